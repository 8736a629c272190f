// Residual addition, RMSNorm and int8 quantisation of a token in one pass.
//
// h = x + delta, z = h * gain / sqrt(mean(h^2) + eps), q = rint(z * 127 / g)
// with g = max |z|.  The factor r = 1 / sqrt(..) is one positive number a
// token, so with t = h * gain the largest |z| is the largest |t| times r, in
// float32 as well (rounding is monotonic): the sum and the maximum come out
// of one reduction, and a token's t stay in registers from the load to q.
// The squares are summed in double: no finite token overflows.
//
// What bounds it is memory, 26 bytes an entry with delta and h (8 + 8 + 8 + 2):
// 2048 tokens of 2048 entries 20.2 us (5.4 TB/s, a plain copy's rate); 77 of 1500
// 4.1 us and one of 2048 3.0 us, an empty launch and two trips to memory.
#include <float.h>

#include "common.h"

namespace fairy2i {

namespace {

// Sum of s and maximum of m (bits of an absolute value: a NaN's are above
// infinity's, so it stays) over the block, the same in every thread.
template <int NT>
__device__ inline void block_sum_max(double& s, uint32_t& m) {
  __shared__ double ss[NT / 64];
  __shared__ uint32_t mm[NT / 64];
  for (int off = 32; off > 0; off >>= 1) {
    s += __shfl_xor(s, off);
    m = max(m, (uint32_t)__shfl_xor((int)m, off));
  }
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) {
      ss[threadIdx.x >> 6] = s;
      mm[threadIdx.x >> 6] = m;
    }
    __syncthreads();
    s = ss[0];
    m = mm[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) {
      s += ss[w];
      m = max(m, mm[w]);
    }
  }
}

struct Norm {
  float r, inv, scale;  // z = t * r, q = rint(z * inv)
};

__device__ inline Norm norm_of(double sum, uint32_t top, int64_t n, float eps) {
  Norm k;
  k.r = (float)(1.0 / sqrt(sum / (double)(2 * n) + (double)eps));
  const float g = __fmul_rn(__uint_as_float(top), k.r);
  if (!(g < INFINITY)) {  // a value that is not finite: the scale says so
    k.r = k.inv = 0.0f;
    k.scale = __builtin_nanf("");
    return k;
  }
  k.inv = g > 0.0f ? 127.0f / g : 0.0f;
  if (k.inv == INFINITY) k.inv = 0.0f;  // g below 2^-121: zeros
  k.scale = k.inv > 0.0f ? g / 127.0f : 0.0f;
  return k;
}

__device__ inline uint32_t quantise(float t, const Norm& k) {
  const float q = fminf(fmaxf(rintf(__fmul_rn(__fmul_rn(t, k.r), k.inv)), -127.0f), 127.0f);
  return (uint32_t)(uint8_t)(int8_t)(int)(k.inv > 0.0f ? q : 0.0f);
}

__device__ inline uint32_t abs_bits(float t) { return __float_as_uint(t) & 0x7FFFFFFFu; }

typedef int8_t i8x2_any __attribute__((ext_vector_type(2), aligned(1)));

// Any size and alignment.  A token is read twice (the second time from h
// where that is written, which may be x or delta): a size that no number of
// registers a thread is right for has nowhere else to wait for its maximum.
__global__ __launch_bounds__(256) void add_rmsnorm_i8_any_kernel(const float2* x, const float2* delta,
                                                                 const float* __restrict__ gain, float eps, int64_t n,
                                                                 float2* h, i8x2_any* __restrict__ q,
                                                                 float* __restrict__ x_scale) {
  const int64_t base = (int64_t)blockIdx.x * n;
  double sum = 0.0;
  uint32_t top = 0;
  for (int64_t j = threadIdx.x; j < n; j += 256) {
    float2 v = x[base + j];
    if (delta) {
      const float2 d = delta[base + j];
      v.x += d.x;
      v.y += d.y;
    }
    if (h) h[base + j] = v;
    sum += (double)v.x * v.x + (double)v.y * v.y;
    top = max(top, max(abs_bits(v.x * gain[j]), abs_bits(v.y * gain[n + j])));
  }
  block_sum_max<256>(sum, top);
  const Norm k = norm_of(sum, top, n, eps);
  for (int64_t j = threadIdx.x; j < n; j += 256) {  // each thread its own entries again
    float2 v = h ? h[base + j] : x[base + j];
    if (!h && delta) {
      const float2 d = delta[base + j];
      v.x += d.x;
      v.y += d.y;
    }
    q[base + j] = i8x2_any{(int8_t)quantise(v.x * gain[j], k), (int8_t)quantise(v.y * gain[n + j], k)};
  }
  if (threadIdx.x == 0) x_scale[blockIdx.x] = k.scale;
}

// n % 4 == 0, everything aligned: groups of four entries, GROUPS a thread.
template <int NT, int GROUPS>
__global__ __launch_bounds__(NT) void add_rmsnorm_i8_kernel(const float4* x, const float4* delta,
                                                            const float4* __restrict__ gain, float eps, int groups,
                                                            float4* h, uint2* __restrict__ q,
                                                            float* __restrict__ x_scale) {
  const int64_t base = (int64_t)blockIdx.x * groups;
  float4 a[GROUPS][2];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int g = threadIdx.x + i * NT;
#pragma unroll
    for (int e = 0; e < 2; ++e) a[i][e] = g < groups ? x[2 * (base + g) + e] : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if (delta) {
    float4 d[GROUPS][2];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const int g = threadIdx.x + i * NT;
#pragma unroll
      for (int e = 0; e < 2; ++e) d[i][e] = g < groups ? delta[2 * (base + g) + e] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        a[i][e].x += d[i][e].x;
        a[i][e].y += d[i][e].y;
        a[i][e].z += d[i][e].z;
        a[i][e].w += d[i][e].w;
      }
  }
  double sum = 0.0;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int g = threadIdx.x + i * NT;
    if (g >= groups) break;
    if (h) {
#pragma unroll
      for (int e = 0; e < 2; ++e) h[2 * (base + g) + e] = a[i][e];
    }
    const float4 re = gain[g], im = gain[groups + g];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float4& v = a[i][e];
      sum += (double)v.x * v.x + (double)v.y * v.y;
      sum += (double)v.z * v.z + (double)v.w * v.w;
      v.x *= e ? re.z : re.x;
      v.y *= e ? im.z : im.x;
      v.z *= e ? re.w : re.y;
      v.w *= e ? im.w : im.y;
      top = max(top, max(max(abs_bits(v.x), abs_bits(v.y)), max(abs_bits(v.z), abs_bits(v.w))));
    }
  }
  block_sum_max<NT>(sum, top);
  const Norm k = norm_of(sum, top, 4 * (int64_t)groups, eps);
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int g = threadIdx.x + i * NT;
    if (g >= groups) break;
    uint32_t w[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      w[e] = quantise(a[i][e].x, k) | quantise(a[i][e].y, k) << 8 | quantise(a[i][e].z, k) << 16 |
             quantise(a[i][e].w, k) << 24;
    q[base + g] = make_uint2(w[0], w[1]);
  }
  if (threadIdx.x == 0) x_scale[blockIdx.x] = k.scale;
}

template <int NT, int GROUPS>
void launch_vec(const float* x, const float* delta, const float* gain, float eps, int64_t B, int64_t n, float* h,
                int8_t* q, float* x_scale, hipStream_t s) {
  hipLaunchKernelGGL((add_rmsnorm_i8_kernel<NT, GROUPS>), dim3((unsigned)B), dim3(NT), 0, s,
                     reinterpret_cast<const float4*>(x), reinterpret_cast<const float4*>(delta),
                     reinterpret_cast<const float4*>(gain), eps, (int)(n / 4), reinterpret_cast<float4*>(h),
                     reinterpret_cast<uint2*>(q), x_scale);
}

constexpr int64_t kMostTokens = 1 << 22;  // of a launch, which takes fewer than 2^32 threads

void launch(const float* x, const float* delta, const float* gain, float eps, int64_t B, int64_t n, float* h,
            int8_t* q, float* x_scale, hipStream_t s) {
  auto at = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  // As many threads as take a token at a group each, up to 512, then up to four
  // groups each.  us for 1 | 2048 tokens (a launch in a graph is about 2 of them):
  //   n = 256   64 x 1 3.3 | 5.0    256 x 1 3.3 | 6.2     512 x 1 3.5 | 8.9
  //   n = 1024 256 x 1 3.5 | 11.9    64 x 4 4.6 | 12.0    512 x 1 3.5 | 13.7
  //   n = 2048 512 x 1 3.9 | 20.8   256 x 2 4.1 | 20.1   1024 x 1 4.2 | 22.9
  //   n = 4096 512 x 2 4.6 | 36.6   512 x 4 4.8 | 38.1   1024 x 1 5.0 | 37.4
  //   n = 8192 512 x 4 6.2 | 91.1  1024 x 2 6.6 | 90.4
  // The form for any size reads a token twice: 4.8 | 14.7 at n = 1024, 18.5 | 108
  // at n = 8192.
  if (n % 4 != 0 || n > 8192 || ((at(x) | at(delta) | at(gain) | at(h)) & 15) != 0 || (at(q) & 7) != 0)
    hipLaunchKernelGGL(add_rmsnorm_i8_any_kernel, dim3((unsigned)B), dim3(256), 0, s,
                       reinterpret_cast<const float2*>(x), reinterpret_cast<const float2*>(delta), gain, eps, n,
                       reinterpret_cast<float2*>(h), reinterpret_cast<i8x2_any*>(q), x_scale);
  else if (n <= 256)
    launch_vec<64, 1>(x, delta, gain, eps, B, n, h, q, x_scale, s);
  else if (n <= 1024)
    launch_vec<256, 1>(x, delta, gain, eps, B, n, h, q, x_scale, s);
  else if (n <= 2048)
    launch_vec<512, 1>(x, delta, gain, eps, B, n, h, q, x_scale, s);
  else if (n <= 4096)
    launch_vec<512, 2>(x, delta, gain, eps, B, n, h, q, x_scale, s);
  else
    launch_vec<512, 4>(x, delta, gain, eps, B, n, h, q, x_scale, s);
}

}  // namespace

}  // namespace fairy2i

using namespace fairy2i;

extern "C" fairy2i_status fairy2i_add_rmsnorm_i8(const float* x, const float* delta, const float* gain, float eps,
                                                 int64_t B, int64_t n, float* h, int8_t* q, float* x_scale,
                                                 void* stream) {
  if (!x || !gain || !q || !x_scale) return FAIRY2I_ERR_NULL;
  if (B <= 0 || n <= 0 || B > INT32_MAX || n > ((int64_t)1 << 24) || !(eps > 0.0f) || eps > FLT_MAX) return FAIRY2I_ERR_SHAPE;
  for (int64_t b = 0; b < B; b += kMostTokens) {
    const int64_t e = b * n;  // entries before
    launch(x + 2 * e, delta ? delta + 2 * e : nullptr, gain, eps, min(B - b, kMostTokens), n, h ? h + 2 * e : nullptr,
           q + 2 * e, x_scale + b, static_cast<hipStream_t>(stream));
  }
  return hipGetLastError() == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}
