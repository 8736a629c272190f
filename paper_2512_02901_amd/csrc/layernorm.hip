// Layer norm (or RMSNorm) of a token's 2n reals with the residual addition in
// front, in bf16 or as a row of an 8-bit matrix; and its backward pass.
//
// Forward: h = x + delta, mu = mean(h) (0 for RMSNorm), r = 1 / sqrt(mean((h -
// mu)^2) + eps), z = (h - mu) r gain + bias.  A token stays in registers from
// the load to z, so the squares are summed around the mean itself; both sums
// are in double.  A block of 128 reals of the 8-bit row is 16 neighbouring
// lanes' groups of 8.
//
// Backward, with y = (h - mu) r and w = dz gain:
//   dx = dh + r (w - mean(w) - y mean(w y))  (no mean(w) for RMSNorm),
//   dgain = sum over tokens of dz y,  dbias = sum over tokens of dz.
// One pass: a thread keeps its entries' sums over the tokens of its block in
// registers, blocks' sums are joined by a second kernel in a fixed order.
//
// Both are bound by memory; a copy of 1 GiB reaches 5.06 TB/s.  4096 tokens of 2048
// entries, under the profiler: forward with delta and h into an 8-bit matrix 46 us
// (219 MB, 4.7 TB/s), backward with dh and dz in bf16 46 us (235 MB, 5.1 TB/s) and
// 5.0 for the join of 512 blocks' parts.  In a loop over inputs that no cache holds
// a call of the forward takes 43.8 us (into bf16 45.2), of the backward with dbias
// 56.4 (dz in complex64 64.3).  Past 8192 entries the forward reads a token three
// times, the backward h and dz twice: 1024 tokens of 16384 entries 122 us forward
// and 144 backward, where one reading would be 86 and 93 at the copy's rate.  One
// token takes 3.2 us: a launch, a chain of loads and two sums over a block.  The
// tables below are of loops over three inputs, which the last cache holds in part.
#include <float.h>

#include <algorithm>

#include "fp8.h"

namespace fairy2i {

namespace {

constexpr int64_t kMostTokens = 1 << 22;  // of a launch, which takes fewer than 2^32 threads
constexpr int64_t kMostInRegisters = 8192;  // entries of a token

// Four entries of a token, `count` (1..4) of them there.
struct Group {
  float v[8];
};

__device__ inline Group load_group(const float* p, int count) {
  Group g;
  if (count >= 4) {
    const f32x4_any a = reinterpret_cast<const f32x4_any*>(p)[0], b = reinterpret_cast<const f32x4_any*>(p)[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      g.v[j] = a[j];
      g.v[4 + j] = b[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) g.v[j] = j < 2 * count ? p[j] : 0.0f;
  }
  return g;
}

__device__ inline void store_group(float* p, const Group& g, int count) {
  if (count >= 4) {
    reinterpret_cast<f32x4_any*>(p)[0] = f32x4_any{g.v[0], g.v[1], g.v[2], g.v[3]};
    reinterpret_cast<f32x4_any*>(p)[1] = f32x4_any{g.v[4], g.v[5], g.v[6], g.v[7]};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < 2 * count) p[j] = g.v[j];
  }
}

// Four entries' values of a [2n] array (real parts' first), interleaved.
__device__ inline Group load_gain(const float* p, int64_t n, int64_t j, int count) {
  Group g;
  if (count >= 4) {
    const f32x4_any re = *reinterpret_cast<const f32x4_any*>(p + j), im = *reinterpret_cast<const f32x4_any*>(p + n + j);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      g.v[2 * e] = re[e];
      g.v[2 * e + 1] = im[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      g.v[2 * e] = e < count ? p[j + e] : 0.0f;
      g.v[2 * e + 1] = e < count ? p[n + j + e] : 0.0f;
    }
  }
  return g;
}

__device__ inline void store_gain(float* p, int64_t n, int64_t j, const float* v, int count) {
  if (count >= 4) {
    *reinterpret_cast<f32x4_any*>(p + j) = f32x4_any{v[0], v[2], v[4], v[6]};
    *reinterpret_cast<f32x4_any*>(p + n + j) = f32x4_any{v[1], v[3], v[5], v[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < count) {
        p[j + e] = v[2 * e];
        p[n + j + e] = v[2 * e + 1];
      }
  }
}

__device__ inline int count_of(int64_t n, int64_t g) {  // entries of group g
  const int64_t left = n - 4 * g;
  return left >= 4 ? 4 : (left > 0 ? (int)left : 0);
}

template <int NT>
__device__ inline double block_sum(double s, double* slots) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = s;
    __syncthreads();
    s = slots[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) s += slots[w];
  }
  return s;
}

struct Forward {
  const float* x;
  const float* delta;
  const float* gain;
  const float* bias;
  float eps;
  int center;
  int64_t n;
  float* h;
  uint16_t* z;       // bf16, or
  uint8_t* codes;    // 8-bit, with
  uint8_t* scales;
  int64_t rows;      // of the whole 8-bit matrix
  int64_t row0;      // first row of this launch in it
  float* stats;
};

// For e4m3 z is formed in double and rounded once, at no cost in time: of 16.8
// million values (three seeds) none differs from the definition applied to the h
// that is stored, where float32 on the way puts 19 to 26 on the other side of a
// midpoint (relative L2 7e-5 to 3e-4).  Against x + delta before h was rounded 6 to 9
// differ (1e-5 to 4e-5), with float32 17 to 29.  bf16's own rounding is 1.7e-3.
struct Moments {
  double mean, r;
};

// The float next to v with its last bit set where v is no float: rounding that to
// fewer bits rounds v itself.
__device__ inline float odd_float(double v) {
  const float f = (float)v;
  const double back = (double)f;
  uint32_t b = __float_as_uint(f);
  if (fabs(back) > fabs(v)) b -= 1;
  return __uint_as_float(back != v ? b | 1u : b);
}

__device__ inline void write_z(const Forward& a, int64_t row, int64_t g, int count, const Group& h, const Moments& m) {
  const Group gain = load_gain(a.gain, a.n, 4 * g, count);
  Group z = Group{};
  if (a.bias) z = load_gain(a.bias, a.n, 4 * g, count);
  if (a.z) {
    // h - mean may be beyond the largest float32, and r below its normal numbers
#pragma unroll
    for (int j = 0; j < 8; ++j) z.v[j] += (float)(((double)h.v[j] - m.mean) * m.r) * gain.v[j];
    uint16_t* p = a.z + 2 * (row * a.n + 4 * g);
    if (count >= 4) {
      *reinterpret_cast<u32x4_any*>(p) = u32x4_any{bf16_pair(z.v[0], z.v[1]), bf16_pair(z.v[2], z.v[3]),
                                                   bf16_pair(z.v[4], z.v[5]), bf16_pair(z.v[6], z.v[7])};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < count) reinterpret_cast<u32_any*>(p)[e] = bf16_pair(z.v[2 * e], z.v[2 * e + 1]);
    }
    return;
  }
  // the 16 lanes of this block of 128 reals come here together, past the token's end with zeros
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    z.v[j] = odd_float(((double)h.v[j] - m.mean) * m.r * (double)gain.v[j] + (double)z.v[j]);
    if (j >= 2 * count) z.v[j] = 0.0f;
    top = max(top, __float_as_uint(z.v[j]) & 0x7FFFFFFFu);
  }
  if (top > kFp8Most) {
    top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      z.v[j] = fp8_tame(z.v[j]);
      top = max(top, fp8_magnitude(z.v[j]));
    }
  }
  const int byte = fp8_scale_byte(row16_max(top));
  const float scale = fp8_power(byte);
  const int64_t ld = (2 * a.n + 127) / 128 * 128, r = a.row0 + row;
  *reinterpret_cast<uint2*>(a.codes + r * ld + 8 * g) =
      make_uint2(fp8_codes4(z.v[0], z.v[1], z.v[2], z.v[3], scale), fp8_codes4(z.v[4], z.v[5], z.v[6], z.v[7], scale));
  if ((g & 15) == 0) a.scales[fp8_scale_at(a.rows, r, g >> 4)] = (uint8_t)byte;
}

__device__ inline Moments moments(double mean, double squares, int64_t n, float eps, float* stats) {
  Moments m;
  m.mean = mean;
  m.r = 1.0 / sqrt(squares / (double)(2 * n) + (double)eps);
  if (threadIdx.x == 0) {
    stats[0] = (float)m.mean;
    stats[1] = (float)m.r;
  }
  return m;
}

__device__ inline void add(Group& a, const Group& b) {
#pragma unroll
  for (int j = 0; j < 8; ++j) a.v[j] += b.v[j];
}

template <int NT, int GROUPS>
__global__ __launch_bounds__(NT) void add_layernorm_kernel(Forward a) {
  __shared__ double slots[2][NT / 64];
  const int64_t row = blockIdx.x, base = row * a.n;
  const int64_t groups = a.z ? (a.n + 3) / 4 : (2 * a.n + 127) / 128 * 16;
  Group h[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int64_t g = threadIdx.x + i * NT;
    h[i] = load_group(a.x + 2 * (base + 4 * g), count_of(a.n, g));
  }
  if (a.delta) {
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const int64_t g = threadIdx.x + i * NT;
      add(h[i], load_group(a.delta + 2 * (base + 4 * g), count_of(a.n, g)));
    }
  }
  double mean = 0.0, squares = 0.0;
  if (a.center) {
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) mean += (double)h[i].v[j];
    mean = block_sum<NT>(mean, slots[0]) / (double)(2 * a.n);
  }
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int64_t g = threadIdx.x + i * NT;
    const int count = count_of(a.n, g);
    if (a.h && count) store_group(a.h + 2 * (base + 4 * g), h[i], count);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double c = j < 2 * count ? (double)h[i].v[j] - mean : 0.0;
      squares += c * c;
    }
  }
  const Moments m = moments(mean, block_sum<NT>(squares, slots[1]), a.n, a.eps, a.stats + 2 * row);
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int64_t g = threadIdx.x + i * NT;
    if (g < groups) write_z(a, row, g, count_of(a.n, g), h[i], m);
  }
}

// Tokens too long for registers are read again for each sum and for z.
__global__ __launch_bounds__(512) void add_layernorm_long_kernel(Forward a) {
  __shared__ double slots[2][8];
  const int64_t row = blockIdx.x, base = row * a.n;
  const int64_t own = (a.n + 3) / 4, groups = a.z ? own : (2 * a.n + 127) / 128 * 16;
  auto load = [&](int64_t g) {  // as the first pass left it: each thread meets its own entries again
    const int count = count_of(a.n, g);
    if (a.h) return load_group(a.h + 2 * (base + 4 * g), count);
    Group v = load_group(a.x + 2 * (base + 4 * g), count);
    if (a.delta) add(v, load_group(a.delta + 2 * (base + 4 * g), count));
    return v;
  };
  double mean = 0.0, squares = 0.0;
  for (int64_t g = threadIdx.x; g < own; g += 512) {
    const int count = count_of(a.n, g);
    Group v = load_group(a.x + 2 * (base + 4 * g), count);
    if (a.delta) add(v, load_group(a.delta + 2 * (base + 4 * g), count));
    if (a.h) store_group(a.h + 2 * (base + 4 * g), v, count);
#pragma unroll
    for (int j = 0; j < 8; ++j) mean += (double)v.v[j];
  }
  mean = a.center ? block_sum<512>(mean, slots[0]) / (double)(2 * a.n) : 0.0;
  for (int64_t g = threadIdx.x; g < own; g += 512) {
    const Group v = load(g);
    const int count = count_of(a.n, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const double c = j < 2 * count ? (double)v.v[j] - mean : 0.0;
      squares += c * c;
    }
  }
  const Moments m = moments(mean, block_sum<512>(squares, slots[1]), a.n, a.eps, a.stats + 2 * row);
  for (int64_t g = threadIdx.x; g < groups; g += 512)
    write_z(a, row, g, count_of(a.n, g), g < own ? load(g) : Group{}, m);
}

template <int NT, int GROUPS>
void launch_forward(const Forward& a, int64_t B, hipStream_t s) {
  hipLaunchKernelGGL((add_layernorm_kernel<NT, GROUPS>), dim3((unsigned)B), dim3(NT), 0, s, a);
}

// As many threads a token as it has groups of four entries, 512 at most.  us with
// four groups a thread / two / one: 1 token of 2048 5.1 / 4.1 / 3.7, 4096 of 2048
// 44.2 / 41.9 / 40.0, 4096 of 1024 26.0 / 23.8 / 22.8; 1024 threads where a token
// would have two groups of 512 gain nothing (2048 of 4096: 43.0 and 43.1).
void forward(const Forward& a, int64_t B, hipStream_t s) {
  if (a.n <= 256)
    launch_forward<64, 1>(a, B, s);
  else if (a.n <= 1024)
    launch_forward<256, 1>(a, B, s);
  else if (a.n <= 2048)
    launch_forward<512, 1>(a, B, s);
  else if (a.n <= 4096)
    launch_forward<512, 2>(a, B, s);
  else if (a.n <= kMostInRegisters)
    launch_forward<512, 4>(a, B, s);
  else
    hipLaunchKernelGGL(add_layernorm_long_kernel, dim3((unsigned)B), dim3(512), 0, s, a);
}

// ---------------------------------------------------------------- backward

struct Backward {
  const void* dz;  // bf16 or float32 pairs
  const float* h;
  const float* stats;
  const float* gain;
  const float* dh;  // may be null
  int center;
  int64_t B, n;
  float* dx;
  float* parts;  // [blocks][dgain 2n, dbias 2n where wanted]; the outputs themselves where one block does all
  float* dbias;  // with one block
  float* coef;   // tokens too long for registers: [B][3], the two means and what is taken off y
  int64_t rows_per_block;
};

template <bool BF16>
__device__ inline Group load_dz(const void* dz, int64_t entry, int count) {
  if constexpr (BF16) {
    const uint16_t* p = static_cast<const uint16_t*>(dz) + 2 * entry;
    Group g;
    if (count >= 4) {
      const u32x4_any a = *reinterpret_cast<const u32x4_any*>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        g.v[2 * e] = bf16_lo(a[e]);
        g.v[2 * e + 1] = bf16_hi(a[e]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) g.v[j] = j < 2 * count ? __uint_as_float((uint32_t)p[j] << 16) : 0.0f;
    }
    return g;
  } else {
    return load_group(static_cast<const float*>(dz) + 2 * entry, count);
  }
}

__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// The forward pass takes its mean off in double, stats hold it in float32: y is
// off by up to 2^-24 |mu| r, the same for the whole token.  Where that is above
// 2^-18 the mean of y, which ought to be 0, is taken off y.
constexpr float kFarMean = 64.0f;  // |mu| r

// (h - mu) r by way of halves: the difference may be beyond the largest float32.
__device__ inline float scaled(float h, float half_mu, float twice_r) { return fmaf(h, 0.5f, -half_mu) * twice_r; }

// NT threads take a token, 512 / NT tokens a block at a time.
template <int NT, int GROUPS, bool BF16, bool BIAS>
__global__ __launch_bounds__(512) void layernorm_backward_kernel(Backward a) {
  constexpr int TEAMS = 512 / NT, WAVES = NT / 64;
  __shared__ float2 slots[2][8];
  __shared__ float offsets[2][8];
  __shared__ float others[TEAMS > 1 ? (TEAMS - 1) * NT * GROUPS * 8 * (BIAS ? 2 : 1) : 1];
  const int team = threadIdx.x / NT, t = threadIdx.x % NT;
  const float over = 1.0f / (float)(2 * a.n);
  const int64_t first = blockIdx.x * a.rows_per_block, last = min(first + a.rows_per_block, a.B);

  Group gain[GROUPS], sum_g[GROUPS], sum_b[BIAS ? GROUPS : 1];
  int count[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int64_t g = t + i * NT;
    count[i] = count_of(a.n, g);
    gain[i] = load_gain(a.gain, a.n, 4 * g, count[i]);
    sum_g[i] = Group{};
    if constexpr (BIAS) sum_b[i] = Group{};
  }
  int parity = 0;
  for (int64_t at = first; at < last; at += TEAMS, parity ^= 1) {
    const int64_t row = at + team;
    const bool there = row < last;
    Group y[GROUPS], dz[GROUPS];
    float mu = 0.0f, r = 0.0f;
    if (there) {
      mu = a.stats[2 * row];
      r = a.stats[2 * row + 1];
    }
    const bool far = a.center && fabsf(mu) * r > kFarMean;  // the whole team
    float s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const int64_t e = row * a.n + 4 * (int64_t)(t + i * NT);
      const int c = there ? count[i] : 0;
      y[i] = load_group(a.h + 2 * e, c);
      dz[i] = load_dz<BF16>(a.dz, e, c);
    }
#pragma unroll
    for (int i = 0; i < GROUPS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = scaled(y[i].v[j], 0.5f * mu, 2.0f * r);
        y[i].v[j] = v;
        sum_g[i].v[j] += dz[i].v[j] * v;
        if constexpr (BIAS) sum_b[i].v[j] += dz[i].v[j];
        const float w = dz[i].v[j] * gain[i].v[j];
        s1 += w;
        s2 += w * v;
      }
    s1 = wave_sum(s1);
    s2 = wave_sum(s2);
    if (far) {
#pragma unroll
      for (int i = 0; i < GROUPS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < 2 * count[i]) s3 += y[i].v[j];
      s3 = wave_sum(s3);
    }
    if constexpr (WAVES > 1) {
      if ((threadIdx.x & 63) == 0) {
        slots[parity][threadIdx.x >> 6] = make_float2(s1, s2);
        offsets[parity][threadIdx.x >> 6] = s3;
      }
      __syncthreads();  // the other parity's slots are free: they were read before the last barrier
      s1 = s2 = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float2 v = slots[parity][team * WAVES + w];
        s1 += v.x;
        s2 += v.y;
      }
    }
    const float m1 = a.center ? s1 * over : 0.0f;
    float m2 = s2 * over;
    if (far) {
      if constexpr (WAVES > 1) {
        s3 = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s3 += offsets[parity][team * WAVES + w];
      }
      const float off = s3 * over;
      m2 -= m1 * off;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          sum_g[i].v[j] -= dz[i].v[j] * off;
          y[i].v[j] -= off;
        }
    }
    if (there) {
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        if (count[i] == 0) continue;
        const int64_t e = row * a.n + 4 * (int64_t)(t + i * NT);
        Group d = Group{};
        if (a.dh) d = load_group(a.dh + 2 * e, count[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) d.v[j] += ((dz[i].v[j] * gain[i].v[j] - m1) - y[i].v[j] * m2) * r;
        store_group(a.dx + 2 * e, d, count[i]);
      }
    }
  }
  if constexpr (TEAMS > 1) {
    constexpr int PER = GROUPS * 8 * (BIAS ? 2 : 1);
    if (team > 0) {
      float* o = others + (team - 1) * NT * PER;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          o[(i * 8 + j) * NT + t] = sum_g[i].v[j];
          if constexpr (BIAS) o[((GROUPS + i) * 8 + j) * NT + t] = sum_b[i].v[j];
        }
    }
    __syncthreads();
    if (team > 0) return;
    for (int k = 0; k < TEAMS - 1; ++k) {
      const float* o = others + k * NT * PER;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          sum_g[i].v[j] += o[(i * 8 + j) * NT + t];
          if constexpr (BIAS) sum_b[i].v[j] += o[((GROUPS + i) * 8 + j) * NT + t];
        }
    }
  }
  float* part = a.parts + blockIdx.x * (BIAS ? 4 : 2) * a.n;
  float* part_b = gridDim.x == 1 ? a.dbias : part + 2 * a.n;
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int64_t j = 4 * (int64_t)(t + i * NT);
    if (count[i] == 0) continue;
    store_gain(part, a.n, j, sum_g[i].v, count[i]);
    if constexpr (BIAS) store_gain(part_b, a.n, j, sum_b[i].v, count[i]);
  }
}

// Tokens too long for registers: a token's means first, then the entries,
// a thread one entry of a run of tokens.  The run is as long as the grid makes it
// (all tokens from 2^19 entries on), so a thread's sums are in double.
template <bool BF16>
__global__ __launch_bounds__(512) void layernorm_backward_means_kernel(Backward a) {
  __shared__ float slots[3][8];
  const int64_t row = blockIdx.x;
  const float mu = a.stats[2 * row], r = a.stats[2 * row + 1];
  double s1 = 0.0, s2 = 0.0, s3 = 0.0;
  for (int64_t g = threadIdx.x; 4 * g < a.n; g += 512) {
    const int count = count_of(a.n, g);
    const Group h = load_group(a.h + 2 * (row * a.n + 4 * g), count);
    const Group dz = load_dz<BF16>(a.dz, row * a.n + 4 * g, count), gain = load_gain(a.gain, a.n, 4 * g, count);
    float p1 = 0.0f, p2 = 0.0f, p3 = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float w = dz.v[j] * gain.v[j], y = scaled(h.v[j], 0.5f * mu, 2.0f * r);
      p1 += w;
      p2 += w * y;
      p3 += j < 2 * count ? y : 0.0f;
    }
    s1 += (double)p1;
    s2 += (double)p2;
    s3 += (double)p3;
  }
  const float f1 = wave_sum((float)s1), f2 = wave_sum((float)s2), f3 = wave_sum((float)s3);
  if ((threadIdx.x & 63) == 0) {
    slots[0][threadIdx.x >> 6] = f1;
    slots[1][threadIdx.x >> 6] = f2;
    slots[2][threadIdx.x >> 6] = f3;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double m[3] = {};
    for (int i = 0; i < 3; ++i) {
      for (int w = 0; w < 8; ++w) m[i] += (double)slots[i][w];
      m[i] /= (double)(2 * a.n);
    }
    if (!a.center) m[0] = 0.0;
    const bool far = a.center && fabsf(mu) * r > kFarMean;
    if (far) m[1] -= m[0] * m[2];
    a.coef[3 * row] = (float)m[0];
    a.coef[3 * row + 1] = (float)m[1];
    a.coef[3 * row + 2] = far ? (float)m[2] : 0.0f;
  }
}

template <bool BF16, bool BIAS>
__global__ __launch_bounds__(256) void layernorm_backward_long_kernel(Backward a) {
  const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (j >= a.n) return;
  const int64_t first = blockIdx.y * a.rows_per_block, last = min(first + a.rows_per_block, a.B);
  const float gr = a.gain[j], gi = a.gain[a.n + j];
  double sgr = 0.0, sgi = 0.0, sbr = 0.0, sbi = 0.0;
  for (int64_t row = first; row < last; ++row) {
    const int64_t e = row * a.n + j;
    const float mu = a.stats[2 * row], r = a.stats[2 * row + 1];
    const float m1 = a.coef[3 * row], m2 = a.coef[3 * row + 1], off = a.coef[3 * row + 2];
    const f32x2_any h = *reinterpret_cast<const f32x2_any*>(a.h + 2 * e);
    float dr, di;
    if constexpr (BF16) {
      const uint32_t w = *reinterpret_cast<const u32_any*>(static_cast<const uint16_t*>(a.dz) + 2 * e);
      dr = bf16_lo(w);
      di = bf16_hi(w);
    } else {
      const f32x2_any w = *reinterpret_cast<const f32x2_any*>(static_cast<const float*>(a.dz) + 2 * e);
      dr = w[0];
      di = w[1];
    }
    const float yr = scaled(h[0], 0.5f * mu, 2.0f * r) - off, yi = scaled(h[1], 0.5f * mu, 2.0f * r) - off;
    sgr += (double)dr * (double)yr;
    sgi += (double)di * (double)yi;
    sbr += (double)dr;
    sbi += (double)di;
    f32x2_any d = {0.0f, 0.0f};
    if (a.dh) d = *reinterpret_cast<const f32x2_any*>(a.dh + 2 * e);
    d[0] += ((dr * gr - m1) - yr * m2) * r;
    d[1] += ((di * gi - m1) - yi * m2) * r;
    *reinterpret_cast<f32x2_any*>(a.dx + 2 * e) = d;
  }
  float* part = a.parts + blockIdx.y * (BIAS ? 4 : 2) * a.n;
  part[j] = (float)sgr;
  part[a.n + j] = (float)sgi;
  if constexpr (BIAS) {
    float* part_b = gridDim.y == 1 ? a.dbias : part + 2 * a.n;
    part_b[j] = (float)sbr;
    part_b[a.n + j] = (float)sbi;
  }
}

// Sums of the blocks' parts: 32 columns a block, 32 threads a column.
__global__ __launch_bounds__(1024) void layernorm_join_kernel(const float* __restrict__ parts, int64_t blocks,
                                                              int64_t width, int64_t n2, float* __restrict__ dgain,
                                                              float* __restrict__ dbias) {
  __shared__ double sums[32][32];
  const int c = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int64_t col = (int64_t)blockIdx.x * 32 + c;
  double s = 0.0;
  if (col < width) {
#pragma unroll 8
    for (int64_t b = k; b < blocks; b += 32) s += (double)parts[b * width + col];
  }
  sums[k][c] = s;
  __syncthreads();
  if (k == 0 && col < width) {
#pragma unroll
    for (int i = 1; i < 32; ++i) s += sums[i][c];
    if (col < n2)
      dgain[col] = (float)s;
    else
      dbias[col - n2] = (float)s;
  }
}

// Up to this many tokens a team one block does them all, without a join: us of one
// block / a block for each step, 2 tokens of 2048 4.6 / 5.9, 5 of 512 4.5 / 5.7, 2 of
// 4096 6.5 / 7.2; with three tokens a team 5.6 / 5.8, 6.0 / 5.8 and 8.4 / 7.2.
constexpr int64_t kOneBlock = 2;

// A team adds up to this many tokens in float32; what is above is the join's, in
// double, so an error does not grow with the tokens.  us with 256 or 512 blocks for
// any number of tokens / with 64 a team: 65536 of 2048 725 / 722, 65536 of 4096 1596 /
// 1506, 262144 of 300 455 / 458, 524288 of 130 497 / 504.
constexpr int64_t kMostSteps = 64;
constexpr int64_t kMostBlocks = 1 << 22;  // a launch takes fewer than 2^32 threads

// How the tokens are cut over blocks.
struct Cut {
  int64_t blocks, rows_per_block;
};

int teams_of(int64_t n) {  // tokens of a block at a time, as backward() has them
  return n <= 256 ? 8 : n <= 512 ? 4 : n <= 1024 ? 2 : 1;
}

Cut cut_of(int64_t B, int64_t n) {
  if (n <= kMostInRegisters) {
    // One block a CU, two where the threads' registers allow it and each has more
    // than two tokens a team still: each block leaves a part of 8 or 16 bytes an
    // entry to the join.  us, one / two a CU, of dz in bf16 with dbias and dh: 4096
    // tokens of 2048 54.7 / 51.5, 4096 of 1024 30.8 / 26.9, 4096 of 512 15.2 / 14.9;
    // 1024 of 2048 16.6 / 17.5, 2048 of 512 11.3 / 11.9.
    const int64_t teams = teams_of(n), steps = (B + teams - 1) / teams;
    int64_t most = steps <= kOneBlock ? 1 : n <= 2048 && steps > 1024 ? 512 : 256;
    most = std::max(most, std::min((steps + kMostSteps - 1) / kMostSteps, kMostBlocks));
    const int64_t rows = (steps + most - 1) / most * teams;
    return {(B + rows - 1) / rows, rows};
  }
  const int64_t col_blocks = (n + 255) / 256;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(B, 2048 / col_blocks));
  const int64_t rows = (B + want - 1) / want;
  return {(B + rows - 1) / rows, rows};
}

int64_t parts_floats(int64_t B, int64_t n) {
  const Cut c = cut_of(B, n);
  return c.blocks == 1 ? 0 : c.blocks * 4 * n;
}

template <int NT, int GROUPS, bool BF16, bool BIAS>
void launch_backward(const Backward& a, int64_t blocks, hipStream_t s) {
  hipLaunchKernelGGL((layernorm_backward_kernel<NT, GROUPS, BF16, BIAS>), dim3((unsigned)blocks), dim3(512), 0, s, a);
}

template <bool BF16, bool BIAS>
hipError_t backward(Backward a, float* dgain, float* dbias, float* workspace, hipStream_t s) {
  const Cut c = cut_of(a.B, a.n);
  a.rows_per_block = c.rows_per_block;
  a.parts = c.blocks == 1 ? dgain : workspace;
  a.dbias = dbias;
  // As many threads a token as it has groups of four entries, 512 at most: few
  // tokens wait for their loads and sums.  us with two groups a thread / one: 1
  // token of 2048 4.6 / 3.5, 77 of 2048 8.1 / 7.5, 4096 of 1024 29.9 / 30.6.
  if (a.n <= 256)
    launch_backward<64, 1, BF16, BIAS>(a, c.blocks, s);
  else if (a.n <= 512)
    launch_backward<128, 1, BF16, BIAS>(a, c.blocks, s);
  else if (a.n <= 1024)
    launch_backward<256, 1, BF16, BIAS>(a, c.blocks, s);
  else if (a.n <= 2048)
    launch_backward<512, 1, BF16, BIAS>(a, c.blocks, s);
  else if (a.n <= 4096)
    launch_backward<512, 2, BF16, BIAS>(a, c.blocks, s);
  else if (a.n <= kMostInRegisters)
    launch_backward<512, 4, BF16, BIAS>(a, c.blocks, s);
  else {
    a.coef = workspace + parts_floats(a.B, a.n);
    for (int64_t b = 0; b < a.B; b += kMostTokens) {
      Backward p = a;
      p.B = std::min(a.B - b, kMostTokens);
      p.dz = static_cast<const char*>(a.dz) + 2 * b * a.n * (BF16 ? 2 : 4);
      p.h += 2 * b * a.n;
      p.stats += 2 * b;
      p.coef += 3 * b;
      hipLaunchKernelGGL((layernorm_backward_means_kernel<BF16>), dim3((unsigned)p.B), dim3(512), 0, s, p);
    }
    hipLaunchKernelGGL((layernorm_backward_long_kernel<BF16, BIAS>),
                       dim3((unsigned)((a.n + 255) / 256), (unsigned)c.blocks), dim3(256), 0, s, a);
  }
  if (c.blocks > 1) {
    const int64_t width = (BIAS ? 4 : 2) * a.n;
    hipLaunchKernelGGL(layernorm_join_kernel, dim3((unsigned)((width + 31) / 32)), dim3(1024), 0, s, workspace,
                       c.blocks, width, 2 * a.n, dgain, dbias);
  }
  return hipGetLastError();
}

bool sizes_ok(int64_t B, int64_t n) { return B >= 1 && B <= INT32_MAX && n >= 1 && n <= ((int64_t)1 << 24); }

}  // namespace

}  // namespace fairy2i

using namespace fairy2i;

extern "C" {

fairy2i_status fairy2i_add_layernorm(const float* x, const float* delta, const float* gain, const float* bias,
                                     float eps, int32_t center, int64_t B, int64_t n, float* h, void* z,
                                     const fairy2i_fp8_matrix* z8, float* stats, void* stream) {
  if (!x || !gain || !stats || (!z && !z8)) return FAIRY2I_ERR_NULL;
  if (!sizes_ok(B, n) || !(eps > 0.0f) || eps > FLT_MAX || (center != 0 && center != 1)) return FAIRY2I_ERR_SHAPE;
  if (z && z8) return FAIRY2I_ERR_UNSUPPORTED;
  if (z8) {
    const fairy2i_status st = fp8_check(z8);
    if (st != FAIRY2I_OK) return st;
    if (z8->rows != B || z8->cols != 2 * n) return FAIRY2I_ERR_SHAPE;
  }
  for (int64_t b = 0; b < B; b += kMostTokens) {
    const int64_t e = b * n;  // entries before
    const Forward a{x + 2 * e,
                    delta ? delta + 2 * e : nullptr,
                    gain,
                    bias,
                    eps,
                    center,
                    n,
                    h ? h + 2 * e : nullptr,
                    z ? static_cast<uint16_t*>(z) + 2 * e : nullptr,
                    z8 ? z8->codes : nullptr,
                    z8 ? z8->scales : nullptr,
                    B,
                    b,
                    stats + 2 * b};
    forward(a, std::min(B - b, kMostTokens), static_cast<hipStream_t>(stream));
  }
  return hipGetLastError() == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

size_t fairy2i_layernorm_backward_workspace_bytes(int64_t B, int64_t n) {
  if (!sizes_ok(B, n)) return 0;
  return sizeof(float) * (size_t)(parts_floats(B, n) + (n > kMostInRegisters ? 3 * B : 0));
}

fairy2i_status fairy2i_layernorm_backward(const void* dz, int32_t dtype, const float* h, const float* stats,
                                          const float* gain, const float* dh, int32_t center, int64_t B, int64_t n,
                                          float* dx, float* dgain, float* dbias, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  if (!dz || !h || !stats || !gain || !dx || !dgain) return FAIRY2I_ERR_NULL;
  if (!sizes_ok(B, n) || (center != 0 && center != 1)) return FAIRY2I_ERR_SHAPE;
  if (dtype != FAIRY2I_ACT_F32 && dtype != FAIRY2I_ACT_BF16) return FAIRY2I_ERR_DTYPE;
  const size_t need = fairy2i_layernorm_backward_workspace_bytes(B, n);
  if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 3)))
    return FAIRY2I_ERR_WORKSPACE;
  const Backward a{dz, h, stats, gain, dh, center, B, n, dx, nullptr, nullptr, nullptr, 0};
  float* ws = static_cast<float*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = dtype == FAIRY2I_ACT_BF16;
  const hipError_t e = bf16 ? (dbias ? backward<true, true>(a, dgain, dbias, ws, s)
                                     : backward<true, false>(a, dgain, dbias, ws, s))
                            : (dbias ? backward<false, true>(a, dgain, dbias, ws, s)
                                     : backward<false, false>(a, dgain, dbias, ws, s));
  return e == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

}  // extern "C"
