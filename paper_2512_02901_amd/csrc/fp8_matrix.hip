// 8-bit matrices: from float32 or bf16 along the rows, along the columns
// (transposed) or both in one pass; an 8-bit matrix turned; and back to bf16.
//
// A product C = A B^T on the matrix cores wants both operands along the axis
// that is summed over, and a block of 128 along that axis to share its scale.
// A training step's three products sum over three axes, so X, G_Y and R are
// wanted in both forms.  A block of threads takes 128 x 128 reals into
// registers once: a thread holds 8 rows x 8 columns, so a row's maximum is 8
// values and a DPP row of 16 lanes, a column's 8 values, the wave's four DPP
// rows and four waves.  The turned codes go through 16 KB of LDS (8-byte slots
// exchanged by column) and leave as whole 128-byte rows.  A wave writes rows
// 1024 bytes apart, into one span of 128 bytes of the banks: conflicts are 18 % of
// the LDS cycles, which are 8 % of the kernel's.
//
// Bound by memory: bf16 of 11008 x 4096 in, both forms out, is 182 MB in 39.5
// us, 4.6 TB/s of the 5.06 that a large copy reaches, at a third of the VALU's
// issue.  The 149 registers of a thread allow three waves a SIMD; held to 128
// (four waves) it spills: 65 us.  Turning an 8-bit matrix fits in 128 but for one
// register: 4096 x 4096 9.6 us, with three waves 10.5.  Read once a form instead,
// 4096 x 4096 takes 9.8 + 11.4 us where both at once take 14.8.  What the last
// columns cost: 1003 x 1376 of bf16 5.1 us, 1003 x 1378 6.1 (a multiple of 8
// columns costs nothing more).
#include <algorithm>

#include "fp8.h"

namespace fairy2i {

namespace {

enum { kF32, kBf16, kFp8 };  // what is read

struct Source {
  const void* x;
  const uint8_t* scales;  // kFp8
  int64_t ld;             // elements of a row
};

// Eight neighbours of row r from column c on.
template <int SRC>
__device__ inline void load8_at(const Source& s, int64_t rows, int64_t r, int64_t c, float v[8]) {
  if constexpr (SRC == kFp8) {  // rows are padded with zeros to whole blocks
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(s.x) + r * s.ld + c);
    const float unit = fp8_power(s.scales[fp8_scale_at(rows, r, c / kFp8Block)]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t word = h ? w.y : w.x;
      const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, unit, false);
      const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, unit, true);
      v[4 * h] = lo[0];
      v[4 * h + 1] = lo[1];
      v[4 * h + 2] = hi[0];
      v[4 * h + 3] = hi[1];
    }
  } else if constexpr (SRC == kF32) {
    const f32x4_any* p = reinterpret_cast<const f32x4_any*>(static_cast<const float*>(s.x) + r * s.ld + c);
    const f32x4_any a = p[0], b = p[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = a[j];
      v[4 + j] = b[j];
    }
  } else {
    const u32x4_any a = *reinterpret_cast<const u32x4_any*>(static_cast<const uint16_t*>(s.x) + r * s.ld + c);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = bf16_lo(a[j]);
      v[2 * j + 1] = bf16_hi(a[j]);
    }
  }
}

// One element's bits, bf16's in the low half.
template <int SRC>
__device__ inline uint32_t load1_at(const Source& s, int64_t r, int64_t c) {
  if constexpr (SRC == kF32) return static_cast<const uint32_t*>(s.x)[r * s.ld + c];
  return static_cast<const uint16_t*>(s.x)[r * s.ld + c];
}

// Eight rows of eight from (r, c) on, zeros outside; rows and columns outside are
// asked for at the last ones.
template <int SRC>
__device__ inline void load64(const Source& s, int64_t rows, int64_t cols, int64_t r, int64_t c, float v[8][8]) {
  const int there = (int)min(rows - r, (int64_t)8), left = (int)min(cols - c, (int64_t)8);  // below 1: none
  if (SRC == kFp8 || cols >= 8) {
    const int64_t first = SRC == kFp8 ? c : min(c, cols - 8), top = min(r, rows - 1);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      load8_at<SRC>(s, rows, top + min(p, max(there - 1, 0)), first, v[p]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[p][j] = p < there && (SRC == kFp8 || left > 0) ? v[p][j] : 0.0f;
    }
  }
  if constexpr (SRC != kFp8) {
    // the lanes whose group the matrix ends in, value by value: 64 loads on the way at once
    if (cols < 8 || (left > 0 && left < 8)) {
      uint32_t w[8][8];
#pragma unroll
      for (int p = 0; p < 8; ++p)
#pragma unroll
        for (int j = 0; j < 8; ++j) w[p][j] = load1_at<SRC>(s, min(r + p, rows - 1), min(c + j, cols - 1));
#pragma unroll
      for (int p = 0; p < 8; ++p)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          // else the compiler loads bf16 into upper halves, each after a wait for the load before it: 9.3 us
          // instead of 6.1 at 1003 x 1378
          asm volatile("" : "+v"(w[p][j]));
          v[p][j] = p < there && j < left ? __uint_as_float(SRC == kF32 ? w[p][j] : w[p][j] << 16) : 0.0f;
        }
    }
  }
}

template <int SRC, bool DIRECT, bool TURNED>
__global__ __launch_bounds__(256, SRC == kFp8 ? 4 : 3) void fp8_quantize_kernel(Source src, int64_t rows, int64_t cols, int col_tiles,
                                                              uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                                              uint8_t* __restrict__ codes_t,
                                                              uint8_t* __restrict__ scales_t) {
  __shared__ __attribute__((aligned(16))) uint2 tile[TURNED ? 128 * 16 : 1];
  __shared__ __attribute__((aligned(16))) uint32_t tops[TURNED ? 4 * 128 : 4];
  const int t = threadIdx.x, cg = t & 15, rg = t >> 4;
  const int64_t rb = blockIdx.x / (uint32_t)col_tiles, cb = blockIdx.x % (uint32_t)col_tiles;
  const int64_t r0 = rb * 128 + 8 * rg, c0 = cb * 128 + 8 * cg;
  float v[8][8];
  load64<SRC>(src, rows, cols, r0, c0, v);

  uint32_t row[8] = {}, col[8] = {}, all = 0;  // largest magnitudes of this thread's rows and columns
#pragma unroll
  for (int p = 0; p < 8; ++p)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t a = __float_as_uint(v[p][j]) & 0x7FFFFFFFu;
      if constexpr (DIRECT) row[p] = max(row[p], a);
      if constexpr (TURNED) col[j] = max(col[j], a);
    }
#pragma unroll
  for (int p = 0; p < 8; ++p) all = max(all, DIRECT ? row[p] : col[p]);
  if (__any(all > kFp8Most)) {
#pragma unroll
    for (int p = 0; p < 8; ++p) row[p] = col[p] = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[p][j] = fp8_tame(v[p][j]);
        const uint32_t a = fp8_magnitude(v[p][j]);
        row[p] = max(row[p], a);
        col[j] = max(col[j], a);
      }
  }
  if constexpr (TURNED) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      col[j] = max(col[j], (uint32_t)__shfl_xor((int)col[j], 16));
      col[j] = max(col[j], (uint32_t)__shfl_xor((int)col[j], 32));
    }
    if ((t & 63) < 16) {
      uint4* to = reinterpret_cast<uint4*>(&tops[(t >> 6) * 128 + 8 * cg]);
      to[0] = make_uint4(col[0], col[1], col[2], col[3]);
      to[1] = make_uint4(col[4], col[5], col[6], col[7]);
    }
  }
  if constexpr (DIRECT) {
    const int64_t ld = (cols + 127) / 128 * 128;
    uint8_t* to = codes + r0 * ld + c0;
    uint8_t* scale_to = scales + fp8_scale_at(rows, r0, cb);
    const int there = (int)min(rows - r0, (int64_t)8);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int byte = fp8_scale_byte(row16_max(row[p]));
      const float scale = fp8_power(byte);
      const uint2 w = make_uint2(fp8_codes4(v[p][0], v[p][1], v[p][2], v[p][3], scale),
                                 fp8_codes4(v[p][4], v[p][5], v[p][6], v[p][7], scale));
      if (p < there) {
        *reinterpret_cast<uint2*>(to) = w;
        if (cg == 0) scale_to[4 * p] = (uint8_t)byte;
      }
      to += ld;
    }
  }
  if constexpr (TURNED) {
    __syncthreads();
    const int64_t ld = (rows + 127) / 128 * 128;
    uint8_t* scale_to = scales_t + fp8_scale_at(cols, c0, rb);
    const int there = (int)min(max(cols - c0, (int64_t)0), (int64_t)8);
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 o = *reinterpret_cast<const uint4*>(&tops[w * 128 + 8 * cg + 4 * h]);
        col[4 * h] = max(col[4 * h], o.x);
        col[4 * h + 1] = max(col[4 * h + 1], o.y);
        col[4 * h + 2] = max(col[4 * h + 2], o.z);
        col[4 * h + 3] = max(col[4 * h + 3], o.w);
      }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int byte = fp8_scale_byte(col[j]);
      const float scale = fp8_power(byte);
      tile[(8 * cg + j) * 16 + (rg ^ cg)] = make_uint2(fp8_codes4(v[0][j], v[1][j], v[2][j], v[3][j], scale),
                                                       fp8_codes4(v[4][j], v[5][j], v[6][j], v[7][j], scale));
      if (rg == j && j < there) scale_to[4 * j] = (uint8_t)byte;
    }
    __syncthreads();
    // a row of turned codes is eight lanes' 16 bytes: two of the 8-byte slots
    const int c = t >> 3, pair = t & 7;
    const int64_t left = cols - cb * 128 - c;
    uint8_t* to = codes_t + (cb * 128 + c) * ld + rb * 128 + 16 * pair;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = c + 32 * i;
      const uint4 w = *reinterpret_cast<const uint4*>(&tile[at * 16 + 2 * (pair ^ (at >> 4))]);
      const bool swap = (at >> 3) & 1;
      if (32 * i < left) *reinterpret_cast<uint4*>(to) = swap ? make_uint4(w.z, w.w, w.x, w.y) : w;
      to += 32 * ld;
    }
  }
}

template <int SRC>
hipError_t launch(const Source& src, int64_t rows, int64_t cols, const fairy2i_fp8_matrix* direct,
                  const fairy2i_fp8_matrix* turned, hipStream_t s) {
  const int64_t row_tiles = (rows + 127) / 128, col_tiles = (cols + 127) / 128;
  const dim3 grid((unsigned)(row_tiles * col_tiles)), block(256);
  uint8_t *c = direct ? direct->codes : nullptr, *f = direct ? direct->scales : nullptr;
  uint8_t *ct = turned ? turned->codes : nullptr, *ft = turned ? turned->scales : nullptr;
  if constexpr (SRC != kFp8) {  // an 8-bit matrix is only ever turned
    if (direct) {
      if (turned)
        hipLaunchKernelGGL((fp8_quantize_kernel<SRC, true, true>), grid, block, 0, s, src, rows, cols, (int)col_tiles,
                           c, f, ct, ft);
      else
        hipLaunchKernelGGL((fp8_quantize_kernel<SRC, true, false>), grid, block, 0, s, src, rows, cols, (int)col_tiles,
                           c, f, ct, ft);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((fp8_quantize_kernel<SRC, false, true>), grid, block, 0, s, src, rows, cols, (int)col_tiles, c, f,
                     ct, ft);
  return hipGetLastError();
}

// Eight codes a thread -> eight bf16 values: exact (four significant bits, a
// normal power of two).
__global__ __launch_bounds__(256) void fp8_dequantize_kernel(Source src, int64_t rows, int64_t cols,
                                                             uint16_t* __restrict__ out) {
  const int64_t groups = src.ld / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * groups; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / groups, c = i % groups * 8;
    if (c >= cols) continue;
    float v[8];
    load8_at<kFp8>(src, rows, r, c, v);
    uint16_t* p = out + r * cols + c;
    if (c + 8 <= cols) {
      *reinterpret_cast<u32x4_any*>(p) =
          u32x4_any{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j < cols) p[j] = bf16_one(v[j]);
    }
  }
}

// A launch takes fewer than 2^32 threads.
bool too_many_tiles(int64_t rows, int64_t cols) {
  return ((rows + 127) / 128) * ((cols + 127) / 128) >= ((int64_t)1 << 24);
}

}  // namespace

}  // namespace fairy2i

using namespace fairy2i;

extern "C" {

size_t fairy2i_fp8_codes_bytes(int64_t rows, int64_t cols) {
  if (rows < 1 || cols < 1 || rows > kFp8MostSide || cols > kFp8MostSide) return 0;
  return (size_t)(rows * fp8_ld(cols));
}

size_t fairy2i_fp8_scales_bytes(int64_t rows, int64_t cols) {
  if (rows < 1 || cols < 1 || rows > kFp8MostSide || cols > kFp8MostSide) return 0;
  return (size_t)((cols + 511) / 512 * rows * 4);
}

fairy2i_status fairy2i_fp8_quantize(const void* x, int32_t dtype, int64_t ld, const fairy2i_fp8_matrix* direct,
                                    const fairy2i_fp8_matrix* turned, void* stream) {
  if (!x || (!direct && !turned)) return FAIRY2I_ERR_NULL;
  for (const fairy2i_fp8_matrix* m : {direct, turned})
    if (m) {
      const fairy2i_status st = fp8_check(m);
      if (st != FAIRY2I_OK) return st;
    }
  const int64_t rows = direct ? direct->rows : turned->cols, cols = direct ? direct->cols : turned->rows;
  if (turned && (turned->cols != rows || turned->rows != cols)) return FAIRY2I_ERR_SHAPE;
  if (ld < cols) return FAIRY2I_ERR_SHAPE;
  if (dtype != FAIRY2I_ACT_F32 && dtype != FAIRY2I_ACT_BF16) return FAIRY2I_ERR_DTYPE;
  if (too_many_tiles(rows, cols) || (direct && turned && fp8_overlap(direct, turned))) return FAIRY2I_ERR_UNSUPPORTED;
  const int size = dtype == FAIRY2I_ACT_F32 ? 4 : 2;
  for (const fairy2i_fp8_matrix* m : {direct, turned})
    if (m && fp8_overlap(m, x, rows, cols, ld, size)) return FAIRY2I_ERR_UNSUPPORTED;
  const Source src{x, nullptr, ld};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const hipError_t e = dtype == FAIRY2I_ACT_F32 ? launch<kF32>(src, rows, cols, direct, turned, s)
                                                : launch<kBf16>(src, rows, cols, direct, turned, s);
  return e == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

fairy2i_status fairy2i_fp8_transpose(const fairy2i_fp8_matrix* in, const fairy2i_fp8_matrix* out, void* stream) {
  for (const fairy2i_fp8_matrix* m : {in, out}) {
    const fairy2i_status st = fp8_check(m);
    if (st != FAIRY2I_OK) return st;
  }
  if (out->rows != in->cols || out->cols != in->rows) return FAIRY2I_ERR_SHAPE;
  if (too_many_tiles(in->rows, in->cols) || fp8_overlap(in, out)) return FAIRY2I_ERR_UNSUPPORTED;
  const Source src{in->codes, in->scales, fp8_ld(in->cols)};
  const hipError_t e = launch<kFp8>(src, in->rows, in->cols, nullptr, out, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

fairy2i_status fairy2i_fp8_dequantize(const fairy2i_fp8_matrix* in, void* out, void* stream) {
  const fairy2i_status st = fp8_check(in);
  if (st != FAIRY2I_OK) return st;
  if (!out) return FAIRY2I_ERR_NULL;
  if (fp8_overlap(in, out, 1, in->rows * in->cols, 0, 2)) return FAIRY2I_ERR_UNSUPPORTED;
  const Source src{in->codes, in->scales, fp8_ld(in->cols)};
  const int64_t work = in->rows * (src.ld / 8);
  const unsigned blocks = (unsigned)std::min<int64_t>((work + 255) / 256, 1 << 20);
  hipLaunchKernelGGL(fp8_dequantize_kernel, dim3(blocks), dim3(256), 0, static_cast<hipStream_t>(stream), src,
                     in->rows, in->cols, static_cast<uint16_t*>(out));
  return hipGetLastError() == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

}  // extern "C"
