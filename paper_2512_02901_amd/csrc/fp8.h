// The 8-bit matrices of the training operators (fairy2i_fp8_matrix): e4m3
// codes with one power of two for 128 neighbours of a row.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "common.h"

namespace fairy2i {

constexpr int kFp8Block = 128;
constexpr int64_t kFp8MostSide = (int64_t)1 << 22;  // rows or columns
constexpr int kFp8LeastScale = 127 - 117, kFp8MostScale = 127 + 119;

// Loads and stores of any element's alignment: the hardware takes them whole.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));

inline int64_t fp8_ld(int64_t cols) { return (cols + kFp8Block - 1) / kFp8Block * kFp8Block; }

// Sizes, pointers and alignment.
inline fairy2i_status fp8_check(const fairy2i_fp8_matrix* m) {
  if (!m || !m->codes || !m->scales) return FAIRY2I_ERR_NULL;
  if (m->rows < 1 || m->cols < 1 || m->rows > kFp8MostSide || m->cols > kFp8MostSide) return FAIRY2I_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(m->codes) & 15) || (reinterpret_cast<uintptr_t>(m->scales) & 3))
    return FAIRY2I_ERR_UNSUPPORTED;
  return FAIRY2I_OK;
}

// Memory of a matrix: codes, scales.
struct Fp8Range {
  uint64_t first, last;
};
inline Fp8Range fp8_codes_range(const fairy2i_fp8_matrix* m) {
  const uint64_t p = reinterpret_cast<uintptr_t>(m->codes);
  return {p, p + (uint64_t)(m->rows * fp8_ld(m->cols))};
}
inline Fp8Range fp8_scales_range(const fairy2i_fp8_matrix* m) {
  const uint64_t p = reinterpret_cast<uintptr_t>(m->scales);
  return {p, p + (uint64_t)((m->cols + 511) / 512 * m->rows * 4)};
}

// Whether two matrices share memory.
inline bool fp8_overlap(const fairy2i_fp8_matrix* a, const fairy2i_fp8_matrix* b) {
  for (const Fp8Range& x : {fp8_codes_range(a), fp8_scales_range(a)})
    for (const Fp8Range& y : {fp8_codes_range(b), fp8_scales_range(b)})
      if (x.first < y.last && y.first < x.last) return true;
  return false;
}

// Whether a matrix shares memory with `rows` rows of `width` elements of `size`
// bytes, ld >= width elements apart: what lies between the rows is others'.
inline bool fp8_overlap(const fairy2i_fp8_matrix* m, const void* p, int64_t rows, int64_t width, int64_t ld, int size) {
  const uint64_t base = reinterpret_cast<uintptr_t>(p), bytes = (uint64_t)(width * size);
  // rows further apart than memory is large: the first is all that could
  const uint64_t pitch = rows > 1 ? (uint64_t)std::min(ld, (int64_t)1 << 56) * (uint64_t)size : bytes;
  for (const Fp8Range& x : {fp8_codes_range(m), fp8_scales_range(m)}) {
    if (x.last <= base) continue;
    // the first row that ends behind x.first
    const uint64_t row = x.first < base + bytes ? 0 : (x.first - base - bytes) / pitch + 1;
    if (row < (uint64_t)rows && base + row * pitch < x.last) return true;
  }
  return false;
}

// Byte of block `kb` of row r in the scales of a matrix of `rows` rows.
__host__ __device__ inline int64_t fp8_scale_at(int64_t rows, int64_t r, int64_t kb) {
  return ((kb >> 2) * rows + r) * 4 + (kb & 3);
}

// |v| as bits for the maximum; what is not finite does not count.
__device__ inline uint32_t fp8_magnitude(float v) {
  const uint32_t a = __float_as_uint(v) & 0x7FFFFFFFu;
  return a < 0x7F800000u ? a : 0u;
}

// Largest magnitude of a block -> its scale byte: the smallest e with
// top <= 448 * 2^e = 1.75 * 2^(8 + e), within [-117, 119].  The ends keep every
// value and both powers normal float32 and bf16 numbers.
__device__ inline int fp8_scale_byte(uint32_t top) {
  const int e = (int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u);
  return min(max(e, kFp8LeastScale), kFp8MostScale);
}

__device__ inline float fp8_power(int byte) { return __uint_as_float((uint32_t)byte << 23); }  // 2^(byte - 127)

// Above this lie what e = 119 cannot hold and what is not finite (as bits of an absolute value).
constexpr uint32_t kFp8Most = 0x7F600000u;  // 448 * 2^119

// A value as it is held: beyond the largest that one, a NaN for what is not
// finite.  Only blocks with a magnitude past kFp8Most need it.
__device__ inline float fp8_tame(float v) {
  const uint32_t a = __float_as_uint(v) & 0x7FFFFFFFu;
  if (a >= 0x7F800000u) return __builtin_nanf("");
  return a > kFp8Most ? copysignf(__uint_as_float(kFp8Most), v) : v;
}

// Four reals of a block of scale 2^e -> four codes, rounded to nearest even by the
// conversion instruction, which divides by the power of two on its way.
__device__ inline uint32_t fp8_codes4(float a, float b, float c, float d, float scale) {
  typedef short v2s __attribute__((ext_vector_type(2)));
  v2s w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, w);
}

// Maximum over the 16 lanes of a DPP row, in all of them.
__device__ inline uint32_t row16_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));  // row_ror:8
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, false));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, false));
  return v;
}

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two floats -> two bf16, nearest even (a NaN stays one).
__device__ inline uint32_t bf16_pair(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}

__device__ inline uint16_t bf16_one(float a) { return __builtin_bit_cast(uint16_t, (__bf16)a); }

}  // namespace fairy2i
