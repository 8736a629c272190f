// Product of two 8-bit matrices, C = A B^T, on the matrix cores.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 codes and
// takes a power of two for every 32 codes of a row; a block of 128 along the
// summed axis has one, so a step of 128 is one instruction a 16 x 16 tile of C
// with both rows' scale bytes as operands and no other arithmetic.
//
// A block of waves takes BM x BN of C and walks K in steps of 128, double
// buffered in LDS: a step's codes arrive by direct-to-LDS loads (1 KB of eight
// rows an instruction) while the step before is multiplied.  The 16-byte chunk
// c of row r lies at chunk c ^ (r & 7), which the loading lanes' addresses
// arrange, so neither side of LDS meets a bank conflict.  Scales come four
// steps at a time, a dword a row.
#include <algorithm>

#include "fp8.h"

namespace fairy2i {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;

struct Gemm {
  const uint8_t* a;
  const uint8_t* a_scales;
  const uint8_t* b;
  const uint8_t* b_scales;
  int64_t M, N, ld;  // ld: bytes of a row, K rounded up to whole steps
  int steps;
  int steps_per_split;  // a multiple of 4
  int tiles_m, tiles_n;
  void* c;
  int64_t ldc;
  int bf16, accumulate;
  float* parts;  // [splits][M][N], or null
};

// Row of C from column n on, four values (fewer at the end of a row).
__device__ inline void store4(const Gemm& g, int64_t m, int64_t n, v4f v, int split) {
  const int count = (int)min((int64_t)4, g.N - n);
  if (g.parts) {
    float* p = g.parts + ((int64_t)split * g.M + m) * g.N + n;
    if (count == 4)
      *reinterpret_cast<f32x4_any*>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
    else
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < count) p[j] = v[j];
  } else if (g.bf16) {
    uint16_t* p = static_cast<uint16_t*>(g.c) + m * g.ldc + n;
    typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
    if (count == 4) {
      if (g.accumulate) {
        const u32x2_any o = *reinterpret_cast<const u32x2_any*>(p);
        v += v4f{bf16_lo(o[0]), bf16_hi(o[0]), bf16_lo(o[1]), bf16_hi(o[1])};
      }
      *reinterpret_cast<u32x2_any*>(p) = u32x2_any{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < count) p[j] = bf16_one(v[j] + (g.accumulate ? __uint_as_float((uint32_t)p[j] << 16) : 0.0f));
    }
  } else {
    float* p = static_cast<float*>(g.c) + m * g.ldc + n;
    if (count == 4) {
      if (g.accumulate) {
        const f32x4_any o = *reinterpret_cast<const f32x4_any*>(p);
        v += v4f{o[0], o[1], o[2], o[3]};
      }
      *reinterpret_cast<f32x4_any*>(p) = f32x4_any{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < count) p[j] = v[j] + (g.accumulate ? p[j] : 0.0f);
    }
  }
}

// Which tile of C a block takes: the blocks that one XCD runs at a time
// (every eighth of the grid) take neighbouring tiles, eight rows of tiles deep,
// so they meet each other's operands in their L2.
__device__ inline void tile_of(const Gemm& g, int id, int& tm, int& tn) {
  const int total = g.tiles_m * g.tiles_n;
  const int per = total / 8, left = total % 8, xcd = id % 8;
  const int t = xcd * per + min(xcd, left) + id / 8;
  const int deep = 8, band = t / (deep * g.tiles_n), in = t % (deep * g.tiles_n);
  const int rows = min(deep, g.tiles_m - band * deep);
  tm = band * deep + in % rows;
  tn = in / rows;
}

template <int BM, int BN, int WM, int WN, int BLOCKS>
__global__ __launch_bounds__(64 * WM * WN, BLOCKS) void gemm_fp8_kernel(Gemm g) {
#if defined(__HIP_DEVICE_COMPILE__)  // LDS-DMA and buffer-descriptor code: device pass only
  constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr int PIECES = (BM + BN) / 8 / WAVES;  // 1 KB loads of a wave and step
  constexpr int SCALE_LOADS = (BM + BN) / 64;    // of 64 rows
  __shared__ __attribute__((aligned(16))) uint8_t codes[2][(BM + BN) * 128];
  __shared__ uint32_t scales[2][BM + BN];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int wm = wave % WM, wn = wave / WM;
  int tm, tn;
  tile_of(g, (int)blockIdx.x, tm, tn);
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  const int split = (int)blockIdx.y;
  const int k0 = split * g.steps_per_split, k1 = min(k0 + g.steps_per_split, g.steps);

  // This wave's pieces of a step: eight rows each, of A's tile first, then of B's.
  // Rows past the matrix's end read its last row.
  const uint8_t* piece_at[PIECES];
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int p = wave * PIECES + i;
    const bool of_a = p < BM / 8;
    const int64_t r = (of_a ? m0 + 8 * p : n0 + 8 * (p - BM / 8)) + (lane >> 3);
    const int64_t row = min(r, (of_a ? g.M : g.N) - 1);
    piece_at[i] = (of_a ? g.a : g.b) + row * g.ld + 16 * ((lane & 7) ^ (lane >> 3));
  }
  auto issue = [&](int k, int buf) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(piece_at[i] + (int64_t)k * 128),
          (lds_ptr_t)&codes[buf][(wave * PIECES + i) * 1024], 16, 0, 0);
  };
  auto issue_scales = [&](int k4, int buf) {
#pragma unroll
    for (int i = 0; i < (SCALE_LOADS + WAVES - 1) / WAVES; ++i) {
      const int p = wave + i * WAVES;
      if (p >= SCALE_LOADS) break;
      const bool of_a = p < BM / 64;
      const int64_t rows = of_a ? g.M : g.N;
      const int64_t row = min((of_a ? m0 + 64 * p : n0 + 64 * (p - BM / 64)) + lane, rows - 1);
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)((of_a ? g.a_scales : g.b_scales) + (k4 * rows + row) * 4),
          (lds_ptr_t)&scales[buf][p * 64], 4, 0, 0);
    }
  };

  v4f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
  uint32_t sa[TM], sb[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) sa[i] = 0;
#pragma unroll
  for (int j = 0; j < TN; ++j) sb[j] = 0;

  const int r16 = lane & 15, q = lane >> 4;
  // chunks q and q + 4 of a row are this lane's 32 codes (of both operands alike)
  const int lo = 16 * (q ^ (r16 & 7)), hi = 16 * ((q + 4) ^ (r16 & 7));
  auto load = [&](int buf, int row) {
    const uint8_t* p = &codes[buf][(row + r16) * 128];
    const v4i x = *reinterpret_cast<const v4i*>(p + lo), y = *reinterpret_cast<const v4i*>(p + hi);
    return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto compute = [&](int k, int buf) {
    if ((k & 3) == 0) {
      const int sbuf = (k >> 2) & 1;
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = scales[sbuf][wm * TM * 16 + 16 * i + r16];
#pragma unroll
      for (int j = 0; j < TN; ++j) sb[j] = scales[sbuf][BM + wn * TN * 16 + 16 * j + r16];
    }
    v8i fb[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j] = load(buf, BM + wn * TN * 16 + 16 * j);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const v8i fa = load(buf, wm * TM * 16 + 16 * i);
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa, acc[i][j], 0, 0, 0, (int)sb[j], 0,
                                                                     (int)sa[i]);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) sa[i] >>= 8;
#pragma unroll
    for (int j = 0; j < TN; ++j) sb[j] >>= 8;
  };

  // One barrier a step: after it every wave has its share of step k in LDS and
  // has done with step k - 1, whose buffer step k + 1 then fills.  k0 is a
  // multiple of 4.
  issue_scales(k0 >> 2, (k0 >> 2) & 1);
  issue(k0, 0);
  for (int k = k0; k < k1; ++k) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (k + 1 < k1) {
      issue(k + 1, (k + 1) & 1);
      if (((k + 1) & 3) == 0) issue_scales((k + 1) >> 2, ((k + 1) >> 2) & 1);
    }
    compute(k, k & 1);
  }

#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int64_t m = m0 + wm * TM * 16 + 16 * i + r16;
    if (m >= g.M) continue;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int64_t n = n0 + wn * TN * 16 + 16 * j + 4 * q;
      if (n < g.N) store4(g, m, n, acc[i][j], split);
    }
  }
#endif
}

// Sums of the splits' parts, in order.
__global__ __launch_bounds__(256) void gemm_fp8_join_kernel(Gemm g, int splits) {
  const int64_t groups = (g.N + 3) / 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < g.M * groups; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / groups, n = i % groups * 4;
    const int count = (int)min((int64_t)4, g.N - n);
    v4f v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) {
      const float* p = g.parts + ((int64_t)s * g.M + m) * g.N + n;
      if (count == 4) {
        const f32x4_any o = *reinterpret_cast<const f32x4_any*>(p);
        v += v4f{o[0], o[1], o[2], o[3]};
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < count) v[j] += p[j];
      }
    }
    Gemm out = g;
    out.parts = nullptr;
    store4(out, m, n, v, 0);
  }
}

// Tile sizes, and how many splits of K: see plan_of.
struct Plan {
  int tile;  // 0: 256 x 256, 1: 128 x 128, 2: 64 x 64
  int splits, steps_per_split;
};

constexpr int kSide[3] = {256, 128, 64};

Plan plan_of(int64_t M, int64_t N, int64_t K) {
  const int steps = (int)((K + 127) / 128);
  auto tiles = [&](int side) { return ((M + side - 1) / side) * ((N + side - 1) / side); };
  Plan p;
  p.tile = tiles(256) >= 192 ? 0 : tiles(128) >= 128 ? 1 : 2;
  const int64_t t = tiles(kSide[p.tile]);
  int64_t splits = 1;
  if (p.tile > 0) splits = std::max<int64_t>(1, std::min<int64_t>(512 / t, steps / 8));
  const int64_t quads = (steps + 3) / 4;
  splits = std::min(splits, quads);
  p.steps_per_split = (int)((quads + splits - 1) / splits * 4);
  p.splits = (steps + p.steps_per_split - 1) / p.steps_per_split;
  return p;
}

bool sizes_ok(int64_t M, int64_t N, int64_t K) {
  return M >= 1 && N >= 1 && K >= 1 && M <= kFp8MostSide && N <= kFp8MostSide && K <= kFp8MostSide;
}

}  // namespace

}  // namespace fairy2i

using namespace fairy2i;

extern "C" {

size_t fairy2i_gemm_fp8_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  if (!sizes_ok(M, N, K)) return 0;
  const Plan p = plan_of(M, N, K);
  return p.splits > 1 ? sizeof(float) * (size_t)p.splits * (size_t)M * (size_t)N : 0;
}

fairy2i_status fairy2i_gemm_fp8(const fairy2i_fp8_matrix* A, const fairy2i_fp8_matrix* B, void* C, int32_t dtype,
                                int64_t ldc, int32_t accumulate, void* workspace, size_t workspace_bytes,
                                void* stream) {
  for (const fairy2i_fp8_matrix* m : {A, B}) {
    const fairy2i_status st = fp8_check(m);
    if (st != FAIRY2I_OK) return st;
  }
  if (!C) return FAIRY2I_ERR_NULL;
  if (A->cols != B->cols || ldc < B->rows || (accumulate != 0 && accumulate != 1)) return FAIRY2I_ERR_SHAPE;
  if (dtype != FAIRY2I_ACT_F32 && dtype != FAIRY2I_ACT_BF16) return FAIRY2I_ERR_DTYPE;
  const int64_t M = A->rows, N = B->rows, K = A->cols;
  const Plan p = plan_of(M, N, K);
  const size_t need = fairy2i_gemm_fp8_workspace_bytes(M, N, K);
  if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 3)))
    return FAIRY2I_ERR_WORKSPACE;
  const int side = kSide[p.tile];
  Gemm g{A->codes,
         A->scales,
         B->codes,
         B->scales,
         M,
         N,
         fp8_ld(K),
         (int)(fp8_ld(K) / 128),
         p.steps_per_split,
         (int)((M + side - 1) / side),
         (int)((N + side - 1) / side),
         C,
         ldc,
         dtype == FAIRY2I_ACT_BF16,
         accumulate,
         need > 0 ? static_cast<float*>(workspace) : nullptr};
  const int64_t tiles = (int64_t)g.tiles_m * g.tiles_n;
  if (tiles >= ((int64_t)1 << 22)) return FAIRY2I_ERR_UNSUPPORTED;  // a launch takes fewer than 2^32 threads
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)tiles, (unsigned)p.splits);
  if (p.tile == 0)
    hipLaunchKernelGGL((gemm_fp8_kernel<256, 256, 2, 4, 1>), grid, dim3(512), 0, s, g);
  else if (p.tile == 1)
    hipLaunchKernelGGL((gemm_fp8_kernel<128, 128, 2, 2, 2>), grid, dim3(256), 0, s, g);
  else
    hipLaunchKernelGGL((gemm_fp8_kernel<64, 64, 2, 2, 2>), grid, dim3(256), 0, s, g);
  if (p.splits > 1) {
    const int64_t groups = M * ((N + 3) / 4);
    const unsigned blocks = (unsigned)std::min<int64_t>((groups + 255) / 256, 4096);
    hipLaunchKernelGGL(gemm_fp8_join_kernel, dim3(blocks), dim3(256), 0, s, g, p.splits);
  }
  return hipGetLastError() == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

}  // extern "C"
