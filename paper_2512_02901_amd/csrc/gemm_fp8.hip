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
//
// 4096 x 4096 over 11008: 122-132 us on different cards, 2.8-3.0 PFLOP/s (a library product of codes
// without scales: 114-118); 8192^3: 363 us, 3.0 PFLOP/s (341).  The matrix cores are
// busy for 70 and 76 % of the cycles, at the 1.9-1.96 GHz that the card holds under
// them; no LDS conflicts.  What is left are the barrier of each step and the codes'
// way into LDS, some 43 bytes a clock and CU.  Four waves of 128 x 128 sums each read
// 32 KB of LDS a wave and step; eight of 128 x 64 read 1.5 times as much in all and
// take 201 us for the first product.  The instruction for 32 x 32 x 64 sums runs at
// 4.37 PFLOP/s on random codes, this one at 4.72.  Small products are bound by the
// chain of steps: 16 x 512 over 512 4.0 us.
#include <algorithm>
#include <utility>

#include "fp8.h"

namespace fairy2i {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;

__device__ inline __amdgpu_buffer_rsrc_t rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)bytes, 0x00020000);
}

template <int V>
struct Constant {
  static constexpr int value = V;
};

// f(Constant<0>) .. f(Constant<N - 1>): what stands between two products is placed at compile time.
template <int... I, typename F>
__device__ __attribute__((always_inline)) inline void each_of(std::integer_sequence<int, I...>, F&& f) {
  (f(Constant<I>{}), ...);
}
template <int N, typename F>
__device__ __attribute__((always_inline)) inline void each(F&& f) {
  each_of(std::make_integer_sequence<int, N>{}, f);
}
// Slot T's share of N things that are spread over IN slots.
template <int N, int IN, int T, typename F>
__device__ __attribute__((always_inline)) inline void some(F&& f) {
  if constexpr (T < IN)
    each<(T + 1) * N / IN - T * N / IN>(
        [&](auto i) __attribute__((always_inline)) { f(Constant<T * N / IN + decltype(i)::value>{}); });
}

// c += 16 x 128 codes of a times those of b, scaled by byte U of sa and sb.  The
// sums are asked for in accumulation registers and the operands in vector ones:
// left to itself the compiler moves both to and fro where a wave has 256 sums.
// It does not see the hazards of an instruction written so: an operand that it
// has just written needs two wait states (the s_nop), a sum read by anything but a
// product needs settle() first.
template <int U>
__device__ __attribute__((always_inline)) inline void product(v4f& c, const v8i& a, const v8i& b, uint32_t sa, uint32_t sb) {
  if constexpr (U == 0)
    asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]"
                 : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
  else if constexpr (U == 1)
    asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0]"
                 : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
  else if constexpr (U == 2)
    asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[1,1,0]"
                 : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
  else
    asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[1,1,0]"
                 : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb));
}

// Past the last product's eight passes: its sums may be read.
template <int TM, int TN>
__device__ __attribute__((always_inline)) inline void settle(v4f (&acc)[TM][TN]) {
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) asm volatile("" : "+a"(acc[i][j]));
}

// Operand of s_waitcnt: no LDS operation under way, `loads` loads at most.
constexpr int wait_loads(int loads) { return 0x70 | (loads & 15) | loads >> 4 << 14; }

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
  if (count <= 0) return;
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
// (every eighth of the grid) take neighbouring tiles, four rows of tiles deep,
// so they meet each other's operands in their L2.
__device__ inline void tile_of(const Gemm& g, int id, int& tm, int& tn) {
  const int total = g.tiles_m * g.tiles_n;
  const int per = total / 8, left = total % 8, xcd = id % 8;
  const int t = xcd * per + min(xcd, left) + id / 8;
  const int deep = 4, band = t / (deep * g.tiles_n), in = t % (deep * g.tiles_n);
  const int rows = min(deep, g.tiles_m - band * deep);
  tm = band * deep + in % rows;
  tn = in / rows;
}

// BM x BN of C by WM x WN waves, BLOCKS blocks a CU; STAGES steps in LDS (2 or 4);
// AHEAD: how many steps ahead lines are asked for (0: not).
template <int BM, int BN, int WM, int WN, int STAGES, int BLOCKS, int AHEAD>
__global__ __launch_bounds__(64 * WM * WN, BLOCKS) void gemm_fp8_kernel(Gemm g) {
#if defined(__HIP_DEVICE_COMPILE__)  // LDS-DMA and buffer-descriptor code: device pass only
  constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
  constexpr int PA = BM / 8 / WAVES, PB = BN / 8 / WAVES;  // 1 KB loads of a wave and step
  constexpr int SA = (BM + 63) / 64, SB = (BN + 63) / 64, SCALES = 64 * (SA + SB);  // loads of 64 rows' scales
  constexpr int SLOTS = TM * TN, HALF = SLOTS / 2;
  constexpr int STAGE = (BM + BN) * 128;
  // several arrays and not one of several: loads into one never order reads of another
  __shared__ __attribute__((aligned(16))) uint8_t codes0[STAGE];
  __shared__ __attribute__((aligned(16))) uint8_t codes1[STAGE];
  __shared__ __attribute__((aligned(16))) uint8_t codes2[STAGES > 2 ? STAGE : 16];
  __shared__ __attribute__((aligned(16))) uint8_t codes3[STAGES > 2 ? STAGE : 16];
  __shared__ uint32_t scales[2 * SCALES];
  __shared__ uint32_t asked[AHEAD ? 64 : 1];  // never read
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int wm = wave % WM, wn = wave / WM;
  auto buffer = [&](auto k) __attribute__((always_inline)) {  // of step k
    constexpr int b = decltype(k)::value % STAGES;
    if constexpr (b == 0) return &codes0[0];
    else if constexpr (b == 1) return &codes1[0];
    else if constexpr (b == 2) return &codes2[0];
    else return &codes3[0];
  };
  int tm, tn;
  tile_of(g, (int)blockIdx.x, tm, tn);
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  const int split = (int)blockIdx.y;
  const int k0 = split * g.steps_per_split, k1 = min(k0 + g.steps_per_split, g.steps);

  // A tile's rows as a buffer: rows past the matrix's end are past the buffer's
  // and read as zeros, steps past the last one find an empty buffer.
  const uint32_t ld = (uint32_t)g.ld;
  const uint8_t *base_a = g.a + m0 * g.ld, *base_b = g.b + n0 * g.ld;
  const uint32_t bytes_a = (uint32_t)min((int64_t)BM, g.M - m0) * ld;
  const uint32_t bytes_b = (uint32_t)min((int64_t)BN, g.N - n0) * ld;
  const uint32_t at = (uint32_t)(8 * wave + (lane >> 3)) * ld + 16u * (uint32_t)((lane & 7) ^ (lane >> 3));
  auto issue = [&](int k, int i, uint8_t* codes) {  // load i (A's, then B's) of step k
    const bool of_a = i < PA;
    const int p = of_a ? i : i - PA;
    const __amdgpu_buffer_rsrc_t r = rsrc(of_a ? base_a : base_b, k < k1 ? (of_a ? bytes_a : bytes_b) : 0u);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)&codes[((of_a ? 0 : BM / 8) + p * WAVES + wave) * 1024], 16,
                                             at + (uint32_t)(p * WAVES * 8) * ld, (uint32_t)k * 128u, 0, 0);
  };
  // One line of each row a few steps on, into the L2: the tiles that run beside this
  // one on its XCD (eight in a row of tiles, four in a column) share the rows out.
  const uint32_t ask_a =
      lane < BM / 8 / WAVES ? (uint32_t)(BM / 8 * (tn & 7) + BM / 8 / WAVES * wave + lane) * ld : 0xFFFFFFF0u;
  const uint32_t ask_b =
      lane < BN / 4 / WAVES ? (uint32_t)(BN / 4 * (tm & 3) + BN / 4 / WAVES * wave + lane) * ld : 0xFFFFFFF0u;
  auto ask = [&](int k) {
    const bool there = k < k1;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(base_a, there ? bytes_a : 0u), (lds_ptr_t)&asked[0], 4, ask_a,
                                             (uint32_t)k * 128u, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(base_b, there ? bytes_b : 0u), (lds_ptr_t)&asked[0], 4, ask_b,
                                             (uint32_t)k * 128u, 0, 0);
  };
  // Scales of four steps, a dword a row: 64 rows a load.
  auto issue_scales = [&](int k4) {
#pragma unroll
    for (int i = 0; i < (SA + SB + WAVES - 1) / WAVES; ++i) {
      const int p = wave + i * WAVES;
      const bool of_a = p < SA;
      const int64_t rows = of_a ? g.M : g.N, first = of_a ? m0 : n0;
      const __amdgpu_buffer_rsrc_t r = rsrc((of_a ? g.a_scales : g.b_scales) + (k4 * rows + first) * 4,
                                            4 * k4 < k1 ? (uint32_t)min(rows - first, (int64_t)256) * 4u : 0u);
      if ((SA + SB) % WAVES == 0 || p < SA + SB)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr_t)&scales[(k4 & 1) * SCALES + p * 64], 4,
                                                 4u * (uint32_t)(64 * (of_a ? p : p - SA) + lane), 0, 0, 0);
    }
  };

  v4f acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};

  const int r16 = lane & 15, q = lane >> 4;
  // chunks q and q + 4 of a row are this lane's 32 codes (of both operands alike)
  const int lo = r16 * 128 + 16 * (q ^ (r16 & 7)), hi = r16 * 128 + 16 * ((q + 4) ^ (r16 & 7));
  const int row_a = wm * TM * 16, row_b = BM + wn * TN * 16;
  auto half = [&](const uint8_t* codes, int row, int h) {
    return *reinterpret_cast<const v4i*>(&codes[row * 128 + (h ? hi : lo)]);
  };
  auto whole = [](const v4i& x, const v4i& y) { return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7); };

  uint32_t sa[TM], sb[TN], sa_next[TM], sb_next[TN];
  auto read_scale = [&](int k4, int i) {
    const uint32_t* f = &scales[(k4 & 1) * SCALES];
    if (i < TM)
      sa_next[i] = f[row_a + 16 * i + r16];
    else
      sb_next[i - TM] = f[64 * SA + wn * TN * 16 + 16 * (i - TM) + r16];
  };
  // Step k, whose first fragments (A's first, B's all) are in registers and whose
  // codes are in `mine`.  First half, rows of tiles 0 .. TM / 2 - 1: reads of the
  // rest of its A fragments.  Then `mine` is free and step k + 1 is in `other`: one
  // barrier.  Second half, the other rows' tiles column by column: step k + 2's
  // loads into `mine`, and as a column's B fragment has served, step k + 1's in its
  // place.  A product keeps the matrix core busy for 32 cycles, an instruction or
  // two stand between two of them.
  v4i fb[TN][2], first[2];
  auto step = [&](int k, auto which) __attribute__((always_inline)) {
    constexpr int U = decltype(which)::value;
    uint8_t *mine = buffer(which), *other = buffer(Constant<U + 1>{});
    v4i fa[TM][2];
    fa[0][0] = first[0];
    fa[0][1] = first[1];
    each<SLOTS>([&](auto slot) __attribute__((always_inline)) {
      constexpr int s = decltype(slot)::value, t = s - HALF, R = TM / 2;
      constexpr int i = s < HALF ? s / TN : R + t % R, j = s < HALF ? s % TN : t / R;
      product<U>(acc[i][j], whole(fb[j][0], fb[j][1]), whole(fa[i][0], fa[i][1]), sb[j], sa[i]);
      if constexpr (s < HALF) {
        constexpr int READS = 2 * (TM - 1), IN = HALF > 8 ? HALF - 4 : HALF > 2 ? HALF - 2 : 1;
        some<READS, IN, s>([&](auto r) __attribute__((always_inline)) {
          constexpr int n = 1 + decltype(r)::value / 2, h = decltype(r)::value % 2;
          fa[n][h] = half(mine, row_a + 16 * n, h);
        });
      } else {
        constexpr int IN = HALF - 1;
        if constexpr (t == 0 && (U + STAGES) % 4 == 0) issue_scales((k + STAGES) >> 2);
        some<PA + PB, IN, t>([&](auto r) __attribute__((always_inline)) { issue(k + STAGES, decltype(r)::value, mine); });
        if constexpr (t < 2) first[t] = half(other, row_a, t);
        if constexpr (t % R == R - 1) {
          fb[j][0] = half(other, row_b + 16 * j, 0);
          fb[j][1] = half(other, row_b + 16 * j, 1);
        }
        if constexpr (U == 3)
          some<TM + TN, IN, t>([&](auto r) __attribute__((always_inline)) { read_scale((k >> 2) + 1, decltype(r)::value); });
        if constexpr (AHEAD && s == SLOTS - 1) ask(k + AHEAD);
      }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (s == HALF - 1) {
        asm volatile("" ::: "memory");
        // all LDS reads; all loads but the later steps' and ask()'s last two
        __builtin_amdgcn_s_waitcnt(wait_loads((STAGES - 2) * (PA + PB) + (AHEAD > 0 ? 2 : 0)));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    if constexpr (U == 3) {
#pragma unroll
      for (int i = 0; i < TM; ++i) sa[i] = sa_next[i];
#pragma unroll
      for (int j = 0; j < TN; ++j) sb[j] = sb_next[j];
    }
  };

  // k0 is a multiple of 4
  each<STAGES>([&](auto stage) __attribute__((always_inline)) {
    constexpr int k = decltype(stage)::value;
    if constexpr (k == 0) issue_scales(k0 >> 2);
#pragma unroll
    for (int i = 0; i < PA + PB; ++i) issue(k0 + k, i, buffer(stage));
  });
#pragma unroll
  for (int k = STAGES; k < AHEAD; ++k) ask(k0 + k);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(wait_loads((STAGES - 1) * (PA + PB) + (AHEAD > 0 ? 2 * (AHEAD - STAGES) : 0)));
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    first[h] = half(buffer(Constant<0>{}), row_a, h);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j][h] = half(buffer(Constant<0>{}), row_b + 16 * j, h);
  }
#pragma unroll
  for (int i = 0; i < TM + TN; ++i) read_scale(k0 >> 2, i);
#pragma unroll
  for (int i = 0; i < TM; ++i) sa[i] = sa_next[i];
#pragma unroll
  for (int j = 0; j < TN; ++j) sb[j] = sb_next[j];

  int k = k0;
  for (; k + 4 <= k1; k += 4)
    each<4>([&](auto u) __attribute__((always_inline)) { step(k + decltype(u)::value, u); });
  each<3>([&](auto u) __attribute__((always_inline)) {
    if (k + decltype(u)::value < k1) step(k + decltype(u)::value, u);
  });
  __builtin_amdgcn_s_waitcnt(0);  // loads into this block's LDS end before it does
  settle(acc);
  __syncthreads();  // every wave has done with LDS

  // A lane holds four neighbours of a row in each tile.  Whole tiles in bf16 go out
  // two at a time, lanes 16 apart exchanging halves: 16 bytes a lane, 64 of a row
  // at a time, half the stores.
  const int64_t nw = n0 + wn * TN * 16;
  if (m0 + BM <= g.M && n0 + BN <= g.N && !g.parts && g.bf16 && !g.accumulate) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      uint16_t* p = static_cast<uint16_t*>(g.c) + (m0 + row_a + 16 * i + r16) * g.ldc + nw + (q & 1 ? 16 + 4 * (q - 1) : 4 * q);
#pragma unroll
      for (int j = 0; j < TN; j += 2) {
        uint32_t w[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const v4f& c = acc[i][j + h];
          w[h][0] = bf16_pair(c[0], c[1]);
          w[h][1] = bf16_pair(c[2], c[3]);
        }
        const auto x = __builtin_amdgcn_permlane16_swap(w[0][0], w[1][0], false, false);
        const auto y = __builtin_amdgcn_permlane16_swap(w[0][1], w[1][1], false, false);
        *reinterpret_cast<u32x4_any*>(p + 16 * j) = u32x4_any{x[0], y[0], x[1], y[1]};
      }
    }
    return;
  }
  // Everything else goes through LDS, 16 rows of the wave's tiles at a time.
  constexpr int LD = TN * 16 + 4, PER_ROW = TN * 2;  // floats of a row there, groups of eight
  static_assert(WAVES * 16 * LD * 4 <= STAGE, "");
  float* rows = reinterpret_cast<float*>(codes0) + wave * 16 * LD;
  each<TM>([&](auto tile) __attribute__((always_inline)) {
    constexpr int i = decltype(tile)::value;
#pragma unroll
    for (int j = 0; j < TN; ++j) *reinterpret_cast<v4f*>(&rows[r16 * LD + 16 * j + 4 * q]) = acc[i][j];
    wave_sync();
#pragma unroll 1
    for (int e = lane; e < 16 * PER_ROW; e += 64) {
      const int64_t m = m0 + row_a + 16 * i + e / PER_ROW;
      const int n = e % PER_ROW * 8;
      const float* v = &rows[e / PER_ROW * LD + n];
      if (m < g.M) {
        store4(g, m, nw + n, *reinterpret_cast<const v4f*>(v), split);
        store4(g, m, nw + n + 4, *reinterpret_cast<const v4f*>(v + 4), split);
      }
    }
    wave_sync();
  });
#endif
}

// Sums of the splits' parts, in order.
__global__ __launch_bounds__(256) void gemm_fp8_join_kernel(Gemm g, int splits) {
  const int64_t groups = (g.N + 3) / 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < g.M * groups; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / groups, n = i % groups * 4;
    const int count = (int)min((int64_t)4, g.N - n);
    v4f v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
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

// A block's time is taken as a fixed part and a part a step, fitted so that the
// differences between variants come out: what all of them share is left out.  A call
// takes some 4 us more (128 x 128: 500^3 3.9 by the estimate and 7.5 measured, 1500^3
// 7.4 and 11.4).  `room` blocks run at once; with two a CU each has half of it, so
// up to 256 blocks a step takes `alone`.
struct Variant {
  int bm, bn, threads, room;
  float alone, step, fixed;  // us
  void (*kernel)(Gemm);
};

// us on the GPU with C in bf16, every variant at some sizes (plan_of takes the least but for a few %):
//   M, N, K            256x256  256x128  128x128  128x128x2  64x128  64x64x2  64x32x3
//   1, 4096, 4096         37.9     26.4     14.3       20.9    10.6      9.0      8.1
//   77, 4096, 4096        41.4     28.8     16.5       23.3    11.2      9.1      8.4
//   500, 500, 500         16.8     10.6      7.5        7.3     5.1      4.2      4.1
//   256, 4096, 4096       39.6     26.6     15.4       21.8    11.5      9.4
//   512, 4096, 4096       39.7     26.6     15.7       22.1    13.1     15.0
//   1024, 4096, 4096      40.5     27.2     18.7       23.8    23.2     26.9
//   1400, 4096, 4096      44.6     31.5     32.4       28.9    33.8     37.8
//   2048, 4096, 4096      41.9     31.9     34.7       32.3    44.5     50.7
//   4096, 4096, 4096      53.6     61.2     66.7       61.8    87.6     99.0
//   4096, 11008, 4096    146.7    183.3    203.4      191.2   263.4    277.0
//   4096, 4096, 512       16.3     16.8     20.4       16.6    27.4     27.5
//   1500, 1500, 1500      26.0     19.0     11.4       13.2    12.9     11.0
// A smaller tile moves more bytes a product into LDS (some 43 a clock arrive on a CU,
// whatever the number of stages) and reads LDS more often; a larger one leaves CUs
// without work.
const Variant kVariants[] = {
    {256, 256, 256, 256, 1.3f, 1.3f, 8.0f, gemm_fp8_kernel<256, 256, 2, 2, 2, 1, 3>},
    {256, 128, 256, 256, 0.8f, 0.8f, 4.5f, gemm_fp8_kernel<256, 128, 2, 2, 2, 1, 3>},
    {128, 128, 256, 256, 0.43f, 0.43f, 2.2f, gemm_fp8_kernel<128, 128, 2, 2, 4, 1, 0>},
    {128, 128, 256, 512, 0.55f, 0.85f, 2.5f, gemm_fp8_kernel<128, 128, 2, 2, 2, 2, 0>},
    {64, 128, 256, 256, 0.28f, 0.28f, 1.4f, gemm_fp8_kernel<64, 128, 2, 2, 4, 1, 0>},
    {64, 64, 256, 512, 0.17f, 0.34f, 0.9f, gemm_fp8_kernel<64, 64, 2, 2, 4, 2, 0>},
    {64, 32, 128, 768, 0.14f, 0.32f, 1.2f, gemm_fp8_kernel<64, 32, 2, 1, 4, 3, 0>},
};

struct Plan {
  const Variant* v;
  int64_t tiles_m, tiles_n;
  int splits, steps_per_split;
};

// The variant, and how many parts K is cut into, with the least expected time: the
// rounds of blocks, and for a split K the second launch (4 us of a call), a chain of
// loads and the parts' way to memory and back (8 bytes each at 2.5 TB/s).  16 x 16
// over 16384: 25.1 us in one part, 10.7 in four, 8.7 in eight, 9.6 in sixteen; 300 x
// 300 over 16384: 26.2, 13.5, 13.4, 16.9.
Plan plan_of(int64_t M, int64_t N, int64_t K) {
  const int steps = (int)((K + 127) / 128), quads = (steps + 3) / 4;
  Plan best{};
  double least = 0;
  for (const Variant& v : kVariants) {
    Plan p{&v, (M + v.bm - 1) / v.bm, (N + v.bn - 1) / v.bn, 1, 0};
    for (int want = 1; want <= 32 && want <= quads; want *= 2) {
      p.steps_per_split = (quads + want - 1) / want * 4;
      p.splits = (steps + p.steps_per_split - 1) / p.steps_per_split;
      const int64_t blocks = p.tiles_m * p.tiles_n * p.splits, rounds = blocks / v.room, rest = blocks % v.room;
      const int run = std::min(p.steps_per_split, steps);
      double us = (double)rounds * (run * v.step + v.fixed);
      if (rest > 0) us += run * (rest > 256 ? v.step : v.alone) + v.fixed;
      if (p.splits > 1) us += 4.0 + p.splits * (0.35 + (double)M * (double)N * 8e-6 / 2.5);
      if (!best.v || us < least) {
        best = p;
        least = us;
      }
    }
  }
  return best;
}

size_t parts_bytes(const Plan& p, int64_t M, int64_t N) {
  return p.splits > 1 ? sizeof(float) * (size_t)p.splits * (size_t)M * (size_t)N : 0;
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
  return parts_bytes(plan_of(M, N, K), M, N);
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
  const size_t need = parts_bytes(p, M, N);
  if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 3)))
    return FAIRY2I_ERR_WORKSPACE;
  const int64_t tiles = p.tiles_m * p.tiles_n;
  if (tiles * p.splits >= ((int64_t)1 << 24)) return FAIRY2I_ERR_UNSUPPORTED;  // a launch takes fewer than 2^32 threads
  for (const fairy2i_fp8_matrix* m : {A, B})  // blocks read operands while others store C
    if (fp8_overlap(m, C, M, N, ldc, dtype == FAIRY2I_ACT_F32 ? 4 : 2)) return FAIRY2I_ERR_UNSUPPORTED;
  const Gemm g{A->codes,
               A->scales,
               B->codes,
               B->scales,
               M,
               N,
               fp8_ld(K),
               (int)(fp8_ld(K) / 128),
               p.steps_per_split,
               (int)p.tiles_m,
               (int)p.tiles_n,
               C,
               ldc,
               dtype == FAIRY2I_ACT_BF16,
               accumulate,
               need > 0 ? static_cast<float*>(workspace) : nullptr};
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(p.v->kernel, dim3((unsigned)tiles, (unsigned)p.splits), dim3(p.v->threads), 0, s, g);
  if (p.splits > 1) {
    const int64_t groups = M * ((N + 3) / 4);
    const unsigned blocks = (unsigned)std::min<int64_t>((groups + 255) / 256, 4096);
    hipLaunchKernelGGL(gemm_fp8_join_kernel, dim3(blocks), dim3(256), 0, s, g, p.splits);
  }
  return hipGetLastError() == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

}  // extern "C"
