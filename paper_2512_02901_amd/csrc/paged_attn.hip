// Hermitian-score attention over the paged 4-bit cache (fairy2i_kv_attend).
//
// Per key head the G query heads that share it and the sequence's new tokens
// are rows (row = token * G + query head).  With one complex entry as two
// reals, s = scale * Re(q^H k) is a real product, so everything is matrix
// work: S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_16x16x32_bf16, one block
// of 32 reals (one scale) a product.  The 4-bit values become bf16 exactly
// (a power of two times two bits) on their way into the operands, one
// conversion for two values; the cache's layout is the operands' own, so a
// lane's codes are its own 16-byte loads and S^T's accumulators are P^T's
// operand as they stand.
//
// One pass with a running maximum and sum; positions are split over blocks
// (chunks) and over a block's waves, joined through LDS and, where a row has
// several chunks, by a second kernel.
//
// What bounds it, with us of a whole call:
//  - a few tokens a sequence: memory.  One token over 262144 positions, 32 heads
//    on 8 of dc = 64 (285 MB), 60 us, its first kernel 53 (5.4 TB/s, a copy's
//    rate); 63 sequences of up to 8192 (302 MB) 67, 62 (4.8 TB/s: blocks start with
//    a chain of lookups, about 6 us under load, that their own loads wait for);
//  - short contexts: that chain and the join's; one token over 40 positions 4.4,
//    over 2048 (32 heads) 9.2, of which the join 3.0;
//  - prompts: the vector work of softmax and weights, issued beside the matrix
//    products of other waves only.  2048 tokens, 32 heads of dc = 64, 73 us (0.47
//    PFLOP/s of 4 products of 2 flops an entry, 0.7 as executed, the weights' two
//    parts counted); 811 tokens behind 15872, 16 on 4 of dc = 32, 86 us (0.42).
#include <float.h>
#include <math.h>

#include <type_traits>

#include "paged_kv.h"

namespace fairy2i {

namespace {

constexpr int kRows = 16;         // that a matrix product takes
constexpr int kCus = 256;
constexpr int kWaves = 4, kThreads = 64 * kWaves;
// Blocks of 16 rows in a row tile: one, or, past kWideRows rows a sequence in
// the mean, as many as share a conversion of the cache: two of a wave up to
// dc = 32, one of each of eight waves at dc = 48 and 64, and one again above
// (dc = 128, 1024 tokens behind 1024, 16 heads on 4: 16 rows 66 us, 32 111).
// us, one block | shared: dc = 64, 32 heads on 32, a prompt of 2048 107 | 74;
// 32 on 8, 2048 behind 2048 220 | 152, 8 prompts of up to 700 80 | 49; dc = 32,
// 16 on 4, 509 behind 15872 and 302 behind 2065 111 | 97 (by eight waves 106);
// dc = 16, 8 on 1, 2 x 512 behind 7680 50 | 46 (78).
constexpr int wide_rb(int nb) { return nb <= 2 ? 2 : 1; }
constexpr int kSharedWaves = 8;
constexpr bool shared(int nb) { return nb == 3 || nb == 4; }
constexpr int wide_blocks(int nb) { return shared(nb) ? kSharedWaves : wide_rb(nb); }
// Small blocks leave fewer rows idle and fill more of the machine.  64
// sequences of up to 2000 positions, rows each, us, one block | shared: dc = 64,
// 32 heads on 8: 32 rows 44 | 70, 64 56 | 73, 128 75 | 80, 256 140 | 120;
// dc = 32, 16 on 4: 32 23 | 25, 128 40 | 42, 256 53 | 56.  One sequence, 16381
// positions: dc = 64 32 18.6 | 21.5, 128 32.2 | 32.7, 256 52 | 46.
constexpr int kWideRows = 128;
// Blocks that are resident at once, which a call is cut into where its rows
// alone are fewer: by the kernels' registers.  us for 512 | 768 | 1024 items:
// 32 heads on 8, dc = 64 (768 resident), one token over 262144 positions 63 | 61 |
// 65, 31 over up to 16384 80 | 78 | 80, 16 over 8192 33.7 | 32.7 | 35; 16 on 16,
// dc = 32 (1024), 31 over up to 16384 97 | 84 | 82; 16 on 4, dc = 128 (512), 7 over
// up to 16384 25.3 | 30.4 (256: 26.4), 64 over 4096 57 | 62 (65).
constexpr int resident(int nb, bool wide) { return kCus * (wide ? (nb <= 2 ? 3 : 2) : nb <= 2 ? 4 : nb <= 4 ? 3 : 2); }
constexpr int kMaxItems = 4 * kCus;
// Tiles of a chunk at least, by row blocks of a tile: shorter ones cost a join and
// lookups for little work.  us for 4 | 8 | 16 | 32 tiles: one block, one token over
// 2048, 32 heads on 32 (dc = 64) 9.7 | 9.1 | 10.4, 6 x up to 5 over up to 4099, 8 on
// 2 (dc = 128) 17.6 | 15.2 | 16.4; two, a prompt of 600, 16 on 4 (dc = 32) 8: 13.7 |
// 12.5 | 10.4, 128 tokens over 800 10.6 | 11.9 | 11.3; eight, 3 prompts of up to 400,
// 32 on 8 (dc = 64) 26.6 | 18.7 | 18.6, 256 over 1500 29 | 26 | 37.6, a prompt of
// 600 21.7 | 24.8 | 22.1.
constexpr int min_chunk(int rb) { return rb == 1 ? 8 : rb == kSharedWaves ? 16 : 32; }
constexpr int kMostTiles = 1 << 25;  // 2^30 positions
constexpr int kClasses = 9;

// The running reference of a row's weights is raised once a score is 2^8 past
// it: raising it at every new maximum scales 64 sums a lane in nearly every
// tile of a prompt, and weights of up to 2^8 lose nothing in float32 or bf16.
constexpr float kRaise = 8.0f;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
  KvCache c;
  KvBatch b;
  const u32_any* q;   // [n_new][heads][dc] bf16 pairs
  u32_any* out;       // the same
  int32_t heads, group;
  float scale;        // log2(e) times the score scale
  float* part;        // [items][rows of a tile][D] unnormalised sums
  float2* ml;         // [items][rows of a tile] running maximum and sum
  int2* meta;         // [slots][kv_heads]: first of a row block's records, chunks
  int32_t items, tile_rows;
};

// Row blocks of a sequence: sequence i's start at slot row0 * G / 16 + i (its
// ceil(n G / 16) blocks end before the next one's start).
__device__ inline int row_slot(const AttnArgs& a, int i) {
  return (int)((int64_t)kv_row(a.b, i) * a.group / kRows) + i;
}
int64_t row_slots(int64_t n_new, int64_t n_seqs, int group) { return n_new * group / kRows + n_seqs; }

__device__ inline int row_blocks(const AttnArgs& a, const KvSeq& s) { return (int)(((int64_t)s.n * a.group + kRows - 1) / kRows); }
// Tiles of `RB` blocks; a sequence with one block has a tile of one.
template <int RB>
__device__ inline int row_tiles(const AttnArgs& a, const KvSeq& s) { return (row_blocks(a, s) + RB - 1) / RB; }
__device__ inline int kv_tiles(int len) { return (len + kKvTile - 1) / kKvTile; }

// Sum over the lanes below and this one, without a trip through LDS.
template <typename T>
__device__ inline T up_to(T v) {
  auto add = [&](auto shift) {
    constexpr int ctrl = decltype(shift)::value, rows = ctrl == 0x142 ? 0xA : ctrl == 0x143 ? 0xC : 0xF;
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xF, false);
    if constexpr (sizeof(T) == 8) {
      const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), ctrl, rows, 0xF, false);
      v += (uint64_t)hi << 32 | lo;
    } else {
      v += lo;
    }
  };
  add(std::integral_constant<int, 0x111>{});  // one lane up in rows of 16, two, four, eight
  add(std::integral_constant<int, 0x112>{});
  add(std::integral_constant<int, 0x114>{});
  add(std::integral_constant<int, 0x118>{});
  add(std::integral_constant<int, 0x142>{});  // row 0's last to row 1, 2's to 3
  add(std::integral_constant<int, 0x143>{});  // row 1's last to rows 2 and 3
  return v;
}

__device__ inline int of_lane(int v, int i) { return __builtin_amdgcn_readlane(v, i); }
__device__ inline uint32_t of_lane(uint32_t v, int i) { return __builtin_amdgcn_readlane((int)v, i); }
__device__ inline uint64_t of_lane(uint64_t v, int i) {
  const uint32_t lo = of_lane((uint32_t)v, i), hi = of_lane((uint32_t)(v >> 32), i);
  return (uint64_t)hi << 32 | lo;
}

struct Item {
  int seq, tile, head, chunk;  // row tile and chunk of the sequence, key head
  int chunk_tiles;
  int id;  // where its sums go, if the chunk is one of several
  KvSeq s;
};

// One or two blocks of eight waves a CU, the longest first: the second ones in
// the other order, so that a CU's two are as long together as any other's.
template <int RB>
__device__ inline uint32_t in_turn(uint32_t at, uint32_t items) {
  return RB == kSharedWaves && items > kCus && items <= 2 * kCus && at >= kCus && at < items ? items - 1 - (at - kCus) : at;
}

// Chunks are as long as makes `target` of them over all sequences, and
// min_chunk tiles at least.  Whole chunks go first, then what is left of the
// sequences in kClasses - 1 classes of its length, the longest first, so that the
// short ones fill the gaps; of a sequence's, the last row tiles (which see most)
// go first and heads are neighbours.  (In the sequences' own order 31 tokens over
// up to 16384 positions, 32 heads on 8, dc = 64, took 92 us for 77, 63 over up to
// 8192 77 for 67.)  `hist`: kClasses words of LDS for the wave.
// A cu_new that decreases somewhere can name more rows than there are: counts may
// then wrap, and an item is taken only if everything in it is in range.
template <int RB>
__device__ inline bool find_item(const AttnArgs& a, uint32_t at, int target, uint32_t* hist, Item& it) {
  const int lane = threadIdx.x & 63, n = a.b.n_seqs, kv = a.c.kv_heads;
  if (n > 1 && lane < kClasses) hist[lane] = 0;
  auto seq = [&](int i) { return i < n ? kv_seq(a.b, a.c, i) : KvSeq{0, 0, 0, 0}; };
  const KvSeq first = seq(lane);
  uint64_t work = (uint64_t)kv_tiles(first.len) * row_tiles<RB>(a, first);
  for (int i = 64 + lane; i < n; i += 64) {
    const KvSeq s = seq(i);
    work += (uint64_t)kv_tiles(s.len) * row_tiles<RB>(a, s);
  }
  // of one sequence, its lane's number; of more, the last lane's sum
  auto total = [&](auto v) { return n > 1 ? of_lane(up_to(v), 63) : of_lane(v, 0); };
  work = total(work);
  const int ct = (int)max((uint64_t)min_chunk(RB), min((work * kv + target - 1) / target, (uint64_t)kMostTiles));
  const float classes = (kClasses - 1.0f) / ct;
  struct Share {
    int row_tiles, chunks, kind;  // row tiles, whole chunks of each, the class of what is left
    uint32_t whole, rest;         // items of whole chunks and others
  };
  auto share_of = [&](const KvSeq& s) {
    const int t = kv_tiles(s.len), chunks = t / ct, left = t - chunks * ct, rt = row_tiles<RB>(a, s);
    const uint32_t items = (uint32_t)rt * kv;
    return Share{rt, chunks, kClasses - 1 - min((int)(left * classes), kClasses - 2), chunks * items,
                 left > 0 || chunks == 0 ? items : 0};
  };
  const Share mine = share_of(first);
  int kind;        // the item's class, 0 for whole chunks
  uint32_t start;  // items of the classes before
  if (n > 1) {
    uint32_t whole = mine.whole;
    auto add = [&](const Share& x) {
      if (x.rest) __hip_atomic_fetch_add(hist + x.kind, x.rest, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    };
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    add(mine);
    for (int i = 64 + lane; i < n; i += 64) {
      const Share x = share_of(seq(i));
      whole += x.whole;
      add(x);
    }
    whole = total(whole);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const uint32_t here = lane == 0 ? whole : lane < kClasses ? hist[lane] : 0, upto = up_to(here);
    at = in_turn<RB>(at, of_lane(upto, 63));
    const uint64_t past = __ballot(upto > at);
    if (past == 0) return false;
    kind = __builtin_ctzll(past);
    start = of_lane(upto - here, kind);
  } else {
    start = of_lane(mine.whole, 0);
    at = in_turn<RB>(at, start + of_lane(mine.rest, 0));
    kind = at < start ? 0 : of_lane(mine.kind, 0);
    if (kind == 0) start = 0;
  }
  at -= start;
  uint32_t before = 0, ids = 0;  // items of the sequences before: of this class, and all
  for (int i0 = 0; i0 < n; i0 += 64) {
    const KvSeq s = i0 == 0 ? first : seq(i0 + lane);
    const Share x = i0 == 0 ? mine : share_of(s);
    const uint32_t all = x.whole + x.rest, here = kind == 0 ? x.whole : x.kind == kind ? x.rest : 0;
    const uint32_t upto = n > 1 ? up_to(here) : here, ids_upto = n > 1 ? up_to(all) : all;
    const uint64_t past = __ballot(before + upto > at);
    if (past != 0) {
      const int w = __builtin_ctzll(past);
      auto of = [&](auto v) { return of_lane(v, w); };
      const int local = (int)(at - before - of(upto - here)), rt = of(x.row_tiles), chunks = of(x.chunks);
      const int per = kind == 0 ? chunks : 1;  // chunks of this class that a row tile has
      const int hc = local / kv, t = hc / max(per, 1);
      it.seq = i0 + w;
      it.s = {of(s.row0), of(s.n), of(s.p0), of(s.len)};
      it.head = local - hc * kv;
      it.chunk = kind == 0 ? hc - t * per : chunks;
      it.tile = rt - 1 - t;
      it.chunk_tiles = ct;
      const uint32_t id = ids + of(ids_upto - all) + ((uint32_t)t * (chunks + (of(x.rest) != 0)) + it.chunk) * kv + it.head;
      it.id = (int)id;
      return local >= 0 && it.tile >= 0 && id < (uint32_t)a.items;  // not so only for a cu_new that decreases
    }
    before += of_lane(upto, 63);
    ids += of_lane(ids_upto, 63);
  }
  return false;
}

// Codes and scales of a tile (PARTS = 1) or of about half of its blocks, part
// PART of two, of one lane.
template <int NB, int PARTS>
struct TileRegs {
  static constexpr KvTile T{NB};
  static constexpr int kUnits = 2 * NB / T.unit, kBlocks = T.unit / 2;  // loads of each array, blocks a load
  static constexpr int kMax = (kUnits + PARTS - 1) / PARTS;
  uint32_t k[kMax * T.unit], v[kMax * T.unit];
  uint32_t ks[2][(T.sb + 3) / 4], vs[2 * T.sb];

  static constexpr int first(int part) { return part * (kUnits / PARTS); }
  static constexpr int last(int part) { return part + 1 == PARTS ? kUnits : first(part + 1); }

  template <int PART>
  __device__ inline void load(const uint8_t* tile) {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int u = first(PART); u < last(PART); ++u) {
      load_n<T.unit>(k + (u - first(PART)) * T.unit, tile + T.dword(u * T.unit, lane));
      load_n<T.unit>(v + (u - first(PART)) * T.unit, tile + T.v_codes() + T.dword(u * T.unit, lane));
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint8_t* at = tile + T.k_scales() + (16 * s + r) * T.sb;
      if constexpr (T.sb == 1) ks[s][0] = *at;
      else if constexpr (T.sb == 2) ks[s][0] = *reinterpret_cast<const uint16_t*>(at);
      else load_n<T.sb / 4>(ks[s], at);
    }
    load_n<2 * T.sb>(vs, tile + T.v_scales() + g * 8 * T.sb);
  }

  template <int N>
  __device__ static inline void load_n(uint32_t* to, const uint8_t* at) {
    if constexpr (N >= 4) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        const uint4 x = reinterpret_cast<const uint4*>(at)[i];
        to[4 * i] = x.x;
        to[4 * i + 1] = x.y;
        to[4 * i + 2] = x.z;
        to[4 * i + 3] = x.w;
      }
    } else if constexpr (N == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(at);
      to[0] = x.x;
      to[1] = x.y;
    } else {
      to[0] = *reinterpret_cast<const uint32_t*>(at);
    }
  }

  // Byte `i` of `words` as the scale operand: only its exponent field counts.
  __device__ static inline float scale_at(const uint32_t* words, int i) {
    const uint32_t w = words[i / 4];
    const int b = i % 4;
    return __uint_as_float(b == 3 ? w >> 1 : w << (23 - 8 * b));
  }

  // Keys of half `s` (16 positions), block b: the A operand of S^T.
  template <int PART>
  __device__ inline bf16x8 key(int b, int s) const {
    const float scale = scale_at(ks[s], b);
    const uint32_t w = k[2 * (b - first(PART) * kBlocks) + s];
    u32x4 o;
    o[0] = pair<0>(w, scale);
    o[1] = pair<1>(w, scale);
    o[2] = pair<2>(w, scale);
    o[3] = pair<3>(w, scale);
    return __builtin_bit_cast(bf16x8, o);
  }

  // Values of block b: the A operands of O^T, real and imaginary parts.
  template <int PART>
  __device__ inline void value(int b, bf16x8& re, bf16x8& im) const {
    uint32_t c[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t w = v[2 * (b - first(PART) * kBlocks) + h];
      c[4 * h + 0] = pair<0>(w, scale_at(vs, (4 * h + 0) * T.sb + b));
      c[4 * h + 1] = pair<1>(w, scale_at(vs, (4 * h + 1) * T.sb + b));
      c[4 * h + 2] = pair<2>(w, scale_at(vs, (4 * h + 2) * T.sb + b));
      c[4 * h + 3] = pair<3>(w, scale_at(vs, (4 * h + 3) * T.sb + b));
    }
    u32x4 lo, hi;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lo[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100);
      hi[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302);
    }
    re = __builtin_bit_cast(bf16x8, lo);
    im = __builtin_bit_cast(bf16x8, hi);
  }

  template <int B>
  __device__ static inline uint32_t pair(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
  }

  // For a tile with positions that some row does not see: nobody may have written
  // them, past the length or past the rotation table, and under a weight of zero
  // what stands there has to be finite.  Scale bytes of the values above 252, the
  // largest that is ever stored, become 252.
  __device__ inline void make_finite() {
#pragma unroll
    for (uint32_t& w : vs) {
      const uint32_t two = w & w << 1;                                      // bits 7, 5, 3: that and the one below
      const uint32_t above = two & two << 2 & two << 4 & 0x80808080u;       // bits 7 to 2 all set
      w &= ~(above >> 6 | above >> 7);
    }
  }
};

// max over the four lanes that share a row
__device__ inline float row_max(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const uint32_t x = __float_as_uint(v);
  const auto c = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return fmaxf(__uint_as_float(c[0]), __uint_as_float(c[1]));
}

__device__ inline float row_sum(float v) {
  const uint32_t u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t x = __float_as_uint(v);
  const auto c = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return __uint_as_float(c[0]) + __uint_as_float(c[1]);
}

__device__ inline uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 p;
  p[0] = (__bf16)lo;
  p[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, p);
}

__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// Sums of the waves that hand theirs over: all for one row block, else two.
template <int NB, int RB>
constexpr int kLds = (RB > 1 ? 2 : kWaves) * 16 * RB * ((32 * NB + 4) * 4 + 8);

// Four tiles' operands and whether the table has them.
template <int NB>
constexpr int kSharedLds = kSharedWaves / 2 * (4096 * NB + 4);

// The queries of rows row0 .. row0 + 15 of a tile: operand B of S^T.
template <int NB>
__device__ inline void load_q(const AttnArgs& a, const Item& it, int row0, bf16x8 (&q)[NB]) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int row = row0 + r, token = row / a.group, hq = it.head * a.group + (row - token * a.group);
  const u32x4_any* at = reinterpret_cast<const u32x4_any*>(a.q + ((int64_t)(it.s.row0 + token) * a.heads + hq) * (16 * NB)) + g;
  const bool real = row < it.s.n * a.group;
#pragma unroll
  for (int b = 0; b < NB; ++b) q[b] = __builtin_bit_cast(bf16x8, real ? u32x4(at[4 * b]) : u32x4{0, 0, 0, 0});
}

// Scores past what the lane's row sees, in tiles from position t0 on.
template <int H>
__device__ inline void mask(f32x4 (&s)[H], int t0, int last) {
  int from = t0 + 4 * ((threadIdx.x & 63) >> 4);
  asm volatile("" : "+v"(from));  // keeps the comparisons out of the tiles that need none
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (from + 16 * h + i > last) s[h][i] = -INFINITY;
}

// A row block's running softmax: the score that its weights are relative to, and
// the lane's share of their sum.  It starts below every finite score and takes
// no part until one is seen: masked ones are -infinity, and weigh nothing.
struct Softmax {
  float m = -FLT_MAX, l = 0.0f;
};

// Over the scores of H times 16 positions: raises the reference where they ask
// for it (scaling l and o), adds to l and leaves the weights in p.  The reference
// is subtracted before the scale: one fused multiply-add of its product would
// save an instruction, but its rounding passes 2^7 once scores pass 2^31.
template <int NB, int H>
__device__ inline void weigh(const f32x4 (&s)[H], float scale, Softmax& x, f32x4 (&o)[2 * NB], float (&p)[4 * H]) {
  float top = s[0][0];
#pragma unroll
  for (int i = 1; i < 4 * H; ++i) top = fmaxf(top, s[i / 4][i % 4]);
  if (__any(top > x.m + kRaise / scale)) {
    asm volatile("");
    top = fmaxf(x.m, row_max(top));  // the row's own, in all of its lanes
    const float f = exp2_of((x.m - top) * scale);
    x.m = top;
    x.l *= f;
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) o[i] *= f;
  }
#pragma unroll
  for (int i = 0; i < 4 * H; ++i) {
    p[i] = exp2_of((s[i / 4][i % 4] - x.m) * scale);
    x.l += p[i];
  }
}

// p as the sum of two bf16 numbers each (2^-16 relative).
__device__ inline void split_bf16(const float* p, bf16x8& ph, bf16x8& pl) {
  u32x4 hi, lo;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    hi[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
    asm("" : "+v"(hi[i]));  // one conversion, its halves taken apart
    lo[i] = pack_bf16(p[2 * i] - __uint_as_float(hi[i] << 16), p[2 * i + 1] - __uint_as_float(hi[i] & 0xFFFF0000u));
  }
  ph = __builtin_bit_cast(bf16x8, hi);
  pl = __builtin_bit_cast(bf16x8, lo);
}

// A tile of 16 RB rows, a chunk of positions over four waves: each streams tiles
// of its own.  A tile is converted once for its RB row blocks; the weights go
// in as two bf16 parts, since what rounding them to one would leave is of the
// size of the output's own rounding.
template <int NB, int RB>
__device__ inline void attend_tile(const AttnArgs& a, const Item& it, char* lds) {
  constexpr int D = 32 * NB, kStride = D + 4, kTileRows = kRows * RB;
  auto os = reinterpret_cast<float(*)[kTileRows][kStride]>(lds);
  auto mls = reinterpret_cast<float2(*)[kTileRows]>(lds + sizeof(float) * (RB > 1 ? 2 : kWaves) * kTileRows * kStride);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int r = lane & 15, g = lane >> 4;
  const int rows = it.s.n * a.group, row0 = it.tile * kTileRows;
  const int p0 = it.s.p0;  // position of the first new token
  // the least and the most that any row of the tile sees
  const int least = p0 + row0 / a.group;
  const int most = min(p0 + (min(row0 + kTileRows, rows) - 1) / a.group, it.s.len - 1);
  const int tiles = kv_tiles(most + 1), chunks = max(1, (tiles + it.chunk_tiles - 1) / it.chunk_tiles);
  if (it.chunk == 0 && threadIdx.x < RB && row0 + kRows * (int)threadIdx.x < rows)
    a.meta[(int64_t)(row_slot(a, it.seq) + it.tile * RB + threadIdx.x) * a.c.kv_heads + it.head] =
        make_int2(it.id * kTileRows + kRows * (int)threadIdx.x, chunks);
  if (it.chunk >= chunks) return;
  const int t_end = min(tiles, (it.chunk + 1) * it.chunk_tiles);
  int last[RB];  // what the lane's rows see; rows past the end compute what nobody stores
  bf16x8 q[RB][NB];
  f32x4 o[RB][2 * NB];
  Softmax sm[RB];
#pragma unroll
  for (int y = 0; y < RB; ++y) {
    last[y] = min(p0 + (row0 + kRows * y + r) / a.group, most);
    load_q<NB>(a, it, row0 + kRows * y, q[y]);
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) o[y][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // the wave's k-th tile: the pages of 64 at a time, one a lane
  const int t_first = it.chunk * it.chunk_tiles + wave;
  int ids = 0;
  auto tile_at = [&](int k) -> const uint8_t* {
    if (k % 64 == 0) {
      const int t = t_first + kWaves * (k + lane);
      ids = t < t_end ? kv_tile_index(a.c, a.b, it.seq, t, it.head) : -1;
    }
    const int id = __builtin_amdgcn_readlane(ids, k % 64);
    return id < 0 ? nullptr : a.c.data + (int64_t)id * KvTile(NB).bytes;
  };
  auto step = [&](int t, TileRegs<NB, 1>& x) {
    f32x4 s[RB][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int y = 0; y < RB; ++y) s[y][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const bf16x8 k = x.template key<0>(b, h);
#pragma unroll
        for (int y = 0; y < RB; ++y) s[y][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[y][b], s[y][h], 0, 0, 0);
      }
    }
    if constexpr (RB > 1) __builtin_amdgcn_sched_barrier(0);  // the values' conversions would take registers from here on
    const int t0 = t * kKvTile;
    const bool edge = t0 + kKvTile - 1 > least;
    if (edge) x.make_finite();
    bf16x8 ph[RB], pl[RB];
#pragma unroll
    for (int y = 0; y < RB; ++y) {
      if (edge) mask<2>(s[y], t0, last[y]);
      float p[8];
      weigh<NB, 2>(s[y], a.scale, sm[y], o[y], p);
      split_bf16(p, ph[y], pl[y]);
    }
    if constexpr (RB > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      bf16x8 re, im;
      x.template value<0>(b, re, im);
#pragma unroll
      for (int y = 0; y < RB; ++y) {
        o[y][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(re, ph[y], o[y][2 * b], 0, 0, 0);
        o[y][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(im, ph[y], o[y][2 * b + 1], 0, 0, 0);
      }
#pragma unroll
      for (int y = 0; y < RB; ++y) {
        o[y][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(re, pl[y], o[y][2 * b], 0, 0, 0);
        o[y][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(im, pl[y], o[y][2 * b + 1], 0, 0, 0);
      }
    }
  };
  {
    // two sets of registers, one loaded while the other is used
    TileRegs<NB, 1> xa, xb;
    int k = 0, t = t_first;
    const uint8_t* at = tile_at(0);
    if (at) xa.template load<0>(at);
    while (t < t_end) {
      const uint8_t* next = tile_at(k + 1);
      if (next) xb.template load<0>(next);
      if (at) step(t, xa);
      t += kWaves;
      if (t >= t_end) break;
      at = tile_at(k + 2);
      if (at) xa.template load<0>(at);
      if (next) step(t, xb);
      t += kWaves;
      k += 2;
    }
  }
  // Join the waves: one row block's through LDS by all threads, more by the
  // upper two waves handing over to the lower two, and those to one.
#pragma unroll
  for (int y = 0; y < RB; ++y) sm[y].l = row_sum(sm[y].l);
  auto put = [&](int w) {
#pragma unroll
    for (int y = 0; y < RB; ++y) {
      if (g == 0) mls[w][kRows * y + r] = make_float2(sm[y].m, sm[y].l);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; i += 2)  // entries 16 b + 4 g + i, + 1
          *reinterpret_cast<float4*>(&os[w][kRows * y + r][32 * b + 8 * g + 2 * i]) =
              make_float4(o[y][2 * b][i], o[y][2 * b + 1][i], o[y][2 * b][i + 1], o[y][2 * b + 1][i + 1]);
    }
  };
  if constexpr (RB > 1) {
    auto add = [&](int w) {
#pragma unroll
      for (int y = 0; y < RB; ++y) {
        const float2 ml = mls[w][kRows * y + r];
        const float top = fmaxf(sm[y].m, ml.x);
        const float f = exp2_of((sm[y].m - top) * a.scale), h = exp2_of((ml.x - top) * a.scale);
        sm[y].m = top;
        sm[y].l = f * sm[y].l + h * ml.y;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            const float4 v = *reinterpret_cast<const float4*>(&os[w][kRows * y + r][32 * b + 8 * g + 2 * i]);
            o[y][2 * b][i] = f * o[y][2 * b][i] + h * v.x;
            o[y][2 * b + 1][i] = f * o[y][2 * b + 1][i] + h * v.y;
            o[y][2 * b][i + 1] = f * o[y][2 * b][i + 1] + h * v.z;
            o[y][2 * b + 1][i + 1] = f * o[y][2 * b + 1][i + 1] + h * v.w;
          }
      }
    };
    if (wave >= 2) put(wave - 2);
    __syncthreads();
    if (wave < 2) add(wave);
    __syncthreads();
    if (wave == 1) put(0);
    __syncthreads();
    if (wave != 0) return;
    add(0);
#pragma unroll
    for (int y = 0; y < RB; ++y) {
      const int row = row0 + kRows * y + r, token = row / a.group, hq = it.head * a.group + (row - token * a.group);
      if (row >= rows) continue;
      if (chunks == 1) {
        const float inv = sm[y].l == 0.0f ? 0.0f : 1.0f / sm[y].l;
        u32x4_any* to = reinterpret_cast<u32x4_any*>(a.out + ((int64_t)(it.s.row0 + token) * a.heads + hq) * (16 * NB)) + g;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          u32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = pack_bf16(o[y][2 * b][i] * inv, o[y][2 * b + 1][i] * inv);
          to[4 * b] = v;
        }
      } else {
        const int64_t rec = (int64_t)it.id * kTileRows + (row - row0);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 4; i += 2)
            *reinterpret_cast<float4*>(a.part + rec * D + 32 * b + 8 * g + 2 * i) =
                make_float4(o[y][2 * b][i], o[y][2 * b + 1][i], o[y][2 * b][i + 1], o[y][2 * b + 1][i + 1]);
        if (g == 0) a.ml[rec] = make_float2(sm[y].m, sm[y].l);
      }
    }
  } else {
    put(wave);
    __syncthreads();
    for (int e = threadIdx.x; e < kRows * (D / 2); e += kThreads) {
      const int rr = e / (D / 2), c = e - rr * (D / 2), w = row0 + rr;
      if (w >= rows) continue;
      float top = mls[0][rr].x;
#pragma unroll
      for (int i = 1; i < kWaves; ++i) top = fmaxf(top, mls[i][rr].x);
      float sum = 0.0f;
      float2 y = make_float2(0.0f, 0.0f);
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        const float f = exp2_of((mls[i][rr].x - top) * a.scale);
        sum += f * mls[i][rr].y;
        const float2 v = *reinterpret_cast<const float2*>(&os[i][rr][2 * c]);
        y.x += f * v.x;
        y.y += f * v.y;
      }
      if (chunks == 1) {
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int tk = w / a.group, hh = it.head * a.group + (w - tk * a.group);
        a.out[((int64_t)(it.s.row0 + tk) * a.heads + hh) * (D / 2) + c] = pack_bf16(y.x * inv, y.y * inv);
      } else {
        const int64_t rec = (int64_t)it.id * kTileRows + rr;
        *reinterpret_cast<float2*>(a.part + rec * D + 2 * c) = y;
        if (c == 0) a.ml[rec] = make_float2(top, sum);
      }
    }
  }
}

// Many rows of heads whose conversions cost as much as their softmax (dc = 48,
// 64): a wave for each 16 of a tile's 128 rows, all walking the chunk's tiles
// together, four at a time from LDS.  Two waves convert a tile for all of them
// into the operands' order, its codes loaded a round before.  What counts is
// four waves a SIMD (128 registers): alone, a wave issues a vector instruction
// every seventh cycle or so, and none beside its own matrix products.  Operands
// are asked for four products ahead; left to the compiler, each is waited for
// right after it is asked for.
template <int NB>
__device__ inline void attend_shared(const AttnArgs& a, const Item& it, char* lds) {
  constexpr int D = 32 * NB, W = kSharedWaves, R = W / 2;
  using Regs = TileRegs<NB, 2>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int r = lane & 15, g = lane >> 4, mine = wave / 2;
  auto operand = [&](int tile, int i) {  // i: keys 2 b + s, values 2 NB + 2 b + (0 re, 1 im)
    return reinterpret_cast<bf16x8*>(lds + tile * 4096 * NB + i * 1024) + lane;
  };
  int* there = reinterpret_cast<int*>(lds + R * 4096 * NB);  // whether the table has the round's tiles
  const int rows = it.s.n * a.group, tile0 = it.tile * kRows * W, row0 = tile0 + wave * kRows;
  const int p0 = it.s.p0;  // position of the first new token
  const int tile_most = min(p0 + (min(tile0 + kRows * W, rows) - 1) / a.group, it.s.len - 1);
  const int tiles = kv_tiles(tile_most + 1), chunks = max(1, (tiles + it.chunk_tiles - 1) / it.chunk_tiles);
  if (it.chunk == 0 && threadIdx.x < W && tile0 + kRows * (int)threadIdx.x < rows)
    a.meta[(int64_t)(row_slot(a, it.seq) + it.tile * W + threadIdx.x) * a.c.kv_heads + it.head] =
        make_int2(it.id * a.tile_rows + kRows * (int)threadIdx.x, chunks);
  if (it.chunk >= chunks) return;
  const int t_end = min(tiles, (it.chunk + 1) * it.chunk_tiles);
  // the least and the most that any of the wave's rows sees, and the least of all
  const int least = p0 + row0 / a.group, tile_least = p0 + tile0 / a.group;
  const int most = row0 < rows ? min(p0 + (min(row0 + kRows, rows) - 1) / a.group, it.s.len - 1) : -1;
  const int last = min(p0 + (row0 + r) / a.group, most);  // rows past the end compute what nobody stores
  bf16x8 q[NB];
  load_q<NB>(a, it, row0, q);
  f32x4 o[2 * NB];
#pragma unroll
  for (int i = 0; i < 2 * NB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  Softmax sm;

  Regs x;
  const int t_first = it.chunk * it.chunk_tiles;
  int ids = 0;  // of 64 tiles, one a lane
  auto fetch = [&](int k) {  // the wave's part of tile k + mine: whether there is one
    if (k % 64 == 0) {
      const int t = t_first + k + lane;
      ids = t < t_end ? kv_tile_index(a.c, a.b, it.seq, t, it.head) : -1;
    }
    const int id = __builtin_amdgcn_readlane(ids, k % 64 + mine);
    if (id >= 0) {
      const uint8_t* at = a.c.data + (int64_t)id * KvTile(NB).bytes;
      if (wave % 2 == 0) x.template load<0>(at);
      else x.template load<1>(at);
    }
    return id >= 0;
  };
  auto convert = [&](auto part) {
    constexpr int P = decltype(part)::value;
#pragma unroll
    for (int b = Regs::first(P) * Regs::kBlocks; b < Regs::last(P) * Regs::kBlocks; ++b) {
      *operand(mine, 2 * b) = x.template key<P>(b, 0);
      *operand(mine, 2 * b + 1) = x.template key<P>(b, 1);
      bf16x8 re, im;
      x.template value<P>(b, re, im);
      *operand(mine, 2 * NB + 2 * b) = re;
      *operand(mine, 2 * NB + 2 * b + 1) = im;
    }
  };
  bool have = fetch(0);
  for (int k = 0; t_first + k < t_end; k += R) {
    __syncthreads();  // the last round's readers
    if (have) {
      const int t0 = (t_first + k + mine) * kKvTile;
      if (t0 + kKvTile - 1 > tile_least) x.make_finite();
      if (wave % 2 == 0) convert(std::integral_constant<int, 0>{});
      else convert(std::integral_constant<int, 1>{});
    }
    if (lane == 0 && wave % 2 == 0) there[mine] = have;
    have = fetch(k + R);
    __syncthreads();
#pragma unroll 1
    for (int u = 0; u < R; ++u) {
      const int t0 = (t_first + k + u) * kKvTile;
      if (t0 > most) break;
      if (!__builtin_amdgcn_readfirstlane(there[u])) continue;  // no such page: nothing to see there
      constexpr int N = 2 * NB, AHEAD = 4;
      bf16x8 buf[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) buf[i] = *operand(u, i);
      __builtin_amdgcn_sched_barrier(0);
      f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int i = 0; i < N; ++i) {
        s[i % 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(buf[i % AHEAD], q[i / 2], s[i % 2], 0, 0, 0);
        buf[i % AHEAD] = *operand(u, i + AHEAD);  // the last ones: the first values
        __builtin_amdgcn_sched_barrier(0);
      }
      if (t0 + kKvTile - 1 > least) mask<2>(s, t0, last);
      float p[8];
      weigh<NB, 2>(s, a.scale, sm, o, p);
      bf16x8 ph, pl;
      split_bf16(p, ph, pl);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(buf[(i + N) % AHEAD], ph, o[i], 0, 0, 0);
        o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(buf[(i + N) % AHEAD], pl, o[i], 0, 0, 0);
        if (i + AHEAD < N) buf[(i + N) % AHEAD] = *operand(u, N + i + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  const float sum = row_sum(sm.l);
  const int row = row0 + r, token = row / a.group, hq = it.head * a.group + (row - token * a.group);
  if (row >= rows) return;
  if (chunks == 1) {
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    u32x4_any* to = reinterpret_cast<u32x4_any*>(a.out + ((int64_t)(it.s.row0 + token) * a.heads + hq) * (16 * NB)) + g;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      u32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = pack_bf16(o[2 * b][i] * inv, o[2 * b + 1][i] * inv);
      to[4 * b] = v;
    }
  } else {
    const int64_t rec = (int64_t)it.id * a.tile_rows + (row - tile0);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        *reinterpret_cast<float4*>(a.part + rec * D + 32 * b + 8 * g + 2 * i) =
            make_float4(o[2 * b][i], o[2 * b + 1][i], o[2 * b][i + 1], o[2 * b + 1][i + 1]);
    if (g == 0) a.ml[rec] = make_float2(sm.m, sum);
  }
}

// The block's item, looked up by one wave for all; seq < 0: none.
template <int RB>
__device__ inline Item block_item(const AttnArgs& a, int target, char* lds) {
  Item it{};
  Item* found = reinterpret_cast<Item*>(lds);
  if (threadIdx.x < 64) {
    if (!find_item<RB>(a, blockIdx.x, target, reinterpret_cast<uint32_t*>(lds + sizeof(Item)), it)) it.seq = -1;
    if (threadIdx.x == 0) *found = it;
  }
  __syncthreads();
  it = *found;
  int* word = reinterpret_cast<int*>(&it);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(Item) / 4); ++i) word[i] = __builtin_amdgcn_readfirstlane(word[i]);
  __syncthreads();  // what else stands there comes after this
  return it;
}

template <int NB, int RB>
__global__ __launch_bounds__(kThreads, RB > 1 ? 2 : 1) void kv_attend_kernel(AttnArgs a) {
  __shared__ __align__(16) char lds[kLds<NB, RB>];
  static_assert(sizeof(Item) + 4 * kClasses <= kLds<NB, RB>);
  const Item it = block_item<RB>(a, resident(NB, RB > 1), lds);
  if (it.seq >= 0) attend_tile<NB, RB>(a, it, lds);
}

template <int NB>
__global__ __launch_bounds__(64 * kSharedWaves, 4) void kv_attend_shared_kernel(AttnArgs a) {
  __shared__ __align__(16) char lds[kSharedLds<NB>];
  const Item it = block_item<kSharedWaves>(a, resident(NB, true), lds);
  if (it.seq >= 0) attend_shared<NB>(a, it, lds);
}

constexpr int kJoinThreads = 256;

// Joins a row block's chunks.  What bounds it is a chain of loads (of the
// sequences, of the chunks' maxima and sums), so the first sums are asked for
// before their weights are known, eight a lane at a time.  Up to 8 chunks: a
// lane for four reals, so a wave has several rows (with a wave a row, 32 x up to
// 64 tokens over up to 4096 positions, dc = 64, took 141 us for 130, 2 x 512 over
// 8192, dc = 16, 46 for 39); up to 64: a wave a row; more: a block a row.
// blockIdx.y: which rows, of 16.
template <int NB>
__global__ __launch_bounds__(kJoinThreads) void kv_attend_join_kernel(AttnArgs a) {
  constexpr int D = 32 * NB, kQuads = D / 4, kLanes = kQuads <= 8 ? 8 : kQuads <= 16 ? 16 : kQuads <= 32 ? 32 : 64;
  constexpr int kAhead = 8, kWavesJ = kJoinThreads / 64;
  __shared__ float weight[kMaxItems + 1];
  __shared__ float4 ys[kJoinThreads];
  __shared__ float tops[kWavesJ], sums[kWavesJ];
  const int slot = blockIdx.x / a.c.kv_heads, head = blockIdx.x - slot * a.c.kv_heads;
  const int2 meta = a.meta[(int64_t)slot * a.c.kv_heads + head];
  const int i = kv_find(a.b.n_seqs, slot, [&](int s) { return row_slot(a, s); });
  if (i < 0) return;
  const int row0 = kv_row(a.b, i), rows = max(kv_row(a.b, i + 1) - row0, 0) * a.group;
  const int block = slot - row_slot(a, i);
  if (block < 0 || block * kRows >= rows) return;
  const int chunks = meta.y;
  if (chunks < 2) return;
  // a chunk is kv_heads items after the one before; nothing else can stand
  // there unless cu_new decreases somewhere and no item wrote it
  const int64_t stride = (int64_t)a.c.kv_heads * a.tile_rows, records = (int64_t)a.items * a.tile_rows;
  if (chunks > kMaxItems + 1 || meta.x < 0 || meta.x + (int64_t)(chunks - 1) * stride + kRows > records) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto store = [&](int w, int c, const float4& y, float sum) {
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const int tk = w / a.group, hh = head * a.group + (w - tk * a.group);
    *reinterpret_cast<u32x2_any*>(a.out + ((int64_t)(row0 + tk) * a.heads + hh) * (D / 2) + 2 * c) =
        u32x2_any{pack_bf16(y.x * inv, y.y * inv), pack_bf16(y.z * inv, y.w * inv)};
  };
  if (chunks <= kAhead) {
    constexpr int kPer = 64 / kLanes;
    const int c = lane % kLanes;
    for (int rr = (blockIdx.y * kWavesJ + wave) * kPer + lane / kLanes; rr < kRows; rr += gridDim.y * kWavesJ * kPer) {
      const int w = block * kRows + rr;
      if (w >= rows) break;
      float2 ml[kAhead];
      float4 v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int64_t rec = meta.x + k * stride + rr;
        ml[k] = k < chunks ? a.ml[rec] : make_float2(-FLT_MAX, 0.0f);
        v[k] = k < chunks && c < kQuads ? *reinterpret_cast<const float4*>(a.part + rec * D + 4 * c) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      float top = ml[0].x, sum = 0.0f;
#pragma unroll
      for (int k = 1; k < kAhead; ++k) top = fmaxf(top, ml[k].x);
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float f = exp2_of((ml[k].x - top) * a.scale);
        sum += f * ml[k].y;
        y.x += f * v[k].x;
        y.y += f * v[k].y;
        y.z += f * v[k].z;
        y.w += f * v[k].w;
      }
      if (c < kQuads) store(w, c, y, sum);
    }
    return;
  }
  // threads of a row: of a wave, or of the block
  const bool few = chunks <= 64;
  const int mine = few ? lane : tid, parts = (few ? 64 : kJoinThreads) / kLanes, part = mine / kLanes, c = mine % kLanes;
  const int step = gridDim.y * (few ? kWavesJ : 1);
  for (int rr = few ? blockIdx.y * kWavesJ + wave : blockIdx.y; rr < kRows; rr += step) {
    const int w = block * kRows + rr;
    if (w >= rows) break;
    auto record = [&](int k) { return meta.x + (int64_t)k * stride + rr; };
    float4 v[kAhead];
    auto ask = [&](int k0) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int k = k0 + j * parts;
        v[j] = k < chunks && c < kQuads ? *reinterpret_cast<const float4*>(a.part + record(k) * D + 4 * c)
                                        : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    };
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](int j, float f) {
      y.x += f * v[j].x;
      y.y += f * v[j].y;
      y.z += f * v[j].z;
      y.w += f * v[j].w;
    };
    float top = -FLT_MAX, sum = 0.0f;
    ask(part);
    if (few) {
      const float2 ml = lane < chunks ? a.ml[record(lane)] : make_float2(-FLT_MAX, 0.0f);
      top = ml.x;
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
      const float f = exp2_of((ml.x - top) * a.scale);
      sum = f * ml.y;
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
      for (int k0 = part; k0 - part < chunks; k0 += kAhead * parts) {
        if (k0 != part) ask(k0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int k = k0 + j * parts;
          const float g = __shfl(f, k & 63);
          add(j, k < chunks ? g : 0.0f);
        }
      }
#pragma unroll
      for (int off = kLanes; off < 64; off <<= 1) {
        y.x += __shfl_xor(y.x, off);
        y.y += __shfl_xor(y.y, off);
        y.z += __shfl_xor(y.z, off);
        y.w += __shfl_xor(y.w, off);
      }
    } else {
      for (int k = tid; k < chunks; k += kJoinThreads) {
        const float m = a.ml[record(k)].x;
        weight[k] = m;
        top = fmaxf(top, m);
      }
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
      if (lane == 0) tops[wave] = top;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kWavesJ; ++j) top = fmaxf(top, tops[j]);
      for (int k = tid; k < chunks; k += kJoinThreads) {
        const float f = exp2_of((weight[k] - top) * a.scale);
        weight[k] = f;
        sum += f * a.ml[record(k)].y;
      }
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
      if (lane == 0) sums[wave] = sum;
      __syncthreads();
      for (int k0 = part; k0 < chunks; k0 += kAhead * parts) {
        if (k0 != part) ask(k0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int k = k0 + j * parts;
          add(j, k < chunks ? weight[k] : 0.0f);
        }
      }
      ys[tid] = y;
      __syncthreads();
      if (part == 0) {
#pragma unroll
        for (int k = 1; k < kJoinThreads / kLanes; ++k) {
          const float4 u = ys[k * kLanes + c];
          y.x += u.x;
          y.y += u.y;
          y.z += u.z;
          y.w += u.w;
        }
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kWavesJ; ++j) sum += sums[j];
      }
      __syncthreads();  // the next row's writers
    }
    if (part == 0 && c < kQuads) store(w, c, y, sum);
  }
}

struct Layout {
  bool wide;
  int64_t items, slots, tile_rows;
  size_t part, ml, meta, bytes;
};

Layout layout_of(const fairy2i_kv_cache* c, int64_t n_new, int64_t n_seqs, int32_t n_heads) {
  Layout l{};
  const int64_t G = n_heads / c->n_kv_heads;
  l.wide = n_new * G > kWideRows * n_seqs && wide_blocks((int)c->dc / 16) > 1;
  l.tile_rows = l.wide ? kRows * wide_blocks(c->dc / 16) : kRows;
  // a row tile more than its rows fill for each sequence that has any, and a
  // chunk more than its work fills for each row tile
  l.items = resident((int)c->dc / 16, l.wide) + c->n_kv_heads * (n_new * G / l.tile_rows + (n_seqs < n_new ? n_seqs : n_new));
  l.slots = row_slots(n_new, n_seqs, (int)G);
  auto up = [](size_t b) { return (b + 255) / 256 * 256; };
  l.part = up((size_t)l.items * l.tile_rows * 2 * c->dc * sizeof(float));
  l.ml = up((size_t)l.items * l.tile_rows * sizeof(float2));
  l.meta = up((size_t)l.slots * c->n_kv_heads * sizeof(int2));
  l.bytes = l.part + l.ml + l.meta;
  return l;
}

template <int NB>
void launch(const AttnArgs& a, const Layout& l, bool one_chunk, hipStream_t s) {
  auto kernel = kv_attend_kernel<NB, 1>;
  int threads = kThreads;
  if constexpr (shared(NB)) {
    if (l.wide) {
      kernel = kv_attend_shared_kernel<NB>;
      threads = 64 * kSharedWaves;
    }
  } else if constexpr (wide_rb(NB) > 1) {
    if (l.wide) kernel = kv_attend_kernel<NB, wide_rb(NB)>;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)l.items), dim3(threads), 0, s, a);
  if (one_chunk) return;
  const int64_t blocks = l.slots * a.c.kv_heads;
  // Blocks a row block: more only where few rows leave the machine empty, each
  // costs its chain of lookups.  us of the whole call, 16 | 4 | 1: one token
  // behind 131071, 64 heads on 4 (dc = 64) 27 | 37; 16 sequences of 4096, 32 on 8
  // (dc = 64) 23.3 | 22.2; 2 x 512 tokens behind 7680, 8 on 1 (dc = 16) 4: 39, 1: 37.
  const unsigned split = blocks <= 32 ? kRows : blocks <= 512 ? 4 : 1;
  hipLaunchKernelGGL(kv_attend_join_kernel<NB>, dim3((unsigned)blocks, split), dim3(kJoinThreads), 0, s, a);
}

bool valid_heads(const fairy2i_kv_cache* c, int32_t n_heads) {
  return n_heads >= 1 && n_heads <= 65535 && n_heads % c->n_kv_heads == 0;
}

}  // namespace

}  // namespace fairy2i

using namespace fairy2i;

extern "C" {

size_t fairy2i_kv_attend_workspace_bytes(const fairy2i_kv_cache* cache, int64_t n_new, int64_t n_seqs,
                                         int32_t n_heads) {
  if (!cache || fairy2i_kv_cache_bytes(cache->n_pages, cache->page_size, cache->n_kv_heads, cache->dc) == 0 ||
      !valid_heads(cache, n_heads) || n_new < 1 || n_new > (1 << 26) || n_seqs < 1 || n_seqs > (1 << 20))
    return 0;
  return layout_of(cache, n_new, n_seqs, n_heads).bytes;
}

fairy2i_status fairy2i_kv_attend(const fairy2i_kv_cache* cache, const fairy2i_kv_batch* batch, const void* q,
                                 int32_t n_heads, float scale, void* out, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  if (const fairy2i_status s = kv_check(cache, batch)) return s;
  if (!q || !out) return FAIRY2I_ERR_NULL;
  if (!valid_heads(cache, n_heads) || !(scale >= 1e-30f) || !(scale <= 1e30f)) return FAIRY2I_ERR_SHAPE;
  const Layout l = layout_of(cache, batch->n_new, batch->n_seqs, n_heads);
  if (!workspace || workspace_bytes < l.bytes || (reinterpret_cast<uintptr_t>(workspace) & 15) != 0)
    return FAIRY2I_ERR_WORKSPACE;
  if (l.items > INT32_MAX / 512 || l.items * l.tile_rows > INT32_MAX || l.slots * cache->n_kv_heads > INT32_MAX / 512)
    return FAIRY2I_ERR_UNSUPPORTED;
  AttnArgs a{};
  a.c = kv_cache_of(cache);
  a.b = kv_batch_of(batch);
  a.q = static_cast<const u32_any*>(q);
  a.out = static_cast<u32_any*>(out);
  a.heads = n_heads;
  a.group = n_heads / cache->n_kv_heads;
  a.scale = scale * 1.44269504088896341f;
  a.items = (int32_t)l.items;
  a.tile_rows = (int32_t)l.tile_rows;
  char* ws = static_cast<char*>(workspace);
  a.part = reinterpret_cast<float*>(ws);
  a.ml = reinterpret_cast<float2*>(ws + l.part);
  a.meta = reinterpret_cast<int2*>(ws + l.part + l.ml);
  const bool one_chunk = (int64_t)batch->max_pages * cache->page_size <= min_chunk((int)l.tile_rows / kRows) * kKvTile;
  auto s = static_cast<hipStream_t>(stream);
  switch (cache->dc / 16) {
    case 1: launch<1>(a, l, one_chunk, s); break;
    case 2: launch<2>(a, l, one_chunk, s); break;
    case 3: launch<3>(a, l, one_chunk, s); break;
    case 4: launch<4>(a, l, one_chunk, s); break;
    case 5: launch<5>(a, l, one_chunk, s); break;
    case 6: launch<6>(a, l, one_chunk, s); break;
    case 7: launch<7>(a, l, one_chunk, s); break;
    default: launch<8>(a, l, one_chunk, s); break;
  }
  return hipGetLastError() == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

}  // extern "C"
