// The paged 4-bit cache: its layout, and which sequence a piece of work is of.
#pragma once

#include "common.h"

namespace fairy2i {

constexpr int kKvTile = 32;     // positions of a tile
constexpr int kKvMaxDc = 128;   // complex entries of a head

// Sizes of a tile for dc = 16 nb entries a head (fairy2i.h has the layout).
struct KvTile {
  int nb;     // blocks of 16 entries that share a scale
  int unit;   // dwords that a lane's codes come in: 4 (even nb) or 2
  int sb;     // bytes of a position's scales
  int bytes;  // codes of keys, codes of values, scales of keys, scales of values
  __host__ __device__ explicit constexpr KvTile(int nb_)
      : nb(nb_), unit(nb_ % 2 == 0 ? 4 : 2), sb(nb_ <= 2 ? nb_ : (nb_ + 3) / 4 * 4), bytes(1024 * nb_ + 64 * sb) {}
  __host__ __device__ constexpr int v_codes() const { return 512 * nb; }
  __host__ __device__ constexpr int k_scales() const { return 1024 * nb; }
  __host__ __device__ constexpr int v_scales() const { return 1024 * nb + 32 * sb; }
  // byte offset of dword w = 2 block + half of `lane`
  __host__ __device__ constexpr int dword(int w, int lane) const {
    return 4 * ((w / unit * 64 + lane) * unit + w % unit);
  }
};

// Tensors of bf16 pairs and of floats may begin at any element.  Accesses to them
// promise no more than that and are one instruction all the same.
typedef uint32_t u32_any __attribute__((aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));

struct KvCache {
  uint8_t* data;
  int64_t n_pages;
  int32_t page_size, kv_heads, dc;
};

// The sequences of a call.  What the arrays hold is the device's, so every
// number from them is bounded before it is used.
struct KvBatch {
  const int32_t* pages;   // [n_seqs][max_pages]
  const int32_t* cu_new;  // [n_seqs + 1]
  const int32_t* lens;    // [n_seqs]
  int32_t n_seqs, max_pages;
  int32_t n_new;          // rows of q, k, v
};

// Rows that q, k and v do not have (cu_new past n_new) and positions that the
// table does not have (lens past it) are left out; the others stay in place, so p0
// may lie outside [0, len).
struct KvSeq {
  int row0, n, p0, len;  // first row, rows, the first one's position, positions of the table up to the last one's
};

constexpr int kKvMaxNew = 1 << 26, kKvMaxLen = 1 << 30;  // rows of a call, positions of a table

#if defined(__HIPCC__)

__device__ inline int kv_row(const KvBatch& b, int i) { return min(max(b.cu_new[i], 0), b.n_new); }

__device__ inline KvSeq kv_seq(const KvBatch& b, const KvCache& c, int i) {
  KvSeq s;
  s.row0 = kv_row(b, i);
  const int end = b.cu_new[i + 1];  // a row there would stand at lens[i]
  s.n = max(min(max(end, 0), b.n_new) - s.row0, 0);
  // saturated and bounded to where all rows are outside as well
  const int p0 = __builtin_elementwise_add_sat(__builtin_elementwise_sub_sat(b.lens[i], end), s.row0);
  s.p0 = min(max(p0, -kKvMaxNew), kKvMaxLen);
  s.len = min(max(s.p0 + s.n, 0), b.max_pages * c.page_size);
  return s;
}

// The last i in [0, n_seqs) with start(i) <= at (start increasing), or -1;
// 64 guesses at a time, the same in every lane.
template <typename F>
__device__ inline int kv_find(int n_seqs, int at, F start) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = n_seqs;
  bool first = true;
  while (first || n > 1) {
    const int step = (n + 63) / 64, i = lo + lane * step;
    const int found = __popcll(__ballot(i < lo + n && start(i) <= at));
    if (found == 0) return -1;  // only at the first round
    const int hi = lo + n;
    lo += (found - 1) * step;
    n = min(step, hi - lo);
    first = false;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// Number of tile t (of a sequence's positions) of head h in the cache; -1 where
// the table names no page.
__device__ inline int kv_tile_index(const KvCache& c, const KvBatch& b, int i, int t, int h) {
  const int tiles = c.page_size / kKvTile, page = t / tiles;
  const int id = b.pages[(int64_t)i * b.max_pages + page];
  return (uint32_t)id < (uint64_t)c.n_pages ? (id * c.kv_heads + h) * tiles + (t - page * tiles) : -1;
}

// Tile of position p of sequence i and head h; null where the table names no page.
__device__ inline uint8_t* kv_tile(const KvCache& c, const KvBatch& b, int i, int p, int h, int bytes) {
  const int id = kv_tile_index(c, b, i, p / kKvTile, h);
  return id < 0 ? nullptr : c.data + (int64_t)id * bytes;
}

#endif

// Argument checks shared by the entry points.
inline fairy2i_status kv_check(const fairy2i_kv_cache* c, const fairy2i_kv_batch* b) {
  if (!c || !b || !c->data || !b->pages || !b->cu_new || !b->lens) return FAIRY2I_ERR_NULL;
  if (fairy2i_kv_cache_bytes(c->n_pages, c->page_size, c->n_kv_heads, c->dc) == 0) return FAIRY2I_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(c->data) & 15) != 0) return FAIRY2I_ERR_UNSUPPORTED;
  if (b->n_seqs < 1 || b->n_seqs > (1 << 20) || b->max_pages < 1 || b->n_new < 1 || b->n_new > kKvMaxNew ||
      (int64_t)b->max_pages * c->page_size > kKvMaxLen)
    return FAIRY2I_ERR_SHAPE;
  return FAIRY2I_OK;
}

inline KvCache kv_cache_of(const fairy2i_kv_cache* c) {
  return {c->data, c->n_pages, c->page_size, c->n_kv_heads, c->dc};
}

inline KvBatch kv_batch_of(const fairy2i_kv_batch* b) {
  return {b->pages, b->cu_new, b->lens, b->n_seqs, b->max_pages, (int32_t)b->n_new};
}

}  // namespace fairy2i
