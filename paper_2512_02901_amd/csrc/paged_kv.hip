// Append to and read from the paged 4-bit cache.
//
// A wave owns four neighbouring positions (4 g .. 4 g + 3) of a head, a lane
// one or two complex entries of them.  Four positions are what a dword of
// either code array holds: a value dword is four positions of an entry, a key
// dword four entries of a position, so both go out whole (the keys' bytes
// transposed within four lanes), and no two waves share a byte.
//
// What bounds the append is memory: 8 bytes an entry of q, k and v in, 4 of q
// and about 1 of k and v each out.  3926 tokens of 32 heads on 8 (dc = 64) 28.6 us
// (5.3 TB/s, a plain copy's rate, with q's turns in blocks beside the keys');
// 15 single tokens of 32 on 32 4.8 us, a chain of loads (which sequence, its
// page, its values).  Reading the same tokens back 7.6 and 3.5 us.
#include <math.h>

#include <type_traits>

#include "paged_kv.h"

namespace fairy2i {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMostBlocks = ((int64_t)1 << 32) / kThreads - 1;  // a launch takes fewer than 2^32 threads

// Groups of four positions: sequence i's start at slot cu_new[i] / 4 + 2 i, so
// a slot's sequence is found without adding up anything.  (n positions touch
// at most (n + 2) / 4 + 1 <= n / 4 + 2 groups.)
__device__ inline int slot_of(const KvBatch& b, int i) { return (kv_row(b, i) >> 2) + 2 * i; }
inline int64_t slots(int64_t n_new, int64_t n_seqs) { return n_new / 4 + 2 * n_seqs; }

// 4 x 4 bytes transposed over four lanes: byte j of lane i's result is byte i
// of lane j's argument.
__device__ inline uint32_t transpose4(uint32_t x) {
  const int sh = 8 * (threadIdx.x & 3);
  uint32_t r = ((uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x00, 0xF, 0xF, true) >> sh & 0xFF);
  r |= ((uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x55, 0xF, 0xF, true) >> sh & 0xFF) << 8;
  r |= ((uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xAA, 0xF, 0xF, true) >> sh & 0xFF) << 16;
  r |= ((uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xFF, 0xF, 0xF, true) >> sh & 0xFF) << 24;
  return r;
}

__device__ inline float2 turn_at(const f32x2_any* p) {
  const f32x2_any t = *p;
  return make_float2(t.x, t.y);
}

// (re + i im)(c + i s), each product and sum rounded once.
__device__ inline float2 turn(float2 v, float2 cs) {
#pragma clang fp contract(off)
  return make_float2(v.x * cs.x - v.y * cs.y, v.x * cs.y + v.y * cs.x);
}

__device__ inline uint32_t bf16_pair(float2 v) {  // nearest even
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 p;
  p[0] = (__bf16)v.x;
  p[1] = (__bf16)v.y;
  return __builtin_bit_cast(uint32_t, p);
}

__device__ inline uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Biased exponent of the scale for a block whose largest magnitude has the
// bits `top`: the smallest e with top <= 7 2^e, so that what saturates at 6 is
// off by at most the half step of [4, 6]; from 2^-125 (0.5 2^e stays normal)
// to 2^125 (6 2^e stays finite).
__device__ inline uint32_t scale_of(uint32_t top) {
  const int e = (int)(top >> 23) - 2 + ((top & 0x7FFFFFu) > 0x600000u);
  return (uint32_t)min(max(e, 2), 252);
}

// Largest over the 16 lanes of a row, in all of them.
__device__ inline uint32_t row_top(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, true));  // rotated by 8, 4, 2, 1
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x124, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x122, 0xF, 0xF, true));
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x121, 0xF, 0xF, true));
}

// Byte J of `to`: v / 2^e, each part to the nearest of 0 .5 1 1.5 2 3 4 6 (ties
// to the even code, above 6 as 6), the real one in the low nibble.  The
// conversion takes the exponent of the scale.  The tests hold it at every midpoint
// and the floats next to it, scales from 2^-122 to 2^124.
template <int J>
__device__ inline uint32_t e2m1(uint32_t to, float2 v, uint32_t scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(to, v.x, v.y, __uint_as_float(scale << 23), J);
}

struct AppendArgs {
  KvCache c;
  KvBatch b;
  const float2 *q, *k, *v;
  int64_t q_ld, k_ld, v_ld;
  const f32x2_any* rope;  // [rope_len][dc]
  int64_t rope_len;
  u32_any* q_out;      // [n_new][heads][dc] bf16 pairs, or null
  int32_t heads;
  int32_t head_groups; // of keys and values: waves that a slot takes
  int32_t kv_blocks, q_chunks;
};

// EPL: entries a lane (2 for dc > 64, since a head's values meet in one wave to
// be found finite).  Heads of up to 32 entries share a wave.
template <int EPL>
__device__ void append_kv(const AppendArgs& a) {
  const int lane = threadIdx.x & 63, dc = a.c.dc;
  const int job = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)));
  const int slot = job / a.head_groups, hg = job - slot * a.head_groups;
  const int i = kv_find(a.b.n_seqs, slot, [&](int s) { return slot_of(a.b, s); });
  if (i < 0) return;
  const KvSeq s = kv_seq(a.b, a.c, i);
  const int group = (s.p0 >> 2) + slot - slot_of(a.b, i), u0 = 4 * group % kKvTile;
  if (s.n == 0 || group < 0 || 4 * (int64_t)group >= s.len) return;
  const int hpw = dc <= 32 ? 64 / dc : 1;  // heads a wave
  const int sub = hpw > 1 ? lane / dc : 0, h = hg * hpw + sub;
  const KvTile t(dc / 16);
  const bool head = h < a.c.kv_heads;
  uint8_t* tile = kv_tile(a.c, a.b, i, 4 * group, head ? h : 0, t.bytes);
  if (!tile) return;
  uint32_t valid = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int p = 4 * group + j;
    if (p >= s.p0 && p < s.len && p < a.rope_len) valid |= 1u << j;
  }
  float2 kx[EPL][4], vx[EPL][4];
#pragma unroll
  for (int x = 0; x < EPL; ++x) {
    const int e = lane - sub * dc + 64 * x;
    const bool mine = head && e < dc;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool load = mine && (valid >> j & 1);
      const int64_t row = s.row0 + (4 * group + j - s.p0);
      const float2 zero = make_float2(0.0f, 0.0f);
      const float2 cs = load ? turn_at(a.rope + (int64_t)(4 * group + j) * dc + e) : zero;
      const float2 k = load ? a.k[row * a.k_ld + (int64_t)h * dc + e] : zero;
      kx[x][j] = turn(k, cs);
      vx[x][j] = load ? a.v[row * a.v_ld + (int64_t)h * dc + e] : zero;
    }
  }
  // whole-wave work from here on: every lane takes part in the exchanges
  uint32_t bad = 0;  // positions of the lane's head that hold a value that is not finite
  const uint64_t of_head = hpw > 1 ? ((1ull << dc) - 1) << (sub * dc) : ~0ull;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t top = 0;
#pragma unroll
    for (int x = 0; x < EPL; ++x)
      top = max(top, max(max(abs_bits(kx[x][j].x), abs_bits(kx[x][j].y)), max(abs_bits(vx[x][j].x), abs_bits(vx[x][j].y))));
    if (__ballot(top >= 0x7F800000u) & of_head) bad |= 1u << j;
  }
#pragma unroll
  for (int x = 0; x < EPL; ++x) {
    const int e = lane - sub * dc + 64 * x, b = e / 16, r = e % 16;
    const bool mine = head && e < dc;
    uint32_t kc = 0, vc = 0, my_ks = 0, my_vs = 0;
    auto quantise = [&](auto of) {
      constexpr int j = decltype(of)::value;
      const uint32_t kt = row_top(max(abs_bits(kx[x][j].x), abs_bits(kx[x][j].y)));
      uint32_t vt = row_top(max(abs_bits(vx[x][j].x), abs_bits(vx[x][j].y)));
      // a value block that is not finite is stored as zeros: its position's
      // keys carry the NaN, so whoever attends to it sees one, nobody else
      float2 v = vx[x][j];
      if (vt >= 0x7F800000u) {
        vt = 0;
        v = make_float2(0.0f, 0.0f);
      }
      const uint32_t ks = scale_of(kt), vs = scale_of(vt);
      kc = e2m1<j>(kc, kx[x][j], ks);
      vc = e2m1<j>(vc, v, vs);
      if (r == j) {
        my_ks = bad >> j & 1 ? 255u : ks;
        my_vs = vs;
      }
    };
    quantise(std::integral_constant<int, 0>{});
    quantise(std::integral_constant<int, 1>{});
    quantise(std::integral_constant<int, 2>{});
    quantise(std::integral_constant<int, 3>{});
    const uint32_t kd = transpose4(kc);
    if (mine) {
      const int w = 2 * b + u0 / 16, g = u0 % 16 / 4, j = lane & 3;
      if (valid >> j & 1) *reinterpret_cast<uint32_t*>(tile + t.dword(w, r / 4 * 16 + u0 % 16 + j)) = kd;
      uint8_t* at = tile + t.v_codes() + t.dword(w, g * 16 + r);
      if (valid == 15) {
        *reinterpret_cast<uint32_t*>(at) = vc;
      } else {
#pragma unroll
        for (int m = 0; m < 4; ++m)
          if (valid >> m & 1) at[m] = (uint8_t)(vc >> (8 * m));
      }
      if (r < 4 && (valid >> r & 1)) {
        tile[t.k_scales() + (u0 + r) * t.sb + b] = (uint8_t)my_ks;
        tile[t.v_scales() + (g * 8 + u0 / 16 * 4 + r) * t.sb + b] = (uint8_t)my_vs;
      }
    }
  }
}

// 1024 entries of a token's q, asked for before its position is known.
__device__ void rotate_q(const AppendArgs& a) {
  const int id = (int)blockIdx.x - a.kv_blocks, row = id / a.q_chunks, e0 = (id - row * a.q_chunks) * 1024;
  const int n = a.heads * a.c.dc;
  const float2* q = a.q + (int64_t)row * a.q_ld;
  float2 x[4], cs[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int e = e0 + m * kThreads + threadIdx.x;
    x[m] = e < n ? q[e] : make_float2(0.0f, 0.0f);
  }
  const int i = kv_find(a.b.n_seqs, row, [&](int s) { return kv_row(a.b, s); });
  int64_t p = -1;
  if (i >= 0) {
    const KvSeq s = kv_seq(a.b, a.c, i);
    if (row < s.row0 + s.n && s.p0 + (row - s.row0) < s.len) p = s.p0 + (row - s.row0);
  }
  const bool known = p >= 0 && p < a.rope_len;
  const f32x2_any* turns = a.rope + (known ? p : 0) * a.c.dc;
  int c = (e0 + (int)threadIdx.x) % a.c.dc;
  const int step = kThreads % a.c.dc;
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    cs[m] = known ? turn_at(turns + c) : make_float2(__builtin_nanf(""), __builtin_nanf(""));
    c += step;
    if (c >= a.c.dc) c -= a.c.dc;
  }
  u32_any* out = a.q_out + (int64_t)row * n;
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int e = e0 + m * kThreads + threadIdx.x;
    if (e < n) out[e] = bf16_pair(turn(x[m], cs[m]));
  }
}

template <int EPL>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(AppendArgs a) {
  if ((int)blockIdx.x < a.kv_blocks) append_kv<EPL>(a);
  else rotate_q(a);
}

struct ReadArgs {
  KvCache c;
  KvBatch b;
  u32_any *k, *v;  // [n_new][kv_heads][dc] bf16 pairs
  int32_t head_groups;
};

// For checks and for moving sequences, between steps and not in them, so it is the
// plain form, scales a byte at a time: 3926 tokens (20 MB) 7.5 us, where a copy's
// rate would be 3.9.
template <int EPL>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(ReadArgs a) {
  const int lane = threadIdx.x & 63, dc = a.c.dc;
  const int job = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)));
  const int slot = job / a.head_groups, hg = job - slot * a.head_groups;
  const int i = kv_find(a.b.n_seqs, slot, [&](int s) { return slot_of(a.b, s); });
  if (i < 0) return;
  const KvSeq s = kv_seq(a.b, a.c, i);
  const int group = (s.p0 >> 2) + slot - slot_of(a.b, i), u0 = 4 * group & (kKvTile - 1);
  if (s.n == 0 || 4 * group >= s.p0 + s.n) return;
  const int hpw = dc <= 32 ? 64 / dc : 1;
  const int sub = hpw > 1 ? lane / dc : 0, h = hg * hpw + sub;
  const KvTile t(dc / 16);
  const bool head = h < a.c.kv_heads;
  // before position 0 and past the table there is no page either
  const bool inside = group >= 0 && 4 * (int64_t)group < s.len;
  const uint8_t* tile = inside ? kv_tile(a.c, a.b, i, 4 * group, head ? h : 0, t.bytes) : nullptr;
#pragma unroll
  for (int x = 0; x < EPL; ++x) {
    const int e = lane - sub * dc + 64 * x, b = e / 16, r = e % 16;
    const bool mine = head && e < dc;
    const int w = 2 * b + u0 / 16, g = u0 % 16 / 4;
    uint32_t kd = 0, vd = 0, ks[4] = {255, 255, 255, 255}, vs[4] = {255, 255, 255, 255};  // no page: NaN
    if (mine && tile) {
      kd = *reinterpret_cast<const uint32_t*>(tile + t.dword(w, r / 4 * 16 + u0 % 16 + (lane & 3)));
      vd = *reinterpret_cast<const uint32_t*>(tile + t.v_codes() + t.dword(w, g * 16 + r));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ks[j] = tile[t.k_scales() + (u0 + j) * t.sb + b];
        vs[j] = tile[t.v_scales() + (g * 8 + u0 / 16 * 4 + j) * t.sb + b];
      }
    }
    kd = transpose4(kd);
    auto pair = [](uint32_t codes, uint32_t scale) {  // a power of two times a value of two bits: exact in bf16
      return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, __uint_as_float(scale << 23), 0));
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t row = 4 * (int64_t)group + j - s.p0;
      if (mine && row >= 0 && row < s.n) {
        const int64_t at = ((s.row0 + row) * a.c.kv_heads + h) * dc + e;
        a.k[at] = pair(kd >> (8 * j), ks[j]);
        a.v[at] = pair(vd >> (8 * j), vs[j]);
      }
    }
  }
}

__global__ __launch_bounds__(kThreads) void rope_table_kernel(int64_t n, int dc, double base, float2* __restrict__ out) {
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
    const int64_t p = i / dc;
    double sn, cs;
    sincos((double)p * pow(base, -(double)(i - p * dc) / dc), &sn, &cs);
    out[i] = make_float2((float)cs, (float)sn);
  }
}

int head_groups(int kv_heads, int dc) {
  const int hpw = dc <= 32 ? 64 / dc : 1;
  return (kv_heads + hpw - 1) / hpw;
}

}  // namespace

}  // namespace fairy2i

using namespace fairy2i;

extern "C" {

size_t fairy2i_kv_cache_bytes(int64_t n_pages, int32_t page_size, int32_t n_kv_heads, int32_t dc) {
  if (n_pages < 1 || n_pages > INT32_MAX || page_size < kKvTile || page_size > 65536 || page_size % kKvTile != 0 ||
      n_kv_heads < 1 || n_kv_heads > 65535 || dc < 16 || dc > kKvMaxDc || dc % 16 != 0)
    return 0;
  if ((double)n_pages * n_kv_heads * (page_size / kKvTile) > INT32_MAX) return 0;  // tiles are numbered in 32 bits
  return (size_t)n_pages * (size_t)n_kv_heads * (size_t)(page_size / kKvTile) * (size_t)KvTile(dc / 16).bytes;
}

fairy2i_status fairy2i_rope_table(int64_t n_pos, int32_t dc, double base, float* out, void* stream) {
  if (!out) return FAIRY2I_ERR_NULL;
  if (n_pos < 1 || n_pos > ((int64_t)1 << 30) || dc < 1 || dc > 4096 || !(base > 0.0) || !(base <= 1e300))
    return FAIRY2I_ERR_SHAPE;
  const int64_t n = n_pos * dc, blocks = min((n + kThreads - 1) / kThreads, kMostBlocks);
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream), n,
                     (int)dc, base, reinterpret_cast<float2*>(out));
  return hipGetLastError() == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

fairy2i_status fairy2i_kv_append(const fairy2i_kv_cache* cache, const fairy2i_kv_batch* batch, const float* q,
                                 int64_t q_ld, int32_t n_heads, const float* k, int64_t k_ld, const float* v,
                                 int64_t v_ld, const float* rope, int64_t rope_len, void* q_out, void* stream) {
  if (const fairy2i_status s = kv_check(cache, batch)) return s;
  if (!k || !v || !rope || (q && !q_out) || (!q && q_out)) return FAIRY2I_ERR_NULL;
  const int64_t nkv = (int64_t)cache->n_kv_heads * cache->dc, nq = q ? (int64_t)n_heads * cache->dc : 0;
  if (rope_len < 1 || k_ld < nkv || v_ld < nkv || (q && (n_heads < 1 || n_heads > 65535 || q_ld < nq)))
    return FAIRY2I_ERR_SHAPE;
  AppendArgs a{};
  a.c = kv_cache_of(cache);
  a.b = kv_batch_of(batch);
  a.q = reinterpret_cast<const float2*>(q);
  a.k = reinterpret_cast<const float2*>(k);
  a.v = reinterpret_cast<const float2*>(v);
  a.q_ld = q_ld;
  a.k_ld = k_ld;
  a.v_ld = v_ld;
  a.rope = reinterpret_cast<const f32x2_any*>(rope);
  a.rope_len = rope_len;
  a.q_out = static_cast<u32_any*>(q_out);
  a.heads = n_heads;
  a.head_groups = head_groups(cache->n_kv_heads, cache->dc);
  const int64_t waves = slots(batch->n_new, batch->n_seqs) * a.head_groups, kv_blocks = (waves + 3) / 4;
  const int64_t chunks = (nq + 1023) / 1024, blocks = kv_blocks + chunks * batch->n_new;
  if (blocks > kMostBlocks) return FAIRY2I_ERR_UNSUPPORTED;
  a.kv_blocks = (int32_t)kv_blocks;
  a.q_chunks = (int32_t)chunks;
  auto kernel = cache->dc <= 64 ? kv_append_kernel<1> : kv_append_kernel<2>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

fairy2i_status fairy2i_kv_read(const fairy2i_kv_cache* cache, const fairy2i_kv_batch* batch, void* k_out, void* v_out,
                               void* stream) {
  if (const fairy2i_status s = kv_check(cache, batch)) return s;
  if (!k_out || !v_out) return FAIRY2I_ERR_NULL;
  ReadArgs a{};
  a.c = kv_cache_of(cache);
  a.b = kv_batch_of(batch);
  a.k = static_cast<u32_any*>(k_out);
  a.v = static_cast<u32_any*>(v_out);
  a.head_groups = head_groups(cache->n_kv_heads, cache->dc);
  const int64_t waves = slots(batch->n_new, batch->n_seqs) * a.head_groups, blocks = (waves + 3) / 4;
  if (blocks > kMostBlocks) return FAIRY2I_ERR_UNSUPPORTED;
  auto kernel = cache->dc <= 64 ? kv_read_kernel<1> : kv_read_kernel<2>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? FAIRY2I_OK : FAIRY2I_ERR_HIP;
}

}  // extern "C"
