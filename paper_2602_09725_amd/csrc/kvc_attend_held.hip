// Attention of a batch over pages held in 4 bits (kvc_attend_paged on a pool of KVC_HELD_Q4).
//
// A token's key is k = s c + m with codes c of 0 .. 15 and a pair (s, m) of its head, so that q . k = s (q . c) + m sum(q); its value likewise, so that
//   sum_t w_t v_t = sum_t (w_t s_t) c_t + sum_t w_t m_t.
// Codes go into the matrix unit as they are: the products with keys are of exact numbers, and nothing is dequantized element by element.
//   Keys: four bits in the low mantissa bits of an fp16 number are c 2^-24, a subnormal that the matrix unit takes exactly; the next four bits are c 2^-20.  Queries are
//   made fp16 numbers of their row's size (a power of two, exact but for elements 2^34 below the row's largest), those that meet the second kind a sixteenth of it.
//   Values: four bits in the mantissa of 128 are 128 + c in bf16.  Weights w s are rounded to bf16 (half a step, as the inputs of such a pool have), or for a pool
//   of fp16 to two of them, which hold 16 bits.  A third product, with ones, sums the rounded weights: 136 of these sums are taken off and w (m + 8 s)
//   is added in fp32, so that a weight's rounding counts by the distance from the middle of the codes, not from 0.
//
// A tile is 64 tokens of a wave's own.  S^T = K Q^T and O^T += V^T W^T are 16x16x32 products: a lane has one row (lane % 16), and of a tile the 16 tokens from
// 16 (lane / 16) on.  A page has each word of four tokens side by side (a quad), so that a lane's 16 bytes are the operands of four products with keys, and
// of values, whose operands take two tokens' codes of one element, words of two tokens are merged half by half.  No operand passes through LDS; the pairs do, a token a lane.
#include <hip/hip_runtime.h>

#include "kvc_attend.h"
#include "kvc_device.h"
#include "kvc_serve.h"

namespace kvc {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 mfma_f16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

constexpr uint32_t kTile = 64;  // tokens

// Sizes of a body: DP elements of a head at most, RB blocks of 16 rows.
template <int DP>
struct Sizes {
  static constexpr int KS = DP / 32;                  // products of 32 elements, and vectors of keys that a lane loads
  static constexpr int VS = DP > 128 ? 2 : 1;         // vectors of values of a quad that it loads
  static constexpr int NJ = DP == 64 ? 4 : 8;         // elements of a word that a lane's values go to products of
};

// The exchange of a row's four lanes.
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float row_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// What a wave knows of its unit.
template <bool BIG>
struct Unit {
  using Offset = typename std::conditional<BIG, uint64_t, uint32_t>::type;  // within a layer's keys, or values
  const uint8_t KVC_GLOBAL *codes, *pairs;  // of the head's keys, page 0
  uint64_t values;                          // from keys to values
  const int32_t* table;
  uint32_t t0, t1, bound;  // tokens of the unit that are there; none that the host knows of lies at or beyond `bound`
  uint32_t quad_bytes;     // codes of a quad
};

// A tile's loads.
template <int DP>
struct Tile {
  u32x4 k[Sizes<DP>::KS], v[Sizes<DP>::VS][4];
  uint32_t kp, vp;   // pairs of token `lane`
  uint32_t missing;  // bit: the quad is on no page of the pool
};

template <int DP, int RB>
struct State {
  float m[RB], l[RB], low[RB];  // a number near the largest product, sum of this lane's weights, of what they add to all elements
  f32x4 total[RB];              // sums of the rounded weights
  f32x4 sum[RB][Sizes<DP>::VS][Sizes<DP>::NJ];
};

template <int RB>
struct Rows {
  float unit[RB], whole[RB];    // log2 of a weight for one step of a product; sum of the query
  float slack[RB];
  uint32_t limit[RB];           // positions below it are seen
};

template <bool BIG>
__device__ __forceinline__ uint32_t page_of_lane(const AttendParams& p, const Unit<BIG>& u, uint32_t at) {
  return (uint32_t)u.table[fd_div(p.pool.dbs, min(at + (threadIdx.x & 15u) * 4, u.bound - 1))];
}

template <typename T>
__device__ __forceinline__ T of_lane(uint32_t lane, T v) {
  if constexpr (sizeof(T) == 8)
    return (uint64_t)(uint32_t)__builtin_amdgcn_ds_bpermute((int)(lane * 4), (int)(uint32_t)(v >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_ds_bpermute((int)(lane * 4), (int)(uint32_t)v);
  else
    return (uint32_t)__builtin_amdgcn_ds_bpermute((int)(lane * 4), (int)v);
}

// Loads the tile at position `at`; page: that of the lane's quad.  A quad that is not there is read from page 0, which is.
template <int DP, bool BIG>
__device__ __forceinline__ void load_tile(const AttendParams& p, const Unit<BIG>& u, uint32_t at, uint32_t page, Tile<DP>& t) {
  using S = Sizes<DP>;
  using Offset = typename Unit<BIG>::Offset;
  const uint32_t lane = threadIdx.x & 63u, quad = lane & 15u, g = lane >> 4, W = p.D / 8;
  const uint32_t pos = at + quad * 4;
  const bool gone = pos >= u.t1, bad = page >= p.pool.num_blocks;
  t.missing = (uint32_t)__ballot(bad && !gone) & 0xffffu;
  const uint32_t slot = pos - fd_div(p.pool.dbs, pos) * p.pool.block_size;
  const bool none = bad || gone;
  const Offset begin = none ? (Offset)0 : (Offset)page * (Offset)p.pool.page_bytes;
  const Offset codes = begin + (none ? 0u : slot / 4 * u.quad_bytes), pairs = begin + (none ? 0u : slot * 4);
  const uint8_t KVC_GLOBAL* const value_codes = u.codes + u.values;
#pragma unroll
  for (int e = 0; e < S::KS; ++e) {
    const uint32_t w = min((uint32_t)e * 4 + g, W - 1);  // (words that the head lacks meet a query's zeros)
    t.k[e] = *(const u32x4 KVC_GLOBAL*)(u.codes + (codes + w * 16));
  }
  const Offset pair = of_lane(lane / 4, pairs) + (lane & 3u) * 4;
  t.kp = *(const uint32_t KVC_GLOBAL*)(u.pairs + pair);
  t.vp = *(const uint32_t KVC_GLOBAL*)(u.pairs + u.values + pair);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const Offset from = of_lane(g * 4 + i, codes);
#pragma unroll
    for (int s = 0; s < S::VS; ++s) {
      const uint32_t w = min(DP == 64 ? quad & 7u : quad + 16 * s, W - 1);  // (elements that the head lacks are not written)
      t.v[s][i] = *(const u32x4 KVC_GLOBAL*)(value_codes + (from + w * 16));
    }
  }
}

// Eight codes -> an operand of the products with keys.
__device__ __forceinline__ u32x4 key_operand(uint32_t w) {
  const uint32_t h = w >> 8;
  return u32x4{w & 0x000f000fu, w & 0x00f000f0u, h & 0x000f000fu, h & 0x00f000f0u};
}

// One tile.  MASKED: not all of it is there and seen by all rows.
template <int DT, int DP, int RB, bool MASKED>
__device__ __forceinline__ void take_tile(const AttendParams& p, uint32_t at, uint32_t t1, const Tile<DP>& t, const Rows<RB>& rows,
                                          const u32x4 (&query)[RB][Sizes<DP>::KS], State<DP, RB>& x, f32x2* kpair, f32x2* vpair) {
  using S = Sizes<DP>;
  const uint32_t lane = threadIdx.x & 63u, g = lane >> 4;
  {
    float s, m;
    widen_pair<DT>(t.kp, s, m);
    kpair[lane] = f32x2{s, m};
    widen_pair<DT>(t.vp, s, m);
    vpair[lane] = f32x2{s, fmaf(8.0f, s, m)};
  }
  // products: s[b][k][i] is token 16 g + 4 i + k
  f32x4 s[RB][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int e = 0; e < S::KS; ++e) {
      const u32x4 a = key_operand(t.k[e][k]);
#pragma unroll
      for (int b = 0; b < RB; ++b) s[b][k] = mfma_f16(a, query[b][e], e ? s[b][k] : f32x4{0, 0, 0, 0});
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x2 pair = kpair[16 * g + 4 * i + k];
#pragma unroll
      for (int b = 0; b < RB; ++b) s[b][k][i] = fmaf(pair.x, s[b][k][i], pair.y * rows.whole[b]);
    }
  if constexpr (MASKED) {
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const int32_t seen = (int32_t)(min(rows.limit[b], t1) - at - 16 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (4 * i + k >= seen || (t.missing >> (4 * g + i) & 1u)) s[b][k][i] = kNone;
    }
  }
  // bases
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    float top = kNone;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[b][k][i]);
    if (__any(top > x.m[b] + rows.slack[b])) {
      const float now = fmaxf(x.m[b], row_max(top)), keep = weight(x.m[b] * rows.unit[b], now * rows.unit[b]);
      x.m[b] = now;
      x.l[b] *= keep;
      x.low[b] *= keep;
      x.total[b] *= keep;
#pragma unroll
      for (int v = 0; v < S::VS; ++v)
#pragma unroll
        for (int j = 0; j < S::NJ; ++j) x.sum[b][v][j] *= keep;
    }
  }
  // weights: w[b][h] is the operand of tokens 16 g + 8 h .. + 7
  u32x4 w[RB][2], fine[RB][2];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const float shift = x.m[b] == kNone ? 0.0f : x.m[b] * rows.unit[b];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const f32x2 pair = vpair[16 * g + 4 * i + k];
        const float y = __builtin_amdgcn_exp2f(fmaf(s[b][k][i], rows.unit[b], -shift));
        x.l[b] += y;
        a[k] = y * pair.x;
        const float low = fmaf(y, pair.y, x.low[b]);
        if constexpr (MASKED) {  // (what is not seen may be held with anything)
          const bool none = s[b][k][i] == kNone;
          a[k] = none ? 0.0f : a[k];
          x.low[b] = none ? x.low[b] : low;
        } else {
          x.low[b] = low;
        }
      }
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
        const uint32_t r = narrow_pair<KVC_BF16>(a[k], a[k + 1]);
        w[b][i / 2][i % 2 * 2 + k / 2] = r;
        if constexpr (DT == KVC_F16) fine[b][i / 2][i % 2 * 2 + k / 2] = narrow_pair<KVC_BF16>(a[k] - widen_bits<KVC_BF16>(r & 0xffffu), a[k + 1] - widen_bits<KVC_BF16>(r >> 16));
      }
    }
  }
  // values
  const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      x.total[b] = mfma_bf16(ones, w[b][h], x.total[b]);
      if constexpr (DT == KVC_F16) x.total[b] = mfma_bf16(ones, fine[b][h], x.total[b]);
    }
#pragma unroll
    for (int v = 0; v < S::VS; ++v) {
      const u32x4 y = t.v[v][2 * h], z = t.v[v][2 * h + 1];
#pragma unroll
      for (int half = 0; half < (DP == 64 ? 1 : 2); ++half) {
        // (of up to 64 elements the lanes from 8 on have the odd elements of the words that the others have)
        const uint32_t sel = DP == 64 ? ((lane & 8u) ? 0x07060302u : 0x05040100u) : half ? 0x07060302u : 0x05040100u;
        const u32x4 both = {__builtin_amdgcn_perm(y.y, y.x, sel), __builtin_amdgcn_perm(y.w, y.z, sel), __builtin_amdgcn_perm(z.y, z.x, sel),
                            __builtin_amdgcn_perm(z.w, z.z, sel)};
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const u32x4 a = {(both.x >> 4 * n & 0x000f000fu) | 0x43004300u, (both.y >> 4 * n & 0x000f000fu) | 0x43004300u,
                           (both.z >> 4 * n & 0x000f000fu) | 0x43004300u, (both.w >> 4 * n & 0x000f000fu) | 0x43004300u};
          const int j = DP == 64 ? n : 2 * n + half;
#pragma unroll
          for (int b = 0; b < RB; ++b) {
            x.sum[b][v][j] = mfma_bf16(a, w[b][h], x.sum[b][v][j]);
            if constexpr (DT == KVC_F16) x.sum[b][v][j] = mfma_bf16(a, fine[b][h], x.sum[b][v][j]);
          }
        }
      }
    }
  }
}

// The query of a row as the products take it, and what its weights are computed with.
template <int DT, int DP, int RB>
__device__ __forceinline__ void load_queries(const AttendParams& p, const uint16_t* const (&from)[RB], const bool (&there)[RB], u32x4 (&query)[RB][Sizes<DP>::KS],
                                             Rows<RB>& rows) {
  using S = Sizes<DP>;
  const uint32_t g = (threadIdx.x & 63u) >> 4, W = p.D / 8;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    u32x4 raw[S::KS];
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < S::KS; ++e) {
      const uint32_t w = e * 4 + g;
      raw[e] = *(const KVC_GLOBAL u32x4*)(from[b] + min(w, W - 1) * 8);
      if (!there[b] || w >= W) raw[e] = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) most = max(most, max(raw[e][i] & 0x7fffu, raw[e][i] >> 16 & 0x7fffu));
    }
    const float largest = row_max(widen_bits<DT>(most));
    // its largest element comes to lie in [2^14, 2^15).  (An infinity or a NaN stays one; beyond 2^115 the step would pass fp32's range.)
    int up = largest > 0.0f && largest < __builtin_inff() ? 15 - __builtin_amdgcn_frexp_expf(largest) : 0;
    up = max(up, -100);
    float whole = 0.0f;
#pragma unroll
    for (int e = 0; e < S::KS; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x, y;
        widen_pair<DT>(raw[e][i], x, y);
        x = __builtin_amdgcn_ldexpf(x, up), y = __builtin_amdgcn_ldexpf(y, up);
        whole += x + y;
        query[b][e][i] = i % 2 ? narrow_pair<KVC_F16>(x * 0.0625f, y * 0.0625f) : narrow_pair<KVC_F16>(x, y);
      }
    rows.whole[b] = row_sum(whole) * 5.9604644775390625e-8f;  // (2^-24, as the codes)
    rows.unit[b] = __builtin_amdgcn_ldexpf(p.scale_log2, 24 - up);
    rows.slack[b] = fminf(8.0f / rows.unit[b], 1e30f);
  }
}

template <int DP, int RB>
struct Lds {
  struct {
    f32x2 k[kTile], v[kTile];
  } pairs[4];
  float sums[4][16 * RB][DP];
  float m[4][16 * RB], l[4][16 * RB];
};

// Element of a head that sum j of row i of a lane's is.
template <int DP>
__device__ __forceinline__ uint32_t element_of(uint32_t g, int v, int j, int i) {
  if constexpr (DP == 64) {
    const uint32_t c = 4 * g + i;
    return 8 * (c & 7u) + 2 * j + (c >> 3);
  }
  return 8 * (16 * v + 4 * g + i) + j;
}

// From the lanes' rows to all of a block's: the most and the least that one sees.
__device__ __forceinline__ void lanes_see(uint32_t& most, uint32_t& least) {
#pragma unroll
  for (int d = 1; d < 16; d *= 2) {
    most = max(most, (uint32_t)__shfl_xor((int)most, d));
    least = min(least, (uint32_t)__shfl_xor((int)least, d));
  }
}

// One unit: 16 RB rows x head x piece of the tokens; a workgroup's, whose waves have every fourth tile, or (LONE) a wave's.
template <int DT, int DP, int RB, bool BIG, bool LONE>
__device__ __forceinline__ void attend_unit(const AttendParams& p, const AttendPart& part, const bool shared, uint32_t unit, Lds<DP, RB>& lds) {
  using S = Sizes<DP>;
  constexpr uint32_t ROWS = 16 * RB;
  const uint32_t lane = threadIdx.x & 63u, wave = wave_uniform(threadIdx.x >> 6), col = lane & 15u, g = lane >> 4;
  const uint32_t speaker = LONE ? lane : threadIdx.x;
  const Place at_work = place_of_unit(p, part, shared, unit);

  Request q{};
  if (!shared) q = request_at(p, at_work.request);
  const uint32_t new_tokens = shared ? p.batch.n_new : covered(p, q);
  if (!shared && p.pieces == 1 && at_work.block == 0 && q.faults)  // (of several pieces the join writes what these rows hold)
    write_uncovered(p, q, at_work.request, at_work.head, speaker, LONE ? 64 : 256);
  if (!shared && at_work.block * ROWS >= wave_uniform(new_tokens) * p.G) {  // (a request with fewer new tokens than others)
    if (speaker == 0) fault(p, q.faults);
    return;
  }
  Unit<BIG> u;
  u.bound = shared ? p.prefix : p.most_tokens;
  u.t0 = (shared ? 0 : p.own_from) + at_work.split * part.tokens;
  u.table = p.pool.tables + (uint64_t)(shared ? p.prefix_row : wave_uniform(q.row)) * p.pool.table_len;
  constexpr uint32_t NEXT = LONE ? kTile : 4 * kTile;
  const uint32_t start = u.t0 + (LONE ? 0 : wave * kTile);
  // (the table has an entry for every position below the bound, and need not wait for the row's length)
  uint32_t page[2] = {page_of_lane<BIG>(p, u, start), page_of_lane<BIG>(p, u, start + NEXT)};

  const uint32_t base_row = at_work.block * ROWS;
  const uint16_t* from[RB];
  bool there[RB];
  uint32_t token[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    uint32_t t, k;
    fd_divmod(p.dG, base_row + b * 16 + col, t, k);
    there[b] = t < new_tokens;
    token[b] = (there[b] ? t : 0) + (shared ? 0 : min(q.first, p.batch.n_new - 1));
    from[b] = p.q + (int64_t)token[b] * p.q_token + (int64_t)(at_work.head * p.G + k) * p.q_head;
  }
  const uint64_t block = p.pool.block_size, W = p.D / 8;
  const uint8_t KVC_GLOBAL* const layer = (const uint8_t KVC_GLOBAL*)as_const(p.pool.layers)[p.layer];
  u.codes = layer + at_work.head * block * W * 4;
  u.pairs = layer + (p.H * W + at_work.head) * block * 4;
  u.values = (uint64_t)p.pool.num_blocks * p.pool.page_bytes;
  u.quad_bytes = (uint32_t)W * 16;
  u.t1 = shared ? prefix_there(p) : min(wave_uniform(q.len), p.most_tokens);
  if (shared && u.t1 < p.prefix && speaker == 0) fault(p, KVC_FAULT_LIST);
  u.t1 = min(u.t1, u.t0 + part.tokens);
  Tile<DP> tile[2];
  if (start < u.t1) load_tile<DP, BIG>(p, u, start, page[0], tile[0]);

  // How far the rows see.
  Rows<RB> rows;
  u32x4 query[RB][S::KS];
  load_queries<DT, DP, RB>(p, from, there, query, rows);
  uint32_t most = 0, least = ~0u;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    Request r = q;
    if (shared) r = request_at(p, request_of(p.batch, token[b]));
    if (shared ? there[b] && at_work.split == 0 && at_work.head == 0 && g == 0 : speaker == 0 && b == 0) fault(p, r.faults);
    rows.limit[b] = there[b] ? limit_of(p, r, token[b]) : 0;
    most = max(most, rows.limit[b]);
    if (there[b]) least = min(least, rows.limit[b]);
  }
  lanes_see(most, least);
  least = wave_uniform(least);
  const uint32_t end = min(u.t1, wave_uniform(most)), plain = min(least, u.t1);

  State<DP, RB> x;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    x.m[b] = kNone;
    x.l[b] = x.low[b] = 0.0f;
    x.total[b] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < S::VS; ++v)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) x.sum[b][v][j] = f32x4{0, 0, 0, 0};
  }
  uint32_t missing = 0;
  auto step = [&](uint32_t pos, const Tile<DP>& now, Tile<DP>& next, uint32_t& page_of_next) {
    if (pos + NEXT < end) {
      load_tile<DP, BIG>(p, u, pos + NEXT, page_of_next, next);
      page_of_next = page_of_lane<BIG>(p, u, pos + 2 * NEXT);
    }
    missing |= now.missing;
    f32x2 *const kpair = lds.pairs[wave].k, *const vpair = lds.pairs[wave].v;
    if (pos + kTile <= plain && now.missing == 0) take_tile<DT, DP, RB, false>(p, pos, u.t1, now, rows, query, x, kpair, vpair);
    else take_tile<DT, DP, RB, true>(p, pos, u.t1, now, rows, query, x, kpair, vpair);
  };
  for (uint32_t pos = start; pos < end;) {
    step(pos, tile[0], tile[1], page[1]);
    pos += NEXT;
    tile[0] = tile[1];
  }
  if (missing && lane == 0) fault(p, KVC_FAULT_PAGE);
  if (u.t0 >= end && p.pieces > 1) return;  // the join does not look for it

  // Results go through LDS, so that a row's are written side by side; waves along the tokens are joined there.
  if constexpr (!LONE) __syncthreads();
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const float low = row_sum(x.low[b]), total = row_sum(x.l[b]);
    const float off = fmaf(-136.0f, x.total[b][0], low);
    float* const to = lds.sums[wave][b * 16 + col];
#pragma unroll
    for (int v = 0; v < S::VS; ++v)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t at = element_of<DP>(g, v, j, i);
          to[((at / 4) ^ col) * 4 + at % 4] = x.sum[b][v][j][i] + off;
        }
    if (g == 0) {
      lds.m[wave][b * 16 + col] = x.m[b] != kNone ? x.m[b] * rows.unit[b] : total == 0.0f ? kNone : 0.0f;  // (a row that saw NaN alone is not empty)
      lds.l[wave][b * 16 + col] = total;
    }
  }
  if constexpr (!LONE) __syncthreads();
  else __builtin_amdgcn_wave_barrier();
  constexpr uint32_t QD = DP / 4, THREADS = LONE ? 64 : 256, SIDE = THREADS / QD, PARTS = LONE ? 1 : 4;
  const uint32_t self = LONE ? lane : threadIdx.x, at = self % QD;
  for (uint32_t r = self / QD; r < ROWS; r += SIDE) {
    uint32_t t, k;
    fd_divmod(p.dG, base_row + r, t, k);
    if (t >= new_tokens) break;
    float share[PARTS], top = kNone, total = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < PARTS; ++i) top = fmaxf(top, lds.m[LONE ? wave : i][r]);
#pragma unroll
    for (uint32_t i = 0; i < PARTS; ++i) {
      const float m = lds.m[LONE ? wave : i][r];
      share[i] = m == kNone ? -1.0f : weight(m, top);
      if (m != kNone) total += share[i] * lds.l[LONE ? wave : i][r];
    }
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (uint32_t i = 0; i < PARTS; ++i) {
      const f32x4 v = *(const f32x4*)&lds.sums[LONE ? wave : i][r][(at ^ (r & 15u)) * 4];
      if (!(share[i] < 0.0f)) o += share[i] * v;
    }
    const uint32_t at_token = shared ? t : q.first + t, head = at_work.head * p.G + k;
    if (p.pieces > 1) {
      const uint32_t piece = shared ? at_work.split : p.part[0].splits + at_work.split;
      const uint64_t slot = ((uint64_t)piece * p.batch.n_new + at_token) * (p.H * p.G) + head;
      if (at * 4 < p.D) *(KVC_GLOBAL f32x4*)(p.sums + slot * p.D + at * 4) = o;
      if (at == 0) *(KVC_GLOBAL f32x2*)(p.tops + slot * 2) = f32x2{top, total};
    } else {
      const float y = total == 0.0f ? 0.0f : 1.0f / total;
      uint16_t* const to = p.out + (int64_t)at_token * p.o_token + (int64_t)head * p.o_head + at * 4;
      if (at * 4 < p.D) *(KVC_GLOBAL u32x2*)to = u32x2{narrow_pair<DT>(o.x * y, o.y * y), narrow_pair<DT>(o.z * y, o.w * y)};
      if (at == 0 && p.lse) p.lse[(uint64_t)at_token * (p.H * p.G) + head] = total == 0.0f ? kNone : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
    }
  }
}

template <int DT, int DP, bool BIG>
__global__ void __launch_bounds__(256) attend_held_kernel(AttendParams p) {
  constexpr int MOST = DP > 128 ? 1 : 2;
  __shared__ Lds<DP, MOST> lds;
  bool shared;
  uint32_t unit;
  if (!unit_of(p, shared, unit)) return;
  const AttendPart& part = p.part[shared ? 0 : 1];
  Lds<DP, 1>& small = *reinterpret_cast<Lds<DP, 1>*>(&lds);
  if (part.lone) {
    unit = unit * 4 + wave_uniform(threadIdx.x >> 6);
    if (unit < part.lone) attend_unit<DT, DP, 1, BIG, true>(p, part, shared, unit, small);
  } else if (MOST == 1 || part.waves == 1) attend_unit<DT, DP, 1, BIG, false>(p, part, shared, unit, small);
  else attend_unit<DT, DP, MOST, BIG, false>(p, part, shared, unit, lds);
}

template <int DT, int DP>
kvc_status launch_of(const AttendParams& p, hipStream_t stream) {
  const uint32_t groups = (uint32_t)attend_groups(p);
  const bool big = (uint64_t)p.pool.num_blocks * p.pool.page_bytes >> 32;
  if (groups && big) hipLaunchKernelGGL((attend_held_kernel<DT, DP, true>), dim3(groups), dim3(256), 0, stream, p);
  if (groups && !big) hipLaunchKernelGGL((attend_held_kernel<DT, DP, false>), dim3(groups), dim3(256), 0, stream, p);
  if (hipGetLastError() != hipSuccess) return KVC_ERR_RUNTIME;
  return p.pieces == 1 ? KVC_OK : launch_join(p, stream);
}

}  // namespace

kvc_status plan_attend_held(AttendParams& p) {
  p.pieces = 0;
  p.dheads = make_fastdiv(p.H * p.G);
  p.slack = p.lift = 0.0f;
  const uint64_t chip = 512;  // workgroups that run at a time
  // Tiles lie on quads of the pages: up to three last tokens of a prefix that ends inside one are read through each row's own table, which has them too.
  p.prefix &= ~3u;
  p.own_from = p.prefix;
  for (int i = 0; i < 2; ++i) {
    AttendPart& a = p.part[i];
    a = AttendPart{};
    const uint64_t tokens = i == 0 ? p.own_from : p.most_tokens - p.own_from;
    const uint64_t rows = (uint64_t)(i == 0 ? p.batch.n_new : p.batch.most_new) * p.G;
    a.waves = rows <= 16 || p.D > 128 ? 1 : 2;  // blocks of 16 rows
    const uint64_t each_block = a.waves * 16, blocks = (rows + each_block - 1) / each_block;
    const uint64_t whole = blocks * p.H * (i == 0 ? 1 : p.batch.n_requests);
    a.drows = a.dsplits = a.drequests = make_fastdiv(1);
    if (tokens == 0) continue;
    if (whole >> 31) return KVC_ERR_UNSUPPORTED;
    uint64_t splits = whole <= chip ? chip / whole : 1;
    uint64_t each = (tokens + splits - 1) / splits;
    const uint64_t least = 4 * kTile;
    each = (each + least - 1) / least * least;
    splits = (tokens + each - 1) / each;
    if (whole * splits >> 31) return KVC_ERR_UNSUPPORTED;
    a.row_blocks = (uint32_t)blocks;
    a.splits = (uint32_t)splits;
    a.tokens = (uint32_t)each;
    a.units = (uint32_t)(whole * splits);
    a.drows = make_fastdiv(a.row_blocks);
    a.dsplits = make_fastdiv(a.splits);
    a.drequests = make_fastdiv(p.batch.n_requests);
    a.dtokens = make_fastdiv(a.tokens);
    p.pieces += a.splits;
  }
  return attend_fits(p) ? KVC_OK : KVC_ERR_UNSUPPORTED;
}

kvc_status launch_attend_held(const AttendParams& p, hipStream_t stream) {
  const bool half = p.dtype == KVC_F16;
  if (p.D <= 64) return half ? launch_of<KVC_F16, 64>(p, stream) : launch_of<KVC_BF16, 64>(p, stream);
  if (p.D <= 128) return half ? launch_of<KVC_F16, 128>(p, stream) : launch_of<KVC_BF16, 128>(p, stream);
  return half ? launch_of<KVC_F16, 256>(p, stream) : launch_of<KVC_BF16, 256>(p, stream);
}

}  // namespace kvc
