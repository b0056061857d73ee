// Attention of a batch over pages held in 4 bits (kvc_attend_paged on a pool of KVC_HELD_Q4).
//
// A token's key is k = s (c - 8) + (m + 8 s) with codes c of 0 .. 15 and a pair (s, m) of its head, so that q . k = s (q . (c - 8)) + (m + 8 s) sum(q); its value
// likewise, so that, with z = m / s + 8,
//   sum_t w_t v_t = sum_t (w_t s_t) (c_t - 8) + sum_t (w_t s_t) z_t.
// Codes go into the matrix unit as they are: nothing is dequantized element by element, and the products with keys are of exact numbers, whose sums are
// no larger than the products that they stand for.
//   Four bits in the low mantissa bits of 1024 are 1024 + c in fp16, the next four bits 1024 + 16 c; one instruction takes 1032 or 1152 off two of them.
//   (Without the 1024 they are c 2^-24, subnormals that the matrix unit takes as well; but sums of such products have been seen to hold some 14 bits only.)
//   Queries are made fp16 numbers by a power of two that all rows of a workgroup share (exact but for what lies 2^-35 below the largest of their elements), those that
//   meet the second kind a sixteenth of it.
//   Weights w s, with s in the exponent, are rounded to fp16 (an eighth of the step that a bf16 pool's results have), or for a pool of fp16 to two such numbers, which
//   hold 22 bits.  One more product has rows of z (in two numbers): it sums the second term of the same rounded weights.
//
// A tile is 64 tokens.  S^T = K Q^T and O^T += V^T W^T are 16x16x32 products: a lane has one row (lane % 16), and of a tile the 16 tokens from
// 16 (lane / 16) on.  A page has each word of four tokens side by side (a quad), so that a lane's 16 bytes are the operands of four products with keys, and
// of values, whose operands take two tokens' codes of one element, words of two tokens are merged half by half.  No operand passes through LDS; what the pairs
// give does, a token a lane.
#include <hip/hip_runtime.h>

#include <math.h>

#include <type_traits>

#include "kvc_attend.h"
#include "kvc_device.h"
#include "kvc_serve.h"

namespace kvc {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
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
  uint32_t first;          // tokens below it are the other part's: up to three, where the prefix ends inside the quad that t0 is
  uint32_t quad_bytes;     // codes of a quad
};

// Where a lane's part of a tile lies: the codes and pairs of quad lane % 16.
template <bool BIG>
struct Source {
  typename Unit<BIG>::Offset codes, pairs;
  uint32_t missing;  // bit: the quad is on no page of the pool
};

// A tile's loads.
template <int DP>
struct Tile {
  u32x4 k[Sizes<DP>::KS], v[Sizes<DP>::VS][4];
  uint32_t kp, vp;  // pairs of token `lane`
};

// What the pairs of a tile's tokens give.
struct alignas(16) PairSpace {
  float ks[kTile], km[kTile];  // scale and m + 8 s of keys, times what a product is multiplied with
  float lv[kTile], rv[kTile];  // logarithm and reciprocal of the scale of values
  uint16_t z[2][kTile];        // rows of the product that sums weights, fp16: z, what is left of it
};

template <int DP, int RB>
struct State {
  float m[RB], l[RB];  // a number near the largest exponent of a weight times its value's scale, sum of this lane's weights
  f32x4 total[RB];     // what the rounded weights add to all elements, in two parts
  f32x4 sum[RB][Sizes<DP>::VS][Sizes<DP>::NJ];
};

template <int RB>
struct Rows {
  float whole[RB];      // sum of the query
  uint32_t limit[RB];   // positions below it are seen
  float unit;           // log2 of a weight for one step of a product
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

// Where the tile at position `at` lies; page: that of the lane's quad.  A quad that is not there is read from page 0, which is.
template <bool BIG>
__device__ __forceinline__ Source<BIG> source_of(const AttendParams& p, const Unit<BIG>& u, uint32_t at, uint32_t page) {
  using Offset = typename Unit<BIG>::Offset;
  const uint32_t pos = at + (threadIdx.x & 15u) * 4;
  const bool gone = pos >= u.t1, bad = page >= p.pool.num_blocks, none = bad || gone;
  const uint32_t slot = pos - fd_div(p.pool.dbs, pos) * p.pool.block_size;
  const Offset begin = none ? (Offset)0 : (Offset)page * (Offset)p.pool.page_bytes;
  return Source<BIG>{begin + (none ? (Offset)0 : (Offset)(slot / 4) * u.quad_bytes), begin + (none ? (Offset)0 : (Offset)slot * 4), (uint32_t)__ballot(bad && !gone) & 0xffffu};
}

template <int DP, bool BIG>
__device__ __forceinline__ void load_keys(const AttendParams& p, const Unit<BIG>& u, const Source<BIG>& from, Tile<DP>& t) {
  const uint32_t lane = threadIdx.x & 63u, g = lane >> 4, W = p.D / 8;
  const auto pair = of_lane(lane / 4, from.pairs) + (lane & 3u) * 4;
  t.kp = *(const uint32_t KVC_GLOBAL*)(u.pairs + pair);
  t.vp = *(const uint32_t KVC_GLOBAL*)(u.pairs + u.values + pair);
#pragma unroll
  for (int e = 0; e < Sizes<DP>::KS; ++e)  // (words that the head lacks meet a query's zeros)
    t.k[e] = *(const u32x4 KVC_GLOBAL*)(u.codes + (from.codes + min((uint32_t)e * 4 + g, W - 1) * 16));
}

template <int DP, bool BIG>
__device__ __forceinline__ void load_values(const AttendParams& p, const Unit<BIG>& u, const Source<BIG>& from, Tile<DP>& t) {
  const uint32_t lane = threadIdx.x & 63u, quad = lane & 15u, g = lane >> 4, W = p.D / 8;
  const uint8_t KVC_GLOBAL* const codes = u.codes + u.values;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto at = of_lane(g * 4 + i, from.codes);
#pragma unroll
    for (int s = 0; s < Sizes<DP>::VS; ++s)  // (elements that the head lacks are not written)
      t.v[s][i] = *(const u32x4 KVC_GLOBAL*)(codes + (at + min(DP == 64 ? quad & 7u : quad + 16 * s, W - 1) * 16));
  }
}

// Scales of values lie in [2^-60, 2^40]: a sum of weights, each held times its value's scale, has what it needs of fp32's range then.  (fp16's all do.)  Larger ones count as not
// finite.
constexpr float kLeastScale = 8.67361738e-19f, kMostScale = 1.09951163e12f;

// A head whose values are all alike has scale 0.  It is given a scale of its value's size, and codes of 0 (as one of smaller steps than that, or whose least value is beyond
// 2^15 steps, which no values of 16 bits have).
__device__ __forceinline__ bool is_flat(float s, float m) { return fabsf(m) * 3.0517578125e-5f >= s || s < kLeastScale; }

// The least value in steps of the scale.
__device__ __forceinline__ void steps_of(float& s, float m, float& z) {
  if (is_flat(s, m)) s = fmaxf(fabsf(m), kLeastScale);
  const float r = __builtin_amdgcn_rcpf(s);
  z = m * r;
  z = fmaf(fmaf(-z, s, m), r, z);
}

template <int DT>
__device__ __forceinline__ void put_key_pair(PairSpace& to, uint32_t token, uint32_t pair, float unit) {
  float s, m;
  widen_pair<DT>(pair, s, m);
  to.ks[token] = s * unit;
  to.km[token] = fmaf(8.0f, s, m) * unit;
}

// Tokens of a tile whose values are flat; pair: token `lane`'s.
template <int DT>
__device__ __forceinline__ uint64_t flat_tokens(uint32_t pair) {
  float s, m;
  widen_pair<DT>(pair, s, m);
  return __ballot(is_flat(s, m));
}

// A pair that is not finite makes NaN of the weights that see it, and nothing of the others.  there: the token is the part's own; one that is not has weight 0 for all rows.
// (Only a part's first tile has such tokens.  Decided here it costs a token a lane; among the masks of scores, 16 a lane, calls without a prefix took 7 % longer.)
template <int DT>
__device__ __forceinline__ void put_value_pair(PairSpace& to, uint32_t token, uint32_t pair, bool there) {
  constexpr uint32_t kExp = DT == KVC_F16 ? 0x7c00u : 0x7f80u;
  bool wild = (pair & kExp) == kExp || (pair >> 16 & kExp) == kExp;
  float s, m, z;
  widen_pair<DT>(pair, s, m);
  steps_of(s, m, z);
  if (DT == KVC_BF16) wild |= s > kMostScale;
  z = wild ? 0.0f : z + 8.0f;
  to.lv[token] = !there ? kNone : wild ? __builtin_nanf("") : __builtin_amdgcn_logf(s);
  to.rv[token] = __builtin_amdgcn_rcpf(s);
  const uint32_t high = narrow_pair<KVC_F16>(z, 0.0f);
  to.z[0][token] = (uint16_t)high;
  to.z[1][token] = (uint16_t)narrow_pair<KVC_F16>(z - widen_bits<KVC_F16>(high & 0xffffu), 0.0f);
}

// Codes c in the low mantissa bits of two halves, or c 16 in those above -> c - 8 or 16 (c - 8): 1024 and more, less 1032 or 1152.
template <int SHIFT>
__device__ __forceinline__ uint32_t centred(uint32_t w) {
  uint32_t mask = SHIFT ? 0x00f000f0u : 0x000f000fu, big = 0x64006400u;  // (in registers, so that one instruction takes both)
  asm("" : "+s"(mask));
  asm("" : "+v"(big));
  const uint32_t codes = (w & mask) | big, less = SHIFT ? 0x64806480u : 0x64086408u;
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2v, codes) - __builtin_bit_cast(f16x2v, less));
}

// Eight codes -> an operand of the products with keys.
__device__ __forceinline__ u32x4 key_operand(uint32_t w) {
  const uint32_t h = w >> 8;
  return u32x4{centred<0>(w), centred<4>(w), centred<0>(h), centred<4>(h)};
}

// Words of eight tokens -> two tokens' elements 2 n (or, with the selector's other value, 2 n + 1) side by side.
__device__ __forceinline__ u32x4 halves(u32x4 y, u32x4 z, uint32_t selector) {
  return u32x4{__builtin_amdgcn_perm(y.y, y.x, selector), __builtin_amdgcn_perm(y.w, y.z, selector), __builtin_amdgcn_perm(z.y, z.x, selector),
               __builtin_amdgcn_perm(z.w, z.z, selector)};
}
constexpr uint32_t kLow = 0x05040100u, kHigh = 0x07060302u;
// (Elements of odd n come 16 times too large.)
__device__ __forceinline__ u32x4 value_operand(u32x4 both, int n) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = n % 2 ? centred<4>(both[i] >> n / 2 * 8) : centred<0>(both[i] >> n / 2 * 8);
  return r;
}
template <int DP>
constexpr float size_of(int j) { return (DP == 64 ? j : j / 2) % 2 ? 0.0625f : 1.0f; }

// Sums of more than 128 elements have no room among the registers that other arithmetic takes: they stay in the matrix unit's own also where they are multiplied, once in
// many tiles.  (Left to itself the compiler moves all of them there and back for every tile; and 16 rows' fit two
// waves a SIMD so: a prompt of 8000 tokens, 16 query heads of 256, 974 -> 860 us, 64 requests of up to 2000 tokens 76 -> 45.  The 16-row body is short of registers
// then: 7 of a lane, 10 with fp16's second weights, lie in memory; of 128 elements with offsets of 64 bits 2 with fp16.)
template <int DP>
__device__ __forceinline__ void stay(f32x4& v) {
  if constexpr (DP > 128) asm volatile("" : "+a"(v));
}

// Weights of a tile from its products s[k][i], those of token 16 g + 4 i + k (they are overwritten): operands w[h] of tokens 16 g + 8 h .. + 7, and for fp16
// what their rounding left.  masked: not all of it is there and seen by all rows (wave-uniform); missing: quads on no page.  The number subtracted from an exponent need not be
// the largest one, as long as no weight leaves fp16; so that small ones stay in it too it lies 2^8 below the product that moves it.  Weights times scales down to 2^-33 of a row's largest
// count then; they are rounded to steps of 2^-24, and those below half of one are lost, while the sum of weights has them.  (The order is the source's: a few of LDS's numbers at a time.)
template <int DT, int DP, int RB>
__device__ __forceinline__ void weights(bool masked, uint32_t at, uint32_t t1, uint32_t missing, const PairSpace& pairs, const Rows<RB>& rows, int b, f32x4 (&s)[4],
                                        State<DP, RB>& x, u32x4 (&w)[2], u32x4 (&fine)[2]) {
  const uint32_t g = (threadIdx.x & 63u) >> 4;
  constexpr float kLift = 8.0f, kMost = 15.0f;
  const float shift = x.m[b] == kNone ? 0.0f : x.m[b];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 ks = *(const f32x4*)&pairs.ks[16 * g + 4 * i], km = *(const f32x4*)&pairs.km[16 * g + 4 * i], lv = *(const f32x4*)&pairs.lv[16 * g + 4 * i];
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k][i] = fmaf(s[k][i], ks[k], fmaf(km[k], rows.whole[b], lv[k] - shift));
    __builtin_amdgcn_sched_barrier(0);
  }
  if (masked) {
    const int32_t left = (int32_t)(min(rows.limit[b], t1) - at - 16 * g);
    const uint32_t gone = missing >> (4 * g);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k][i] = 4 * i + k < left && !(gone >> i & 1u) ? s[k][i] : kNone;
  }
  float top = kNone;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, s[k][i]);
  if (__any(top > kMost || x.m[b] == kNone)) {
    top = row_max(top);
    const bool first = x.m[b] == kNone;
    const float up = top == kNone ? 0.0f : first ? top - kLift : fmaxf(top - kLift, 0.0f), keep = __builtin_amdgcn_exp2f(first ? 0.0f : -up);
    if (!first || top != kNone) x.m[b] = shift + up;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k][i] -= up;
    x.l[b] *= keep;  // (a row that had no base has sums of 0)
    x.total[b] *= keep;
#pragma unroll
    for (int v = 0; v < Sizes<DP>::VS; ++v)
#pragma unroll
      for (int j = 0; j < Sizes<DP>::NJ; ++j) {
        stay<DP>(x.sum[b][v][j]);
        x.sum[b][v][j] *= keep;
        stay<DP>(x.sum[b][v][j]);
      }
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x4 rv = *(const f32x4*)&pairs.rv[16 * g + 4 * i];
    if (masked) {  // (what is not seen may be held with anything)
#pragma unroll
      for (int k = 0; k < 4; ++k) rv[k] = s[k][i] == kNone ? 0.0f : rv[k];
    }
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
      const float y = __builtin_amdgcn_exp2f(s[k][i]), z = __builtin_amdgcn_exp2f(s[k + 1][i]);
      x.l[b] = fmaf(y, rv[k], fmaf(z, rv[k + 1], x.l[b]));
      const uint32_t r = narrow_pair<KVC_F16>(y, z);
      w[i / 2][i % 2 * 2 + k / 2] = r;
      if constexpr (DT == KVC_F16)
        fine[i / 2][i % 2 * 2 + k / 2] = narrow_pair<KVC_F16>(y - widen_bits<KVC_F16>(r & 0xffffu), z - widen_bits<KVC_F16>(r >> 16));
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Operand of the product that sums weights: even rows of z, odd ones of its rest.
__device__ __forceinline__ u32x4 sums_operand(const PairSpace& pairs, int h) {
  const uint32_t lane = threadIdx.x & 63u;
  return *(const u32x4*)&pairs.z[lane & 1u][16 * (lane >> 4) + 8 * h];
}

// One tile of a wave's own.  The next tile's loads follow as soon as this one's have been used.
template <int DT, int DP, int RB, bool BIG>
__device__ __forceinline__ void take_tile(const AttendParams& p, const Unit<BIG>& u, bool masked, uint32_t at, uint32_t missing, const Source<BIG>& next, Tile<DP>& t,
                                          const Rows<RB>& rows, const u32x4 (&query)[RB][Sizes<DP>::KS], State<DP, RB>& x, PairSpace& pairs) {
  using S = Sizes<DP>;
  const uint32_t lane = threadIdx.x & 63u, g = lane >> 4;
  const bool there = at + lane >= u.first;
  put_key_pair<DT>(pairs, lane, there ? t.kp : 0, rows.unit);
  put_value_pair<DT>(pairs, lane, there ? t.vp : 0, there);
  const uint64_t flat = flat_tokens<DT>(t.vp);
  // (The order is the source's: left to itself the compiler makes all operands first, and has no registers for them.)
  f32x4 s[RB][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int e = 0; e < S::KS; ++e) {
      const u32x4 a = key_operand(t.k[e][k]);
#pragma unroll
      for (int b = 0; b < RB; ++b) s[b][k] = product(a, query[b][e], e ? s[b][k] : f32x4{0, 0, 0, 0});
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  load_keys<DP, BIG>(p, u, next, t);
  __builtin_amdgcn_sched_barrier(0);
  u32x4 w[RB][2], fine[RB][2];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    weights<DT, DP, RB>(masked, at, u.t1, missing, pairs, rows, b, s[b], x, w[b], fine[b]);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (flat) {  // (codes that their scale makes nothing of)
    const uint32_t mine = (uint32_t)(flat >> (16 * g)) & 0xffffu;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int v = 0; v < S::VS; ++v) t.v[v][i][k] = mine >> (4 * i + k) & 1u ? 0u : t.v[v][i][k];
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const u32x4 rows_of_sums = sums_operand(pairs, h);
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      x.total[b] = product(rows_of_sums, w[b][h], x.total[b]);
      if constexpr (DT == KVC_F16) x.total[b] = product(rows_of_sums, fine[b][h], x.total[b]);
    }
#pragma unroll
    for (int v = 0; v < S::VS; ++v)
#pragma unroll
      for (int half = 0; half < (DP == 64 ? 1 : 2); ++half) {
        // (of up to 64 elements the lanes from 8 on have the odd elements of the words that the others have)
        const u32x4 both = halves(t.v[v][2 * h], t.v[v][2 * h + 1], DP == 64 ? ((lane & 8u) ? kHigh : kLow) : half ? kHigh : kLow);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const u32x4 a = value_operand(both, n);
          const int j = DP == 64 ? n : 2 * n + half;
#pragma unroll
          for (int b = 0; b < RB; ++b) {
            x.sum[b][v][j] = product(a, w[b][h], x.sum[b][v][j]);
            if constexpr (DT == KVC_F16) x.sum[b][v][j] = product(a, fine[b][h], x.sum[b][v][j]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
  }
  load_values<DP, BIG>(p, u, next, t);
}

// The queries of a wave's rows as the products take them, and what weights are computed with.  Rows that see nothing, whose queries may be anything, do not count.
template <int DT, int DP, int RB>
__device__ __forceinline__ uint32_t load_queries(const AttendParams& p, const uint16_t* const (&from)[RB], u32x4 (&raw)[RB][Sizes<DP>::KS], const Rows<RB>& rows) {
  const uint32_t g = (threadIdx.x & 63u) >> 4, W = p.D / 8;
  constexpr uint32_t kExp = DT == KVC_F16 ? 0x7c00u : 0x7f80u;
  uint32_t most = 0;
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int e = 0; e < Sizes<DP>::KS; ++e) {
      const uint32_t w = e * 4 + g;
      raw[b][e] = *(const KVC_GLOBAL u32x4*)(from[b] + min(w, W - 1) * 8);
      if (rows.limit[b] == 0 || w >= W) raw[b][e] = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = raw[b][e][i] & 0x7fffu, y = raw[b][e][i] >> 16 & 0x7fffu;
        most = max(most, max(x < kExp ? x : 0, y < kExp ? y : 0));
      }
    }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, d));
  return most;
}

// most: the largest of the workgroup's elements (bits).  It comes to lie in [2^14, 2^15); a step beyond 2^115 would pass fp32's range.
template <int DT, int DP, int RB>
__device__ __forceinline__ void make_queries(const AttendParams& p, uint32_t most, u32x4 (&query)[RB][Sizes<DP>::KS], Rows<RB>& rows) {
  const int up = most ? max(15 - __builtin_amdgcn_frexp_expf(widen_bits<DT>(most)), -100) : 0;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    float whole = 0.0f;
#pragma unroll
    for (int e = 0; e < Sizes<DP>::KS; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x, y;
        widen_pair<DT>(query[b][e][i], x, y);
        x = __builtin_amdgcn_ldexpf(x, up), y = __builtin_amdgcn_ldexpf(y, up);
        whole += x + y;
        query[b][e][i] = i % 2 ? narrow_pair<KVC_F16>(x * 0.0625f, y * 0.0625f) : narrow_pair<KVC_F16>(x, y);
      }
    rows.whole[b] = row_sum(whole);
  }
  rows.unit = __builtin_amdgcn_ldexpf(p.scale_log2, -up);
}

// ---- up to 16 rows --------------------------------------------------------------------------------------------------------
//
// What few rows read bounds it: 24 rows of up to 16 000 tokens of 32 heads, 871 MB, 183 - 197 us, 4.4 - 4.8 TB/s with twelve waves a CU, each of which asks for its next tile's
// vectors as soon as the present one's have become operands.  Where there are few units their chain of answers does (four rows over 1000 tokens 10 us).

// LDS of a wave: the pairs of its tile, and in the end its sums.
template <int DP>
struct Lds {
  union Wave {
    PairSpace pairs;
    float sums[16][DP];
  } of[4];
  float m[4][16], l[4][16];
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

// A wave's sums into LDS, in vectors of four, and its rows' bases and sums of weights.
template <int DP, int RB>
__device__ __forceinline__ void put_sums(const State<DP, RB>& x, float (*sums)[DP], float* m, float* l) {
  const uint32_t lane = threadIdx.x & 63u, col = lane & 15u, g = lane >> 4;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const float total = row_sum(x.l[b]), off = x.total[b][0] + x.total[b][1];
    float* const to = sums[b * 16 + col];
#pragma unroll
    for (int v = 0; v < Sizes<DP>::VS; ++v)
#pragma unroll
      for (int j = 0; j < Sizes<DP>::NJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t at = element_of<DP>(g, v, j, i);
          to[((at / 4) ^ col) * 4 + at % 4] = fmaf(x.sum[b][v][j][i], size_of<DP>(j), off);
        }
    if (g == 0) {
      m[b * 16 + col] = x.m[b] != kNone ? x.m[b] : total == 0.0f ? kNone : 0.0f;  // (a row that saw NaN alone is not empty)
      l[b * 16 + col] = total;
    }
  }
}

// Writes a block's rows: PARTS waves have sums of each of them, THREADS threads write.
template <int DT, int DP, int ROWS, int PARTS, int THREADS>
__device__ __forceinline__ void write_rows(const AttendParams& p, bool shared, const Place& at_work, const Request& q, uint32_t new_tokens, uint32_t base_row,
                                           const float (*sums)[ROWS][DP], const float (*m)[ROWS], const float (*l)[ROWS], uint32_t self) {
  constexpr uint32_t QD = DP / 4, SIDE = THREADS / QD;
  const uint32_t at = self % QD;
#pragma unroll 1
  for (uint32_t r = self / QD; r < ROWS; r += SIDE) {
    uint32_t t, k;
    fd_divmod(p.dG, base_row + r, t, k);
    if (t >= new_tokens) break;
    float share[PARTS], top = kNone, total = 0.0f;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) top = fmaxf(top, m[i][r]);
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
      share[i] = m[i][r] == kNone ? -1.0f : weight(m[i][r], top);  // (below 0: the wave saw nothing)
      if (m[i][r] != kNone) total += share[i] * l[i][r];
    }
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
      const f32x4 v = *(const f32x4*)&sums[i][r][(at ^ (r & 15u)) * 4];
      if (!(share[i] < 0.0f)) o += share[i] * v;
    }
    const uint32_t token = shared ? t : q.first + t, head = at_work.head * p.G + k;
    if (p.pieces > 1) {
      const uint32_t piece = shared ? at_work.split : p.part[0].splits + at_work.split;
      const uint64_t slot = ((uint64_t)piece * p.batch.n_new + token) * (p.H * p.G) + head;
      if (at * 4 < p.D) *(KVC_GLOBAL f32x4*)(p.sums + slot * p.D + at * 4) = o;
      if (at == 0) *(KVC_GLOBAL f32x2*)(p.tops + slot * 2) = f32x2{top, total};
    } else {
      const float y = total == 0.0f ? 0.0f : 1.0f / total;
      uint16_t* const to = p.out + (int64_t)token * p.o_token + (int64_t)head * p.o_head + at * 4;
      if (at * 4 < p.D) *(KVC_GLOBAL u32x2*)to = u32x2{narrow_pair<DT>(o.x * y, o.y * y), narrow_pair<DT>(o.z * y, o.w * y)};
      if (at == 0 && p.lse) p.lse[(uint64_t)token * (p.H * p.G) + head] = total == 0.0f ? kNone : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
    }
  }
}

// Where a head's codes and pairs lie.
template <bool BIG>
__device__ __forceinline__ void place_of_head(const AttendParams& p, uint32_t head, Unit<BIG>& u) {
  const uint64_t block = p.pool.block_size, W = p.D / 8;
  const uint8_t KVC_GLOBAL* const layer = (const uint8_t KVC_GLOBAL*)as_const(p.pool.layers)[p.layer];
  u.codes = layer + head * block * W * 4;
  u.pairs = layer + (p.H * W + head) * block * 4;
  u.values = (uint64_t)p.pool.num_blocks * p.pool.page_bytes;
  u.quad_bytes = (uint32_t)W * 16;
}

// From the lanes' rows to all of a block's: the most and the least that one sees.
__device__ __forceinline__ void lanes_see(uint32_t& most, uint32_t& least) {
#pragma unroll
  for (int d = 1; d < 16; d *= 2) {
    most = max(most, (uint32_t)__shfl_xor((int)most, d));
    least = min(least, (uint32_t)__shfl_xor((int)least, d));
  }
}

// One unit: 16 rows x head x piece of the tokens; a workgroup's, whose waves have every fourth tile, or (LONE) a wave's.
template <int DT, int DP, bool BIG, bool LONE>
__device__ __forceinline__ void attend_unit(const AttendParams& p, const AttendPart& part, const bool shared, uint32_t unit, Lds<DP>& lds) {
  using S = Sizes<DP>;
  constexpr int RB = 1;
  constexpr uint32_t ROWS = 16;
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
  u.first = shared ? 0 : p.prefix;
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
  place_of_head(p, at_work.head, u);
  u.t1 = shared ? prefix_there(p) : min(wave_uniform(q.len), p.most_tokens);
  if (shared && u.t1 < p.prefix && speaker == 0) fault(p, KVC_FAULT_LIST);
  u.t1 = min(u.t1, at_work.split + 1 < part.splits ? u.t0 + part.tokens : ~0u);  // (the prefix's last piece has its last tokens too)
  const bool has_tile = start < u.t1;
  Tile<DP> tile;
  Source<BIG> at_tile = source_of<BIG>(p, u, start, page[0]);
  if (has_tile) {
    load_keys<DP, BIG>(p, u, at_tile, tile);
    load_values<DP, BIG>(p, u, at_tile, tile);
  }

  // How far the rows see.
  Rows<RB> rows;
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
  const uint32_t seen = min(u.t1, wave_uniform(most)), plain = min(least, u.t1);
  const uint32_t end = seen > u.first ? seen : 0;  // (a quad that has none of the part's tokens is not looked at)
  u32x4 query[RB][S::KS];
  make_queries<DT, DP, RB>(p, load_queries<DT, DP, RB>(p, from, query, rows), query, rows);

  State<DP, RB> x;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    x.m[b] = there[b] ? kNone : 0.0f;  // (a row that is not there asks for no base)
    x.l[b] = 0.0f;
    x.total[b] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < S::VS; ++v)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) x.sum[b][v][j] = f32x4{0, 0, 0, 0};
  }
  PairSpace& pairs = lds.of[wave].pairs;
  uint32_t missing = 0;
#pragma unroll 1
  for (uint32_t pos = start; pos < end; pos += NEXT) {
    const uint32_t holes = at_tile.missing;
    missing |= holes;
    at_tile = source_of<BIG>(p, u, pos + NEXT, page[1]);  // (one that is not there reads page 0)
    page[1] = page_of_lane<BIG>(p, u, pos + 2 * NEXT);
    take_tile<DT, DP, RB, BIG>(p, u, pos + kTile > plain || holes, pos, holes, at_tile, tile, rows, query, x, pairs);
  }
  if (missing && lane == 0) fault(p, KVC_FAULT_PAGE);
  if (u.t0 >= seen && p.pieces > 1) return;  // the join does not look for it

  // Results go through LDS, so that a row's are written side by side; waves along the tokens are joined there.
  put_sums<DP, 1>(x, lds.of[wave].sums, lds.m[wave], lds.l[wave]);
  if constexpr (LONE) {
    __builtin_amdgcn_wave_barrier();
    write_rows<DT, DP, 16, 1, 64>(p, shared, at_work, q, new_tokens, base_row, &lds.of[wave].sums, &lds.m[wave], &lds.l[wave], lane);
  } else {
    __syncthreads();
    write_rows<DT, DP, 16, 4, 256>(p, shared, at_work, q, new_tokens, base_row, &lds.of[0].sums, lds.m, lds.l, threadIdx.x);
  }
}

// ---- many rows ------------------------------------------------------------------------------------------------------------
//
// Four waves side by side along the rows, 32 each, take the same tiles.  What a tile's codes become as operands is made once: each wave makes a quarter of it,
// for the tile after the present one, into LDS, where an operand's 16 bytes a lane lie side by side.  One barrier a tile.
// Scores and products, which take turns in a wave, bound it (scale, shift, exp2, rounding, a sum: vector instructions are issued nearly half of the time, the matrix unit is busy 34 %), and
// reads of LDS are not far behind (79 instructions a wave and tile, most of 16 bytes a lane, which take 8 cycles each: 80 %): 10 000 rows of 128 over 32K tokens of 8 heads 1.73 ms, 782
// TFLOP/s; fp16, whose weights are two numbers, 2.2 ms.  Two workgroups a CU (69 KB of LDS, 252 registers) let one's products run beside the other's scores; waves in products go first (1765 -> 1745 us).  Of heads of
// more than 128 one fits (135 KB, sums of 128 registers), whose phases take turns.

template <int DP>
struct Made {
  u32x4 k[4][Sizes<DP>::KS][64];                       // operands of keys
  u32x4 v[2][Sizes<DP>::VS][Sizes<DP>::NJ][64];        // and of values
  PairSpace pairs;
};

constexpr int kRB = 2;  // blocks of 16 rows of a wave

template <int DP>
struct BlockLds {
  union {
    Made<DP> made[2];
    float sums[4][16 * kRB][DP];
  };
  float m[4][16 * kRB], l[4][16 * kRB];
  uint32_t most[4], seen[4];
};

// A wave's share of a tile's loads: keys' vectors, words of values of two quads, pairs.
template <int DP>
struct Share {
  static constexpr int KE = DP > 128 ? 2 : 1;
  u32x4 k[KE], v[Sizes<DP>::VS][2];
  uint32_t kp, vp;
};

template <int DP, bool BIG>
__device__ __forceinline__ void load_share(const AttendParams& p, const Unit<BIG>& u, const Source<BIG>& from, uint32_t wave, Share<DP>& t) {
  const uint32_t lane = threadIdx.x & 63u, quad = lane & 15u, g = lane >> 4, W = p.D / 8;
  const auto pair = of_lane(lane / 4, from.pairs) + (lane & 3u) * 4;
  t.kp = *(const uint32_t KVC_GLOBAL*)(u.pairs + pair);
  t.vp = *(const uint32_t KVC_GLOBAL*)(u.pairs + u.values + pair);
#pragma unroll
  for (int i = 0; i < Share<DP>::KE; ++i) {
    const uint32_t e = DP == 64 ? wave & 1u : wave * Share<DP>::KE + i;
    t.k[i] = *(const u32x4 KVC_GLOBAL*)(u.codes + (from.codes + min(e * 4 + g, W - 1) * 16));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto at = of_lane(g * 4 + (wave >> 1) * 2 + i, from.codes);
#pragma unroll
    for (int s = 0; s < Sizes<DP>::VS; ++s)
      t.v[s][i] = *(const u32x4 KVC_GLOBAL*)(u.codes + u.values + (at + min(DP == 64 ? quad & 7u : quad + 16 * s, W - 1) * 16));
  }
}

// Makes a wave's share of a tile's operands.  there: token `lane` is the part's own.
template <int DT, int DP>
__device__ __forceinline__ void make_share(const Share<DP>& t, uint32_t wave, bool there, float unit, Made<DP>& to) {
  const uint32_t lane = threadIdx.x & 63u, h = wave >> 1;
  if (wave == 0) put_key_pair<DT>(to.pairs, lane, there ? t.kp : 0, unit);
  if (wave == 1) put_value_pair<DT>(to.pairs, lane, there ? t.vp : 0, there);
  const uint64_t flat = flat_tokens<DT>(t.vp);
#pragma unroll
  for (int i = 0; i < Share<DP>::KE; ++i) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (DP == 64) {
        if ((uint32_t)k >> 1 == h) to.k[k][wave & 1u][lane] = key_operand(t.k[0][k]);
      } else {
        to.k[k][wave * Share<DP>::KE + i][lane] = key_operand(t.k[i][k]);
      }
    }
  }
#pragma unroll
  for (int s = 0; s < Sizes<DP>::VS; ++s) {
    u32x4 y = t.v[s][0], z = t.v[s][1];
    if (flat) {  // (codes that their scale makes nothing of)
      const uint32_t mine = (uint32_t)(flat >> (16 * (lane >> 4) + 8 * h));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        y[k] = mine >> k & 1u ? 0u : y[k];
        z[k] = mine >> (4 + k) & 1u ? 0u : z[k];
      }
    }
    if constexpr (DP == 64) {
      const u32x4 both = halves(y, z, (lane & 8u) ? kHigh : kLow);
#pragma unroll
      for (int n = 0; n < 4; ++n)
        if ((uint32_t)n >> 1 == (wave & 1u)) to.v[h][s][n][lane] = value_operand(both, n);
    } else {
      const u32x4 both = halves(y, z, (wave & 1u) ? kHigh : kLow);
#pragma unroll
      for (int n = 0; n < 4; ++n) to.v[h][s][2 * n + (wave & 1u)][lane] = value_operand(both, n);
    }
  }
}

constexpr int kAhead = 2;  // pairs of operands that are read before the products that take them

// The first pairs of a tile's operands of keys.
template <int DP>
__device__ __forceinline__ void read_first(const Made<DP>& made, u32x4 (&a)[kAhead + 1][2]) {
#pragma unroll
  for (int n = 0; n < kAhead; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) a[n][i] = made.k[2 * n / Sizes<DP>::KS][2 * n % Sizes<DP>::KS + i][threadIdx.x & 63u];
}

// A tile that has been made.  Operands are read from LDS some products ahead of those that take them; the order is the source's.  ask(): a call in between.
template <int DT, int DP, typename Ask>
__device__ __forceinline__ void take_made(bool masked, uint32_t at, uint32_t t1, uint32_t missing, const Made<DP>& made, const Rows<kRB>& rows,
                                          const u32x4 (&query)[kRB][Sizes<DP>::KS], State<DP, kRB>& x, u32x4 (&a)[kAhead + 1][2], Ask ask) {
  using S = Sizes<DP>;
  constexpr int KS = S::KS, NV = S::VS * S::NJ, RING = kAhead + 1;
  const uint32_t lane = threadIdx.x & 63u;
  f32x4 s[kRB][4];
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int n = 0; n < 2 * KS; ++n) {
    const int k = 2 * n / KS, first = 2 * n % KS, m = n + kAhead;
    if (m < 2 * KS) {
#pragma unroll
      for (int i = 0; i < 2; ++i) a[m % RING][i] = made.k[2 * m / KS][2 * m % KS + i][lane];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < kRB; ++b) s[b][k] = product(a[n % RING][i], query[b][first + i], first + i ? s[b][k] : f32x4{0, 0, 0, 0});
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
  ask();
  __builtin_amdgcn_sched_barrier(0);
  u32x4 w[kRB][2], fine[kRB][2];
#pragma unroll
  for (int b = 0; b < kRB; ++b) {
    if (b == kRB - 1) {
#pragma unroll
      for (int n = 0; n < kAhead; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) a[n][i] = ((const u32x4(*)[64])made.v)[2 * n + i][lane];
    }
    weights<DT, DP, kRB>(masked, at, t1, missing, made.pairs, rows, b, s[b], x, w[b], fine[b]);
  }
  const u32x4(*const values)[64] = (const u32x4(*)[64])made.v;
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int n = 0; n < NV; ++n) {
    const int h = 2 * n / NV, first = 2 * n % NV, m = n + kAhead;
    if (m < NV) {
#pragma unroll
      for (int i = 0; i < 2; ++i) a[m % RING][i] = values[2 * m + i][lane];
    }
    if (first == 0) {
      const u32x4 rows_of_sums = sums_operand(made.pairs, h);
#pragma unroll
      for (int b = 0; b < kRB; ++b) {
        x.total[b] = product(rows_of_sums, w[b][h], x.total[b]);
        if constexpr (DT == KVC_F16) x.total[b] = product(rows_of_sums, fine[b][h], x.total[b]);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int b = 0; b < kRB; ++b) {
        f32x4& sum = x.sum[b][(first + i) / S::NJ][(first + i) % S::NJ];
        sum = product(a[n % RING][i], w[b][h], sum);
        if constexpr (DT == KVC_F16) sum = product(a[n % RING][i], fine[b][h], sum);
      }
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_setprio(0);
}

// One unit: 128 rows x head x piece of the tokens.
template <int DT, int DP, bool BIG>
__device__ __forceinline__ void attend_block(const AttendParams& p, const AttendPart& part, const bool shared, uint32_t unit, BlockLds<DP>& lds) {
  using S = Sizes<DP>;
  constexpr uint32_t ROWS = 16 * kRB;
  const uint32_t lane = threadIdx.x & 63u, wave = wave_uniform(threadIdx.x >> 6), col = lane & 15u, g = lane >> 4;
  const Place at_work = place_of_unit(p, part, shared, unit);

  Request q{};
  if (!shared) q = request_at(p, at_work.request);
  const uint32_t new_tokens = shared ? p.batch.n_new : covered(p, q);
  if (!shared && p.pieces == 1 && at_work.block == 0 && q.faults)  // (of several pieces the join writes what these rows hold)
    write_uncovered(p, q, at_work.request, at_work.head, threadIdx.x, 256);
  if (!shared && at_work.block * (4 * ROWS) >= wave_uniform(new_tokens) * p.G) {  // (a request with fewer new tokens than others)
    if (threadIdx.x == 0) fault(p, q.faults);
    return;
  }
  Unit<BIG> u;
  u.bound = shared ? p.prefix : p.most_tokens;
  u.t0 = (shared ? 0 : p.own_from) + at_work.split * part.tokens;
  u.first = shared ? 0 : p.prefix;
  u.table = p.pool.tables + (uint64_t)(shared ? p.prefix_row : wave_uniform(q.row)) * p.pool.table_len;
  uint32_t page[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) page[i] = page_of_lane<BIG>(p, u, u.t0 + i * kTile);

  const uint32_t base_row = (at_work.block * 4 + wave) * ROWS;
  const uint16_t* from[kRB];
  bool there[kRB];
  uint32_t token[kRB];
#pragma unroll
  for (int b = 0; b < kRB; ++b) {
    uint32_t t, k;
    fd_divmod(p.dG, base_row + b * 16 + col, t, k);
    there[b] = t < new_tokens;
    token[b] = (there[b] ? t : 0) + (shared ? 0 : min(q.first, p.batch.n_new - 1));
    from[b] = p.q + (int64_t)token[b] * p.q_token + (int64_t)(at_work.head * p.G + k) * p.q_head;
  }
  place_of_head(p, at_work.head, u);
  u.t1 = shared ? prefix_there(p) : min(wave_uniform(q.len), p.most_tokens);
  if (shared && u.t1 < p.prefix && threadIdx.x == 0) fault(p, KVC_FAULT_LIST);
  u.t1 = min(u.t1, at_work.split + 1 < part.splits ? u.t0 + part.tokens : ~0u);  // (the prefix's last piece has its last tokens too)
  // (a tile that is not there is read from page 0)
  Share<DP> share;
  Source<BIG> source = source_of<BIG>(p, u, u.t0, page[0]);
  uint32_t holes = source.missing, next_holes;  // of the present tile and the next one
  load_share<DP, BIG>(p, u, source, wave, share);

  // How far the rows see.
  Rows<kRB> rows;
  uint32_t most = 0, least = ~0u;
#pragma unroll
  for (int b = 0; b < kRB; ++b) {
    Request r = q;
    if (shared) r = request_at(p, request_of(p.batch, token[b]));
    if (shared ? there[b] && at_work.split == 0 && at_work.head == 0 && g == 0 : threadIdx.x == 0 && b == 0) fault(p, r.faults);
    rows.limit[b] = there[b] ? limit_of(p, r, token[b]) : 0;
    most = max(most, rows.limit[b]);
    if (there[b]) least = min(least, rows.limit[b]);
  }
  lanes_see(most, least);
  most = wave_uniform(most), least = wave_uniform(least);
  u32x4 query[kRB][S::KS];
  uint32_t largest = load_queries<DT, DP, kRB>(p, from, query, rows);
  if (lane == 0) lds.most[wave] = largest, lds.seen[wave] = most;
  meet();
  largest = wave_uniform(max(max(lds.most[0], lds.most[1]), max(lds.most[2], lds.most[3])));
  const uint32_t seen = min(u.t1, wave_uniform(max(max(lds.seen[0], lds.seen[1]), max(lds.seen[2], lds.seen[3]))));
  const uint32_t end = seen > u.first ? seen : 0;  // (a quad that has none of the part's tokens is not looked at)
  const uint32_t mine = min(u.t1, most), plain = min(least, u.t1);
  make_queries<DT, DP, kRB>(p, largest, query, rows);

  State<DP, kRB> x;
#pragma unroll
  for (int b = 0; b < kRB; ++b) {
    x.m[b] = there[b] ? kNone : 0.0f;  // (a row that is not there asks for no base)
    x.l[b] = 0.0f;
    x.total[b] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < S::VS; ++v)
#pragma unroll
      for (int j = 0; j < S::NJ; ++j) x.sum[b][v][j] = f32x4{0, 0, 0, 0};
  }
  uint32_t missing = 0;
  if (u.t0 < end) make_share<DT, DP>(share, wave, u.t0 + lane >= u.first, rows.unit, lds.made[0]);
  source = source_of<BIG>(p, u, u.t0 + kTile, page[1]);
  next_holes = source.missing;
  load_share<DP, BIG>(p, u, source, wave, share);
  uint32_t turn = 0;
#pragma unroll 1
  for (uint32_t pos = u.t0; pos < end; pos += kTile, turn ^= 1u) {
    const Made<DP>& now = lds.made[turn];
    meet();  // what is in `now` is there, and the other one has been read
    u32x4 first[kAhead + 1][2];
    read_first<DP>(now, first);
    if (pos + kTile < end) make_share<DT, DP>(share, wave, true, rows.unit, lds.made[turn ^ 1u]);
    __builtin_amdgcn_sched_barrier(0);
    missing |= holes;
    auto ask = [&]() {
      source = source_of<BIG>(p, u, pos + 2 * kTile, page[2]);
      load_share<DP, BIG>(p, u, source, wave, share);
      page[2] = page_of_lane<BIG>(p, u, pos + 3 * kTile);
    };
    // (with one wave a SIMD a wave that has seen all of its tokens would wait for the others; a branch around its sums has them all moved between registers)
    if (DP <= 128 && pos >= mine) ask();
    else take_made<DT, DP>(pos + kTile > plain || holes, pos, u.t1, holes, now, rows, query, x, first, ask);
    holes = next_holes;
    next_holes = source.missing;
  }
  if (missing && threadIdx.x == 0) fault(p, KVC_FAULT_PAGE);
  if (u.t0 >= seen && p.pieces > 1) return;  // the join does not look for it
  meet();  // the sums lie where the operands were
  put_sums<DP, kRB>(x, lds.sums[wave], lds.m[wave], lds.l[wave]);
  __builtin_amdgcn_wave_barrier();
  write_rows<DT, DP, ROWS, 1, 64>(p, shared, at_work, q, new_tokens, base_row, &lds.sums[wave], &lds.m[wave], &lds.l[wave], lane);
}

// BLOCKS: a part has four waves side by side.
template <int DT, int DP, bool BIG, bool BLOCKS>
__global__ void __launch_bounds__(256, DP > 128 ? (BLOCKS || BIG ? 1 : 2) : BLOCKS ? 2 : 3) attend_held_kernel(AttendParams p) {
  union Both {
    Lds<DP> few;
    typename std::conditional<BLOCKS, BlockLds<DP>, uint32_t>::type many;
  };
  __shared__ __align__(16) uint8_t memory[sizeof(Both)];
  Both& lds = *reinterpret_cast<Both*>(memory);
  bool shared;
  uint32_t unit;
  if (!unit_of(p, shared, unit)) return;
  const AttendPart& part = p.part[shared ? 0 : 1];
  if constexpr (BLOCKS) {
    if (part.waves == 4) {
      attend_block<DT, DP, BIG>(p, part, shared, unit, lds.many);
      return;
    }
  }
  if (part.lone) {
    unit = unit * 4 + wave_uniform(threadIdx.x >> 6);
    if (unit < part.lone) attend_unit<DT, DP, BIG, true>(p, part, shared, unit, lds.few);
  } else {
    attend_unit<DT, DP, BIG, false>(p, part, shared, unit, lds.few);
  }
}

bool is_big(const AttendParams& p) { return (uint64_t)p.pool.num_blocks * p.pool.page_bytes >> 32; }

template <int DT, int DP>
kvc_status launch_of(const AttendParams& p, hipStream_t stream) {
  const uint32_t groups = (uint32_t)attend_groups(p);
  const bool big = is_big(p);
  const bool blocks = p.part[0].waves == 4 || p.part[1].waves == 4;
  if (groups && big && blocks) hipLaunchKernelGGL((attend_held_kernel<DT, DP, true, true>), dim3(groups), dim3(256), 0, stream, p);
  else if (groups && big) hipLaunchKernelGGL((attend_held_kernel<DT, DP, true, false>), dim3(groups), dim3(256), 0, stream, p);
  else if (groups && blocks) hipLaunchKernelGGL((attend_held_kernel<DT, DP, false, true>), dim3(groups), dim3(256), 0, stream, p);
  else if (groups) hipLaunchKernelGGL((attend_held_kernel<DT, DP, false, false>), dim3(groups), dim3(256), 0, stream, p);
  if (hipGetLastError() != hipSuccess) return KVC_ERR_RUNTIME;
  return p.pieces == 1 ? KVC_OK : launch_join(p, stream);
}

}  // namespace

namespace {


// What a part of the work takes in units of 16 or 128 rows and of so many tokens each.
struct Shape {
  uint32_t waves;  // that stand side by side along the rows: 1 or 4
  uint64_t blocks, splits, each;
  double time;  // us, roughly
};

// The times are a fit to calls of 1 to 128 requests over 50 to 32K tokens: with c workgroups to a CU a unit takes `start` and, for each token, `alone` and `shared` c times.
// (Which body is taken is worth up to a factor of two: 24 rows over 4000 tokens of 32 heads 26 us in units of 16 rows, 39 in units of 128; 10 000 rows over 32K of 8
// heads 2.00 and 1.69 ms.  How the tokens are cut: one row over 32K tokens of 8 heads in 14 or 42 pieces 27 or 22.7 us.)
Shape shape_of(const AttendParams& p, uint32_t waves, uint64_t tokens, uint64_t rows, uint64_t requests, bool joined) {
  Shape best{};
  if (tokens == 0) return best;
  const bool many = waves == 4;
  const double size = (p.D <= 64 ? 0.7 : p.D <= 128 ? 1.0 : many ? 1.3 : 1.5) * (p.dtype == KVC_F16 ? 1.0 : many ? 0.73 : 0.82), start = !many ? 4.0 : p.D <= 128 ? 3.0 : 4.5;
  const double alone = size * (many ? 0.0195 : 0.0028), shared = size * (many ? 0.0195 : 0.0034);
  const uint64_t most = p.D > 128 ? (many || is_big(p) ? 1 : 2) : many ? 2 : 3;  // workgroups to a CU
  const uint64_t step = many ? kTile : 4 * kTile, block = many ? 64 * kRB : 16;
  best.waves = waves;
  best.time = 1e300;
  best.blocks = (rows + block - 1) / block;
  const double whole = (double)best.blocks * p.H * requests, lines = (double)p.batch.n_new * p.H * p.G;
  for (uint64_t splits = 1, last = 0; splits <= 256; ++splits) {
    const uint64_t each = ((tokens + splits - 1) / splits + step - 1) / step * step, pieces = (tokens + each - 1) / each;
    if (each == last) continue;
    last = each;
    // (rows of their own are of all lengths: little more than half of the units' tokens are there)
    const double units = whole * pieces * (requests > 1 ? 0.6 : 1.0), slots = 256.0 * most;
    const double full = floor(units / slots), rest = units - full * slots;
    double time = full * (each * (alone + shared * most) + start);
    if (rest > 0 || full == 0) time += each * (alone + shared * ceil(rest > 0 ? rest / 256 : 1)) + start;
    if (pieces > 1 || joined) time += (joined ? 0 : 3) + lines * pieces * p.D * 8 / 6e6;  // sums of pieces, written and read
    if (time < best.time) best.time = time, best.each = each, best.splits = pieces;
  }
  return best;
}

}  // namespace

kvc_status plan_attend_held(AttendParams& p) {
  p.pieces = 0;
  p.dheads = make_fastdiv(p.H * p.G);
  p.slack = p.lift = 0.0f;
  // Tiles lie on quads of the pages: a quad that the prefix ends in is a tile's in both parts, the prefix's through its row's table and the rows' own through theirs, each
  // with its tokens alone.  The prefix's pieces are cut as if it ended where that quad begins, and the last one has what follows (128 rows of 8 heads over 515 tokens: 25.1 us
  // with a piece of 3 tokens, 22.0 so).
  p.own_from = p.prefix & ~3u;
  const uint64_t tokens[2] = {p.own_from ? p.own_from : p.prefix, p.most_tokens > p.prefix ? p.most_tokens - p.own_from : 0}, requests[2] = {1, p.batch.n_requests};
  const uint64_t rows[2] = {(uint64_t)p.batch.n_new * p.G, (uint64_t)p.batch.most_new * p.G};
  Shape few[2], many[2];
  for (int i = 0; i < 2; ++i) {
    if (tokens[i] && (rows[i] + 15) / 16 * p.H * requests[i] >> 31) return KVC_ERR_UNSUPPORTED;
    few[i] = shape_of(p, 1, tokens[i], rows[i], requests[i], tokens[1 - i] > 0);
    many[i] = rows[i] > 16 ? shape_of(p, 4, tokens[i], rows[i], requests[i], tokens[1 - i] > 0) : few[i];
    // (in a kernel that has both bodies the first one has fewer waves to a CU)
    if (few[i].time * 1.2 < many[i].time) many[i] = few[i], many[i].time *= 1.2;
  }
  const bool both = many[0].time + many[1].time < few[0].time + few[1].time;
  for (int i = 0; i < 2; ++i) {
    AttendPart& a = p.part[i];
    a = AttendPart{};
    a.drows = a.dsplits = a.drequests = make_fastdiv(1);
    if (tokens[i] == 0) continue;
    const Shape s = both ? many[i] : few[i];
    const uint64_t units = s.blocks * p.H * requests[i] * s.splits;
    if (units >> 31) return KVC_ERR_UNSUPPORTED;
    a.waves = s.waves;
    a.row_blocks = (uint32_t)s.blocks;
    a.splits = (uint32_t)s.splits;
    a.tokens = (uint32_t)s.each;
    a.units = (uint32_t)units;
    // A wave each has a unit of few tokens where there are many (64 rows of 32 heads with up to 300 tokens over a prefix of 500: 45 -> 35 us; with pieces of 1024, 128 rows
    // of 8 heads 31 -> 36, so these keep a workgroup).
    if (i == 1 && a.waves == 1 && s.each <= 512 && units >= 512) {
      a.lone = a.units;
      a.units = (a.units + 3) / 4;
    }
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
