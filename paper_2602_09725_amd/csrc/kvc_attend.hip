// Attention of a batch over paged rows that share their first tokens (kvc_attend_paged).
//
// Of a query row (a token and one of the G query heads of a KV head) with s_j = q . k_j, the result is
//   out = sum_j w_j v_j / sum_j w_j,  w_j = exp2(scale_log2 * (s_j - m)),  m any number near the largest s_j,
// and results over disjoint sets of tokens join by their m and sums.  So the work is cut into pieces: the shared prefix is
// one sequence for the rows of all requests (read once for 32 or 128 of them), each row's own tokens another for the rows
// of its request, and both are cut along the tokens until the chip is full.  A second, small launch joins the pieces.  Where many new tokens
// meet a short prefix the pieces' sums would be most of the work: then each row's tokens are one sequence, the prefix's and its own.
//
// A wave holds 32 rows.  It computes S^T = K Q^T and O^T += V^T W^T with 32x32x16 matrix instructions, so that a lane has
// one row (lane % 32) in all of its registers: the softmax needs one exchange between the halves of a wave for a
// maximum, and W^T leaves the first product in the order that the second one takes, if V's tokens are taken in
// the same order: lanes 0-31 hold tokens {0..3, 8..11}, lanes 32-63 {4..7, 12..15} of 16.  V^T comes from V's rows in LDS by
// transposing reads.
#include <hip/hip_runtime.h>

#include "kvc_attend.h"
#include "kvc_device.h"
#include "kvc_serve.h"

namespace kvc {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define KVC_LDS __attribute__((address_space(3)))

template <int DT>
__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (DT == KVC_F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Values of a lane and of its partner 32 lanes away.
__device__ __forceinline__ float half_max(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// ---- tiles ----------------------------------------------------------------------------------------------------------------

// Where the 16-byte vector `chunk` of a token's row lies in the row in LDS, whose 64 banks hold 16 such vectors.  Reads of K take one chunk of 16
// tokens that follow one another at a time, transposing reads of V four chunks of four tokens: both find them in different banks.
template <int CH>
__device__ __forceinline__ uint32_t place(uint32_t token, uint32_t chunk) {
  if constexpr (CH >= 16) return chunk ^ ((token & 3u) << 2 | ((token >> 2) & 3u));
  else return chunk ^ (((token >> 1) & 1u) << 2 | ((token >> 2) & 3u));  // (two rows lie side by side)
}

template <int DT>
__device__ __forceinline__ bool not_finite(uint32_t w) {
  const uint32_t e = DT == KVC_F16 ? 0x7c00u : 0x7f80u;
  return (w & e) == e || ((w >> 16) & e) == e;
}

// Bits 15 and 31: which of the two values of a word are not finite.
template <int DT>
__device__ __forceinline__ uint32_t wild_bits(uint32_t w) {
  return DT == KVC_F16 ? (w & 0x7c007c00u) + 0x04000400u : (w & 0x7f807f80u) + 0x00800080u;
}

// The two values of a word, 0 in the place of those that are not finite.
template <int DT>
__device__ __forceinline__ uint32_t only_finite(uint32_t w) {
  const uint32_t e = DT == KVC_F16 ? 0x7c00u : 0x7f80u;
  if ((w & e) == e) w &= 0xffff0000u;
  if (((w >> 16) & e) == e) w &= 0xffffu;
  return w;
}

// Sizes of a body: R waves side by side along the rows; tokens of a tile; vectors of a tile's K (and V).
template <int DP, int R>
struct Shape {
  static constexpr int CH = DP / 8;                          // vectors of a token's row
  static constexpr int TT = R == 1 ? 32 : 64;                // tokens of a tile
  static constexpr int GROUPS = 4 / R;                       // waves along the tokens, each with tiles of its own
  static constexpr int LOADS = TT * CH / (R * 64);           // vectors of K (and of V) that a thread loads
  static constexpr int STEP = R * 64 / CH;                   // tokens from one of them to the next
  static constexpr int TILE = TT * CH;                       // vectors of a tile
};

// LDS of a workgroup: four arrays of this many vectors, so that the compiler sees which reads a load does not touch.  Four waves
// side by side have the K and V of two tiles in them, single waves the K of two waves in each of the first two and the V in
// the others; in the end each wave its sums.
template <int DP>
constexpr int quarter() {
  constexpr int a = Shape<DP, 4>::TILE, b = 2 * Shape<DP, 1>::TILE, c = 32 * DP / 4;
  return a > b ? (a > c ? a : c) : (b > c ? b : c);
}

struct Lds {
  u32x4 KVC_LDS *a, *b, *c, *d;
  __device__ __forceinline__ u32x4 KVC_LDS* of(uint32_t i) const { return i == 0 ? a : i == 1 ? b : i == 2 ? c : d; }
};

struct Tops {
  float m[4][32], l[4][32];
  uint32_t most[4], least[4];
};

// What a wave knows of its unit.
struct Unit {
  const uint8_t KVC_GLOBAL *keys, *values;  // of the head: slot 0
  const int32_t* table;
  uint32_t span;           // bytes from there to the end of the layer's keys (and values), if they fit
  uint32_t t0, t1, bound;  // tokens of the unit that are there; none that the host knows of lies at or beyond `bound`
  uint32_t limit, least;   // those below `limit` are seen by the lane's row, below `least` by all of them
  bool bad_pages;          // a page outside the pool has been met: an error of the caller's, and only then looked for token by token
  bool page_fault;
  // Four waves side by side may have the prefix before a row's own tokens: those below `front` are read through this table, and are there below `known`.
  const int32_t* front_table;
  uint32_t front, known;
};

// Page of a position, and whether it is one of the prefix's that are not there.
template <int TT>
__device__ __forceinline__ uint32_t page_of(const AttendParams& p, const Unit& u, uint32_t pos) {
  const int32_t* table = u.table;
  if (TT == 64 && pos < u.front) table = u.front_table;
  return (uint32_t)table[fd_div(p.pool.dbs, pos)];
}
template <int TT>
__device__ __forceinline__ bool in_hole(const Unit& u, uint32_t pos) { return TT == 64 && pos < u.front && pos >= u.known; }

// Running state of a lane's row: a number near the largest product so far, sum of this half's weights, sums of values.
template <int DP>
struct State {
  float m, l;
  f32x16 sum[DP / 32];
};

// Waits until at most LEFT of the wave's loads are on their way.  (The builtin, which the compiler takes into account: it adds no wait
// of its own then for loads that the wave has waited for.)
template <int LEFT>
__device__ __forceinline__ void wait_loads() {
  static_assert(LEFT < 64, "six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (LEFT & 15) | (LEFT >> 4) << 14);
  asm volatile("" ::: "memory");
}

// Page of token lane % TT of the tile at position `at`, if it is there.  (Always one load: waits count it.  It lies within the table,
// and need not wait for the row's length.)
template <int TT>
__device__ __forceinline__ uint32_t page_of_lane(const AttendParams& p, const Unit& u, uint32_t at) {
  const uint32_t pos = at + (threadIdx.x & (uint32_t)(TT - 1));
  return page_of<TT>(p, u, min(pos, u.bound - 1));
}

// What has been loaded is not looked at before this point, so that no wait is put in front of it.
__device__ __forceinline__ void from_here(uint32_t& v) { asm volatile("" : "+v"(v)); }

// Where a thread's vectors of a tile come from.  They are loaded through a descriptor of the memory, so that a vector that is not there
// reads as 0 if its offset lies beyond the end.  Offsets have 32 bits: where a layer's K is larger than that (BIG), bits 31 and up
// go into the descriptor's base, which differs from lane to lane then, and the compiler makes a loop over the bases that occur.
// (Loads by address instead, which need no such loop, have the compiler wait for all of a wave's reads of LDS where it would
// wait for the oldest.)
template <int DP, int R, bool BIG>
struct Sources {
  uint32_t at[Shape<DP, R>::LOADS];
  uint32_t base[BIG ? Shape<DP, R>::LOADS : 1];
};

template <int DP, int R, bool BIG>
__device__ __forceinline__ Sources<DP, R, BIG> sources_of(const AttendParams& p, Unit& u, uint32_t at, uint32_t page) {
  using S = Shape<DP, R>;
  const uint32_t self = R == 1 ? threadIdx.x & 63u : threadIdx.x, first = self / S::CH, lane = threadIdx.x & 63u;
  const uint32_t pos = at + (lane & (uint32_t)(S::TT - 1));
  const uint32_t slot = page * p.pool.block_size + (pos - fd_div(p.pool.dbs, pos) * p.pool.block_size);
  const bool hole = in_hole<S::TT>(u, pos), bad = (int)(page >= p.pool.num_blocks) | (int)hole, gone = pos >= u.t1;
  if (__any((int)bad & (int)!gone)) {
    u.bad_pages = true;
    u.page_fault |= __any((int)bad & (int)!gone & (int)!hole);
  }
  uint32_t offset, base = 0;
  if constexpr (BIG) {
    const uint64_t all = (uint64_t)slot * p.pool.token_bytes;
    offset = (uint32_t)all & 0x7fffffffu;
    base = (int)bad | (int)gone ? 0 : (uint32_t)(all >> 31);
  } else {
    offset = slot * p.pool.token_bytes;
  }
  if ((int)bad | (int)gone) offset = ~0u;
  Sources<DP, R, BIG> s;
  s.base[0] = 0;
#pragma unroll
  for (int i = 0; i < S::LOADS; ++i) {
    const int from = (int)(first * 4 + i * S::STEP * 4);
    const uint32_t chunk = place<S::CH>(first + i * S::STEP, self % S::CH);
    s.at[i] = __builtin_elementwise_add_sat((uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)offset), chunk * 8 < p.D ? chunk * 16 : ~0u);
    if constexpr (BIG) s.base[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)base);
  }
  return s;
}

// Loads a tile's K or V, or COUNT of a thread's vectors of it from FIRST on, from memory straight into LDS: a wave's 64 vectors of one
// instruction lie side by side there.
template <int FIRST, int COUNT, int DP, int R, bool BIG>
__device__ __forceinline__ void load_part(const Unit& u, const uint8_t KVC_GLOBAL* from, const Sources<DP, R, BIG>& s, u32x4 KVC_LDS* to) {
  const uint32_t wave = R == 1 ? 0 : wave_uniform(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < COUNT; ++i) {
    // (a row begins below bit 31, but may end above it)
    const auto memory = __builtin_amdgcn_make_buffer_rsrc((void*)(from + (BIG ? (uint64_t)s.base[BIG ? FIRST + i : 0] << 31 : 0)), 0,
                                                          BIG ? 0x80000000u + DP * 2 : u.span, 0x00027000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(memory, (void KVC_LDS*)(to + i * (R * 64) + wave * 64), 16, (int)s.at[FIRST + i], 0, 0, 0);
  }
}
template <int DP, int R, bool BIG>
__device__ __forceinline__ void load_tile(const Unit& u, const uint8_t KVC_GLOBAL* from, const Sources<DP, R, BIG>& s, u32x4 KVC_LDS* to) {
  load_part<0, Shape<DP, R>::LOADS>(u, from, s, to);
}

// V^T of dims 32 d .., tokens 16 k .. in the lane's order.
template <int CH>
__device__ __forceinline__ u32x4 values_at(const u32x4 KVC_LDS* v, int k, int d) {
  const uint32_t lane = threadIdx.x & 63u, half = lane >> 5;
  u32x4 a;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t t = k * 16 + half * 4 + ((lane & 15u) >> 2) + j * 8;
    const uint32_t dim = d * 32 + (lane & 16u) + (lane & 3u) * 4;
    const u32x4 KVC_LDS* at = v + t * CH + place<CH>(t, dim / 8);
    const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 KVC_LDS*)((const uint16_t KVC_LDS*)at + (dim & 4u))));
    a[2 * j] = w.x;
    a[2 * j + 1] = w.y;
  }
  return a;
}

// S^T of a tile.  K's vectors are read 32 tokens ahead of the products that take them: left to itself the compiler reads each one just
// before its product and waits for it.
template <int DT, int DP, int NS>
__device__ __forceinline__ void products(const u32x4 KVC_LDS* k, const u32x4 (&query)[DP / 16], f32x16 (&s)[NS]) {
  constexpr int CH = DP / 8, KK = DP / 16;
  const uint32_t lane = threadIdx.x & 63u, col = lane & 31u, half = lane >> 5;
  u32x4 f[2][KK];
#pragma unroll
  for (int e = 0; e < KK; ++e) f[0][e] = k[col * CH + place<CH>(col, e * 2 + half)];
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    __builtin_amdgcn_sched_barrier(0);
    if (n + 1 < NS) {
      const uint32_t t = (n + 1) * 32 + col;
#pragma unroll
      for (int e = 0; e < KK; ++e) f[(n + 1) & 1][e] = k[t * CH + place<CH>(t, e * 2 + half)];
    }
    s[n] = mfma<DT>(f[n & 1][0], query[0], f32x16{});
#pragma unroll
    for (int e = 1; e < KK; ++e) s[n] = mfma<DT>(f[n & 1][e], query[e], s[n]);
  }
}

// -inf in the place of products that the lane's row does not see, in 32 tokens at position `at`.  TT: of a tile of the body.
template <int TT>
__device__ __forceinline__ void mask(const AttendParams& p, const Unit& u, uint32_t at, f32x16& s) {
  const uint32_t lane = threadIdx.x & 63u, half = lane >> 5;
  const int32_t seen = (int32_t)(min(u.limit, u.t1) - at - half * 4);  // (below 2^31 each)
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if ((i / 4) * 8 + i % 4 >= seen) s[i] = kNone;
  if (u.bad_pages) {
    const uint32_t pos = at + (lane & 31u);
    const bool there = !in_hole<TT>(u, pos) && page_of<TT>(p, u, min(pos, u.t1 - 1)) < p.pool.num_blocks;
    const uint32_t bits = (uint32_t)__ballot(there) >> (half * 4);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!(bits >> ((i / 4) * 8 + i % 4) & 1u)) s[i] = kNone;
  }
}

// Moves the state's base if a product exceeds it by too much; top: the largest of the lane's.  (The number subtracted need not be the
// maximum: as long as no weight exceeds 2^8, or 2^15 of fp16, sums and types hold them as well.  fp16 holds numbers down to 2^-24, and a weight below
// that is lost to the values' sum: so its base lies 2^7 below the product that moves it, and weights down to 2^-32 of the largest count.)
template <int DP>
__device__ __forceinline__ void move_base(const AttendParams& p, State<DP>& x, float top) {
  top = half_max(top);
  if (__any(top > x.m + p.slack)) {
    const float now = fmaxf(x.m, top - p.lift), keep = weight(x.m * p.scale_log2, now * p.scale_log2);
    x.m = now;
    x.l *= keep;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) x.sum[d][i] *= keep;
  }
}

// Weights of a tile, rounded to the type, from its products; the state is moved to them.  (The matrix unit takes 16 bits: half a step a weight, as the inputs
// themselves have.  Their sum is of the weights before that: its logarithm is a result in fp32, which rounded weights would leave with 2^-12 or 2^-9.)
template <int DT, int DP, int NS>
__device__ __forceinline__ void weights(const AttendParams& p, State<DP>& x, const f32x16 (&s)[NS], u32x4 (&w)[NS][2]) {
  float top = kNone;
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
  move_base<DP>(p, x, top);
  const float shift = x.m == kNone ? 0.0f : x.m * p.scale_log2;
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float a = __builtin_amdgcn_exp2f(fmaf(s[n][i], p.scale_log2, -shift));
      const float b = __builtin_amdgcn_exp2f(fmaf(s[n][i + 1], p.scale_log2, -shift));
      x.l += a + b;
      w[n][i / 8][(i % 8) / 2] = narrow_pair<DT>(a, b);
    }
}

template <int DT, int DP, int NS>
__device__ __forceinline__ void add_values(State<DP>& x, const u32x4 KVC_LDS* v, const u32x4 (&w)[NS][2]) {
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) x.sum[d] = mfma<DT>(values_at<DP / 8>(v, n * 2 + h, d), w[n][h], x.sum[d]);
}

// The same for a tile that not all rows see all of.  A weight of 0 does not hide an infinity: values that are not finite are kept
// out of the product, rows that see their token get them by an addition, the others not at all.
template <int DT, int DP, int NS>
__device__ __forceinline__ void add_seen_values(const Unit& u, uint32_t at, State<DP>& x, const u32x4 KVC_LDS* v, const u32x4 (&w)[NS][2]) {
  constexpr int CH = DP / 8, TT = NS * 32;
  const uint32_t lane = threadIdx.x & 63u, half = lane >> 5;
  uint32_t wild = 0;
#pragma unroll
  for (int i = 0; i < TT * CH / 64; ++i) {
    const u32x4 y = v[i * 64 + lane];
    wild |= wild_bits<DT>(y.x) | wild_bits<DT>(y.y) | wild_bits<DT>(y.z) | wild_bits<DT>(y.w);
  }
  if (!__any((wild & 0x80008000u) != 0)) {
    add_values<DT, DP, NS>(x, v, w);
    return;
  }
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        u32x4 a = values_at<CH>(v, n * 2 + h, d);
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = only_finite<DT>(a[i]);
        x.sum[d] = mfma<DT>(a, w[n][h], x.sum[d]);
      }
  for (uint32_t t = 0; t < (uint32_t)TT; ++t) {
    const bool seen = at + t < u.limit && at + t < u.t1;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t dim = d * 32 + (i / 4) * 8 + half * 4 + i % 4;
        const uint32_t y = ((const uint16_t KVC_LDS*)(v + t * CH + place<CH>(t, dim / 8)))[dim & 7u];
        if (seen && not_finite<DT>(y)) x.sum[d][i] += widen_bits<DT>(y);
      }
  }
}

// Whether a tile at position `at` has a token that is there and not seen by all rows.
template <int TT>
__device__ __forceinline__ bool hides_tokens(const Unit& u, uint32_t at) { return u.bad_pages || u.least < min(at + TT, u.t1); }

// Tokens from t0 on that are all there and seen by all rows: tiles among them need no mask.
__device__ __forceinline__ uint32_t plain_end(const Unit& u) { return max(u.t0, min(u.least, u.t1)); }

// The e-th vector of 32 tokens of K, the one that a lane has in the product.
template <int DP>
__device__ __forceinline__ u32x4 key_at(const u32x4 KVC_LDS* k, int e) {
  const uint32_t lane = threadIdx.x & 63u, col = lane & 31u, half = lane >> 5;
  return k[col * (DP / 8) + place<DP / 8>(col, (uint32_t)e * 2 + half)];
}

constexpr int kReads = 3;  // reads of LDS that are under way

// 32 tokens that all rows see all of: their products are in s, V in v; s gets the products of the 32 at k.  `first` holds K's first
// vectors, and gets those of the 32 tokens after these, at k2, if they are there by now (NEXT).  more: what is at k will be taken.  The matrix unit and the other
// ones work side by side if they are given their instructions in turn: beside each product stands some of the weights' arithmetic, and
// reads of LDS are kReads vectors ahead.  The order is the source's (left to itself the compiler makes blocks of either).
template <int DT, int DP, bool NEXT>
__device__ __forceinline__ void take_tokens(const AttendParams& p, State<DP>& x, const u32x4 (&query)[DP / 16], f32x16& s, u32x4 (&first)[kReads],
                                            const u32x4 KVC_LDS* k, const u32x4 KVC_LDS* v, const u32x4 KVC_LDS* k2, bool more) {
  constexpr int KK = DP / 16, DD = DP / 32, STEPS = 2 * DD, A = kReads;
  f32x16 next;
  u32x4 w[2], f[A + 1];
#pragma unroll
  for (int e = 0; e < A; ++e) f[e] = first[e];
  const float shift = x.m == kNone ? 0.0f : x.m * p.scale_log2;
#pragma unroll
  for (int e = 0; e < KK; ++e) {
    f[(e + A) % (A + 1)] = e + A < KK ? key_at<DP>(k, e + A) : values_at<DP / 8>(v, (e + A - KK) / DD, (e + A - KK) % DD);
    next = mfma<DT>(f[e % (A + 1)], query[e], e ? next : f32x16{});
#pragma unroll
    for (int i = e * 16 / KK; i < (e + 1) * 16 / KK; i += 2) {  // (16 / KK of them: one pair, two or a half)
      if (i % 2) continue;
      const float a = __builtin_amdgcn_exp2f(fmaf(s[i], p.scale_log2, -shift));
      const float b = __builtin_amdgcn_exp2f(fmaf(s[i + 1], p.scale_log2, -shift));
      x.l += a + b;
      w[i / 8][(i % 8) / 2] = narrow_pair<DT>(a, b);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  float top = kNone;
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    if (j + A < STEPS) f[(KK + j + A) % (A + 1)] = values_at<DP / 8>(v, (j + A) / DD, (j + A) % DD);
    else if (NEXT) first[j + A - STEPS] = key_at<DP>(k2, j + A - STEPS);
    x.sum[j % DD] = mfma<DT>(f[(KK + j) % (A + 1)], w[j / DD], x.sum[j % DD]);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i * STEPS / 16 == j) top = fmaxf(top, next[i]);
    __builtin_amdgcn_sched_barrier(0);
  }
  s = next;
  if (more) move_base<DP>(p, x, top);
}

// Four waves side by side take a tile's 64 tokens in a step.  The products run 32 tokens ahead of the values, so a step needs the K
// of its tile's second half and of the next tile's first: these two lie together in LDS, and there is one barrier a
// step, behind which stands all that it reads, and before which all has been read that its loads replace.  Each load has a whole step's time.

// The begin of the step of the tile at `at`: V of the next tile goes to v2, K of its second half and of the first half after it to k2.
// `next` holds the next tile's sources, `page` the page after it.
template <int DP, bool BIG>
__device__ __forceinline__ void begin_step(const AttendParams& p, Unit& u, uint32_t at, Sources<DP, 4, BIG>& next, uint32_t& page, u32x4 (&first)[kReads],
                                           const u32x4 KVC_LDS* k, u32x4 KVC_LDS* k2, u32x4 KVC_LDS* v2) {
  using S = Shape<DP, 4>;
  wait_loads<0>();
  meet();
#pragma unroll
  for (int e = 0; e < kReads; ++e) first[e] = key_at<DP>(k, e);
  load_tile(u, u.values, next, v2);
  load_part<S::LOADS / 2, S::LOADS / 2>(u, u.keys, next, k2);
  from_here(page);
  next = sources_of<DP, 4, BIG>(p, u, at + 2 * S::TT, page);
  load_part<0, S::LOADS / 2>(u, u.keys, next, k2 + S::TILE / 2);
  page = page_of_lane<S::TT>(p, u, at + 3 * S::TT);
}

// Rows of more than 128 elements take a wave's whole registers, half of which only matrix instructions use at once: what they use goes there.
// (Left to itself the compiler keeps the queries in memory, and reading them waits for the loads of the next tile as well.)
template <int DP>
__device__ __forceinline__ void hold(u32x4 (&query)[DP / 16], State<DP>& x) {
  if constexpr (DP > 128) {
#pragma unroll
    for (int e = 0; e < DP / 16; ++e) asm volatile("" : "+a"(query[e]));
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) asm volatile("" : "+a"(x.sum[d]));
  }
}

// A tile that all rows see all of.  s holds the products of its first half, and gets those of the next tile's.  more: these are seen by
// all rows as well.
template <int DT, int DP, bool BIG>
__device__ __forceinline__ void step_of_four(const AttendParams& p, Unit& u, uint32_t at, Sources<DP, 4, BIG>& next, uint32_t& page, u32x4 (&query)[DP / 16],
                                             State<DP>& x, f32x16& s, const u32x4 KVC_LDS* k, const u32x4 KVC_LDS* v, u32x4 KVC_LDS* k2, u32x4 KVC_LDS* v2,
                                             bool more) {
  constexpr int HALF = Shape<DP, 4>::TILE / 2;
  u32x4 first[kReads];
  hold<DP>(query, x);
  begin_step<DP, BIG>(p, u, at, next, page, first, k, k2, v2);
  take_tokens<DT, DP, true>(p, x, query, s, first, k, v, k + HALF, true);
  take_tokens<DT, DP, false>(p, x, query, s, first, k + HALF, v + HALF, nullptr, more);
}

// 32 tokens at `at` that need a mask, or come after some that do.
template <int DT, int DP>
__device__ __forceinline__ void take_masked(const AttendParams& p, const Unit& u, uint32_t at, State<DP>& x, const f32x16& products, const u32x4 KVC_LDS* v) {
  f32x16 s[1] = {products};
  u32x4 w[1][2];
  mask<64>(p, u, at, s[0]);
  weights<DT, DP, 1>(p, x, s, w);
  if (hides_tokens<32>(u, at)) add_seen_values<DT, DP, 1>(u, at, x, v, w);
  else add_values<DT, DP, 1>(x, v, w);
}

template <int DT, int DP, bool BIG>
__device__ __forceinline__ void masked_step_of_four(const AttendParams& p, Unit& u, uint32_t at, Sources<DP, 4, BIG>& next, uint32_t& page,
                                                    const u32x4 (&query)[DP / 16], State<DP>& x, f32x16& s, const u32x4 KVC_LDS* k, const u32x4 KVC_LDS* v,
                                                    u32x4 KVC_LDS* k2, u32x4 KVC_LDS* v2) {
  constexpr int HALF = Shape<DP, 4>::TILE / 2;
  u32x4 unused[kReads];
  begin_step<DP, BIG>(p, u, at, next, page, unused, k, k2, v2);
  f32x16 second[1], after[1];
  products<DT, DP, 1>(k, query, second);
  take_masked<DT, DP>(p, u, at, x, s, v);
  products<DT, DP, 1>(k + HALF, query, after);
  take_masked<DT, DP>(p, u, at + 32, x, second[0], v + HALF);
  s = after[0];
}

// One step of a wave that has its tokens to itself: the tile's K and V are in (k, v) or on their way there, the next tile's
// follow them as soon as each has been read.
template <int DT, int DP, bool BIG, bool PLAIN>
__device__ __forceinline__ void step_of_one(const AttendParams& p, Unit& u, const uint8_t KVC_GLOBAL* keys, const uint8_t KVC_GLOBAL* values, uint32_t at,
                                            uint32_t next, uint32_t& page, u32x4 (&query)[DP / 16], State<DP>& x, u32x4 KVC_LDS* k, u32x4 KVC_LDS* v) {
  using S = Shape<DP, 1>;
  constexpr int N = S::LOADS;
  f32x16 s[1];
  u32x4 w[1][2];
  hold<DP>(query, x);
  wait_loads<N>();  // K and the page are there, V may be on its way
  from_here(page);
  const Sources<DP, 1, BIG> from = sources_of<DP, 1, BIG>(p, u, at + next, page);
  products<DT, DP, 1>(k, query, s);
  wait_reads();
  load_tile(u, keys, from, k);
  asm volatile("" ::: "memory");
  page = page_of_lane<S::TT>(p, u, at + 2 * next);  // (between this line and the wait below: it is one of the loads counted there)
  if constexpr (!PLAIN) mask<S::TT>(p, u, at, s[0]);
  weights<DT, DP, 1>(p, x, s, w);
  wait_loads<N + 1>();  // V is there; the next K and its successor's page follow
  if (!PLAIN && hides_tokens<S::TT>(u, at)) add_seen_values<DT, DP, 1>(u, at, x, v, w);
  else add_values<DT, DP, 1>(x, v, w);
  wait_reads();
  load_tile(u, values, from, v);
}

// The step for tiles that need no mask.  Loads of K do not touch V: told so the compiler does not have reads of one wait for the other.
// (It keeps such notes for few loads of a kernel only; the steps with a mask go without.)
template <int DT, int DP, bool BIG>
__device__ __forceinline__ void plain_step_of_one(const AttendParams& p, Unit& u, const uint8_t KVC_GLOBAL* __restrict__ keys,
                                                  const uint8_t KVC_GLOBAL* __restrict__ values, uint32_t at, uint32_t next, uint32_t& page,
                                                  u32x4 (&query)[DP / 16], State<DP>& x, u32x4 KVC_LDS* __restrict__ k, u32x4 KVC_LDS* __restrict__ v) {
  step_of_one<DT, DP, BIG, true>(p, u, keys, values, at, next, page, query, x, k, v);
}

// The query of a row, element 16 k + 8 half of it in the k-th vector; 0 where there is none.  Returns whether there is a row, and its token.
template <int DP>
__device__ __forceinline__ bool load_query(const AttendParams& p, const Request& q, bool shared, uint32_t new_tokens, uint32_t row, uint32_t head,
                                           uint32_t& token, u32x4 (&query)[DP / 16]) {
  const uint32_t half = (threadIdx.x >> 5) & 1u;
  uint32_t t, g;
  fd_divmod(p.dG, row, t, g);
  const bool there = t < new_tokens;
  token = (there ? t : 0) + (shared ? 0 : min(q.first, p.batch.n_new - 1));
  const uint16_t* from = p.q + (int64_t)token * p.q_token + (int64_t)(head * p.G + g) * p.q_head;
#pragma unroll
  for (int k = 0; k < DP / 16; ++k) {
    const uint32_t at = k * 16 + half * 8;
    query[k] = *(const KVC_GLOBAL u32x4*)(from + (at < p.D ? at : 0));
    if (!there || at >= p.D) query[k] = u32x4{0, 0, 0, 0};
  }
  return there;
}

// From the lanes' rows to all rows of a workgroup of four waves side by side: the most and the least that one sees.
__device__ __forceinline__ void lanes_see(uint32_t& most, uint32_t& least) {
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    most = max(most, (uint32_t)__shfl_xor((int)most, d));
    least = min(least, (uint32_t)__shfl_xor((int)least, d));
  }
}
__device__ __forceinline__ void rows_see(Tops& tops, uint32_t& most, uint32_t& least) {
  const uint32_t wave = threadIdx.x >> 6;
  lanes_see(most, least);
  if ((threadIdx.x & 63u) == 0) tops.most[wave] = most, tops.least[wave] = least;
  meet();
  most = wave_uniform(max(max(tops.most[0], tops.most[1]), max(tops.most[2], tops.most[3])));
  least = wave_uniform(min(min(tops.least[0], tops.least[1]), min(tops.least[2], tops.least[3])));
}

// A wave's 32 rows of sums into LDS, in vectors of four, and their bases and sums of weights.
template <int DP>
__device__ __forceinline__ void put_sums(const AttendParams& p, const State<DP>& x, f32x4 KVC_LDS* sums, float* m, float* l) {
  constexpr uint32_t QD = DP / 4;
  const uint32_t lane = threadIdx.x & 63u, col = lane & 31u, half = lane >> 5;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t at = d * 8 + i * 2 + half;
      sums[col * QD + (at ^ (col & 15u))] = f32x4{x.sum[d][i * 4], x.sum[d][i * 4 + 1], x.sum[d][i * 4 + 2], x.sum[d][i * 4 + 3]};
    }
  const float total = half_sum(x.l);
  if (half == 0) {
    m[col] = x.m != kNone ? x.m * p.scale_log2 : total == 0.0f ? kNone : 0.0f;  // (a row that saw NaN alone is not empty)
    l[col] = total;
  }
}

// One unit: rows x head x piece of the tokens; a workgroup's, or (LONE) a wave's.
template <int DT, int DP, int R, bool BIG, bool LONE = false>
__device__ __forceinline__ void attend_unit(const AttendParams& p, const AttendPart& part, const bool shared, uint32_t unit, const Lds& lds, Tops& tops) {
  using S = Shape<DP, R>;
  constexpr int TT = S::TT, KK = DP / 16, DD = DP / 32;
  constexpr bool JOINED = R == 1 && !LONE;  // the waves of a workgroup have tokens of the same rows
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, col = lane & 31u, half = lane >> 5;
  const uint32_t speaker = LONE ? lane : threadIdx.x;

  const Place at_work = place_of_unit(p, part, shared, unit);

  // What can be asked for at once is: lists, pages, queries; then lengths; then the first tiles, and only then is worked out who sees
  // what.  (One after the other these made half of a short call's time.)
  Unit u;
  Request q{};
  if (!shared) q = request_at(p, at_work.request);
  const uint32_t new_tokens = shared ? p.batch.n_new : covered(p, q);
  if (!shared && p.pieces == 1 && at_work.block == 0 && q.faults)  // (of several pieces the join writes what these rows hold)
    write_uncovered(p, q, at_work.request, at_work.head, speaker, LONE ? 64 : 256);
  if (!shared && at_work.block * (R * 32) >= wave_uniform(new_tokens) * p.G) {  // (a request with fewer new tokens than others)
    if (speaker == 0) fault(p, q.faults);
    return;
  }
  u.bound = shared ? p.prefix : p.most_tokens;
  u.t0 = (shared ? 0 : p.own_from) + at_work.split * part.tokens;
  u.front = shared || p.own_from ? 0 : p.prefix;
  u.front_table = p.pool.tables + (uint64_t)p.prefix_row * p.pool.table_len;
  u.page_fault = false;
  u.table = p.pool.tables + (uint64_t)(shared ? p.prefix_row : wave_uniform(q.row)) * p.pool.table_len;
  constexpr uint32_t NEXT = LONE ? TT : S::GROUPS * TT;  // from a tile of a wave to its next
  const uint32_t start = u.t0 + (JOINED ? wave_uniform(wave) * TT : 0);
  uint32_t page[3];
#pragma unroll
  for (int i = 0; i < (R == 1 ? 2 : 3); ++i) page[i] = page_of_lane<TT>(p, u, start + i * NEXT);

  const uint32_t base_row = (at_work.block * R + (R == 1 ? 0 : wave)) * 32;
  uint32_t token;
  u32x4 query[KK];
  const bool there = load_query<DP>(p, q, shared, new_tokens, base_row + col, at_work.head, token, query);
  u.keys = (const uint8_t KVC_GLOBAL*)as_const(p.pool.layers)[p.layer] + (uint64_t)at_work.head * p.D * 2;
  u.values = u.keys + (uint64_t)p.pool.num_blocks * p.pool.page_bytes;
  u.span = (uint32_t)((uint64_t)p.pool.num_blocks * p.pool.page_bytes - (uint64_t)at_work.head * p.D * 2);
  if (shared) q = request_at(p, request_of(p.batch, token));
  u.t1 = shared ? prefix_there(p) : min(wave_uniform(q.len), p.most_tokens);
  u.known = u.front ? prefix_there(p) : 0;
  if ((shared ? u.t1 < p.prefix : u.known < u.front) && speaker == 0) fault(p, KVC_FAULT_LIST);
  u.t1 = min(u.t1, u.t0 + part.tokens);
  u.bad_pages = false;
  u.limit = u.least = 0;

  // The first tiles.
  const bool any = u.t0 < u.t1, has_tile = start < u.t1;
  u32x4 KVC_LDS *k0, *v0, *k1 = nullptr, *v1 = nullptr;
  Sources<DP, 4, BIG> next;
  if constexpr (R == 1) {
    const uint32_t self = wave_uniform(wave);
    if constexpr (LONE) {
      k0 = lds.of(self);  // (its sums follow there)
      v0 = k0 + S::TILE;
    } else {
      k0 = (self < 2 ? lds.a : lds.b) + (self & 1u) * S::TILE;
      v0 = (self < 2 ? lds.c : lds.d) + (self & 1u) * S::TILE;
    }
    if (has_tile) {
      const Sources<DP, 1, BIG> from = sources_of<DP, 1, BIG>(p, u, start, page[0]);
      load_tile(u, u.keys, from, k0);
      load_tile(u, u.values, from, v0);
      wait_loads<2 * S::LOADS>();  // (what has been asked for before)
    }
  } else {
    k0 = lds.a, v0 = lds.b, k1 = lds.c, v1 = lds.d;
    if (any) {
      const Sources<DP, 4, BIG> from = sources_of<DP, 4, BIG>(p, u, start, page[0]);
      next = sources_of<DP, 4, BIG>(p, u, start + TT, page[1]);
      load_part<0, S::LOADS / 2>(u, u.keys, from, k1 + S::TILE / 2);
      load_part<S::LOADS / 2, S::LOADS / 2>(u, u.keys, from, k0);
      load_tile(u, u.values, from, v0);
      load_part<0, S::LOADS / 2>(u, u.keys, next, k0 + S::TILE / 2);
      wait_loads<5 * S::LOADS / 2>();
    }
  }

  // How far the rows see.
  if (shared ? there && at_work.split == 0 && at_work.head == 0 && half == 0 : speaker == 0) fault(p, q.faults);
  u.limit = there ? limit_of(p, q, token) : 0;
  uint32_t most = u.limit, least = there ? u.limit : ~0u;
  if constexpr (R == 1) lanes_see(most, least);
  else rows_see(tops, most, least);
  u.least = wave_uniform(least);
  const uint32_t end = min(u.t1, wave_uniform(most)), plain = min(plain_end(u), end);

  State<DP> x;
  x.m = kNone;
  x.l = 0.0f;
#pragma unroll
  for (int d = 0; d < DD; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) x.sum[d][i] = 0.0f;
  uint32_t pos = start;
  if constexpr (R == 1) {
    for (; pos + TT <= plain && !u.bad_pages; pos += NEXT) plain_step_of_one<DT, DP, BIG>(p, u, u.keys, u.values, pos, NEXT, page[1], query, x, k0, v0);
    for (; pos < end; pos += NEXT) step_of_one<DT, DP, BIG, false>(p, u, u.keys, u.values, pos, NEXT, page[1], query, x, k0, v0);
  } else {
    f32x16 s[1];
    wait_loads<2 * S::LOADS>();  // K of the first 32 tokens
    meet();
    products<DT, DP, 1>(k1 + S::TILE / 2, query, s);
    if (pos + TT <= plain && !u.bad_pages) {
      float top = s[0][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[0][i]);
      move_base<DP>(p, x, top);
      // (whether a page is bad is known two tiles ahead)
      for (; pos + 2 * TT <= plain && !u.bad_pages; pos += 2 * TT) {
        step_of_four<DT, DP, BIG>(p, u, pos, next, page[2], query, x, s[0], lds.a, lds.b, lds.c, lds.d, true);
        // (the first step has seen the pages of the tile whose products the second one begins)
        step_of_four<DT, DP, BIG>(p, u, pos + TT, next, page[2], query, x, s[0], lds.c, lds.d, lds.a, lds.b, pos + 3 * TT <= plain && !u.bad_pages);
      }
      if (pos + TT <= plain && !u.bad_pages) {
        step_of_four<DT, DP, BIG>(p, u, pos, next, page[2], query, x, s[0], lds.a, lds.b, lds.c, lds.d, false);
        pos += TT;
        k0 = lds.c, v0 = lds.d, k1 = lds.a, v1 = lds.b;
      }
    }
    for (; pos < end; pos += TT) {
      masked_step_of_four<DT, DP, BIG>(p, u, pos, next, page[2], query, x, s[0], k0, v0, k1, v1);
      u32x4 KVC_LDS* const k2 = k0;
      u32x4 KVC_LDS* const v2 = v0;
      k0 = k1, v0 = v1;
      k1 = k2, v1 = v2;
    }
  }
  wait_loads<0>();  // (of tiles that nobody reads: they may not land on the sums, nor after the workgroup's end)
  if (u.page_fault && lane == 0) fault(p, KVC_FAULT_PAGE);
  if (u.t0 >= end && p.pieces > 1) return;  // the join does not look for it
  // Results: sums go through LDS, so that a row's are written side by side; waves along the tokens are joined there.
  if constexpr (LONE) wait_reads();
  else __syncthreads();
  f32x4 KVC_LDS* const mine = (f32x4 KVC_LDS*)lds.of(wave_uniform(wave));
  put_sums<DP>(p, x, mine, tops.m[wave], tops.l[wave]);
  if constexpr (LONE) wait_reads();
  else __syncthreads();
  constexpr uint32_t QD = DP / 4;                         // vectors of four sums of a row
  constexpr uint32_t SIDE = 64 / QD == 0 ? 1 : 64 / QD;  // rows that a wave writes at a time
  constexpr uint32_t MINE = JOINED ? 8 : 32;             // rows that it writes in all
  constexpr int PARTS = JOINED ? 4 : 1;                  // waves that have a sum of a row
  // A lane knows where its row goes and what the waves' sums of it weigh; those who write it ask the lane.
  float share[PARTS];  // below 0: the wave saw nothing
  uint64_t to = 0;
  {
    float m[PARTS], top = kNone, total = 0.0f;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) m[k] = tops.m[JOINED ? k : wave][col], top = fmaxf(top, m[k]);
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      share[k] = JOINED ? weight(m[k], top) : 1.0f;
      total += share[k] * tops.l[JOINED ? k : wave][col];
    }
    const float y = p.pieces > 1 ? 1.0f : total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int k = 0; k < PARTS; ++k) share[k] = m[k] == kNone ? -1.0f : share[k] * y;
    uint32_t t, g;
    fd_divmod(p.dG, base_row + col, t, g);
    if (t < new_tokens) {
      const uint32_t at_token = shared ? t : q.first + t, head = at_work.head * p.G + g;
      const uint32_t piece = shared ? at_work.split : p.part[0].splits + at_work.split;
      const uint64_t slot = ((uint64_t)piece * p.batch.n_new + at_token) * (p.H * p.G) + head;
      to = p.pieces > 1 ? (uint64_t)(p.sums + slot * p.D) : (uint64_t)(p.out + (int64_t)at_token * p.o_token + (int64_t)head * p.o_head);
      if (half == 0 && (!JOINED || wave == 0)) {
        if (p.pieces > 1) *(KVC_GLOBAL f32x2*)(p.tops + slot * 2) = f32x2{top, total};
        else if (p.lse) p.lse[slot] = total == 0.0f ? kNone : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
      }
    }
  }
  const uint32_t begin = JOINED ? wave * 8 : 0, at = lane % QD;
  const uint32_t rows = LONE ? min(MINE, wave_uniform(new_tokens) * p.G - base_row) : MINE;
#pragma unroll LONE ? 1 : 8
  for (uint32_t i = 0; i < rows; i += SIDE) {
    const uint32_t r = begin + i + lane / QD;
    auto of_row = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_ds_bpermute((int)(r * 4), (int)v); };
    uint8_t* const there_to = (uint8_t*)((uint64_t)of_row((uint32_t)(to >> 32)) << 32 | of_row((uint32_t)to));
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      const float x = __builtin_bit_cast(float, of_row(__builtin_bit_cast(uint32_t, share[k])));
      const f32x4 v = (JOINED ? (const f32x4 KVC_LDS*)lds.of(k) : (const f32x4 KVC_LDS*)mine)[r * QD + (at ^ (r & 15u))];
      if (!(x < 0.0f)) o += x * v;
    }
    if (!there_to || at * 4 >= p.D) continue;
    if (p.pieces > 1) *(KVC_GLOBAL f32x4*)(there_to + at * 16) = o;
    else *(KVC_GLOBAL u32x2*)(there_to + at * 8) = u32x2{narrow_pair<DT>(o.x, o.y), narrow_pair<DT>(o.z, o.w)};
  }
}

// ONES: neither part has four waves side by side.
template <int DT, int DP, bool BIG, bool ONES>
__global__ void __launch_bounds__(256, DP > 128 ? 1 : 2) attend_kernel(AttendParams p) {
  __shared__ u32x4 a[quarter<DP>()], b[quarter<DP>()], c[quarter<DP>()], d[quarter<DP>()];
  __shared__ Tops tops;
  const Lds lds = {(u32x4 KVC_LDS*)a, (u32x4 KVC_LDS*)b, (u32x4 KVC_LDS*)c, (u32x4 KVC_LDS*)d};
  bool shared;
  uint32_t unit;
  if (!unit_of(p, shared, unit)) return;
  const AttendPart& part = p.part[shared ? 0 : 1];
  if (part.lone) {
    unit = unit * 4 + wave_uniform(threadIdx.x >> 6);
    if (unit < part.lone) attend_unit<DT, DP, 1, BIG, true>(p, part, shared, unit, lds, tops);
  } else if (ONES || part.waves == 1) attend_unit<DT, DP, 1, BIG>(p, part, shared, unit, lds, tops);
  else if constexpr (!ONES) attend_unit<DT, DP, 4, BIG>(p, part, shared, unit, lds, tops);
}

// Joins the pieces of rows: a workgroup takes LINES rows (a token and a head), and 256 / LINES threads a row.  First the weights of all of
// its pieces are computed from their maxima, then the sums are added with many loads under way.
template <int DT, int DP, int LINES>
__global__ void __launch_bounds__(256) join_kernel(AttendParams p) {
  fetch_params<AttendParams>();
  extern __shared__ float weight_of[];  // [LINES][pieces]
  __shared__ f32x4 part[256];
  __shared__ float tops[8];
  constexpr uint32_t QD = DP / 4, EACH = 256 / LINES, SIDE = EACH / QD;  // lanes and groups of lanes of a row
  constexpr uint32_t AHEAD = 4;
  const uint32_t self = threadIdx.x % EACH, mine = threadIdx.x / EACH;
  const uint64_t lines = (uint64_t)p.batch.n_new * p.H * p.G, line = (uint64_t)blockIdx.x * LINES + mine;
  const bool there = line < lines;
  uint32_t token, head;
  fd_divmod(p.dheads, there ? (uint32_t)line : 0u, token, head);
  const uint32_t at = self % QD, group = self / QD;
  auto slot = [&](uint32_t i) { return (uint64_t)i * lines + (there ? line : 0); };
  // What the row's pieces hold is asked for before it is known which of them hold something: all are memory of the call's.
  f32x4 ahead[AHEAD];
#pragma unroll
  for (uint32_t k = 0; k < AHEAD; ++k) {
    const uint32_t i = group + k * SIDE;
    if (i < p.pieces && at * 4 < p.D) ahead[k] = *(const KVC_GLOBAL f32x4*)(p.sums + slot(i) * p.D + at * 4);
  }
  f32x2 first = {kNone, 0.0f};
  if (self < p.pieces) first = *(const KVC_GLOBAL f32x2*)(p.tops + slot(self) * 2);
  const Request q = request_at(p, request_of(p.batch, token));
  if (p.pieces == 0 && there && head == 0 && self == 0) fault(p, q.faults);  // (no other kernel has looked at it)
  const uint32_t limit = limit_of(p, q, token), prefix = min(limit, prefix_there(p));
  // pieces that hold something: those that begin below what the row sees
  // (over 4 bits the prefix's last piece may have up to three tokens more than the others)
  uint32_t a = p.part[0].splits ? min(p.part[0].splits, fd_div(p.part[0].dtokens, prefix + p.part[0].tokens - 1)) : 0;
  uint32_t n = p.part[1].splits && limit > p.own_from ? fd_div(p.part[1].dtokens, limit - p.own_from + p.part[1].tokens - 1) : 0;
  if (!there) a = n = 0;
  const uint32_t split = p.part[0].splits, end = split + n;
  auto holds = [&](uint32_t i) { return i < a || (i >= split && i < end); };
  // maxima, weights and the sum of weights: a row's threads share its pieces
  float* const w = weight_of + mine * p.pieces;
  float top = kNone, total = 0.0f;
  for (uint32_t i = self; i < p.pieces; i += EACH) {
    f32x2 t = i == self ? first : *(const KVC_GLOBAL f32x2*)(p.tops + slot(i) * 2);
    if (!holds(i)) t.x = kNone;
    w[i] = t.x;
    const float now = fmaxf(top, t.x), keep = weight(top, now);
    total = total * keep + (t.x == kNone ? 0.0f : t.y * weight(t.x, now));
    top = now;
  }
#pragma unroll
  for (uint32_t d = 1; d < (EACH < 64 ? EACH : 64); d *= 2) {
    const float m = __shfl_xor(top, d), l = __shfl_xor(total, d), now = fmaxf(top, m);
    total = (top == kNone ? 0.0f : total * weight(top, now)) + (m == kNone ? 0.0f : l * weight(m, now));
    top = now;
  }
  if constexpr (EACH > 64) {
    if ((threadIdx.x & 63u) == 0) tops[threadIdx.x / 64] = top, tops[4 + threadIdx.x / 64] = total;
    __syncthreads();
    constexpr uint32_t WAVES = EACH / 64;
    float m[WAVES], l[WAVES];
#pragma unroll
    for (uint32_t k = 0; k < WAVES; ++k) m[k] = tops[mine * WAVES + k], l[k] = tops[4 + mine * WAVES + k];
    top = kNone;
    total = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < WAVES; ++k) top = fmaxf(top, m[k]);
#pragma unroll
    for (uint32_t k = 0; k < WAVES; ++k) total += m[k] == kNone ? 0.0f : l[k] * weight(m[k], top);
  }
  for (uint32_t i = self; i < p.pieces; i += EACH) w[i] = weight(w[i], top);
  __syncthreads();
  // sums: group g of a row takes pieces g, g + SIDE, ..
  f32x4 o = {0, 0, 0, 0};
#pragma unroll
  for (uint32_t k = 0; k < AHEAD; ++k) {
    const float x = group + k * SIDE < p.pieces ? w[group + k * SIDE] : 0.0f;
    if (x != 0.0f) o += ahead[k] * x;  // (the sums of a piece that saw nothing mean nothing)
  }
  if (at * 4 < p.D) {
#pragma unroll 4
    for (uint32_t i = group + AHEAD * SIDE; i < p.pieces; i += SIDE) {
      const float x = w[i];
      const f32x4 v = *(const KVC_GLOBAL f32x4*)(p.sums + slot(i) * p.D + at * 4);
      if (x != 0.0f) o += v * x;
    }
  }
  if constexpr (SIDE > 1) {
    part[threadIdx.x] = o;
    __syncthreads();
    if (group == 0) {
#pragma unroll
      for (uint32_t k = 1; k < SIDE; ++k) o += part[threadIdx.x + k * QD];
    }
  }
  if (!there || group != 0) return;
  const float y = total == 0.0f ? 0.0f : 1.0f / total;
  if (at * 4 < p.D) {
    const u32x2 r = {narrow_pair<DT>(o.x * y, o.y * y), narrow_pair<DT>(o.z * y, o.w * y)};
    *(KVC_GLOBAL u32x2*)(p.out + (int64_t)token * p.o_token + (int64_t)head * p.o_head + at * 4) = r;
  }
  if (at == 0 && p.lse) p.lse[line] = total == 0.0f ? kNone : (top + __builtin_amdgcn_logf(total)) * 0.69314718055994531f;
}

// Rows that share a workgroup of the join.  Few rows of many pieces take a workgroup each; many rows share one, a row having as many threads as it has
// vectors of four sums (up to 128 elements, so that a workgroup's life, which is that of its loads one after the other, is spent on eight rows).
constexpr uint32_t join_lines(uint32_t D) { return D > 128 ? 4 : 8; }

template <int DT, int DP>
kvc_status join_of(const AttendParams& p, hipStream_t stream) {
  constexpr uint32_t kLines = join_lines(DP);
  const uint32_t lines = p.batch.n_new * p.H * p.G;
  if (lines <= 2048)
    hipLaunchKernelGGL((join_kernel<DT, DP, 1>), dim3(lines), dim3(256), p.pieces * 4, stream, p);
  else
    hipLaunchKernelGGL((join_kernel<DT, DP, kLines>), dim3((lines + kLines - 1) / kLines), dim3(256), p.pieces * kLines * 4, stream, p);
  return hipGetLastError() == hipSuccess ? KVC_OK : KVC_ERR_RUNTIME;
}

template <int DT, int DP>
kvc_status launch_of(const AttendParams& p, hipStream_t stream) {
  const uint32_t groups = (uint32_t)attend_groups(p);
  const bool big = (uint64_t)p.pool.num_blocks * p.pool.page_bytes > 0xffff0000u;  // (offsets of what is not there lie above)
  // Few rows have a kernel of the one body alone, with fewer registers (4 rows over 1000 tokens 14.6 -> 13.9 us, 30 rows of 32 heads over 3000 tokens 40.8 ->
  // 39.2); caches beyond 32 bits go without.
  const bool ones = p.part[0].waves <= 1 && p.part[1].waves <= 1;
  if (groups && big) hipLaunchKernelGGL((attend_kernel<DT, DP, true, false>), dim3(groups), dim3(256), 0, stream, p);
  if (groups && !big && ones) hipLaunchKernelGGL((attend_kernel<DT, DP, false, true>), dim3(groups), dim3(256), 0, stream, p);
  if (groups && !big && !ones) hipLaunchKernelGGL((attend_kernel<DT, DP, false, false>), dim3(groups), dim3(256), 0, stream, p);
  if (hipGetLastError() != hipSuccess) return KVC_ERR_RUNTIME;
  return p.pieces == 1 ? KVC_OK : join_of<DT, DP>(p, stream);  // (no piece at all: every row is empty)
}

}  // namespace

uint64_t attend_groups(const AttendParams& p) { return ((uint64_t)p.part[0].units + 7) / 8 * 8 + ((uint64_t)p.part[1].units + 7) / 8 * 8; }

bool attend_fits(const AttendParams& p) {
  const uint64_t lines = (uint64_t)p.batch.n_new * p.H * p.G, each = join_lines(p.D);
  return attend_groups(p) <= kMostGroups && (p.pieces == 1 || (lines + each - 1) / each <= kMostGroups);
}

kvc_status launch_join(const AttendParams& p, hipStream_t stream) {
  const bool half = p.dtype == KVC_F16;
  if (p.D <= 64) return half ? join_of<KVC_F16, 64>(p, stream) : join_of<KVC_BF16, 64>(p, stream);
  if (p.D <= 128) return half ? join_of<KVC_F16, 128>(p, stream) : join_of<KVC_BF16, 128>(p, stream);
  return half ? join_of<KVC_F16, 256>(p, stream) : join_of<KVC_BF16, 256>(p, stream);
}

// Whether the prefix is read anew for each request.  It costs the products of about 64 rows of a block that a request does not fill, over the
// prefix's tokens and at 900 TFLOP/s, and spares the writing and reading of a sum of each part for each row, at 4 TB/s, and the join's launch.  (Calls of 2 or 8
// requests over 60 to 500 tokens, 16 to 64 query heads: from 32 blocks of 128 rows on the sequences are 34 % faster to 13 % slower, the median 6 % faster; of 8
// to 32 blocks, where most of the gain is the launch, 25 % faster to 6 % slower, 4 %: no border shows, and these keep the pieces.)
bool one_sequence(const AttendParams& p) {
  const uint64_t rows = (uint64_t)p.batch.n_new * p.G;
  if (p.prefix == 0 || p.most_tokens == p.prefix || (uint64_t)p.batch.most_new * p.G <= 32) return false;
  return rows * p.H >= 128 * 32 && (uint64_t)p.batch.n_requests * p.prefix < 14 * rows;
}

kvc_status plan_attend(AttendParams& p) {
  p.pieces = 0;
  p.dheads = make_fastdiv(p.H * p.G);
  p.slack = 8.0f / p.scale_log2 < 1e30f ? 8.0f / p.scale_log2 : 1e30f;
  p.lift = p.dtype == KVC_F16 ? p.slack * 0.875f : 0.0f;
  p.slack += p.lift;
  const uint64_t chip = p.D <= 128 ? 512 : 256;  // workgroups that run at a time
  p.own_from = one_sequence(p) ? 0 : p.prefix;
  for (int i = 0; i < 2; ++i) {
    AttendPart& a = p.part[i];
    a = AttendPart{};
    const uint64_t tokens = i == 0 ? p.own_from : p.most_tokens - p.own_from;
    const uint64_t rows = (uint64_t)(i == 0 ? p.batch.n_new : p.batch.most_new) * p.G;
    a.waves = rows <= 32 ? 1 : 4;
    const uint64_t each_block = a.waves == 1 ? 32 : 128, blocks = (rows + each_block - 1) / each_block;
    const uint64_t whole = blocks * p.H * (i == 0 ? 1 : p.batch.n_requests);
    a.drows = a.dsplits = a.drequests = make_fastdiv(1);
    if (tokens == 0) continue;
    if (whole >> 31) return KVC_ERR_UNSUPPORTED;
    // One workgroup a CU where a piece is short (32 query heads of 8 KV heads, one or two workgroups: 8 requests over 32K tokens 34 or 39 us, over 64K 60 or
    // 65), two of them where it is long (64 requests over 64K 123 or 112 us; over 32K 73 or 69, but where the rows' own 500 tokens each take the
    // second workgroup's place 83 or 86); where more than two a CU wait, in halves if the last round would be mostly empty (79 blocks of 8 heads 1.51 ms
    // instead of 1.75).
    // Of a row's own tokens four waves side by side take pieces of 512 (19 requests of 56 heads with up to 2000 tokens each 55 or 47 us).
    const uint64_t lengthy = i == 0 && p.most_tokens > p.prefix ? 2048 : a.waves == 4 ? 256 : 1024;
    uint64_t splits = whole <= chip && tokens * whole >= lengthy * chip ? chip / whole : whole <= 256 ? 256 / whole : 1;
    if (whole > chip && tokens >= 4096 && 20 * ((whole + chip - 1) / chip) * chip > 23 * whole) splits = 2;
    uint64_t each = (tokens + splits - 1) / splits;
    const uint64_t least = 128;
    each = (each + least - 1) / least * least;
    splits = (tokens + each - 1) / each;
    if (whole * splits >> 31) return KVC_ERR_UNSUPPORTED;
    a.row_blocks = (uint32_t)blocks;
    a.splits = (uint32_t)splits;
    a.tokens = (uint32_t)each;
    a.units = (uint32_t)(whole * splits);
    // A wave each has a unit of few tokens where there are many: a workgroup's life is mostly that of memory's answers one after the other, and it has four
    // at a time so (over a prefix of 1000: 91 requests of 32 heads with up to 6 tokens 56 -> 30 us, 128 of 8 heads with up to 60 or 250: 36 -> 32, 42 -> 36, 32
    // with 20: 23.6 -> 22.6; 64 with up to 500 beside a prefix of 32K 81 -> 85, and with 1000 46 -> 53, so these keep a workgroup).
    if (i == 1 && a.waves == 1 && each <= 256 && 2 * whole * splits >= chip) {
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

kvc_status launch_attend(const AttendParams& p, hipStream_t stream) {
  const bool half = p.dtype == KVC_F16;
  if (p.D <= 64) return half ? launch_of<KVC_F16, 64>(p, stream) : launch_of<KVC_BF16, 64>(p, stream);
  if (p.D <= 128) return half ? launch_of<KVC_F16, 128>(p, stream) : launch_of<KVC_BF16, 128>(p, stream);
  return half ? launch_of<KVC_F16, 256>(p, stream) : launch_of<KVC_BF16, 256>(p, stream);
}

}  // namespace kvc
