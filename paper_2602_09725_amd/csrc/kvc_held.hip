// Pages held in 4 bits: tokens quantized as they are written, read back, and pages moved between a 16-bit pool and a 4-bit one.
//
// All of it is memory's time: 2 bytes an element on one side, half a byte and 4 bytes a token's head on the other.  A thread has one word (eight
// elements) of four tokens that follow one another in a page (a quad), 64 bytes on the wide side and 16 on the other, so that both sides are read and written in
// vectors; the threads of a head, its least and largest value known to all of them after a few exchanges, lie side by side in a wave.
#include <hip/hip_runtime.h>

#include "kvc_codes.h"
#include "kvc_device.h"
#include "kvc_serve.h"

namespace kvc {

namespace {

__device__ __forceinline__ void fault(const PoolView& p, uint32_t bits) {
  if (p.err && bits) atomicOr(p.err, bits);
}

__device__ __forceinline__ uint32_t lane_id() { return threadIdx.x & 63u; }

__device__ __forceinline__ uint8_t* page_at(const PoolView& p, uint32_t layer, uint32_t kind, uint32_t page) {
  uint8_t* base = (uint8_t*)as_const(p.layers)[layer];
  return base + ((uint64_t)kind * p.num_blocks + page) * p.page_bytes;
}

// Where a quad of a head lies in a page in 4 bits: its codes and its pairs.
__device__ __forceinline__ uint64_t codes_at(const PoolView& p, uint32_t W, uint32_t head, uint32_t slot) {
  return ((uint64_t)head * p.block_size + slot) * (W * 4);
}
__device__ __forceinline__ uint64_t pairs_at(const PoolView& p, uint32_t W, uint32_t H, uint32_t head, uint32_t slot) {
  return ((uint64_t)(H * W + head) * p.block_size + slot) * 4;
}

// A value of another lane of the row of 16.
template <int CONTROL>
__device__ __forceinline__ uint32_t of_neighbour(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, 0xf, 0xf, true);
}

// The least of P lanes, two numbers at a time, in all of them.
template <int P>
__device__ __forceinline__ s16x2 least_of(s16x2 v) {
  auto with = [&](uint32_t other) { v = __builtin_elementwise_min(v, __builtin_bit_cast(s16x2, other)); };
  if constexpr (P >= 2) with(of_neighbour<0xb1>(__builtin_bit_cast(uint32_t, v)));    // the other one of two lanes
  if constexpr (P >= 4) with(of_neighbour<0x4e>(__builtin_bit_cast(uint32_t, v)));    // of the other two of four
  if constexpr (P >= 8) with(of_neighbour<0x141>(__builtin_bit_cast(uint32_t, v)));   // the lane that lies opposite in eight
  if constexpr (P >= 16) with(of_neighbour<0x140>(__builtin_bit_cast(uint32_t, v)));  // and in sixteen
  if constexpr (P >= 32) with((uint32_t)__shfl_xor(__builtin_bit_cast(int, v), 16));
  return v;
}

// Quantizes a quad's vectors: P lanes have a head.  All lanes of a wave call it.  What a token's head is held with takes two divisions: each of
// four lanes makes that of one of the tokens, and tells the others (8500 tokens of 8 heads 16.4 -> 14.0 us).
template <int DT, int P>
__device__ __forceinline__ void quantize(const u32x4 (&v)[4], u32x4& codes, u32x4& pairs) {
  s16x2 both[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    Extremes e = {s16x2{0x7fff, 0x7fff}, s16x2{-0x8000, -0x8000}};
#pragma unroll
    for (int i = 0; i < 4; ++i) widen_to(e, as_ordered(v[k][i]));
    // the least in the low half, the most, its bits turned over, in the high one: one exchange for both
    const short low = e.low.x < e.low.y ? e.low.x : e.low.y, high = e.high.x > e.high.y ? e.high.x : e.high.y;
    both[k] = least_of<P>(s16x2{low, (short)~high});
  }
  Pair p[4];
  if constexpr (P < 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = pair_of<DT>(both[k].x, (short)~both[k].y);
  } else {
    const uint32_t mine = threadIdx.x & 3u;
    const s16x2 of = mine == 0 ? both[0] : mine == 1 ? both[1] : mine == 2 ? both[2] : both[3];
    const Pair one = pair_of<DT>(of.x, (short)~of.y);
    const uint32_t mn = __builtin_bit_cast(uint32_t, one.mn), inv = __builtin_bit_cast(uint32_t, one.inv), wild = one.wild;
    auto tell = [&](Pair& to, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
      to.mn = __builtin_bit_cast(float, a), to.inv = __builtin_bit_cast(float, b), to.bits = c, to.wild = d != 0;
    };
    tell(p[0], of_neighbour<0x00>(mn), of_neighbour<0x00>(inv), of_neighbour<0x00>(one.bits), of_neighbour<0x00>(wild));
    tell(p[1], of_neighbour<0x55>(mn), of_neighbour<0x55>(inv), of_neighbour<0x55>(one.bits), of_neighbour<0x55>(wild));
    tell(p[2], of_neighbour<0xaa>(mn), of_neighbour<0xaa>(inv), of_neighbour<0xaa>(one.bits), of_neighbour<0xaa>(wild));
    tell(p[3], of_neighbour<0xff>(mn), of_neighbour<0xff>(inv), of_neighbour<0xff>(one.bits), of_neighbour<0xff>(wild));
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    codes[k] = word_of<DT>(v[k], p[k]);
    pairs[k] = p[k].bits;
  }
}

// A request's tokens as quads of its pages: quad j of all holds the positions [4 m, 4 m + 4) of a row.
struct Quad {
  uint32_t row, position;  // of its first token
  uint32_t token;          // new token that lies there (it may be below the request's first one: taken says which are its own)
  uint32_t taken;          // bit k: the k-th token is there
  uint32_t page, slot;
};

// Request r has the quads from this one on: as many as n tokens can touch, n / 4 + 2, fit below the next one's.
__device__ __forceinline__ uint32_t first_quad(const BatchView& b, uint32_t r) { return (b.starts ? min((uint32_t)b.starts[r], b.n_new) / 4 + 2 * r : r); }

// What quads of a batch are; `first`: position of each request's first token, or null for the row's last ones.  Of a quad that has nothing, taken is 0.
// PAGED: a quad lies in one page.  Each question waits for the answer to the one before: those of all U quads are asked side by side, with indexes that
// are in range whatever the answers were.
template <bool PAGED, int U>
__device__ __forceinline__ void quads_of(const PoolView& p, const BatchView& b, const int32_t* first, const uint32_t (&j)[U], const uint32_t (&r)[U], const bool (&there)[U],
                                         bool tells, Quad (&q)[U]) {
  uint32_t from[U], n[U], bad = 0, len[U];
  int64_t begin[U], here[U], low[U], high[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    from[u] = r[u];
    n[u] = 1;
    if (b.starts) {
      const uint32_t a = (uint32_t)b.starts[r[u]], e = (uint32_t)b.starts[r[u] + 1];
      from[u] = min(a, b.n_new);
      const uint32_t end = min(e, b.n_new);
      n[u] = end > from[u] ? end - from[u] : 0;
      if (a > e || e > b.n_new || n[u] > b.most_new) bad |= KVC_FAULT_LIST;
      if ((r[u] == 0 && a != 0) || (r[u] + 1 == b.n_requests && e != b.n_new)) bad |= KVC_FAULT_LIST;
    }
    q[u].row = b.rows ? (uint32_t)b.rows[r[u]] : r[u];
    begin[u] = first ? (int64_t)first[r[u]] : 0;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool known = q[u].row < p.n_rows;
    if (!known) q[u].row = 0;
    len[u] = (uint32_t)p.lens[q[u].row];
    if (!known || len[u] > p.capacity) {
      if (there[u]) bad |= KVC_FAULT_LIST;
      n[u] = 0;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    // positions [begin, begin + covered) are asked for, those within the row are there
    if (!first) begin[u] = (int64_t)len[u] - n[u];
    const uint32_t covered = min(n[u], b.most_new);
    low[u] = begin[u] < 0 ? 0 : begin[u];
    high[u] = begin[u] + covered < (int64_t)len[u] ? begin[u] + covered : (int64_t)len[u];
    if (there[u] && n[u] && (begin[u] < 0 || begin[u] + covered > (int64_t)len[u])) bad |= KVC_FAULT_LIST;
    here[u] = (low[u] / 4 + (j[u] - first_quad(b, r[u]))) * 4;
    q[u].taken = 0;
    q[u].page = q[u].slot = 0;
    const bool some = there[u] && n[u] && here[u] < high[u];
    q[u].position = some ? (uint32_t)here[u] : 0;
    q[u].token = (uint32_t)((int64_t)from[u] + here[u] - begin[u]);
    if (some) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (here[u] + k >= low[u] && here[u] + k < high[u]) q[u].taken |= 1u << k;
    }
    if constexpr (PAGED) {
      uint32_t block;
      fd_divmod(p.dbs, q[u].position, block, q[u].slot);
      q[u].page = (uint32_t)p.tables[(uint64_t)q[u].row * p.table_len + block];
    }
  }
  if (tells) fault(p, bad);
}

// Leaves out quads on no page of the pool.
template <int U>
__device__ __forceinline__ void look_at_pages(const PoolView& p, bool tells, Quad (&q)[U]) {
  uint32_t bad = 0;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (q[u].taken && q[u].page >= p.num_blocks) {
      bad |= KVC_FAULT_PAGE;
      q[u].taken = 0;
    }
  if (tells) fault(p, bad);
}

// Request of quad j, the workgroup's first one; all threads of a wave call it.
__device__ __forceinline__ uint32_t request_of_quad(const BatchView& b, uint32_t j) {
  if (!b.starts) return j;
  uint32_t c = 0;
  for (uint32_t r = lane_id(); r < ((b.n_requests + 63) & ~63u); r += 64) c += (uint32_t)__popcll(__ballot(r < b.n_requests && first_quad(b, r) <= j));
  return c ? c - 1 : 0;
}

// A column is a kind and a head.  A thread's units are the same column of U quads that follow one another.
template <int U>
struct Column {
  uint32_t quad[U], request[U], kind, head;
  bool there[U];
};
template <int U>
__device__ __forceinline__ Column<U> column_of(const HeldParams& p, uint64_t unit, uint64_t first_unit) {
  Column<U> c;
  const uint32_t H2 = 2 * p.H;
  const uint64_t all = (uint64_t)((p.quads + U - 1) / U) * H2;
  const bool mine = unit < all;
  auto group_of = [&](uint64_t at, uint32_t& column) {
    if (all >> 31) {
      const uint32_t g = (uint32_t)(at / H2);
      column = (uint32_t)(at - (uint64_t)g * H2);
      return g;
    }
    uint32_t g;
    fd_divmod(p.dcolumns, (uint32_t)at, g, column);
    return g;
  };
  uint32_t column, unused;
  const uint32_t group = group_of(mine ? unit : first_unit, column);
  c.kind = column >= p.H;
  c.head = column - c.kind * p.H;
  uint32_t r = request_of_quad(p.batch, group_of(first_unit, unused) * U);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    c.quad[u] = group * U + u;
    c.there[u] = mine && c.quad[u] < p.quads;
    if (p.batch.starts)
      while (r + 1 < p.batch.n_requests && first_quad(p.batch, r + 1) <= c.quad[u]) ++r;
    else
      r = min(c.quad[u], p.batch.n_requests - 1);
    c.request[u] = r;
  }
  return c;
}

// Tokens of a batch to their slots: P threads have a head of U quads.
template <int DT, int P, int U>
__global__ void __launch_bounds__(256) write_kernel(HeldParams p) {
  fetch_params<HeldParams>();
  const uint64_t first = (uint64_t)blockIdx.x * (256 / P);
  const uint32_t w = threadIdx.x % P;
  const Column<U> c = column_of<U>(p, first + threadIdx.x / P, first);
  Quad q[U];
  const bool tells = w == 0 && c.kind == 0 && c.head == 0;
  quads_of<true, U>(p.pool, p.batch, nullptr, c.quad, c.request, c.there, tells, q);
  // (lanes beyond a head's words have what its first one has)
  const uint16_t* const from = (c.kind ? p.v : p.k) + (uint64_t)(c.head * p.W + (w < p.W ? w : 0)) * 8;
  u32x4 v[U][4];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[u][k] = u32x4{0, 0, 0, 0};
      if (q[u].taken >> k & 1u) v[u][k] = stream_load<u32x4>(from + (int64_t)(uint32_t)(q[u].token + k) * p.token_stride);
    }
  look_at_pages<U>(p.pool, tells, q);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    u32x4 codes, pairs;
    quantize<DT, P>(v[u], codes, pairs);
    if (w >= p.W || !q[u].taken) continue;
    uint8_t* const page = page_at(p.pool, p.layer, c.kind, q[u].page);
    uint8_t* const to = page + codes_at(p.pool, p.W, c.head, q[u].slot) + w * 16;
    uint8_t* const pair_to = page + pairs_at(p.pool, p.W, p.H, c.head, q[u].slot);
    if (q[u].taken == 15) {
      *(KVC_GLOBAL u32x4*)to = codes;
      if (w == 0) *(KVC_GLOBAL u32x4*)pair_to = pairs;
      continue;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (!(q[u].taken >> k & 1u)) continue;
      ((KVC_GLOBAL uint32_t*)to)[k] = codes[k];
      if (w == 0) ((KVC_GLOBAL uint32_t*)pair_to)[k] = pairs[k];
    }
  }
}

// A thread's unit and word of so many threads.
__device__ __forceinline__ uint64_t unit_of_thread(const HeldParams& p, uint64_t all, uint64_t at, uint32_t& w) {
  if (all >> 31) {
    const uint64_t unit = at / p.W;
    w = (uint32_t)(at - unit * p.W);
    return unit;
  }
  uint32_t unit;
  fd_divmod(p.dwords, (uint32_t)at, unit, w);
  return unit;
}

// Tokens of rows back: a thread has a word of U quads.
template <int DT, int U>
__global__ void __launch_bounds__(256) read_kernel(HeldParams p) {
  fetch_params<HeldParams>();
  const uint64_t all = (uint64_t)((p.quads + U - 1) / U) * 2 * p.H * p.W, begin = (uint64_t)blockIdx.x * 256, here = begin + threadIdx.x;
  uint32_t w, unused;
  const uint64_t unit = unit_of_thread(p, all, here < all ? here : all - 1, w);
  const Column<U> c = column_of<U>(p, unit, unit_of_thread(p, all, begin, unused));
  Quad q[U];
  const bool tells = here < all && w == 0 && c.kind == 0 && c.head == 0;
  quads_of<true, U>(p.pool, p.batch, p.first, c.quad, c.request, c.there, tells, q);
  look_at_pages<U>(p.pool, tells, q);
  if (here >= all) return;
  u32x4 codes[U], pairs[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint8_t* const page = page_at(p.pool, p.layer, c.kind, q[u].taken ? q[u].page : 0);
    codes[u] = stream_load<u32x4>(page + codes_at(p.pool, p.W, c.head, q[u].slot) + w * 16);
    pairs[u] = *(const KVC_GLOBAL u32x4*)(page + pairs_at(p.pool, p.W, p.H, c.head, q[u].slot));
  }
  uint16_t* const to = (c.kind ? p.v_out : p.k_out) + (uint64_t)(c.head * p.W + w) * 8;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (q[u].taken >> k & 1u)
        stream_store<u32x4>(to + (int64_t)(uint32_t)(q[u].token + k) * p.token_stride, values_of<DT>(codes[u][k], pairs[u][k]));
}

// The same from a pool of 16 bits: a thread has eight elements of a quad's tokens.
__global__ void __launch_bounds__(256) read_wide_kernel(HeldParams p) {
  const uint64_t all = (uint64_t)p.quads * 2 * p.H * p.W, begin = (uint64_t)blockIdx.x * 256, here = begin + threadIdx.x;
  uint32_t w, unused;
  const uint64_t unit = unit_of_thread(p, all, here < all ? here : all - 1, w);
  const Column<1> c = column_of<1>(p, unit, unit_of_thread(p, all, begin, unused));
  Quad qs[1];
  quads_of<false, 1>(p.pool, p.batch, p.first, c.quad, c.request, c.there, here < all && w == 0 && c.kind == 0 && c.head == 0, qs);
  if (here >= all) return;
  const Quad& q = qs[0];
  uint16_t* const to = (c.kind ? p.v_out : p.k_out) + (uint64_t)(c.head * p.W + w) * 8;
  uint32_t bad = 0, page[4], slot[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t block;  // (a page of any number of tokens may end inside a quad)
    fd_divmod(p.pool.dbs, q.taken >> k & 1u ? q.position + k : 0u, block, slot[k]);
    page[k] = (uint32_t)p.pool.tables[(uint64_t)q.row * p.pool.table_len + block];
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (!(q.taken >> k & 1u)) continue;
    if (page[k] >= p.pool.num_blocks) {
      bad |= KVC_FAULT_PAGE;
      continue;
    }
    const uint8_t* const from = page_at(p.pool, p.layer, c.kind, page[k]) + (uint64_t)slot[k] * p.pool.token_bytes + (uint64_t)(c.head * p.W + w) * 16;
    stream_store<u32x4>(to + (int64_t)(uint32_t)(q.token + k) * p.token_stride, stream_load<u32x4>(from));
  }
  if (w == 0 && c.head == 0 && c.kind == 0) fault(p.pool, bad);
}

// Pages between the pools: which (pair, layer and kind, quad, head) a thread's unit is.
struct PageQuad {
  uint32_t wide_page, held_page, layer, kind, slot, head;
  bool there;
};
__device__ __forceinline__ PageQuad page_quad_of(const ConvertParams& p, uint64_t unit) {
  PageQuad q;
  const uint64_t each = (uint64_t)p.H * (p.held.block_size / 4);  // units of a page, layer and kind
  const uint64_t all = each * 2 * p.held.L * p.n;
  q.there = unit < all;
  const uint64_t at = q.there ? unit : all - 1;
  uint64_t rest;
  uint32_t within;
  if (all >> 31) {
    rest = at / each, within = (uint32_t)(at - rest * each);
  } else {
    uint32_t r;
    fd_divmod(p.deach, (uint32_t)at, r, within);
    rest = r;
  }
  uint32_t pair, layer_kind, quad;
  fd_divmod(p.dkinds, (uint32_t)rest, pair, layer_kind);
  fd_divmod(p.dheads, within, quad, q.head);
  q.layer = layer_kind / 2;
  q.kind = layer_kind % 2;
  q.slot = quad * 4;
  const uint32_t from = (uint32_t)p.src[pair], to = (uint32_t)p.dst[pair];
  q.wide_page = p.back ? to : from;
  q.held_page = p.back ? from : to;
  const bool no_wide = q.wide_page >= p.wide.num_blocks, no_held = q.held_page >= p.held.num_blocks;
  if (q.there && within == 0 && layer_kind == 0) {
    if (no_wide) fault(p.wide, KVC_FAULT_PAGE);
    if (no_held) fault(p.held, KVC_FAULT_PAGE);
  }
  q.there = q.there && !no_wide && !no_held;
  return q;
}

template <int DT, int P>
__global__ void __launch_bounds__(256) convert_kernel(ConvertParams p) {
  const uint32_t w = threadIdx.x % P;
  const PageQuad q = page_quad_of(p, (uint64_t)blockIdx.x * (256 / P) + threadIdx.x / P);
  u32x4 v[4];
  const uint32_t word = w < p.W ? w : 0;  // (lanes beyond a head's words have what its first one has)
  if (q.there) {
    const uint8_t* const from = page_at(p.wide, q.layer, q.kind, q.wide_page) + (uint64_t)q.slot * p.wide.token_bytes + (q.head * p.W + word) * 16;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = stream_load<u32x4>(from + (uint64_t)k * p.wide.token_bytes);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = u32x4{0, 0, 0, 0};
  }
  u32x4 codes, pairs;
  quantize<DT, P>(v, codes, pairs);
  if (!q.there || w >= p.W) return;
  uint8_t* const page = page_at(p.held, q.layer, q.kind, q.held_page);
  *(KVC_GLOBAL u32x4*)(page + codes_at(p.held, p.W, q.head, q.slot) + w * 16) = codes;
  if (w == 0) *(KVC_GLOBAL u32x4*)(page + pairs_at(p.held, p.W, p.H, q.head, q.slot)) = pairs;
}

template <int DT>
__global__ void __launch_bounds__(256) convert_back_kernel(ConvertParams p) {
  const uint64_t first = (uint64_t)blockIdx.x * 256, unit0 = first / p.W;  // (uniform)
  uint32_t more, w;
  fd_divmod(p.dwords, (uint32_t)(first - unit0 * p.W) + threadIdx.x, more, w);
  const PageQuad q = page_quad_of(p, unit0 + more);
  if (!q.there) return;
  const uint8_t* const page = page_at(p.held, q.layer, q.kind, q.held_page);
  const u32x4 codes = stream_load<u32x4>(page + codes_at(p.held, p.W, q.head, q.slot) + w * 16);
  const u32x4 pairs = *(const KVC_GLOBAL u32x4*)(page + pairs_at(p.held, p.W, p.H, q.head, q.slot));
  uint8_t* const to = page_at(p.wide, q.layer, q.kind, q.wide_page) + (uint64_t)q.slot * p.wide.token_bytes + (q.head * p.W + w) * 16;
#pragma unroll
  for (int k = 0; k < 4; ++k) stream_store<u32x4>(to + (uint64_t)k * p.wide.token_bytes, values_of<DT>(codes[k], pairs[k]));
}

kvc_status launched() { return hipGetLastError() == hipSuccess ? KVC_OK : KVC_ERR_RUNTIME; }

// Threads that have a head: the next power of two of its words.
uint32_t threads_of(uint32_t W) {
  uint32_t P = 1;
  while (P < W) P *= 2;
  return P;
}

template <int DT, int U>
void launch_write_of(const HeldParams& p, uint32_t P, uint32_t groups, hipStream_t stream) {
  switch (P) {
    case 1: hipLaunchKernelGGL((write_kernel<DT, 1, U>), dim3(groups), dim3(256), 0, stream, p); break;
    case 2: hipLaunchKernelGGL((write_kernel<DT, 2, U>), dim3(groups), dim3(256), 0, stream, p); break;
    case 4: hipLaunchKernelGGL((write_kernel<DT, 4, U>), dim3(groups), dim3(256), 0, stream, p); break;
    case 8: hipLaunchKernelGGL((write_kernel<DT, 8, U>), dim3(groups), dim3(256), 0, stream, p); break;
    case 16: hipLaunchKernelGGL((write_kernel<DT, 16, U>), dim3(groups), dim3(256), 0, stream, p); break;
    default: hipLaunchKernelGGL((write_kernel<DT, 32, U>), dim3(groups), dim3(256), 0, stream, p); break;
  }
}

// Quads of a thread: one while that is fewer than twelve workgroups a CU; of more, whose loads the chip cannot have in flight at once, several that ask side by
// side.  8 heads of 128, one quad / several: 8500 tokens (8 workgroups a CU) written 15.7 / 15.7 us, read 14.3 / 14.3; 16 000 tokens (16 a CU) written
// 25.1 / 20.8, read 23.5 / 19.5; 160 000 tokens written 200 / 166; 32 rows of up to 8000 tokens read 177 / 132.  Two to write (with four: 16 000 tokens 24.3 us,
// 160 000 173), four to read (with two: 20.7 and 179 against 19.5 and 160).
constexpr uint32_t kQuadsRead = 4, kQuadsWritten = 2;
uint32_t quads_each(const HeldParams& p, uint32_t P, uint32_t most) { return (uint64_t)p.quads * 2 * p.H * P < 12ull * 256 * 256 ? 1 : most; }
uint64_t groups_of(const HeldParams& p, uint32_t P, uint32_t each) { return ((uint64_t)((p.quads + each - 1) / each) * 2 * p.H * P + 255) / 256; }

template <int DT>
void launch_convert_of(const ConvertParams& p, uint32_t P, uint32_t groups, hipStream_t stream) {
  switch (P) {
    case 1: hipLaunchKernelGGL((convert_kernel<DT, 1>), dim3(groups), dim3(256), 0, stream, p); break;
    case 2: hipLaunchKernelGGL((convert_kernel<DT, 2>), dim3(groups), dim3(256), 0, stream, p); break;
    case 4: hipLaunchKernelGGL((convert_kernel<DT, 4>), dim3(groups), dim3(256), 0, stream, p); break;
    case 8: hipLaunchKernelGGL((convert_kernel<DT, 8>), dim3(groups), dim3(256), 0, stream, p); break;
    case 16: hipLaunchKernelGGL((convert_kernel<DT, 16>), dim3(groups), dim3(256), 0, stream, p); break;
    default: hipLaunchKernelGGL((convert_kernel<DT, 32>), dim3(groups), dim3(256), 0, stream, p); break;
  }
}

}  // namespace

kvc_status launch_write_held(const HeldParams& p, hipStream_t stream) {
  const uint32_t P = threads_of(p.W), each = quads_each(p, P, kQuadsWritten);
  const uint64_t groups = groups_of(p, P, each);
  if (groups > kMostGroups) return KVC_ERR_UNSUPPORTED;
  if (p.dtype == KVC_F16) each == 1 ? launch_write_of<KVC_F16, 1>(p, P, (uint32_t)groups, stream) : launch_write_of<KVC_F16, kQuadsWritten>(p, P, (uint32_t)groups, stream);
  else each == 1 ? launch_write_of<KVC_BF16, 1>(p, P, (uint32_t)groups, stream) : launch_write_of<KVC_BF16, kQuadsWritten>(p, P, (uint32_t)groups, stream);
  return launched();
}

kvc_status launch_read(const HeldParams& p, hipStream_t stream) {
  const uint32_t each = p.pool.held ? quads_each(p, p.W, kQuadsRead) : 1;
  const uint64_t groups = groups_of(p, p.W, each);
  if (groups > kMostGroups) return KVC_ERR_UNSUPPORTED;
  const dim3 grid((uint32_t)groups);
  if (!p.pool.held) hipLaunchKernelGGL(read_wide_kernel, grid, dim3(256), 0, stream, p);
  else if (p.dtype == KVC_F16 && each == 1) hipLaunchKernelGGL((read_kernel<KVC_F16, 1>), grid, dim3(256), 0, stream, p);
  else if (p.dtype == KVC_F16) hipLaunchKernelGGL((read_kernel<KVC_F16, kQuadsRead>), grid, dim3(256), 0, stream, p);
  else if (each == 1) hipLaunchKernelGGL((read_kernel<KVC_BF16, 1>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((read_kernel<KVC_BF16, kQuadsRead>), grid, dim3(256), 0, stream, p);
  return launched();
}

kvc_status launch_convert(const ConvertParams& p, hipStream_t stream) {
  const uint32_t P = p.back ? p.W : threads_of(p.W);
  const uint64_t units = (uint64_t)p.H * (p.held.block_size / 4) * 2 * p.held.L;
  if (units > (kMostGroups * 256) / P || units * p.n > (kMostGroups * 256) / P || (uint64_t)p.n * 2 * p.held.L >> 31) return KVC_ERR_UNSUPPORTED;
  const uint32_t groups = (uint32_t)((units * p.n * P + 255) / 256);
  if (p.back) {
    if (p.dtype == KVC_F16) hipLaunchKernelGGL(convert_back_kernel<KVC_F16>, dim3(groups), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL(convert_back_kernel<KVC_BF16>, dim3(groups), dim3(256), 0, stream, p);
  } else {
    if (p.dtype == KVC_F16) launch_convert_of<KVC_F16>(p, P, groups, stream);
    else launch_convert_of<KVC_BF16>(p, P, groups, stream);
  }
  return launched();
}

}  // namespace kvc
