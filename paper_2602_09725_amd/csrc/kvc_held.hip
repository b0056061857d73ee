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

// Quantizes a quad's vectors: P lanes have a head.  All lanes of a wave call it.
template <int DT, int P>
__device__ __forceinline__ void quantize(const u32x4 (&v)[4], u32x4& codes, u32x4& pairs) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    Extremes e = {s16x2{0x7fff, 0x7fff}, s16x2{-0x8000, -0x8000}};
#pragma unroll
    for (int i = 0; i < 4; ++i) widen_to(e, as_ordered(v[k][i]));
    // the least in the low half, the most, its bits turned over, in the high one: one exchange for both
    const short low = e.low.x < e.low.y ? e.low.x : e.low.y, high = e.high.x > e.high.y ? e.high.x : e.high.y;
    s16x2 both = {low, (short)~high};
#pragma unroll
    for (int d = 1; d < P; d *= 2)
      both = __builtin_elementwise_min(both, __builtin_bit_cast(s16x2, __shfl_xor(__builtin_bit_cast(uint32_t, both), d)));
    const Pair p = pair_of<DT>(both.x, (short)~both.y);
    codes[k] = word_of<DT>(v[k], p);
    pairs[k] = p.bits;
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

// What quad j of a batch is; `first`: position of each request's first token, or null for the row's last ones.  Of a quad that has nothing, taken is 0.
// PAGED: a quad lies in one page.
template <bool PAGED>
__device__ __forceinline__ Quad quad_of(const PoolView& p, const BatchView& b, const int32_t* first, uint32_t j, uint32_t r, bool tells) {
  Quad q{};
  uint32_t from = r, n = 1, bad = 0;
  if (b.starts) {
    const uint32_t a = (uint32_t)b.starts[r], e = (uint32_t)b.starts[r + 1];
    from = min(a, b.n_new);
    const uint32_t end = min(e, b.n_new);
    n = end > from ? end - from : 0;
    if (a > e || e > b.n_new || n > b.most_new) bad |= KVC_FAULT_LIST;
    if ((r == 0 && a != 0) || (r + 1 == b.n_requests && e != b.n_new)) bad |= KVC_FAULT_LIST;
  }
  q.row = b.rows ? (uint32_t)b.rows[r] : r;
  const bool known = q.row < p.n_rows;
  if (!known) q.row = 0;
  const uint32_t len = (uint32_t)p.lens[q.row];
  if (!known || len > p.capacity) {
    bad |= KVC_FAULT_LIST;
    n = 0;
  }
  // positions [begin, begin + covered) are asked for, those within the row are there
  const int64_t begin = first ? (int64_t)first[r] : (int64_t)len - n;
  const uint32_t covered = min(n, b.most_new);
  const int64_t low = begin < 0 ? 0 : begin, high = begin + covered < (int64_t)len ? begin + covered : (int64_t)len;
  if (n && (begin < 0 || begin + covered > (int64_t)len)) bad |= KVC_FAULT_LIST;
  const int64_t here = (low / 4 + (j - first_quad(b, r))) * 4;
  if (n && here < high) {
    q.position = (uint32_t)here;
    q.token = (uint32_t)((int64_t)from + here - begin);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (here + k >= low && here + k < high) q.taken |= 1u << k;
    if constexpr (PAGED) {
      uint32_t block;
      fd_divmod(p.dbs, q.position, block, q.slot);
      q.page = (uint32_t)p.tables[(uint64_t)q.row * p.table_len + block];
      if (q.page >= p.num_blocks) {
        bad |= KVC_FAULT_PAGE;
        q.taken = 0;
      }
    }
  }
  if (tells) fault(p, bad);
  return q;
}

// Request of quad j, the workgroup's first one; all threads of a wave call it.
__device__ __forceinline__ uint32_t request_of_quad(const BatchView& b, uint32_t j) {
  if (!b.starts) return j;
  uint32_t c = 0;
  for (uint32_t r = lane_id(); r < ((b.n_requests + 63) & ~63u); r += 64) c += (uint32_t)__popcll(__ballot(r < b.n_requests && first_quad(b, r) <= j));
  return c ? c - 1 : 0;
}

// Threads of a workgroup that have a quad's column (a kind and a head) each, and which one a thread's is.
struct Column {
  uint32_t quad, kind, head, request;
  bool there;
};
__device__ __forceinline__ Column column_of(const HeldParams& p, uint64_t unit, uint64_t first_unit) {
  Column c;
  const uint32_t H2 = 2 * p.H, first = (uint32_t)(first_unit / H2);
  c.there = unit < (uint64_t)p.quads * H2;
  const uint64_t at = c.there ? unit : first_unit;
  uint32_t column;
  if ((uint64_t)p.quads * H2 >> 31) c.quad = (uint32_t)(at / H2), column = (uint32_t)(at - (uint64_t)c.quad * H2);
  else fd_divmod(p.dcolumns, (uint32_t)at, c.quad, column);
  c.kind = column >= p.H;
  c.head = column - c.kind * p.H;
  c.request = request_of_quad(p.batch, first);
  if (p.batch.starts)
    while (c.request + 1 < p.batch.n_requests && first_quad(p.batch, c.request + 1) <= c.quad) ++c.request;
  else
    c.request = c.quad;
  return c;
}

// Tokens of a batch to their slots: P threads have a head of a quad.
template <int DT, int P>
__global__ void __launch_bounds__(256) write_kernel(HeldParams p) {
  const uint64_t first = (uint64_t)blockIdx.x * (256 / P);
  const uint32_t w = threadIdx.x % P;
  const Column c = column_of(p, first + threadIdx.x / P, first);
  const Quad q = quad_of<true>(p.pool, p.batch, nullptr, c.quad, c.request, c.there && w == 0 && c.kind == 0 && c.head == 0);
  const bool mine = c.there && w < p.W;
  const uint16_t* const from = (c.kind ? p.v : p.k) + (uint64_t)(c.head * p.W + w) * 8;
  u32x4 v[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const bool live = mine && (q.taken >> k & 1u);
    v[k] = u32x4{0, 0, 0, 0};
    if (live) v[k] = *(const KVC_GLOBAL u32x4*)(from + (int64_t)(uint32_t)(q.token + k) * p.token_stride);
  }
  if (w >= p.W) {  // lanes beyond a head's words have what its first one has
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c.there && (q.taken >> k & 1u)) v[k] = *(const KVC_GLOBAL u32x4*)((c.kind ? p.v : p.k) + (uint64_t)c.head * p.W * 8 + (int64_t)(uint32_t)(q.token + k) * p.token_stride);
  }
  u32x4 codes, pairs;
  quantize<DT, P>(v, codes, pairs);
  if (!mine || !q.taken) return;
  uint8_t* const page = page_at(p.pool, p.layer, c.kind, q.page);
  uint8_t* const to = page + codes_at(p.pool, p.W, c.head, q.slot) + w * 16;
  uint8_t* const pair_to = page + pairs_at(p.pool, p.W, p.H, c.head, q.slot);
  if (q.taken == 15) {
    *(KVC_GLOBAL u32x4*)to = codes;
    if (w == 0) *(KVC_GLOBAL u32x4*)pair_to = pairs;
    return;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (!(q.taken >> k & 1u)) continue;
    ((KVC_GLOBAL uint32_t*)to)[k] = codes[k];
    if (w == 0) ((KVC_GLOBAL uint32_t*)pair_to)[k] = pairs[k];
  }
}

// Tokens of rows back: a thread has a word of a quad.
template <int DT>
__global__ void __launch_bounds__(256) read_kernel(HeldParams p) {
  const uint64_t all = (uint64_t)p.quads * 2 * p.H * p.W, begin = (uint64_t)blockIdx.x * 256;
  const uint64_t here = begin + threadIdx.x, at = here < all ? here : all - 1;
  uint64_t unit;
  uint32_t w;
  if (all >> 31) {
    unit = at / p.W, w = (uint32_t)(at - unit * p.W);
  } else {
    uint32_t u;
    fd_divmod(p.dwords, (uint32_t)at, u, w);
    unit = u;
  }
  const Column c = column_of(p, unit, begin / p.W);
  const Quad q = quad_of<true>(p.pool, p.batch, p.first, c.quad, c.request, here < all && w == 0 && c.kind == 0 && c.head == 0);
  if (here >= all || !q.taken) return;
  const uint8_t* const page = page_at(p.pool, p.layer, c.kind, q.page);
  const u32x4 codes = *(const KVC_GLOBAL u32x4*)(page + codes_at(p.pool, p.W, c.head, q.slot) + w * 16);
  const u32x4 pairs = *(const KVC_GLOBAL u32x4*)(page + pairs_at(p.pool, p.W, p.H, c.head, q.slot));
  uint16_t* const to = (c.kind ? p.v_out : p.k_out) + (uint64_t)(c.head * p.W + w) * 8;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (q.taken >> k & 1u) stream_store<u32x4>(to + (int64_t)(uint32_t)(q.token + k) * p.token_stride, values_of<DT>(codes[k], pairs[k]));
}

// The same from a pool of 16 bits: a thread has eight elements of a quad's tokens.
__global__ void __launch_bounds__(256) read_wide_kernel(HeldParams p) {
  const uint64_t all = (uint64_t)p.quads * 2 * p.H * p.W, begin = (uint64_t)blockIdx.x * 256;
  const uint64_t here = begin + threadIdx.x, at = here < all ? here : all - 1;
  const uint64_t unit = at / p.W;
  const uint32_t w = (uint32_t)(at - unit * p.W);
  const Column c = column_of(p, unit, begin / p.W);
  const Quad q = quad_of<false>(p.pool, p.batch, p.first, c.quad, c.request, here < all && w == 0 && c.kind == 0 && c.head == 0);
  if (here >= all) return;
  uint16_t* const to = (c.kind ? p.v_out : p.k_out) + (uint64_t)(c.head * p.W + w) * 8;
  uint32_t bad = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (!(q.taken >> k & 1u)) continue;
    uint32_t block, slot;  // (a page of any number of tokens may end inside a quad)
    fd_divmod(p.pool.dbs, q.position + k, block, slot);
    const uint32_t page = (uint32_t)p.pool.tables[(uint64_t)q.row * p.pool.table_len + block];
    if (page >= p.pool.num_blocks) {
      bad |= KVC_FAULT_PAGE;
      continue;
    }
    const uint8_t* const from = page_at(p.pool, p.layer, c.kind, page) + (uint64_t)slot * p.pool.token_bytes + (uint64_t)(c.head * p.W + w) * 16;
    stream_store<u32x4>(to + (int64_t)(uint32_t)(q.token + k) * p.token_stride, *(const KVC_GLOBAL u32x4*)from);
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
  const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint64_t unit = at / p.W;
  const uint32_t w = (uint32_t)(at - unit * p.W);
  const PageQuad q = page_quad_of(p, unit);
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

template <int DT>
void launch_write_of(const HeldParams& p, uint32_t P, uint32_t groups, hipStream_t stream) {
  switch (P) {
    case 1: hipLaunchKernelGGL((write_kernel<DT, 1>), dim3(groups), dim3(256), 0, stream, p); break;
    case 2: hipLaunchKernelGGL((write_kernel<DT, 2>), dim3(groups), dim3(256), 0, stream, p); break;
    case 4: hipLaunchKernelGGL((write_kernel<DT, 4>), dim3(groups), dim3(256), 0, stream, p); break;
    case 8: hipLaunchKernelGGL((write_kernel<DT, 8>), dim3(groups), dim3(256), 0, stream, p); break;
    case 16: hipLaunchKernelGGL((write_kernel<DT, 16>), dim3(groups), dim3(256), 0, stream, p); break;
    default: hipLaunchKernelGGL((write_kernel<DT, 32>), dim3(groups), dim3(256), 0, stream, p); break;
  }
}

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
  const uint32_t P = threads_of(p.W);
  const uint64_t groups = ((uint64_t)p.quads * 2 * p.H * P + 255) / 256;
  if (groups > kMostGroups) return KVC_ERR_UNSUPPORTED;
  if (p.dtype == KVC_F16) launch_write_of<KVC_F16>(p, P, (uint32_t)groups, stream);
  else launch_write_of<KVC_BF16>(p, P, (uint32_t)groups, stream);
  return launched();
}

kvc_status launch_read(const HeldParams& p, hipStream_t stream) {
  const uint64_t groups = ((uint64_t)p.quads * 2 * p.H * p.W + 255) / 256;
  if (groups > kMostGroups) return KVC_ERR_UNSUPPORTED;
  if (!p.pool.held) hipLaunchKernelGGL(read_wide_kernel, dim3((uint32_t)groups), dim3(256), 0, stream, p);
  else if (p.dtype == KVC_F16) hipLaunchKernelGGL(read_kernel<KVC_F16>, dim3((uint32_t)groups), dim3(256), 0, stream, p);
  else hipLaunchKernelGGL(read_kernel<KVC_BF16>, dim3((uint32_t)groups), dim3(256), 0, stream, p);
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
