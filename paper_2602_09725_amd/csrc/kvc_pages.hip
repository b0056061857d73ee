// Pages of a pool: copied, forked, taken, freed, compacted; and the tokens of a step written to their slots.
//
// The books are small (four bytes a page) and the pages large, so every call that takes pages has two launches: a survey
// that leaves a bit for each free page, the number of free ones of each segment of 4096 pages and, from the list, how
// many pages the entries before each entry take; then one in which every workgroup finds the pages of its own entry in the
// bits by their rank.  Nothing depends on the order in which workgroups run: the k-th page taken is the k-th free one,
// counts change by atomic additions of whole numbers, and what one workgroup reads of the books no other one of the launch writes.
#include <hip/hip_runtime.h>

#include "kvc_device.h"
#include "kvc_serve.h"

namespace kvc {

namespace {

__device__ __forceinline__ void fault(const PoolView& p, uint32_t bits) {
  if (p.err && bits) atomicOr(p.err, bits);
}

__device__ __forceinline__ uint32_t lane_id() { return threadIdx.x & 63u; }

// Sum over the lanes before and with this one.
template <typename T>
__device__ __forceinline__ T wave_scan(T v) {
#pragma unroll
  for (uint32_t d = 1; d < 64; d *= 2) {
    const T u = __shfl_up(v, d);
    if (lane_id() >= d) v += u;
  }
  return v;
}

__device__ __forceinline__ uint32_t wave_total(uint32_t inclusive) { return __shfl(inclusive, 63); }

__device__ __forceinline__ uint32_t pages_of(const PoolView& p, uint32_t tokens) { return fd_div(p.dbs, tokens + p.block_size - 1); }

// ---- survey -------------------------------------------------------------------------------------------------------------

// Sum over a workgroup's threads before this one; *total gets the sum over all.
__device__ uint64_t group_scan(uint32_t v, uint64_t* sums, uint64_t* total) {
  const uint64_t inclusive = wave_scan<unsigned long long>(v);
  const uint32_t wave = threadIdx.x / 64, waves = blockDim.x / 64;
  __syncthreads();
  if (lane_id() == 63) sums[wave] = inclusive;
  __syncthreads();
  uint64_t before = 0, all = 0;
  for (uint32_t w = 0; w < waves; ++w) {
    if (w < wave) before += sums[w];
    all += sums[w];
  }
  *total = all;
  return before + inclusive - v;
}

// Checks a fork's or a grow's list and counts the pages its entries take.  `seen` has a bit for each row.
template <PageList LIST>
__device__ void plan_list(const PoolView& p, const PageSpace& w, const int32_t* a, const int32_t* b, uint32_t n, uint32_t* seen, uint64_t* sums) {
  for (uint32_t i = threadIdx.x; i < (p.n_rows + 31) / 32; i += blockDim.x) seen[i] = 0;
  __syncthreads();
  uint32_t bad = 0;
  const int32_t* written = LIST == PageList::kFork ? b : a;  // rows that the call changes
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
    const uint32_t row = (uint32_t)written[i];
    if (row >= p.n_rows) {
      bad |= KVC_FAULT_LIST;
      continue;
    }
    if (atomicOr(&seen[row / 32], 1u << (row % 32)) >> (row % 32) & 1u) bad |= KVC_FAULT_LIST;
    if (LIST == PageList::kFork && p.lens[row] != 0) bad |= KVC_FAULT_LIST;
  }
  __syncthreads();
  uint64_t all = 0;
  for (uint32_t base = 0; base < n; base += blockDim.x) {
    const uint32_t i = base + threadIdx.x;
    uint32_t need = 0;
    if (i < n) {
      const uint32_t row = (uint32_t)a[i];
      const uint32_t len = row < p.n_rows ? (uint32_t)p.lens[row] : ~0u;
      if (row >= p.n_rows || len > p.capacity) {
        bad |= KVC_FAULT_LIST;
      } else if (LIST == PageList::kFork) {
        if (seen[row / 32] >> (row % 32) & 1u) bad |= KVC_FAULT_LIST;
        need = len - fd_div(p.dbs, len) * p.block_size != 0;
      } else {
        const int32_t more = b ? b[i] : 1;
        const uint32_t held = pages_of(p, len), whole = fd_div(p.dbs, len);
        if (more < 0) {
          bad |= KVC_FAULT_LIST;
        } else if ((uint32_t)more > p.capacity - len) {
          bad |= KVC_FAULT_NO_ROOM;
        } else {
          need = pages_of(p, len + (uint32_t)more) - held;
          if (held != whole && more > 0) {  // its last page will be written to
            const uint32_t page = (uint32_t)p.tables[(uint64_t)row * p.table_len + whole];
            if (page >= p.num_blocks) fault(p, KVC_FAULT_PAGE);
            else if (p.refs[page] > 1) bad |= KVC_FAULT_LIST;
          }
        }
      }
    }
    uint64_t total;
    const uint64_t before = group_scan(need, sums, &total);
    if (i < n) w.first[i] = (uint32_t)(all + before);  // (used only where all of them are fewer than 2^31)
    all += total;
  }
  if (all > p.num_blocks) bad |= KVC_FAULT_NO_ROOM;
  const uint32_t faults = (__syncthreads_or(bad & KVC_FAULT_LIST) ? KVC_FAULT_LIST : 0u) | (__syncthreads_or(bad & KVC_FAULT_NO_ROOM) ? KVC_FAULT_NO_ROOM : 0u);
  if (threadIdx.x == 0) {
    w.head[kPlanFaults] = faults;
    w.head[kPlanNeed] = (uint32_t)all;
    fault(p, faults);
  }
}

// The last workgroup looks at the list, if there is one, the others at a segment of the pages each.
__global__ void __launch_bounds__(256) survey_kernel(PoolView p, PageSpace w, PageList list, const int32_t* a, const int32_t* b, uint32_t n) {
  extern __shared__ uint32_t seen[];
  __shared__ uint64_t sums[4];
  if (blockIdx.x == w.segments) {
    if (list == PageList::kFork) plan_list<PageList::kFork>(p, w, a, b, n, seen, sums);
    if (list == PageList::kGrow) plan_list<PageList::kGrow>(p, w, a, b, n, seen, sums);
    return;
  }
  const uint32_t seg = blockIdx.x, wave = threadIdx.x / 64;
  uint32_t free_pages = 0;
  int32_t refs[kSegment / 256];
#pragma unroll
  for (uint32_t i = 0; i < kSegment / 256; ++i) {
    const uint32_t page = seg * kSegment + i * 256 + threadIdx.x;
    refs[i] = page < p.num_blocks ? p.refs[page] : 1;
  }
  bool below = false;
#pragma unroll
  for (uint32_t i = 0; i < kSegment / 256; ++i) {
    const uint64_t bits = __ballot(refs[i] <= 0);
    below |= refs[i] < 0;
    if (lane_id() == 0) {
      uint32_t* to = w.bits + (uint64_t)seg * kSegmentWords + i * 8 + wave * 2;
      to[0] = (uint32_t)bits;
      to[1] = (uint32_t)(bits >> 32);
    }
    free_pages += (uint32_t)__popcll(bits);
  }
  if (__any(below) && lane_id() == 0) fault(p, KVC_FAULT_LIST);
  if (lane_id() == 0) sums[wave] = free_pages;
  __syncthreads();
  if (threadIdx.x == 0) w.counts[seg] = (uint32_t)(sums[0] + sums[1] + sums[2] + sums[3]);
}

// ---- taking pages ---------------------------------------------------------------------------------------------------------

// Free pages of segments [0, end); all lanes of a wave call it.
__device__ uint32_t free_before(const PageSpace& w, uint32_t end) {
  uint32_t sum = 0;
  for (uint32_t s = lane_id(); s < end; s += 64) sum += w.counts[s];
  return wave_total(wave_scan(sum));
}

// Whether the plan of a list stands; all lanes of a wave call it.
__device__ bool plan_stands(const PoolView& p, const PageSpace& w) {
  if (w.head[kPlanFaults]) return false;
  if (free_before(w, w.segments) >= w.head[kPlanNeed]) return true;
  if (blockIdx.x == 0 && threadIdx.x == 0) fault(p, KVC_FAULT_NO_ROOM);
  return false;
}

// Calls emit(j, page) for the free pages of ranks first + j, j < m, which there are; all lanes of a wave call it, and each
// page comes to one of them.
template <typename Emit>
__device__ void take_pages(const PageSpace& w, uint32_t first, uint32_t m, Emit emit) {
  if (m == 0) return;
  uint32_t seg = 0, before = 0;
  for (;; seg += 64) {
    if (seg >= w.segments) return;
    const uint32_t c = seg + lane_id() < w.segments ? w.counts[seg + lane_id()] : 0u;
    const uint32_t inclusive = wave_scan(c);
    const uint64_t there = __ballot(before + inclusive > first);
    if (there) {
      const uint32_t at = (uint32_t)__ffsll((unsigned long long)there) - 1;
      before += __shfl(inclusive - c, at);
      seg += at;
      break;
    }
    before += wave_total(inclusive);
  }
  for (; seg < w.segments && before < first + m; ++seg) {
    const uint64_t at = (uint64_t)seg * kSegmentWords + lane_id() * 2;
    uint64_t bits = w.bits[at] | (uint64_t)w.bits[at + 1] << 32;
    const uint32_t c = (uint32_t)__popcll(bits), inclusive = wave_scan(c);
    uint32_t rank = before + inclusive - c;
    if (rank + c > first && rank < first + m) {
      for (; bits; bits &= bits - 1, ++rank)
        if (rank >= first && rank < first + m) emit(rank - first, seg * kSegment + lane_id() * 64 + (uint32_t)__ffsll((unsigned long long)bits) - 1);
    }
    before += wave_total(inclusive);
  }
}

// ---- moving data ----------------------------------------------------------------------------------------------------------

constexpr uint32_t kPiece = 32768;  // bytes that a workgroup of 256 threads moves in one go, eight loads a thread in flight

// Copies up to kPiece bytes, a multiple of 16.
__device__ __forceinline__ void copy_piece(uint8_t* dst, const uint8_t* src, uint32_t bytes) {
  constexpr uint32_t U = kPiece / 16 / 256;
  const uint32_t first = threadIdx.x * 16;
  if (bytes == kPiece) {
    u32x4 v[U];
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) v[u] = stream_load<u32x4>(src + first + u * 4096);
#pragma unroll
    for (uint32_t u = 0; u < U; ++u) stream_store<u32x4>(dst + first + u * 4096, v[u]);
  } else {  // two at a time
    for (uint32_t at = first; at < bytes; at += 8192) {
      const bool two = at + 4096 < bytes;
      const u32x4 a = stream_load<u32x4>(src + at), b = stream_load<u32x4>(src + (two ? at + 4096 : at));
      stream_store<u32x4>(dst + at, a);
      if (two) stream_store<u32x4>(dst + at + 4096, b);
    }
  }
}

__device__ __forceinline__ uint8_t* page_at(const PoolView& p, uint32_t layer, uint32_t kind, uint32_t page) {
  uint8_t* base = (uint8_t*)as_const(p.layers)[layer];
  return base + ((uint64_t)kind * p.num_blocks + page) * p.page_bytes;
}

// Workgroup: one piece of one kind of one layer of one pair.
__global__ void __launch_bounds__(256) copy_kernel(PoolView p, const int32_t* src, const int32_t* dst, FastDiv dpieces, FastDiv dkinds) {
  uint32_t pair, rest, unit = blockIdx.x, piece;
  fd_divmod(dpieces, unit, rest, piece);
  uint32_t layer_kind;
  fd_divmod(dkinds, rest, pair, layer_kind);
  const uint32_t from = (uint32_t)as_const(src)[pair], to = (uint32_t)as_const(dst)[pair];
  if (from >= p.num_blocks || to >= p.num_blocks) {
    if (threadIdx.x == 0) fault(p, KVC_FAULT_PAGE);
    return;
  }
  const uint64_t at = (uint64_t)piece * kPiece, left = p.page_bytes - at;
  copy_piece(page_at(p, layer_kind / 2, layer_kind % 2, to) + at, page_at(p, layer_kind / 2, layer_kind % 2, from) + at,
             left < kPiece ? (uint32_t)left : kPiece);
}

// Workgroup: one layer of one fork.
__global__ void __launch_bounds__(256) fork_kernel(PoolView p, PageSpace w, const int32_t* parents, const int32_t* children, FastDiv dL) {
  uint32_t i, layer;
  fd_divmod(dL, blockIdx.x, i, layer);
  if (!plan_stands(p, w)) return;
  const uint32_t parent = (uint32_t)as_const(parents)[i], child = (uint32_t)as_const(children)[i];
  const uint32_t len = (uint32_t)p.lens[parent], whole = fd_div(p.dbs, len), part = len - whole * p.block_size;
  const int32_t* from = p.tables + (uint64_t)parent * p.table_len;
  int32_t* to = p.tables + (uint64_t)child * p.table_len;
  if (layer == 0) {
    for (uint32_t j = threadIdx.x; j < whole; j += 256) {
      const uint32_t page = (uint32_t)from[j];
      to[j] = (int32_t)page;
      if (page < p.num_blocks) atomicAdd(p.refs + page, 1);
      else fault(p, KVC_FAULT_PAGE);
    }
    if (threadIdx.x == 0) p.lens[child] = (int32_t)len;
  }
  if (part == 0) return;
  __shared__ uint32_t taken;
  if (threadIdx.x < 64)
    take_pages(w, w.first[i], 1, [&](uint32_t, uint32_t page) {
      taken = page;
      if (layer == 0) {
        to[whole] = (int32_t)page;
        p.refs[page] = 1;
      }
    });
  __syncthreads();
  const uint32_t page = taken, source = (uint32_t)from[whole];
  if (source >= p.num_blocks) {
    if (threadIdx.x == 0) fault(p, KVC_FAULT_PAGE);
    return;
  }
  const uint64_t bytes = (uint64_t)part * p.token_bytes;
  for (uint32_t kind = 0; kind < 2; ++kind) {
    uint8_t* d = page_at(p, layer, kind, page);
    const uint8_t* s = page_at(p, layer, kind, source);
    for (uint64_t at = 0; at < bytes; at += kPiece) copy_piece(d + at, s + at, bytes - at < kPiece ? (uint32_t)(bytes - at) : kPiece);
  }
}

// Wave: one row of the list.
__global__ void __launch_bounds__(256) grow_kernel(PoolView p, PageSpace w, const int32_t* rows, const int32_t* counts, uint32_t n) {
  if (!plan_stands(p, w)) return;
  const uint32_t i = blockIdx.x * 4 + threadIdx.x / 64;
  if (i >= n) return;
  const uint32_t row = (uint32_t)rows[i], len = (uint32_t)p.lens[row], now = len + (uint32_t)(counts ? counts[i] : 1);
  const uint32_t held = pages_of(p, len);
  int32_t* to = p.tables + (uint64_t)row * p.table_len + held;
  take_pages(w, w.first[i], pages_of(p, now) - held, [&](uint32_t j, uint32_t page) {
    to[j] = (int32_t)page;
    p.refs[page] = 1;
  });
  if (lane_id() == 0) p.lens[row] = (int32_t)now;
}

// Wave: one row of the list.  The first one that takes a row's length frees its pages.
__global__ void __launch_bounds__(256) free_kernel(PoolView p, const int32_t* rows, uint32_t n) {
  const uint32_t i = blockIdx.x * 4 + threadIdx.x / 64;
  if (i >= n) return;
  const uint32_t row = (uint32_t)rows[i];
  if (row >= p.n_rows) {
    if (lane_id() == 0) fault(p, KVC_FAULT_LIST);
    return;
  }
  uint32_t len = 0;
  if (lane_id() == 0) len = (uint32_t)atomicExch(p.lens + row, 0);
  len = wave_uniform(len);
  uint32_t bad = 0;
  if (len > p.capacity) {  // nobody knows what it holds
    bad = KVC_FAULT_LIST;
    len = 0;
  }
  for (uint32_t j = lane_id(); j < pages_of(p, len); j += 64) {
    const uint32_t page = (uint32_t)p.tables[(uint64_t)row * p.table_len + j];
    if (page >= p.num_blocks) {
      bad |= KVC_FAULT_PAGE;
    } else if (atomicSub(p.refs + page, 1) <= 0) {  // it was free: take it back
      atomicAdd(p.refs + page, 1);
      bad |= KVC_FAULT_LIST;
    }
  }
  fault(p, bad);
}

// ---- compact --------------------------------------------------------------------------------------------------------------

// Workgroup: a segment.  Of a page in use at a place below the number of pages in use `moved` gets the place, of a free one -1, of one that
// moves -2 - its rank among these.
__global__ void __launch_bounds__(256) compact_lists_kernel(PoolView p, PageSpace w) {
  __shared__ uint32_t words[kSegmentWords], before[kSegmentWords];
  const uint32_t seg = blockIdx.x;
  const uint32_t used = p.num_blocks - free_before(w, w.segments);
  // free places below `used`: as many as pages that move
  const uint32_t edge = used / kSegment;
  uint32_t moves = free_before(w, edge < w.segments ? edge : w.segments);
  if (edge < w.segments) {
    uint32_t c = 0;
    for (uint32_t k = lane_id(); k < kSegmentWords; k += 64) {
      const uint32_t base = edge * kSegment + k * 32, bits = w.bits[(uint64_t)edge * kSegmentWords + k];
      c += base >= used ? 0 : (uint32_t)__popc(used - base >= 32 ? bits : bits & ((1u << (used - base)) - 1u));
    }
    moves += wave_total(wave_scan(c));
  }
  const uint32_t free_earlier = free_before(w, seg);
  if (threadIdx.x < 64) {
    const uint64_t at = (uint64_t)seg * kSegmentWords + lane_id() * 2;
    const uint32_t a = w.bits[at], b = w.bits[at + 1], c = (uint32_t)(__popc(a) + __popc(b)), inclusive = wave_scan(c);
    words[lane_id() * 2] = a;
    words[lane_id() * 2 + 1] = b;
    before[lane_id() * 2] = inclusive - c;
    before[lane_id() * 2 + 1] = inclusive - c + (uint32_t)__popc(a);
  }
  __syncthreads();
  for (uint32_t i = 0; i < kSegment / 256; ++i) {
    const uint32_t at = i * 256 + threadIdx.x, page = seg * kSegment + at;
    if (page >= p.num_blocks) break;
    const uint32_t word = words[at / 32], bit = at % 32;
    const uint32_t free_rank = free_earlier + before[at / 32] + (uint32_t)__popc(word & ((1u << bit) - 1u));
    int32_t to = -1;
    if (word >> bit & 1u) {
      if (page < used) w.places[free_rank] = (int32_t)page;
    } else if (page < used) {
      to = (int32_t)page;
    } else {
      const uint32_t rank = page - free_rank - (used - moves);  // pages in use before it, but for those below `used`
      w.sources[rank] = (int32_t)page;
      to = -2 - (int32_t)rank;
    }
    w.moved[page] = to;
    w.refs[page] = p.refs[page] < 0 ? 0 : p.refs[page];
  }
  if (seg == 0 && threadIdx.x == 0) {
    w.head[kPlanUsed] = used;
    w.head[kPlanMoves] = moves;
  }
}

__device__ __forceinline__ int32_t place_of(const PageSpace& w, uint32_t page) {
  const int32_t to = w.moved[page];
  return to <= -2 ? w.places[-2 - to] : to;
}

// The first `movers` workgroups move pages, the others write the books.
__global__ void __launch_bounds__(256) compact_kernel(PoolView p, PageSpace w, int32_t* map, int32_t* tables, int32_t* refs, uint32_t movers,
                                                      uint32_t pieces, FastDiv dlen) {
  const uint32_t moves = as_const(w.head)[kPlanMoves];
  if (blockIdx.x < movers) {
    const uint32_t a_page = 2 * p.L * pieces;
    const uint64_t units = (uint64_t)moves * a_page;
    for (uint64_t unit = blockIdx.x; unit < units; unit += movers) {
      const uint32_t k = (uint32_t)(unit / a_page), rest = (uint32_t)(unit - (uint64_t)k * a_page), lk = rest / pieces;
      const uint64_t at = (uint64_t)(rest - lk * pieces) * kPiece, left = p.page_bytes - at;
      copy_piece(page_at(p, lk / 2, lk % 2, (uint32_t)as_const(w.places)[k]) + at, page_at(p, lk / 2, lk % 2, (uint32_t)as_const(w.sources)[k]) + at,
                 left < kPiece ? (uint32_t)left : kPiece);
    }
    return;
  }
  const uint32_t threads = (gridDim.x - movers) * 256, self = (blockIdx.x - movers) * 256 + threadIdx.x;
  const uint32_t used = as_const(w.head)[kPlanUsed];
  for (uint32_t page = self; page < p.num_blocks; page += threads) {
    map[page] = place_of(w, page);
    int32_t held = 0;
    if (page < used) {
      const int32_t here = w.refs[page];
      if (here) {
        held = here;
      } else {  // the place of a page that moves here: its rank is the free place's
        uint32_t low = 0, high = moves;
        while (low + 1 < high) {
          const uint32_t mid = (low + high) / 2;
          if ((uint32_t)w.places[mid] <= page) low = mid;
          else high = mid;
        }
        held = w.refs[w.sources[low]];
      }
    }
    refs[page] = held;
  }
  uint32_t bad = 0;
  const uint64_t entries = (uint64_t)p.n_rows * p.table_len;
  for (uint64_t e = self; e < entries; e += threads) {
    const uint32_t row = e >> 31 ? (uint32_t)(e / p.table_len) : fd_div(dlen, (uint32_t)e), j = (uint32_t)(e - (uint64_t)row * p.table_len);
    uint32_t len = (uint32_t)p.lens[row];
    if (len > p.capacity) {
      bad |= KVC_FAULT_LIST;
      len = 0;
    }
    const int32_t was = p.tables[e];
    int32_t now = was;
    if (j < pages_of(p, len)) {
      if ((uint32_t)was >= p.num_blocks) {
        bad |= KVC_FAULT_PAGE;
      } else if ((now = place_of(w, (uint32_t)was)) < 0) {
        bad |= KVC_FAULT_LIST;
        now = was;
      }
    }
    tables[e] = now;
  }
  fault(p, bad);
}

// ---- append ---------------------------------------------------------------------------------------------------------------

// Request of new token t, given one at or before it.
__device__ __forceinline__ uint32_t request_from(const BatchView& b, uint32_t t, uint32_t r) {
  while (r + 1 < b.n_requests && (uint32_t)b.starts[r + 1] <= t) ++r;
  return r;
}

// Thread: U vectors of 8 elements; a token's vectors are those of its key, then those of its value.
template <int U>
__global__ void __launch_bounds__(256) append_kernel(AppendParams p) {
  fetch_params<AppendParams>();
  const uint32_t per_token = 2 * p.atoms;
  const uint64_t begin = (uint64_t)blockIdx.x * (256 * U), all = (uint64_t)p.batch.n_new * per_token;
  uint32_t r0 = 0;
  if (p.batch.starts) {  // the request of the workgroup's first token: how many begin at or before it
    const uint32_t t = (uint32_t)(begin / per_token);
    uint32_t c = 0;
    for (uint32_t r = lane_id(); r < ((p.batch.n_requests + 63) & ~63u); r += 64)
      c += (uint32_t)__popcll(__ballot(r < p.batch.n_requests && (uint32_t)p.batch.starts[r] <= t));
    r0 = c ? c - 1 : 0;
  }
  u32x4 value[U];
  uint8_t* to[U];
  uint32_t bad = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint64_t at = begin + (uint32_t)u * 256 + threadIdx.x;
    to[u] = nullptr;
    if (at >= all) continue;
    uint32_t t, atom, twice;
    if (all >> 31) twice = (uint32_t)(at / p.atoms), atom = (uint32_t)(at - (uint64_t)twice * p.atoms);
    else fd_divmod(p.datoms, (uint32_t)at, twice, atom);
    t = twice / 2;
    const uint32_t kind = twice % 2;
    uint32_t r = t, back = 1;  // the token is its request's last but back - 1
    if (p.batch.starts) {
      r = request_from(p.batch, t, r0);
      const uint32_t end = (uint32_t)p.batch.starts[r + 1];
      back = end - t;
    }
    const uint32_t row = p.batch.rows ? (uint32_t)p.batch.rows[r] : r;
    const uint32_t len = row < p.pool.n_rows ? (uint32_t)p.pool.lens[row] : ~0u;
    if (len > p.pool.capacity || back - 1 >= len) {
      bad |= KVC_FAULT_LIST;
      continue;
    }
    uint32_t block, slot;
    fd_divmod(p.pool.dbs, len - back, block, slot);
    const uint32_t page = (uint32_t)p.pool.tables[(uint64_t)row * p.pool.table_len + block];
    if (page >= p.pool.num_blocks) {
      bad |= KVC_FAULT_PAGE;
      continue;
    }
    value[u] = *(const KVC_GLOBAL u32x4*)((kind ? p.v : p.k) + (int64_t)t * p.token_stride + atom * 8);
    to[u] = page_at(p.pool, p.layer, kind, page) + (uint64_t)slot * p.pool.token_bytes + atom * 16;
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (to[u]) *(KVC_GLOBAL u32x4*)to[u] = value[u];
  fault(p.pool, bad);
}

kvc_status launched() { return hipGetLastError() == hipSuccess ? KVC_OK : KVC_ERR_RUNTIME; }

}  // namespace

kvc_status launch_survey(const PoolView& pool, const PageSpace& w, PageList list, const int32_t* a, const int32_t* b, uint32_t n,
                         hipStream_t stream) {
  const uint32_t seen = list == PageList::kNone ? 0 : (pool.n_rows + 31) / 32 * 4;
  hipLaunchKernelGGL(survey_kernel, dim3(w.segments + (list != PageList::kNone)), dim3(256), seen, stream, pool, w, list, a, b, n);
  return launched();
}

kvc_status launch_fork(const PoolView& pool, const PageSpace& w, const int32_t* parents, const int32_t* children, uint32_t n,
                       hipStream_t stream) {
  if ((uint64_t)n * pool.L >> 31) return KVC_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(fork_kernel, dim3(n * pool.L), dim3(256), 0, stream, pool, w, parents, children, make_fastdiv(pool.L));
  return launched();
}

kvc_status launch_grow(const PoolView& pool, const PageSpace& w, const int32_t* rows, const int32_t* counts, uint32_t n,
                       hipStream_t stream) {
  hipLaunchKernelGGL(grow_kernel, dim3((n + 3) / 4), dim3(256), 0, stream, pool, w, rows, counts, n);
  return launched();
}

kvc_status launch_free(const PoolView& pool, const int32_t* rows, uint32_t n, hipStream_t stream) {
  hipLaunchKernelGGL(free_kernel, dim3((n + 3) / 4), dim3(256), 0, stream, pool, rows, n);
  return launched();
}

kvc_status launch_compact(const PoolView& pool, const PageSpace& w, int32_t* map, int32_t* tables, int32_t* refs, hipStream_t stream) {
  const uint64_t pieces = (pool.page_bytes + kPiece - 1) / kPiece;
  if (2 * pool.L * pieces >> 31) return KVC_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(compact_lists_kernel, dim3(w.segments), dim3(256), 0, stream, pool, w);
  if (hipGetLastError() != hipSuccess) return KVC_ERR_RUNTIME;
  const uint32_t movers = 2048;
  const uint64_t books = ((uint64_t)pool.n_rows * pool.table_len + pool.num_blocks + 1023) / 1024;
  hipLaunchKernelGGL(compact_kernel, dim3(movers + (uint32_t)(books < 512 ? books : 512)), dim3(256), 0, stream, pool, w, map, tables, refs,
                     movers, (uint32_t)pieces, make_fastdiv(pool.table_len));
  return launched();
}

kvc_status launch_copy_pages(const PoolView& pool, const int32_t* src, const int32_t* dst, uint32_t n, hipStream_t stream) {
  const uint64_t pieces = (pool.page_bytes + kPiece - 1) / kPiece;
  if (2 * pool.L * pieces >> 31 || (uint64_t)n * (2 * pool.L * pieces) >> 31) return KVC_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(copy_kernel, dim3((uint32_t)(n * 2 * pool.L * pieces)), dim3(256), 0, stream, pool, src, dst, make_fastdiv((uint32_t)pieces),
                     make_fastdiv(2 * pool.L));
  return launched();
}

kvc_status launch_append(const AppendParams& p, hipStream_t stream) {
  const uint64_t vectors = (uint64_t)p.batch.n_new * 2 * p.atoms;
  const bool many = vectors >= 256 * 4 * 512;
  const uint64_t groups = (vectors + (many ? 1023 : 255)) / (many ? 1024 : 256);
  if (groups >> 31) return KVC_ERR_UNSUPPORTED;
  if (many) hipLaunchKernelGGL(append_kernel<4>, dim3((uint32_t)groups), dim3(256), 0, stream, p);
  else hipLaunchKernelGGL(append_kernel<1>, dim3((uint32_t)groups), dim3(256), 0, stream, p);
  return launched();
}

}  // namespace kvc
