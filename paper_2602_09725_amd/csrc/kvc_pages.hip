// Pages of a pool: copied, forked, taken, freed, compacted; and the tokens of a step written to their slots.
//
// The books are small (four bytes a page) and the pages large.  The books of a pool of up to kOnePages pages are one workgroup's
// work, which has a bit for each free page in LDS: growing rows is one launch, and forking and compacting are this one and a second one that moves
// the data.  In larger pools a survey by many workgroups leaves a bit for each free page, the number of free ones of each segment of
// 4096 pages and, from the list, how many pages the entries before each entry take; then every workgroup finds the pages of its
// own entry in the bits by their rank.  Nothing depends on the order in which workgroups run: the k-th page taken is the k-th free one,
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

// Notes a row that an entry of a list changes in `seen`, a bit for each row; len: its length.
template <PageList LIST>
__device__ __forceinline__ uint32_t note_row(const PoolView& p, uint32_t row, int32_t len, uint32_t* seen) {
  if (row >= p.n_rows) return KVC_FAULT_LIST;
  const bool twice = atomicOr(&seen[row / 32], 1u << (row % 32)) >> (row % 32) & 1u;
  return twice || (LIST == PageList::kFork && len != 0) ? KVC_FAULT_LIST : 0u;
}

// A fork's parent may not be a row that the call changes.
__device__ __forceinline__ uint32_t parent_noted(const PoolView& p, uint32_t row, const uint32_t* seen) {
  return row < p.n_rows && (seen[row / 32] >> (row % 32) & 1u) ? KVC_FAULT_LIST : 0u;
}

// What an entry of a list takes: its row (a fork's parent), the row's length and pages, and how many pages it needs for `more` tokens.
struct Entry {
  uint32_t row, len, held, need, more;
  uint32_t last;  // page that is filled in part, if there is one
};

template <PageList LIST>
__device__ __forceinline__ Entry entry_of(const PoolView& p, uint32_t row, int32_t more, uint32_t& bad) {
  Entry e{};
  const uint32_t len = row < p.n_rows ? (uint32_t)p.lens[row] : ~0u;
  if (row >= p.n_rows || len > p.capacity) {
    bad |= KVC_FAULT_LIST;
    return e;
  }
  e.row = row;
  e.len = len;
  const uint32_t whole = fd_div(p.dbs, len);
  e.held = pages_of(p, len);
  const bool part = e.held != whole;
  if (part) e.last = (uint32_t)p.tables[(uint64_t)row * p.table_len + whole];
  if (LIST == PageList::kFork) {
    e.need = part;
  } else if (more < 0) {
    bad |= KVC_FAULT_LIST;
  } else if ((uint32_t)more > p.capacity - len) {
    bad |= KVC_FAULT_NO_ROOM;
  } else {
    e.more = (uint32_t)more;
    e.need = pages_of(p, len + e.more) - e.held;
    if (part && more > 0) {  // its last page will be written to: it has to be this row's alone
      if (e.last >= p.num_blocks) fault(p, KVC_FAULT_PAGE);
      else if (p.refs[e.last] != 1) bad |= KVC_FAULT_LIST;
    }
  }
  return e;
}

// The faults that any thread of a workgroup has met; all of them call it.
__device__ __forceinline__ uint32_t all_faults(uint32_t bad) {
  return (__syncthreads_or(bad & KVC_FAULT_LIST) ? KVC_FAULT_LIST : 0u) | (__syncthreads_or(bad & KVC_FAULT_NO_ROOM) ? KVC_FAULT_NO_ROOM : 0u);
}

// Checks a fork's or a grow's list and counts the pages its entries take.
template <PageList LIST>
__device__ void plan_list(const PoolView& p, const PageSpace& w, const int32_t* a, const int32_t* b, uint32_t n, uint32_t* seen, uint64_t* sums) {
  for (uint32_t i = threadIdx.x; i < (p.n_rows + 31) / 32; i += blockDim.x) seen[i] = 0;
  __syncthreads();
  uint32_t bad = 0;
  const int32_t* written = LIST == PageList::kFork ? b : a;
  for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
    const uint32_t row = (uint32_t)written[i];
    bad |= note_row<LIST>(p, row, row < p.n_rows ? p.lens[row] : 0, seen);
  }
  __syncthreads();
  uint64_t all = 0;
  for (uint32_t base = 0; base < n; base += blockDim.x) {
    const uint32_t i = base + threadIdx.x;
    uint32_t need = 0;
    if (i < n) {
      const uint32_t row = (uint32_t)a[i];
      if (LIST == PageList::kFork) bad |= parent_noted(p, row, seen);
      const Entry e = entry_of<LIST>(p, row, LIST == PageList::kGrow && b ? b[i] : 1, bad);
      need = e.need;
      if (LIST == PageList::kFork && need && e.last < p.num_blocks && p.refs[e.last] <= 0) bad |= KVC_FAULT_LIST;  // (its tokens are nobody's)
    }
    uint64_t total;
    const uint64_t before = group_scan(need, sums, &total);
    if (i < n) w.first[i] = (uint32_t)(all + before);  // (used only where all of them are fewer than 2^31)
    all += total;
  }
  if (all > p.num_blocks) bad |= KVC_FAULT_NO_ROOM;
  const uint32_t faults = all_faults(bad);
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

// Compact's lists, at one page: of a page in use at a place below the number of pages in use `moved` gets the place, of a free one -1, of one
// that moves -2 - its rank among these.  word: the bits of its 32 pages; before: free pages before these; low: free places below `used`.
__device__ __forceinline__ void list_page(const PoolView& p, const PageSpace& w, uint32_t page, uint32_t word, uint32_t before, uint32_t used,
                                          uint32_t low) {
  const uint32_t bit = page % 32, free_rank = before + (uint32_t)__popc(word & ((1u << bit) - 1u));
  int32_t to = -1;
  if (word >> bit & 1u) {
    if (page < used) w.places[free_rank] = (int32_t)page;
  } else if (page < used) {
    to = (int32_t)page;
  } else {
    const uint32_t rank = page - free_rank - (used - low);  // pages in use before it, but for those below `used`
    w.sources[rank] = (int32_t)page;
    to = -2 - (int32_t)rank;
  }
  w.moved[page] = to;
  w.refs[page] = p.refs[page] < 0 ? 0 : p.refs[page];
}

// ---- small pools ----------------------------------------------------------------------------------------------------------

// The books of a small pool in one workgroup: a bit for each free page, and the free ones before each word of them.
constexpr uint32_t kOneThreads = 1024, kOneWords = kOnePages / 32;
struct OneBooks {
  uint64_t sums[kOneThreads / 64];
  uint32_t words[kOneWords], before[kOneWords];
  uint32_t faults;
};

// What a thread's entry of a list takes, how many pages the entries before it take, and what is true of all.
struct OnePlan {
  Entry e;
  uint32_t first, free_pages, total, faults;
};

// Fills the books and checks a fork's or a grow's list, an entry a thread.  The call's time is that of memory's answers one after the other, so what can be
// asked for at once is, and free pages and needs are added up together (2^14 free ones at most, the needs below them).
template <PageList LIST>
__device__ __forceinline__ OnePlan plan_one(const PoolView& p, OneBooks& s, const int32_t* a, const int32_t* b, uint32_t n, uint32_t* seen) {
  constexpr uint32_t kWaves = kOneThreads / 64;
  const uint32_t self = threadIdx.x, wave = self / 64;
  const bool mine = LIST != PageList::kNone && self < n;
  OnePlan plan{};
  uint32_t row = ~0u, bad = 0;
  int32_t other = 1, other_len = 0;
  if (mine) {
    row = (uint32_t)a[self];
    if (LIST == PageList::kFork || b) other = b[self];
  }
  int32_t refs[kOnePages / kOneThreads];
#pragma unroll
  for (uint32_t i = 0; i < kOnePages / kOneThreads; ++i) {
    const uint32_t page = i * kOneThreads + self;
    refs[i] = page < p.num_blocks ? p.refs[page] : 1;
  }
  if (LIST != PageList::kNone)
    for (uint32_t i = self; i < (p.n_rows + 31) / 32; i += kOneThreads) seen[i] = 0;
  if (self == 0) s.faults = 0;
  if (mine) {
    if (LIST == PageList::kFork && (uint32_t)other < p.n_rows) other_len = p.lens[other];
    plan.e = entry_of<LIST>(p, row, other, bad);
  }
  bool below = false;
#pragma unroll
  for (uint32_t i = 0; i < kOnePages / kOneThreads; ++i) {
    const uint64_t bits = __ballot(refs[i] <= 0);
    below |= refs[i] < 0;
    if (lane_id() == 0) {
      uint32_t* to = s.words + (i * kOneThreads + self) / 32;
      to[0] = (uint32_t)bits;
      to[1] = (uint32_t)(bits >> 32);
    }
  }
  if (__any(below) && lane_id() == 0) fault(p, KVC_FAULT_LIST);
  __syncthreads();
  if (mine) bad |= note_row<LIST>(p, LIST == PageList::kFork ? (uint32_t)other : row, other_len, seen);
  if (LIST == PageList::kFork && plan.e.need && plan.e.last < p.num_blocks && (s.words[plan.e.last / 32] >> plan.e.last % 32 & 1u))
    bad |= KVC_FAULT_LIST;  // (its tokens are nobody's)
  const uint64_t v = (uint64_t)(self < kOneWords ? __popc(s.words[self]) : 0) << 44 | plan.e.need;
  const uint64_t inclusive = wave_scan<unsigned long long>(v);
  if (lane_id() == 63) s.sums[wave] = inclusive;
  if (LIST == PageList::kFork) {
    __syncthreads();
    if (mine) bad |= parent_noted(p, row, seen);
  }
  if (bad) atomicOr(&s.faults, bad);
  __syncthreads();
  uint64_t before = inclusive - v, all = 0;
#pragma unroll
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w < wave) before += s.sums[w];
    all += s.sums[w];
  }
  if (self < kOneWords) s.before[self] = (uint32_t)(before >> 44);
  const uint64_t needs = (1ull << 44) - 1;
  plan.first = (uint32_t)(before & needs);  // (used only where all of them are fewer than the free pages)
  plan.free_pages = (uint32_t)(all >> 44);
  plan.total = (uint32_t)(all & needs);
  plan.faults = s.faults & (KVC_FAULT_LIST | KVC_FAULT_NO_ROOM);
  if (!plan.faults && (all & needs) > plan.free_pages) plan.faults = KVC_FAULT_NO_ROOM;
  if (self == 0) fault(p, plan.faults);
  return plan;  // (s.before is there for all threads after the next barrier)
}

// The free page of a rank that there is.
__device__ uint32_t page_of_rank(const OneBooks& s, uint32_t rank) {
  uint32_t k = 0;
#pragma unroll
  for (uint32_t step = kOneWords / 2; step; step /= 2)
    if (s.before[k + step] <= rank) k += step;
  uint32_t bits = s.words[k];
  for (uint32_t skip = rank - s.before[k]; skip; --skip) bits &= bits - 1;
  return k * 32 + (uint32_t)__ffs(bits) - 1;
}

// What a fork leaves for the launch that copies: where the tokens of the parent's last page come from and go to, and how many they are.
__global__ void __launch_bounds__(kOneThreads) plan_fork_kernel(PoolView p, PageSpace w, const int32_t* parents, const int32_t* children, uint32_t n) {
  extern __shared__ uint32_t seen[];
  __shared__ OneBooks s;
  const uint32_t i = threadIdx.x;
  const uint32_t child = i < n ? (uint32_t)children[i] : 0u;
  const OnePlan plan = plan_one<PageList::kFork>(p, s, parents, children, n, seen);
  const Entry& e = plan.e;
  if (i == 0) w.head[kPlanFaults] = plan.faults;
  if (i < w.segments * kSegmentWords) w.bits[i] = s.words[i];  // (kOneWords at most)
  __syncthreads();
  if (i >= n || plan.faults) return;
  ForkJob job = {0, 0, 0, e.len};
  if (e.need) {
    const uint64_t whole = e.held - 1;
    job.to = page_of_rank(s, plan.first);
    job.from = e.last;
    job.tokens = e.len - (uint32_t)whole * p.block_size;
    p.tables[(uint64_t)child * p.table_len + whole] = (int32_t)job.to;
    p.refs[job.to] = 1;
    if (job.from >= p.num_blocks) {
      fault(p, KVC_FAULT_PAGE);
      job.tokens = 0;
    }
  }
  p.lens[child] = (int32_t)e.len;
  w.jobs[i] = job;
}

__global__ void __launch_bounds__(kOneThreads) grow_one_kernel(PoolView p, const int32_t* rows, const int32_t* counts, uint32_t n) {
  extern __shared__ uint32_t seen[];
  __shared__ OneBooks s;
  __shared__ uint32_t first[kOneThreads];
  __shared__ uint64_t to[kOneThreads];
  const uint32_t i = threadIdx.x;
  const OnePlan plan = plan_one<PageList::kGrow>(p, s, rows, counts, n, seen);
  const Entry& e = plan.e;
  first[i] = i < n ? plan.first : ~0u;
  to[i] = (uint64_t)e.row * p.table_len + e.held;
  __syncthreads();
  if (plan.faults) return;
  for (uint32_t rank = i; rank < plan.total; rank += kOneThreads) {
    uint32_t k = 0;  // the last entry that begins at or before it: those after it that need none begin later
#pragma unroll
    for (uint32_t step = kOneThreads / 2; step; step /= 2)
      if (first[k + step] <= rank) k += step;
    const uint32_t page = page_of_rank(s, rank);
    p.tables[to[k] + rank - first[k]] = (int32_t)page;
    p.refs[page] = 1;
  }
  if (i < n) p.lens[e.row] = (int32_t)(e.len + e.more);
}

// The lists of compact, as compact_lists_kernel leaves them.
__global__ void __launch_bounds__(kOneThreads) compact_one_kernel(PoolView p, PageSpace w) {
  __shared__ OneBooks s;
  const uint32_t used = p.num_blocks - plan_one<PageList::kNone>(p, s, nullptr, nullptr, 0, nullptr).free_pages;
  __syncthreads();
  const uint32_t word = used / 32;  // (none is free if all are in use)
  const uint32_t low = used < p.num_blocks ? s.before[word] + (uint32_t)__popc(s.words[word] & ((1u << used % 32) - 1u)) : 0u;
  for (uint32_t page = threadIdx.x; page < p.num_blocks; page += kOneThreads)
    list_page(p, w, page, s.words[page / 32], s.before[page / 32], used, low);
  if (threadIdx.x == 0) {
    w.head[kPlanUsed] = used;
    w.head[kPlanMoves] = low;
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
  } else {
    u32x4 v[U];
#pragma unroll
    for (uint32_t u = 0; u < U; ++u)
      if (first + u * 4096 < bytes) v[u] = stream_load<u32x4>(src + first + u * 4096);
#pragma unroll
    for (uint32_t u = 0; u < U; ++u)
      if (first + u * 4096 < bytes) stream_store<u32x4>(dst + first + u * 4096, v[u]);
  }
}

// Bytes of the k-th piece of so many.  (In 32 bits: of a choice by a 64-bit comparison of uniform values the compiler has been seen to take
// the wrong side, the comparison in one flag and the choice by another.)
__device__ __forceinline__ uint32_t piece_bytes(uint64_t all, uint32_t k) {
  return k < (uint32_t)(all / kPiece) ? kPiece : (uint32_t)all % kPiece;
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
  const uint64_t at = (uint64_t)piece * kPiece;
  copy_piece(page_at(p, layer_kind / 2, layer_kind % 2, to) + at, page_at(p, layer_kind / 2, layer_kind % 2, from) + at,
             piece_bytes(p.page_bytes, piece));
}

// Workgroup: one kind of one layer of one fork.  KNOWN: plan_fork_kernel has written the books but for the pages that are shared.
// Whether a page was free before the call is asked of the survey's bits: the call itself may have taken it since.
template <bool KNOWN>
__global__ void __launch_bounds__(256) fork_kernel(PoolView p, PageSpace w, const int32_t* parents, const int32_t* children, FastDiv dkinds) {
  uint32_t i, layer_kind;
  fd_divmod(dkinds, blockIdx.x, i, layer_kind);
  ForkJob job;
  if constexpr (KNOWN) {
    job = __builtin_bit_cast(ForkJob, as_const(reinterpret_cast<const u32x4*>(w.jobs))[i]);
    if (as_const(w.head)[kPlanFaults]) return;
  } else {
    if (!plan_stands(p, w)) return;
    job.len = (uint32_t)p.lens[as_const(parents)[i]];
  }
  const uint32_t whole = fd_div(p.dbs, job.len);
  if (layer_kind == 0 || !KNOWN) {
    const uint32_t parent = (uint32_t)as_const(parents)[i], child = (uint32_t)as_const(children)[i];
    const int32_t* from = p.tables + (uint64_t)parent * p.table_len;
    int32_t* to = p.tables + (uint64_t)child * p.table_len;
    if (layer_kind == 0) {
      for (uint32_t j = threadIdx.x; j < whole; j += 256) {
        const uint32_t page = (uint32_t)from[j];
        to[j] = (int32_t)page;
        if (page >= p.num_blocks) fault(p, KVC_FAULT_PAGE);
        else if (w.bits[page / 32] >> page % 32 & 1u) fault(p, KVC_FAULT_LIST);
        else atomicAdd(p.refs + page, 1);
      }
    }
    if constexpr (!KNOWN) {
      job.tokens = job.len - whole * p.block_size;
      if (layer_kind == 0 && threadIdx.x == 0) p.lens[child] = (int32_t)job.len;
      if (job.tokens == 0) return;
      __shared__ uint32_t taken;
      if (threadIdx.x < 64)
        take_pages(w, w.first[i], 1, [&](uint32_t, uint32_t page) {
          taken = page;
          if (layer_kind == 0) {
            to[whole] = (int32_t)page;
            p.refs[page] = 1;
          }
        });
      __syncthreads();
      job.to = taken;
      job.from = (uint32_t)from[whole];
      if (job.from >= p.num_blocks) {
        if (threadIdx.x == 0) fault(p, KVC_FAULT_PAGE);
        return;
      }
    }
  }
  if (job.tokens == 0) return;
  // (a page in 4 bits has the tokens of a head, not the heads of a token, side by side: it is copied whole)
  const uint64_t bytes = (uint64_t)(p.held ? p.block_size : job.tokens) * p.token_bytes;
  uint8_t* d = page_at(p, layer_kind / 2, layer_kind % 2, job.to);
  const uint8_t* s = page_at(p, layer_kind / 2, layer_kind % 2, job.from);
  const uint32_t pieces = (uint32_t)((bytes + kPiece - 1) / kPiece);
  for (uint32_t k = 0; k < pieces; ++k) copy_piece(d + (uint64_t)k * kPiece, s + (uint64_t)k * kPiece, piece_bytes(bytes, k));
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

// Workgroup: a segment.
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
    list_page(p, w, page, words[at / 32], free_earlier + before[at / 32], used, moves);
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
      const uint32_t piece = rest - lk * pieces;
      const uint64_t at = (uint64_t)piece * kPiece;
      copy_piece(page_at(p, lk / 2, lk % 2, (uint32_t)as_const(w.places)[k]) + at, page_at(p, lk / 2, lk % 2, (uint32_t)as_const(w.sources)[k]) + at,
                 piece_bytes(p.page_bytes, piece));
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
  // Each of a vector's questions (request, row, length, page) waits for the one before: those of a thread's vectors are asked side by side, with
  // indexes that are in range whatever the answers were.
  const uint64_t most = begin + 256 * U < all ? begin + 256 * U - 1 : all - 1;
  bool several = false;
  if (p.batch.starts && r0 + 1 < p.batch.n_requests) several = (uint32_t)p.batch.starts[r0 + 1] <= (uint32_t)(most / per_token);
  u32x4 value[U];
  uint32_t t[U], kind[U], atom[U], r[U], first[U], back[U], row[U], len[U], page[U], slot[U];
  bool live[U];
  uint32_t bad = 0;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint64_t here = begin + (uint32_t)u * 256 + threadIdx.x, at = here < all ? here : all - 1;
    live[u] = here < all;
    uint32_t twice;
    if (all >> 31) twice = (uint32_t)(at / p.atoms), atom[u] = (uint32_t)(at - (uint64_t)twice * p.atoms);
    else fd_divmod(p.datoms, (uint32_t)at, twice, atom[u]);
    t[u] = twice / 2;
    kind[u] = twice % 2;
    value[u] = *(const KVC_GLOBAL u32x4*)((kind[u] ? p.v : p.k) + (int64_t)t[u] * p.token_stride + atom[u] * 8);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {  // the token is its request's last but back - 1
    r[u] = p.batch.starts ? r0 : t[u];
    if (several) r[u] = request_from(p.batch, t[u], u ? r[u - 1] : r0);
    first[u] = p.batch.starts ? (uint32_t)p.batch.starts[r[u]] : t[u];
    back[u] = p.batch.starts ? (uint32_t)p.batch.starts[r[u] + 1] - t[u] : 1u;
    row[u] = p.batch.rows ? (uint32_t)p.batch.rows[r[u]] : r[u];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool known = row[u] < p.pool.n_rows;
    len[u] = (uint32_t)p.pool.lens[known ? row[u] : 0];
    if (live[u] && (!known || len[u] > p.pool.capacity || back[u] - 1 >= len[u] || t[u] - first[u] >= p.batch.most_new)) {
      bad |= KVC_FAULT_LIST;
      live[u] = false;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t block;
    fd_divmod(p.pool.dbs, live[u] ? len[u] - back[u] : 0u, block, slot[u]);
    page[u] = (uint32_t)p.pool.tables[(uint64_t)(live[u] ? row[u] : 0u) * p.pool.table_len + block];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!live[u]) continue;
    if (page[u] < p.pool.num_blocks)
      *(KVC_GLOBAL u32x4*)(page_at(p.pool, p.layer, kind[u], page[u]) + (uint64_t)slot[u] * p.pool.token_bytes + atom[u] * 16) = value[u];
    else
      bad |= KVC_FAULT_PAGE;
  }
  fault(p.pool, bad);
}

kvc_status launched() { return hipGetLastError() == hipSuccess ? KVC_OK : KVC_ERR_RUNTIME; }

}  // namespace

namespace {

// Whether one workgroup looks after a call's books: of pools of kOnePages pages, and lists of an entry a thread.  (One layer, lists of 4 to 1024
// entries, pools of 500 to 16384 pages, kernels: a grow 4.4-7.2 us, by many workgroups 12-18; a fork 8.1-10.2, 7.8-13.0; a compact of few pages 7.0-15.4,
// 10-23.)
bool one_group(const PoolView& pool, uint32_t n) { return pool.num_blocks <= kOnePages && n <= kOneThreads; }

kvc_status launch_survey(const PoolView& pool, const PageSpace& w, PageList list, const int32_t* a, const int32_t* b, uint32_t n,
                         hipStream_t stream) {
  const uint32_t seen = list == PageList::kNone ? 0 : (pool.n_rows + 31) / 32 * 4;
  hipLaunchKernelGGL(survey_kernel, dim3(w.segments + (list != PageList::kNone)), dim3(256), seen, stream, pool, w, list, a, b, n);
  return launched();
}

}  // namespace

kvc_status launch_fork(const PoolView& pool, const PageSpace& w, const int32_t* parents, const int32_t* children, uint32_t n,
                       hipStream_t stream) {
  const uint32_t kinds = 2 * pool.L;
  if ((uint64_t)n * kinds > kMostGroups) return KVC_ERR_UNSUPPORTED;
  if (one_group(pool, n)) {
    hipLaunchKernelGGL(plan_fork_kernel, dim3(1), dim3(kOneThreads), (pool.n_rows + 31) / 32 * 4, stream, pool, w, parents, children, n);
    if (hipGetLastError() != hipSuccess) return KVC_ERR_RUNTIME;
    hipLaunchKernelGGL(fork_kernel<true>, dim3(n * kinds), dim3(256), 0, stream, pool, w, parents, children, make_fastdiv(kinds));
    return launched();
  }
  const kvc_status st = launch_survey(pool, w, PageList::kFork, parents, children, n, stream);
  if (st != KVC_OK) return st;
  hipLaunchKernelGGL(fork_kernel<false>, dim3(n * kinds), dim3(256), 0, stream, pool, w, parents, children, make_fastdiv(kinds));
  return launched();
}

kvc_status launch_grow(const PoolView& pool, const PageSpace& w, const int32_t* rows, const int32_t* counts, uint32_t n,
                       hipStream_t stream) {
  if (one_group(pool, n)) {
    hipLaunchKernelGGL(grow_one_kernel, dim3(1), dim3(kOneThreads), (pool.n_rows + 31) / 32 * 4, stream, pool, rows, counts, n);
    return launched();
  }
  const kvc_status st = launch_survey(pool, w, PageList::kGrow, rows, counts, n, stream);
  if (st != KVC_OK) return st;
  hipLaunchKernelGGL(grow_kernel, dim3((n + 3) / 4), dim3(256), 0, stream, pool, w, rows, counts, n);
  return launched();
}

kvc_status launch_free(const PoolView& pool, const int32_t* rows, uint32_t n, hipStream_t stream) {
  if ((n + 3) / 4 > kMostGroups) return KVC_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(free_kernel, dim3((n + 3) / 4), dim3(256), 0, stream, pool, rows, n);
  return launched();
}

kvc_status launch_compact(const PoolView& pool, const PageSpace& w, int32_t* map, int32_t* tables, int32_t* refs, hipStream_t stream) {
  const uint64_t pieces = (pool.page_bytes + kPiece - 1) / kPiece;
  if (2 * pool.L * pieces >> 31) return KVC_ERR_UNSUPPORTED;
  if (one_group(pool, 0)) {
    hipLaunchKernelGGL(compact_one_kernel, dim3(1), dim3(kOneThreads), 0, stream, pool, w);
  } else {
    const kvc_status st = launch_survey(pool, w, PageList::kNone, nullptr, nullptr, 0, stream);
    if (st != KVC_OK) return st;
    hipLaunchKernelGGL(compact_lists_kernel, dim3(w.segments), dim3(256), 0, stream, pool, w);
  }
  if (hipGetLastError() != hipSuccess) return KVC_ERR_RUNTIME;
  const uint32_t movers = 2048;
  const uint64_t books = ((uint64_t)pool.n_rows * pool.table_len + pool.num_blocks + 1023) / 1024;
  hipLaunchKernelGGL(compact_kernel, dim3(movers + (uint32_t)(books < 512 ? books : 512)), dim3(256), 0, stream, pool, w, map, tables, refs,
                     movers, (uint32_t)pieces, make_fastdiv(pool.table_len));
  return launched();
}

kvc_status launch_copy_pages(const PoolView& pool, const int32_t* src, const int32_t* dst, uint32_t n, hipStream_t stream) {
  const uint64_t pieces = (pool.page_bytes + kPiece - 1) / kPiece;
  if (2 * pool.L * pieces > kMostGroups || (uint64_t)n * (2 * pool.L * pieces) > kMostGroups) return KVC_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(copy_kernel, dim3((uint32_t)(n * 2 * pool.L * pieces)), dim3(256), 0, stream, pool, src, dst, make_fastdiv((uint32_t)pieces),
                     make_fastdiv(2 * pool.L));
  return launched();
}

kvc_status launch_append(const AppendParams& p, hipStream_t stream) {
  const uint64_t vectors = (uint64_t)p.batch.n_new * 2 * p.atoms;
  const bool many = vectors >= 256 * 4 * 512;
  const uint64_t groups = (vectors + (many ? 1023 : 255)) / (many ? 1024 : 256);
  if (groups > kMostGroups) return KVC_ERR_UNSUPPORTED;
  if (many) hipLaunchKernelGGL(append_kernel<4>, dim3((uint32_t)groups), dim3(256), 0, stream, p);
  else hipLaunchKernelGGL(append_kernel<1>, dim3((uint32_t)groups), dim3(256), 0, stream, p);
  return launched();
}

}  // namespace kvc
