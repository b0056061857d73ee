// Parameter blocks of the serving kernels (pages, appended tokens, attention over pages) and their launch functions.
#pragma once

#include <hip/hip_runtime.h>

#include "kvc_common.h"

namespace kvc {

// Workgroups of 256 threads that a launch can have: fewer than 2^32 threads.
constexpr uint64_t kMostGroups = (1ull << 24) - 1;

// The pool as the kernels see it.
struct PoolView {
  void* const* layers;
  int32_t *tables, *lens, *refs;
  uint32_t* err;
  uint32_t num_blocks, n_rows, table_len, block_size, L;
  uint32_t capacity;      // tokens of a row
  uint32_t token_bytes;   // of one token, layer and kind
  uint64_t page_bytes;    // of one page, layer and kind
  FastDiv dbs;
};

// Books are surveyed in segments of this many pages: for each of them the number of free ones, and a bit for each page.
constexpr uint32_t kSegment = 4096, kSegmentWords = kSegment / 32;
// Pools of up to this many pages are surveyed by one workgroup.
constexpr uint32_t kOnePages = 16384;

struct ForkJob {
  uint32_t from, to, tokens, len;  // pages, tokens that are copied, tokens of the parent
};

// The workspace of fork, grow and compact.
struct PageSpace {
  uint32_t* head;    // kPlan*
  uint32_t* counts;  // [segments] free pages
  uint32_t* bits;    // [segments][kSegmentWords] 1: free
  uint32_t* first;   // [n_rows + 1] pages that the entries of the list before this one take
  ForkJob* jobs;     // [n_rows] fork of a small pool
  int32_t *places, *sources, *moved, *refs;  // compact, [num_blocks] each
  uint32_t segments;
};
enum { kPlanFaults = 0, kPlanNeed = 1, kPlanUsed = 2, kPlanMoves = 3, kPlanWords = 64 };

enum class PageList { kNone, kFork, kGrow };

kvc_status launch_fork(const PoolView& pool, const PageSpace& w, const int32_t* parents, const int32_t* children, uint32_t n,
                       hipStream_t stream);
kvc_status launch_grow(const PoolView& pool, const PageSpace& w, const int32_t* rows, const int32_t* counts, uint32_t n,
                       hipStream_t stream);
kvc_status launch_free(const PoolView& pool, const int32_t* rows, uint32_t n, hipStream_t stream);
kvc_status launch_compact(const PoolView& pool, const PageSpace& w, int32_t* map, int32_t* tables, int32_t* refs, hipStream_t stream);
kvc_status launch_copy_pages(const PoolView& pool, const int32_t* src, const int32_t* dst, uint32_t n, hipStream_t stream);

// The tokens of a step as the kernels see them.
struct BatchView {
  const int32_t *rows, *starts;  // either may be null
  uint32_t n_requests, n_new, most_new;
};

struct AppendParams {
  PoolView pool;
  BatchView batch;
  const uint16_t *k, *v;
  int64_t token_stride;
  uint32_t layer, atoms;  // atoms: vectors of 8 elements of a token and kind
  FastDiv datoms;
};
kvc_status launch_append(const AppendParams& p, hipStream_t stream);

// One of the two parts of an attention call: the shared prefix, or the rows' own tokens.
struct AttendPart {
  uint32_t waves;       // waves of a workgroup that stand side by side along the rows: 1 or 4
  uint32_t row_blocks;  // blocks of 32 * waves rows
  uint32_t splits;      // pieces of the tokens, 0: the part is empty
  uint32_t tokens;      // of a piece
  uint32_t units;       // workgroups
  uint32_t lone;        // units in all, a wave each; 0: a workgroup each
  FastDiv drows, dsplits, drequests, dtokens;
};

struct AttendParams {
  PoolView pool;
  BatchView batch;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t q_token, q_head, o_token, o_head;
  uint32_t layer, H, G, D, dtype;
  uint32_t prefix, prefix_row, most_tokens;
  uint32_t own_from;    // first token of the rows' own part: the prefix's end, or 0 where each row's tokens are one sequence
  FastDiv dG, dheads;   // dheads: query heads
  AttendPart part[2];   // prefix, own
  float scale_log2;
  float slack;          // products that exceed a row's base by no more than this leave it as it is
  float lift;           // a base that is moved comes to lie this much below the product that moved it
  uint32_t pieces;      // results of a row that are joined afterwards; 1: the row is written at once; 0: nobody sees anything
  float *sums, *tops;   // [pieces][n_new][heads][D] unnormalized sums, [pieces][n_new][heads][2] {maximum (log2), sum of weights}
};

// Splits the work (everything but the pointers is set); launch_attend needs what it returns.
kvc_status plan_attend(AttendParams& p);
kvc_status launch_attend(const AttendParams& p, hipStream_t stream);

}  // namespace kvc
