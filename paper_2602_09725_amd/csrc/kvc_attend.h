// What the kernels of attention over pages share: who sees what, and which part of the work is whose.
#pragma once

#include <hip/hip_runtime.h>

#include "kvc_device.h"
#include "kvc_serve.h"

namespace kvc {

namespace {

__device__ __forceinline__ void fault(const AttendParams& p, uint32_t bits) {
  if (p.pool.err && bits) atomicOr(p.pool.err, bits);
}

constexpr float kNone = -__builtin_inff();

// exp2(a - b) where a is -inf if b is: 0 then.
__device__ __forceinline__ float weight(float a, float b) { return a == kNone ? 0.0f : __builtin_amdgcn_exp2f(a - b); }

// ---- waits ----------------------------------------------------------------------------------------------------------------

// Waits until the wave's reads of LDS have come back.
__device__ __forceinline__ void wait_reads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("" ::: "memory");
}

// All waves of a workgroup have come here, and their reads of LDS have come back; loads stay under way.
__device__ __forceinline__ void meet() {
  wait_reads();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---- who sees what --------------------------------------------------------------------------------------------------------

struct Request {
  uint32_t row, first, n, len;  // row of the table; first new token, new tokens; tokens (the true length)
  uint32_t faults;
};

// All of a request; what is out of range is told and made harmless.
__device__ __forceinline__ Request request_at(const AttendParams& p, uint32_t r) {
  Request q;
  q.faults = 0;
  q.first = r;
  q.n = 1;
  q.row = p.batch.rows ? (uint32_t)p.batch.rows[r] : r;
  if (p.batch.starts) {
    const uint32_t a = (uint32_t)p.batch.starts[r], b = (uint32_t)p.batch.starts[r + 1];
    q.first = a < p.batch.n_new ? a : p.batch.n_new;
    const uint32_t end = b < p.batch.n_new ? b : p.batch.n_new;
    q.n = end > q.first ? end - q.first : 0;
    if (a > b || b > p.batch.n_new || q.n > p.batch.most_new) q.faults |= KVC_FAULT_LIST;
    if ((r == 0 && a != 0) || (r + 1 == p.batch.n_requests && b != p.batch.n_new)) q.faults |= KVC_FAULT_LIST;
  }
  const bool known = q.row < p.pool.n_rows;
  q.row = known ? q.row : 0;
  q.len = (uint32_t)p.pool.lens[q.row];
  if (!known || q.len > p.most_tokens) q.faults |= KVC_FAULT_LIST;
  if (!known || q.len > 0x7fffffffu) q.len = 0;
  return q;
}

// New tokens of a request that have a result.
__device__ __forceinline__ uint32_t covered(const AttendParams& p, const Request& q) { return min(q.n, p.batch.most_new); }

// Positions that new token t of a request sees: those below this.  (A token whose request does not cover it sees none.)
__device__ __forceinline__ uint32_t limit_of(const AttendParams& p, const Request& q, uint32_t t) {
  if (t - q.first >= covered(p, q)) return 0;
  const int64_t seen = (int64_t)q.len - q.n + (t - q.first) + 1;
  return seen < 0 ? 0 : seen < (int64_t)p.most_tokens ? (uint32_t)seen : p.most_tokens;
}

// Request of new token t.
__device__ __forceinline__ uint32_t request_of(const BatchView& b, uint32_t t) {
  if (!b.starts) return t;
  uint32_t low = 0, high = b.n_requests;
  while (low + 1 < high) {
    const uint32_t mid = (low + high) / 2;
    if ((uint32_t)b.starts[mid] <= t) low = mid;
    else high = mid;
  }
  return low;
}

// Writes the result of new tokens [from, to) for a KV head's query heads: that of rows that see nothing.  self: one of so many threads.
__device__ __forceinline__ void write_none(const AttendParams& p, uint32_t from, uint32_t to, uint32_t head, uint32_t self, uint32_t threads) {
  const uint32_t rows = from < to ? (to - from) * p.G : 0;
  for (uint32_t row = self; row < rows; row += threads) {
    uint32_t t, g;
    fd_divmod(p.dG, row, t, g);
    const uint32_t token = from + t, h = head * p.G + g;
    uint16_t* const out = p.out + (int64_t)token * p.o_token + (int64_t)h * p.o_head;
    for (uint32_t at = 0; at < p.D; at += 8) *(KVC_GLOBAL u32x4*)(out + at) = u32x4{0, 0, 0, 0};
    if (p.lse) p.lse[(uint64_t)token * (p.H * p.G) + h] = kNone;
  }
}

// The new tokens around a request's that no request covers: its own beyond the bound, and those before the first request's and after the last one's.
__device__ __forceinline__ void write_uncovered(const AttendParams& p, const Request& q, uint32_t request, uint32_t head, uint32_t self, uint32_t threads) {
  const uint32_t end = q.first + q.n;
  write_none(p, q.first + covered(p, q), request + 1 == p.batch.n_requests ? p.batch.n_new : end, head, self, threads);
  if (request == 0) write_none(p, 0, q.first, head, self, threads);
}

// Tokens of the shared prefix that there are.
__device__ __forceinline__ uint32_t prefix_there(const AttendParams& p) {
  if (p.prefix == 0) return 0;
  const uint32_t len = (uint32_t)as_const(p.pool.lens)[p.prefix_row];
  return len > p.pool.capacity ? 0 : len < p.prefix ? len : p.prefix;
}

// ---- units ----------------------------------------------------------------------------------------------------------------

// Which part of the work a unit is.
struct Place {
  uint32_t block, split, head, request;
};

__device__ __forceinline__ Place place_of_unit(const AttendParams& p, const AttendPart& part, bool shared, uint32_t unit) {
  Place w;
  uint32_t rest;
  fd_divmod(part.drows, unit, rest, w.block);
  if (!shared) w.block = part.row_blocks - 1 - w.block;  // (of a prompt the last rows see the most, and are begun first)
  fd_divmod(part.dsplits, rest, rest, w.split);
  w.head = rest;
  w.request = 0;
  if (!shared) fd_divmod(part.drequests, rest, w.head, w.request);
  return w;
}

// Workgroups go to the XCDs round-robin.  Each XCD has an eighth of a part's units, which follow one another (blocks of rows of the
// same tokens, then pieces of the same head); the prefix's units, which may be long, are begun first.
__device__ __forceinline__ bool unit_of(const AttendParams& p, bool& shared, uint32_t& unit) {
  const uint32_t front = (p.part[0].units + 7) / 8 * 8;
  shared = blockIdx.x < front;
  const uint32_t units = p.part[shared ? 0 : 1].units, at = shared ? blockIdx.x : blockIdx.x - front;
  unit = (at & 7u) * ((units + 7) / 8) + (at >> 3);
  return unit < units;
}

}  // namespace

}  // namespace kvc
