// Host layer of the serving calls of include/kvc.h: argument checks, workspaces, launches.
#include <hip/hip_runtime.h>

#include <math.h>

#include "kvc_serve.h"

namespace kvc {

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

// Checks a pool and fills the kernels' view of it.
kvc_status view_of(const kvc_pool* p, bool books, PoolView* v) {
  if (!p || p->struct_size != sizeof(kvc_pool) || p->abi_version != KVC_ABI_VERSION) return KVC_ERR_INVALID_ARG;
  if (p->num_layers < 1 || p->num_kv_heads < 1 || p->head_dim < 1) return KVC_ERR_INVALID_ARG;
  if (p->num_blocks < 1 || p->n_rows < 1 || p->block_size < 1 || p->table_len < 1) return KVC_ERR_INVALID_ARG;
  if (p->dtype != KVC_F16 && p->dtype != KVC_BF16) return KVC_ERR_INVALID_ARG;
  if (!p->d_layer_cache || !p->d_tables || !p->d_lens || (books && !p->d_refs)) return KVC_ERR_INVALID_ARG;
  if (!aligned(p->d_layer_cache, 8) || !aligned(p->d_tables, 4) || !aligned(p->d_lens, 4) || !aligned(p->d_refs, 4) || !aligned(p->d_err, 4))
    return KVC_ERR_INVALID_ARG;
  const int64_t C = (int64_t)p->num_kv_heads * p->head_dim;
  if (p->head_dim % 8 != 0 || C > (1 << 20) || p->num_layers > (1 << 20) || p->n_rows >= (1 << 18)) return KVC_ERR_UNSUPPORTED;
  if (p->num_blocks >= (1ll << 31) || p->num_blocks * p->block_size >= (1ll << 32)) return KVC_ERR_UNSUPPORTED;
  if ((int64_t)p->table_len * p->block_size >= (1ll << 31)) return KVC_ERR_UNSUPPORTED;
  v->layers = p->d_layer_cache;
  v->tables = p->d_tables;
  v->lens = p->d_lens;
  v->refs = p->d_refs;
  v->err = p->d_err;
  v->num_blocks = (uint32_t)p->num_blocks;
  v->n_rows = (uint32_t)p->n_rows;
  v->table_len = (uint32_t)p->table_len;
  v->block_size = (uint32_t)p->block_size;
  v->L = (uint32_t)p->num_layers;
  v->capacity = v->table_len * v->block_size;
  v->token_bytes = (uint32_t)(2 * C);
  v->page_bytes = (uint64_t)v->block_size * v->token_bytes;
  v->dbs = make_fastdiv(v->block_size);
  return KVC_OK;
}

// The workspace of fork, grow and compact laid out at `base`; returns its size.
size_t lay_out(const PoolView& v, uint8_t* base, PageSpace* w) {
  size_t at = 0;
  auto take = [&](size_t bytes) {
    uint8_t* p = base ? base + at : nullptr;
    at += (bytes + 255) & ~(size_t)255;
    return p;
  };
  w->segments = (v.num_blocks + kSegment - 1) / kSegment;
  w->head = reinterpret_cast<uint32_t*>(take(kPlanWords * 4));
  w->counts = reinterpret_cast<uint32_t*>(take((size_t)w->segments * 4));
  w->bits = reinterpret_cast<uint32_t*>(take((size_t)w->segments * kSegmentWords * 4));
  w->first = reinterpret_cast<uint32_t*>(take(((size_t)v.n_rows + 1) * 4));
  w->jobs = reinterpret_cast<ForkJob*>(take((size_t)v.n_rows * sizeof(ForkJob)));
  for (int32_t** list : {&w->places, &w->sources, &w->moved, &w->refs}) *list = reinterpret_cast<int32_t*>(take((size_t)v.num_blocks * 4));
  return at;
}

kvc_status space_of(const PoolView& v, void* workspace, size_t bytes, PageSpace* w) {
  if (!workspace || !aligned(workspace, 256)) return KVC_ERR_INVALID_ARG;
  return lay_out(v, static_cast<uint8_t*>(workspace), w) > bytes ? KVC_ERR_BUFFER_TOO_SMALL : KVC_OK;
}

kvc_status view_of(const kvc_batch* b, BatchView* v) {
  if (!b || b->struct_size != sizeof(kvc_batch) || b->abi_version != KVC_ABI_VERSION) return KVC_ERR_INVALID_ARG;
  if (b->n_requests < 0 || b->most_new < 0 || b->n_new < 0 || b->n_new >= (1ll << 31)) return KVC_ERR_INVALID_ARG;
  if (!aligned(b->d_rows, 4) || !aligned(b->d_starts, 4)) return KVC_ERR_INVALID_ARG;
  if (!b->d_starts && b->n_new != b->n_requests) return KVC_ERR_INVALID_ARG;
  if (b->n_new > 0 && (b->n_requests < 1 || b->most_new < 1)) return KVC_ERR_INVALID_ARG;
  if (b->n_new > (int64_t)b->most_new * b->n_requests) return KVC_ERR_INVALID_ARG;
  v->rows = b->d_rows;
  v->starts = b->d_starts;
  v->n_requests = (uint32_t)b->n_requests;
  v->n_new = (uint32_t)b->n_new;
  v->most_new = !b->d_starts ? 1 : (uint32_t)(b->most_new < b->n_new ? b->most_new : b->n_new);
  return KVC_OK;
}

// Checks an attention call but for its pointers and plans it.
kvc_status plan_of(const kvc_pool* pool, const kvc_batch* batch, const kvc_attention* a, AttendParams* p) {
  kvc_status st = view_of(pool, false, &p->pool);
  if (st != KVC_OK) return st;
  if ((st = view_of(batch, &p->batch)) != KVC_OK) return st;
  if (!a || a->struct_size != sizeof(kvc_attention) || a->abi_version != KVC_ABI_VERSION) return KVC_ERR_INVALID_ARG;
  if (a->num_q_heads < 1 || a->num_q_heads % pool->num_kv_heads != 0) return KVC_ERR_INVALID_ARG;
  if (!(a->scale > 0.0f) || !isfinite(a->scale)) return KVC_ERR_INVALID_ARG;
  if (a->most_tokens < 0 || a->most_tokens > (int64_t)p->pool.capacity) return KVC_ERR_INVALID_ARG;
  if (a->prefix_tokens < 0 || a->prefix_tokens > a->most_tokens) return KVC_ERR_INVALID_ARG;
  if (a->prefix_row < 0 || a->prefix_row >= pool->n_rows) return KVC_ERR_INVALID_ARG;
  for (int64_t s : {a->q_token_stride, a->q_head_stride, a->out_token_stride, a->out_head_stride})
    if (s < 0 || s % 8 != 0) return KVC_ERR_INVALID_ARG;
  if (pool->head_dim > 256) return KVC_ERR_UNSUPPORTED;
  const int64_t group = a->num_q_heads / pool->num_kv_heads;
  if (batch->n_new * group >= (1ll << 31) - 128 || batch->n_new * a->num_q_heads >= (1ll << 31)) return KVC_ERR_UNSUPPORTED;
  p->q_token = a->q_token_stride;
  p->q_head = a->q_head_stride;
  p->o_token = a->out_token_stride;
  p->o_head = a->out_head_stride;
  p->H = (uint32_t)pool->num_kv_heads;
  p->G = (uint32_t)group;
  p->D = (uint32_t)pool->head_dim;
  p->dtype = (uint32_t)pool->dtype;
  p->prefix = (uint32_t)a->prefix_tokens;
  p->prefix_row = (uint32_t)a->prefix_row;
  p->most_tokens = (uint32_t)a->most_tokens;
  p->dG = make_fastdiv(p->G);
  p->scale_log2 = (float)((double)a->scale * 1.4426950408889634);
  return batch->n_new == 0 ? KVC_OK : plan_attend(*p);
}

// Bytes of the joined pieces' sums, and in all.
size_t attend_space(const AttendParams& p, size_t* sums) {
  const size_t lines = p.pieces > 1 ? (size_t)p.pieces * p.batch.n_new * p.H * p.G : 0;
  *sums = (lines * p.D * 4 + 255) & ~(size_t)255;
  return *sums + lines * 8;
}

}  // namespace

}  // namespace kvc

using namespace kvc;

extern "C" {

kvc_status kvc_pool_validate(const kvc_pool* pool) {
  PoolView v{};
  return view_of(pool, false, &v);
}

size_t kvc_pages_workspace(const kvc_pool* pool) {
  PoolView v{};
  PageSpace w{};
  return view_of(pool, false, &v) == KVC_OK ? lay_out(v, nullptr, &w) : 0;
}

kvc_status kvc_pages_copy(const kvc_pool* pool, const int32_t* d_src, const int32_t* d_dst, int64_t n, void* stream) {
  PoolView v{};
  const kvc_status st = view_of(pool, false, &v);
  if (st != KVC_OK) return st;
  if (n < 0 || n >= (1ll << 31)) return KVC_ERR_INVALID_ARG;
  if (n == 0) return KVC_OK;
  if (!d_src || !d_dst || !aligned(d_src, 4) || !aligned(d_dst, 4)) return KVC_ERR_INVALID_ARG;
  return launch_copy_pages(v, d_src, d_dst, (uint32_t)n, as_stream(stream));
}

kvc_status kvc_pages_fork(const kvc_pool* pool, const int32_t* d_parents, const int32_t* d_children, int64_t n, void* workspace,
                          size_t workspace_bytes, void* stream) {
  PoolView v{};
  PageSpace w{};
  kvc_status st = view_of(pool, true, &v);
  if (st != KVC_OK) return st;
  if (n < 0 || n > v.n_rows) return KVC_ERR_INVALID_ARG;
  if (n == 0) return KVC_OK;
  if (!d_parents || !d_children || !aligned(d_parents, 4) || !aligned(d_children, 4)) return KVC_ERR_INVALID_ARG;
  if ((st = space_of(v, workspace, workspace_bytes, &w)) != KVC_OK) return st;
  return launch_fork(v, w, d_parents, d_children, (uint32_t)n, as_stream(stream));
}

kvc_status kvc_pages_grow(const kvc_pool* pool, const int32_t* d_rows, const int32_t* d_counts, int64_t n, void* workspace,
                          size_t workspace_bytes, void* stream) {
  PoolView v{};
  PageSpace w{};
  kvc_status st = view_of(pool, true, &v);
  if (st != KVC_OK) return st;
  if (n < 0 || n > v.n_rows) return KVC_ERR_INVALID_ARG;
  if (n == 0) return KVC_OK;
  if (!d_rows || !aligned(d_rows, 4) || !aligned(d_counts, 4)) return KVC_ERR_INVALID_ARG;
  if ((st = space_of(v, workspace, workspace_bytes, &w)) != KVC_OK) return st;
  return launch_grow(v, w, d_rows, d_counts, (uint32_t)n, as_stream(stream));
}

kvc_status kvc_pages_free(const kvc_pool* pool, const int32_t* d_rows, int64_t n, void* stream) {
  PoolView v{};
  const kvc_status st = view_of(pool, true, &v);
  if (st != KVC_OK) return st;
  if (n < 0 || n >= (1ll << 31) - 4) return KVC_ERR_INVALID_ARG;
  if (n == 0) return KVC_OK;
  if (!d_rows || !aligned(d_rows, 4)) return KVC_ERR_INVALID_ARG;
  return launch_free(v, d_rows, (uint32_t)n, as_stream(stream));
}

kvc_status kvc_pages_compact(const kvc_pool* pool, int32_t* d_map, int32_t* d_tables_out, int32_t* d_refs_out, void* workspace,
                             size_t workspace_bytes, void* stream) {
  PoolView v{};
  PageSpace w{};
  kvc_status st = view_of(pool, true, &v);
  if (st != KVC_OK) return st;
  if (!d_map || !d_tables_out || !d_refs_out) return KVC_ERR_INVALID_ARG;
  if (!aligned(d_map, 4) || !aligned(d_tables_out, 4) || !aligned(d_refs_out, 4)) return KVC_ERR_INVALID_ARG;
  if ((st = space_of(v, workspace, workspace_bytes, &w)) != KVC_OK) return st;
  return launch_compact(v, w, d_map, d_tables_out, d_refs_out, as_stream(stream));
}

kvc_status kvc_append_paged(const kvc_pool* pool, const kvc_batch* batch, int32_t layer, const void* k, const void* v,
                            int64_t token_stride, void* stream) {
  AppendParams p{};
  kvc_status st = view_of(pool, false, &p.pool);
  if (st != KVC_OK) return st;
  if ((st = view_of(batch, &p.batch)) != KVC_OK) return st;
  if (layer < 0 || layer >= pool->num_layers) return KVC_ERR_INVALID_ARG;
  if (batch->n_new == 0) return KVC_OK;
  if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) return KVC_ERR_INVALID_ARG;
  if (token_stride < 0 || token_stride % 8 != 0) return KVC_ERR_INVALID_ARG;
  p.k = static_cast<const uint16_t*>(k);
  p.v = static_cast<const uint16_t*>(v);
  p.token_stride = token_stride;
  p.layer = (uint32_t)layer;
  p.atoms = p.pool.token_bytes / 16;
  p.datoms = make_fastdiv(p.atoms);
  return launch_append(p, as_stream(stream));
}

size_t kvc_attention_workspace(const kvc_pool* pool, const kvc_batch* batch, const kvc_attention* attention) {
  AttendParams p{};
  size_t sums;
  return plan_of(pool, batch, attention, &p) == KVC_OK ? attend_space(p, &sums) : (size_t)-1;
}

kvc_status kvc_attend_paged(const kvc_pool* pool, const kvc_batch* batch, const kvc_attention* attention, int32_t layer, const void* q,
                            void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  AttendParams p{};
  const kvc_status st = plan_of(pool, batch, attention, &p);
  if (st != KVC_OK) return st;
  if (layer < 0 || layer >= pool->num_layers) return KVC_ERR_INVALID_ARG;
  if (batch->n_new == 0) return KVC_OK;
  if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4)) return KVC_ERR_INVALID_ARG;
  size_t sums;
  const size_t bytes = attend_space(p, &sums);
  if (bytes) {
    if (!workspace || !aligned(workspace, 256)) return KVC_ERR_INVALID_ARG;
    if (bytes > workspace_bytes) return KVC_ERR_BUFFER_TOO_SMALL;
    p.sums = static_cast<float*>(workspace);
    p.tops = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + sums);
  }
  p.layer = (uint32_t)layer;
  p.q = static_cast<const uint16_t*>(q);
  p.out = static_cast<uint16_t*>(out);
  p.lse = lse;
  return launch_attend(p, as_stream(stream));
}

}  // extern "C"
