// What the planner of attention over pools in 4 bits makes of a call, for tests that have to know which body they meet.
#include "kvc_serve.h"

namespace {

struct Part {
  int32_t waves, splits, lone, tokens;
};
struct Plan {
  int32_t pieces;
  Part part[2];
};

}  // namespace

extern "C" int held_plan(const kvc_pool* pool, const kvc_batch* batch, const kvc_attention* a, Plan* to) {
  kvc::AttendParams p{};
  p.H = (uint32_t)pool->num_kv_heads;
  p.G = (uint32_t)(a->num_q_heads / pool->num_kv_heads);
  p.D = (uint32_t)pool->head_dim;
  p.dtype = (uint32_t)(pool->dtype & ~KVC_HELD_Q4);
  p.pool.num_blocks = (uint32_t)pool->num_blocks;
  p.pool.page_bytes = kvc_page_bytes(pool);
  p.pool.held = 4;
  p.batch.n_requests = (uint32_t)batch->n_requests;
  p.batch.n_new = (uint32_t)batch->n_new;
  p.batch.most_new = !batch->d_starts ? 1 : (uint32_t)(batch->most_new < batch->n_new ? batch->most_new : batch->n_new);
  p.prefix = (uint32_t)a->prefix_tokens;
  p.most_tokens = (uint32_t)a->most_tokens;
  const int status = kvc::plan_attend_held(p);
  to->pieces = (int32_t)p.pieces;
  for (int i = 0; i < 2; ++i) to->part[i] = Part{(int32_t)p.part[i].waves, (int32_t)p.part[i].splits, (int32_t)p.part[i].lone, (int32_t)p.part[i].tokens};
  return status;
}
