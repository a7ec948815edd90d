// Entry points of the calls that write rows with their positions' rotation, keep the bounds of blocks
// and attend to selected blocks (include/fastcache.h).  Nothing is queued before everything has
// been checked.

#include "fc_call.h"

using namespace fc;

namespace {

// The layer, the tables and the chunks of a call on the pool; 1: there is nothing to do.
int plan_call(const fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks, const int32_t* host_seq_lens,
              const int32_t* host_n_new, int n_req, ChunkPlan* plan) {
  if (layer < 0 || layer >= p->n_layers) return fail(FC_EINVAL, "layer %d outside 0..%d", layer, p->n_layers - 1);
  if (n_req > 0 && (!dev_block_tables || !host_n_new)) return fail(FC_EINVAL, "NULL argument");
  if (n_req > 0 && max_blocks < 1) return fail(FC_EINVAL, "max_blocks_per_req < 1");
  if (plan_chunk(n_req, max_blocks, host_seq_lens, host_n_new, plan) != PLAN_OK) return fail(plan->code, "%s", plan->message);
  return plan->reqs.empty() ? 1 : FC_OK;
}

int check_aligned(const void* at, size_t to, const char* name) {
  if (!at) return fail(FC_EINVAL, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(at) & (to - 1)) return fail(FC_EINVAL, "%s must be %zu-byte aligned", name, to);
  return FC_OK;
}

size_t bounds_elems(const fc_pool* p) { return (size_t)p->n_blocks * p->n_heads * 2 * p->head_dim; }  // of a layer

// What a selection and an attention of its blocks have in common.
void set_selection(const fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks, const void* dev_bounds, int n_select,
                   const fc_rows* q, int n_q_heads, int32_t* dev_selected, const SparsePlan& plan, SelectParams* sp) {
  sp->bounds = static_cast<const _Float16*>(dev_bounds) + (size_t)layer * bounds_elems(p);
  sp->n_blocks = p->n_blocks;
  sp->n_heads = p->n_heads;
  sp->group = n_q_heads / p->n_heads;
  sp->head_dim = p->head_dim;
  sp->block_tables = dev_block_tables;
  sp->max_blocks = max_blocks;
  sp->n_tokens = (int)plan.tokens.size();
  sp->q = view(q);
  sp->n_select = n_select;
  sp->selected = dev_selected;
  sp->lds_keys = plan.longest;
}

// Scores, selection and attention, a launch each.
int select_then_attend(fc_pool* p, SparsePlan* plan, int n_q_heads, SelectParams* sp, AttnParams* ap, hipStream_t stream) {
  AttnLaunch launches[ATTN_KINDS];
  if (plan_attention(geometry(p), p->n_cu, sp->group, true, p->max_states, &plan->attention, launches, p->dtype == FC_DTYPE_E2M1) != PLAN_OK)
    return fail(plan->attention.code, "%s", plan->attention.message);
  // (what may grow grows before the descriptors are on their way)
  int rc;
  const size_t heads = plan->tokens.size() * p->n_heads;
  const size_t score_bytes = heads * plan->longest * sizeof(float), most_bytes = (size_t)plan->n_units * p->n_heads * sizeof(uint32_t);
  if ((rc = scratch_for(p, &p->sparse, score_bytes + most_bytes + heads * sp->n_select * sizeof(int32_t), stream))) return rc;
  std::vector<ChunkReq> reqs(plan->tokens);
  const std::vector<ChunkReq> attended = attention_reqs(launches);
  ChunkReqs token_reqs, scored_reqs, attention_inline;
  if (reqs.size() <= ChunkReqs::kInline) {
    std::copy(reqs.begin(), reqs.end(), token_reqs.req);
    std::copy(plan->scored.begin(), plan->scored.end(), scored_reqs.req);
    std::copy(attended.begin(), attended.end(), attention_inline.req);
  } else {
    reqs.insert(reqs.end(), attended.begin(), attended.end());
    reqs.insert(reqs.end(), plan->scored.begin(), plan->scored.end());
    const void* at = nullptr;
    if ((rc = meta_to_device(p, reqs.data(), reqs.size() * sizeof(ChunkReq), &at, stream))) return rc;
    sp->tokens = static_cast<const ChunkReq*>(at);
    ap->reqs = sp->tokens + plan->tokens.size();
    sp->reqs = ap->reqs + attended.size();
  }
  sp->scores = reinterpret_cast<float*>(p->sparse.data);
  sp->most = reinterpret_cast<uint32_t*>(p->sparse.data + score_bytes);
  sp->ids = reinterpret_cast<int32_t*>(p->sparse.data + score_bytes + most_bytes);
  sp->part_blocks = plan->part_blocks;
  sp->tile_tokens = plan->tile_tokens;
  sp->n_req = (int)plan->scored.size();
  sp->n_units = (int)plan->n_units;
  sp->score_stride = plan->longest;
  FC_HIP(launch_select_blocks(*sp, token_reqs, scored_reqs, stream));
  ap->block_tables = sp->ids;
  ap->max_blocks = sp->n_select;
  ap->table_heads = p->n_heads;
  set_launches(p, launches, n_q_heads, ap);
  FC_HIP(launch_attention(*ap, attention_inline, stream));
  return FC_OK;
}

int sparse_attention(fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks, const ChunkPlan& chunk,
                     const void* dev_bounds, int n_select, const fc_rows* q, int n_q_heads, const fc_rows* out,
                     int32_t* dev_selected, float scale, hipStream_t stream) {
  int rc;
  if ((rc = check_q_heads(p, n_q_heads)) || (rc = check_aligned(dev_bounds, 16, "dev_bounds"))) return rc;
  if (reinterpret_cast<uintptr_t>(dev_selected) & 3) return fail(FC_EINVAL, "dev_selected must be 4-byte aligned");
  SparsePlan plan;
  if (plan_sparse(geometry(p), p->n_cu, n_q_heads / p->n_heads, n_select, chunk, &plan) != PLAN_OK) return fail(plan.code, "%s", plan.message);
  if ((rc = check_rows(q, "q", chunk.n_rows, n_q_heads, p->head_dim, false)) ||
      (rc = check_rows(out, "out", chunk.n_rows, n_q_heads, p->head_dim, true)))
    return rc;
  SelectParams sp = {};
  set_selection(p, layer, dev_block_tables, max_blocks, dev_bounds, n_select, q, n_q_heads, dev_selected, plan, &sp);
  AttnParams ap = {};
  ap.kv = layer_blocks(p, layer);
  ap.source = p->dtype == FC_DTYPE_E4M3 ? ATTN_E4M3 : p->dtype == FC_DTYPE_E2M1 ? ATTN_E2M1 : ATTN_F16;
  set_queries(p, q, out, n_q_heads, scale, &ap);
  if (plan.part_blocks) return select_then_attend(p, &plan, n_q_heads, &sp, &ap, stream);
  ChunkReqs token_reqs;
  if ((rc = pass_reqs(p, plan.tokens, &token_reqs, &sp.tokens, stream))) return rc;
  FC_HIP(launch_selected_attention(sp, ap, token_reqs, stream));
  return FC_OK;
}

}  // namespace

extern "C" {

int fc_rotate_store_chunk(fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks_per_req,
                          const int32_t* host_seq_lens, const int32_t* host_n_new, const int32_t* host_positions,
                          const fc_rotation* rotation, const fc_rows* q, int n_q_heads, const fc_rows* q_out, const fc_rows* k,
                          const fc_rows* v, int n_req, void* stream_) {
  return guarded("fc_rotate_store_chunk", [&]() -> int {
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    FC_CHECK_POOL(p);
    ChunkPlan plan;
    int rc = plan_call(p, layer, dev_block_tables, max_blocks_per_req, host_seq_lens, host_n_new, n_req, &plan);
    if (rc) return rc < 0 ? rc : FC_OK;
    if (!rotation) return fail(FC_EINVAL, "rotation is NULL");
    if ((rc = check_aligned(rotation->table, 16, "the rotation's table"))) return rc;
    if (rotation->rotary_dim < 16 || rotation->rotary_dim > p->head_dim || rotation->rotary_dim % 16)
      return fail(FC_EINVAL, "rotary_dim %d: a multiple of 16, at most head_dim", rotation->rotary_dim);
    if (rotation->n_positions < 1) return fail(FC_EINVAL, "n_positions < 1");
    if (n_q_heads < 0 || n_q_heads > p->n_heads * (int64_t)FC_MAX_GROUP) return fail(FC_EINVAL, "n_q_heads %d", n_q_heads);
    if ((rc = check_rows(k, "k", plan.n_rows, p->n_heads, p->head_dim, false)) ||
        (rc = check_rows(v, "v", plan.n_rows, p->n_heads, p->head_dim, false)))
      return rc;
    if (n_q_heads > 0 && ((rc = check_rows(q, "q", plan.n_rows, n_q_heads, p->head_dim, false)) ||
                          (rc = check_rows(q_out, "q_out", plan.n_rows, n_q_heads, p->head_dim, true))))
      return rc;
    if (plan_positions(host_positions, rotation->n_positions, &plan) != PLAN_OK || plan_store_units(&plan) != PLAN_OK)
      return fail(plan.code, "%s", plan.message);
    RotateParams rp = {};
    ChunkReqs inline_reqs;
    if ((rc = pass_reqs(p, plan.reqs, &inline_reqs, &rp.store.reqs, stream))) return rc;
    rp.store.kv = layer_blocks(p, layer);
    rp.store.e4m3 = row_format(p);
    rp.store.n_blocks = p->n_blocks;
    rp.store.n_heads = p->n_heads;
    rp.store.head_dim = p->head_dim;
    rp.store.block_tables = dev_block_tables;
    rp.store.max_blocks = max_blocks_per_req;
    rp.store.n_req = (int)plan.reqs.size();
    rp.store.n_rows = (int)plan.n_rows;
    rp.store.k = view(k);
    rp.store.v = view(v);
    if (n_q_heads > 0) {
      rp.q = view(q);
      rp.q_out = view(q_out);
    }
    rp.n_q_heads = n_q_heads;
    rp.table = rotation->table;
    rp.rotary = rotation->rotary_dim;
    rp.interleaved = rotation->interleaved ? 1 : 0;
    FC_HIP(launch_rotate_store(rp, inline_reqs, stream));
    return FC_OK;
  });
}

int fc_block_bounds(fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks_per_req,
                    const int32_t* host_seq_lens, const int32_t* host_n_new, void* dev_bounds, int n_req, void* stream_) {
  return guarded("fc_block_bounds", [&]() -> int {
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    FC_CHECK_POOL(p);
    ChunkPlan plan;
    int rc = plan_call(p, layer, dev_block_tables, max_blocks_per_req, host_seq_lens, host_n_new, n_req, &plan);
    if (rc) return rc < 0 ? rc : FC_OK;
    if ((rc = check_aligned(dev_bounds, 16, "dev_bounds"))) return rc;
    if (plan_bounds(&plan) != PLAN_OK) return fail(plan.code, "%s", plan.message);
    BoundsParams bp = {};
    ChunkReqs inline_reqs;
    if ((rc = pass_reqs(p, plan.reqs, &inline_reqs, &bp.reqs, stream))) return rc;
    bp.kv = layer_blocks(p, layer);
    bp.format = row_format(p);
    bp.n_blocks = p->n_blocks;
    bp.n_heads = p->n_heads;
    bp.head_dim = p->head_dim;
    bp.block_tables = dev_block_tables;
    bp.max_blocks = max_blocks_per_req;
    bp.n_req = (int)plan.reqs.size();
    bp.n_units = (int)plan.n_rows;
    bp.bounds = static_cast<_Float16*>(dev_bounds) + (size_t)layer * bounds_elems(p);
    FC_HIP(launch_bounds(bp, inline_reqs, stream));
    return FC_OK;
  });
}

int fc_sparse_attention(fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks_per_req,
                        const int32_t* host_seq_lens, const int32_t* host_n_new, const void* dev_bounds, int n_select,
                        const fc_rows* q, int n_q_heads, const fc_rows* out, int32_t* dev_selected, int n_req, float scale,
                        void* stream) {
  return guarded("fc_sparse_attention", [&]() -> int {
    FC_CHECK_POOL(p);
    ChunkPlan plan;
    const int rc = plan_call(p, layer, dev_block_tables, max_blocks_per_req, host_seq_lens, host_n_new, n_req, &plan);
    if (rc) return rc < 0 ? rc : FC_OK;
    return sparse_attention(p, layer, dev_block_tables, max_blocks_per_req, plan, dev_bounds, n_select, q, n_q_heads, out,
                            dev_selected, scale, static_cast<hipStream_t>(stream));
  });
}

}  // extern "C"
