// Entry points of the calls on chunks of new tokens and whole prompts and of the copy into a
// pool of fewer bits (include/fastcache.h).  Validation and descriptors as in fc_api.hip: nothing is
// queued or changed before everything has been checked.

#include "fc_call.h"

#include <string.h>

using namespace fc;

namespace {

// k and v: packed rows, or NULL for the cache in the pool.
int attention(fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks, const int32_t* host_seq_lens,
              const int32_t* host_n_new, const fc_rows* q, const fc_rows* k, const fc_rows* v, int n_q_heads,
              const fc_rows* out, float* dev_lse, int window, int n_req, float scale, hipStream_t stream) {
  const bool paged = !k;
  if (layer < 0 || layer >= p->n_layers) return fail(FC_EINVAL, "layer %d outside 0..%d", layer, p->n_layers - 1);
  if (int rc = check_q_heads(p, n_q_heads)) return rc;
  if (window < 0 || (dev_lse && window < 1)) return fail(FC_EINVAL, "window %d", window);
  if (reinterpret_cast<uintptr_t>(dev_lse) & 3) return fail(FC_EINVAL, "dev_lse must be 4-byte aligned");
  ChunkPlan plan;
  if (plan_chunk(n_req, paged ? max_blocks : -1, host_seq_lens, host_n_new, &plan) != PLAN_OK)
    return fail(plan.code, "%s", plan.message);
  if (plan.reqs.empty()) return FC_OK;
  int rc;
  if ((rc = check_rows(q, "q", plan.n_rows, n_q_heads, p->head_dim, false)) ||
      (rc = check_rows(out, "out", plan.n_rows, n_q_heads, p->head_dim, true)))
    return rc;
  if (!paged && ((rc = check_rows(k, "k", plan.n_rows, p->n_heads, p->head_dim, false)) ||
                 (rc = check_rows(v, "v", plan.n_rows, p->n_heads, p->head_dim, false))))
    return rc;
  AttnLaunch launches[ATTN_KINDS];
  if (plan_attention(geometry(p), p->n_cu, n_q_heads / p->n_heads, paged, p->max_states, &plan, launches, p->dtype == FC_DTYPE_E2M1) != PLAN_OK)
    return fail(plan.code, "%s", plan.message);

  AttnParams ap = {};
  ap.kv = paged ? layer_blocks(p, layer) : nullptr;
  ap.source = !paged ? ATTN_ROWS : p->dtype == FC_DTYPE_E4M3 ? ATTN_E4M3 : p->dtype == FC_DTYPE_E2M1 ? ATTN_E2M1 : ATTN_F16;
  set_queries(p, q, out, n_q_heads, scale, &ap);
  ap.block_tables = dev_block_tables;
  ap.max_blocks = max_blocks;
  ap.table_heads = 1;
  if (!paged) {
    ap.k = view(k);
    ap.v = view(v);
  }
  ap.window = window;
  if (dev_lse) {
    ap.lse = dev_lse + (int64_t)layer * n_q_heads * window;
    ap.lse_stride = (int64_t)p->n_layers * n_q_heads * window;
  }
  ChunkReqs inline_reqs;
  if ((rc = pass_reqs(p, attention_reqs(launches), &inline_reqs, &ap.reqs, stream))) return rc;
  set_launches(p, launches, n_q_heads, &ap);
  FC_HIP(launch_attention(ap, inline_reqs, stream));
  return FC_OK;
}

}  // namespace

extern "C" {

int fc_extend_batch(fc_pool* p, int32_t* dev_block_tables, int max_blocks_per_req, int32_t* host_seq_lens,
                    const int32_t* host_n_new, int n_req, void* stream_) {
  return guarded("fc_extend_batch", [&]() -> int {
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    FC_CHECK_POOL(p);
    if (n_req > 0 && !dev_block_tables) return fail(FC_EINVAL, "NULL argument");
    ExtendPlan plan;
    if (plan_extend(geometry(p), n_req, max_blocks_per_req, host_seq_lens, host_n_new, &plan) != PLAN_OK)
      return fail(plan.code, "%s", plan.message);
    if (!plan.reqs.empty()) {
      ExtendParams ep = {};
      ExtendReqs inline_reqs;
      if (int rc = pass_reqs(p, plan.reqs, &inline_reqs, &ep.reqs, stream)) return rc;
      ep.stack = p->stack;
      ep.top_before = p->top;
      ep.n_blocks = p->n_blocks;
      ep.block_tables = dev_block_tables;
      ep.max_blocks = max_blocks_per_req;
      ep.n_req = (int)plan.reqs.size();
      ep.owner = p->debug_checks ? p->owner : nullptr;
      ep.error_flag = p->error_flag;
      FC_HIP_STAGE(p, launch_extend(ep, inline_reqs, stream));
      p->top -= plan.n_pop;
    }
    for (int r = 0; r < n_req; ++r) host_seq_lens[r] += host_n_new[r];
    return FC_OK;
  });
}

int fc_store_chunk(fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks_per_req,
                   const int32_t* host_seq_lens, const int32_t* host_n_new, const fc_rows* k, const fc_rows* v,
                   int n_req, void* stream_) {
  return guarded("fc_store_chunk", [&]() -> int {
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    FC_CHECK_POOL(p);
    if (layer < 0 || layer >= p->n_layers) return fail(FC_EINVAL, "layer %d outside 0..%d", layer, p->n_layers - 1);
    if (n_req > 0 && (!dev_block_tables || !host_n_new)) return fail(FC_EINVAL, "NULL argument");
    if (n_req > 0 && max_blocks_per_req < 1) return fail(FC_EINVAL, "max_blocks_per_req < 1");
    ChunkPlan plan;
    if (plan_chunk(n_req, max_blocks_per_req, host_seq_lens, host_n_new, &plan) != PLAN_OK)
      return fail(plan.code, "%s", plan.message);
    if (plan.reqs.empty()) return FC_OK;
    int rc;
    if ((rc = check_rows(k, "k", plan.n_rows, p->n_heads, p->head_dim, false)) ||
        (rc = check_rows(v, "v", plan.n_rows, p->n_heads, p->head_dim, false)))
      return rc;
    if (plan_store_units(&plan) != PLAN_OK) return fail(plan.code, "%s", plan.message);
    StoreParams sp = {};
    ChunkReqs inline_reqs;
    if ((rc = pass_reqs(p, plan.reqs, &inline_reqs, &sp.reqs, stream))) return rc;
    sp.kv = layer_blocks(p, layer);
    sp.e4m3 = row_format(p);
    sp.n_blocks = p->n_blocks;
    sp.n_heads = p->n_heads;
    sp.head_dim = p->head_dim;
    sp.block_tables = dev_block_tables;
    sp.max_blocks = max_blocks_per_req;
    sp.n_req = (int)plan.reqs.size();
    sp.n_rows = (int)plan.n_rows;
    sp.k = view(k);
    sp.v = view(v);
    FC_HIP(launch_store_chunk(sp, inline_reqs, stream));
    return FC_OK;
  });
}

int fc_chunk_attention(fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks_per_req,
                       const int32_t* host_seq_lens, const int32_t* host_n_new, const fc_rows* q, int n_q_heads,
                       const fc_rows* out, float* dev_lse, int window, int n_req, float scale, void* stream) {
  return guarded("fc_chunk_attention", [&]() -> int {
    FC_CHECK_POOL(p);
    if (n_req > 0 && (!dev_block_tables || !host_n_new)) return fail(FC_EINVAL, "NULL argument");
    if (n_req > 0 && max_blocks_per_req < 1) return fail(FC_EINVAL, "max_blocks_per_req < 1");
    return attention(p, layer, dev_block_tables, max_blocks_per_req, host_seq_lens, host_n_new, q, nullptr, nullptr,
                     n_q_heads, out, dev_lse, window, n_req, scale, static_cast<hipStream_t>(stream));
  });
}

int fc_prefill_attention(fc_pool* p, int layer, const int32_t* host_seq_lens, const fc_rows* q, const fc_rows* k,
                         const fc_rows* v, int n_q_heads, const fc_rows* out, float* dev_lse, int window, int n_req,
                         float scale, void* stream) {
  return guarded("fc_prefill_attention", [&]() -> int {
    FC_CHECK_POOL(p);
    if (n_req > 0 && (!k || !v)) return fail(FC_EINVAL, "NULL argument");
    const fc_rows none = {nullptr, 0, 0};
    return attention(p, layer, nullptr, 0, host_seq_lens, nullptr, q, k ? k : &none, v ? v : &none, n_q_heads, out,
                     dev_lse, window, n_req, scale, static_cast<hipStream_t>(stream));
  });
}

int fc_quantise_batch(fc_pool* dst, const int32_t* dev_dst_tables, int dst_max_blocks_per_req, fc_pool* src,
                      const int32_t* dev_src_tables, int src_max_blocks_per_req, const int32_t* host_seq_lens,
                      const int32_t* host_enable, int n_req, void* stream_) {
  return guarded("fc_quantise_batch", [&]() -> int {
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    FC_CHECK_POOL(dst);
    FC_CHECK_POOL(src);
    if ((dst->dtype != FC_DTYPE_E4M3 && dst->dtype != FC_DTYPE_E2M1) || src->dtype != FC_DTYPE_F16)
      return fail(FC_EINVAL, "fc_quantise_batch reads a pool of FC_DTYPE_F16 and writes one of FC_DTYPE_E4M3 or FC_DTYPE_E2M1");
    if (dst->n_layers != src->n_layers || dst->n_heads != src->n_heads || dst->head_dim != src->head_dim)
      return fail(FC_EINVAL, "the pools' geometries do not match");
    if (n_req > 0 && (!dev_dst_tables || !dev_src_tables)) return fail(FC_EINVAL, "NULL argument");
    ChunkPlan plan;
    if (plan_quantise(n_req, dst_max_blocks_per_req, src_max_blocks_per_req, host_seq_lens, host_enable, &plan) != PLAN_OK)
      return fail(plan.code, "%s", plan.message);
    if (plan.reqs.empty()) return FC_OK;
    if (plan.n_rows * src->n_layers > kPlanMaxWorkgroups) return fail(FC_EINVAL, "batch too large for one launch");
    QuantiseParams qp = {};
    ChunkReqs inline_reqs;
    if (int rc = pass_reqs(dst, plan.reqs, &inline_reqs, &qp.reqs, stream)) return rc;
    qp.src = src->kv;
    qp.dst = reinterpret_cast<uint8_t*>(dst->kv);
    qp.e2m1 = dst->dtype == FC_DTYPE_E2M1 ? 1 : 0;
    qp.src_blocks = src->n_blocks;
    qp.dst_blocks = dst->n_blocks;
    qp.n_layers = src->n_layers;
    qp.n_heads = src->n_heads;
    qp.head_dim = src->head_dim;
    qp.src_tables = dev_src_tables;
    qp.dst_tables = dev_dst_tables;
    qp.src_max_blocks = src_max_blocks_per_req;
    qp.dst_max_blocks = dst_max_blocks_per_req;
    qp.n_req = (int)plan.reqs.size();
    qp.n_units = (int)plan.n_rows;
    FC_HIP(launch_quantise(qp, inline_reqs, stream));
    return FC_OK;
  });
}

}  // extern "C"
