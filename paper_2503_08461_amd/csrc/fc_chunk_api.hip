// Entry points of the calls on chunks of new tokens and whole prompts and of the copy into an
// 8-bit pool (include/fastcache.h).  Validation and descriptors as in fc_api.hip: nothing is
// queued or changed before everything has been checked.

#include "fc_chunk_plan.h"
#include "fc_pool.h"

#include <math.h>
#include <string.h>

#include <algorithm>
#include <exception>

using namespace fc;

namespace {

static_assert(kPlanMaxGroup == FC_MAX_GROUP && kAttnKinds == ATTN_KINDS, "limits");

// (a vector that cannot grow must not throw into C)
template <typename F>
int guarded(const char* what, F f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(FC_ENOMEM, "%s: %s", what, e.what());
  }
}

// The requests as the kernel's argument (*on_device stays NULL) if they fit, else to the device.
template <typename Reqs, typename Req>
int pass_reqs(fc_pool* p, const std::vector<Req>& reqs, Reqs* inline_reqs, const Req** on_device, hipStream_t stream) {
  *on_device = nullptr;
  if (reqs.size() <= Reqs::kInline) {
    std::copy(reqs.begin(), reqs.end(), inline_reqs->req);
    return FC_OK;
  }
  const void* at = nullptr;
  if (int rc = meta_to_device(p, reqs.data(), reqs.size() * sizeof(Req), &at, stream)) return rc;
  *on_device = static_cast<const Req*>(at);
  return FC_OK;
}

// written: every row has its own place, row by row of a token or token by token of a head.
int check_rows(const fc_rows* rows, const char* name, int64_t n_rows, int n_heads, int head_dim, bool written) {
  if (!rows || !rows->data) return fail(FC_EINVAL, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(rows->data) & 15) return fail(FC_EINVAL, "%s must be 16-byte aligned", name);
  const int64_t t = rows->token_stride, h = rows->head_stride;
  if ((t | h) & 7 || t < 0 || h < 0) return fail(FC_EINVAL, "strides of %s must be multiples of 8, 0 or more", name);
  // (16 rows span less than 2^31 bytes; products with numbers of tokens and heads are of 32 bits each)
  if (t > FC_MAX_TOKEN_STRIDE || h > FC_MAX_HEAD_STRIDE) return fail(FC_EINVAL, "strides of %s are too large", name);
  if (written && !(h >= head_dim && t >= (n_heads - 1) * h + head_dim) && !(t >= head_dim && h >= (n_rows - 1) * t + head_dim))
    return fail(FC_EINVAL, "rows of %s overlap", name);
  return FC_OK;
}

RowsView view(const fc_rows* r) { return {static_cast<_Float16*>(r->data), r->token_stride, r->head_stride}; }

PoolView geometry(const fc_pool* p) {
  PoolView v;
  v.n_layers = p->n_layers;
  v.n_heads = p->n_heads;
  v.head_dim = p->head_dim;
  v.n_free = p->top;
  return v;
}

// the blocks of one layer
void* layer_blocks(const fc_pool* p, int layer) {
  const size_t row = p->dtype == FC_DTYPE_E4M3 ? p->head_dim + 1 : 2 * p->head_dim;
  return reinterpret_cast<char*>(p->kv) + (size_t)layer * p->n_blocks * 2 * p->n_heads * FC_BLOCK_SIZE * row;
}

// k and v: packed rows, or NULL for the cache in the pool.
int attention(fc_pool* p, int layer, const int32_t* dev_block_tables, int max_blocks, const int32_t* host_seq_lens,
              const int32_t* host_n_new, const fc_rows* q, const fc_rows* k, const fc_rows* v, int n_q_heads,
              const fc_rows* out, float* dev_lse, int window, int n_req, float scale, hipStream_t stream) {
  const bool paged = !k;
  if (layer < 0 || layer >= p->n_layers) return fail(FC_EINVAL, "layer %d outside 0..%d", layer, p->n_layers - 1);
  if (n_q_heads < 1 || n_q_heads % p->n_heads || n_q_heads / p->n_heads > FC_MAX_GROUP)
    return fail(FC_EINVAL, "%d query heads for %d heads of K and V", n_q_heads, p->n_heads);
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
  if (plan_attention(geometry(p), p->n_cu, n_q_heads / p->n_heads, paged, p->max_states, &plan, launches) != PLAN_OK)
    return fail(plan.code, "%s", plan.message);

  AttnParams ap = {};
  ap.kv = paged ? layer_blocks(p, layer) : nullptr;
  ap.source = !paged ? ATTN_ROWS : p->dtype == FC_DTYPE_E4M3 ? ATTN_E4M3 : ATTN_F16;
  ap.n_blocks = p->n_blocks;
  ap.n_heads = p->n_heads;
  ap.group = n_q_heads / p->n_heads;
  ap.group_inverse = (uint32_t)((((uint64_t)1 << 31) + ap.group - 1) / ap.group);
  ap.head_dim = p->head_dim;
  ap.block_tables = dev_block_tables;
  ap.max_blocks = max_blocks;
  ap.q = view(q);
  if (!paged) {
    ap.k = view(k);
    ap.v = view(v);
  }
  ap.out = view(out);
  ap.window = window;
  if (dev_lse) {
    ap.lse = dev_lse + (int64_t)layer * n_q_heads * window;
    ap.lse_stride = (int64_t)p->n_layers * n_q_heads * window;
  }
  ap.scale_log2e = ((scale > 0.f) ? scale : 1.0f / sqrtf((float)p->head_dim)) * 1.44269504088896340736f;
  std::vector<ChunkReq> reqs(launches[ATTN_TALL].reqs);
  reqs.insert(reqs.end(), launches[ATTN_FLAT].reqs.begin(), launches[ATTN_FLAT].reqs.end());
  ChunkReqs inline_reqs;
  if ((rc = pass_reqs(p, reqs, &inline_reqs, &ap.reqs, stream))) return rc;
  int first_req = 0;
  int64_t states = 0;
  for (int s = 0; s < ATTN_KINDS; ++s) {
    const AttnLaunch& l = launches[s];
    AttnLaunchView& a = ap.launch[s];
    a.first_req = first_req;
    a.n_req = (int)l.reqs.size();
    a.n_units = (int)l.n_units;
    a.seg_blocks = std::max(l.seg_blocks, 1);
    a.n_seg = l.n_seg;
    first_req += a.n_req;
    if (l.n_seg > 1) {
      a.state_rows = (int)l.state_rows;
      a.states = p->decode_partial + states * DecodeParams::state_words(p->head_dim);
      states += l.state_rows * n_q_heads * l.n_seg;
    }
  }
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
    sp.e4m3 = p->dtype == FC_DTYPE_E4M3 ? 1 : 0;
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
    if (dst->dtype != FC_DTYPE_E4M3 || src->dtype != FC_DTYPE_F16)
      return fail(FC_EINVAL, "fc_quantise_batch reads a pool of FC_DTYPE_F16 and writes one of FC_DTYPE_E4M3");
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
