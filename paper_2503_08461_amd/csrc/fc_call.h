// What the entry points on packed rows share: their checks, and how descriptors and launches are
// made of a plan.  Host code, not part of the public ABI.
#pragma once

#include "fc_chunk_plan.h"
#include "fc_pool.h"

#include <math.h>

#include <algorithm>
#include <exception>

namespace fc {

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
inline int check_rows(const fc_rows* rows, const char* name, int64_t n_rows, int n_heads, int head_dim, bool written) {
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

inline int check_q_heads(const fc_pool* p, int n_q_heads) {
  if (n_q_heads < 1 || n_q_heads % p->n_heads || n_q_heads / p->n_heads > FC_MAX_GROUP)
    return fail(FC_EINVAL, "%d query heads for %d heads of K and V", n_q_heads, p->n_heads);
  return FC_OK;
}

inline RowsView view(const fc_rows* r) { return {static_cast<_Float16*>(r->data), r->token_stride, r->head_stride}; }

inline PoolView geometry(const fc_pool* p) {
  PoolView v;
  v.n_layers = p->n_layers;
  v.n_heads = p->n_heads;
  v.head_dim = p->head_dim;
  v.n_free = p->top;
  return v;
}

// the blocks of one layer
inline void* layer_blocks(const fc_pool* p, int layer) {
  return reinterpret_cast<char*>(p->kv) + (size_t)layer * p->n_blocks * block_bytes(p->dtype, p->n_heads, p->head_dim);
}
// how a pool's rows are held, for the kernels' parameters
inline int row_format(const fc_pool* p) {
  return p->dtype == FC_DTYPE_E4M3 ? ROWS_E4M3 : p->dtype == FC_DTYPE_E2M1 ? ROWS_E2M1 : ROWS_F16;
}

// The parameters of an attention that do not depend on where its keys are.
inline void set_queries(const fc_pool* p, const fc_rows* q, const fc_rows* out, int n_q_heads, float scale, AttnParams* ap) {
  ap->n_blocks = p->n_blocks;
  ap->n_heads = p->n_heads;
  ap->group = n_q_heads / p->n_heads;
  ap->group_inverse = (uint32_t)((((uint64_t)1 << 31) + ap->group - 1) / ap->group);
  ap->head_dim = p->head_dim;
  ap->q = view(q);
  ap->out = view(out);
  ap->scale_log2e = ((scale > 0.f) ? scale : 1.0f / sqrtf((float)p->head_dim)) * 1.44269504088896340736f;
}
// The requests of both kinds, as the kernel finds them one after the other.
inline std::vector<ChunkReq> attention_reqs(const AttnLaunch launches[ATTN_KINDS]) {
  std::vector<ChunkReq> reqs(launches[ATTN_TALL].reqs);
  reqs.insert(reqs.end(), launches[ATTN_FLAT].reqs.begin(), launches[ATTN_FLAT].reqs.end());
  return reqs;
}
inline void set_launches(const fc_pool* p, const AttnLaunch launches[ATTN_KINDS], int n_q_heads, AttnParams* ap) {
  int first_req = 0;
  int64_t states = 0;
  for (int s = 0; s < ATTN_KINDS; ++s) {
    const AttnLaunch& l = launches[s];
    AttnLaunchView& a = ap->launch[s];
    a.first_req = first_req;
    a.n_req = (int)l.reqs.size();
    a.n_units = (int)l.n_units;
    a.seg_blocks = std::max(l.seg_blocks, 1);
    a.n_seg = l.n_seg;
    for (const ChunkReq& q : l.reqs) a.most_rows = (int)std::max<int64_t>(a.most_rows, (int64_t)q.n_new * ap->group);
    first_req += a.n_req;
    if (l.n_seg > 1) {
      a.state_rows = (int)l.state_rows;
      a.states = p->decode_partial + states * DecodeParams::state_words(p->head_dim);
      states += l.state_rows * n_q_heads * l.n_seg;
    }
  }
}

}  // namespace fc
