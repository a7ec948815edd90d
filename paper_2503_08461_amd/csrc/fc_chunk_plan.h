// Host-side planning of the calls on chunks of new tokens and whole prompts
// (fc_extend_batch, fc_store_chunk, fc_chunk_attention, fc_prefill_attention)
// and of fc_quantise_batch.  Plain C++, as fc_plan.h.
#pragma once

#include "fc_plan.h"

namespace fc {

static constexpr int kPlanMaxGroup = 64;

struct ExtendPlan {
  int code = PLAN_OK;
  char message[256] = "";
  std::vector<ExtendReq> reqs;  // those that get blocks, batch order
  int n_pop = 0;
};
int plan_extend(const PoolView& pool, int n_req, int max_blocks, const int32_t* seq_lens,
                const int32_t* n_new, ExtendPlan* plan);

// The requests of a batch that have new rows, in batch order.
struct ChunkPlan {
  int code = PLAN_OK;
  char message[256] = "";
  std::vector<ChunkReq> reqs;
  int64_t n_rows = 0;  // packed rows
};
// n_new NULL: whole prompts (every token is new); max_blocks -1: no table.
int plan_chunk(int n_req, int max_blocks, const int32_t* seq_lens, const int32_t* n_new, ChunkPlan* plan);
// fc_store_chunk: a unit is a packed row.  FC_EINVAL (plan->code) where they are too many for a launch.
int plan_store_units(ChunkPlan* plan);

// The requests of an attention by kind: those with many rows to a head of K and V take
// workgroups whose wavefronts have rows of their own, those with few rows wavefronts that
// share the keys (fc_attention.hip).  AttnLaunch[0] has many rows, [1] few.
static constexpr int kAttnKinds = 2;
static constexpr int kTallRows = 128;  // rows (new tokens x query heads of a group) of a workgroup
static constexpr int kFlatRows = 32;
static constexpr int kPlanMinSegment = 32;  // blocks
// Most states of a call's split rows, what the pool's buffer holds if the card has the room (42 MB
// at 128 channels; else kMaxDecodeSegments, or none).
static constexpr int kMaxAttnStates = 65536;
struct AttnLaunch {
  std::vector<ChunkReq> reqs;  // longest first; unit = (row tile, segment), heads not counted
  int64_t n_units = 0;
  int seg_blocks = 0, n_seg = 1;  // blocks per segment of a head, segments of the longest one
  int64_t state_rows = 0;         // rows (tokens) that have states
};
// group: query heads per head of K and V; max_states: states that fit the pool's memory, 0 for
// none.  FC_EINVAL (plan->code) where the launch would be too large.
int plan_attention(const PoolView& pool, int n_cu, int group, bool may_split, int64_t max_states,
                   ChunkPlan* plan, AttnLaunch launches[kAttnKinds]);

// fc_quantise_batch: a unit is a block of a request.
int plan_quantise(int n_req, int dst_max_blocks, int src_max_blocks, const int32_t* seq_lens,
                  const int32_t* enable, ChunkPlan* plan);

}  // namespace fc
