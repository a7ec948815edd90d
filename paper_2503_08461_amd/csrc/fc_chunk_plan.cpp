#include "fc_chunk_plan.h"

#include <stdarg.h>
#include <stdio.h>

#include <algorithm>

namespace fc {

namespace {

int blocks_for(int tokens) { return (tokens + kPlanBlockSize - 1) / kPlanBlockSize; }

template <typename Plan>
int fail(Plan* plan, int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(plan->message, sizeof(plan->message), fmt, ap);
  va_end(ap);
  plan->code = code;
  return code;
}

constexpr int64_t kMaxRows = 0x7fffffff;

}  // namespace

int plan_extend(const PoolView& pool, int n_req, int max_blocks, const int32_t* seq_lens,
                const int32_t* n_new, ExtendPlan* plan) {
  *plan = ExtendPlan();
  if (n_req < 0) return fail(plan, PLAN_EINVAL, "n_req < 0");
  if (n_req == 0) return PLAN_OK;
  if (!seq_lens || !n_new) return fail(plan, PLAN_EINVAL, "NULL argument");
  if (max_blocks < 1) return fail(plan, PLAN_EINVAL, "max_blocks_per_req < 1");
  int64_t n_pop = 0;
  for (int r = 0; r < n_req; ++r) {
    const int L = seq_lens[r], n = n_new[r];
    if (L < 0 || n < 0 || L > kPlanMaxSeqLen || n > kPlanMaxSeqLen - L)
      return fail(plan, PLAN_EINVAL, "request %d: %d tokens and %d new ones outside 0..%d", r, L, n, kPlanMaxSeqLen);
    const int before = blocks_for(L), after = blocks_for(L + n);
    if (after > max_blocks)
      return fail(plan, PLAN_EINVAL, "request %d: %d tokens exceed max_blocks_per_req", r, L + n);
    if (after == before) continue;
    plan->reqs.push_back({r, before, after - before, (int32_t)std::min(n_pop, kMaxRows)});
    n_pop += after - before;
  }
  if (n_pop > pool.n_free)
    return fail(plan, PLAN_ENOMEM, "the new tokens need %lld new blocks, %d free", (long long)n_pop, pool.n_free);
  plan->n_pop = (int)n_pop;
  return PLAN_OK;
}

int plan_chunk(int n_req, int max_blocks, const int32_t* seq_lens, const int32_t* n_new, ChunkPlan* plan) {
  *plan = ChunkPlan();
  if (n_req < 0) return fail(plan, PLAN_EINVAL, "n_req < 0");
  if (n_req == 0) return PLAN_OK;
  if (!seq_lens) return fail(plan, PLAN_EINVAL, "NULL argument");
  if (max_blocks == 0 || max_blocks < -1) return fail(plan, PLAN_EINVAL, "max_blocks_per_req < 1");
  for (int r = 0; r < n_req; ++r) {
    const int L = seq_lens[r], n = n_new ? n_new[r] : L;
    if (L < 0 || L > kPlanMaxSeqLen)
      return fail(plan, PLAN_EINVAL, "request %d: length %d outside 0..%d", r, L, kPlanMaxSeqLen);
    if (n < 0 || n > L) return fail(plan, PLAN_EINVAL, "request %d: %d new tokens of %d", r, n, L);
    if (max_blocks > 0 && blocks_for(L) > max_blocks)
      return fail(plan, PLAN_EINVAL, "request %d: %d tokens exceed max_blocks_per_req", r, L);
    if (n == 0) continue;
    if (plan->n_rows + n > kMaxRows) return fail(plan, PLAN_EINVAL, "batch too large for one launch");
    plan->reqs.push_back({r, L, n, (int32_t)plan->n_rows, 0, 0});
    plan->n_rows += n;
  }
  return PLAN_OK;
}

int plan_store_units(ChunkPlan* plan) {
  if (plan->n_rows > kPlanMaxWorkgroups) return fail(plan, PLAN_EINVAL, "batch too large for one launch");
  for (ChunkReq& q : plan->reqs) q.unit_start = q.row_off;
  return PLAN_OK;
}

int plan_attention(const PoolView& pool, int n_cu, int group, bool may_split, int64_t max_states,
                   ChunkPlan* plan, AttnLaunch launches[kAttnKinds]) {
  for (int s = 0; s < kAttnKinds; ++s) launches[s] = AttnLaunch();
  // Few rows of a head are those of one tile that shares the keys.  What 33-127 rows cost as many
  // rows / as two to four tiles of few, each of which reads the keys again (the attention, us):
  //                                            fp16             8-bit
  //   40 rows, 48 caches of 1280-7040, 8 heads  179 / 195        138 / 110
  //   120 rows                                  189 / 332        165 / 180
  //   40 rows, 32 of 256-1408, 8 heads         31.6 / 31.9      34.4 / 22.6
  //   96 rows                                  49.2 / 43.0      50.1 / 33.5
  //   40 rows, 1 of 30000, 8 heads             31.6 / 45.3      29.7 / 31.0
  //   40 rows, 24 of 256-4000, 32 heads         169 / 222        124 / 128
  // (one border for both: 8-bit caches of grouped heads would gain with one of two tiles)
  for (const ChunkReq& q : plan->reqs)
    launches[(int64_t)q.n_new * group <= kFlatRows ? 1 : 0].reqs.push_back(q);
  int64_t states_left = may_split ? max_states : 0;
  for (int s = 0; s < kAttnKinds; ++s) {
    AttnLaunch& l = launches[s];
    if (l.reqs.empty()) continue;
    std::stable_sort(l.reqs.begin(), l.reqs.end(),
                     [](const ChunkReq& a, const ChunkReq& b) { return a.seq_len > b.seq_len; });
    const int tile = s == 0 ? kTallRows : kFlatRows;
    auto tiles = [&](const ChunkReq& q) { return ((int64_t)q.n_new * group + tile - 1) / tile; };
    const int longest = blocks_for(l.reqs.front().seq_len);
    l.seg_blocks = std::max(longest, 1);
    int64_t total = 0, units = 0;  // blocks that workgroups walk, workgroups, all heads
    for (const ChunkReq& q : l.reqs) {
      units += tiles(q) * pool.n_heads;
      total += tiles(q) * blocks_for(q.seq_len) * pool.n_heads;
      l.state_rows += q.n_new;
    }
    // Keys are split where workgroups are few or uneven, at least in two.  Two workgroups fit a
    // CU.  Many rows: as many segments as make that many workgroups, of 32 blocks and more
    // (rows x tokens cached; us, 8 heads of K and V, 4 query heads each):
    //   whole / split     64 x 16000 (two)  256 x 20000   150 x 5000-9000 (three)
    //                     92 / 60           204 / 109     61 / 40
    // Few rows: segments of half of a CU's share (a CU whose neighbours are done draws more
    // than that), of 32 blocks and more: each costs the merge as much as reading one or two.
    //   a share's                      whole  half  third  quarter, at least 16  32  64
    //   64 caches of 500-4000            97    102    102    105
    //   16 of 1000-9000, 4 heads         44     36     41     38
    //   24 of 3000-20000                209    204    188    203
    //   the same in 8 bits              135    129    118    120
    //   1 of 30000                                                            34  28  28
    //   1 of 8000                                                             15  15  18
    const int64_t n_q_heads = (int64_t)group * pool.n_heads;
    const int64_t slots = 2 * (int64_t)std::max(n_cu, 1);
    const int64_t room = states_left / (l.state_rows * n_q_heads);  // segments of a row
    if (room >= 2) {
      const int64_t wanted = s == 0 ? (slots + units - 1) / units : 1;
      const int64_t seg = std::max<int64_t>({s == 0 ? (longest + wanted - 1) / wanted : total / slots, kPlanMinSegment,
                                             (longest + room - 1) / room});
      if (2 * seg <= longest) {
        l.seg_blocks = (int)seg;
        l.n_seg = decode_segments(longest, l.seg_blocks);
        states_left -= l.state_rows * n_q_heads * l.n_seg;
      }
    }
    int64_t state_off = 0;
    for (ChunkReq& q : l.reqs) {
      q.unit_start = (int32_t)l.n_units;
      q.state_off = (int32_t)state_off;
      state_off += q.n_new;
      l.n_units += tiles(q) * decode_segments(blocks_for(q.seq_len), l.seg_blocks);
      if ((launches[0].n_units + launches[1].n_units) * pool.n_heads > kPlanMaxWorkgroups)
        return fail(plan, PLAN_EINVAL, "batch too large for one launch");
    }
  }
  return PLAN_OK;
}

int plan_quantise(int n_req, int dst_max_blocks, int src_max_blocks, const int32_t* seq_lens,
                  const int32_t* enable, ChunkPlan* plan) {
  *plan = ChunkPlan();
  if (n_req < 0) return fail(plan, PLAN_EINVAL, "n_req < 0");
  if (n_req == 0) return PLAN_OK;
  if (!seq_lens) return fail(plan, PLAN_EINVAL, "NULL argument");
  if (dst_max_blocks < 1 || src_max_blocks < 1) return fail(plan, PLAN_EINVAL, "max_blocks_per_req < 1");
  for (int r = 0; r < n_req; ++r) {
    if (enable && !enable[r]) continue;
    const int L = seq_lens[r];
    if (L < 0 || L > kPlanMaxSeqLen)
      return fail(plan, PLAN_EINVAL, "request %d: length %d outside 0..%d", r, L, kPlanMaxSeqLen);
    if (blocks_for(L) > std::min(dst_max_blocks, src_max_blocks))
      return fail(plan, PLAN_EINVAL, "request %d: %d tokens exceed max_blocks_per_req", r, L);
    if (L == 0) continue;
    plan->reqs.push_back({r, L, 0, 0, (int32_t)plan->n_rows, 0});
    plan->n_rows += blocks_for(L);
    if (plan->n_rows > kMaxRows) return fail(plan, PLAN_EINVAL, "batch too large for one launch");
  }
  return PLAN_OK;
}

}  // namespace fc
