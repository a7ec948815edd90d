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
                   ChunkPlan* plan, AttnLaunch launches[kAttnKinds], bool four_bits) {
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
    int64_t most_rows = 0;
    for (const ChunkReq& q : l.reqs) {
      most_rows = std::max(most_rows, (int64_t)q.n_new * group);
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
      const bool few = four_bits && s == 1 && launches[0].reqs.empty() && most_rows <= kFewRows4;
      const int64_t share = few ? total / (2 * slots) : total / slots;
      const int64_t least = few ? std::max(16, (longest + 63) / 64) : kPlanMinSegment;
      int64_t seg = std::max<int64_t>({s == 0 ? (longest + wanted - 1) / wanted : share, least, (longest + room - 1) / room});
      if (few) {
        // (a few more than fit at once would run after all others)
        auto segments = [&] {
          int64_t n = 0;
          for (const ChunkReq& q : l.reqs) n += decode_segments(blocks_for(q.seq_len), (int)seg);
          return n * pool.n_heads;
        };
        for (int64_t n = segments(); n > 2 * slots && n < 3 * slots && 2 * seg <= longest; n = segments()) seg += seg / 32 + 1;
      }
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

int plan_positions(const int32_t* positions, int n_positions, ChunkPlan* plan) {
  for (ChunkReq& q : plan->reqs) {
    const int first = positions ? positions[q.table_row] : q.seq_len - q.n_new;
    if (first < 0 || first > n_positions - q.n_new)
      return fail(plan, PLAN_EINVAL, "request %d: %d tokens from position %d on, the table has %d", q.table_row, q.n_new, first, n_positions);
    q.state_off = first;
  }
  return PLAN_OK;
}

int plan_bounds(ChunkPlan* plan) {
  plan->n_rows = 0;
  for (ChunkReq& q : plan->reqs) {
    q.row_off = (q.seq_len - q.n_new) / kPlanBlockSize;
    q.unit_start = (int32_t)plan->n_rows;
    plan->n_rows += blocks_for(q.seq_len) - q.row_off;
    if (plan->n_rows > kPlanMaxWorkgroups) return fail(plan, PLAN_EINVAL, "batch too large for one launch");
  }
  return PLAN_OK;
}

int plan_sparse(const PoolView& pool, int n_cu, int group, int n_select, const ChunkPlan& chunk, SparsePlan* plan) {
  *plan = SparsePlan();
  if (n_select < 1 || n_select > kPlanMaxSeqLen / kPlanBlockSize)
    return fail(plan, PLAN_EINVAL, "n_select %d outside 1..%d", n_select, kPlanMaxSeqLen / kPlanBlockSize);
  // (workgroups that select have 512 threads)
  if (chunk.n_rows * pool.n_heads > kPlanMaxWorkgroups / 2) return fail(plan, PLAN_EINVAL, "batch too large for one launch");
  bool single = true;
  int read = 0;  // most blocks of a token
  // (with one block, the token's own, nothing is scored)
  auto scores = [&](int nb) { return nb > n_select && n_select > 1; };
  for (const ChunkReq& q : chunk.reqs) {
    single = single && q.n_new == 1;
    for (int i = 0; i < q.n_new; ++i) {
      const int seen = q.seq_len - q.n_new + i + 1, nb = blocks_for(seen), row = q.row_off + i;
      plan->tokens.push_back({q.table_row, seen, 0, row, 0, 0});
      if (scores(nb)) plan->longest = std::max(plan->longest, nb - 1);
      read = std::max(read, std::min(nb, n_select));
    }
  }
  // One launch, a workgroup of four wavefronts for a token's head, where each has little to read and to score, or where
  // there are many, of single tokens; else the scores are made by as many workgroups as fill the card, and for the tokens of a
  // request together.  us a step, fp16, n_select 64, one / apart, for so many single tokens times heads:
  //   tokens cached     8            32           64           128          192
  //   2000-2500         29.2 / 32.6  30.1 / 34.8  31.0 / 35.8  33.2 / 41.3  36.0 / 48.5
  //   4000-5000         30.5 / 31.8  31.6 / 34.2  32.8 / 36.5  35.3 / 42.0  38.4 / 50.4
  //   8000-10000        33.3 / 32.0  37.0 / 36.6  38.0 / 38.8  40.0 / 47.4  43.5 / 56.8
  //   30000             52.0 / 32.4  53.6 / 37.9  54.8 / 41.6  59.0 / 60.9  65.8 / 85.1
  // five tokens of 32 caches of 1000-1250, 8 heads: 91 / 93, of 16 of 4000-5000 77 / 72; 256 of two of 16000: 463 / 302.
  // By the blocks read, of 5000:
  //   96                30.5 / 31.4  36.3 / 34.8  38.1 / 38.5  40.6 / 47.3  (256: 54 / 64)
  //   256               56.4 / 32.5  59.6 / 38.8  62.7 / 48.9  68.9 / 69.8  (256: 104 / 114)
  // and 384 of 1024 in caches of 100-30000 436 / 424, of whole ones 553 / 467: whole heads end unevenly.
  // 8 bits and 4, which the rule treats alike, one / apart:
  //   tokens cached     8            64           192              8            64           192
  //   2000-2500         24.8 / 23.9  27.2 / 29.1  28.5 / 37.9      20.7 / 20.9  23.4 / 26.5  24.3 / 33.7
  //   4000-5000         26.3 / 24.3  29.8 / 31.1  31.1 / 40.1      23.0 / 21.8  26.0 / 28.1  27.0 / 35.7
  //   8000-10000        30.7 / 25.0  34.0 / 32.0  35.9 / 45.6      26.2 / 21.6  30.2 / 29.3  31.7 / 41.2
  //   30000             51.3 / 26.9  52.6 / 38.4  60.6 / 77.6      47.3 / 24.2  48.5 / 35.5  55.9 / 72.9
  //   256 of 5000       55.3 / 25.5  56.8 / 39.5  58.4 / 70.7      42.0 / 22.3  43.8 / 33.7  45.0 / 49.1
  // Near a border the other side is ahead by 2 to 3 us in some, most where 128 heads read 256 blocks (8 bits 57 / 50) and for
  // five tokens of 16 caches of 4000-5000 (fp16 75 / 72, 8 bits 59 / 55, 4 bits 40 / 42).
  // (Up to half of the rows: what else is kept of the queries and blocks would not fit the LDS beside more.)
  const int cu = std::max(n_cu, 1);
  const bool many = 2 * chunk.n_rows * pool.n_heads >= cu;
  if (group <= kScoreRows / 2 && read <= (many ? 256 : 64) && (plan->longest <= 384 || (single && many))) return PLAN_OK;
  for (const ChunkReq& t : plan->tokens) {
    // (whole blocks, but for the token's own, the last one)
    const int keys = (std::min(blocks_for(t.seq_len), n_select) - 1) * kPlanBlockSize + (t.seq_len - 1) % kPlanBlockSize + 1;
    plan->attention.reqs.push_back({t.row_off, keys, 1, t.row_off, 0, 0});
  }
  plan->attention.n_rows = chunk.n_rows;
  plan->tile_tokens = std::max(1, kScoreRows / group);
  int64_t total = 0;  // blocks of all workgroups
  auto tiles = [&](const ChunkReq& q) { return ((int64_t)q.n_new + plan->tile_tokens - 1) / plan->tile_tokens; };
  for (const ChunkReq& q : chunk.reqs) {
    const int nb = blocks_for(q.seq_len);
    if (!scores(nb)) continue;
    plan->scored.push_back(q);
    plan->scored.back().state_off = nb - 1;
    total += tiles(q) * (nb - 1) * pool.n_heads;
  }
  plan->part_blocks = (int)std::max<int64_t>(64, (total + 2 * cu - 1) / (2 * cu) + 15) & ~15;
  for (ChunkReq& q : plan->scored) {
    const int parts = (q.state_off + plan->part_blocks - 1) / plan->part_blocks;
    q.unit_start = (int32_t)plan->n_units;
    for (int i = 0; i < q.n_new; ++i) {
      ChunkReq& t = plan->tokens[q.row_off + i];
      t.unit_start = (int32_t)plan->n_units + i / plan->tile_tokens * parts;
      t.n_new = parts;
    }
    plan->n_units += tiles(q) * parts;
    if (plan->n_units * pool.n_heads > kPlanMaxWorkgroups) return fail(plan, PLAN_EINVAL, "batch too large for one launch");
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
