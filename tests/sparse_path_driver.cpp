// Which launches a call over selected blocks makes, and how its attention is cut (csrc/fc_chunk_plan.cpp): batches
// from stdin, a line each; built and checked by test_sparse_paths.py.
//   S heads group n_select n  (L n_new) * n  ->  parts a tile of the longest, tiles, segments in fp16 and in 4 bits
//   C heads group n  (L n_new) * n           ->  units of many rows, of few, segments of few, most rows, in 4 bits
#include <algorithm>
#include <cstdio>

#include "../paper_2503_08461_amd/csrc/fc_chunk_plan.h"

using namespace fc;

int main() {
  char what;
  while (scanf(" %c", &what) == 1) {
    int heads, group, n_select = 0, n;
    if (scanf("%d %d", &heads, &group) != 2 || (what == 'S' && scanf("%d", &n_select) != 1) || scanf("%d", &n) != 1) return 1;
    std::vector<int32_t> lens(n), news(n);
    for (int i = 0; i < n; ++i)
      if (scanf("%d %d", &lens[i], &news[i]) != 2) return 1;
    PoolView pool;
    pool.n_layers = 1;
    pool.n_heads = heads;
    ChunkPlan p;
    if (plan_chunk(n, 1 << 20, lens.data(), news.data(), &p) != PLAN_OK) return 1;
    AttnLaunch l[kAttnKinds];
    if (what == 'C') {
      if (plan_attention(pool, 256, group, true, kMaxAttnStates, &p, l, true) != PLAN_OK) return 1;
      int rows = 0;
      for (const ChunkReq& q : l[1].reqs) rows = std::max(rows, q.n_new * group);
      printf("%lld %lld %d %d\n", (long long)l[0].n_units, (long long)l[1].n_units, l[1].n_seg, rows);
      continue;
    }
    SparsePlan s;
    if (plan_sparse(pool, 256, group, n_select, p, &s) != PLAN_OK) return 1;
    int parts = 0, tiles = 0, seg[2] = {};
    for (const ChunkReq& q : s.scored) {
      parts = std::max(parts, (q.state_off + s.part_blocks - 1) / s.part_blocks);
      tiles = std::max(tiles, (q.n_new + s.tile_tokens - 1) / s.tile_tokens);
    }
    for (int four = 0; four < 2 && s.part_blocks; ++four) {
      ChunkPlan a = s.attention;
      if (plan_attention(pool, 256, group, true, kMaxAttnStates, &a, l, four != 0) != PLAN_OK) return 1;
      seg[four] = std::max(l[0].n_seg, l[1].n_seg);
    }
    printf("%d %d %d %d\n", parts, tiles, seg[0], seg[1]);
  }
  return 0;
}
