// Host planning of positions, bounds, selected blocks and attention over 4-bit rows (csrc/fc_chunk_plan.cpp) on
// its own: batches from stdin, plans to stdout, one line each; built with the host sanitizers by test_cache_plan.py.
//   P n_positions given n  (L n_new position) * n       B n  (L n_new) * n
//   S heads group n_cu n_select n  (L n_new) * n        F heads group n_cu max_states n  (L n_new) * n
#include <cstdio>

#include "../paper_2503_08461_amd/csrc/fc_chunk_plan.h"

using namespace fc;

int main() {
  char what;
  while (scanf(" %c", &what) == 1) {
    int a[4] = {}, n = 0;
    const int n_args = what == 'P' ? 2 : what == 'B' ? 0 : 4;
    for (int i = 0; i < n_args; ++i)
      if (scanf("%d", &a[i]) != 1) return 1;
    if (scanf("%d", &n) != 1) return 1;
    std::vector<int32_t> x(n), y(n), z(n);
    for (int i = 0; i < n; ++i) {
      if (scanf("%d %d", &x[i], &y[i]) != 2) return 1;
      if (what == 'P' && scanf("%d", &z[i]) != 1) return 1;
    }
    ChunkPlan p;
    int rc = plan_chunk(n, 1 << 20, x.data(), y.data(), &p);
    PoolView pool;
    pool.n_layers = 1;
    pool.n_heads = a[0];
    printf("%c ", what);
    if (what == 'P') {
      if (!rc) rc = plan_positions(a[1] ? z.data() : nullptr, a[0], &p);
      printf("%d", rc);
      for (const ChunkReq& q : p.reqs)
        if (!rc) printf(" %d,%d", q.table_row, q.state_off);
    } else if (what == 'B') {
      if (!rc) rc = plan_bounds(&p);
      printf("%d %lld", rc, (long long)p.n_rows);
      for (const ChunkReq& q : p.reqs)
        if (!rc) printf(" %d,%d,%d", q.table_row, q.row_off, q.unit_start);
    } else if (what == 'S') {
      SparsePlan s;
      if (!rc) rc = plan_sparse(pool, a[2], a[1], a[3], p, &s);
      printf("%d %d %d %lld %d", rc, s.part_blocks, s.tile_tokens, (long long)s.n_units, s.longest);
      if (!rc) {
        for (const ChunkReq& q : s.scored) printf(" q%d,%d,%d,%d", q.table_row, q.n_new, q.unit_start, q.state_off);
        for (const ChunkReq& q : s.tokens) printf(" t%d,%d,%d,%d,%d", q.table_row, q.seq_len, q.row_off, q.unit_start, q.n_new);
        for (const ChunkReq& q : s.attention.reqs) printf(" a%d,%d,%d,%d", q.table_row, q.seq_len, q.n_new, q.row_off);
      }
    } else {
      AttnLaunch l[kAttnKinds];
      if (!rc) rc = plan_attention(pool, a[2], a[1], true, a[3], &p, l, true);
      printf("%d", rc);
      for (int s = 0; !rc && s < kAttnKinds; ++s) {
        printf(" | %lld %d %d %lld", (long long)l[s].n_units, l[s].seg_blocks, l[s].n_seg, (long long)l[s].state_rows);
        for (const ChunkReq& q : l[s].reqs) printf(" %d,%d,%d,%d,%d", q.table_row, q.seq_len, q.n_new, q.unit_start, q.state_off);
      }
    }
    printf("\n");
  }
  return 0;
}
