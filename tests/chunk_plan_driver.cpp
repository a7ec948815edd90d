// Host planning of the calls on chunks (csrc/fc_chunk_plan.cpp) on its own: batches from stdin,
// plans to stdout, one line each; built with the host sanitizers by test_chunk_plan.py.
//   A layers heads group n_cu may_split max_states n  (L n_new) * n
//   E free max_blocks n  (L n_new) * n        C max_blocks n  (L n_new) * n
//   Q dst src n  (L enable) * n
#include <cstdio>

#include "../paper_2503_08461_amd/csrc/fc_chunk_plan.h"

using namespace fc;

int main() {
  char what;
  while (scanf(" %c", &what) == 1) {
    int a[6] = {}, n = 0;
    const int n_args = what == 'A' ? 6 : what == 'C' ? 1 : 2;
    for (int i = 0; i < n_args; ++i)
      if (scanf("%d", &a[i]) != 1) return 1;
    if (scanf("%d", &n) != 1) return 1;
    std::vector<int32_t> x(n > 0 ? n : 0), y(x.size());
    for (size_t i = 0; i < x.size(); ++i)
      if (scanf("%d %d", &x[i], &y[i]) != 2) return 1;
    if (what == 'E') {
      PoolView pool;
      pool.n_free = a[0];
      ExtendPlan p;
      const int rc = plan_extend(pool, n, a[1], x.data(), y.data(), &p);
      printf("E %d %d", rc, rc ? 0 : p.n_pop);
      if (!p.code)
        for (const ExtendReq& q : p.reqs) printf(" %d,%d,%d,%d", q.table_row, q.first, q.n_pop, q.pop_index);
      printf("\n");
    } else if (what == 'C') {
      ChunkPlan p;
      printf("C %d", plan_chunk(n, a[0], x.data(), a[0] == -1 ? nullptr : y.data(), &p));
      if (!p.code)
        for (const ChunkReq& q : p.reqs) printf(" %d,%d,%d,%d", q.table_row, q.seq_len, q.n_new, q.row_off);
      printf("\n");
    } else if (what == 'Q') {
      ChunkPlan p;
      printf("Q %d", plan_quantise(n, a[0], a[1], x.data(), y.data(), &p));
      if (!p.code) printf(" %lld", (long long)p.n_rows);
      printf("\n");
    } else {
      PoolView pool;
      pool.n_layers = a[0];
      pool.n_heads = a[1];
      ChunkPlan p;
      AttnLaunch l[kAttnKinds];
      int rc = plan_chunk(n, 1 << 20, x.data(), y.data(), &p);
      if (!rc) rc = plan_attention(pool, a[3], a[2], a[4] != 0, a[5], &p, l);
      printf("A %d", rc);
      for (int s = 0; !rc && s < kAttnKinds; ++s) {
        printf(" | %lld %d %d %lld", (long long)l[s].n_units, l[s].seg_blocks, l[s].n_seg, (long long)l[s].state_rows);
        for (const ChunkReq& q : l[s].reqs)
          printf(" %d,%d,%d,%d,%d,%d", q.table_row, q.seq_len, q.n_new, q.row_off, q.unit_start, q.state_off);
      }
      printf("\n");
    }
  }
  return 0;
}
