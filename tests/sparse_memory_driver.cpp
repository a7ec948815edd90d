// Scratch memory of fc_sparse_attention (csrc/fc_cache_api.hip) on the CPU, over the HIP runtime of
// api_host_driver.cpp.  Built and checked by test_sparse_memory.py.
//   batches from stdin: heads group n_select n  (L n_new) * n  ->  code, bytes of scratch that the call took
//   then a call whose memory is not there, a smaller one, and the same again with the memory there
#define main api_host_main
#include "api_host_driver.cpp"
#undef main

#include "../paper_2503_08461_amd/csrc/fc_cache_api.hip"

namespace fc {
hipError_t launch_rotate_store(const RotateParams&, const ChunkReqs&, hipStream_t) { return hipGetLastError(); }
hipError_t launch_bounds(const BoundsParams&, const ChunkReqs&, hipStream_t) { return hipGetLastError(); }
hipError_t launch_select_blocks(const SelectParams&, const ChunkReqs&, const ChunkReqs&, hipStream_t) { return launched("select"); }
hipError_t launch_attention(const AttnParams&, const ChunkReqs&, hipStream_t) { return launched("attention"); }
hipError_t launch_selected_attention(const SelectParams&, const AttnParams&, const ChunkReqs&, hipStream_t) { return launched("selected"); }
}  // namespace fc

int main() {
  int32_t* table = somewhere<int32_t>();
  auto pool_of = [&](int heads) {
    fc_pool* p = nullptr;
    if (fc_pool_create(&p, somewhere<void>(), ~(size_t)0, 64, 16, 1, heads, 128, FC_DTYPE_F16) != FC_OK) exit(1);
    g_launched.clear();
    return p;
  };
  auto call = [&](fc_pool* p, int group, int n_select, const std::vector<int32_t>& lens, const std::vector<int32_t>& news) {
    const int n_q = p->n_heads * group;
    const fc_rows rows = {somewhere<void>(), n_q * 128, 128};
    return fc_sparse_attention(p, 0, table, 2048, lens.data(), news.data(), somewhere<void>(), n_select, &rows, n_q, &rows, nullptr, (int)lens.size(),
                               0.f, nullptr);
  };
  int heads, group, n_select, n;
  while (scanf("%d %d %d %d", &heads, &group, &n_select, &n) == 4) {
    std::vector<int32_t> lens(n), news(n);
    for (int i = 0; i < n; ++i)
      if (scanf("%d %d", &lens[i], &news[i]) != 2) return 1;
    fc_pool* p = pool_of(heads);
    const int rc = call(p, group, n_select, lens, news);
    printf("batch %d %zu\n", rc, p->sparse.cap);
    fc_pool_destroy(p);
  }
  fc_pool* p = pool_of(32);
  const std::vector<int32_t> one_len = {30000}, chunk = {2048}, few = {2};
  g_launched.clear();
  report("few", call(p, 1, 64, one_len, few));
  g_largest = 100 << 20;
  report("chunk_without", call(p, 1, 64, one_len, chunk));
  report("few_after", call(p, 1, 64, one_len, few));
  g_largest = ~(size_t)0;
  report("chunk", call(p, 1, 64, one_len, chunk));
  fc_pool_destroy(p);
  return 0;
}
