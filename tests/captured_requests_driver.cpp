// Descriptors of captured calls on many requests (csrc/fc_api.hip, meta_to_device) on the CPU, over
// the HIP runtime of api_host_driver.cpp.  Built and checked by test_captured_requests.py.
#define main api_host_main
#include "api_host_driver.cpp"
#undef main

#include "../paper_2503_08461_amd/csrc/fc_chunk_api.hip"

namespace fc {
hipError_t launch_extend(const ExtendParams&, const ExtendReqs&, hipStream_t) { return hipSuccess; }
hipError_t launch_store_chunk(const StoreParams&, const ChunkReqs&, hipStream_t) { return hipSuccess; }
hipError_t launch_quantise(const QuantiseParams&, const ChunkReqs&, hipStream_t) { return hipSuccess; }
hipError_t launch_attention(const AttnParams&, const ChunkReqs&, hipStream_t) { return hipSuccess; }
}  // namespace fc

int main() {
  int32_t* table = somewhere<int32_t>();
  fc_pool* p = nullptr;
  fc_pool_create(&p, somewhere<void>(), ~(size_t)0, 64, 16, 2, 4, 128, FC_DTYPE_F16);
  g_launched.clear();
  const fc_rows rows = {somewhere<void>(), 512, 128};
  std::vector<int32_t> l(100000, 20), ones(100000, 1);
  auto call = [&](const char* name, int n, bool captured) {
    g_capturing = captured;
    const int rc = fc_store_chunk(p, 0, table, 2, l.data(), ones.data(), &rows, &rows, n, nullptr);
    g_capturing = false;
    report(name, rc);
    printf("kept %zu\n", p->meta_retired.size());
  };
  call("captured_first", 150, true);  // nothing to put the descriptors in
  call("eager", 150, false);
  call("eager_more", 1000, false);  // grows; nothing captured
  const char* none = p->dev_meta;
  call("captured", 150, true);
  const char* used = p->dev_meta;
  call("captured_more", 50000, true);
  printf("same %d\n", none == used && p->dev_meta == used);
  call("eager_grows", 10000, false);
  printf("grown %d\n", p->dev_meta != used && p->meta_retired.size() == 1 && p->meta_retired[0] == used);
  call("eager_grows_again", 50000, false);  // no graph uses the one before
  call("captured_again", 40000, true);
  call("eager_last", 100000, false);
  fc_pool_destroy(p);
  return 0;
}
