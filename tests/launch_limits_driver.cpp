// Calls just within and just beyond what one launch takes (csrc/fc_api.hip, fc_chunk_api.hip) on the
// CPU, over the HIP runtime and the launchers of api_host_driver.cpp, and these.  Built and checked by
// test_launch_limits.py.
#define main api_host_main
#include "api_host_driver.cpp"
#undef main

#include "../paper_2503_08461_amd/csrc/fc_chunk_api.hip"

namespace fc {
hipError_t launch_extend(const ExtendParams&, const ExtendReqs&, hipStream_t) { return launched("extend"); }
hipError_t launch_store_chunk(const StoreParams&, const ChunkReqs&, hipStream_t) { return launched("store"); }
hipError_t launch_quantise(const QuantiseParams&, const ChunkReqs&, hipStream_t) { return launched("quantise"); }
hipError_t launch_attention(const AttnParams&, const ChunkReqs&, hipStream_t) { return launched("attention"); }
}  // namespace fc

int main() {
  auto pool_of = [&](int layers, int heads, int dtype) {
    fc_pool* p = nullptr;
    fc_pool_create(&p, somewhere<void>(), ~(size_t)0, 64, 16, layers, heads, 128, dtype);
    g_launched.clear();
    return p;
  };
  int32_t* table = somewhere<int32_t>();
  const fc_rows same = {somewhere<void>(), 0, 0};
  for (int beyond : {0, 1}) {
    const std::string s = beyond ? "_beyond" : "_within";
    // a workgroup a new token: 512 * 32768 = 2^24
    std::vector<int32_t> lens(511 + beyond, 32768);
    fc_pool *p = pool_of(1, 1, FC_DTYPE_F16), *p8 = pool_of(1, 1, FC_DTYPE_E4M3);
    for (fc_pool* at : {p, p8})
      report(((at == p ? "store" : "store8") + s).c_str(),
             fc_store_chunk(at, 0, table, 2048, lens.data(), lens.data(), &same, &same, (int)lens.size(), nullptr));
    fc_pool_destroy(p);
    fc_pool_destroy(p8);
    // 128 rows a workgroup, 32768 * 64 rows a head: 2^14 workgroups
    const int heads = 1023 + beyond;
    p = pool_of(1, heads, FC_DTYPE_F16);
    const int32_t whole[1] = {32768};
    const fc_rows out = {somewhere<void>(), heads * 64 * 128, 128};
    report(("prefill" + s).c_str(), fc_prefill_attention(p, 0, whole, &same, &same, &same, heads * 64, &out, nullptr, 0, 1, 0.f, nullptr));
    report(("chunk" + s).c_str(), fc_chunk_attention(p, 0, table, 2048, whole, whole, &same, heads * 64, &out, nullptr, 0, 1, 0.f, nullptr));
    fc_pool_destroy(p);
    // a workgroup a block and layer: 2048 * 8192
    p = pool_of(8192, 1, FC_DTYPE_F16), p8 = pool_of(8192, 1, FC_DTYPE_E4M3);
    const int32_t cached[1] = {32767 - 16 + 16 * beyond};
    report(("quantise" + s).c_str(), fc_quantise_batch(p8, table, 2048, p, table, 2048, cached, nullptr, 1, nullptr));
    // a workgroup a request and layer: 2048 * 8192
    std::vector<int32_t> few(2047 + beyond, 20);
    report(("append" + s).c_str(), fc_append_batch(p, table, 4, few.data(), somewhere<void>(), nullptr, (int)few.size(), nullptr));
    printf("append%s_left %d\n", s.c_str(), few[0]);
    report(("append8" + s).c_str(), fc_append_batch(p8, table, 4, few.data(), somewhere<void>(), nullptr, (int)few.size(), nullptr));
    fc_pool_destroy(p);
    fc_pool_destroy(p8);
    // a workgroup a head: 2048 * 8192
    p = pool_of(8192, 2047 + beyond, FC_DTYPE_F16), p8 = pool_of(8192, 2047 + beyond, FC_DTYPE_E4M3);
    const int32_t one[1] = {20};
    for (fc_pool* at : {p, p8})
      report(((at == p ? "decode" : "decode8") + s).c_str(),
             fc_decode_attention(at, table, 2, one, somewhere<void>(), somewhere<float>(), 1, 0.f, nullptr));
    report(("kept" + s).c_str(), fc_decode_attention_kept(p, table, 2, one, one, table, somewhere<void>(), somewhere<float>(), 1, 0.f, nullptr));
    fc_pool_destroy(p);
    fc_pool_destroy(p8);
  }
  return 0;
}
