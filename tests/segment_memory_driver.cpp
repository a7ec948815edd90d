// Attention over split caches in a pool whose card is nearly full (csrc/fc_api.hip, fc_chunk_api.hip)
// on the CPU, over the HIP runtime of api_host_driver.cpp: the largest allocation that succeeds is the
// argument.  Built and checked by test_segment_memory.py.
#define main api_host_main
#include "api_host_driver.cpp"
#undef main

#include "../paper_2503_08461_amd/csrc/fc_chunk_api.hip"

namespace fc {
hipError_t launch_extend(const ExtendParams&, const ExtendReqs&, hipStream_t) { return hipSuccess; }
hipError_t launch_store_chunk(const StoreParams&, const ChunkReqs&, hipStream_t) { return hipSuccess; }
hipError_t launch_quantise(const QuantiseParams&, const ChunkReqs&, hipStream_t) { return hipSuccess; }
hipError_t launch_attention(const AttnParams& p, const ChunkReqs&, hipStream_t) {
  int64_t states = 0;  // all of both kinds, and where the last one ends in the pool's buffer
  float* end = nullptr;
  for (const AttnLaunchView& l : p.launch) {
    if (l.n_seg <= 1) continue;
    const int64_t n = (int64_t)l.state_rows * p.n_heads * p.group * l.n_seg;
    states += n;
    end = std::max(end, l.states + n * DecodeParams::state_words(p.head_dim));
  }
  g_launched += std::to_string(states) + " " + std::to_string((uintptr_t)end) + " ";
  return hipSuccess;
}
}  // namespace fc

int main(int argc, char** argv) {
  g_largest = (size_t)atoll(argc > 1 ? argv[1] : "0");
  fc_pool* p = nullptr;
  if (fc_pool_create(&p, somewhere<void>(), ~(size_t)0, 1024, 16, 1, 32, 128, FC_DTYPE_F16) != FC_OK) return 1;
  g_launched.clear();
  const int32_t lens[2] = {8000, 30000}, news[2] = {1, 200};
  report("decode", fc_decode_attention(p, somewhere<int32_t>(), 2048, lens, somewhere<void>(), somewhere<float>(), 2, 0.f, nullptr));
  const fc_rows rows = {somewhere<void>(), 32 * 128, 128};
  report("chunk", fc_chunk_attention(p, 0, somewhere<int32_t>(), 2048, lens, news, &rows, 32, &rows, nullptr, 0, 2, 0.f, nullptr));
  printf("buffer %zu %d\n", (size_t)p->decode_partial, (int)DecodeParams::state_words(128));
  fc_pool_destroy(p);
  return 0;
}
