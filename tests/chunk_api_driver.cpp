// The entry points on chunks of new tokens and 8-bit pools (csrc/fc_chunk_api.hip) on the CPU: the
// HIP runtime and the launchers of api_host_driver.cpp, and these.  Built and checked by
// test_chunk_api.py; every line says what was called, its code and what was launched.
#define main api_host_main
#include "api_host_driver.cpp"
#undef main

#include "../paper_2503_08461_amd/csrc/fc_chunk_api.hip"

namespace fc {
hipError_t launch_extend(const ExtendParams& p, const ExtendReqs&, hipStream_t) { return launched(p.reqs ? "extend" : "extend_inline"); }
hipError_t launch_store_chunk(const StoreParams& p, const ChunkReqs&, hipStream_t) {
  return launched(((p.e4m3 ? "store8" : "store") + std::string(p.reqs ? "" : "_inline") + ":" + std::to_string(p.n_rows)).c_str());
}
hipError_t launch_quantise(const QuantiseParams& p, const ChunkReqs&, hipStream_t) { return launched(("quantise:" + std::to_string(p.n_units)).c_str()); }
hipError_t launch_attention(const AttnParams& p, const ChunkReqs&, hipStream_t) {
  std::string s = "attention" + std::to_string(p.source) + (p.reqs ? "" : "_inline");
  for (const AttnLaunchView& l : p.launch) s += ":" + std::to_string(l.n_req) + "x" + std::to_string(l.n_seg);
  return launched(s.c_str());
}
}  // namespace fc

int main() {
  int32_t* table = somewhere<int32_t>();
  float* out32 = somewhere<float>();
  auto pool_of = [&](int dtype, int heads, int dim, size_t bytes) {
    fc_pool* p = nullptr;
    const int rc = fc_pool_create(&p, somewhere<void>(), bytes, 64, 16, 2, heads, dim, dtype);
    g_launched.clear();
    return rc == FC_OK ? p : nullptr;
  };
  // sizes: an 8-bit row is head_dim + 1 bytes
  const size_t bytes8 = (size_t)2 * 64 * 2 * 4 * 16 * 129;
  fc_pool* none = pool_of(FC_DTYPE_E4M3, 4, 128, bytes8 - 1);
  report("create8_small", none ? 0 : -1);
  report("create_dtype", pool_of(2, 4, 128, ~(size_t)0) ? 0 : -1);
  fc_pool *p8 = pool_of(FC_DTYPE_E4M3, 4, 128, bytes8), *p16 = pool_of(FC_DTYPE_F16, 4, 128, ~(size_t)0);
  fc_pool* other = pool_of(FC_DTYPE_F16, 4, 64, ~(size_t)0);
  report("create8", p8 ? 0 : -1);

  // what an 8-bit pool refuses, before anything is launched
  int32_t lens[2] = {100, 40}, method[2] = {FC_METHOD_KNORM, FC_METHOD_SNAPKV}, budget[2] = {40, 40}, width[2] = {7, 7}, window[2] = {16, 16};
  const int32_t zeros[2] = {0, 0};
  report("compress8", fc_compress_batch(p8, table, 8, lens, table, 16, method, budget, 2, 7, 0.f, nullptr, nullptr, nullptr));
  report("noalloc8", fc_compress_batch_noalloc(p8, table, 8, lens, table, 16, method, budget, 2, 7, 0.f, nullptr, nullptr, nullptr));
  report("var8", fc_compress_batch_var(p8, table, 8, lens, table, window, method, budget, width, 2, 0.f, nullptr, nullptr, nullptr));
  report("lse8", fc_compress_batch_lse(p8, table, 8, lens, table, out32, 16, method, budget, 2, 7, 0.f, nullptr, nullptr, nullptr));
  report("window8", fc_window_lse(p8, table, 8, lens, table, 16, nullptr, 2, 0.f, out32, nullptr));
  report("kept8", fc_decode_attention_kept(p8, table, 8, lens, budget, table, table, out32, 2, 0.f, nullptr));
  report("mlp8", fc_compress_batch_mlp(p8, table, 8, lens, zeros, zeros, nullptr, 2, nullptr));
  fc_mlp_weights weights = {};
  report("weights8", fc_mlp_set_weights(p8, &weights, nullptr));
  // ... and takes
  report("append8", fc_append_batch(p8, table, 8, lens, table, nullptr, 2, nullptr));
  report("decode8", fc_decode_attention(p8, table, 8, lens, table, out32, 2, 0.f, nullptr));
  printf("lens %d %d\n", lens[0], lens[1]);

  // extend
  int32_t more[2] = {0, 30}, fewer[2] = {0, -1}, far[2] = {1 << 15, 0};
  report("extend", fc_extend_batch(p16, table, 8, lens, more, 2, nullptr));
  printf("lens %d %d free %d\n", lens[0], lens[1], fc_pool_num_free(p16));
  report("extend_negative", fc_extend_batch(p16, table, 8, lens, fewer, 2, nullptr));
  report("extend_far", fc_extend_batch(p16, table, 4096, lens, far, 2, nullptr));
  report("extend_table", fc_extend_batch(p16, nullptr, 8, lens, more, 2, nullptr));
  report("extend_news", fc_extend_batch(p16, table, 8, lens, nullptr, 2, nullptr));
  report("extend_pool", fc_extend_batch(nullptr, table, 8, lens, more, 2, nullptr));
  report("extend_none", fc_extend_batch(p16, nullptr, 8, nullptr, nullptr, 0, nullptr));
  int32_t long_lens[2] = {0, 0}, many[2] = {520, 520};
  report("extend_full", fc_extend_batch(p16, table, 64, long_lens, many, 2, nullptr));
  printf("lens %d %d free %d\n", lens[0] + long_lens[0], lens[1] + long_lens[1], fc_pool_num_free(p16));

  // rows
  const fc_rows ok = {somewhere<void>(), 12 * 128, 128};
  const int32_t news[2] = {1, 33};
  auto store = [&](const char* what, const fc_rows* k, const fc_rows* v, int layer = 1, const int32_t* n = nullptr, int mb = 8) {
    report(what, fc_store_chunk(p16, layer, table, mb, lens, n ? n : news, k, v, 2, nullptr));
  };
  store("store", &ok, &ok);
  report("store8", fc_store_chunk(p8, 0, table, 8, lens, news, &ok, &ok, 2, nullptr));
  store("store_layer", &ok, &ok, 2);
  store("store_below", &ok, &ok, -1);
  store("store_null", nullptr, &ok);
  const fc_rows no_data = {nullptr, 512, 128}, odd_stride = {somewhere<void>(), 12 * 128 + 4, 128}, backwards = {somewhere<void>(), -512, 128},
                askew = {somewhere<char>() + 8, 512, 128}, wide = {somewhere<void>(), (1 << 24) + 8, 128},
                tall = {somewhere<void>(), 128, (int64_t)1 << 31}, same = {somewhere<void>(), 0, 0};
  store("store_no_data", &ok, &no_data);
  store("store_odd_stride", &odd_stride, &ok);
  store("store_backwards", &ok, &backwards);
  store("store_askew", &askew, &ok);
  store("store_wide", &wide, &ok);
  store("store_tall", &ok, &tall);
  store("store_broadcast", &same, &ok);
  const int32_t too_many[2] = {200, 0}, nothing[2] = {0, 0};
  store("store_too_many", &ok, &ok, 0, too_many);
  store("store_short_table", &ok, &ok, 0, news, 2);
  store("store_nothing", nullptr, nullptr, 0, nothing);

  // attention
  auto attend = [&](const char* what, const fc_rows* q, const fc_rows* o, int n_q = 8, float* lse = nullptr, int win = 0, int layer = 0) {
    report(what, fc_chunk_attention(p16, layer, table, 8, lens, news, q, n_q, o, lse, win, 2, 0.f, nullptr));
  };
  attend("attend", &ok, &ok);
  report("attend8", fc_chunk_attention(p8, 0, table, 8, lens, news, &ok, 8, &ok, out32, 4, 2, 0.f, nullptr));
  attend("attend_heads", &ok, &ok, 6);
  attend("attend_few_heads", &ok, &ok, 0);
  const fc_rows all = {somewhere<void>(), 260 * 128, 128};
  attend("attend_group", &all, &all, 4 * 64);
  attend("attend_large_group", &all, &all, 4 * 65);
  attend("attend_window", &ok, &ok, 8, out32, 0);
  attend("attend_negative_window", &ok, &ok, 8, nullptr, -1);
  attend("attend_lse_askew", &ok, &ok, 8, reinterpret_cast<float*>(somewhere<char>() + 2), 4);
  attend("attend_layer", &ok, &ok, 8, nullptr, 0, 2);
  attend("attend_q", nullptr, &ok);
  attend("attend_out", &ok, nullptr);
  const fc_rows overlap = {somewhere<void>(), 128, 128}, broadcast = {somewhere<void>(), 0, 128}, head_major = {somewhere<void>(), 128, 34 * 128},
                close = {somewhere<void>(), 128, 33 * 128};
  attend("attend_overlap", &ok, &overlap);
  attend("attend_broadcast_out", &ok, &broadcast);
  attend("attend_broadcast_q", &broadcast, &ok);
  attend("attend_head_major", &head_major, &head_major);
  attend("attend_close", &ok, &close);
  int32_t long_chunk[1] = {900}, one[1] = {1};
  report("attend_split", fc_chunk_attention(p16, 0, table, 64, (long_chunk[0] = 30000, long_chunk), one, &ok, 4, &ok, nullptr, 0, 1, 0.f, nullptr));
  report("attend_split_table", fc_chunk_attention(p16, 0, table, 2048, long_chunk, one, &ok, 4, &ok, nullptr, 0, 1, 0.f, nullptr));

  // prompts
  const int32_t prompts[2] = {70, 3};
  report("prefill", fc_prefill_attention(p8, 1, prompts, &ok, &ok, &ok, 8, &ok, out32, 16, 2, 0.f, nullptr));
  report("prefill_k", fc_prefill_attention(p16, 1, prompts, &ok, nullptr, &ok, 8, &ok, nullptr, 0, 2, 0.f, nullptr));
  report("prefill_v", fc_prefill_attention(p16, 1, prompts, &ok, &ok, &no_data, 8, &ok, nullptr, 0, 2, 0.f, nullptr));
  report("prefill_lens", fc_prefill_attention(p16, 1, nullptr, &ok, &ok, &ok, 8, &ok, nullptr, 0, 2, 0.f, nullptr));
  report("prefill_none", fc_prefill_attention(p16, 1, nullptr, nullptr, nullptr, nullptr, 8, nullptr, nullptr, 0, 0, 0.f, nullptr));
  const int32_t beyond[1] = {32769};
  report("prefill_beyond", fc_prefill_attention(p16, 1, beyond, &ok, &ok, &ok, 8, &ok, nullptr, 0, 1, 0.f, nullptr));

  // quantise
  const int32_t cached[2] = {100, 16};
  report("quantise", fc_quantise_batch(p8, table, 8, p16, table, 8, cached, nullptr, 2, nullptr));
  report("quantise_back", fc_quantise_batch(p16, table, 8, p8, table, 8, cached, nullptr, 2, nullptr));
  report("quantise_other", fc_quantise_batch(p8, table, 8, other, table, 8, cached, nullptr, 2, nullptr));
  report("quantise_table", fc_quantise_batch(p8, table, 6, p16, table, 8, cached, nullptr, 2, nullptr));
  report("quantise_null", fc_quantise_batch(p8, nullptr, 8, p16, table, 8, cached, nullptr, 2, nullptr));
  report("quantise_off", fc_quantise_batch(p8, table, 8, p16, table, 8, cached, nothing, 2, nullptr));

  // more requests than fit the arguments: to the device, in a captured call as arguments
  const int n = 150;
  std::vector<int32_t> l(n, 20), ones(n, 1);
  for (bool captured : {false, true}) {
    g_capturing = captured;
    const std::string s = captured ? "_captured" : "";
    report(("many_store" + s).c_str(), fc_store_chunk(p16, 0, table, 2, l.data(), ones.data(), &ok, &ok, n, nullptr));
    report(("many_attend" + s).c_str(), fc_chunk_attention(p16, 0, table, 2, l.data(), ones.data(), &ok, 4, &ok, nullptr, 0, n, 0.f, nullptr));
    g_capturing = false;
  }
  for (fc_pool* p : {p8, p16, other}) fc_pool_destroy(p);
  return 0;
}
