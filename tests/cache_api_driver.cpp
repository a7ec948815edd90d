// The entry points on rotated rows, bounds of blocks and selected blocks (csrc/fc_cache_api.hip) and a 4-bit
// pool's calls on the CPU: the HIP runtime and the launchers of api_host_driver.cpp, and these.  Built and
// checked by test_cache_api.py; every line says what was called, its code and what was launched.  With an argument:
// calls at the limits of a launch.
#define main api_host_main
#include "api_host_driver.cpp"
#undef main

#include "../paper_2503_08461_amd/csrc/fc_cache_api.hip"
#include "../paper_2503_08461_amd/csrc/fc_chunk_api.hip"

static std::vector<ChunkReq> g_attended;
namespace fc {
hipError_t launch_extend(const ExtendParams& p, const ExtendReqs&, hipStream_t) { return launched("extend"); }
hipError_t launch_store_chunk(const StoreParams& p, const ChunkReqs&, hipStream_t) { return launched(("store" + std::to_string(p.e4m3)).c_str()); }
hipError_t launch_quantise(const QuantiseParams& p, const ChunkReqs&, hipStream_t) { return launched(("quantise" + std::to_string(p.e2m1)).c_str()); }
hipError_t launch_attention(const AttnParams& p, const ChunkReqs& reqs, hipStream_t) {
  std::string s = "attention" + std::to_string(p.source) + "x" + std::to_string(p.table_heads);
  g_attended.clear();
  if (!p.reqs) g_attended.assign(reqs.req, reqs.req + p.launch[0].n_req + p.launch[1].n_req);
  return launched(s.c_str());
}
hipError_t launch_rotate_store(const RotateParams& p, const ChunkReqs& reqs, hipStream_t) {
  std::string s = "rotate" + std::to_string(p.store.e4m3) + (p.store.reqs ? "" : "_inline") + ":" + std::to_string(p.store.n_rows) + "x" +
                  std::to_string(p.n_q_heads);
  if (!p.store.reqs)
    for (int i = 0; i < p.store.n_req; ++i) s += ":" + std::to_string(reqs.req[i].state_off);
  return launched(s.c_str());
}
hipError_t launch_bounds(const BoundsParams& p, const ChunkReqs&, hipStream_t) {
  return launched(("bounds" + std::to_string(p.format) + ":" + std::to_string(p.n_units)).c_str());
}
hipError_t launch_select_blocks(const SelectParams& p, const ChunkReqs&, const ChunkReqs&, hipStream_t) {
  std::string s = "select" + std::string(p.tokens ? "" : "_inline") + ":" + std::to_string(p.n_tokens) + ":" + std::to_string(p.n_req) + "x" +
                  std::to_string(p.n_units) + ":" + std::to_string(p.lds_keys);
  return launched(s.c_str());
}
hipError_t launch_selected_attention(const SelectParams& sp, const AttnParams& p, const ChunkReqs& tokens, hipStream_t) {
  std::string s = "selected" + std::to_string(p.source) + (sp.tokens ? "" : "_inline") + ":" + std::to_string(sp.n_tokens) + ":" +
                  std::to_string(sp.lds_keys);
  if (!sp.tokens)
    for (int i = 0; i < sp.n_tokens && i < 3; ++i)
      s += ":" + std::to_string(tokens.req[i].table_row) + "," + std::to_string(tokens.req[i].seq_len) + "," + std::to_string(tokens.req[i].row_off);
  return launched(s.c_str());
}
}  // namespace fc

// Calls just within and just beyond what one launch takes: fewer than 2^32 threads.
static int limits() {
  int32_t* table = somewhere<int32_t>();
  const fc_rows same = {somewhere<void>(), 0, 0};
  const fc_rotation turn = {somewhere<float>(), 32768, 128, 0};
  for (int beyond : {0, 1}) {
    const std::string s = beyond ? "_beyond" : "_within";
    auto pool_of = [&](int heads, int dtype) {
      fc_pool* p = nullptr;
      fc_pool_create(&p, somewhere<void>(), ~(size_t)0, 64, 16, 1, heads, 128, dtype);
      g_launched.clear();
      return p;
    };
    for (int dtype : {FC_DTYPE_F16, FC_DTYPE_E2M1}) {
      // workgroups of 256 threads, one a new token: 512 * 32768 = 2^24
      fc_pool* p = pool_of(1, dtype);
      std::vector<int32_t> lens(511 + beyond, 32768);
      report(("rotate" + s).c_str(), fc_rotate_store_chunk(p, 0, table, 2048, lens.data(), lens.data(), nullptr, &turn, nullptr, 0, nullptr, &same,
                                                           &same, (int)lens.size(), nullptr));
      // ... one a block: 8192 * 2048
      lens.assign(8191 + beyond, 32768);
      report(("bounds" + s).c_str(), fc_block_bounds(p, 0, table, 2048, lens.data(), lens.data(), somewhere<void>(), (int)lens.size(), nullptr));
      fc_pool_destroy(p);
      // of 512 threads, one a new token and head: 1024 * 8192 = 2^23
      p = pool_of(8192, dtype);
      const int32_t news[1] = {1023 + beyond};
      const fc_rows out = {somewhere<void>(), 8192 * 128, 128};
      for (int n_select : {1, 2048})
        report(("sparse" + s).c_str(), fc_sparse_attention(p, 0, table, 2048, news, news, somewhere<void>(), n_select, &same, 8192, &out, nullptr, 1,
                                                           0.f, nullptr));
      fc_pool_destroy(p);
    }
  }
  return 0;
}

int main(int argc, char**) {
  if (argc > 1) return limits();
  int32_t* table = somewhere<int32_t>();
  float* out32 = somewhere<float>();
  auto pool_of = [&](int dtype, int heads, int dim, size_t bytes) {
    fc_pool* p = nullptr;
    const int rc = fc_pool_create(&p, somewhere<void>(), bytes, 64, 16, 2, heads, dim, dtype);
    g_launched.clear();
    return rc == FC_OK ? p : nullptr;
  };
  // sizes: 17 / 32 bytes a channel
  for (int dim : {64, 128}) {
    const size_t bytes = (size_t)2 * 64 * 17 * 4 * dim;
    fc_pool *none = pool_of(FC_DTYPE_E2M1, 4, dim, bytes - 1), *some = pool_of(FC_DTYPE_E2M1, 4, dim, bytes);
    report("create4_small", none ? 0 : -1);
    report("create4", some ? 0 : -1);
    fc_pool_destroy(some);
  }
  fc_pool *p4 = pool_of(FC_DTYPE_E2M1, 4, 128, ~(size_t)0), *p8 = pool_of(FC_DTYPE_E4M3, 4, 128, ~(size_t)0);
  fc_pool *p16 = pool_of(FC_DTYPE_F16, 4, 128, ~(size_t)0), *other = pool_of(FC_DTYPE_F16, 4, 64, ~(size_t)0);

  // what a 4-bit pool refuses, before anything is launched
  int32_t lens[2] = {100, 40}, method[2] = {FC_METHOD_KNORM, FC_METHOD_SNAPKV}, budget[2] = {40, 40}, width[2] = {7, 7}, window[2] = {16, 16};
  const int32_t zeros[2] = {0, 0}, news[2] = {1, 33};
  report("compress4", fc_compress_batch(p4, table, 8, lens, table, 16, method, budget, 2, 7, 0.f, nullptr, nullptr, nullptr));
  report("noalloc4", fc_compress_batch_noalloc(p4, table, 8, lens, table, 16, method, budget, 2, 7, 0.f, nullptr, nullptr, nullptr));
  report("var4", fc_compress_batch_var(p4, table, 8, lens, table, window, method, budget, width, 2, 0.f, nullptr, nullptr, nullptr));
  report("lse4", fc_compress_batch_lse(p4, table, 8, lens, table, out32, 16, method, budget, 2, 7, 0.f, nullptr, nullptr, nullptr));
  report("window4", fc_window_lse(p4, table, 8, lens, table, 16, nullptr, 2, 0.f, out32, nullptr));
  report("kept4", fc_decode_attention_kept(p4, table, 8, lens, budget, table, table, out32, 2, 0.f, nullptr));
  report("mlp4", fc_compress_batch_mlp(p4, table, 8, lens, zeros, zeros, nullptr, 2, nullptr));
  // ... and takes
  const fc_rows ok = {somewhere<void>(), 12 * 128, 128};
  report("append4", fc_append_batch(p4, table, 8, lens, table, nullptr, 2, nullptr));
  report("decode4", fc_decode_attention(p4, table, 8, lens, table, out32, 2, 0.f, nullptr));
  report("store4", fc_store_chunk(p4, 0, table, 8, lens, news, &ok, &ok, 2, nullptr));
  report("attend4", fc_chunk_attention(p4, 0, table, 8, lens, news, &ok, 8, &ok, nullptr, 0, 2, 0.f, nullptr));
  report("prefill4", fc_prefill_attention(p4, 0, news, &ok, &ok, &ok, 8, &ok, nullptr, 0, 2, 0.f, nullptr));
  report("quantise4", fc_quantise_batch(p4, table, 8, p16, table, 8, lens, nullptr, 2, nullptr));
  report("quantise8", fc_quantise_batch(p8, table, 8, p16, table, 8, lens, nullptr, 2, nullptr));
  report("quantise4_from8", fc_quantise_batch(p4, table, 8, p8, table, 8, lens, nullptr, 2, nullptr));
  report("quantise4_back", fc_quantise_batch(p16, table, 8, p4, table, 8, lens, nullptr, 2, nullptr));
  report("quantise4_other", fc_quantise_batch(p4, table, 8, other, table, 8, lens, nullptr, 2, nullptr));

  // rotated rows
  const fc_rotation turn = {out32, 1000, 128, 0};
  auto rotate = [&](const char* what, const fc_rotation* r, const int32_t* positions = nullptr, const fc_rows* q = nullptr, int n_q = 0,
                    const fc_rows* o = nullptr, const fc_rows* k = nullptr, const fc_rows* v = nullptr, int layer = 0, fc_pool* p = nullptr,
                    const int32_t* n = nullptr, const int32_t* t = nullptr) {
    report(what, fc_rotate_store_chunk(p ? p : p16, layer, t ? t : table, 8, lens, n ? n : news, positions, r, q, n_q, o, k ? k : &ok, v ? v : &ok, 2,
                                       nullptr));
  };
  rotate("rotate", &turn);
  rotate("rotate4", &turn, nullptr, &ok, 8, &ok, &ok, &ok, 1, p4);
  rotate("rotate8", &turn, nullptr, &ok, 1, &ok, &ok, &ok, 1, p8);
  int32_t last[2] = {999, 967}, past[2] = {999, 968}, before[2] = {-1, 0}, far[2] = {0, 0x7fffffff};
  rotate("rotate_last", &turn, last);
  rotate("rotate_past", &turn, past);
  rotate("rotate_before", &turn, before);
  rotate("rotate_far", &turn, far);
  const int32_t only[2] = {0, 33};
  rotate("rotate_unused", &turn, before, nullptr, 0, nullptr, nullptr, nullptr, 0, nullptr, only);
  rotate("rotate_nothing", nullptr, nullptr, nullptr, 0, nullptr, nullptr, nullptr, 0, nullptr, zeros);
  rotate("rotate_null", nullptr);
  const fc_rotation no_table = {nullptr, 1000, 128, 0}, askew = {out32 + 1, 1000, 128, 0}, odd = {out32, 1000, 40, 0}, wide = {out32, 1000, 144, 0},
                    none = {out32, 1000, 0, 0}, empty = {out32, 0, 128, 0}, part = {out32, 1000, 48, 1};
  rotate("rotate_no_table", &no_table);
  rotate("rotate_askew", &askew);
  rotate("rotate_odd", &odd);
  rotate("rotate_wide", &wide);
  rotate("rotate_none", &none);
  rotate("rotate_empty", &empty);
  rotate("rotate_part", &part);
  rotate("rotate_q", &turn, nullptr, nullptr, 8, &ok);
  rotate("rotate_q_out", &turn, nullptr, &ok, 8, nullptr);
  rotate("rotate_heads", &turn, nullptr, &ok, -1, &ok);
  rotate("rotate_many_heads", &turn, nullptr, &ok, 4 * 64 + 1, &ok);
  const fc_rows same = {somewhere<void>(), 0, 0}, crooked = {somewhere<char>() + 8, 512, 128}, uneven = {somewhere<void>(), 12 * 128 + 4, 128};
  rotate("rotate_broadcast", &turn, nullptr, &same, 8, &ok, &same, &same);
  rotate("rotate_overlap", &turn, nullptr, &ok, 8, &same);
  rotate("rotate_k", &turn, nullptr, &ok, 8, &ok, &crooked);
  rotate("rotate_v", &turn, nullptr, &ok, 8, &ok, &ok, &uneven);
  rotate("rotate_layer", &turn, nullptr, nullptr, 0, nullptr, nullptr, nullptr, 2);
  report("rotate_tables", fc_rotate_store_chunk(p16, 0, nullptr, 8, lens, news, nullptr, &turn, nullptr, 0, nullptr, &ok, &ok, 2, nullptr));
  report("rotate_pool", fc_rotate_store_chunk(nullptr, 0, table, 8, lens, news, nullptr, &turn, nullptr, 0, nullptr, &ok, &ok, 2, nullptr));

  // bounds
  void* bounds = somewhere<void>();
  auto bound = [&](const char* what, fc_pool* p, void* b, const int32_t* n, int layer = 0, int mb = 8, const int32_t* t = nullptr) {
    report(what, fc_block_bounds(p, layer, t ? t : table, mb, lens, n, b, 2, nullptr));
  };
  printf("lens %d %d\n", lens[0], lens[1]);  // 101, 41
  bound("bounds", p16, bounds, lens);
  bound("bounds_new", p4, bounds, news);
  bound("bounds8", p8, bounds, news, 1);
  bound("bounds_null", p16, nullptr, news);
  bound("bounds_askew", p16, static_cast<char*>(bounds) + 8, news);
  bound("bounds_layer", p16, bounds, news, -1);
  bound("bounds_short_table", p16, bounds, news, 0, 6);
  bound("bounds_news", p16, bounds, nullptr);
  bound("bounds_nothing", p16, nullptr, zeros);
  int32_t more[2] = {102, 0};
  bound("bounds_more", p16, bounds, more);

  // selected blocks
  auto sparse = [&](const char* what, int n_select, const fc_rows* q, const fc_rows* o, int n_q = 8, void* b = nullptr, int32_t* sel = nullptr,
                    fc_pool* p = nullptr, const int32_t* n = nullptr) {
    report(what, fc_sparse_attention(p ? p : p16, 0, table, 8, lens, n ? n : news, b ? b : bounds, n_select, q, n_q, o, sel, 2, 0.f, nullptr));
  };
  const int32_t one[2] = {1, 1};
  sparse("sparse", 3, &ok, &ok, 8, nullptr, table, nullptr, one);
  sparse("sparse4", 2048, &ok, &ok, 4, nullptr, nullptr, p4);
  sparse("sparse8", 1, &ok, &ok, 4, nullptr, nullptr, p8);
  sparse("sparse_none", 0, &ok, &ok);
  sparse("sparse_many", 2049, &ok, &ok);
  sparse("sparse_q", 3, nullptr, &ok);
  sparse("sparse_out", 3, &ok, nullptr);
  sparse("sparse_overlap", 3, &ok, &same);
  sparse("sparse_heads", 3, &ok, &ok, 6);
  sparse("sparse_askew", 3, &ok, &ok, 8, static_cast<char*>(bounds) + 2);
  sparse("sparse_selected", 3, &ok, &ok, 8, nullptr, reinterpret_cast<int32_t*>(somewhere<char>() + 2));
  report("sparse_bounds", fc_sparse_attention(p16, 0, table, 8, lens, news, nullptr, 3, &ok, 8, &ok, nullptr, 2, 0.f, nullptr));
  sparse("sparse_nothing", 0, nullptr, nullptr, 0, nullptr, nullptr, nullptr, zeros);
  int32_t long_lens[1] = {30000}, first[1] = {1};
  report("sparse_long", fc_sparse_attention(p16, 0, table, 2048, long_lens, first, bounds, 64, &ok, 4, &ok, nullptr, 1, 0.f, nullptr));
  for (const ChunkReq& r : g_attended) printf("reads %d %d %d %d\n", r.table_row, r.seq_len, r.n_new, r.row_off);

  // two tokens of one of 8001 (the first one's block ends there), one of 41
  int32_t some_lens[2] = {8001, 41}, some_news[2] = {2, 1};
  report("sparse_apart", fc_sparse_attention(p8, 0, table, 2048, some_lens, some_news, bounds, 64, &ok, 4, &ok, nullptr, 2, 0.f, nullptr));
  for (const ChunkReq& r : g_attended) printf("reads %d %d %d %d\n", r.table_row, r.seq_len, r.n_new, r.row_off);
  // 33 query heads of a head
  const fc_rows many_q = {somewhere<void>(), 4 * 33 * 128, 128};
  report("sparse_rows", fc_sparse_attention(p16, 0, table, 8, lens, one, bounds, 3, &many_q, 4 * 33, &many_q, nullptr, 2, 0.f, nullptr));

  // captured: nothing is allocated (two tokens of 8000, so that scores need memory)
  const int n = 80;
  std::vector<int32_t> l(n, 8000), twos(n, 2);
  fc_pool* fresh = pool_of(FC_DTYPE_F16, 4, 128, ~(size_t)0);
  auto many = [&](const char* what, int n_req, bool captured) {
    g_capturing = captured;
    report(what, fc_sparse_attention(fresh, 0, table, 2048, l.data(), twos.data(), bounds, 3, &ok, 4, &ok, nullptr, n_req, 0.f, nullptr));
    g_capturing = false;
  };
  many("captured_first", 70, true);
  many("eager", 70, false);
  const char* used = fresh->sparse.data;
  many("captured", 70, true);
  printf("kept %d\n", (int)(fresh->sparse.captured && fresh->sparse.data == used));
  many("captured_many", n, true);  // (descriptors that no call left room for)
  l.assign(4000, 8000);
  twos.assign(4000, 2);
  report("eager_more", fc_sparse_attention(fresh, 0, table, 2048, l.data(), twos.data(), bounds, 3, &ok, 4, &ok, nullptr, 4000, 0.f, nullptr));
  printf("retired %d\n", (int)(fresh->retired.size() == 1 && fresh->retired[0] == used && !fresh->sparse.captured));
  for (fc_pool* p : {p4, p8, p16, other, fresh}) fc_pool_destroy(p);
  return 0;
}
