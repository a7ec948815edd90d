// Scratch memory of captured calls (csrc/fc_api.hip) on the CPU, over the HIP runtime of
// api_host_driver.cpp, whose device allocations and frees are counted here.  Built and checked by
// test_captured_scratch.py.  A line per step: its name, code, device buffers made and freed by it.
#include <hip/hip_runtime.h>

#include <cstdlib>
#include <cstring>
#include <set>

static std::set<void*> g_live;  // device buffers (pinned ones are not counted)
static int g_made = 0, g_freed = 0;
static void* counted_calloc(size_t n, size_t size, const char* by) {
  void* at = calloc(n, size);
  if (!strcmp(by, "give") && g_live.insert(at).second) ++g_made;
  return at;
}
static void counted_free(void* at, const char* by) {
  if (!strcmp(by, "hipFree") && g_live.erase(at)) ++g_freed;
  free(at);
}
#define calloc(n, size) counted_calloc(n, size, __func__)
#define free(at) counted_free(at, __func__)
#define main api_host_main
#include "api_host_driver.cpp"
#undef main

int main() {
  fc_pool* p = nullptr;
  auto line = [&](const char* what, int rc) {
    printf("%s %d %d %d %s\n", what, rc, g_made, g_freed, g_launched.c_str());
    g_made = g_freed = 0;
    g_launched.clear();
  };
  auto create = [&] {
    fc_pool_create(&p, somewhere<void>(), ~(size_t)0, 1 << 22, 16, 1, 32, 128, FC_DTYPE_F16);
    g_launched.clear();
    g_made = g_freed = 0;
  };
  auto call = [&](const char* what, const char* name, bool captured, int n, int len) {
    std::vector<int32_t> lens(n, len), budgets(n, len / 4), methods(n, FC_METHOD_KNORM), zeros(n, 0);
    std::vector<int32_t> snap(n, FC_METHOD_SNAPKV);
    g_capturing = captured;
    int rc = 0;
    if (!strcmp(what, "window_lse"))
      rc = fc_window_lse(p, somewhere<int32_t>(), 2048, lens.data(), somewhere<void>(), 32, nullptr, n, 0.f,
                         somewhere<float>(), nullptr);
    else if (!strcmp(what, "mlp"))
      rc = fc_compress_batch_mlp(p, somewhere<int32_t>(), 2048, lens.data(), zeros.data(), lens.data(), nullptr, n, nullptr);
    else if (!strcmp(what, "noalloc"))
      rc = fc_compress_batch_noalloc(p, somewhere<int32_t>(), 2048, lens.data(), nullptr, 32, methods.data(), budgets.data(),
                                     n, 7, 0.f, nullptr, nullptr, nullptr);
    else
      rc = fc_compress_batch(p, somewhere<int32_t>(), 2048, lens.data(), nullptr, 32, methods.data(), budgets.data(), n, 7,
                             0.f, nullptr, nullptr, nullptr);
    g_capturing = false;
    const int free_now = fc_pool_num_free(p), unchanged = lens[0] == len;
    line(name, rc);
    if (rc != FC_OK) printf("%s_left %d %d\n", name, free_now == 1 << 22, unchanged);
    fc_pool_import_state_dev(p, somewhere<int32_t>(), 1 << 22, nullptr);
    g_launched.clear();
  };
  auto weights = [&](const char* name, bool captured = false) {
    const _Float16 w1[256 * 128] = {}, w2[128 * 256] = {};
    const float b1[256] = {}, b2[128] = {};
    const fc_mlp_weights w = {1, 256, FC_ACT_GELU_ERF, {w1, w1}, {b1, b1}, {w2, w2}, {b2, b2}};
    g_capturing = captured;
    const int rc = fc_mlp_set_weights(p, &w, nullptr);
    g_capturing = false;
    line(name, rc);
  };
  auto destroy = [&](const char* name) {
    fc_pool_destroy(p);
    printf("%s %zu\n", name, g_live.size());
    g_made = g_freed = 0;
  };

  // the log-sum-exps' descriptors
  create();
  call("window_lse", "lse_first", true, 100, 200);  // nothing there to put them in
  call("window_lse", "lse_eager", false, 100, 200);
  call("window_lse", "lse_captured", true, 100, 200);
  call("window_lse", "lse_grows", false, 2000, 200);
  call("window_lse", "lse_grows_again", false, 40000, 200);  // no graph uses the one before
  destroy("lse_end");

  // a compression in the fused kernels: block ids and descriptors
  create();
  call("compress", "fused_first", true, 64, 800);
  call("noalloc", "fused_noalloc", true, 64, 800);  // (its scratch is always there)
  call("compress", "fused_eager", false, 64, 800);
  call("compress", "fused_captured", true, 64, 800);
  call("compress", "fused_more", true, 4000, 800);
  call("compress", "fused_grows", false, 4000, 800);
  call("compress", "fused_grows_again", false, 40000, 800);
  destroy("fused_end");

  // heads split over workgroups: scores and kept lists as well
  create();
  call("compress", "split_eager", false, 1, 8000);
  call("compress", "split_captured", true, 1, 8000);
  call("compress", "split_grows", false, 1, 30000);
  call("compress", "split_grows_again", false, 2, 32000);
  destroy("split_end");

  // the separate kernels
  create();
  fc_set_score_mode(p, FC_SCORE_TWO_PASS);
  call("compress", "separate_first", true, 8, 800);
  call("compress", "separate_eager", false, 8, 800);
  call("compress", "separate_captured", true, 8, 800);
  call("compress", "separate_grows", false, 200, 800);
  destroy("separate_end");

  // the chunk MLP: and the weights, which new ones replace
  create();
  weights("weights");
  call("mlp", "mlp_first", true, 64, 800);
  call("mlp", "mlp_eager", false, 64, 800);
  weights("weights_replaced");
  call("mlp", "mlp_captured", true, 64, 800);
  weights("weights_captured", true);
  weights("weights_kept");
  weights("weights_replaced_again");
  call("mlp", "mlp_grows", false, 4000, 800);
  destroy("mlp_end");

  // ownership checks read their verdict on the host
  create();
  weights("weights_checked");
  call("compress", "checked_eager", false, 64, 800);
  call("mlp", "checked_mlp_eager", false, 64, 800);
  fc_set_debug_checks(p, 1);
  g_launched.clear();
  g_made = g_freed = 0;
  call("compress", "checked_first", true, 64, 800);
  call("mlp", "checked_mlp", true, 64, 800);
  fc_pool_import_state_dev(p, somewhere<int32_t>(), 100, nullptr);
  g_launched.clear();
  g_capturing = true;
  line("checked_free", fc_pool_free(p, somewhere<int32_t>(), 5, nullptr));
  g_capturing = false;
  printf("checked_free_left %d 1\n", fc_pool_num_free(p) == 100);
  destroy("checked_end");
  return 0;
}
