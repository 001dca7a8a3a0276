// Host-only driver of the encoder operators' C ABI for a build whose host code carries AddressSanitizer
// and UndefinedBehaviorSanitizer (see abi_sanitize.cpp): refusals, size queries at the ends of their
// types, and valid arguments, which on a machine without a GPU must come back as HPR_ERR_HIP from the
// first runtime call.  No pointer is ever dereferenced by the host code.
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>

#include <hip/hip_runtime_api.h>

#include "hiperrag.h"

static int failures = 0;

static void expect(const char* what, hpr_status got, hpr_status want) {
  if (got == want) return;
  std::fprintf(stderr, "FAIL %s: got %s, want %s (%s)\n", what, hpr_status_string(got),
               hpr_status_string(want), hpr_last_error());
  ++failures;
}

static void expect_size(const char* what, size_t got, size_t want) {
  if (got == want) return;
  std::fprintf(stderr, "FAIL %s: got %zu, want %zu\n", what, got, want);
  ++failures;
}

int main() {
  int n_dev = 0;
  if (hipGetDeviceCount(&n_dev) == hipSuccess && n_dev > 0) {
    std::printf("skipped: a GPU is visible\n");
    return 0;
  }
  uint16_t* p = reinterpret_cast<uint16_t*>(0x10000);
  const int64_t* off = reinterpret_cast<const int64_t*>(0x30000);
  const int32_t* ad = reinterpret_cast<const int32_t*>(0x40000);
  float* f = reinterpret_cast<float*>(0x50000);
  void* ws = reinterpret_cast<void*>(0x70000);
  const size_t big = size_t(1) << 40;
  const hpr_status H = HPR_ERR_HIP;

  const hpr_attention one = {100, 100, 1024, 128, 256, 128, 256, 128, 3, 8, 2, 128, HPR_BF16, 1, 0, 0.1f};
  auto fwd = [&](const hpr_attention& d, size_t bytes) {
    return packed_attention_fwd(&d, p, p, p, off, off, nullptr, p, f, ws, bytes, nullptr);
  };
  auto bwd = [&](const hpr_attention& d, size_t bytes) {
    return packed_attention_bwd(&d, p, p, p, p, p, f, off, off, nullptr, p, p, p, ws, bytes, nullptr);
  };
  // every size of a call that the checks accept, small to large: the workspace that is asked for is enough
  for (int64_t n_q : {int64_t(1), int64_t(33), int64_t(4096), int64_t(1) << 22})
    for (int64_t n_k : {int64_t(0), int64_t(1), int64_t(5000), int64_t(1) << 25})
      for (int32_t n_seq : {1, 7, 100000})
        for (int32_t group : {1, 3, 32}) {
          hpr_attention d = one;
          d.n_q = n_q;
          d.n_k = n_k;
          d.n_seq = n_seq;
          d.heads = 4 * group;
          d.kv_heads = 4;
          expect("attention fwd", fwd(d, packed_attention_workspace_size(&d)), H);
          expect("attention bwd", bwd(d, packed_attention_bwd_workspace_size(&d)), H);
          expect("attention bwd ws", bwd(d, packed_attention_bwd_workspace_size(&d) - 1), 5);
        }
  // sizes that no call takes
  for (int64_t n : {int64_t(-1), int64_t(1) << 31, INT64_MAX / 8, INT64_MAX, INT64_MIN}) {
    hpr_attention d = one;
    d.n_q = n;
    expect_size("fwd size, n_q", packed_attention_workspace_size(&d), 0);
    expect_size("bwd size, n_q", packed_attention_bwd_workspace_size(&d), 0);
    d = one;
    d.n_k = n;
    expect_size("fwd size, n_k", packed_attention_workspace_size(&d), 0);
    expect_size("bwd size, n_k", packed_attention_bwd_workspace_size(&d), 0);
    expect_size("adapter size, n", adapter_linear_bwd_workspace_size(n, 64, 32, 8, 2, 3), 0);
  }
  for (int32_t n : {-1, 0, INT_MAX, INT_MIN}) {
    hpr_attention d = one;
    d.heads = d.kv_heads = n;
    expect_size("fwd size, heads", packed_attention_workspace_size(&d), 0);
    expect_size("bwd size, heads", packed_attention_bwd_workspace_size(&d), 0);
    d = one;
    d.dim = n;
    expect_size("fwd size, dim", packed_attention_workspace_size(&d), 0);
    expect_size("adapter size, k", adapter_linear_bwd_workspace_size(10, n, 32, 8, 2, 3), 0);
    expect_size("adapter size, m", adapter_linear_bwd_workspace_size(10, 64, n, 8, 2, 3), 0);
    expect_size("adapter size, r", adapter_linear_bwd_workspace_size(10, 64, 32, n, 2, 3), 0);
    if (n != 0)
      expect_size("adapter size, n_ad", adapter_linear_bwd_workspace_size(10, 64, 32, 8, n, 3), 0);
    if (n < 0) {
      d = one;
      d.n_seq = n;
      expect_size("fwd size, n_seq", packed_attention_workspace_size(&d), 0);
      expect_size("bwd size, n_seq", packed_attention_bwd_workspace_size(&d), 0);
      expect_size("adapter size, n_req", adapter_linear_bwd_workspace_size(10, 64, 32, 8, 2, n), 0);
    }
  }
  expect_size("no description", packed_attention_workspace_size(nullptr), 0);
  expect_size("no description", packed_attention_bwd_workspace_size(nullptr), 0);
  for (int i = 0; i < 8; ++i) {  // the ends of every field, all at once and by turns
    hpr_attention d = one;
    if (i & 1) d.n_q = d.n_k = INT64_MAX;
    if (i & 2) d.n_seq = INT_MAX;
    if (i & 4) d.q_row = d.k_row = d.v_head = INT64_MAX;
    if (i == 0) d.scale = NAN;
    expect("attention ends", fwd(d, big), i == 0 ? 1 : 4);
    expect("attention ends", bwd(d, big), i == 0 ? 1 : 4);
  }

  auto afwd = [&](int64_t n, int32_t k, int32_t m, int32_t r, int32_t n_ad, int32_t n_req) {
    return adapter_linear_fwd(p, n, k, p, m, p, p, r, n_ad, f, off, ad, n_req, HPR_F16, p, p, nullptr);
  };
  auto abwd = [&](int64_t n, int32_t k, int32_t m, int32_t r, int32_t n_ad, int32_t n_req, size_t bytes) {
    return adapter_linear_bwd(p, p, n, k, p, m, p, p, r, n_ad, f, off, ad, n_req, HPR_F16, p, p, p, p, ws,
                              bytes, nullptr);
  };
  for (int64_t n : {int64_t(1), int64_t(777), int64_t(1) << 21})
    for (int32_t k : {8, 4096, 65536})
      for (int32_t m : {8, 2304})
        for (int32_t r : {1, 20, 128})
          for (int32_t n_req : {0, 1, 5000}) {
            const size_t need = adapter_linear_bwd_workspace_size(n, k, m, r, 3, n_req);
            expect("adapters fwd", afwd(n, k, m, r, 3, n_req), H);
            expect("adapters bwd", abwd(n, k, m, r, 3, n_req, need), H);
            expect("adapters bwd ws", abwd(n, k, m, r, 3, n_req, need - 1), 5);
          }
  expect("adapters n", afwd(INT64_MAX, 64, 32, 8, 2, 3), 4);
  expect("adapters n", abwd(INT64_MAX, 64, 32, 8, 2, 3, big), 4);
  expect("adapters k", abwd(10, INT_MAX - 7, 32, 8, 2, 3, big), 4);
  expect("adapters m", abwd(10, 64, INT_MAX - 7, 8, 2, 3, big), 4);
  expect("adapters n_req", abwd(10, 64, 32, 8, 2, INT_MAX, big), 4);
  expect("adapters n_ad", abwd(10, 64, 32, 8, INT_MAX, 3, big), 4);

  auto rot = [&](int64_t n, int64_t row, int32_t heads, int32_t dim) {
    return rotary_apply(p, row, 64, heads, p, row, 64, 2, n, dim, 64, ad, f, f, INT64_MAX, 0, HPR_BF16, p, p,
                        nullptr);
  };
  expect("rotary", rot(10, 512, 8, 64), H);
  expect("rotary large", rot(INT_MAX, INT64_MAX & ~int64_t(7), 4096, 1024), H);
  expect("rotary n", rot(INT64_MAX, 512, 8, 64), 1);
  expect("rotary heads", rot(10, 512, INT_MAX, 64), 4);
  std::printf("%s: %d failures\n", failures ? "FAILED" : "ok", failures);
  return failures ? 1 : 0;
}
