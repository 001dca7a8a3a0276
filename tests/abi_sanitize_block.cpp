// Host-only driver of the C ABI of the gated projections, the norms around a block and the checkpoints, for a
// build whose host code carries AddressSanitizer and UndefinedBehaviorSanitizer (see abi_sanitize.cpp): size
// queries at the ends of their types, refusals, and valid arguments, which on a machine without a GPU must come
// back as HPR_ERR_HIP from the first runtime call.  No pointer is ever dereferenced by the host code.
#include <climits>
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

int main() {
  int n_dev = 0;
  if (hipGetDeviceCount(&n_dev) == hipSuccess && n_dev > 0) {
    std::printf("skipped: a GPU is visible\n");
    return 0;
  }
  uint16_t* p = reinterpret_cast<uint16_t*>(0x10000);
  uint8_t* exps = reinterpret_cast<uint8_t*>(0x20000);
  int8_t* codes = reinterpret_cast<int8_t*>(0x30000);
  void* ws = reinterpret_cast<void*>(0x70000);
  const size_t big = size_t(1) << 46;
  const hpr_status H = HPR_ERR_HIP;

  // every size of a call that the checks accept, small to large: the workspace that is asked for is enough, and one
  // byte less is not
  for (int64_t n : {int64_t(1), int64_t(33), int64_t(700), int64_t(6001), int64_t(1) << 18})
    for (int32_t k : {8, 72, 4096, 65536})
      for (int32_t f : {8, 1000, 65536})
        for (int dtype : {HPR_BF16, HPR_F16})
          for (int packed : {0, 1}) {
            expect("gated forward", gated_linear_fwd(p, k, n, k, p, p, f, HPR_GELU, dtype, p, nullptr), H);
            for (int needs : {1, 2, 3}) {
              uint16_t* dx = needs & 1 ? p : nullptr;
              uint16_t* dw = needs & 2 ? p : nullptr;
              const size_t need = gated_linear_bwd_workspace_size(n, k, f, packed, needs & 1, needs >> 1);
              auto call = [&](size_t bytes) {
                return gated_linear_bwd(p, p, packed ? exps : nullptr, k, n, k, p, p, f, HPR_SILU, dtype, dx, dw, dw,
                                        ws, bytes, nullptr);
              };
              expect("gated gradients", call(need), H);
              expect("gated gradients, workspace", call(need - 1), HPR_ERR_WORKSPACE_TOO_SMALL);
            }
          }
  for (int64_t n : {int64_t(1), int64_t(100), int64_t(5000), int64_t(1) << 22})
    for (int32_t d : {8, 512, 520, 1032, 4096, 4104, 8200, 16384})
      for (int kind : {HPR_RMS_NORM, HPR_LAYER_NORM})
        for (int rows : {0, 1}) {
          const hpr_norm q = {n, d, d, d, HPR_BF16, kind, rows, 0.5f, 1e-6f};
          uint16_t* bias = kind == HPR_LAYER_NORM ? p : nullptr;
          expect("norm forward", residual_norm_fwd(&q, p, p, p, bias, p, bias, p, p, p, nullptr), H);
          const size_t need = residual_norm_bwd_workspace_size(&q);
          for (int packed : {0, 1}) {
            const uint8_t* e = packed ? exps : nullptr;
            expect("norm gradients", residual_norm_bwd(&q, p, p, p, e, p, e, p, p, bias, p, p, p, p, bias, p, bias, p,
                                                       ws, need, nullptr), H);
            expect("norm gradients, workspace",
                   residual_norm_bwd(&q, p, p, p, e, p, e, p, p, bias, p, p, p, p, bias, p, bias, p, ws, need - 1,
                                     nullptr), HPR_ERR_WORKSPACE_TOO_SMALL);
          }
        }
  for (int64_t n : {int64_t(1), int64_t(1000), int64_t(1) << 18})
    for (int32_t d : {8, 1000, 65536}) {
      expect("pack", checkpoint_pack(p, d, n, d, HPR_F16, codes, exps, nullptr), H);
      expect("unpack", checkpoint_unpack(codes, exps, n, d, HPR_BF16, p, nullptr), H);
    }
  // the ends of the types
  for (int64_t n : {INT64_MIN, int64_t(-1), int64_t(1) << 31, INT64_MAX}) {
    expect("n", gated_linear_fwd(p, 64, n, 64, p, p, 64, 0, 0, p, nullptr), HPR_ERR_INVALID_ARG);
    expect("n", gated_linear_bwd(p, p, nullptr, 64, n, 64, p, p, 64, 0, 0, p, p, p, ws, big, nullptr),
           HPR_ERR_INVALID_ARG);
    expect("n", checkpoint_pack(p, 64, n, 64, 0, codes, exps, nullptr), HPR_ERR_INVALID_ARG);
    expect("n", checkpoint_unpack(codes, exps, n, 64, 0, p, nullptr), HPR_ERR_INVALID_ARG);
    const hpr_norm q = {n, 64, 64, 64, 0, 0, 0, 1.f, 1e-6f};
    expect("n", residual_norm_fwd(&q, p, p, p, nullptr, p, nullptr, p, p, p, nullptr), HPR_ERR_INVALID_ARG);
    if (gated_linear_bwd_workspace_size(n, 64, 64, 0, 1, 1) || residual_norm_bwd_workspace_size(&q)) ++failures;
  }
  for (int32_t k : {INT32_MIN, -8, 0, 4, 65544, INT32_MAX}) {
    expect("k", gated_linear_fwd(p, 64, 10, k, p, p, 64, 0, 0, p, nullptr), HPR_ERR_UNSUPPORTED_SHAPE);
    expect("f", gated_linear_fwd(p, 64, 10, 64, p, p, k, 0, 0, p, nullptr), HPR_ERR_UNSUPPORTED_SHAPE);
    const hpr_norm q = {10, 64, 64, k, 0, 0, 0, 1.f, 1e-6f};
    expect("dim", residual_norm_fwd(&q, p, p, p, nullptr, p, nullptr, p, p, p, nullptr),
           HPR_ERR_UNSUPPORTED_SHAPE);
    if (gated_linear_bwd_workspace_size(10, k, 64, 1, 1, 1) && (k < 8 || k > 65536)) ++failures;
  }
  for (int64_t row : {INT64_MIN, int64_t(-8), int64_t(3), int64_t(1) << 20, INT64_MAX}) {
    expect("row", gated_linear_fwd(p, row, 10, 64, p, p, 64, 0, 0, p, nullptr), HPR_ERR_UNSUPPORTED_SHAPE);
    expect("row", checkpoint_pack(p, row, 10, 64, 0, codes, exps, nullptr), HPR_ERR_UNSUPPORTED_SHAPE);
  }
  // the most rows of the widest rows
  if (!gated_linear_bwd_workspace_size(INT32_MAX, 65536, 65536, 1, 1, 1)) ++failures;
  std::printf("ok: %d failures\n", failures);
  return failures != 0;
}
