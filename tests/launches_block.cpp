// Host-only recorder of the launches that the gated projections' gradients make: the HIP runtime's launch entry points
// are this program's own, which write down what they are given, so that a machine without a GPU can say what a call would
// launch and on which addresses.  No pointer is ever dereferenced.
//
//   launches_block n k f dtype packed needs      (needs: 1 dx, 2 the weights' gradients, 3 both)
// prints the call's status, and a line a launch: kernel, workgroups, threads and, of a kernel of d, where the largest
// |dh| of the columns are (bytes from the workspace).
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <string>

#include <hip/hip_runtime.h>

#include "hiperrag.h"
#include "kernels.h"

static std::map<const void*, std::string>& names() {
  static std::map<const void*, std::string> m;
  return m;
}
static struct {
  dim3 grid, block;
  size_t lds;
  hipStream_t stream;
} given;
static char* const kWorkspace = reinterpret_cast<char*>(uintptr_t(1) << 40);

extern "C" {
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*,
                           int*) {
  names()[host] = name;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
  given = {grid, block, lds, stream};
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* stream) {
  *grid = given.grid;
  *block = given.block;
  *lds = given.lds;
  *stream = given.stream;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
  const std::string& name = names()[f];
  std::printf("%s %u %u", name.c_str(), grid.x, block.x);
  if (name.find("gated_kernel") != std::string::npos || name.find("gated_few_kernel") != std::string::npos) {
    const hpr::GatedArgs& a = *static_cast<const hpr::GatedArgs*>(args[0]);
    std::printf(" %lld", (long long)(reinterpret_cast<const char*>(a.col_max) - kWorkspace));
  }
  std::printf("\n");
  return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetLastError(void) { return hipSuccess; }
}

int main(int argc, char** argv) {
  if (argc != 7) return 2;
  const int64_t n = std::atoll(argv[1]);
  const int32_t k = std::atoi(argv[2]), f = std::atoi(argv[3]), dtype = std::atoi(argv[4]);
  const int packed = std::atoi(argv[5]), needs = std::atoi(argv[6]);
  uint16_t* const p = reinterpret_cast<uint16_t*>(0x10000);
  const size_t size = gated_linear_bwd_workspace_size(n, k, f, packed, needs & 1, needs >> 1);
  const hpr_status st = gated_linear_bwd(
      p, p, packed ? reinterpret_cast<const uint8_t*>(p) : nullptr, k, n, k, p, p, f, HPR_SILU, dtype,
      needs & 1 ? p : nullptr, needs & 2 ? p : nullptr, needs & 2 ? p : nullptr, kWorkspace, size, nullptr);
  std::printf("status %s\n", hpr_status_string(st));
  return 0;
}
