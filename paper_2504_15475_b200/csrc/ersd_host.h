// What the entry points of every translation unit share on the host.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include "ersd.h"

namespace ersd {

__attribute__((visibility("hidden"))) int cuda_fail(cudaError_t e);  // keeps the error for ersd_last_cuda_error()
__attribute__((visibility("hidden"))) int sm_count();                // multiprocessors of the current device
__attribute__((visibility("hidden"))) void note_launch(const char* format, ...);  // text of ersd_last_launch()

// A launch that may start while the kernel before it on the stream still runs (see
// wait_for_previous_kernel), in clusters of CL blocks.
struct Launch {
  cudaLaunchConfig_t cfg;
  cudaLaunchAttribute at[2];
  Launch(dim3 grid, unsigned threads, size_t smem, cudaStream_t st, unsigned CL = 1) {
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = CL;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = CL > 1 ? 2 : 1;
  }
  Launch(const Launch&) = delete;
};

// A caller's structure of options, cut or filled with zeros to the size this library knows.
template <typename T>
static inline T read_struct(const T* given) {
  T o;
  memset(&o, 0, sizeof o);
  if (given) {
    size_t n = given->struct_size;
    if (n == 0 || n > sizeof o) n = sizeof o;
    memcpy(&o, given, n);
  }
  return o;
}

static inline bool aligned_to(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// Whether parent[0..R) is a draft tree: node 0 the root, every other node behind its parent.
static inline bool is_tree(const int32_t* parent, int R) {
  if (parent[0] != -1) return false;
  for (int n = 1; n < R; ++n)
    if (parent[n] < 0 || parent[n] >= n) return false;
  return true;
}

}  // namespace ersd
