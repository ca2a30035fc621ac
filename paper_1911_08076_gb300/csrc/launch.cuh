// Host-side helpers of the translation units that launch kernels: launches with programmatic
// dependent launch, the driver's tensor-map encoder, small arithmetic.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>

#include <cstdint>
#include <cstdlib>
#include <mutex>
#include <utility>

namespace {

constexpr int kMaxDevices = 64;

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }
inline size_t round_up(size_t a, size_t b) { return (a + b - 1) / b * b; }
inline cudaStream_t S(void* s) { return (cudaStream_t)s; }

// ---------------------------------------------------------------- driver entry point for TMA descriptors

PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;
std::once_flag g_encode_once;

bool get_encode() {
  std::call_once(g_encode_once, [] {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) ==
            cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      g_encode = (PFN_cuTensorMapEncodeTiled_v12000)fn;
  });
  return g_encode != nullptr;
}

// Programmatic dependent launch (on unless IFQ_PDL=0): a kernel may start its
// prologue while the previous kernel in the stream finishes; every kernel here
// waits (griddepcontrol.wait) before it touches global memory.
bool pdl_enabled() {
  static const bool on = [] {
    const char* v = getenv("IFQ_PDL");
    return !(v && v[0] == '0');
  }();
  return on;
}

template <typename... Exp, typename... Act>
cudaError_t launch_k(void (*kern)(Exp...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Act&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<Act>(args)...);
}

// A launch in clusters of `cluster` CTAs along x (grid.x a multiple of it), with programmatic
// dependent launch as in launch_k.
template <typename... Exp, typename... Act>
cudaError_t launch_k_cluster(void (*kern)(Exp...), int cluster, dim3 grid, dim3 block, size_t smem, cudaStream_t st,
                             Act&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = pdl_enabled() ? 1 : 0;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<Act>(args)...);
}

}  // namespace
