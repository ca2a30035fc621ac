// Host-side checks that the entry points of the language-model operators share.
#pragma once
#include <climits>
#include <mutex>

#include "../launch.cuh"
#include "ifq.h"

namespace {

inline bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline int done(cudaError_t e) { return e == cudaSuccess ? IFQ_OK : IFQ_ECUDA; }
inline bool is16(int dtype) { return dtype == IFQ_F16 || dtype == IFQ_BF16; }

// Rows, tokens and columns are ints, and so are the ends of the blocks that they are rounded up to.
constexpr int kMaxSize = INT_MAX - 1023;

std::mutex g_lm_mu;   // guards a unit's per-device state

// A row stride in elements (0: dense): at least a row, in units of 16 bytes of a 16-bit type.
inline int stride_of(int64_t given, long long width, long long* out) {
  if (given < 0 || (given != 0 && (given < width || given % 8 != 0))) return IFQ_EINVAL;
  *out = given ? given : width;
  return IFQ_OK;
}

// SM count of the current device, or a full GB300's where there is none.
inline int sm_count() {
  static int known[kMaxDevices];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 152;
  std::lock_guard<std::mutex> lk(g_lm_mu);
  if (!known[dev] && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess) known[dev] = n;
  return known[dev] ? known[dev] : 152;
}

// Whether the instance's shared memory has been allowed on the current device; if not, do so.
template <typename K>
int allow_smem(K kern, int bytes, bool (&set)[kMaxDevices]) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return IFQ_ECUDA;
  std::lock_guard<std::mutex> lk(g_lm_mu);
  if (!set[dev]) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return IFQ_ECUDA;
    set[dev] = true;
  }
  return IFQ_OK;
}

}  // namespace
