// The handle behind the C ABI and the small host helpers its entry points share.
#pragma once
#include <stdio.h>

#include "ckv_internal.h"

struct criticalkv_handle_s {
  int device;
  int sm_count;
  int cc_major, cc_minor;
  int* status_word;  // device
  int smem_optin;
  int last_path;
  int last_select_fused;
  int last_decode;   // 1: tensor cores, 2: CUDA cores
  long long launches;
  char cuda_error[256];
  // host-staged path: two copy/compute streams and the events that tie them to the caller's stream
  bool host_ready;
  cudaStream_t host_stream[2];
  cudaEvent_t host_event[3];
};

namespace ckv {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int record_cuda(criticalkv_handle h, cudaError_t e) {
  if (e == cudaSuccess) return CKV_OK;
  if (h) snprintf(h->cuda_error, sizeof(h->cuda_error), "%s: %s", cudaGetErrorName(e), cudaGetErrorString(e));
  return CKV_ECUDA;
}

struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; prev = -1; return; }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    if (prev == dev) prev = -1;
  }
  ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

}  // namespace ckv
