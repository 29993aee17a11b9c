// The context behind the C ABI and the host helpers shared by the files that implement it.
#pragma once

#include <vector>

#include "common.cuh"

struct sp_ctx {
  int device = 0;
  void* ws = nullptr;
  size_t ws_bytes = 0;
  int* status = nullptr;  // device int[4]: {code, where, work counter of the paired kernel, unused}
  int kernel = 0;         // 0 tensor-core (paired where supported), 1 CUDA-core cross-check, 2 tensor-core single-tile
  int64_t launches = 0;
  long long* trace = nullptr;  // caller's device buffer for the phase trace, or null
  int trace_cap = 0;
  // sp_prefill_attn_host: device copies of q, k, v, out (+ masks) and the copy streams
  void* stage = nullptr;
  size_t stage_bytes = 0;
  cudaStream_t s_in = nullptr, s_out = nullptr;
  std::vector<cudaEvent_t> events;
  // sp_tree_attn: partial results of units that several CTAs share.  Sized by the device alone, allocated once and never
  // moved, so that captured graphs keep a valid address.
  void* split_ws = nullptr;
  int n_sm = 0;           // set with it
};

namespace sp {

struct DeviceGuard {
  int prev = -1;
  bool ok = true;
  explicit DeviceGuard(int dev) {
    if (cudaGetDevice(&prev) != cudaSuccess) { ok = false; return; }
    if (prev != dev && cudaSetDevice(dev) != cudaSuccess) ok = false;
    target = dev;
  }
  ~DeviceGuard() {
    if (prev >= 0 && prev != target) cudaSetDevice(prev);
  }
  int target = -1;
};

}  // namespace sp
