// Host side: the device an entry point works on is current for the call, and the caller's is put back.
#pragma once

#include <cuda_runtime.h>

#include <string>

#include "hack_internal.h"

namespace hack {

struct DeviceScope {
  int prev = -1;
  bool switched = false;
  cudaError_t err = cudaSuccess;
  explicit DeviceScope(int want) {
    err = cudaGetDevice(&prev);
    if (err == cudaSuccess && prev != want) {
      err = cudaSetDevice(want);
      switched = err == cudaSuccess;
    }
    if (err != cudaSuccess) cudaGetLastError();      // reported by the caller, not by the next launch
  }
  ~DeviceScope() { if (switched) cudaSetDevice(prev); }
};

}  // namespace hack

#define HACK_ON_DEVICE_OF(device)                                                                     \
  hack::DeviceScope dev_scope_(device);                                                               \
  if (dev_scope_.err != cudaSuccess) {                                                                \
    hack::set_error(std::string("selecting the device: ") + cudaGetErrorString(dev_scope_.err));      \
    return HACK_ERR_CUDA;                                                                             \
  }
