// Host side of the entry points: the device they work on is current for the call and the caller's is put back; checks of
// strided tensors.
#pragma once

#include <cuda_runtime.h>

#include <algorithm>
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

// What is wrong with a [batch, heads, tokens, head_dim] tensor whose rows start on 16-byte boundaries, or NULL; one that is
// written has a place of its own for every row.
inline const char* view_error(const void* ptr, const hack_strides_t& s, int batch, int heads, int tokens, int head_dim, int elt, bool written) {
  if (!ptr) return "a tensor is NULL";
  const int unit = 16 / elt;
  if ((reinterpret_cast<uintptr_t>(ptr) & 15) || s.batch % unit || s.head % unit || s.token % unit) return "rows must start on 16-byte boundaries";
  if (!written) return nullptr;
  struct Dim { long long stride, n; } d[3] = {{s.batch, batch}, {s.head, heads}, {s.token, tokens}};
  std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  long long extent = head_dim;                // elements that the inner dimensions take
  for (const Dim& x : d) {
    if (x.n == 1) continue;
    if (x.stride < extent) return "rows of an output overlap";
    extent += x.stride * (x.n - 1);
  }
  return nullptr;
}

// Whether an array of `elt`-byte numbers (or NULL) starts off their size: the kernels read them one by one.
inline bool off_its_size(const void* ptr, int elt) { return reinterpret_cast<uintptr_t>(ptr) % elt != 0; }

}  // namespace hack

#define HACK_ON_DEVICE_OF(device)                                                                     \
  hack::DeviceScope dev_scope_(device);                                                               \
  if (dev_scope_.err != cudaSuccess) {                                                                \
    hack::set_error(std::string("selecting the device: ") + cudaGetErrorString(dev_scope_.err));      \
    return HACK_ERR_CUDA;                                                                             \
  }
