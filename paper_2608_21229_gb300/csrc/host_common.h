// host_common.h -- what the library's translation units share on the host: the
// error message of the calling thread and the check of the current device.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace rc_host {

constexpr int kMaxDevices = 64;

// Records a message for refcache_last_error and returns `code`.
int fail(int code, const char* fmt, ...);
int cuda_fail(cudaError_t e, const char* what);

// The current device's number of SMs; REFCACHE_ERR_UNSUPPORTED unless it is an sm_103 device.
int device_sms(int* sms);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A launch as a programmatic dependent of the kernel before it on the stream: it
// waits (griddepcontrol.wait) before it touches any tensor.
template <typename Kernel, typename... Args>
cudaError_t launch_dependent(Kernel kernel, dim3 grid, dim3 block, size_t smem, cudaStream_t s, const Args&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  return e == cudaSuccess ? cudaGetLastError() : e;
}

}  // namespace rc_host
