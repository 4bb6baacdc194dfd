// host_common.h -- what the library's translation units share on the host: the
// error message of the calling thread and the check of the current device.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace rc_host {

constexpr int kMaxDevices = 64;

// Records a message for refcache_last_error and returns `code`.
int fail(int code, const char* fmt, ...);
int cuda_fail(cudaError_t e, const char* what);

// The current device's number of SMs; REFCACHE_ERR_UNSUPPORTED unless it is an sm_103 device.
int device_sms(int* sms);

// The current device and its error word (refcache_status), whose address is looked up once.
int device_status_word(int* dev, int** word);

// The limit of every wait in a kernel, and the fault injection of the next launch (cleared).
uint64_t wait_timeout_ns();
int take_debug_stop();

// 2-D tensor maps.  `outer` rows of `inner` bytes, `pitch` bytes apart: boxes of 128 bytes x box_outer
// rows with the 128-byte swizzle; `lines` lines of 512 bytes, one line a box.
int encode_map(CUtensorMap* m, const void* base, int64_t inner, int64_t outer, int64_t pitch, uint32_t box_outer);
int encode_lines(CUtensorMap* m, const void* base, int64_t lines);

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
