// Launches that may begin while the kernel before them in the stream ends, and
// launches on the device that holds a pointer.
#pragma once
#include <atomic>
#include <utility>

#include "common.cuh"

namespace shard {

// Launches `kern` with programmatic dependent launch: its CTAs may take their
// places once every CTA of the preceding kernel has called
// pdl_launch_dependents() (or ended). The kernel calls pdl_wait() before its
// first access to anything another kernel writes or reads.
template <class... Params, class... Args>
cudaError_t launch_behind(void (*kern)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...);
}

// Whether pointers are aligned to values of 4 bytes (null ones are).
template <class... P>
bool aligned4(const P*... p) {
  return (((reinterpret_cast<uintptr_t>(p)) | ...) & 3) == 0;
}

// SMs of a device (0: unknown).
inline int sms_of(int device) {
  static std::atomic<int> known[64];
  int v = device < 64 ? known[device].load() : 0;
  if (!v && cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, device) == cudaSuccess && device < 64) known[device].store(v);
  return v;
}

// Makes the device that holds p current for its lifetime.
class OnDeviceOf {
 public:
  explicit OnDeviceOf(const void* p) {
    cudaPointerAttributes at{};
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
      cudaGetLastError();  // not left for the next launch's check
      return;
    }
    if (at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged) return;
    if (cudaGetDevice(&before_) != cudaSuccess || (before_ != at.device && cudaSetDevice(at.device) != cudaSuccess)) return;
    device_ = at.device;
  }
  ~OnDeviceOf() {
    if (device_ >= 0 && device_ != before_) cudaSetDevice(before_);
  }
  OnDeviceOf(const OnDeviceOf&) = delete;
  OnDeviceOf& operator=(const OnDeviceOf&) = delete;
  bool error() const { return device_ < 0; }
  int device() const { return device_; }

 private:
  int before_ = -1, device_ = -1;
};

}  // namespace shard
