// The device of a call, chosen for as long as it lasts.
#pragma once
#include <cuda_runtime.h>

namespace cllm {

// A handle's device for a call (its memory, its tensor maps and the default stream are that
// device's), then the caller's again.
class OnDevice {
 public:
  explicit OnDevice(int dev) {
    error = cudaGetDevice(&before_);
    if (error != cudaSuccess || before_ == dev) return;
    error = cudaSetDevice(dev);
    back_ = error == cudaSuccess;
  }
  ~OnDevice() {
    if (back_) cudaSetDevice(before_);
  }
  OnDevice(const OnDevice&) = delete;
  OnDevice& operator=(const OnDevice&) = delete;
  cudaError_t error;

 private:
  int before_ = 0;
  bool back_ = false;
};

}  // namespace cllm
