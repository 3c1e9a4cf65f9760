// gpuos_on_device.h -- the device that a call of the C interface works on.
#pragma once
#include <hip/hip_runtime_api.h>

#include "gpuos_model.h"

namespace gpuos {

// The device that a call works on, and the caller's again when it ends.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    int e = (int)hipGetDevice(&before_);
    if (e == (int)hipSuccess && before_ != device) {
      e = (int)hipSetDevice(device);
      changed_ = e == (int)hipSuccess;
    }
    status = hip_status(e, "hipSetDevice");
  }
  ~OnDevice() { if (changed_) (void)hipSetDevice(before_); }
  int status;
 private:
  int before_ = 0;
  bool changed_ = false;
};

}  // namespace gpuos
