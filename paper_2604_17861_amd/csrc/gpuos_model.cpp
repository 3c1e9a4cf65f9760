// gpuos_model.cpp -- model operators as ordinary kernels on a caller's stream (gpuos_launch_model), and how
// their tasks are cut (gpuos_model_plan).  Their checks and packing are in gpuos_model.h.

#include <hip/hip_runtime_api.h>

#include <new>
#include <vector>

#include "../../include/gpuos.h"
#include "gpuos_internal.h"
#include "gpuos_model.h"

using namespace gpuos;

namespace {

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

}  // namespace

extern "C" {

int gpuos_launch_model(int32_t device, const gpuos_model_task* tasks, uint32_t n, const uint32_t* impl_of_op, void* stream) {
  if ((!tasks && n) || !impl_of_op) return GPUOS_E_INVAL;
  if (n == 0) return GPUOS_OK;
  static thread_local std::vector<ModelRecord> staged;
  try {
    staged.resize(n);
  } catch (const std::bad_alloc&) {                             // no exception may cross the C boundary
    return GPUOS_E_NOMEM;
  }
  for (uint32_t i = 0; i < n; ++i) {
    const uint32_t impl = tasks[i].op_id < GPUOS_MAX_OPS ? impl_of_op[tasks[i].op_id] : (uint32_t)GPUOS_IMPL_NONE;
    if (!impl_is_model(impl)) return GPUOS_E_BADOP;             // (GPUOS_IMPL_FAIL, the kill switch, too)
    const int rc = ModelPack::pack(tasks[i], impl, &staged[i], kLaunchCut);
    if (rc != GPUOS_OK) return rc;
  }
  OnDevice on(device);
  if (on.status != GPUOS_OK) return on.status;
  ModelLaunch l;
  uint32_t i = 0;
  while (i < n) {
    uint32_t count = 0, blocks = 0, impl = 0;
    const uint32_t head = i;                                    // (a task waits for those of earlier launches by the stream's order)
    for (; i < n && count < kModelLaunch; ++i) {
      const ModelHead& h = staged[i].h;
      if (h.path == PATH_NOP) continue;
      bool waits = count != 0 && (tasks[i].flags & GPUOS_FLAG_FENCE) != 0;
      for (int k = 0; k < 3; ++k) waits = waits || (count != 0 && tasks[i].dep[k] != 0 && tasks[i].dep[k] <= i - head);
      if (count != 0 && (waits || h.impl != impl)) break;
      impl = h.impl;
      l.rec[count] = staged[i];
      l.first[count++] = blocks;
      blocks += h.nchunks;
    }
    if (count == 0) continue;
    for (uint32_t k = count; k < kModelLaunch; ++k) l.first[k] = 0xffffffffu;
    const int rc = hip_status(launch_model(l, impl, blocks, stream), "launch of a model operator");
    if (rc != GPUOS_OK) return rc;
  }
  return GPUOS_OK;
}

int gpuos_model_plan(const gpuos_model_task* task, uint32_t impl_id, uint32_t out[6]) {
  if (!task || !out) return GPUOS_E_INVAL;
  ModelRecord ring, launch;
  int rc = ModelPack::pack(*task, impl_id, &ring, kRingCut);
  if (rc == GPUOS_OK) rc = ModelPack::pack(*task, impl_id, &launch, kLaunchCut);
  if (rc != GPUOS_OK) return rc;
  out[0] = ring.h.path == PATH_NOP ? 2u : (launch.h.vec != 0 ? 1u : 0u);
  out[1] = ring.h.nchunks; out[2] = ring.h.chunk;
  out[3] = launch.h.nchunks; out[4] = launch.h.chunk;
  out[5] = impl_id == GPUOS_IMPL_LOGIT_PENALTY ? launch.penalty.seg : 0u;
  return GPUOS_OK;
}

}  // extern "C"
