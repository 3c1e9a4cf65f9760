// gpuos_model.cpp -- model operators as ordinary kernels on a caller's stream (gpuos_launch_model), and how
// their tasks are cut (gpuos_model_plan).  Their checks and packing are in gpuos_model.h.

#include <new>
#include <vector>

#include "../../include/gpuos.h"
#include "gpuos_internal.h"
#include "gpuos_model.h"
#include "gpuos_on_device.h"

using namespace gpuos;

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
    uint32_t count = 0, chunks = 0, variant = 0;
    const uint32_t head = i;                                    // (a task waits for those of earlier launches by the stream's order)
    for (; i < n && count < kModelLaunch; ++i) {
      const ModelHead& h = staged[i].h;
      if (h.path == PATH_NOP) continue;
      bool waits = count != 0 && (tasks[i].flags & GPUOS_FLAG_FENCE) != 0;
      for (int k = 0; k < 3; ++k) waits = waits || (count != 0 && tasks[i].dep[k] != 0 && tasks[i].dep[k] <= i - head);
      const uint32_t v = model_variant(h.impl, h.vec, h.dtype[0], h.flags);
      if (count != 0 && (waits || v != variant)) break;
      variant = v;
      l.rec[count++] = staged[i];
      chunks = h.nchunks > chunks ? h.nchunks : chunks;
    }
    if (count == 0) continue;
    const int rc = hip_status(launch_model(l, variant, chunks, count, stream), "launch of a model operator");
    if (rc != GPUOS_OK) return rc;
  }
  return GPUOS_OK;
}

int gpuos_model_plan(const gpuos_model_task* task, uint32_t impl_id, uint32_t out[8]) {
  if (!task || !out) return GPUOS_E_INVAL;
  const ModelCut cuts[2] = {kRingCut, kLaunchCut};
  for (int k = 0; k < 2; ++k) {
    ModelRecord r;
    const int rc = ModelPack::pack(*task, impl_id, &r, cuts[k]);
    if (rc != GPUOS_OK) return rc;
    out[4 * k] = r.h.path == PATH_NOP ? 2u : r.h.vec;
    out[4 * k + 1] = r.h.nchunks;
    out[4 * k + 2] = r.h.chunk;
    out[4 * k + 3] = impl_id == GPUOS_IMPL_LOGIT_PENALTY ? r.penalty.seg : (impl_id == GPUOS_IMPL_GAMMA_SUM ? 1u : r.h.block);
  }
  return GPUOS_OK;
}

}  // extern "C"
