// gpuos_cache.cpp -- cache operators on a caller's stream (gpuos_launch_cache, gpuos_cache_workspace).  Their checks and
// packing are in gpuos_cache.h.

#include "gpuos_cache.h"

#include "gpuos_on_device.h"

using namespace gpuos;

extern "C" {

int gpuos_launch_cache(int32_t device, const gpuos_cache_task* task, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!task) return GPUOS_E_INVAL;
  bool empty = false;
  if (task->op == GPUOS_CACHE_APPEND) {
    AppendArgs a;
    const int rc = CachePack::append(*task, &a, &empty);
    if (rc != GPUOS_OK || empty) return rc;
    OnDevice on(device);
    return on.status != GPUOS_OK ? on.status : hip_status(launch_append(a, stream), "launch of a cache operator");
  }
  AttendArgs a;
  uint32_t format = 0;
  uint64_t bytes = 0;
  const int rc = CachePack::attend(*task, &a, &format, &bytes, &empty);
  if (rc != GPUOS_OK || empty) return rc;
  const uint64_t sums = a.joined ? (uint64_t)a.pieces * GPUOS_CACHE_SUMS_BYTES((uint64_t)a.b, a.s, a.hq, a.d) : 0;
  if (bytes < sums) bytes = sums;
  if (bytes != 0 && (!workspace || (uint64_t)workspace % 16 != 0 || workspace_bytes < bytes)) return GPUOS_E_NOMEM;
  a.part = (uint64_t)workspace;
  a.stats = a.part + (uint64_t)a.pieces * a.b * a.s * a.hq * a.d * 4u;
  OnDevice on(device);
  return on.status != GPUOS_OK ? on.status : hip_status(launch_attend(a, format, stream), "launch of a cache operator");
}

int gpuos_cache_workspace(const gpuos_cache_task* task, uint64_t* bytes) {
  if (!task || !bytes) return GPUOS_E_INVAL;
  bool empty = false;
  *bytes = 0;
  if (task->op == GPUOS_CACHE_APPEND) {
    AppendArgs a;
    return CachePack::append(*task, &a, &empty);
  }
  AttendArgs a;
  uint32_t format = 0;
  return CachePack::attend(*task, &a, &format, bytes, &empty);
}

}  // extern "C"
