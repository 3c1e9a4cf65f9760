// gpuos_model.hip -- the model operators as ordinary kernels on a caller's stream (gpuos_launch_model): the
// executors of gpuos_model_device.h, a block a chunk.  Records and block numbers are kernel arguments, so a launch
// allocates and copies nothing and may be captured.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gpuos_model_device.h"

namespace gpuos {

typedef const __attribute__((address_space(4))) ModelRecord* const_record_t;

template <int IMPL> DEV void run_model(const_record_t r, uint32_t chunk, float* s, uint32_t tid) {
  const uint32_t vec = uni((uint32_t)r->h.vec), dt = uni((uint32_t)r->h.dtype[0]);
  if constexpr (IMPL == GPUOS_IMPL_NORM_ROPE || IMPL == GPUOS_IMPL_NORM_ROPE_GRAD) {
    constexpr bool GRAD = IMPL == GPUOS_IMPL_NORM_ROPE_GRAD;
    const RopeArgs a = rope_args(&r->rope);
    if (vec == 0) rope_elements<POL_PLAIN, GRAD>(a, chunk, s, tid);
    else if (!a.pairs) {
      if (dt == GPUOS_F32) rope_vectors<POL_PLAIN, GPUOS_F32, false, GRAD>(a, chunk, s, tid);
      else if (dt == GPUOS_F16) rope_vectors<POL_PLAIN, GPUOS_F16, false, GRAD>(a, chunk, s, tid);
      else rope_vectors<POL_PLAIN, GPUOS_BF16, false, GRAD>(a, chunk, s, tid);
    } else {
      if (dt == GPUOS_F32) rope_vectors<POL_PLAIN, GPUOS_F32, true, GRAD>(a, chunk, s, tid);
      else if (dt == GPUOS_F16) rope_vectors<POL_PLAIN, GPUOS_F16, true, GRAD>(a, chunk, s, tid);
      else rope_vectors<POL_PLAIN, GPUOS_BF16, true, GRAD>(a, chunk, s, tid);
    }
  } else if constexpr (IMPL == GPUOS_IMPL_GAMMA_SUM) {
    gamma_sum<POL_PLAIN>(rope_args(&r->rope), chunk, tid);
  } else if constexpr (IMPL == GPUOS_IMPL_CACHE_STORE) {
    const CacheArgs a = cache_args(&r->cache);
    if (vec == 0) store_elements<POL_PLAIN>(a, chunk, tid);
    else if (dt == GPUOS_F32) store_vectors<POL_PLAIN, GPUOS_F32>(a, chunk, tid);
    else if (dt == GPUOS_F16) store_vectors<POL_PLAIN, GPUOS_F16>(a, chunk, tid);
    else store_vectors<POL_PLAIN, GPUOS_BF16>(a, chunk, tid);
  } else if constexpr (IMPL == GPUOS_IMPL_CACHE_LOAD) {
    const CacheArgs a = cache_args(&r->cache);
    if (vec == 0) load_elements<POL_PLAIN>(a, chunk, tid);
    else if (dt == GPUOS_F32) load_vectors<POL_PLAIN, GPUOS_F32>(a, chunk, tid);
    else if (dt == GPUOS_F16) load_vectors<POL_PLAIN, GPUOS_F16>(a, chunk, tid);
    else load_vectors<POL_PLAIN, GPUOS_BF16>(a, chunk, tid);
  } else {
    const PenaltyArgs a = penalty_args(&r->penalty);
    if (vec == 0) penalty_segments<POL_PLAIN, -1>(a, chunk, s, tid);
    else if (dt == GPUOS_F32) penalty_segments<POL_PLAIN, GPUOS_F32>(a, chunk, s, tid);
    else if (dt == GPUOS_F16) penalty_segments<POL_PLAIN, GPUOS_F16>(a, chunk, s, tid);
    else penalty_segments<POL_PLAIN, GPUOS_BF16>(a, chunk, s, tid);
  }
}
// LDS of a block, in floats: the partial sums of gamma by groups of lanes; a segment's counts
template <int IMPL> constexpr uint32_t model_lds() {
  return IMPL == GPUOS_IMPL_NORM_ROPE_GRAD ? 2048u : (IMPL == GPUOS_IMPL_LOGIT_PENALTY ? ModelPack::kSegment : 1u);
}

template <int IMPL> __global__ void __launch_bounds__(kThreads) gpuos_model_kernel(ModelLaunch l) {
  __shared__ alignas(16) float s[model_lds<IMPL>()];
  typedef const __attribute__((address_space(4))) ModelLaunch* launch_t;
  const launch_t p = (launch_t)__builtin_amdgcn_kernarg_segment_ptr();
  uint32_t t = 0;
#pragma unroll
  for (uint32_t k = 1; k < kModelLaunch; ++k) t += blockIdx.x >= p->first[k] ? 1u : 0u;
  run_model<IMPL>(&p->rec[t], blockIdx.x - p->first[t], s, threadIdx.x);
}

int launch_model(const ModelLaunch& l, uint32_t impl, uint32_t blocks, void* stream) {
  const dim3 grid(blocks), block(kThreads);
  const hipStream_t st = (hipStream_t)stream;
  switch (impl) {
    case GPUOS_IMPL_NORM_ROPE: hipLaunchKernelGGL(gpuos_model_kernel<GPUOS_IMPL_NORM_ROPE>, grid, block, 0, st, l); break;
    case GPUOS_IMPL_NORM_ROPE_GRAD: hipLaunchKernelGGL(gpuos_model_kernel<GPUOS_IMPL_NORM_ROPE_GRAD>, grid, block, 0, st, l); break;
    case GPUOS_IMPL_GAMMA_SUM: hipLaunchKernelGGL(gpuos_model_kernel<GPUOS_IMPL_GAMMA_SUM>, grid, block, 0, st, l); break;
    case GPUOS_IMPL_CACHE_STORE: hipLaunchKernelGGL(gpuos_model_kernel<GPUOS_IMPL_CACHE_STORE>, grid, block, 0, st, l); break;
    case GPUOS_IMPL_CACHE_LOAD: hipLaunchKernelGGL(gpuos_model_kernel<GPUOS_IMPL_CACHE_LOAD>, grid, block, 0, st, l); break;
    case GPUOS_IMPL_LOGIT_PENALTY: hipLaunchKernelGGL(gpuos_model_kernel<GPUOS_IMPL_LOGIT_PENALTY>, grid, block, 0, st, l); break;
    default: return (int)hipErrorInvalidValue;
  }
  return (int)hipGetLastError();
}

}  // namespace gpuos
