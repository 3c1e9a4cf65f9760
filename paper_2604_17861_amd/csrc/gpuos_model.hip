// gpuos_model.hip -- the model operators as ordinary kernels on a caller's stream (gpuos_launch_model): the
// executors of gpuos_model_device.h, a block a chunk.  Records and block numbers are kernel arguments, so a launch
// allocates and copies nothing and may be captured.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <utility>

#include "gpuos_model_device.h"

namespace gpuos {

// LDS of a block, in floats: the partial sums of gamma by groups of lanes; a segment's counts
constexpr uint32_t model_lds(uint32_t v) { return v < MV_GRAD ? 1u : (v < MV_SUM ? 2048u : (v == MV_SUM ? 4u : (v < MV_PENALTY ? 1u : ModelPack::kSegment))); }
constexpr uint32_t model_threads(uint32_t v) { return v < MV_PENALTY ? kThreads : kPenaltyThreads; }

// Wavefronts of a SIMD that the compiler has to leave room for.  A worker of three workgroups a compute unit, the default, leaves a quarter of every
// register file, 128 of 512 registers: a block has to fit there, or it waits until the worker leaves, which it may never do.  A block of 256
// threads is one wavefront a SIMD, of 512 two; so four and eight.  (Unbounded, the gradient element by element took 133.)
// The penalties gain from it besides: they need more scalar registers than eight may have, and 64 rows of 100,352 in segments of eight
// wavefronts are 1,600 workgroups, of which the card takes 768 at once so, and 1,024 with some of them in lanes: 10.6 and 10.2 us.
// Rotations, 16 times a card's worth, are slower with eight: 36.4 and 38.4.
constexpr uint32_t model_waves(uint32_t v) { return 4u * model_threads(v) / kThreads; }

template <uint32_t V> __global__ void __launch_bounds__(model_threads(V), model_waves(V)) gpuos_model_kernel(ModelLaunch) {
  __shared__ alignas(16) float s[model_lds(V)];
  typedef const __attribute__((address_space(4))) ModelLaunch* launch_t;
  const auto r = &((launch_t)__builtin_amdgcn_kernarg_segment_ptr())->rec[blockIdx.y];
  if (blockIdx.x < r->h.nchunks) run_model<POL_PLAIN, V, model_threads(V)>(r, blockIdx.x, s, threadIdx.x);
}

typedef void (*model_kernel_t)(ModelLaunch);
template <uint32_t... V> struct Kernels { static constexpr model_kernel_t at[] = {gpuos_model_kernel<V>...}; };
template <uint32_t... V> Kernels<V...> kernels_of(std::integer_sequence<uint32_t, V...>);
typedef decltype(kernels_of(std::make_integer_sequence<uint32_t, MV_COUNT>())) AllKernels;

int launch_model(const ModelLaunch& l, uint32_t variant, uint32_t chunks, uint32_t tasks, void* stream) {
  if (variant >= MV_COUNT) return (int)hipErrorInvalidValue;
  void* args[] = {(void*)&l};
  return (int)hipLaunchKernel((const void*)AllKernels::at[variant], dim3(chunks, tasks), dim3(model_threads(variant)), args, 0, (hipStream_t)stream);      // (its own status, not the thread's last one)
}

}  // namespace gpuos
