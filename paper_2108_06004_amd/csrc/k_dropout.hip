// k_dropout.hip -- dropout whose mask is drawn from a counter and never stored (include/gs.h).
//
// Plain form: one element a thread.
#include "gs_lm.hpp"

namespace gs {
namespace {

constexpr int kBlock = 256;
constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;

// SplitMix64's output function (Steele, Lea & Flood, "Fast splittable pseudorandom number
// generators", OOPSLA 2014).
__device__ __forceinline__ uint64_t mix(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

template <int DT>
__global__ void __launch_bounds__(kBlock) k_dropout(DropoutArgs a) {
  using E = typename Elem<DT>::type;
  const int64_t n = a.rows * a.cols;
  const uint64_t key = mix(mix(mix(a.seed) ^ (a.step ? (uint64_t)*a.step : 0ull)) ^ a.site);
  for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n; i += (int64_t)gridDim.x * kBlock) {
    const int64_t row = i / a.cols, col = i % a.cols;
    const uint64_t w = mix(key + (uint64_t)(i / 4 + 1) * kGolden);
    const bool kept = ((uint32_t)(w >> (16 * (i & 3))) & 0xffffu) >= a.below;
    float v = kept ? (float)reinterpret_cast<const E*>(a.x)[row * a.xs + col] * a.factor : 0.0f;
    if (a.res) v = (float)reinterpret_cast<const E*>(a.res)[row * a.rs + col] + v;
    reinterpret_cast<E*>(a.y)[row * a.ys + col] = (E)v;
  }
}

}  // namespace

hipError_t launch_dropout(hipStream_t s, int dtype, const DropoutArgs& a) {
  const int64_t want = (a.rows * a.cols + kBlock - 1) / kBlock;
  const dim3 grid((unsigned)(want < 65536 ? want : 65536));
  if (dtype == GS_F32) k_dropout<GS_F32><<<grid, kBlock, 0, s>>>(a);
  if (dtype == GS_BF16) k_dropout<GS_BF16><<<grid, kBlock, 0, s>>>(a);
  if (dtype == GS_F16) k_dropout<GS_F16><<<grid, kBlock, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace gs
