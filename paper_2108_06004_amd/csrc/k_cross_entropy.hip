// k_cross_entropy.hip -- softmax cross-entropy of rows of logits and its gradient (include/gs.h).
//
// Plain form: one workgroup a row, which it reads three times (maximum, sum, gradient); a kernel
// before it counts the rows that count, one after it sums their losses.
#include "gs_lm.hpp"

namespace gs {
namespace {

constexpr int kBlock = 256;
constexpr int kTail = 1024;

template <int THREADS, typename T, typename F>
__device__ __forceinline__ T block_reduce(T v, T* lds, F f) {
  lds[threadIdx.x] = v;
  __syncthreads();
  for (int n = THREADS / 2; n > 0; n >>= 1) {
    if ((int)threadIdx.x < n) lds[threadIdx.x] = f(lds[threadIdx.x], lds[threadIdx.x + n]);
    __syncthreads();
  }
  const T r = lds[0];
  __syncthreads();
  return r;
}

__global__ void __launch_bounds__(kTail) k_xent_count(gs_xent x) {
  __shared__ int64_t lds[kTail];
  int64_t n = 0;
  for (int64_t i = threadIdx.x; i < x.N; i += kTail) n += x.targets[i] != x.ignore_index;
  n = block_reduce<kTail>(n, lds, [](int64_t p, int64_t q) { return p + q; });
  if (threadIdx.x == 0) *static_cast<float*>(x.work) = 1.0f / (float)(n > 0 ? n : 1);
}

__global__ void __launch_bounds__(kTail) k_xent_mean(gs_xent x) {
  __shared__ double lds[kTail];
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < x.N; i += kTail) sum += x.losses[i];
  sum = block_reduce<kTail>(sum, lds, [](double p, double q) { return p + q; });
  if (threadIdx.x == 0) *x.mean_loss = (float)(sum * *static_cast<const float*>(x.work));
}

template <int DT>
__global__ void __launch_bounds__(kBlock) k_xent(gs_xent x) {
  using E = typename Elem<DT>::type;
  __shared__ float lds[kBlock];
  const int64_t n = blockIdx.x, t = x.targets[n];
  const E* z = static_cast<const E*>(x.logits) + n * x.logits_stride;
  E* grad = x.grad ? static_cast<E*>(x.grad) + n * x.grad_stride : nullptr;
  if (t == x.ignore_index) {
    if (threadIdx.x == 0 && x.losses) x.losses[n] = 0.0f;
    if (grad)
      for (int64_t v = threadIdx.x; v < x.V; v += kBlock) grad[v] = (E)0.0f;
    return;
  }
  const bool known = t >= 0 && t < x.V;
  const float at = known ? (float)z[t] : __builtin_nanf("");
  float top = -__builtin_inff();
  for (int64_t v = threadIdx.x; v < x.V; v += kBlock) top = fmaxf(top, (float)z[v]);
  top = block_reduce<kBlock>(top, lds, [](float p, float q) { return fmaxf(p, q); });
  float sum = 0.0f;
  for (int64_t v = threadIdx.x; v < x.V; v += kBlock) sum += __builtin_amdgcn_exp2f(((float)z[v] - top) * kLog2e);
  sum = block_reduce<kBlock>(sum, lds, [](float p, float q) { return p + q; });
  if (threadIdx.x == 0 && x.losses) x.losses[n] = logf(sum) - (at - top);
  if (!grad) return;
  float m = x.factor;
  if (x.scale) m *= x.scale[n * x.scale_stride];
  if (x.mean) m *= *static_cast<const float*>(x.work);
  const float share = known ? 1.0f / sum : __builtin_nanf("");
  for (int64_t v = threadIdx.x; v < x.V; v += kBlock) {
    const float p = __builtin_amdgcn_exp2f(((float)z[v] - top) * kLog2e) * share;
    grad[v] = (E)(m * (v == t ? p - 1.0f : p));
  }
}

}  // namespace

int64_t cross_entropy_work(int64_t, int64_t, int) { return 8; }

hipError_t launch_cross_entropy(hipStream_t s, const gs_xent& x) {
  if (x.N == 0 && !x.mean_loss) return hipSuccess;
  if (x.mean_loss || (x.mean && x.grad)) k_xent_count<<<1, kTail, 0, s>>>(x);
  if (x.N > 0) {
    const dim3 grid((unsigned)x.N);
    if (x.dtype == GS_F32) k_xent<GS_F32><<<grid, kBlock, 0, s>>>(x);
    if (x.dtype == GS_BF16) k_xent<GS_BF16><<<grid, kBlock, 0, s>>>(x);
    if (x.dtype == GS_F16) k_xent<GS_F16><<<grid, kBlock, 0, s>>>(x);
  }
  if (x.mean_loss) k_xent_mean<<<1, kTail, 0, s>>>(x);
  return hipGetLastError();
}

}  // namespace gs
