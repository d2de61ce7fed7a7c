// k_recurrence.hip -- the gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) x_t, a = sigmoid(f),
// y_t = sigmoid(o_t) h_t, and its backward pass (include/gs.h).
//
// Plain form: one thread walks one channel of one sequence along time. A step is two
// dependent operations, so the time is T steps of memory latency.
#include "gs_lm.hpp"

namespace gs {
namespace {

constexpr int kBlock = 256;
constexpr int kStep = GS_RECURRENCE_BLOCK;

__device__ __forceinline__ int64_t length_of(const RecurrenceArgs& a, int64_t b) {
  if (!a.lengths) return a.T;
  const int64_t n = a.lengths[b];
  return n < 0 ? 0 : n > a.T ? a.T : n;
}

template <int DT>
__device__ __forceinline__ float get(const Rows& r, int64_t b, int64_t t, int64_t c) {
  using E = typename Elem<DT>::type;
  return (float)*reinterpret_cast<const E*>(r.p + b * r.batch + t * r.time + c * (int64_t)sizeof(E));
}

template <int DT>
__device__ __forceinline__ void put(const Rows& r, int64_t b, int64_t t, int64_t c, float v) {
  using E = typename Elem<DT>::type;
  *reinterpret_cast<E*>(r.p + b * r.batch + t * r.time + c * (int64_t)sizeof(E)) = (E)v;
}

template <int DT>
__global__ void __launch_bounds__(kBlock) k_recurrence_fwd(RecurrenceArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (i >= a.B * a.C) return;
  const int64_t b = i / a.C, c = i % a.C, n = length_of(a, b), blocks = GS_RECURRENCE_BLOCKS(a.T);
  float h = a.h0 ? a.h0[i] : 0.0f;
  for (int64_t t = 0; t < n; ++t) {
    if (a.states && t % kStep == 0) a.states[(b * blocks + t / kStep) * a.C + c] = h;
    float k, rest;
    sigmoid_both(get<DT>(a.f, b, t, c), k, rest);
    h = fmaf(k, h, rest * get<DT>(a.x, b, t, c));
    float g = 1.0f, unused;
    if (a.o.p) sigmoid_both(get<DT>(a.o, b, t, c), g, unused);
    put<DT>(a.y, b, t, c, g * h);
  }
  for (int64_t t = n; t < a.T; ++t) put<DT>(a.y, b, t, c, 0.0f);
  a.h_last[i] = h;
}

template <int DT>
__global__ void __launch_bounds__(kBlock) k_recurrence_bwd(RecurrenceArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (i >= a.B * a.C) return;
  const int64_t b = i / a.C, c = i % a.C, n = length_of(a, b), blocks = GS_RECURRENCE_BLOCKS(a.T);
  float carry = a.gh ? a.gh[i] : 0.0f;
  for (int64_t t = n; t < a.T; ++t) {
    put<DT>(a.dx, b, t, c, 0.0f);
    put<DT>(a.df, b, t, c, 0.0f);
    if (a.o.p) put<DT>(a.dout, b, t, c, 0.0f);
  }
  for (int64_t blk = GS_RECURRENCE_BLOCKS(n) - 1; blk >= 0; --blk) {
    float before[kStep];
    const int64_t t0 = blk * kStep;
    const int m = (int)(n - t0 < kStep ? n - t0 : kStep);
    float h = a.states[(b * blocks + blk) * a.C + c];
    for (int j = 0; j < m; ++j) {
      before[j] = h;
      float k, rest;
      sigmoid_both(get<DT>(a.f, b, t0 + j, c), k, rest);
      h = fmaf(k, h, rest * get<DT>(a.x, b, t0 + j, c));
    }
    for (int j = m - 1; j >= 0; --j) {
      const int64_t t = t0 + j;
      float k, rest, g = 1.0f, closed = 0.0f;
      sigmoid_both(get<DT>(a.f, b, t, c), k, rest);
      const float x = get<DT>(a.x, b, t, c), gy = get<DT>(a.gy, b, t, c);
      if (a.o.p) {
        sigmoid_both(get<DT>(a.o, b, t, c), g, closed);
        put<DT>(a.dout, b, t, c, gy * fmaf(k, before[j], rest * x) * (g * closed));
      }
      const float s = fmaf(gy, g, carry);
      put<DT>(a.dx, b, t, c, rest * s);
      put<DT>(a.df, b, t, c, s * (before[j] - x) * (k * rest));
      carry = k * s;
    }
  }
  if (a.dh0) a.dh0[i] = carry;
}

}  // namespace

int64_t recurrence_work(int64_t, int64_t, int64_t, int) { return 0; }

hipError_t launch_recurrence_forward(hipStream_t s, int dtype, const RecurrenceArgs& a) {
  const dim3 grid((unsigned)((a.B * a.C + kBlock - 1) / kBlock));
  if (dtype == GS_F32) k_recurrence_fwd<GS_F32><<<grid, kBlock, 0, s>>>(a);
  if (dtype == GS_BF16) k_recurrence_fwd<GS_BF16><<<grid, kBlock, 0, s>>>(a);
  if (dtype == GS_F16) k_recurrence_fwd<GS_F16><<<grid, kBlock, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_recurrence_backward(hipStream_t s, int dtype, const RecurrenceArgs& a) {
  const dim3 grid((unsigned)((a.B * a.C + kBlock - 1) / kBlock));
  if (dtype == GS_F32) k_recurrence_bwd<GS_F32><<<grid, kBlock, 0, s>>>(a);
  if (dtype == GS_BF16) k_recurrence_bwd<GS_BF16><<<grid, kBlock, 0, s>>>(a);
  if (dtype == GS_F16) k_recurrence_bwd<GS_F16><<<grid, kBlock, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace gs
