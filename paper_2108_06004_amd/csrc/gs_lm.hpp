// gs_lm.hpp -- shared by the language-model operators: element types, argument structs and
// launchers (k_recurrence.hip, k_dropout.hip, k_cross_entropy.hip; C ABI in gs_lm.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/gs.h"

namespace gs {

constexpr int64_t kMaxExtent = 2147483647;  // rows and logits
constexpr int64_t kMaxSteps = 1 << 30;       // sequences and their steps

inline int elem_size(int dtype) { return dtype == GS_F32 ? 4 : 2; }

// Activation types: conversion to and from fp32, to nearest even on the way down (the
// hardware's conversions; NaN stays NaN). VEC neighbouring elements travel as one register set.
template <int DT>
struct Elem;
template <>
struct Elem<GS_F32> {
  using type = float;
};
template <>
struct Elem<GS_BF16> {
  using type = __bf16;
};
template <>
struct Elem<GS_F16> {
  using type = _Float16;
};

template <int DT, int VEC>
struct Pack {
  typedef typename Elem<DT>::type raw __attribute__((ext_vector_type(VEC)));
  typedef float wide __attribute__((ext_vector_type(VEC)));
  __device__ static __forceinline__ wide up(raw v) { return __builtin_convertvector(v, wide); }
  __device__ static __forceinline__ raw down(wide v) { return __builtin_convertvector(v, raw); }
};

constexpr float kLog2e = 1.44269504088896340736f;

// sigmoid(z) and 1 - sigmoid(z) = sigmoid(-z), each to its own digits (1 - s would lose those of a gate near one): with
// e = exp(-z) they are 1 / (1 + e) and e / (1 + e). Each is off by at most (1.25 |z| + 8) 2^-24 of itself, the first part
// from z log2(e), which is rounded once: what half an ulp of an fp32 z changes. Where e is so large that the
// first is 0 or no normal number the second is 1 (e may be infinite there); a NaN stays one.
__device__ __forceinline__ void sigmoid_both(float z, float& s, float& rest) {
  const float e = __builtin_amdgcn_exp2f(-z * kLog2e);
  s = __builtin_amdgcn_rcpf(1.0f + e);
  rest = s < 0x1p-125f ? 1.0f : e * s;
}

__device__ __forceinline__ float sigmoid_of(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-z * kLog2e));
}

// A [B][T][C] array with its strides in bytes.
struct Rows {
  char* p;
  int64_t batch, time;
};

struct RecurrenceArgs {
  int64_t B, T, C;
  Rows x, f, o, y, gy, dx, df, dout;
  const int32_t* lengths;
  const float* h0;
  const float* gh;
  float* h_last;
  float* dh0;
  float* states;
  float* work;
};

int64_t recurrence_work(int64_t B, int64_t T, int64_t C, int dtype);
hipError_t launch_recurrence_forward(hipStream_t s, int dtype, const RecurrenceArgs& a);
hipError_t launch_recurrence_backward(hipStream_t s, int dtype, const RecurrenceArgs& a);

struct DropoutArgs {
  int64_t rows, cols;
  const char *x, *res;
  char* y;
  int64_t xs, rs, ys;  // row strides in elements
  uint32_t below;      // draws below this are dropped, of 65,536
  float factor;
  uint64_t seed, site;
  const int64_t* step;
};

hipError_t launch_dropout(hipStream_t s, int dtype, const DropoutArgs& a);

int64_t cross_entropy_work(int64_t N, int64_t V, int dtype);
hipError_t launch_cross_entropy(hipStream_t s, const gs_xent& x);

}  // namespace gs
