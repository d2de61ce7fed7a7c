// k_dropout.hip -- dropout whose mask is drawn from a counter and never stored (include/gs.h).
//
// A word of the generator covers four neighbouring elements of the flat tensor, so a thread takes
// 16 bytes of a row at a time (eight elements and two words, or four and one) and U of them with
// their loads in flight together. A word is two 64-bit products, about 45 VALU slots, which at
// 16 bits a draw is 11 an element: less than the loads and stores cost. Every array is read or written once, past the
// caches (65,536 x 2,048 bf16 with residual: 154 us through them, 141 past, 5.7 TB/s; without 97 us).
#include "gs_lm.hpp"

namespace gs {
namespace {

constexpr int kBlock = 256;
constexpr int kU = 4;
constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;

// SplitMix64's output function (Steele, Lea & Flood, "Fast splittable pseudorandom number
// generators", OOPSLA 2014).
__device__ __forceinline__ uint64_t mix(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

// A thread's place: blockDim.x threads along a row, blockDim.y rows. WIDE: every row of every array
// is 16-byte aligned; otherwise the same elements go one by one. SHIFT: rows may begin inside a word.
template <int DT, bool RES, bool WIDE, bool SHIFT>
__global__ void __launch_bounds__(kBlock) k_dropout(DropoutArgs a) {
  using E = typename Elem<DT>::type;
  constexpr int N = 16 / (int)sizeof(E);
  using P = Pack<DT, N>;
  const int64_t per_row = (a.cols + N - 1) / N, whole = a.cols / N;
  const int64_t stride = (int64_t)gridDim.x * blockDim.x;
  const uint64_t key = mix(mix(mix(a.seed) ^ (a.step ? (uint64_t)*a.step : 0ull)) ^ a.site);
  for (int64_t r = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; r < a.rows; r += (int64_t)gridDim.y * blockDim.y) {
    const E* x = reinterpret_cast<const E*>(a.x) + r * a.xs;
    const E* res = RES ? reinterpret_cast<const E*>(a.res) + r * a.rs : nullptr;
    E* y = reinterpret_cast<E*>(a.y) + r * a.ys;
    for (int64_t j0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; j0 < per_row; j0 += stride * kU) {
      typename P::raw xv[kU], rv[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t j = j0 + u * stride;
        if (WIDE && j < whole) {
          xv[u] = __builtin_nontemporal_load(reinterpret_cast<const typename P::raw*>(x) + j);
          if (RES) rv[u] = __builtin_nontemporal_load(reinterpret_cast<const typename P::raw*>(res) + j);
        } else if (j < per_row) {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const bool in = j * N + e < a.cols;
            xv[u][e] = in ? x[j * N + e] : (E)0.0f;
            if (RES) rv[u][e] = in ? res[j * N + e] : (E)0.0f;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int64_t j = j0 + u * stride;
        if (j >= per_row) break;
        const int64_t i = r * a.cols + j * N;  // flat index of the first element
        const int first = SHIFT ? (int)(i & 3) : 0;
        uint64_t z = key + (uint64_t)(i / 4 + 1) * kGolden;
        uint64_t w[N / 4 + (SHIFT ? 1 : 0)];
#pragma unroll
        for (int m = 0; m < (int)(sizeof w / sizeof w[0]); ++m, z += kGolden) w[m] = mix(z);
        if (SHIFT && first) {
#pragma unroll
          for (int m = 0; m < N / 4; ++m) w[m] = (w[m] >> (16 * first)) | (w[m + 1] << (64 - 16 * first));
        }
        typename P::wide v = P::up(xv[u]);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const bool kept = ((uint32_t)(w[e / 4] >> (16 * (e & 3))) & 0xffffu) >= a.below;
          v[e] = kept ? v[e] * a.factor : 0.0f;
        }
        if (RES) v = P::up(rv[u]) + v;
        const typename P::raw out = P::down(v);
        if (WIDE && j < whole) {
          __builtin_nontemporal_store(out, reinterpret_cast<typename P::raw*>(y) + j);
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (j * N + e < a.cols) y[j * N + e] = out[e];
        }
      }
    }
  }
}

template <int DT>
void launch(hipStream_t s, const DropoutArgs& a) {
  constexpr int N = 16 / (int)sizeof(typename Elem<DT>::type);
  const int64_t per_row = (a.cols + N - 1) / N;
  auto wide_row = [&](const void* p, int64_t stride) {
    return ((uintptr_t)p & 15) == 0 && (a.rows == 1 || stride % N == 0);
  };
  const bool wide = wide_row(a.x, a.xs) && wide_row(a.y, a.ys) && (!a.res || wide_row(a.res, a.rs));
  const bool shift = a.rows > 1 && a.cols % 4 != 0;
  dim3 block(kBlock, 1);
  while (block.x > 1 && (int64_t)(block.x / 2) * kU >= per_row) {  // short rows share a workgroup
    block.x /= 2;
    block.y *= 2;
  }
  const int64_t gx = (per_row + (int64_t)block.x * kU - 1) / ((int64_t)block.x * kU);
  const int64_t gy = (a.rows + block.y - 1) / block.y;
  const dim3 grid((unsigned)(gx < (1 << 22) ? gx : 1 << 22), (unsigned)(gy < 32768 ? gy : 32768));
#define GS_DROPOUT(RES, WIDE, SHIFT) k_dropout<DT, RES, WIDE, SHIFT><<<grid, block, 0, s>>>(a)
  if (a.res) {
    if (shift)
      wide ? GS_DROPOUT(true, true, true) : GS_DROPOUT(true, false, true);
    else
      wide ? GS_DROPOUT(true, true, false) : GS_DROPOUT(true, false, false);
  } else {
    if (shift)
      wide ? GS_DROPOUT(false, true, true) : GS_DROPOUT(false, false, true);
    else
      wide ? GS_DROPOUT(false, true, false) : GS_DROPOUT(false, false, false);
  }
#undef GS_DROPOUT
}

}  // namespace

hipError_t launch_dropout(hipStream_t s, int dtype, const DropoutArgs& a) {
  if (dtype == GS_F32) launch<GS_F32>(s, a);
  if (dtype == GS_BF16) launch<GS_BF16>(s, a);
  if (dtype == GS_F16) launch<GS_F16>(s, a);
  return hipGetLastError();
}

}  // namespace gs
