// k_cross_entropy.hip -- softmax cross-entropy of rows of logits and its gradient (include/gs.h).
//
// One pass: a workgroup holds its whole row in registers, CH times 16 bytes a thread, so the logits are
// read once: maximum, sum of exponentials and gradient come from the registers (the exponential twice,
// which costs less than keeping fp32 values). Rows too long for that, and few long rows, are split over
// several workgroups: one kernel reduces each part to (maximum, sum), a second joins them and writes the
// gradient, reading the logits again.
//
// What bounds it: memory (4,096 x 22,000 bf16 with gradient: 65 us, 5.4 TB/s; 8,191 x 131,071: 852 us, 5.0 TB/s, one
// workgroup a CU), and for few rows the launches: the row's kernel 4.7 us and the mean's 1.8 at 35 x 22,000 fp32.
//
// Rows need not be aligned: the elements before the first 16-byte boundary of a row and after its last one
// (up to seven each) go one to a thread.
#include "gs_lm.hpp"

namespace gs {
namespace {

constexpr int kTail = 1024;  // threads that count rows and sum losses
// So many rows every wave counts by itself; more are counted by a kernel before (4,096 rows of 22,000 bf16 logits,
// whole call: 128 us counted in the row's kernel, whose own loads the targets' displace, 72 before it; 300 rows: 14.1 and 16.4).
constexpr int kInlineCount = 256;
constexpr int kPartThreads = 256;
constexpr int kPartVecs = 4;          // 16-byte pieces a thread takes of a part, at least
constexpr int kMaxParts = kPartThreads;
constexpr int kRowThreads = 1024;
constexpr int kRowPieces = 16;  // longest row in registers: 16 pieces of 1,024 threads, 256 KB
constexpr int kSplitWant = 2048;  // workgroups that rows are split into
constexpr int kFewRows = 64, kLongRow = 8192;  // rows this few of pieces this many are split although registers hold them

__device__ __forceinline__ float inf() { return __builtin_inff(); }

// e^d for d <= 0 (and NaN).
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// (maximum, sum of e^(z - maximum)) of what has been seen; a maximum of -inf stands for 0 in the sum.
struct Seen {
  float top, sum;
};

__device__ __forceinline__ float base_of(float top) { return top == -inf() ? 0.0f : top; }

// A side that has seen nothing (or only -inf, or NaN) keeps its sum, 0 or NaN, as it is.
__device__ __forceinline__ float moved(Seen p, float top) { return p.top == -inf() ? p.sum : p.sum * exp_of(p.top - top); }

__device__ __forceinline__ Seen join(Seen p, Seen q) {
  const float top = fmaxf(p.top, q.top);
  return Seen{top, moved(p, top) + moved(q, top)};
}

// The sum of the losses and the rows that count.
struct Tally {
  double sum;
  int n;
};

// A value of the lane whose number differs in bit d.
__device__ __forceinline__ float lane_xor(float v, int d) { return __shfl_xor(v, d); }
__device__ __forceinline__ int lane_xor(int v, int d) { return __shfl_xor(v, d); }
__device__ __forceinline__ Seen lane_xor(Seen s, int d) { return Seen{__shfl_xor(s.top, d), __shfl_xor(s.sum, d)}; }
__device__ __forceinline__ Tally lane_xor(Tally t, int d) { return Tally{__shfl_xor(t.sum, d), __shfl_xor(t.n, d)}; }

template <int THREADS, typename T, typename F>
__device__ __forceinline__ T block_reduce(T v, T* lds, F f) {
#pragma unroll
  for (int n = 32; n > 0; n >>= 1) v = f(v, lane_xor(v, n));
  if (THREADS == 64) return v;
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) v = f(v, lds[w]);
  return v;
}

// The rows that count among those of one lane, eight loads at a time. Counts are whole numbers up to 2^31 - 1 and are rounded
// to fp32 once, as a divisor.
__device__ __forceinline__ int count_of(const gs_xent& x, int lane, int lanes) {
  int n = 0;
  for (int64_t i0 = lane; i0 < x.N; i0 += 8 * lanes) {
    int64_t t[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) t[u] = i0 + u * lanes < x.N ? x.targets[i0 + u * lanes] : x.ignore_index;
#pragma unroll
    for (int u = 0; u < 8; ++u) n += t[u] != x.ignore_index;
  }
  return n;
}

__device__ __forceinline__ float inverse_of(int n) { return 1.0f / (float)(n > 1 ? n : 1); }

template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_xent_count(gs_xent x) {
  __shared__ int lds[THREADS / 64];
  const int n = block_reduce<THREADS>(count_of(x, threadIdx.x, THREADS), lds, [](int p, int q) { return p + q; });
  if (threadIdx.x == 0) *static_cast<float*>(x.work) = inverse_of(n);
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_xent_mean(gs_xent x) {
  __shared__ Tally lds[THREADS / 64];
  Tally t{0.0, 0};
  for (int64_t i0 = threadIdx.x; i0 < x.N; i0 += 8 * THREADS) {
    float loss[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) loss[u] = i0 + u * THREADS < x.N ? x.losses[i0 + u * THREADS] : 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) t.sum += loss[u];
  }
  t.n = count_of(x, threadIdx.x, THREADS);
  t = block_reduce<THREADS>(t, lds, [](Tally p, Tally q) { return Tally{p.sum + q.sum, p.n + q.n}; });
  if (threadIdx.x == 0) *x.mean_loss = (float)(t.sum / (t.n > 1 ? t.n : 1));
}

// The factor of a row's gradient. Rows few enough are counted here, by each wave on its own.
__device__ __forceinline__ float factor_of(const gs_xent& x, int64_t n) {
  float m = x.factor;
  if (x.scale) m *= x.scale[n * x.scale_stride];
  if (x.mean) {
    if (x.N <= kInlineCount) {
      int c = count_of(x, threadIdx.x & 63, 64);
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) c += __shfl_xor(c, d);
      m *= inverse_of(c);
    } else {
      m *= *static_cast<const float*>(x.work);
    }
  }
  return m;
}

// Workgroups are counted over two dimensions of the grid: one holds fewer than 2^32 threads.
constexpr int64_t kGridX = 1 << 21;
__device__ __forceinline__ int64_t group_of() { return (int64_t)blockIdx.y * kGridX + blockIdx.x; }
dim3 grid_of(int64_t groups) {
  return dim3((unsigned)(groups < kGridX ? groups : kGridX), (unsigned)((groups + kGridX - 1) / kGridX));
}

template <int DT>
struct Row {
  using E = typename Elem<DT>::type;
  static constexpr int N = 16 / (int)sizeof(E);
  using P = Pack<DT, N>;
  const E* z;
  E* grad;
  int head, vecs, tail;  // elements before the first boundary, 16-byte pieces, elements after the last
  __device__ __forceinline__ Row(const gs_xent& x, int64_t n) {
    z = static_cast<const E*>(x.logits) + n * x.logits_stride;
    grad = x.grad ? static_cast<E*>(x.grad) + n * x.grad_stride : nullptr;
    const int V = (int)x.V, off = (int)((uintptr_t)z & 15) / (int)sizeof(E);
    head = off ? N - off : 0;
    head = head < V ? head : V;
    vecs = (V - head) / N;
    tail = V - head - vecs * N;
  }
  // The element that thread i < head + tail holds beside its pieces; below zero: none.
  __device__ __forceinline__ int edge(int i) const {
    return i < head ? i : i < head + tail ? head + vecs * N + (i - head) : -1;
  }
  // Pieces read for the last time and gradients go past the caches (PAST; 4,096 x 22,000 bf16 with gradient: 78 us
  // through them, 72 past; 2,000 x 32,000 fp32 106 and 98), but for the longest rows where they do not fill their
  // 128-byte lines (8,191 x 131,071 bf16: 873 us through the caches, 902 past).
  template <bool PAST>
  __device__ __forceinline__ typename P::raw get(int j) const {
    const auto* p = reinterpret_cast<const typename P::raw*>(z + head + (int64_t)j * N);
    return PAST ? __builtin_nontemporal_load(p) : *p;
  }
  // Gradients need not have the logits' alignment.
  template <bool SAME, bool PAST>
  __device__ __forceinline__ void put(int j, typename P::raw v) const {
    E* g = grad + head + (int64_t)j * N;
    if (SAME && PAST) {
      __builtin_nontemporal_store(v, reinterpret_cast<typename P::raw*>(g));
    } else if (SAME) {
      *reinterpret_cast<typename P::raw*>(g) = v;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] = v[e];
    }
  }
  // A piece of the gradient m (softmax - [v = t]); `at` is t - head.
  template <bool SAME, bool PAST>
  __device__ __forceinline__ void put_grad(int j, typename P::raw r, float top, float share, float m, int at) const {
    typename P::wide v = P::up(r);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = exp_of(v[e] - top) * share;
    if (at >= 0 && at / N == j) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e == at % N) v[e] -= 1.0f;
    }
    put<SAME, PAST>(j, P::down(v * m));
  }
};

// Keeps the compiler from holding a piece's fp32 form from one pass over the registers to the next (twice
// the registers): converting again is cheap.
template <typename T>
__device__ __forceinline__ void as_stored(T& v) {
  static_assert(sizeof(T) == 16, "a 16-byte piece");
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  u4 w = __builtin_bit_cast(u4, v);
  asm volatile("" : "+v"(w));
  v = __builtin_bit_cast(T, w);
}

template <int DT, int THREADS, int CH, bool GRAD, bool SAME, bool PAST = true>
__global__ void __launch_bounds__(THREADS) k_xent_row(gs_xent x) {
  using R = Row<DT>;
  using P = typename R::P;
  using E = typename R::E;
  __shared__ float lds_top[THREADS / 64], lds_sum[THREADS / 64];
  const int64_t n = group_of();
  if (n >= x.N) return;
  const int64_t t = x.targets[n];
  const R row(x, n);
  const int tid = threadIdx.x, edge = row.edge(tid);
  if (t == x.ignore_index) {
    if (tid == 0 && x.losses) x.losses[n] = 0.0f;
    if (GRAD) {
      for (int j = tid; j < row.vecs; j += THREADS) row.template put<SAME, PAST>(j, P::down((typename P::wide)0.0f));
      if (edge >= 0) row.grad[edge] = (E)0.0f;
    }
    return;
  }
  struct Piece {  // in a struct: the compiler makes one long vector of a plain array (8 fp32 pieces: 252 registers for 64)
    typename P::raw v;
  };
  Piece r[CH];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int j = tid + i * THREADS;
    if (j < row.vecs)
      r[i].v = row.template get<PAST>(j);
    else
      r[i].v = P::down((typename P::wide)(-inf()));
  }
  const float side = edge >= 0 ? (float)row.z[edge] : -inf();
  const bool known = t >= 0 && t < x.V;
  const float at = known ? (float)row.z[t] : __builtin_nanf("");
  const float m = GRAD ? factor_of(x, n) : 0.0f;
  float top = side;
#pragma unroll
  for (int i = 0; i < CH; ++i)
    if (i * THREADS < row.vecs) {
      const typename P::wide v = P::up(r[i].v);
#pragma unroll
      for (int e = 0; e < R::N; ++e) top = fmaxf(top, v[e]);
    }
  top = block_reduce<THREADS>(top, lds_top, [](float p, float q) { return fmaxf(p, q); });
  float sum = edge >= 0 ? exp_of(side - top) : 0.0f;
#pragma unroll
  for (int i = 0; i < CH; ++i)
    if (i * THREADS < row.vecs) {
      as_stored(r[i].v);
      const typename P::wide v = P::up(r[i].v);
#pragma unroll
      for (int e = 0; e < R::N; ++e) sum += exp_of(v[e] - top);
    }
  sum = block_reduce<THREADS>(sum, lds_sum, [](float p, float q) { return p + q; });
  if (tid == 0 && x.losses) x.losses[n] = logf(sum) - (at - top);
  if (!GRAD) return;
  const float share = known ? 1.0f / sum : __builtin_nanf("");
  const int mark = known ? (int)t - row.head : -1;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int j = tid + i * THREADS;
    as_stored(r[i].v);
    if (j < row.vecs) row.template put_grad<SAME, PAST>(j, r[i].v, top, share, m, mark);
  }
  if (edge >= 0) {
    const float p = exp_of(side - top) * share;
    row.grad[edge] = (E)(m * (known && edge == (int)t ? p - 1.0f : p));
  }
}

// Work: one float (1 / rows that count) and one unused, the targets' logits [N], the parts [N][parts].
__device__ __forceinline__ float* targets_of(const gs_xent& x) { return static_cast<float*>(x.work) + 2; }
__device__ __forceinline__ Seen* parts_of(const gs_xent& x, int64_t n, int parts) {
  return reinterpret_cast<Seen*>(static_cast<float*>(x.work) + 2 + (x.N + 1) / 2 * 2) + n * parts;
}

template <int DT, bool PAST>
__global__ void __launch_bounds__(kPartThreads) k_xent_part(gs_xent x, int parts, int part_vecs) {
  using R = Row<DT>;
  using P = typename R::P;
  __shared__ Seen lds[kPartThreads / 64];
  const int64_t id = group_of(), n = id / parts;
  if (n >= x.N) return;
  const int64_t t = x.targets[n];
  if (t == x.ignore_index) return;
  const int part = (int)(id - n * parts), tid = threadIdx.x;
  const R row(x, n);
  const int from = part * part_vecs, to = from + part_vecs < row.vecs ? from + part_vecs : row.vecs;
  Seen mine{-inf(), 0.0f};
  if (part == 0) {
    if (tid == 0) targets_of(x)[n] = t >= 0 && t < x.V ? (float)row.z[t] : __builtin_nanf("");
    const int edge = row.edge(tid);
    if (edge >= 0) {
      const float z = (float)row.z[edge];
      mine = Seen{fmaxf(z, -inf()), exp_of(z - base_of(fmaxf(z, -inf())))};
    }
  }
  constexpr int U = 8;
  for (int j0 = from + tid; j0 < to; j0 += U * kPartThreads) {
    typename P::raw r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kPartThreads;
      if (j < to)
        r[u] = row.template get<PAST>(j);
      else
        r[u] = P::down((typename P::wide)(-inf()));
    }
    Seen now{-inf(), 0.0f};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const typename P::wide v = P::up(r[u]);
#pragma unroll
      for (int e = 0; e < R::N; ++e) now.top = fmaxf(now.top, v[e]);
    }
    const float b = base_of(now.top);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const typename P::wide v = P::up(r[u]);
#pragma unroll
      for (int e = 0; e < R::N; ++e) now.sum += exp_of(v[e] - b);
    }
    mine = join(mine, now);
  }
  mine = block_reduce<kPartThreads>(mine, lds, join);
  if (tid == 0) parts_of(x, n, parts)[part] = mine;
}

// Joins a row's parts (every workgroup, in one order) and writes the gradient of one of them. Without a
// gradient there is one workgroup a row.
template <int DT, bool GRAD, bool SAME>
__global__ void __launch_bounds__(kPartThreads) k_xent_join(gs_xent x, int parts, int part_vecs) {
  using R = Row<DT>;
  using P = typename R::P;
  using E = typename R::E;
  const int64_t id = group_of(), n = GRAD ? id / parts : id;
  if (n >= x.N) return;
  const int64_t t = x.targets[n];
  const int part = GRAD ? (int)(id - n * parts) : 0, tid = threadIdx.x;
  const R row(x, n);
  const int from = part * part_vecs, to = from + part_vecs < row.vecs ? from + part_vecs : row.vecs;
  const int edge = part == 0 ? row.edge(tid) : -1;
  if (t == x.ignore_index) {
    if (part == 0 && tid == 0 && x.losses) x.losses[n] = 0.0f;
    if (GRAD) {
      for (int j = from + tid; j < to; j += kPartThreads)
        row.template put<SAME, true>(j, P::down((typename P::wide)0.0f));
      if (edge >= 0) row.grad[edge] = (E)0.0f;
    }
    return;
  }
  __shared__ Seen lds[kPartThreads / 64];
  Seen s{-inf(), 0.0f};
  if (tid < parts) s = parts_of(x, n, parts)[tid];
  s = block_reduce<kPartThreads>(s, lds, join);
  if (part == 0 && tid == 0 && x.losses) x.losses[n] = logf(s.sum) - (targets_of(x)[n] - s.top);
  if (!GRAD) return;
  const bool known = t >= 0 && t < x.V;
  const float share = known ? 1.0f / s.sum : __builtin_nanf(""), m = factor_of(x, n);
  const int mark = known ? (int)t - row.head : -1;
  constexpr int U = 4;
  for (int j0 = from + tid; j0 < to; j0 += U * kPartThreads) {
    typename P::raw r[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * kPartThreads < to) r[u] = row.template get<true>(j0 + u * kPartThreads);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * kPartThreads < to) row.template put_grad<SAME, true>(j0 + u * kPartThreads, r[u], s.top, share, m, mark);
  }
  if (edge >= 0) {
    const float p = exp_of((float)row.z[edge] - s.top) * share;
    row.grad[edge] = (E)(m * (known && edge == (int)t ? p - 1.0f : p));
  }
}

// How a row is worked on: parts > 0: split.
struct Cut {
  int parts, part_vecs;
};

Cut cut_of(int64_t N, int64_t V, int dtype) {
  const int64_t vecs = V / (16 / elem_size(dtype)), least = kPartThreads * kPartVecs;
  int64_t parts = 0;
  if (vecs > (int64_t)kRowThreads * kRowPieces || (N <= kFewRows && vecs >= kLongRow)) {
    parts = N > 0 ? (kSplitWant + N - 1) / N : 1;
    const int64_t most = (vecs + least - 1) / least;
    parts = parts < most ? parts : most;
    parts = parts < kMaxParts ? parts : kMaxParts;
  }
  Cut k{(int)parts, 0};
  if (parts > 0) k.part_vecs = (int)((vecs + parts - 1) / parts);
  return k;
}

template <int DT, bool GRAD, bool SAME>
void rows(hipStream_t s, const gs_xent& x) {
  const int64_t vecs = x.V / (16 / elem_size(DT));
  const dim3 grid = grid_of(x.N);
  // The fewest threads whose pieces hold the row, one to four pieces a thread in a wave, two to eight from 256 threads on.
  // 2,049 to 3,072 pieces go to 512 threads as well as more do: twelve a thread of 256 took longer (4,096 rows with gradient:
  // 20,000 bf16 logits 70 us for 66, 22,000 78 for 72.5, 24,500 86 for 80; 11,000 fp32 74 for 71; 2,000 x 8,400 33.6 for 31.5).
#define GS_XENT(THREADS, CH) \
  if (vecs <= (THREADS) * (CH)) return k_xent_row<DT, THREADS, CH, GRAD, SAME><<<grid, THREADS, 0, s>>>(x), void()
  GS_XENT(64, 1);
  GS_XENT(64, 2);
  GS_XENT(64, 4);
  GS_XENT(256, 2);
  GS_XENT(256, 4);
  GS_XENT(256, 8);
  GS_XENT(512, 8);
  GS_XENT(1024, 8);
#undef GS_XENT
  if ((((uintptr_t)x.logits | (x.logits_stride * elem_size(DT))) & 127) == 0)
    k_xent_row<DT, kRowThreads, kRowPieces, GRAD, SAME, true><<<grid, kRowThreads, 0, s>>>(x);
  else
    k_xent_row<DT, kRowThreads, kRowPieces, GRAD, SAME, false><<<grid, kRowThreads, 0, s>>>(x);
}

template <int DT, bool GRAD, bool SAME>
void launch(hipStream_t s, const gs_xent& x) {
  const Cut k = cut_of(x.N, x.V, DT);
  if (k.parts == 0) return rows<DT, GRAD, SAME>(s, x);
  const dim3 grid = grid_of(x.N * k.parts);
  // few rows are still in the caches when they are read again; many are not (1,000 x 150,000 bf16: 94 + 103 us with
  // the first read through the caches, 57 + 117 past them)
  if (x.N <= kFewRows)
    k_xent_part<DT, false><<<grid, kPartThreads, 0, s>>>(x, k.parts, k.part_vecs);
  else
    k_xent_part<DT, true><<<grid, kPartThreads, 0, s>>>(x, k.parts, k.part_vecs);
  k_xent_join<DT, GRAD, SAME><<<GRAD ? grid : grid_of(x.N), kPartThreads, 0, s>>>(x, k.parts, k.part_vecs);
}

template <int DT>
void launch(hipStream_t s, const gs_xent& x) {
  const int64_t bytes = elem_size(DT);
  const bool same = x.grad && (((uintptr_t)x.grad - (uintptr_t)x.logits) & 15) == 0 &&
                    (x.N == 1 || ((x.grad_stride - x.logits_stride) * bytes & 15) == 0);
  if (!x.grad)
    launch<DT, false, true>(s, x);
  else if (same)
    launch<DT, true, true>(s, x);
  else
    launch<DT, true, false>(s, x);
}

}  // namespace

int64_t cross_entropy_work(int64_t N, int64_t V, int dtype) {
  const Cut k = cut_of(N, V, dtype);
  if (k.parts == 0 && N <= kInlineCount) return 0;
  return 8 + (k.parts ? (N + 1) / 2 * 8 + N * k.parts * (int64_t)sizeof(Seen) : 0);
}

hipError_t launch_cross_entropy(hipStream_t s, const gs_xent& x) {
  if (x.N == 0 && !x.mean_loss) return hipSuccess;
  if (x.N > 0) {
    if (x.mean && x.grad && x.N > kInlineCount) k_xent_count<kTail><<<1, kTail, 0, s>>>(x);
    if (x.dtype == GS_F32) launch<GS_F32>(s, x);
    if (x.dtype == GS_BF16) launch<GS_BF16>(s, x);
    if (x.dtype == GS_F16) launch<GS_F16>(s, x);
  }
  if (x.mean_loss) {
    if (x.N <= 64)
      k_xent_mean<64><<<1, 64, 0, s>>>(x);
    else
      k_xent_mean<kTail><<<1, kTail, 0, s>>>(x);
  }
  return hipGetLastError();
}

}  // namespace gs
