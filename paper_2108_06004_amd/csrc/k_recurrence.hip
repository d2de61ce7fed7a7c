// k_recurrence.hip -- the gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) x_t, a = sigmoid(f),
// y_t = sigmoid(o_t) h_t, and its backward pass (include/gs.h).
//
// A stretch of steps acts on the state as one affine map, h -> A h + S with A the product of its
// gates and S its result from h = 0, and two stretches join as (A2 A1, A2 S1 + S2). So time splits
// three times:
//   - a thread takes L consecutive steps of VEC neighbouring channels. Their loads are all in flight
//     together (L for each array); it forms its own (A, S) in registers;
//   - a workgroup of W x G threads takes a strip of W VEC channels and a block of G L = 128 steps. The
//     groups' maps go through LDS, every thread joins those before its own and runs its steps
//     again from registers with the true state. One barrier a block: the maps have two buffers;
//   - where B and C give too few workgroups, `segs` workgroups share a sequence's blocks. A first
//     kernel reduces each segment to its map (reading x and f once more), the second starts each segment
//     from the joined maps before it.
// The backward pass runs the blocks from the last to the first. s_t = q_t + a_(t+1) s_(t+1) is the
// same recurrence in reverse, carried as c_t = a_t s_t with the map c -> A c + R; the states are computed
// again from the state before each block that the forward pass saved (4 / 128 bytes a step).
#include <type_traits>

#include "gs_lm.hpp"

namespace gs {
namespace {

constexpr int kWantGroups = 512;            // workgroups that fill the chip: two a CU
constexpr int kMaxSegs = 128;
constexpr int kGridY = 32768;

__device__ __forceinline__ int64_t length_of(const RecurrenceArgs& a, int64_t b) {
  if (!a.lengths) return a.T;
  const int64_t n = a.lengths[b];
  return n < 0 ? 0 : n > a.T ? a.T : n;
}

// How a launch cuts the problem: `strips` of channels x `segs` of blocks x sequences.
struct Cut {
  unsigned strips;
  int segs;
  int64_t blocks, seg_blocks;
};

// Where one workgroup is; a reducing backward kernel leaves out segment 0.
struct Place {
  int64_t b, blk0, blk1;
  unsigned strip;
  int seg;
};

__device__ __forceinline__ Place place_of(const Cut& k, int from) {
  Place p;
  const unsigned part = blockIdx.x / k.strips;
  p.strip = blockIdx.x - part * k.strips;
  p.seg = (int)part + from;
  p.b = (int64_t)blockIdx.z * kGridY + blockIdx.y;
  p.blk0 = p.seg * k.seg_blocks;
  p.blk1 = p.blk0 + k.seg_blocks < k.blocks ? p.blk0 + k.seg_blocks : k.blocks;
  return p;
}

// Step t of a strip of an array, as a base that is the same for the whole workgroup; a thread's own
// part of the offset stays below 2^31 bytes (127 steps of at most GS_RECURRENCE_MAX_STRIDE fp32 elements,
// 64 channels).
__device__ __forceinline__ char* row(const Rows& r, int64_t b, int64_t t, int64_t strip_bytes) {
  return r.p + b * r.batch + t * r.time + strip_bytes;
}

template <int DT, int VEC>
__device__ __forceinline__ typename Pack<DT, VEC>::raw load(const char* base, uint32_t off) {
  return *reinterpret_cast<const typename Pack<DT, VEC>::raw*>(base + off);
}

template <int DT, int VEC>
__device__ __forceinline__ void store(char* base, uint32_t off, typename Pack<DT, VEC>::wide v) {
  *reinterpret_cast<typename Pack<DT, VEC>::raw*>(base + off) = Pack<DT, VEC>::down(v);
}

template <int VEC>
__device__ __forceinline__ typename Pack<GS_F32, VEC>::wide loadf(const float* p) {
  return *reinterpret_cast<const typename Pack<GS_F32, VEC>::wide*>(p);
}

template <int VEC>
__device__ __forceinline__ void storef(float* p, typename Pack<GS_F32, VEC>::wide v) {
  *reinterpret_cast<typename Pack<GS_F32, VEC>::wide*>(p) = v;
}

template <int VEC, typename V>
__device__ __forceinline__ V join(V a, V h, V s) {  // a h + s, one rounding
  V r;
#pragma unroll
  for (int j = 0; j < VEC; ++j) r[j] = fmaf(a[j], h[j], s[j]);
  return r;
}

// L steps of one array for one thread. Steps past the last token read the last token's row again
// (the caller drops what they hold), so nothing beyond the sequence is touched.
template <int DT, int VEC, int L>
struct Steps {
  typename Pack<DT, VEC>::raw v[L];
  __device__ __forceinline__ void get(const Rows& r, int64_t b, int64_t t0, int64_t strip_bytes, int first,
                                      uint32_t coff, int last) {
    const char* base = row(r, b, t0, strip_bytes);
    if (first + L - 1 <= last) {
      const uint32_t off = (uint32_t)first * (uint32_t)r.time + coff;
#pragma unroll
      for (int i = 0; i < L; ++i) v[i] = load<DT, VEC>(base + i * r.time, off);
    } else {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        const int t = first + i < last ? first + i : last;
        v[i] = load<DT, VEC>(base, (uint32_t)t * (uint32_t)r.time + coff);
      }
    }
  }
};

// The gates of L steps: kept a, taken 1 - a; padding keeps everything.
template <int DT, int VEC, int L, typename V>
__device__ __forceinline__ void gates(const Steps<DT, VEC, L>& f, int first, int last, V (&k)[L], V (&rest)[L]) {
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const V z = Pack<DT, VEC>::up(f.v[i]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      float a, r;
      sigmoid_both(z[j], a, r);
      k[i][j] = a;
      rest[i][j] = r;
    }
  }
  if (first + L - 1 > last) {
#pragma unroll
    for (int i = 0; i < L; ++i)
      if (first + i > last) {
        k[i] = (V)1.0f;
        rest[i] = (V)0.0f;
      }
  }
}

// work: for each sequence and segment, the map that its state before the segment joins last: [B][segs][2][C].
// Slot 0 is (0, h0), slot s the map of segment s - 1 (forward); slot segs - 1 is (0, gh), slot s that of segment
// s + 1 (backward). So the second kernel reads no h0, which h_last may overwrite.
__device__ __forceinline__ float* slot_of(float* work, const Cut& k, int64_t b, int64_t s, int64_t C) {
  return work + ((b * k.segs + s) * 2) * C;
}

template <int DT, int VEC, bool GATE, int W, int G, int L, bool REDUCE>
__global__ void __launch_bounds__(W* G) k_recurrence_fwd(RecurrenceArgs a, Cut cut) {
  using V = typename Pack<GS_F32, VEC>::wide;
  constexpr int kSpan = G * L;
  __shared__ V maps[G > 1 ? 2 : 1][2][G > 1 ? G : 1][G > 1 ? W : 1];
  const Place p = place_of(cut, 0);
  if (p.b >= a.B) return;
  const int lane = threadIdx.x % W, g = threadIdx.x / W;
  const int64_t c0 = (int64_t)p.strip * (W * VEC);
  const bool live = c0 + lane * VEC < a.C;
  const int64_t c = live ? c0 + lane * VEC : a.C - VEC;  // lanes past the last channel repeat it and store nothing
  const int64_t sb = c0 * (int64_t)sizeof(typename Elem<DT>::type);
  const uint32_t off = (uint32_t)(c - c0) * (uint32_t)sizeof(typename Elem<DT>::type);
  const int64_t n = length_of(a, p.b);
  V h = (V)0.0f, prod = (V)1.0f;
  if (REDUCE) {
    if (p.seg == 0 && live && g == 0) {
      storef<VEC>(slot_of(a.work, cut, p.b, 0, a.C) + c, (V)0.0f);
      storef<VEC>(slot_of(a.work, cut, p.b, 0, a.C) + a.C + c, a.h0 ? loadf<VEC>(a.h0 + p.b * a.C + c) : (V)0.0f);
    }
  } else if (cut.segs > 1) {
    for (int s = 0; s <= p.seg; ++s) {
      const float* m = slot_of(a.work, cut, p.b, s, a.C) + c;
      h = join<VEC>(loadf<VEC>(m), h, loadf<VEC>(m + a.C));
    }
  } else if (a.h0) {
    h = loadf<VEC>(a.h0 + p.b * a.C + c);
  }
  for (int64_t blk = p.blk0; blk < p.blk1; ++blk) {
    const int64_t t0 = blk * kSpan;
    const int first = g * L;
    if (t0 < n) {
      const int last = n - t0 < kSpan ? (int)(n - t0) - 1 : kSpan - 1;
      if (!REDUCE && a.states && g == 0 && live) storef<VEC>(a.states + (p.b * cut.blocks + blk) * a.C + c, h);
      Steps<DT, VEC, L> xs, fs, os;
      fs.get(a.f, p.b, t0, sb, first, off, last);
      xs.get(a.x, p.b, t0, sb, first, off, last);
      if (GATE && !REDUCE) os.get(a.o, p.b, t0, sb, first, off, last);
      V k[L], in[L];
      gates<DT, VEC, L>(fs, first, last, k, in);
      V A = (V)1.0f, S = (V)0.0f;
#pragma unroll
      for (int i = 0; i < L; ++i) {
        V xi = Pack<DT, VEC>::up(xs.v[i]);
        if (first + i > last) xi = (V)0.0f;  // padding may hold anything, NaN too
        in[i] = in[i] * xi;
        A = A * k[i];
        S = join<VEC>(k[i], S, in[i]);
      }
      V mine = h;
      if (G > 1) {
        const int buf = (int)(blk & 1);
        maps[buf][0][g][lane] = A;
        maps[buf][1][g][lane] = S;
        __syncthreads();
#pragma unroll 4
        for (int s = 0; s < G; ++s) {
          if (s == g) mine = h;
          const V As = maps[buf][0][s][lane];
          h = join<VEC>(As, h, maps[buf][1][s][lane]);
          if (REDUCE) prod = prod * As;
        }
      } else {
        h = join<VEC>(A, h, S);
        if (REDUCE) prod = prod * A;
      }
      if (!REDUCE) {
        char* base = row(a.y, p.b, t0, sb);
#pragma unroll
        for (int i = 0; i < L; ++i) {
          mine = join<VEC>(k[i], mine, in[i]);
          V out = mine;
          if (GATE) {
            const V z = Pack<DT, VEC>::up(os.v[i]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
              float s, r;
              sigmoid_both(z[j], s, r);
              out[j] = s * out[j];
            }
          }
          if (first + i > last) out = (V)0.0f;
          if (live && t0 + first + i < a.T)
            store<DT, VEC>(base, (uint32_t)(first + i) * (uint32_t)a.y.time + off, out);
        }
      }
    } else if (!REDUCE && live) {
      char* base = row(a.y, p.b, t0, sb);
      for (int i = 0; i < L && t0 + first + i < a.T; ++i)
        store<DT, VEC>(base, (uint32_t)(first + i) * (uint32_t)a.y.time + off, (V)0.0f);
    }
  }
  if (g != 0 || !live) return;
  if (REDUCE) {
    float* m = slot_of(a.work, cut, p.b, p.seg + 1, a.C) + c;
    storef<VEC>(m, prod);
    storef<VEC>(m + a.C, h);
  } else if (p.seg == cut.segs - 1) {
    storef<VEC>(a.h_last + p.b * a.C + c, h);
  }
}

template <int DT, int VEC, bool GATE, int W, int G, int L, bool REDUCE>
__global__ void __launch_bounds__(W* G) k_recurrence_bwd(RecurrenceArgs a, Cut cut) {
  using V = typename Pack<GS_F32, VEC>::wide;
  constexpr int kSpan = G * L;
  __shared__ V maps[G > 1 ? 2 : 1][3][G > 1 ? G : 1][G > 1 ? W : 1];
  const Place p = place_of(cut, REDUCE ? 1 : 0);
  if (p.b >= a.B) return;
  const int lane = threadIdx.x % W, g = threadIdx.x / W;
  const int64_t c0 = (int64_t)p.strip * (W * VEC);
  const bool live = c0 + lane * VEC < a.C;
  const int64_t c = live ? c0 + lane * VEC : a.C - VEC;
  const int64_t sb = c0 * (int64_t)sizeof(typename Elem<DT>::type);
  const uint32_t off = (uint32_t)(c - c0) * (uint32_t)sizeof(typename Elem<DT>::type);
  const int64_t n = length_of(a, p.b);
  V carry = (V)0.0f, prod = (V)1.0f;
  if (REDUCE) {
    if (p.seg == cut.segs - 1 && live && g == 0) {
      float* m = slot_of(a.work, cut, p.b, cut.segs - 1, a.C) + c;
      storef<VEC>(m, (V)0.0f);
      storef<VEC>(m + a.C, a.gh ? loadf<VEC>(a.gh + p.b * a.C + c) : (V)0.0f);
    }
  } else if (cut.segs > 1) {
    for (int s = cut.segs - 1; s >= p.seg; --s) {
      const float* m = slot_of(a.work, cut, p.b, s, a.C) + c;
      carry = join<VEC>(loadf<VEC>(m), carry, loadf<VEC>(m + a.C));
    }
  } else if (a.gh) {
    carry = loadf<VEC>(a.gh + p.b * a.C + c);
  }
  for (int64_t blk = p.blk1 - 1; blk >= p.blk0; --blk) {
    const int64_t t0 = blk * kSpan;
    const int first = g * L;
    if (t0 < n) {
      const int last = n - t0 < kSpan ? (int)(n - t0) - 1 : kSpan - 1;
      Steps<DT, VEC, L> xs, fs, os, gs;
      fs.get(a.f, p.b, t0, sb, first, off, last);
      gs.get(a.gy, p.b, t0, sb, first, off, last);
      if (GATE) os.get(a.o, p.b, t0, sb, first, off, last);
      V h = (V)0.0f;
      if (!REDUCE) {
        xs.get(a.x, p.b, t0, sb, first, off, last);
        h = loadf<VEC>(a.states + (p.b * cut.blocks + blk) * a.C + c);
      }
      V k[L], rest[L], q[L], shut[L];  // shut: gy sigmoid(o) (1 - sigmoid(o)), the factor of h in do
      gates<DT, VEC, L>(fs, first, last, k, rest);
      V A = (V)1.0f, S = (V)0.0f, R = (V)0.0f;
#pragma unroll
      for (int i = 0; i < L; ++i) {
        const bool pad = first + i > last;
        q[i] = pad ? (V)0.0f : Pack<DT, VEC>::up(gs.v[i]);
        if (GATE) {
          const V z = Pack<DT, VEC>::up(os.v[i]);
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            float s, r;
            sigmoid_both(pad ? 0.0f : z[j], s, r);
            q[i][j] = q[i][j] * s;
            shut[i][j] = q[i][j] * r;
          }
        }
        A = A * k[i];
        if (!REDUCE) {
          const V xi = pad ? (V)0.0f : Pack<DT, VEC>::up(xs.v[i]);
          S = join<VEC>(k[i], S, rest[i] * xi);
        }
      }
#pragma unroll
      for (int i = L - 1; i >= 0; --i) R = k[i] * (q[i] + R);
      V c_in = carry;
      if (G > 1) {
        const int buf = (int)(blk & 1);
        maps[buf][0][g][lane] = A;
        maps[buf][1][g][lane] = R;
        if (!REDUCE) maps[buf][2][g][lane] = S;
        __syncthreads();
#pragma unroll 4
        for (int s = G - 1; s >= 0; --s) {
          if (s == g) c_in = carry;
          const V As = maps[buf][0][s][lane];
          carry = join<VEC>(As, carry, maps[buf][1][s][lane]);
          if (REDUCE) prod = prod * As;
        }
        if (!REDUCE) {
          V hs = h;
#pragma unroll 4
          for (int s = 0; s < G - 1; ++s) {
            hs = join<VEC>(maps[buf][0][s][lane], hs, maps[buf][2][s][lane]);
            if (s == g - 1) h = hs;
          }
        }
      } else {
        carry = join<VEC>(A, carry, R);
        if (REDUCE) prod = prod * A;
      }
      if (!REDUCE) {
        V before[L];
#pragma unroll
        for (int i = 0; i < L; ++i) {
          const V xi = first + i > last ? (V)0.0f : Pack<DT, VEC>::up(xs.v[i]);
          before[i] = h;
          h = join<VEC>(k[i], h, rest[i] * xi);
          if (GATE) shut[i] = shut[i] * h;
        }
#pragma unroll
        for (int i = L - 1; i >= 0; --i) {
          const bool pad = first + i > last;
          const V xi = pad ? (V)0.0f : Pack<DT, VEC>::up(xs.v[i]);
          const V s = q[i] + c_in;
          c_in = k[i] * s;
          if (live && t0 + first + i < a.T) {
            const uint32_t t = (uint32_t)(first + i);
            // padding: rest = 0 and shut = 0
            const V dx = rest[i] * s, df = s * (before[i] - xi) * (k[i] * rest[i]);
            store<DT, VEC>(row(a.dx, p.b, t0, sb), t * (uint32_t)a.dx.time + off, dx);
            store<DT, VEC>(row(a.df, p.b, t0, sb), t * (uint32_t)a.df.time + off, df);
            if (GATE) store<DT, VEC>(row(a.dout, p.b, t0, sb), t * (uint32_t)a.dout.time + off, shut[i]);
          }
        }
      }
    } else if (!REDUCE && live) {
      for (int i = 0; i < L && t0 + first + i < a.T; ++i) {
        const uint32_t t = (uint32_t)(first + i);
        store<DT, VEC>(row(a.dx, p.b, t0, sb), t * (uint32_t)a.dx.time + off, (V)0.0f);
        store<DT, VEC>(row(a.df, p.b, t0, sb), t * (uint32_t)a.df.time + off, (V)0.0f);
        if (GATE) store<DT, VEC>(row(a.dout, p.b, t0, sb), t * (uint32_t)a.dout.time + off, (V)0.0f);
      }
    }
  }
  if (g != 0 || !live) return;
  if (REDUCE) {
    float* m = slot_of(a.work, cut, p.b, p.seg - 1, a.C) + c;
    storef<VEC>(m, prod);
    storef<VEC>(m + a.C, carry);
  } else if (p.seg == 0 && a.dh0) {
    storef<VEC>(a.dh0 + p.b * a.C + c, carry);
  }
}

// Steps of one thread, threads across the channels, groups along time: single tokens, up to eight
// steps, anything longer.
template <int DT, int VEC, bool GATE, bool REDUCE>
void forward(hipStream_t s, const RecurrenceArgs& a, const Cut& k, dim3 grid) {
  if (a.T <= 1)
    k_recurrence_fwd<DT, VEC, GATE, 64, 1, 1, false><<<grid, 64, 0, s>>>(a, k);
  else if (a.T <= 8)
    k_recurrence_fwd<DT, VEC, GATE, 64, 1, 8, false><<<grid, 64, 0, s>>>(a, k);
  else
    k_recurrence_fwd<DT, VEC, GATE, 32, 16, 8, REDUCE><<<grid, 512, 0, s>>>(a, k);
}

template <int DT, int VEC, bool GATE, bool REDUCE>
void backward(hipStream_t s, const RecurrenceArgs& a, const Cut& k, dim3 grid) {
  if (a.T <= 1)
    k_recurrence_bwd<DT, VEC, GATE, 64, 1, 1, false><<<grid, 64, 0, s>>>(a, k);
  else if (a.T <= 8)
    k_recurrence_bwd<DT, VEC, GATE, 64, 1, 8, false><<<grid, 64, 0, s>>>(a, k);
  else
    k_recurrence_bwd<DT, VEC, GATE, 32, 16, 8, REDUCE><<<grid, 512, 0, s>>>(a, k);
}

Cut cut_of(int64_t B, int64_t T, int64_t C, int vec) {
  Cut k{};
  const int64_t across = (T > 8 ? 32 : 64) * vec;
  k.strips = (unsigned)((C + across - 1) / across);
  k.blocks = T > 8 ? GS_RECURRENCE_BLOCKS(T) : T > 0 ? 1 : 0;
  k.segs = 1;
  k.seg_blocks = k.blocks;
  const int64_t groups = B * (int64_t)k.strips;
  if (2 * groups <= kWantGroups && k.blocks > 1) {
    int64_t segs = kWantGroups / groups;
    segs = segs < k.blocks ? segs : k.blocks;
    segs = segs < kMaxSegs ? segs : kMaxSegs;
    k.seg_blocks = (k.blocks + segs - 1) / segs;
    k.segs = (int)((k.blocks + k.seg_blocks - 1) / k.seg_blocks);
  }
  return k;
}

dim3 grid_of(const Cut& k, int parts, int64_t B) {
  const int64_t y = B < kGridY ? B : kGridY;
  return dim3(k.strips * (unsigned)parts, (unsigned)y, (unsigned)((B + y - 1) / y));
}

// Two channels a lane where every row of every array starts on a pair of elements.
bool pairs(const Rows& r, int bytes) {
  const int64_t m = 2 * bytes - 1;
  return ((uintptr_t)r.p & m) == 0 && (r.batch & m) == 0 && (r.time & m) == 0;
}

bool pairs(const float* p) { return ((uintptr_t)p & 7) == 0; }

template <typename F>
void with_type(int dtype, bool two, bool gate, F f) {
  auto g = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    using True = std::true_type;
    using False = std::false_type;
    if (two)
      gate ? f(dt, std::integral_constant<int, 2>(), True()) : f(dt, std::integral_constant<int, 2>(), False());
    else
      gate ? f(dt, std::integral_constant<int, 1>(), True()) : f(dt, std::integral_constant<int, 1>(), False());
    (void)DT;
  };
  if (dtype == GS_F32) g(std::integral_constant<int, GS_F32>());
  if (dtype == GS_BF16) g(std::integral_constant<int, GS_BF16>());
  if (dtype == GS_F16) g(std::integral_constant<int, GS_F16>());
}

}  // namespace

// For each sequence and segment one map; more segments where a lane takes two channels.
int64_t recurrence_work(int64_t B, int64_t T, int64_t C, int) {
  if (B == 0 || T == 0 || C == 0) return 0;
  const Cut k = cut_of(B, T, C, C % 2 == 0 ? 2 : 1);
  return k.segs > 1 ? B * k.segs * 2 * C * (int64_t)sizeof(float) : 0;
}

hipError_t launch_recurrence_forward(hipStream_t s, int dtype, const RecurrenceArgs& a) {
  const int bytes = elem_size(dtype);
  const bool two = a.C % 2 == 0 && (a.T == 0 || (pairs(a.x, bytes) && pairs(a.f, bytes) && pairs(a.y, bytes) &&
                                                 (!a.o.p || pairs(a.o, bytes)))) &&
                   pairs(a.h0) && pairs(a.h_last) && pairs(a.states) && pairs(a.work);
  const Cut k = cut_of(a.B, a.T, a.C, two ? 2 : 1);
  with_type(dtype, two, a.o.p != nullptr, [&](auto dt, auto vec, auto gate) {
    constexpr int DT = decltype(dt)::value, VEC = decltype(vec)::value;
    constexpr bool GATE = decltype(gate)::value;
    if (k.segs > 1) forward<DT, VEC, false, true>(s, a, k, grid_of(k, k.segs - 1, a.B));
    forward<DT, VEC, GATE, false>(s, a, k, grid_of(k, k.segs, a.B));
  });
  return hipGetLastError();
}

hipError_t launch_recurrence_backward(hipStream_t s, int dtype, const RecurrenceArgs& a) {
  const int bytes = elem_size(dtype);
  const bool two = a.C % 2 == 0 &&
                   (a.T == 0 || (pairs(a.x, bytes) && pairs(a.f, bytes) && pairs(a.gy, bytes) && pairs(a.dx, bytes) &&
                                 pairs(a.df, bytes) && (!a.o.p || (pairs(a.o, bytes) && pairs(a.dout, bytes))))) &&
                   pairs(a.gh) && pairs(a.dh0) && pairs(a.states) && pairs(a.work);
  const Cut k = cut_of(a.B, a.T, a.C, two ? 2 : 1);
  with_type(dtype, two, a.o.p != nullptr, [&](auto dt, auto vec, auto gate) {
    constexpr int DT = decltype(dt)::value, VEC = decltype(vec)::value;
    constexpr bool GATE = decltype(gate)::value;
    if (k.segs > 1) backward<DT, VEC, GATE, true>(s, a, k, grid_of(k, k.segs - 1, a.B));
    backward<DT, VEC, GATE, false>(s, a, k, grid_of(k, k.segs, a.B));
  });
  return hipGetLastError();
}

}  // namespace gs
