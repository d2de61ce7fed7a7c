// k_recurrence.hip -- the gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) x_t, a = sigmoid(f),
// y_t = sigmoid(o_t) h_t, and its backward pass (include/gs.h).
//
// A stretch of steps acts on the state as one affine map, h -> A h + S with A the product of its
// gates and S its result from h = 0, and two stretches join as (A2 A1, A2 S1 + S2). So time splits
// three times:
//   - a thread takes L consecutive steps of VEC neighbouring channels. Their loads are all in flight
//     together (L for each array); it forms its own (A, S) in registers;
//   - a workgroup of W x G threads takes a strip of W VEC channels and blocks of G L steps (32, 64 or
//     128), a wave L of them. The waves' maps go through LDS, every thread joins those before its own and runs
//     its steps again from registers with the true state. One barrier a block: the maps have two buffers. The
//     next block's loads are under way meanwhile;
//   - where B and C give too few workgroups, `segs` workgroups share a sequence's blocks. A first
//     kernel reduces each segment to its map (reading x and f once more), the second starts each segment
//     from the joined maps before it.
// The backward pass runs the blocks from the last to the first. s_t = q_t + a_(t+1) s_(t+1) is the
// same recurrence in reverse, carried as c_t = a_t s_t with the map c -> A c + R; the states are computed
// again from the state before every 32 steps that the forward pass saved (an eighth of a byte a step and channel).
//
// What bounds it: memory for long inputs (16 x 4,096 x 2,048 bf16: forward 205 us, 5.25 TB/s of its 8 bytes an element,
// backward 369 us, 5.1 TB/s of 14; VALU 48 and 42% busy, waves waiting for memory half their time). Short
// ones are bound by the launch (one token of 1,500 channels: 2.8 us). Split along time the reading twice adds to that (1 x
// 65,536 x 1,024: 47 of 151 us forward, 72 of 256 backward).
#include <type_traits>

#include "gs_lm.hpp"

namespace gs {
namespace {

constexpr unsigned kGridX = 1u << 22;  // a grid's first dimension holds fewer than 2^32 threads

// The tokens of a sequence, in a scalar register: what follows from it (blocks, buffers) is the same for the
// whole workgroup, and the compiler has to see that.
__device__ __forceinline__ int length_of(const RecurrenceArgs& a, int64_t b) {
  const int T = (int)a.T;
  const int n = a.lengths ? __builtin_amdgcn_readfirstlane(a.lengths[b]) : T;
  return n < 0 ? 0 : n > T ? T : n;
}

// How a launch cuts the problem: `strips` of channels x `segs` of blocks x sequences.
struct Cut {
  unsigned strips;
  int segs, groups;
  int blocks, all, seg_blocks;  // saved states of a sequence; the workgroups' own blocks, all and a segment's
};

// Where one workgroup is; a reducing kernel leaves out the last segment, or going backward the first (from = 1).
struct Place {
  int64_t b;
  unsigned strip;
  int seg, blk0, blk1;
};

// Workgroups go to the eight XCDs in turn, and each XCD has its own L2. Rows that are no multiple of 128 bytes
// share lines between neighbouring strips, so all strips of a sequence's segment go to one XCD, one after the
// other (NEAR; what is left over past a multiple of eight segments goes as it comes).
template <bool NEAR>
__device__ __forceinline__ Place place_of(const Cut& k, unsigned parts, int from, int64_t B) {
  const unsigned id = blockIdx.y * kGridX + blockIdx.x;
  const unsigned even = NEAR ? (unsigned)B * parts / 8 * 8 : 0;
  Place p;
  unsigned item;
  if (NEAR && id < even * k.strips) {
    const unsigned slot = id / 8;
    item = slot / k.strips;
    p.strip = slot - item * k.strips;
    item = item * 8 + id % 8;
  } else {
    const unsigned left = id - even * k.strips;
    item = left / k.strips;
    p.strip = left - item * k.strips;
    item += even;
  }
  const unsigned b = item / parts;
  p.b = b;
  p.seg = (int)(item - b * parts) + from;
  p.blk0 = p.seg * k.seg_blocks;
  p.blk1 = p.blk0 + k.seg_blocks < k.all ? p.blk0 + k.seg_blocks : k.all;
  return p;
}

// One block of a strip of an array as a buffer: its first byte and the strides are the same for the whole
// workgroup (scalar registers), a thread adds one 32-bit offset, which stays below 2^31 (127 steps of at most
// GS_RECURRENCE_MAX_STRIDE elements of 32 bits are 127/128 of it, the strip's row less than the rest). Offset
// kNowhere is out of the buffer's range: a load there gives zero and a store is dropped, so steps and channels
// that are not there need no branches.
constexpr uint32_t kNowhere = 0x80000000u;
// Cache policies: through the caches, or past them (non-temporal). Rows that start and end on 128-byte lines go past
// them in both directions (16 x 4,096 x 2,048 bf16, both directions: 580 us, 603 with the gradients' pass through
// them), rows that share lines with their neighbours through them (64 x 512 x 1,500: 276 us, 306 past), but for
// y, which is stored past them (1 x 65,536 x 1,024: 440 us, 455 through them).
constexpr int kCached = 0, kPast = 2;

struct Block {
  __amdgpu_buffer_rsrc_t at;
  uint32_t time;
  __device__ __forceinline__ Block(const Rows& r, int64_t b, int t0, int64_t strip_bytes)
      : at(__builtin_amdgcn_make_buffer_rsrc(r.p + b * r.batch + t0 * r.time + strip_bytes, 0, kNowhere, 0x00027000)),
        time((uint32_t)r.time) {}
};

template <int DT, int VEC, int AUX>
__device__ __forceinline__ typename Pack<DT, VEC>::raw load(const Block& k, uint32_t off, uint32_t step) {
  using raw = typename Pack<DT, VEC>::raw;
  static_assert(sizeof(raw) == 4 || sizeof(raw) == 2, "one channel a lane, or two of 16 bits");
  if constexpr (sizeof(raw) == 4)
    return __builtin_bit_cast(raw, __builtin_amdgcn_raw_buffer_load_b32(k.at, off, step * k.time, AUX));
  else
    return __builtin_bit_cast(raw, __builtin_amdgcn_raw_buffer_load_b16(k.at, off, step * k.time, AUX));
}

template <int DT, int VEC, int AUX>
__device__ __forceinline__ void store(const Block& k, uint32_t off, uint32_t step, typename Pack<DT, VEC>::wide v) {
  const auto raw = Pack<DT, VEC>::down(v);
  if constexpr (sizeof raw == 4) {
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, raw), k.at, off, step * k.time, AUX);
  } else {
    __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, raw), k.at, off, step * k.time, AUX);
  }
}

template <int VEC>
__device__ __forceinline__ typename Pack<GS_F32, VEC>::wide loadf(const float* p) {
  return *reinterpret_cast<const typename Pack<GS_F32, VEC>::wide*>(p);
}

template <int VEC>
__device__ __forceinline__ void storef(float* p, typename Pack<GS_F32, VEC>::wide v) {
  *reinterpret_cast<typename Pack<GS_F32, VEC>::wide*>(p) = v;
}

// Makes the compiler hold a value as it is from here on: it neither puts off what computes it nor keeps
// what could be computed from it again (the fp32 form of 16-bit elements) beside it.
template <typename T>
__device__ __forceinline__ void pin(T& v) {
  if constexpr (sizeof(T) == 8) {
    uint64_t w = __builtin_bit_cast(uint64_t, v);
    asm volatile("" : "+v"(w));
    v = __builtin_bit_cast(T, w);
  } else if constexpr (sizeof(T) == 4) {
    uint32_t w = __builtin_bit_cast(uint32_t, v);
    asm volatile("" : "+v"(w));
    v = __builtin_bit_cast(T, w);
  }
}

template <int VEC, typename V>
__device__ __forceinline__ V join(V a, V h, V s) {  // a h + s, one rounding
  V r;
#pragma unroll
  for (int j = 0; j < VEC; ++j) r[j] = fmaf(a[j], h[j], s[j]);
  return r;
}

// L steps of one array for one thread, from step `first` of its block. FULL: the block ends before the
// sequence does; otherwise the steps past `last` are not read and hold zero.
template <int DT, int VEC, int L, int AUX>
struct Steps {
  typename Pack<DT, VEC>::raw v[L];
  template <bool FULL>
  __device__ __forceinline__ void get(const Block& k, int first, uint32_t coff, int last, bool live) {
    const uint32_t off = live ? (uint32_t)first * k.time + coff : kNowhere;
#pragma unroll
    for (int i = 0; i < L; ++i) v[i] = load<DT, VEC, AUX>(k, FULL || first + i <= last ? off : kNowhere, i);
  }
  __device__ __forceinline__ typename Pack<DT, VEC>::wide at(int i) const { return Pack<DT, VEC>::up(v[i]); }
};

// Step i of a thread is padding.
template <bool FULL>
__device__ __forceinline__ bool padded(int first, int i, int last) {
  return !FULL && first + i > last;
}

// The gates of L steps: kept a, taken 1 - a; padding keeps everything.
template <bool FULL, int DT, int VEC, int L, int AUX, typename V>
__device__ __forceinline__ void gates(const Steps<DT, VEC, L, AUX>& f, int first, int last, V (&k)[L], V (&rest)[L]) {
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const V z = f.at(i);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      float a, r;
      sigmoid_both(z[j], a, r);
      k[i][j] = padded<FULL>(first, i, last) ? 1.0f : a;
      rest[i][j] = padded<FULL>(first, i, last) ? 0.0f : r;
    }
  }
}

template <int DT, int VEC, int L>
__device__ __forceinline__ void zero_steps(const Rows& r, int64_t b, int t0, int64_t sb, int first, uint32_t coff,
                                           bool live, int T) {
  const Block k(r, b, t0, sb);
  const uint32_t off = (uint32_t)first * k.time + coff;
#pragma unroll
  for (int i = 0; i < L; ++i)
    store<DT, VEC, kCached>(k, live && t0 + first + i < T ? off : kNowhere, i, (typename Pack<DT, VEC>::wide)0.0f);
}

// work: for each sequence and segment, the map that its state before the segment joins last: [B][segs][2][C].
// Slot 0 is (0, h0), slot s the map of segment s - 1 (forward); slot segs - 1 is (0, gh), slot s that of segment
// s + 1 (backward). So the second kernel reads no h0, which h_last may overwrite.
__device__ __forceinline__ float* slot_of(float* work, const Cut& k, int64_t b, int64_t s, int64_t C) {
  return work + ((b * k.segs + s) * 2) * C;
}

// The state (going backward: the carry) that `count` slots give from zero, slot first, first + by, ... in that
// order: each group joins a part of them, four loads of a slot's map at a time, and every thread the groups' maps.
template <int VEC, int W, int G>
__device__ __forceinline__ typename Pack<GS_F32, VEC>::wide join_slots(
    const float* slots, int64_t C, int first, int by, int count, int g, int lane,
    typename Pack<GS_F32, VEC>::wide (&maps)[G][W], typename Pack<GS_F32, VEC>::wide (&results)[G][W]) {
  using V = typename Pack<GS_F32, VEC>::wide;
  const int per = (count + G - 1) / G, end = (g + 1) * per < count ? (g + 1) * per : count;
  V A = (V)1.0f, S = (V)0.0f;
  for (int s0 = g * per; s0 < end; s0 += 4) {
    V a[4], b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + u < end) {
        const float* m = slots + (int64_t)(first + by * (s0 + u)) * 2 * C;
        a[u] = loadf<VEC>(m);
        b[u] = loadf<VEC>(m + C);
      }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + u < end) {
        A = A * a[u];
        S = join<VEC>(a[u], S, b[u]);
      }
  }
  maps[g][lane] = A;
  results[g][lane] = S;
  __syncthreads();
  V h = (V)0.0f;
#pragma unroll
  for (int s = 0; s < G; ++s) h = join<VEC>(maps[s][lane], h, results[s][lane]);
  __syncthreads();  // the blocks use the same memory
  return h;
}

template <int DT, int VEC, bool GATE, int W, int G, int L, bool REDUCE, int AUX>
__global__ void __launch_bounds__(W* G, G > 1 ? 4 : 1) k_recurrence_fwd(RecurrenceArgs a, Cut cut) {
  using V = typename Pack<GS_F32, VEC>::wide;
  constexpr int kSpan = G * L;
  __shared__ V maps[G > 1 ? 2 : 1][2][G][W];
  const Place p = place_of<(G > 1)>(cut, cut.segs - (REDUCE ? 1 : 0), 0, a.B);
  if (p.b >= a.B) return;
  const int lane = threadIdx.x % W, g = W == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / W) : threadIdx.x / W;
  const int64_t c0 = (int64_t)p.strip * (W * VEC);
  const bool live = c0 + lane * VEC < a.C;
  const int64_t c = live ? c0 + lane * VEC : a.C - VEC;  // for lanes past the last channel another one's state
  const int64_t sb = c0 * (int64_t)sizeof(typename Elem<DT>::type);
  const uint32_t off = (uint32_t)(lane * VEC) * (uint32_t)sizeof(typename Elem<DT>::type);
  const int n = length_of(a, p.b), T = (int)a.T;
  V h = (V)0.0f, prod = (V)1.0f;
  if (REDUCE) {
    if (p.seg == 0 && live && g == 0) {
      storef<VEC>(slot_of(a.work, cut, p.b, 0, a.C) + c, (V)0.0f);
      storef<VEC>(slot_of(a.work, cut, p.b, 0, a.C) + a.C + c, a.h0 ? loadf<VEC>(a.h0 + p.b * a.C + c) : (V)0.0f);
    }
  } else if (G > 1 && cut.segs > 1) {
    h = join_slots<VEC, W, G>(slot_of(a.work, cut, p.b, 0, a.C) + c, a.C, 0, 1, p.seg + 1, g, lane, maps[0][0], maps[0][1]);
  } else if (a.h0) {
    h = loadf<VEC>(a.h0 + p.b * a.C + c);
  }
  const int first = g * L;
  struct Loads {
    Steps<DT, VEC, L, AUX> x, f, o;
  };
  auto fetch = [&](auto full, int blk, int last) {
    constexpr bool FULL = decltype(full)::value;
    const int t0 = blk * kSpan;
    Loads m;
    m.f.template get<FULL>(Block(a.f, p.b, t0, sb), first, off, last, live);
    m.x.template get<FULL>(Block(a.x, p.b, t0, sb), first, off, last, live);
    if (GATE && !REDUCE) m.o.template get<FULL>(Block(a.o, p.b, t0, sb), first, off, last, live);
    return m;
  };
  auto block = [&](auto full, int blk, int last, const Loads& m) {
    constexpr bool FULL = decltype(full)::value;
    const int t0 = blk * kSpan;
    V k[L], in[L];
    gates<FULL>(m.f, first, last, k, in);
    V A = (V)1.0f, S = (V)0.0f;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      in[i] = in[i] * m.x.at(i);
      A = A * k[i];
      S = join<VEC>(k[i], S, in[i]);
    }
    V mine = h;
    if (G > 1) {
      const int buf = blk & 1;
      maps[buf][0][g][lane] = A;
      maps[buf][1][g][lane] = S;
      __syncthreads();
#pragma unroll
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
    if (REDUCE) return;
    if (first % GS_RECURRENCE_BLOCK == 0 && a.states && live && (FULL || first <= last))
      storef<VEC>(a.states + (p.b * cut.blocks + (t0 + first) / GS_RECURRENCE_BLOCK) * a.C + c, mine);
    const Block to(a.y, p.b, t0, sb);
    const uint32_t at = live ? (uint32_t)first * to.time + off : kNowhere;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      mine = join<VEC>(k[i], mine, in[i]);
      V out = mine;
      if (GATE) {
        const V z = m.o.at(i);
#pragma unroll
        for (int j = 0; j < VEC; ++j) out[j] = sigmoid_of(z[j]) * out[j];
      }
      if (padded<FULL>(first, i, last)) out = (V)0.0f;
      store<DT, VEC, kPast>(to, FULL || t0 + first + i < T ? at : kNowhere, i, out);
    }
  };
  // whole blocks, each one's loads under way while the one before is worked on; a last, part one; padding
  const int whole = n / kSpan < p.blk1 ? n / kSpan : p.blk1;
  int blk = p.blk0;
  if (blk < whole) {
    Loads now = fetch(std::true_type(), blk, kSpan - 1);
    for (; blk < whole; ++blk) {
      Loads next;
      if (blk + 1 < whole) next = fetch(std::true_type(), blk + 1, kSpan - 1);
      block(std::true_type(), blk, kSpan - 1, now);
      now = next;
    }
  }
  if (blk < p.blk1 && blk * kSpan < n) {
    const int last = n - blk * kSpan - 1;
    block(std::false_type(), blk, last, fetch(std::false_type(), blk, last));
    ++blk;
  }
  if (!REDUCE)
    for (; blk < p.blk1; ++blk) zero_steps<DT, VEC, L>(a.y, p.b, blk * kSpan, sb, first, off, live, T);
  if (g != 0 || !live) return;
  if (REDUCE) {
    float* m = slot_of(a.work, cut, p.b, p.seg + 1, a.C) + c;
    storef<VEC>(m, prod);
    storef<VEC>(m + a.C, h);
  } else if (p.seg == cut.segs - 1) {
    storef<VEC>(a.h_last + p.b * a.C + c, h);
  }
}

template <int DT, int VEC, bool GATE, int W, int G, int L, bool REDUCE, int AUX>
__global__ void __launch_bounds__(W* G, G == 4 ? 3 : G == 8 ? 2 : 1) k_recurrence_bwd(RecurrenceArgs a, Cut cut) {
  using V = typename Pack<GS_F32, VEC>::wide;
  constexpr int kSpan = G * L;
  __shared__ V maps[G > 1 ? 2 : 1][3][G][W];
  const Place p = place_of<(G > 1)>(cut, cut.segs - (REDUCE ? 1 : 0), REDUCE ? 1 : 0, a.B);
  if (p.b >= a.B) return;
  const int lane = threadIdx.x % W, g = W == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / W) : threadIdx.x / W;
  const int64_t c0 = (int64_t)p.strip * (W * VEC);
  const bool live = c0 + lane * VEC < a.C;
  const int64_t c = live ? c0 + lane * VEC : a.C - VEC;
  const int64_t sb = c0 * (int64_t)sizeof(typename Elem<DT>::type);
  const uint32_t off = (uint32_t)(lane * VEC) * (uint32_t)sizeof(typename Elem<DT>::type);
  const int n = length_of(a, p.b), T = (int)a.T;
  V carry = (V)0.0f, prod = (V)1.0f;
  if (REDUCE) {
    if (p.seg == cut.segs - 1 && live && g == 0) {
      float* m = slot_of(a.work, cut, p.b, cut.segs - 1, a.C) + c;
      storef<VEC>(m, (V)0.0f);
      storef<VEC>(m + a.C, a.gh ? loadf<VEC>(a.gh + p.b * a.C + c) : (V)0.0f);
    }
  } else if (G > 1 && cut.segs > 1) {
    carry = join_slots<VEC, W, G>(slot_of(a.work, cut, p.b, 0, a.C) + c, a.C, cut.segs - 1, -1, cut.segs - p.seg, g, lane,
                                  maps[0][0], maps[0][1]);
  } else if (a.gh) {
    carry = loadf<VEC>(a.gh + p.b * a.C + c);
  }
  const int first = g * L;
  struct Loads {
    Steps<DT, VEC, L, AUX> x, f, o, gy;
    V h;
  };
  auto fetch = [&](auto full, int blk, int last) {
    constexpr bool FULL = decltype(full)::value;
    const int t0 = blk * kSpan;
    Loads m;
    m.f.template get<FULL>(Block(a.f, p.b, t0, sb), first, off, last, live);
    m.gy.template get<FULL>(Block(a.gy, p.b, t0, sb), first, off, last, live);
    if (GATE) m.o.template get<FULL>(Block(a.o, p.b, t0, sb), first, off, last, live);
    if (!REDUCE) {
      m.x.template get<FULL>(Block(a.x, p.b, t0, sb), first, off, last, live);
      m.h = loadf<VEC>(a.states + (p.b * cut.blocks + t0 / GS_RECURRENCE_BLOCK) * a.C + c);
    }
    return m;
  };
  auto block = [&](auto full, int blk, int last, Loads& m) {
    constexpr bool FULL = decltype(full)::value;
    const int t0 = blk * kSpan;
    V h = REDUCE ? (V)0.0f : m.h;
    V k[L], rest[L], q[L], shut[L];  // shut: gy sigmoid(o) (1 - sigmoid(o)), the factor of h in do
    gates<FULL>(m.f, first, last, k, rest);
    V A = (V)1.0f, S = (V)0.0f, R = (V)0.0f;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      q[i] = m.gy.at(i);
      if (GATE) {
        const V z = m.o.at(i);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          if (REDUCE) {
            q[i][j] = q[i][j] * sigmoid_of(z[j]);
          } else {
            float s, r;
            sigmoid_both(z[j], s, r);
            q[i][j] = q[i][j] * s;
            shut[i][j] = q[i][j] * r;
          }
        }
      }
      A = A * k[i];
      if (!REDUCE) S = join<VEC>(k[i], S, rest[i] * m.x.at(i));
    }
#pragma unroll
    for (int i = L - 1; i >= 0; --i) R = k[i] * (q[i] + R);
    if (!REDUCE) {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        pin(k[i]);
        pin(rest[i]);
        if (GATE) pin(shut[i]);
      }
    }
    V c_in = carry;
    if (G > 1) {
      const int buf = blk & 1;
      maps[buf][0][g][lane] = A;
      maps[buf][1][g][lane] = R;
      if (!REDUCE) maps[buf][2][g][lane] = S;
      __syncthreads();
      V hs = h;
#pragma unroll
      for (int s = 0; s < G; ++s) {
        const int r = G - 1 - s;
        if (r == g) c_in = carry;
        const V Ar = maps[buf][0][r][lane];
        carry = join<VEC>(Ar, carry, maps[buf][1][r][lane]);
        if (REDUCE) {
          prod = prod * Ar;
        } else {
          if (s == g) h = hs;
          hs = join<VEC>(maps[buf][0][s][lane], hs, maps[buf][2][s][lane]);
        }
      }
    } else {
      carry = join<VEC>(A, carry, R);
      if (REDUCE) prod = prod * A;
    }
    if (REDUCE) return;
#pragma unroll
    for (int i = 0; i < L; ++i) pin(m.x.v[i]);
#pragma unroll
    for (int i = L - 1; i >= 0; --i) {  // q becomes s
      q[i] = q[i] + c_in;
      c_in = k[i] * q[i];
    }
    const Block to_x(a.dx, p.b, t0, sb), to_f(a.df, p.b, t0, sb), to_o(a.dout, p.b, t0, sb);
    const uint32_t at_x = live ? (uint32_t)first * to_x.time + off : kNowhere;
    const uint32_t at_f = live ? (uint32_t)first * to_f.time + off : kNowhere;
    const uint32_t at_o = live ? (uint32_t)first * to_o.time + off : kNowhere;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const V xi = m.x.at(i);
      V dx = rest[i] * q[i], df = (dx * k[i]) * (h - xi);
      h = join<VEC>(k[i], h, rest[i] * xi);
      V dout = GATE ? shut[i] * h : (V)0.0f;
      if (padded<FULL>(first, i, last)) dx = df = dout = (V)0.0f;  // rest and shut are 0, but h or s may be infinite or NaN
      const bool in = FULL || t0 + first + i < T;
      store<DT, VEC, AUX>(to_x, in ? at_x : kNowhere, i, dx);
      store<DT, VEC, AUX>(to_f, in ? at_f : kNowhere, i, df);
      if (GATE) store<DT, VEC, AUX>(to_o, in ? at_o : kNowhere, i, dout);
    }
  };
  int blk = p.blk1 - 1;
  if (!REDUCE) {
    for (; blk >= p.blk0 && blk * kSpan >= n; --blk) {
      zero_steps<DT, VEC, L>(a.dx, p.b, blk * kSpan, sb, first, off, live, T);
      zero_steps<DT, VEC, L>(a.df, p.b, blk * kSpan, sb, first, off, live, T);
      if (GATE) zero_steps<DT, VEC, L>(a.dout, p.b, blk * kSpan, sb, first, off, live, T);
    }
  } else if (blk * kSpan >= n) {
    blk = (n + kSpan - 1) / kSpan - 1;
  }
  if (blk >= p.blk0 && (blk + 1) * kSpan > n) {
    const int last = n - blk * kSpan - 1;
    Loads m = fetch(std::false_type(), blk, last);
    block(std::false_type(), blk, last, m);
    --blk;
  }
  if (blk >= p.blk0) {
    Loads now = fetch(std::true_type(), blk, kSpan - 1);
    for (; blk >= p.blk0; --blk) {
      Loads next;
      if (blk > p.blk0) next = fetch(std::true_type(), blk - 1, kSpan - 1);
      block(std::true_type(), blk, kSpan - 1, now);
      now = next;
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

constexpr int kSteps = 8;           // of a thread
constexpr int kChip = 256;          // workgroups that give every CU one
constexpr int kMaxSegs = 512;

// How a direction is cut. Single tokens and up to eight steps need no groups; more steps take eight groups a workgroup.
// Up to one workgroup a CU the forward pass takes sixteen, for more waves on each (16 x 4,096 x 2,048 bf16, 256
// workgroups: 223 us with eight, 210 with sixteen; 32 x 512 x 1,500, 384: 56 and 60). The backward pass needs 1.6 times
// the registers and takes four where that still gives the CUs more than one workgroup each (256 workgroups:
// 490 us with four, 412 with eight). At most half a workgroup a CU: time is split to two a CU, which costs reading
// two or three arrays twice (1 x 65,536 x 1,024, both directions: 405 us with two a CU, 441 with four), to four where a
// segment would be shorter than eight blocks (5 x 1,037 x 1,500 fp16: 34 us with two a CU, 27 with four). Few steps are
// done in one kernel all the same (1 x 832, both directions: 200 steps 28 us whole, 37 split, 400 steps 48 and 36).
Cut cut_of(int64_t B, int64_t T, int64_t C, int vec, bool backward) {
  Cut k{};
  k.strips = (unsigned)((C + 64 * vec - 1) / (64 * vec));
  k.blocks = (int)GS_RECURRENCE_BLOCKS(T);
  k.segs = 1;
  const int64_t have = B * (int64_t)k.strips;
  const bool split = T > GS_RECURRENCE_WHOLE && 2 * have <= kChip;
  if (T <= kSteps)
    k.groups = 1;
  else if (backward)
    k.groups = split || 4 * have > 5 * kChip ? 4 : 8;
  else
    k.groups = split || have > kChip ? 8 : 16;
  const int64_t span = T <= 1 ? 1 : k.groups * kSteps;
  k.all = (int)((T + span - 1) / span);
  k.seg_blocks = k.all;
  if (split && k.all > 1) {
    int64_t segs = 2 * kChip / have;
    if (k.all < 8 * segs) segs *= 2;
    segs = segs < k.all ? segs : k.all;
    segs = segs < kMaxSegs ? segs : kMaxSegs;
    k.seg_blocks = (int)((k.all + segs - 1) / segs);
    k.segs = (k.all + k.seg_blocks - 1) / k.seg_blocks;
  }
  return k;
}

template <int DT, int VEC, bool GATE, bool REDUCE>
void forward(hipStream_t s, const RecurrenceArgs& a, const Cut& k, dim3 grid, bool lines) {
  if (a.T <= 1)
    k_recurrence_fwd<DT, VEC, GATE, 64, 1, 1, false, kCached><<<grid, 64, 0, s>>>(a, k);
  else if (k.groups == 1)
    k_recurrence_fwd<DT, VEC, GATE, 64, 1, kSteps, false, kCached><<<grid, 64, 0, s>>>(a, k);
  else if (k.groups == 16 && lines)
    k_recurrence_fwd<DT, VEC, GATE, 64, 16, kSteps, false, kPast><<<grid, 1024, 0, s>>>(a, k);
  else if (k.groups == 16)
    k_recurrence_fwd<DT, VEC, GATE, 64, 16, kSteps, false, kCached><<<grid, 1024, 0, s>>>(a, k);
  else if (lines)
    k_recurrence_fwd<DT, VEC, GATE, 64, 8, kSteps, REDUCE, kPast><<<grid, 512, 0, s>>>(a, k);
  else
    k_recurrence_fwd<DT, VEC, GATE, 64, 8, kSteps, REDUCE, kCached><<<grid, 512, 0, s>>>(a, k);
}

template <int DT, int VEC, bool GATE, bool REDUCE>
void backward(hipStream_t s, const RecurrenceArgs& a, const Cut& k, dim3 grid, bool lines) {
  if (a.T <= 1)
    k_recurrence_bwd<DT, VEC, GATE, 64, 1, 1, false, kCached><<<grid, 64, 0, s>>>(a, k);
  else if (k.groups == 1)
    k_recurrence_bwd<DT, VEC, GATE, 64, 1, kSteps, false, kCached><<<grid, 64, 0, s>>>(a, k);
  else if (k.groups == 8 && lines)
    k_recurrence_bwd<DT, VEC, GATE, 64, 8, kSteps, false, kPast><<<grid, 512, 0, s>>>(a, k);
  else if (k.groups == 8)
    k_recurrence_bwd<DT, VEC, GATE, 64, 8, kSteps, false, kCached><<<grid, 512, 0, s>>>(a, k);
  else if (lines)
    k_recurrence_bwd<DT, VEC, GATE, 64, 4, kSteps, REDUCE, kPast><<<grid, 256, 0, s>>>(a, k);
  else
    k_recurrence_bwd<DT, VEC, GATE, 64, 4, kSteps, REDUCE, kCached><<<grid, 256, 0, s>>>(a, k);
}

// strips x parts x B is below 2^31: the [B][C] states of that many workgroups do not fit any memory.
dim3 grid_of(const Cut& k, int parts, int64_t B) {
  const int64_t n = (int64_t)k.strips * parts * B;
  return dim3((unsigned)(n < kGridX ? n : kGridX), (unsigned)((n + kGridX - 1) / kGridX));
}

// Two channels a lane for 16-bit elements, where every row of every array starts on a pair of them and one channel a
// lane would leave a second strip to do. fp32 takes one: two need twice the registers for loads (8 x 4,096 x
// 2,048: 191 + 72 and 423 + 98 us with two, 194 and 390 with one).
bool in_pairs(int dtype, int64_t C) { return dtype != GS_F32 && C % 2 == 0 && C > 64; }

bool pairs(const Rows& r, int bytes) {
  const int64_t m = 2 * bytes - 1;
  return ((uintptr_t)r.p & m) == 0 && (r.batch & m) == 0 && (r.time & m) == 0;
}

// Every row of every step starts on a 128-byte line.
bool lines(const Rows& r) { return (((uintptr_t)r.p | r.batch | r.time) & 127) == 0; }

bool pairs(const float* p) { return ((uintptr_t)p & 7) == 0; }

// Calls f with the element type, the channels of a lane and whether there is an output gate as constants.
template <typename F>
void with_type(int dtype, bool two, bool gate, F f) {
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  auto g = [&](auto dt, auto vec) { gate ? f(dt, vec, std::true_type()) : f(dt, vec, std::false_type()); };
  const std::integral_constant<int, GS_F32> f32;
  const std::integral_constant<int, GS_BF16> bf16;
  const std::integral_constant<int, GS_F16> f16;
  if (dtype == GS_F32) g(f32, One());
  if (dtype == GS_BF16) two ? g(bf16, Two()) : g(bf16, One());
  if (dtype == GS_F16) two ? g(f16, Two()) : g(f16, One());
}

}  // namespace

// For each sequence and segment one map; more segments where a lane takes two channels.
int64_t recurrence_work(int64_t B, int64_t T, int64_t C, int dtype) {
  if (B == 0 || T == 0 || C == 0) return 0;
  const int vec = in_pairs(dtype, C) ? 2 : 1;
  const int f = cut_of(B, T, C, vec, false).segs, b = cut_of(B, T, C, vec, true).segs, segs = f > b ? f : b;
  return segs > 1 ? B * segs * 2 * C * (int64_t)sizeof(float) : 0;
}

hipError_t launch_recurrence_forward(hipStream_t s, int dtype, const RecurrenceArgs& a) {
  const int bytes = elem_size(dtype);
  const bool two = in_pairs(dtype, a.C) && (a.T == 0 || (pairs(a.x, bytes) && pairs(a.f, bytes) && pairs(a.y, bytes) &&
                                                 (!a.o.p || pairs(a.o, bytes)))) &&
                   pairs(a.h0) && pairs(a.h_last) && pairs(a.states) && pairs(a.work);
  const Cut k = cut_of(a.B, a.T, a.C, two ? 2 : 1, false);
  const bool whole = lines(a.x) && lines(a.f) && lines(a.o);
  with_type(dtype, two, a.o.p != nullptr, [&](auto dt, auto vec, auto gate) {
    constexpr int DT = decltype(dt)::value, VEC = decltype(vec)::value;
    constexpr bool GATE = decltype(gate)::value;
    if (k.segs > 1) forward<DT, VEC, false, true>(s, a, k, grid_of(k, k.segs - 1, a.B), whole);
    forward<DT, VEC, GATE, false>(s, a, k, grid_of(k, k.segs, a.B), whole);
  });
  return hipGetLastError();
}

hipError_t launch_recurrence_backward(hipStream_t s, int dtype, const RecurrenceArgs& a) {
  const int bytes = elem_size(dtype);
  const bool two = in_pairs(dtype, a.C) &&
                   (a.T == 0 || (pairs(a.x, bytes) && pairs(a.f, bytes) && pairs(a.gy, bytes) && pairs(a.dx, bytes) &&
                                 pairs(a.df, bytes) && (!a.o.p || (pairs(a.o, bytes) && pairs(a.dout, bytes))))) &&
                   pairs(a.gh) && pairs(a.dh0) && pairs(a.states) && pairs(a.work);
  const Cut k = cut_of(a.B, a.T, a.C, two ? 2 : 1, true);
  const bool whole = lines(a.x) && lines(a.f) && lines(a.o) && lines(a.gy) && lines(a.dx) && lines(a.df) && lines(a.dout);
  with_type(dtype, two, a.o.p != nullptr, [&](auto dt, auto vec, auto gate) {
    constexpr int DT = decltype(dt)::value, VEC = decltype(vec)::value;
    constexpr bool GATE = decltype(gate)::value;
    if (k.segs > 1) backward<DT, VEC, GATE, true>(s, a, k, grid_of(k, k.segs - 1, a.B), whole);
    backward<DT, VEC, GATE, false>(s, a, k, grid_of(k, k.segs, a.B), whole);
  });
  return hipGetLastError();
}

}  // namespace gs
