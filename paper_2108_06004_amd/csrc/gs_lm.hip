// gs_lm.hip -- the C ABI of the language-model operators (include/gs.h): argument checks, then the
// launchers of k_recurrence.hip, k_dropout.hip and k_cross_entropy.hip.
#include <cmath>
#include <cstdio>

#include "gs_internal.hpp"
#include "gs_lm.hpp"

namespace {

gs_status refuse(gs_status st, const char* call, const char* what) {
  char buf[256];
  std::snprintf(buf, sizeof buf, "%s: %s", call, what);
  gs::set_free_error(buf);
  return st;
}

gs_status launched(hipError_t e, const char* call) {
  return e == hipSuccess ? GS_OK : refuse(GS_ERR_DEVICE, call, hipGetErrorString(e));
}

bool known(int dtype) { return dtype == GS_F32 || dtype == GS_BF16 || dtype == GS_F16; }

bool aligned(const void* p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// One [B][T][C] argument: what is wrong with it, or NULL.
const char* wrong_rows(const gs_rows& a, const gs_recurrence& r, int bytes) {
  if (!a.data) return "NULL array";
  if (!aligned(a.data, bytes)) return "an array is not aligned to its elements";
  if (a.batch < 0 || a.time < 0) return "strides must not be negative";
  return nullptr;
}

gs::Rows rows_of(const gs_rows& a, int bytes) {
  return gs::Rows{static_cast<char*>(a.data), a.batch * bytes, a.time * bytes};
}

// The checks that both directions share. *empty: there is no element to compute.
gs_status check_recurrence(const gs_recurrence* r, const char* call, bool* empty) {
  if (!r) return refuse(GS_ERR_INVALID_ARG, call, "r is NULL");
  if (r->B < 0 || r->T < 0 || r->C < 0) return refuse(GS_ERR_INVALID_ARG, call, "sizes must not be negative");
  if (!known(r->dtype)) return refuse(GS_ERR_INVALID_ARG, call, "dtype must be GS_F32, GS_BF16 or GS_F16");
  if (r->B > gs::kMaxSteps || r->T > gs::kMaxSteps || r->C > GS_RECURRENCE_MAX_CHANNELS)
    return refuse(GS_ERR_UNSUPPORTED, call, "B and T must be at most 2^30, C at most GS_RECURRENCE_MAX_CHANNELS");
  *empty = r->B == 0 || r->C == 0;
  if (*empty) return GS_OK;
  if (!aligned(r->lengths, 4) || !aligned(r->h0, 4))
    return refuse(GS_ERR_INVALID_ARG, call, "an array is not aligned to its elements");
  return GS_OK;
}

gs_status check_rows(const gs_recurrence& r, const char* call, const gs_rows* const* a, int n) {
  for (int j = 0; j < n; ++j) {
    if (const char* w = wrong_rows(*a[j], r, gs::elem_size(r.dtype))) return refuse(GS_ERR_INVALID_ARG, call, w);
    if (r.T > 1 && a[j]->time > GS_RECURRENCE_MAX_STRIDE)
      return refuse(GS_ERR_UNSUPPORTED, call, "a time stride is over GS_RECURRENCE_MAX_STRIDE elements");
  }
  return GS_OK;
}

gs::RecurrenceArgs recurrence_args(const gs_recurrence& r, void* work) {
  const int bytes = gs::elem_size(r.dtype);
  gs::RecurrenceArgs a{};
  a.B = r.B;
  a.T = r.T;
  a.C = r.C;
  a.x = rows_of(r.x, bytes);
  a.f = rows_of(r.f, bytes);
  a.o = rows_of(r.o, bytes);
  a.lengths = r.lengths;
  a.h0 = r.h0;
  a.work = static_cast<float*>(work);
  return a;
}

}  // namespace

extern "C" {

int64_t gs_recurrence_work(int64_t B, int64_t T, int64_t C, int32_t dtype) {
  if (B < 0 || T < 0 || C < 0 || !known(dtype)) return -1;
  if (B > gs::kMaxSteps || T > gs::kMaxSteps || C > GS_RECURRENCE_MAX_CHANNELS) return -1;
  return gs::recurrence_work(B, T, C, dtype);
}

gs_status gs_recurrence_forward(const gs_recurrence* r, void* stream, gs_rows y, float* h_last, float* states,
                                void* work) {
  const char* call = "gs_recurrence_forward";
  gs::set_free_error("");
  bool empty = false;
  gs_status st = check_recurrence(r, call, &empty);
  if (st != GS_OK || empty) return st;
  if (!h_last) return refuse(GS_ERR_INVALID_ARG, call, "h_last is NULL");
  if (!aligned(h_last, 4) || !aligned(states, 4) || !aligned(work, 4))
    return refuse(GS_ERR_INVALID_ARG, call, "an array is not aligned to its elements");
  if (r->T > 0) {
    const gs_rows* used[] = {&r->x, &r->f, &y, &r->o};
    st = check_rows(*r, call, used, r->o.data ? 4 : 3);
    if (st != GS_OK) return st;
  }
  if (!work && gs::recurrence_work(r->B, r->T, r->C, r->dtype) > 0)
    return refuse(GS_ERR_INVALID_ARG, call, "work is NULL and gs_recurrence_work is not 0");
  gs::RecurrenceArgs a = recurrence_args(*r, work);
  a.y = rows_of(y, gs::elem_size(r->dtype));
  a.h_last = h_last;
  a.states = states;
  return launched(gs::launch_recurrence_forward(reinterpret_cast<hipStream_t>(stream), r->dtype, a), call);
}

gs_status gs_recurrence_backward(const gs_recurrence* r, void* stream, gs_rows gy, const float* gh,
                                 const float* states, gs_rows dx, gs_rows df, gs_rows dout, float* dh0, void* work) {
  const char* call = "gs_recurrence_backward";
  gs::set_free_error("");
  bool empty = false;
  gs_status st = check_recurrence(r, call, &empty);
  if (st != GS_OK || empty) return st;
  if (!aligned(gh, 4) || !aligned(states, 4) || !aligned(dh0, 4) || !aligned(work, 4))
    return refuse(GS_ERR_INVALID_ARG, call, "an array is not aligned to its elements");
  if (r->T > 0) {
    if (!states) return refuse(GS_ERR_INVALID_ARG, call, "states is NULL");
    if ((r->o.data != nullptr) != (dout.data != nullptr))
      return refuse(GS_ERR_INVALID_ARG, call, "dout goes with o: both or neither");
    const gs_rows* used[] = {&r->x, &r->f, &gy, &dx, &df, &r->o, &dout};
    st = check_rows(*r, call, used, r->o.data ? 7 : 5);
    if (st != GS_OK) return st;
  }
  if (!work && gs::recurrence_work(r->B, r->T, r->C, r->dtype) > 0)
    return refuse(GS_ERR_INVALID_ARG, call, "work is NULL and gs_recurrence_work is not 0");
  const int bytes = gs::elem_size(r->dtype);
  gs::RecurrenceArgs a = recurrence_args(*r, work);
  a.gy = rows_of(gy, bytes);
  a.dx = rows_of(dx, bytes);
  a.df = rows_of(df, bytes);
  a.dout = rows_of(dout, bytes);
  a.gh = gh;
  a.dh0 = dh0;
  a.states = const_cast<float*>(states);
  return launched(gs::launch_recurrence_backward(reinterpret_cast<hipStream_t>(stream), r->dtype, a), call);
}

gs_status gs_dropout(void* stream, int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride,
                     const void* residual, int64_t res_stride, void* y, int64_t y_stride, double p, uint64_t seed,
                     uint64_t site, const int64_t* step) {
  const char* call = "gs_dropout";
  gs::set_free_error("");
  if (!known(dtype)) return refuse(GS_ERR_INVALID_ARG, call, "dtype must be GS_F32, GS_BF16 or GS_F16");
  if (rows < 0 || cols < 0) return refuse(GS_ERR_INVALID_ARG, call, "sizes must not be negative");
  if (!(p >= 0.0 && p <= 1.0)) return refuse(GS_ERR_INVALID_ARG, call, "p must be in [0, 1]");
  if (!aligned(step, 8)) return refuse(GS_ERR_INVALID_ARG, call, "step is not aligned to its element");
  if (rows == 0 || cols == 0) return GS_OK;
  if (rows > INT64_MAX / 4 / cols) return refuse(GS_ERR_UNSUPPORTED, call, "rows * cols is over 2^61");
  const int bytes = gs::elem_size(dtype);
  if (!x || !y) return refuse(GS_ERR_INVALID_ARG, call, "NULL array");
  if (!aligned(x, bytes) || !aligned(y, bytes) || !aligned(residual, bytes))
    return refuse(GS_ERR_INVALID_ARG, call, "an array is not aligned to its elements");
  if (rows > 1 && (x_stride < cols || y_stride < cols || (residual && res_stride < cols)))
    return refuse(GS_ERR_INVALID_ARG, call, "row strides must be at least cols");
  gs::DropoutArgs a{};
  a.rows = rows;
  a.cols = cols;
  a.x = static_cast<const char*>(x);
  a.res = static_cast<const char*>(residual);
  a.y = static_cast<char*>(y);
  a.xs = x_stride;
  a.rs = residual ? res_stride : x_stride;
  a.ys = y_stride;
  a.below = (uint32_t)std::floor(p * 65536.0 + 0.5);
  a.factor = a.below < 65536u ? (float)(65536.0 / (65536.0 - a.below)) : 0.0f;
  a.seed = seed;
  a.site = site;
  a.step = step;
  return launched(gs::launch_dropout(reinterpret_cast<hipStream_t>(stream), dtype, a), call);
}

int64_t gs_cross_entropy_work(int64_t N, int64_t V, int32_t dtype) {
  if (N < 0 || V < 0 || !known(dtype)) return -1;
  return gs::cross_entropy_work(N, V, dtype);
}

gs_status gs_cross_entropy(const gs_xent* x, void* stream) {
  const char* call = "gs_cross_entropy";
  gs::set_free_error("");
  if (!x) return refuse(GS_ERR_INVALID_ARG, call, "x is NULL");
  if (!known(x->dtype)) return refuse(GS_ERR_INVALID_ARG, call, "dtype must be GS_F32, GS_BF16 or GS_F16");
  if (x->N < 0 || x->V < 0) return refuse(GS_ERR_INVALID_ARG, call, "sizes must not be negative");
  if (x->N > gs::kMaxExtent || x->V > gs::kMaxExtent)
    return refuse(GS_ERR_UNSUPPORTED, call, "N and V must be at most 2^31 - 1");
  if (x->N > 0 && x->V == 0) return refuse(GS_ERR_INVALID_ARG, call, "rows without logits");
  if (x->scale_stride != 0 && x->scale_stride != 1)
    return refuse(GS_ERR_INVALID_ARG, call, "scale_stride must be 0 or 1");
  if (!aligned(x->mean_loss, 4) || !aligned(x->losses, 4) || !aligned(x->scale, 4) || !aligned(x->work, 8) ||
      !aligned(x->targets, 8))
    return refuse(GS_ERR_INVALID_ARG, call, "an array is not aligned to its elements");
  if (x->N > 0) {
    const int bytes = gs::elem_size(x->dtype);
    if (!x->logits || !x->targets || (x->mean_loss && !x->losses)) return refuse(GS_ERR_INVALID_ARG, call, "NULL array");
    if (!aligned(x->logits, bytes) || !aligned(x->grad, bytes))
      return refuse(GS_ERR_INVALID_ARG, call, "an array is not aligned to its elements");
    if (x->N > 1 && (x->logits_stride < x->V || (x->grad && x->grad_stride < x->V)))
      return refuse(GS_ERR_INVALID_ARG, call, "row strides must be at least V");
  }
  if (!x->work && (x->N > 0 || x->mean_loss) && gs::cross_entropy_work(x->N, x->V, x->dtype) > 0)
    return refuse(GS_ERR_INVALID_ARG, call, "work is NULL and gs_cross_entropy_work is not 0");
  return launched(gs::launch_cross_entropy(reinterpret_cast<hipStream_t>(stream), *x), call);
}

}  // extern "C"
