// Distillation from the largest logits of a row's teachers: the loss, its gradient, and both in one launch.
//
// Mathematics.  loss = sum over the listed tokens of t (ln t - s/T) + P lse(s/T), so beside the student's normaliser the loss takes the listed tokens alone
// (both relative to the student's largest logit);
// the gradient is P q everywhere, with t taken off at the listed tokens.  Shares of a token that comes up more than once are added by the first of its
// entries, in order, so results do not depend on timing.
//
// Bound by memory: the loss reads the student once, the gradient reads it and writes as much; the launch with both keeps a row in the shared memory of a
// cluster of blocks between the normaliser and the gradient, and reads it once.  Exponentials are 32-bit (2^-22) and sums of them 64-bit; shares, logarithms and
// the loss are 64-bit; the gradient is rounded once.
#include <cuda_bf16.h>

#include "cos_slice.cuh"

namespace cosv {
namespace {

struct DistillParams {
  const char* student;
  long long stride;
  int rows, V, parts, share, seg, res;
  int lists, k;
  const int* ids;
  const float* values;
  const float* lse;
  float w[COS_MAX_MODELS];
  float T;
  const float* row_weights;
  float* loss;
  float2* statistics;
  char* grad;
  long long stride_grad;
};

// The listed tokens of a row that lie in this block's slice, each once.
struct Shares {
  int id[COS_TOP_MAX];
  double t[COS_TOP_MAX];
  double warp[kSliceWarps];
  int bad;
  double list_max[COS_MAX_MODELS], list_sum[COS_MAX_MODELS];
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ double block_sum(double v, double* per_warp) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) per_warp[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < kSliceWarps; ++w) s += per_warp[w];
  __syncthreads();
  return s;
}

// Every entry's share to shared memory (0 for an empty one); returns their sum, NaN where an entry names no token.
__device__ __forceinline__ double row_shares(const DistillParams& p, int row, Shares& sh) {
  const int n = p.lists * p.k, tid = threadIdx.x;
  const int* ids = p.ids + static_cast<long long>(row) * n;
  const float* values = p.values + static_cast<long long>(row) * n;
  const double inv_T = 1.0 / static_cast<double>(p.T);
  if (!p.lse) {  // softmax over each list: a warp for each
    const int g = tid >> 5;
    if (g < p.lists) {
      double m = -INFINITY, s = 0.0;
      for (int i = tid & 31; i < p.k; i += 32)
        if (ids[g * p.k + i] >= 0) m = fmax(m, static_cast<double>(values[g * p.k + i]));
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) m = fmax(m, __shfl_xor_sync(0xffffffffu, m, d));
      for (int i = tid & 31; i < p.k; i += 32)
        if (ids[g * p.k + i] >= 0 && values[g * p.k + i] != -INFINITY) s += exp((static_cast<double>(values[g * p.k + i]) - m) * inv_T);
      s = warp_sum(s);
      if ((tid & 31) == 0) {
        sh.list_max[g] = m;
        sh.list_sum[g] = s;
      }
    }
    __syncthreads();
  }
  double mine = 0.0;
  for (int e = tid; e < n; e += kSliceThreads) {
    const int id = ids[e], g = e / p.k;
    const float v = values[e];
    double t = 0.0;
    if (id >= 0 && v != -INFINITY) {
      const double w = static_cast<double>(p.w[g]);
      if (p.lse)
        t = w * exp(static_cast<double>(v) * inv_T - static_cast<double>(p.lse[static_cast<long long>(row) * p.lists + g]));
      else
        t = w * (exp((static_cast<double>(v) - sh.list_max[g]) * inv_T) / sh.list_sum[g]);
      if (id >= p.V) t = __longlong_as_double(0x7ff8000000000000ll);
    }
    sh.id[e] = id;
    sh.t[e] = t;
    mine += t;
  }
  return block_sum(mine, sh.warp);
}

// f(token, its whole share) for the listed tokens of the slice with a share, by whichever thread has the first entry.
template <int DT, class F>
__device__ __forceinline__ void each_listed(const DistillParams& p, const RowSlice<DT>& s, const Shares& sh, F&& f) {
  const int n = p.lists * p.k;
  const int lo = max(0, s.token(0)), hi = min(p.V, s.token(s.nv));
  for (int e = threadIdx.x; e < n; e += kSliceThreads) {
    const int id = sh.id[e];
    if (id < lo || id >= hi) continue;
    double t = 0.0;
    bool first = true;
    for (int j = 0; j < n; ++j)
      if (sh.id[j] == id) {
        first = first && j >= e;
        t += sh.t[j];
      }
    if (first && t != 0.0) f(id, t);
  }
}

template <int DT>
__device__ __forceinline__ float student_at(const char* row, int x) {
  return Elem<DT>::load1(row, x);
}

template <int DT>
__device__ __forceinline__ void store_entry(char* row, int x, float v) {
  if (DT == COS_DTYPE_F32)
    reinterpret_cast<float*>(row)[x] = v;
  else if (DT == COS_DTYPE_BF16)
    reinterpret_cast<__nv_bfloat16*>(row)[x] = __float2bfloat16_rn(v);
  else
    reinterpret_cast<__half*>(row)[x] = __float2half_rn(v);
}

template <int DT>
__device__ __forceinline__ uint4 packed(const float (&v)[Elem<DT>::E]) {
  uint4 r;
  unsigned* w = reinterpret_cast<unsigned*>(&r);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (DT == COS_DTYPE_F32) {
      w[k] = __float_as_uint(v[k]);
    } else if constexpr (DT == COS_DTYPE_BF16) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
      w[k] = *reinterpret_cast<const unsigned*>(&h);
    } else {
      const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
      w[k] = *reinterpret_cast<const unsigned*>(&h);
    }
  }
  return r;
}

// The slice of the gradient: f(values) in place of the values.
template <int DT, class F>
__device__ __forceinline__ void write_slice(const RowSlice<DT>& s, char* row, bool read, F&& f) {
  constexpr int E = Elem<DT>::E, B = Elem<DT>::bytes;
  const bool whole = static_cast<int>(reinterpret_cast<unsigned long long>(row) & 15) / B == s.off;
  for (int i = s.begin + (threadIdx.x & 31); i < s.end; i += 32) {
    float v[E] = {};
    if (read) Elem<DT>::unpack(s.at(i), v);
    f(v);
    const int x = s.token(i);
    if (whole && x >= 0 && x <= s.V - E) {
      *reinterpret_cast<uint4*>(row + static_cast<long long>(x) * B) = packed<DT>(v);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (x + e >= 0 && x + e < s.V) store_entry<DT>(row, x + e, v[e]);
    }
  }
}

// A part of a softmax normaliser: a sum of powers of two relative to the largest logit seen.
struct Part {
  float m;
  double sum;
  // a vector (NaN makes both NaN, +inf the sum)
  template <int E>
  __device__ __forceinline__ void add(const float (&v)[E], float c) {
    float top = v[0];
#pragma unroll
    for (int e = 1; e < E; ++e) top = max_nan(top, v[e]);
    if (top > m || top != top) {  // (a maximum that is NaN stays it)
      sum *= static_cast<double>(m == -INFINITY ? 0.0f : ex2_approx((m - top) * c));
      m = top;
    }
    if (m == -INFINITY) return;
    float part = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) part += ex2_approx((v[e] - m) * c);
    sum += static_cast<double>(part);
  }
};

struct Keep {
  __device__ __forceinline__ u64 operator()(u64 a, u64) const { return a; }
};

constexpr int kLoss = 0, kGrad = 1, kStep = 2;

template <int DT, int MODE>
__global__ void __launch_bounds__(kSliceThreads, 2) cos_distill_kernel(const DistillParams p) {
  extern __shared__ uint4 smem[];
  __shared__ Shares sh;
  __shared__ Exchange x;
  constexpr bool kCluster = MODE != kGrad;
  constexpr int E = Elem<DT>::E;
  const int parts = p.parts, rank = blockIdx.x % parts, row = blockIdx.x / parts, tid = threadIdx.x;
  const bool wide = kCluster && parts > 1;
  if (wide) cluster_barrier_arrive();
  int turn = 0;
  const char* student = p.student + static_cast<long long>(row) * p.stride * Elem<DT>::bytes;
  char* grad = MODE != kLoss ? p.grad + static_cast<long long>(row) * p.stride_grad * Elem<DT>::bytes : nullptr;
  RowSlice<DT> s;
  s.init(student, p.V, rank, p.share, p.seg, smem, p.res);
  const float weight = MODE != kLoss ? p.row_weights[row] : 1.0f;
  const double mass = row_shares(p, row, sh);  // (the same in every block)
  const float nan = __int_as_float(0x7fc00000);

  if (!(mass != 0.0) || (MODE == kGrad && weight == 0.0f)) {  // nothing to learn from
    if (MODE != kGrad && rank == 0 && tid == 0) {
      p.loss[row] = 0.0f;
      if (MODE == kLoss) p.statistics[row] = make_float2(0.0f, 0.0f);
    }
    if (MODE != kLoss) write_slice<DT>(s, grad, false, [](float (&)[E]) {});
    if (wide) cluster_barrier_wait();
    return;
  }

  const float c = fminf(static_cast<float>(1.4426950408889634 / static_cast<double>(p.T)), 3e38f);
  float m, log_z;
  if constexpr (MODE != kGrad) {
    Part part = {-INFINITY, 0.0};
    s.load([&](const float (&v)[E]) { part.add(v, c); });
    if (wide) cluster_barrier_wait();
    const auto larger = [](u64 a, u64 b) {
      return static_cast<u64>(__float_as_uint(max_nan(__uint_as_float(static_cast<unsigned>(a)), __uint_as_float(static_cast<unsigned>(b)))));
    };
    const auto add = [](u64 a, u64 b) {
      return static_cast<u64>(__double_as_longlong(__longlong_as_double(static_cast<long long>(a)) + __longlong_as_double(static_cast<long long>(b))));
    };
    m = __uint_as_float(static_cast<unsigned>(exchange(x, turn, parts, rank, __float_as_uint(part.m), 0, larger, Keep()).a));
    // of the listed tokens, relative to the largest logit: t (ln t - (s - m) / T)
    double listed = 0.0;
    each_listed(p, s, sh, [&](int id, double t) { listed += t * (log(t) - (static_cast<double>(student_at<DT>(student, id)) - static_cast<double>(m)) / static_cast<double>(p.T)); });
    const double mine = part.m == -INFINITY ? 0.0 : part.sum * static_cast<double>(ex2_approx((part.m - m) * c));
    const Words sums = exchange(x, turn, parts, rank, static_cast<u64>(__double_as_longlong(mine)), static_cast<u64>(__double_as_longlong(listed)), add, add);
    const double z = __longlong_as_double(static_cast<long long>(sums.a));
    log_z = m == -INFINITY ? nan : static_cast<float>(log2(z));
    if (rank == 0 && tid == 0) {
      p.loss[row] = m == -INFINITY ? nan : static_cast<float>(__longlong_as_double(static_cast<long long>(sums.b)) + mass * log(z));
      if (MODE == kLoss) p.statistics[row] = make_float2(m, log_z);
    }
  } else {
    const float2 st = p.statistics[row];
    m = st.x;
    log_z = st.y;
  }
  if constexpr (MODE != kLoss) {
    if (MODE == kStep && weight == 0.0f) {
      write_slice<DT>(s, grad, false, [](float (&)[E]) {});
      return;
    }
    const double per = static_cast<double>(weight) / static_cast<double>(p.T);
    const float scale = static_cast<float>(per * mass);
    // the listed tokens of the slice, before the gradient takes their place
    struct Listed {
      int id;
      float g;
    } at[2] = {{-1, 0.0f}, {-1, 0.0f}};
    static_assert(2 * kSliceThreads >= COS_TOP_MAX, "a thread has two entries at most");
    int found = 0;
    each_listed(p, s, sh, [&](int id, double t) {
      const double q = exp2(static_cast<double>(student_at<DT>(student, id) - m) * static_cast<double>(c) - static_cast<double>(log_z));
      const Listed l = {id, static_cast<float>(per * (mass * q - t))};
      if (found++ == 0)
        at[0] = l;
      else
        at[1] = l;
    });
    __syncthreads();
    write_slice<DT>(s, grad, true, [&](float (&v)[E]) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = scale * ex2_approx((v[e] - m) * c - log_z);
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (at[i].id >= 0) store_entry<DT>(grad, at[i].id, at[i].g);
  }
}

bool misaligned(const void* p, int to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

template <int MODE>
cos_status distill(const cos_distill_args* a, void* cuda_stream) {
  if (!a) return call_failed(COS_ERR_INVALID_ARG, "null argument");
  if (!a->student || !a->ids || !a->values) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (a->rows < 1 || a->vocab < 1 || a->vocab > 0x7ffffff0) return call_failed(COS_ERR_INVALID_ARG, "rows and vocab must be positive");
  if (a->dtype < COS_DTYPE_F32 || a->dtype > COS_DTYPE_F16) return call_failed(COS_ERR_INVALID_ARG, "unknown dtype");
  if (a->rows > 1 && a->stride_student < a->vocab) return call_failed(COS_ERR_INVALID_ARG, "rows overlap: stride_student is less than vocab");
  if (a->lists < 1 || a->lists > COS_MAX_MODELS || a->k < 1 || a->k > COS_TOP_MAX || a->lists * a->k > COS_TOP_MAX)
    return call_failed(COS_ERR_INVALID_ARG, "lists must be in [1, COS_MAX_MODELS] and lists * k in [1, COS_TOP_MAX]");
  for (int g = 0; g < a->lists; ++g)
    if (!(a->weights[g] >= 0.0f && a->weights[g] < INFINITY)) return call_failed(COS_ERR_INVALID_ARG, "weights must be finite and >= 0");
  if (!(a->temperature > 0.0f && a->temperature < INFINITY)) return call_failed(COS_ERR_INVALID_ARG, "temperature must be finite and > 0");
  const int bytes = a->dtype == COS_DTYPE_F32 ? 4 : 2;
  if (misaligned(a->student, bytes)) return call_failed(COS_ERR_ALIGNMENT, "student pointer not aligned to its element type");
  if (MODE != kGrad && !a->loss) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (MODE != kStep && !a->statistics) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (MODE != kLoss) {
    if (!a->row_weights || !a->grad) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
    if (misaligned(a->grad, bytes)) return call_failed(COS_ERR_ALIGNMENT, "grad pointer not aligned to its element type");
    if (a->rows > 1 && a->stride_grad < a->vocab) return call_failed(COS_ERR_INVALID_ARG, "rows overlap: stride_grad is less than vocab");
    if (a->grad == a->student && a->rows > 1 && a->stride_grad != a->stride_student) return call_failed(COS_ERR_INVALID_ARG, "a gradient in place needs the stride of the student");
  }
  if (misaligned(a->ids, 4) || misaligned(a->values, 4) || misaligned(a->lse, 4) || (MODE != kGrad && misaligned(a->loss, 4)) || (MODE != kLoss && misaligned(a->row_weights, 4)))
    return call_failed(COS_ERR_ALIGNMENT, "an int32/float pointer is not 4-byte aligned");
  if (MODE != kStep && misaligned(a->statistics, 8)) return call_failed(COS_ERR_ALIGNMENT, "statistics is not 8-byte aligned");

  OnDevice on(a->device);
  if (on.error != cudaSuccess) return call_failed("cudaSetDevice", on.error);
  SlicePlan plan;
  cudaError_t e = slice_plan(a->device, a->rows, a->vocab, a->dtype, &plan);
  if (e != cudaSuccess) return call_failed("device query", e);
  if (static_cast<long long>(a->rows) * plan.parts > 0x7fffffffll) return call_failed(COS_ERR_UNSUPPORTED, "too many rows for one launch");
  DistillParams p = {};
  p.student = static_cast<const char*>(a->student);
  p.stride = a->stride_student;
  p.rows = a->rows;
  p.V = a->vocab;
  p.parts = plan.parts;
  p.share = plan.share;
  p.seg = plan.seg;
  p.res = MODE == kStep ? plan.res : 0;
  p.lists = a->lists;
  p.k = a->k;
  p.ids = a->ids;
  p.values = a->values;
  p.lse = a->lse;
  for (int g = 0; g < a->lists; ++g) p.w[g] = a->weights[g];
  p.T = a->temperature;
  p.row_weights = a->row_weights;
  p.loss = a->loss;
  p.statistics = reinterpret_cast<float2*>(a->statistics);
  p.grad = static_cast<char*>(a->grad);
  p.stride_grad = a->stride_grad;
  void (*fn)(DistillParams) = a->dtype == COS_DTYPE_F32    ? cos_distill_kernel<COS_DTYPE_F32, MODE>
                              : a->dtype == COS_DTYPE_BF16 ? cos_distill_kernel<COS_DTYPE_BF16, MODE>
                                                           : cos_distill_kernel<COS_DTYPE_F16, MODE>;
  e = slice_launch(fn, p, a->rows * plan.parts, MODE == kGrad ? 1 : plan.parts, MODE == kStep ? plan.smem : 0, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? COS_OK : call_failed("launch", e);
}

}  // namespace
}  // namespace cosv

extern "C" cos_status cos_distill_loss(const cos_distill_args* a, void* cuda_stream) { return cosv::distill<cosv::kLoss>(a, cuda_stream); }
extern "C" cos_status cos_distill_grad(const cos_distill_args* a, void* cuda_stream) { return cosv::distill<cosv::kGrad>(a, cuda_stream); }
extern "C" cos_status cos_distill_step(const cos_distill_args* a, void* cuda_stream) { return cosv::distill<cosv::kStep>(a, cuda_stream); }
