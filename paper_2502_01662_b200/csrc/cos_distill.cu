// Distillation from the largest logits of a row's teachers: the loss, its gradient, and both in one launch.
//
// Mathematics.  loss = sum over the listed tokens of t (ln t - s/T) + P lse(s/T), so beside the student's normaliser the loss takes the listed tokens alone
// (both relative to the student's logit at one of them, so that nothing large is subtracted); the gradient is P q everywhere, with t taken off at the listed
// tokens.  Shares of a token that comes up more than once are added by the first of its entries, in order, so results do not depend on timing.
//
// Two launches for the loss, and for loss and gradient together: the shares (a block for each row looks at its entries; a few microseconds, in which the first rows of the
// other launch are on their way already), then the rows.  Bound by memory: the loss reads the student once, the gradient reads it and writes as much; the rows of the
// launch with both stay in the shared memory of a cluster of blocks between the normaliser and the gradient, and are read once.  Three blocks of a multiprocessor
// have up to 64 KB each under way, since a row's chain of steps (copies, two sweeps, a barrier, the gradient) takes longer than its bytes.
// Measured: loss of 1024 x 128256 bf16 48 us (5.0 TB/s of what is not padding), its gradient 78 (6.4); both of 2048 x 32000 bf16 59 us, 4.0 TB/s, with the issue slots 68 % busy; both of
// 100 x 50001 fp32 14.4 us, of which the shares are 3.  The shares compare every entry of a row with all of them, which is next to nothing for 64 entries and most of the time for many: both of 2048 x 32000
// bf16 without padding 64 us with 64 entries, 116 with 256, 274 with 512, 900 with 1024.
// Exponentials are 32-bit (2^-22) and sums of them 64-bit; shares, logarithms and the loss are 64-bit; the gradient is rounded once.
#include "cos_slice.cuh"

namespace cosv {
namespace {

// What a row's launches leave for the next (COS_DISTILL_STATISTICS floats): the student's largest logit and log2 of its normaliser; the sum of the shares; the
// reference logit, and the sum over the listed tokens of t (ln t - (s - reference) / T).
struct Statistics {
  float m, log_z, mass, reference;
  double listed, mass64;
};
static_assert(sizeof(Statistics) == COS_DISTILL_STATISTICS * sizeof(float), "as the header says");
constexpr int kMostKept = 64 * 1024;  // bytes of a slice: three blocks of a multiprocessor have room for that
constexpr int kLoss = 0, kGrad = 1, kStep = 2, kShareThreads = 128;

struct DistillParams {
  const char* student;
  long long stride;
  int rows, V, parts, shift, share, seg, res;  // parts: 2^shift
  int early;  // blocks that may start on their rows before the shares are there
  int lists, k;
  const int* ids;
  const float* values;
  const float* lse;
  float w[COS_MAX_MODELS];
  float c;       // log2(e) / T
  double inv_T;
  double inv_c;  // 1 / T as `c` has it: the student's listed logits go by the temperature of its normaliser, or the rounding of c (3e-8) comes in times the distance
                 // of the likely logits from the largest one (15 and more) instead of from the listed ones
  const float* row_weights;
  float* loss;
  float* statistics;
  char* grad;
  long long stride_grad;
};

// The entries of a row, in shared memory.
struct Shares {
  double* t;  // 0 for an empty entry
  int* id;
  float* s;   // the student's logits there
  double *per_warp, *list_max, *list_sum;
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
  for (int w = 0; w < kShareThreads / 32; ++w) s += per_warp[w];
  __syncthreads();
  return s;
}

template <int DT>
__device__ __forceinline__ float student_at(const char* row, int x) {
  return Elem<DT>::load1(row, x);
}

// Every entry's share to shared memory (0 for an empty one); returns their sum, NaN where an entry names no token.
template <int DT>
__device__ __forceinline__ double row_shares(const DistillParams& p, const char* student, int row, const Shares& sh) {
  const int n = p.lists * p.k, tid = threadIdx.x;
  const int* ids = p.ids + static_cast<long long>(row) * n;
  const float* values = p.values + static_cast<long long>(row) * n;
  const double inv_T = p.inv_T;
  if (!p.lse) {  // softmax over each list: a warp for each
    for (int g = tid >> 5; g < p.lists; g += kShareThreads / 32) {
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
  for (int e = tid; e < n; e += kShareThreads) {
    const int id = ids[e], g = e / p.k;
    const float v = values[e], s = id >= 0 && id < p.V ? student_at<DT>(student, id) : 0.0f;
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
    sh.s[e] = s;
    sh.t[e] = t;
    mine += t;
  }
  return block_sum(mine, sh.per_warp);
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

// The slice of the gradient: f(vector) in place of the vectors (read: they are looked at).
template <int DT, class F>
__device__ __forceinline__ void write_slice(const RowSlice<DT>& s, char* row, bool read, F&& f) {
  constexpr int E = Elem<DT>::E, B = Elem<DT>::bytes;
  const bool whole = static_cast<int>(reinterpret_cast<unsigned long long>(row) & 15) / B == s.off;
  for (int i = s.begin + (threadIdx.x & 31); i < s.end; i += 32) {
    const uint4 g = f(read ? s.at(i) : uint4());
    const int x = s.token(i);
    if (whole && x >= 0 && x <= s.V - E) {
      *reinterpret_cast<uint4*>(row + static_cast<long long>(x) * B) = g;
    } else {
      const unsigned* w = reinterpret_cast<const unsigned*>(&g);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (x + e >= 0 && x + e < s.V) {
          if (DT == COS_DTYPE_F32)
            reinterpret_cast<unsigned*>(row)[x + e] = w[e];
          else
            reinterpret_cast<unsigned short*>(row)[x + e] = static_cast<unsigned short>((e & 1) ? w[e >> 1] >> 16 : w[e >> 1]);
        }
    }
  }
}

// The student's normaliser over the row: sum of 2^((s - m) c).
struct Normaliser {
  float m;
  double z;
};
struct NormaliserRoom {
  Normaliser warp[kSliceWarps], block[kSliceParts];
};
// ... from the warps' (m the same for the lanes of one, z a lane's).
template <int kWarps>
__device__ __forceinline__ Normaliser row_normaliser(NormaliserRoom& room, int parts, int rank, float c, float m, double z) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  z = warp_sum(z);
  if (lane == 0) room.warp[warp] = {m, z};
  __syncthreads();
  if (warp == 0) {
    const Normaliser a = room.warp[lane & (kWarps - 1)];
    m = a.m;
#pragma unroll
    for (int d = kWarps / 2; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, d));
    z = lane < kWarps && a.m != -INFINITY ? a.z * static_cast<double>(ex2_approx((a.m - m) * c)) : 0.0;
    z = warp_sum(z);
    if (parts == 1) {
      if (lane == 0) room.block[0] = {m, z};
    } else if (lane < parts) {
      *of_rank(&room.block[rank], lane) = {m, z};
    }
  }
  row_barrier(parts);
  Normaliser n = room.block[0];
  for (int r = 1; r < parts; ++r) n.m = max_nan(n.m, room.block[r].m);
  n.z = 0.0;
  for (int r = 0; r < parts; ++r) {
    const Normaliser a = room.block[r];
    if (a.m != -INFINITY) n.z += a.z * static_cast<double>(ex2_approx((a.m - n.m) * c));
  }
  return n;
}

template <int DT>
__device__ __forceinline__ Normaliser normaliser(NormaliserRoom& room, const RowSlice<DT>& s, int parts, int rank, float c) {
  RunningMax<DT> top;
  s.raw([&](int, const uint4& r) { top.add(r); });
  float m = top.value();
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, d));
  double z = 0.0;
  if (!(m == -INFINITY)) {  // (NaN: all NaN)
    const f32x2 minus_m = pack2(-m, -m), cc = pack2(c, c);
    s.raw([&](int, const uint4& r) { z += static_cast<double>(sum_exp2<DT>(r, minus_m, cc)); });
  }
  return row_normaliser<kSliceWarps>(room, parts, rank, c, m, z);
}

// q(x) times the scale, from the statistics of the student.
template <int DT>
__device__ __forceinline__ uint4 gradient_of(const uint4& r, f32x2 scale, f32x2 minus_m, f32x2 c, f32x2 minus_log_z) {
  f32x2 x[Elem<DT>::E / 2];
  unpack_pairs<DT>(r, x);
  uint4 g;
  unsigned* w = reinterpret_cast<unsigned*>(&g);
#pragma unroll
  for (int k = 0; k < Elem<DT>::E / 2; ++k) {
    const f32x2 a = fma2(add2(x[k], minus_m), c, minus_log_z);
    const f32x2 e = mul2(pack2(ex2_approx(lo2(a)), ex2_approx(hi2(a))), scale);
    if constexpr (DT == COS_DTYPE_F32) {
      w[2 * k] = __float_as_uint(lo2(e));
      w[2 * k + 1] = __float_as_uint(hi2(e));
    } else if constexpr (DT == COS_DTYPE_BF16) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(lo2(e), hi2(e));
      w[k] = *reinterpret_cast<const unsigned*>(&h);
    } else {
      const __half2 h = __floats2half2_rn(lo2(e), hi2(e));
      w[k] = *reinterpret_cast<const unsigned*>(&h);
    }
  }
  return g;
}
// The gradient at a listed token.
__device__ __forceinline__ float listed_gradient(float s, double t, double per, double mass, float m, float c, float log_z) {
  return static_cast<float>(per * (mass * exp2(static_cast<double>(s - m) * static_cast<double>(c) - static_cast<double>(log_z)) - t));
}

__device__ __forceinline__ Statistics* statistics_of(const DistillParams& p, int row) { return reinterpret_cast<Statistics*>(p.statistics) + row; }
__device__ __forceinline__ float* shares_of(const DistillParams& p, int row) {  // (behind the statistics of all rows)
  return p.statistics + static_cast<long long>(p.rows) * COS_DISTILL_STATISTICS + static_cast<long long>(row) * p.lists * p.k;
}

// The shares of a row: of a token's first entry its whole share, of the others 0.
template <int DT>
__global__ void __launch_bounds__(kShareThreads) cos_distill_shares_kernel(const DistillParams p) {
  extern __shared__ uint4 smem[];
  __shared__ double per_warp[kShareThreads / 32], list_max[COS_MAX_MODELS], list_sum[COS_MAX_MODELS];
  wait_for_inputs();
  let_next_launch();  // (the rows: they read the student, which is settled where every block has come here)
  const int row = blockIdx.x, n = p.lists * p.k;
  const Shares sh = {reinterpret_cast<double*>(smem), reinterpret_cast<int*>(smem) + 2 * n, reinterpret_cast<float*>(smem) + 3 * n, per_warp, list_max, list_sum};
  const char* student = p.student + static_cast<long long>(row) * p.stride * Elem<DT>::bytes;
  const double mass = row_shares<DT>(p, student, row, sh);
  if (!(mass != 0.0)) {  // nothing to learn from
    if (threadIdx.x == 0) *statistics_of(p, row) = {0.0f, 0.0f, 0.0f, 0.0f, 0.0, 0.0};
    return;
  }
  int at = 0;
  while (at < n && !(sh.t[at] != 0.0 && sh.id[at] < p.V)) ++at;
  const float ref = at < n ? sh.s[at] : 0.0f;
  const double base = fabsf(ref) < INFINITY ? static_cast<double>(ref) : 0.0;
  float* const shares = shares_of(p, row);
  double listed = 0.0;
  for (int e = threadIdx.x; e < n; e += kShareThreads) {
    const int id = sh.id[e];
    double t = 0.0;
    if (id >= 0 && id < p.V) {
      bool first = true;
#pragma unroll 4
      for (int j = 0; j < n; ++j)
        if (sh.id[j] == id) {
          first = first && j >= e;
          t += sh.t[j];
        }
      if (!first) t = 0.0;
      if (t != 0.0) listed += t * (log(t) - (static_cast<double>(sh.s[e]) - base) * p.inv_c);
    }
    shares[e] = static_cast<float>(t);
  }
  listed = block_sum(listed, per_warp);
  if (threadIdx.x == 0) *statistics_of(p, row) = {0.0f, 0.0f, static_cast<float>(mass), static_cast<float>(base), listed, mass};
}

__device__ __forceinline__ float log2_of(const Normaliser& z) { return z.m == -INFINITY ? __int_as_float(0x7fc00000) : log2f(static_cast<float>(z.z)); }
__device__ __forceinline__ void finish_loss(const DistillParams& p, int row, const Statistics& st, const Normaliser& z, bool keep) {
  const float log_z = log2_of(z);
  p.loss[row] = z.m == -INFINITY ? log_z : static_cast<float>(st.listed + st.mass64 * ((static_cast<double>(z.m) - static_cast<double>(st.reference)) * p.inv_c + log(z.z)));
  if (keep) {
    statistics_of(p, row)->m = z.m;
    statistics_of(p, row)->log_z = log_z;
  }
}

// The loss where there are rows enough for a block each: a row goes by in registers, against a running maximum of each lane.
template <int DT, int kWarps>
__global__ void __launch_bounds__(32 * kWarps, 32 / kWarps) cos_distill_stream_kernel(const DistillParams p) {
  __shared__ NormaliserRoom room;
  const int row = blockIdx.x;
  RowSlice<DT> s;
  s.init(p.student + static_cast<long long>(row) * p.stride * Elem<DT>::bytes, p.V, 0, p.share, p.seg, nullptr, 0);
  const bool early = row < p.early;  // (the student is settled; whether the row has shares is known later)
  Statistics st;
  if (!early) {
    wait_for_inputs();
    st = *statistics_of(p, row);
    if (st.mass64 == 0.0) {
      if (threadIdx.x == 0) p.loss[row] = 0.0f;
      return;
    }
  }
  const float c = p.c;
  RunningSum<DT> sum;
  s.stream(s.begin + (threadIdx.x & 31), s.end, [&](const uint4 (&r)[4]) {
    RunningMax<DT> top;
#pragma unroll
    for (int k = 0; k < 4; ++k) top.add(r[k]);
    sum.add(r, top, c);
  });
  if (early) {
    wait_for_inputs();
    st = *statistics_of(p, row);
    if (st.mass64 == 0.0) {
      if (threadIdx.x == 0) p.loss[row] = 0.0f;
      return;
    }
  }
  float m = sum.m;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, d));
  sum.to(m, c);
  const Normaliser n = row_normaliser<kWarps>(room, 1, 0, c, m, sum.z);
  if (threadIdx.x == 0) finish_loss(p, row, st, n, true);
}

// The rows.  kGrad: the normalisers are there, and every block works for itself.
template <int DT, int MODE>
__global__ void __launch_bounds__(kSliceThreads, 3) cos_distill_kernel(const DistillParams p) {
  extern __shared__ uint4 smem[];
  __shared__ NormaliserRoom room;
  const int parts = p.parts, rank = blockIdx.x & (parts - 1), row = blockIdx.x >> p.shift, tid = threadIdx.x, n = p.lists * p.k;
  const bool wide = MODE != kGrad && parts > 1;
  if (wide) cluster_barrier_arrive();
  const char* student = p.student + static_cast<long long>(row) * p.stride * Elem<DT>::bytes;
  char* grad = MODE != kLoss ? p.grad + static_cast<long long>(row) * p.stride_grad * Elem<DT>::bytes : nullptr;
  RowSlice<DT> s;
  s.init(student, p.V, rank, p.share, p.seg, smem, p.res);
  const bool early = MODE != kGrad && blockIdx.x < p.early;
  if (early) s.start();
  wait_for_inputs();
  const Statistics st = *statistics_of(p, row);
  const float weight = MODE != kLoss ? p.row_weights[row] : 1.0f;
  const bool none = st.mass64 == 0.0;
  if (none || (MODE == kGrad && weight == 0.0f)) {
    if (MODE != kGrad && rank == 0 && tid == 0) p.loss[row] = 0.0f;
    if (MODE != kLoss) write_slice<DT>(s, grad, false, [](const uint4& nothing) { return nothing; });
    s.finish();
    if (wide) cluster_barrier_wait();
    return;
  }
  if (!early) s.start();
  // the listed tokens of the slice, before the gradient takes their place
  struct Listed {
    int id;
    float s, t;
  } mine[2] = {{-1, 0.0f, 0.0f}, {-1, 0.0f, 0.0f}};
  static_assert(2 * kSliceThreads >= COS_TOP_MAX, "a thread has two entries at most");
  if (MODE != kLoss) {
    const int lo = max(0, s.token(0)), hi = min(p.V, s.token(s.nv));
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int e = tid + k * kSliceThreads;
      if (e < n) {
        const int id = p.ids[static_cast<long long>(row) * n + e];
        const float t = shares_of(p, row)[e];
        if (id >= lo && id < hi && t != 0.0f) mine[k] = {id, student_at<DT>(student, id), t};
      }
    }
  }
  s.finish();
  const float c = p.c;
  float m = st.m, log_z = st.log_z;
  if (MODE != kGrad) {
    if (wide) cluster_barrier_wait();  // (every block of the row has started)
    const Normaliser z = normaliser<DT>(room, s, parts, rank, c);
    m = z.m;
    log_z = log2_of(z);
    if (rank == 0 && tid == 0) finish_loss(p, row, st, z, MODE == kLoss);
  } else {
    __syncthreads();  // (the listed tokens have been read)
  }
  if (MODE != kLoss) {
    if (MODE == kStep && weight == 0.0f) {
      write_slice<DT>(s, grad, false, [](const uint4& nothing) { return nothing; });
      return;
    }
    const double per = static_cast<double>(weight) * p.inv_T, mass = static_cast<double>(st.mass);
    const float scale = static_cast<float>(per * mass);
    const f32x2 scales = pack2(scale, scale), minus_m = pack2(-m, -m), cc = pack2(c, c), minus_log_z = pack2(-log_z, -log_z);
    write_slice<DT>(s, grad, true, [&](const uint4& r) { return gradient_of<DT>(r, scales, minus_m, cc, minus_log_z); });
    __syncthreads();  // (the listed tokens' places are written again)
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (mine[k].id >= 0) store_entry<DT>(grad, mine[k].id, listed_gradient(mine[k].s, static_cast<double>(mine[k].t), per, mass, m, c, log_z));
  }
}

bool misaligned(const void* p, int to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

template <int MODE>
cos_status distill(const cos_distill_args* a, void* cuda_stream) {
  if (!a) return call_failed(COS_ERR_INVALID_ARG, "null argument");
  if (!a->student || !a->ids || !a->values) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (a->rows < 1 || a->vocab < 1 || a->vocab > 0x7ffffff0) return call_failed(COS_ERR_INVALID_ARG, "rows and vocab must be positive");
  if (a->dtype < COS_DTYPE_F32 || a->dtype > COS_DTYPE_F16) return call_failed(COS_ERR_INVALID_ARG, "unknown dtype");
  if (a->rows > 1 && a->stride_student < a->vocab && a->stride_student != 0) return call_failed(COS_ERR_INVALID_ARG, "rows overlap: stride_student is less than vocab");
  if (a->lists < 1 || a->lists > COS_MAX_MODELS || a->k < 1 || a->k > COS_TOP_MAX || a->lists * a->k > COS_TOP_MAX)
    return call_failed(COS_ERR_INVALID_ARG, "lists must be in [1, COS_MAX_MODELS] and lists * k in [1, COS_TOP_MAX]");
  for (int g = 0; g < a->lists; ++g)
    if (!(a->weights[g] >= 0.0f && a->weights[g] < INFINITY)) return call_failed(COS_ERR_INVALID_ARG, "weights must be finite and >= 0");
  if (!(a->temperature > 1e-300 && a->temperature < 1e300)) return call_failed(COS_ERR_INVALID_ARG, "temperature must be finite and > 0 (1e-300 to 1e300)");
  const int bytes = a->dtype == COS_DTYPE_F32 ? 4 : 2;
  if (misaligned(a->student, bytes)) return call_failed(COS_ERR_ALIGNMENT, "student pointer not aligned to its element type");
  if (MODE != kGrad && !a->loss) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (!a->statistics) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (MODE != kLoss) {
    if (!a->row_weights || !a->grad) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
    if (misaligned(a->grad, bytes)) return call_failed(COS_ERR_ALIGNMENT, "grad pointer not aligned to its element type");
    if (a->rows > 1 && a->stride_grad < a->vocab) return call_failed(COS_ERR_INVALID_ARG, "rows overlap: stride_grad is less than vocab");
    if (overlap(a->student, a->stride_student, a->grad, a->stride_grad, a->rows, a->vocab, bytes)) return call_failed(COS_ERR_INVALID_ARG, "grad overlaps the student (in place: the same address and stride)");
  }
  if (misaligned(a->ids, 4) || misaligned(a->values, 4) || misaligned(a->lse, 4) || (MODE != kGrad && misaligned(a->loss, 4)) || (MODE != kLoss && misaligned(a->row_weights, 4)))
    return call_failed(COS_ERR_ALIGNMENT, "an int32/float pointer is not 4-byte aligned");
  if (misaligned(a->statistics, 16)) return call_failed(COS_ERR_ALIGNMENT, "statistics is not 16-byte aligned");

  OnDevice on(a->device);
  if (on.error != cudaSuccess) return call_failed("cudaSetDevice", on.error);
  SlicePlan plan;
  cudaError_t e = slice_plan(a->device, a->rows, a->vocab, a->dtype, kMostKept, MODE != kGrad, &plan);
  if (e != cudaSuccess) return call_failed("device query", e);
  if (static_cast<long long>(a->rows) * plan.parts > 0x7fffffffll) return call_failed(COS_ERR_UNSUPPORTED, "too many rows for one launch");
  DistillParams p = {};
  p.student = static_cast<const char*>(a->student);
  p.stride = a->stride_student;
  p.rows = a->rows;
  p.V = a->vocab;
  p.parts = plan.parts;
  p.shift = __builtin_ctz(plan.parts);
  p.share = plan.share;
  p.seg = plan.seg;
  p.res = plan.res;
  p.early = 2 * plan.sms;  // (the first ones to find a place)
  // The loss takes a block for each row, but for few rows that are long (64 rows of 128256 bf16 9.0 us, on clusters 13.9; 256 rows 15 and 28; 16 rows of 256000 14.1 and 10.9, 64 rows 14.4
  // and 19.4), of 8 warps where rows are short (256 rows of 32000 bf16 7.5 us, of 16 warps 8.5; 512 rows of 128256 31.1 and 29.3).
  const long long row_bytes = static_cast<long long>(a->vocab) * bytes;
  const int stream_warps = MODE != kLoss || (row_bytes > 384 * 1024 && a->rows <= 32) ? 0 : (row_bytes < 96 * 1024 ? 8 : 16);
  if (stream_warps) plan_row(a->vocab, a->dtype, stream_warps, &p.share, &p.seg);
  p.lists = a->lists;
  p.k = a->k;
  p.ids = a->ids;
  p.values = a->values;
  p.lse = a->lse;
  for (int g = 0; g < a->lists; ++g) p.w[g] = a->weights[g];
  const Exponent exponent = exponent_of(a->temperature);
  p.c = exponent.c;
  p.inv_T = 1.0 / a->temperature;
  p.inv_c = exponent.value < 3e38 ? exponent.value * 0.6931471805599453 : p.inv_T;
  p.row_weights = a->row_weights;
  p.loss = a->loss;
  p.statistics = a->statistics;
  p.grad = static_cast<char*>(a->grad);
  p.stride_grad = a->stride_grad;
  const auto launches = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (MODE != kGrad) {
      constexpr size_t entry = sizeof(double) + sizeof(int) + sizeof(float);
      const cudaError_t first = slice_launch(cos_distill_shares_kernel<DT>, p, a->rows, 1, static_cast<size_t>(a->lists) * a->k * entry, COS_TOP_MAX * entry, stream, kShareThreads);
      if (first != cudaSuccess) return first;
    }
    if (stream_warps == 8) return slice_launch(cos_distill_stream_kernel<DT, 8>, p, a->rows, 1, 0, 0, stream, 256);
    if (stream_warps == 16) return slice_launch(cos_distill_stream_kernel<DT, 16>, p, a->rows, 1, 0, 0, stream, 512);
    return slice_launch(cos_distill_kernel<DT, MODE>, p, a->rows * plan.parts, MODE == kGrad ? 1 : plan.parts, plan.smem, kMostKept, stream);
  };
  e = a->dtype == COS_DTYPE_F32    ? launches(std::integral_constant<int, COS_DTYPE_F32>())
      : a->dtype == COS_DTYPE_BF16 ? launches(std::integral_constant<int, COS_DTYPE_BF16>())
                                   : launches(std::integral_constant<int, COS_DTYPE_F16>());
  return e == cudaSuccess ? COS_OK : call_failed("launch", e);
}

}  // namespace
}  // namespace cosv

extern "C" cos_status cos_distill_loss(const cos_distill_args* a, void* cuda_stream) { return cosv::distill<cosv::kLoss>(a, cuda_stream); }
extern "C" cos_status cos_distill_grad(const cos_distill_args* a, void* cuda_stream) { return cosv::distill<cosv::kGrad>(a, cuda_stream); }
extern "C" cos_status cos_distill_step(const cos_distill_args* a, void* cuda_stream) { return cosv::distill<cosv::kStep>(a, cuda_stream); }
