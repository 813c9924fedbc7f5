// A row of logits on a cluster of blocks: each block holds a slice of it in shared memory and sweeps it as often as it has to, and the
// blocks exchange what they found.
//
// A slice is a range of the row's 16-byte vectors, counted from the 16-byte boundary at or before the row's first entry, so every vector inside
// the row is one aligned load wherever the row starts; entries of the first and the last vector that are not the row's read as -inf.  A warp has a
// contiguous part of the slice and a lane every 32nd vector of it, the same in every sweep, so sweeps need no barrier between them.
#ifndef COS_SLICE_CUH
#define COS_SLICE_CUH

#include <cuda_bf16.h>

#include <cfloat>
#include <cstring>
#include <type_traits>

#include "cos_common.cuh"
#include "cos_draft.h"

namespace cosv {

constexpr int kSliceThreads = 512, kSliceWarps = kSliceThreads / 32, kSliceParts = 16;  // threads of a block, most blocks of a row
typedef unsigned long long u64;

__device__ __forceinline__ float max_nan(float a, float b) {  // NaN where one is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// The largest entry of vectors (NaN where there is one): 16-bit types two entries at a time.
template <int DT>
struct RunningMax {
  unsigned top[DT == COS_DTYPE_F32 ? 2 : 1];
  __device__ __forceinline__ RunningMax() {
    for (unsigned& w : top) w = neg_inf_vector<DT>().x;
  }
  static __device__ __forceinline__ unsigned larger(unsigned a, unsigned b) {
    if constexpr (DT == COS_DTYPE_F32) {
      return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b)));
    } else if constexpr (DT == COS_DTYPE_BF16) {
      const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
      return *reinterpret_cast<const unsigned*>(&m);
    } else {
      const __half2 m = __hmax2_nan(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
      return *reinterpret_cast<const unsigned*>(&m);
    }
  }
  __device__ __forceinline__ void add(const uint4& r) {
    constexpr int kLast = DT == COS_DTYPE_F32 ? 1 : 0;
    top[0] = larger(top[0], larger(r.x, r.z));
    top[kLast] = larger(top[kLast], larger(r.y, r.w));
  }
  __device__ __forceinline__ void add(const RunningMax& o) {
    for (int i = 0; i < static_cast<int>(sizeof(top) / sizeof(top[0])); ++i) top[i] = larger(top[i], o.top[i]);
  }
  __device__ __forceinline__ float value() const {
    if constexpr (DT == COS_DTYPE_F32) return max_nan(__uint_as_float(top[0]), __uint_as_float(top[1]));
    const uint4 r = make_uint4(top[0], 0, 0, 0);
    return max_nan(entry<DT>(r, 0), entry<DT>(r, 1));
  }
};

// sum of 2^((v - m) c) over a vector's entries
template <int DT>
__device__ __forceinline__ float sum_exp2(const uint4& r, f32x2 minus_m, f32x2 c) {
  f32x2 x[Elem<DT>::E / 2], sum = 0;
  unpack_pairs<DT>(r, x);
#pragma unroll
  for (int k = 0; k < Elem<DT>::E / 2; ++k) {
    const f32x2 a = mul2(add2(x[k], minus_m), c);
    const f32x2 e = pack2(ex2_approx(lo2(a)), ex2_approx(hi2(a)));
    sum = k == 0 ? e : add2(sum, e);
  }
  return lo2(sum) + hi2(sum);
}

// A lane's part of a softmax normaliser, against the largest entry it has seen.
template <int DT>
struct RunningSum {
  float m = -INFINITY;
  double z = 0.0;
  __device__ __forceinline__ void to(float t, float c) {  // (a maximum that is NaN stays it)
    if (t > m || t != t) {
      z *= static_cast<double>(m == -INFINITY ? 0.0f : ex2_approx((m - t) * c));
      m = t;
    }
  }
  __device__ __forceinline__ void add(const uint4 (&r)[4], const RunningMax<DT>& top, float c) {
    to(top.value(), c);
    if (m == -INFINITY) return;
    const f32x2 minus_m = pack2(-m, -m), cc = pack2(c, c);
    float part = sum_exp2<DT>(r[0], minus_m, cc);
#pragma unroll
    for (int k = 1; k < 4; ++k) part += sum_exp2<DT>(r[k], minus_m, cc);
    z += static_cast<double>(part);
  }
};

template <int DT>
struct RowSlice {
  static constexpr int E = Elem<DT>::E;
  const char* base;  // the boundary
  int off, V;        // entries between it and the row, entries of the row
  int v0, nv;        // the slice's vectors
  int begin, end;    // this warp's part of them
  uint4* kept;       // the first `res` are here
  int res;

  // `share` vectors for each block, `seg` of them for each warp (a multiple of 32)
  __device__ __forceinline__ void init(const void* row, int V_, int rank, int share, int seg, uint4* smem, int res_) {
    const unsigned long long at = reinterpret_cast<unsigned long long>(row);
    base = reinterpret_cast<const char*>(at & ~15ull);
    off = static_cast<int>(at & 15ull) / Elem<DT>::bytes;
    V = V_;
    const int all = static_cast<int>((static_cast<long long>(V) + off + E - 1) / E);
    const long long lo = static_cast<long long>(rank) * share;
    v0 = lo < all ? static_cast<int>(lo) : all;
    nv = min(share, all - v0);
    const int w = threadIdx.x >> 5;
    begin = min(nv, w * seg);
    end = min(nv, begin + seg);
    kept = smem;
    res = res_;
  }
  // the warp that has a token of the slice
  __device__ __forceinline__ int warp_of(int token, int seg) const { return static_cast<int>((static_cast<long long>(token) + off) / E - v0) / seg; }
  // the token of a vector's first entry (negative where the row starts inside it)
  __device__ __forceinline__ int token(int i) const { return static_cast<int>(static_cast<long long>(v0 + i) * E - off); }
  __device__ __forceinline__ uint4 fetch(int i) const {
    const int x = token(i);
    const char* at = base + (static_cast<long long>(v0) + i) * 16;
    if (x >= 0 && x <= V - E) return ldg_stream16(at);
    return ragged(at, x);
  }
  __device__ __noinline__ uint4 ragged(const char* at, int x) const {
    uint4 r = neg_inf_vector<DT>();
    unsigned* w = reinterpret_cast<unsigned*>(&r);
    if (DT == COS_DTYPE_F32) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (x + k >= 0 && x + k < V) w[k] = __ldg(reinterpret_cast<const unsigned*>(at) + k);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (x + k >= 0 && x + k < V) {
          const unsigned h = __ldg(reinterpret_cast<const unsigned short*>(at) + k);
          w[k >> 1] = (k & 1) ? ((w[k >> 1] & 0xffffu) | (h << 16)) : ((w[k >> 1] & 0xffff0000u) | h);
        }
    }
    return r;
  }
  __device__ __forceinline__ uint4 at(int i) const { return i < res ? kept[i] : fetch(i); }

  // Begins to bring the warp's part here: asynchronous copies, all of a lane's under way at once.  finish() waits for them (a lane reads only what it copied
  // itself, so no barrier is needed).
  __device__ __forceinline__ void start() const {
    const int last = min(end, res);
    int i = begin + (threadIdx.x & 31);
    const int whole = static_cast<int>(min(static_cast<long long>(last), (static_cast<long long>(V) + off) / E - v0));  // vectors before it end inside the row
    if (i < last && v0 + i == 0 && off != 0) {
      kept[i] = ragged(base, token(i));
      i += 32;
    }
    const char* from = base + (static_cast<long long>(v0) + i) * 16;
    unsigned to = static_cast<unsigned>(__cvta_generic_to_shared(kept + i));
#pragma unroll 4
    for (; i < whole; i += 32, from += 512, to += 512) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    if (i < last) kept[i] = ragged(from, token(i));  // (the row's last vector: no lane has more than one behind `whole`)
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ void finish() const { asm volatile("cp.async.wait_all;" ::: "memory"); }

  // f(token of the first entry, values) for every vector of this lane.
  template <class F>
  __device__ __forceinline__ void vectors(F&& f) const {
    for (int i = begin + (threadIdx.x & 31); i < end; i += 32) {
      const uint4 r = at(i);
      float v[E];
      Elem<DT>::unpack(r, v);
      f(token(i), v);
    }
  }
  // f(four vectors) for the vectors of this lane from `from` on, before `to`, fetched from memory, the next four under way meanwhile (-inf where there are fewer).
  template <class F>
  __device__ __forceinline__ void stream(int from, int to, F&& f) const {
    const int whole = static_cast<int>(min(static_cast<long long>(to), (static_cast<long long>(V) + off) / E - v0));  // vectors before it end inside the row
    const auto get = [&](int i, uint4 (&r)[4]) {
      if (i + 96 < whole && (v0 + i > 0 || off == 0)) {
        const char* at = base + (static_cast<long long>(v0) + i) * 16;
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = ldg_stream16(at + 512 * k);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) r[k] = i + 32 * k < to ? fetch(i + 32 * k) : neg_inf_vector<DT>();
      }
    };
    uint4 a[4], b[4];
    get(from, a);
    for (int i = from; i < to; i += 256) {
      get(i + 128, b);
      f(a);
      if (i + 128 >= to) break;
      get(i + 256, a);
      f(b);
    }
  }
  // f(token of the first entry, vector) likewise.
  template <class F>
  __device__ __forceinline__ void raw(F&& f) const {
    for (int i = begin + (threadIdx.x & 31); i < end; i += 32) f(token(i), at(i));
  }
  // f(token, value) for every entry of this lane.  Two words of a vector at a time: a long body in eight copies is more instructions than are fetched in the time they take.
  template <class F>
  __device__ __forceinline__ void entries(F&& f) const {
    for (int i = begin + (threadIdx.x & 31); i < end; i += 32) {
      uint4 r = at(i);
      int x = token(i);
#pragma unroll 1
      for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) f(x + e, entry<DT>(r, e));
        r.x = r.z;
        r.y = r.w;
        x += E / 2;
      }
    }
  }
};

// Everything that the work ahead in the stream wrote is there (launches take their places while it drains).
__device__ __forceinline__ void wait_for_inputs() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Behind that: the next launch may take its places when every block of this one has come here.  (Not sooner: one that starts on inputs which the work just ahead of it does not write
// relies on what lies before that being complete.)  Saves 0.5 us between small calls of one launch; calls of two lose up to 2.
__device__ __forceinline__ void let_next_launch() { asm volatile("griddepcontrol.launch_dependents;"); }

// ------------------------------------------------------------------------------------
// the cluster
// ------------------------------------------------------------------------------------
__device__ __forceinline__ void cluster_barrier_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void row_barrier(int parts) {
  if (parts > 1) {
    __syncwarp();
    cluster_barrier_arrive();
    cluster_barrier_wait();
  } else {
    __syncthreads();
  }
}
template <class T>
__device__ __forceinline__ T* of_rank(T* p, int rank) {
  return cg::this_cluster().map_shared_rank(p, rank);
}

// How a word is reduced over a warp and over a few words.  (Reductions of 32 bits in one instruction where they do: a shuffle is one for each warp and clock of the
// whole multiprocessor, so 64-bit words by shuffles take 16 warps 500 clocks a word.)
struct Add {  // below 2^64
  using OfBlocks = Add;
  static __device__ __forceinline__ u64 two(u64 a, u64 b) { return a + b; }
  static __device__ __forceinline__ u64 warp(u64 v) {
    const u64 lo = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v) & 0xffffffu);
    const u64 mid = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v >> 24) & 0xffffffu);
    const u64 hi = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(v >> 48));
    return lo + (mid << 24) + (hi << 48);
  }
  static constexpr u64 none = 0;
};
struct AddDouble {
  using OfBlocks = AddDouble;
  static __device__ __forceinline__ u64 two(u64 a, u64 b) {
    return static_cast<u64>(__double_as_longlong(__longlong_as_double(static_cast<long long>(a)) + __longlong_as_double(static_cast<long long>(b))));
  }
  static __device__ __forceinline__ u64 warp(u64 v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = two(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
  }
  static constexpr u64 none = 0;
};
struct Max {
  using OfBlocks = Max;
  static __device__ __forceinline__ u64 two(u64 a, u64 b) { return a > b ? a : b; }
  static __device__ __forceinline__ u64 warp(u64 v) {
    const unsigned hi = __reduce_max_sync(0xffffffffu, static_cast<unsigned>(v >> 32));
    const unsigned lo = __reduce_max_sync(0xffffffffu, static_cast<unsigned>(v >> 32) == hi ? static_cast<unsigned>(v) : 0u);
    return static_cast<u64>(hi) << 32 | lo;
  }
  static constexpr u64 none = 0;
};
struct Min {
  using OfBlocks = Min;
  static __device__ __forceinline__ u64 two(u64 a, u64 b) { return a < b ? a : b; }
  static __device__ __forceinline__ u64 warp(u64 v) { return ~Max::warp(~v); }
  static constexpr u64 none = ~0ull;
};
struct Nothing {  // a word that is not used
  using OfBlocks = Nothing;
  static __device__ __forceinline__ u64 two(u64, u64) { return 0; }
  static __device__ __forceinline__ u64 warp(u64) { return 0; }
  static constexpr u64 none = 0;
};
struct OfFirst {  // the sum of the blocks' first threads' words
  using OfBlocks = Add;
  static __device__ __forceinline__ u64 two(u64 a, u64 b) { return a + b; }
  static __device__ __forceinline__ u64 warp(u64 v) { return v; }
  static constexpr u64 none = 0;
};
__device__ __forceinline__ u64 bits_of(double v) { return static_cast<u64>(__double_as_longlong(v)); }
__device__ __forceinline__ double double_of(u64 v) { return __longlong_as_double(static_cast<long long>(v)); }

// Three words from every block of the row.  Used in turns: a block may write the next exchange while another still reads this one, not the one after
// (the barrier of the next one is between them).
struct Exchange {
  u64 a[2][kSliceParts], b[2][kSliceParts], c[2][kSliceParts];
  u64 warp_a[kSliceWarps], warp_b[kSliceWarps], warp_c[kSliceWarps];
};
struct Words {
  u64 a, b, c;
};
// The words reduced over the row, the same in every thread.  `turn` counts the exchanges of the kernel.  Every block has started (the caller has waited once for
// the cluster) and all threads come here.
template <class A, class B = Nothing, class C = Nothing>
__device__ __forceinline__ Words exchange(Exchange& x, int& turn, int parts, int rank, u64 a, u64 b = 0, u64 c = 0) {
  constexpr bool kB = !std::is_same<B, Nothing>::value, kC = !std::is_same<C, Nothing>::value;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = turn & 1;
  ++turn;
  a = A::warp(a);
  if (kB) b = B::warp(b);
  if (kC) c = C::warp(c);
  if (lane == 0) {
    x.warp_a[warp] = a;
    if (kB) x.warp_b[warp] = b;
    if (kC) x.warp_c[warp] = c;
  }
  __syncthreads();
  if (warp == 0) {
    const auto block = [&](auto word, const u64 (&of)[kSliceWarps]) {
      using W = decltype(word);
      if (std::is_same<W, OfFirst>::value) return of[0];
      return W::warp(lane < kSliceWarps ? of[lane & (kSliceWarps - 1)] : W::none);
    };
    a = block(A(), x.warp_a);
    if (kB) b = block(B(), x.warp_b);
    if (kC) c = block(C(), x.warp_c);
    if (parts == 1) {
      if (lane == 0) {
        x.a[t][0] = a;
        if (kB) x.b[t][0] = b;
        if (kC) x.c[t][0] = c;
      }
    } else if (lane < parts) {
      Exchange* o = of_rank(&x, lane);
      o->a[t][rank] = a;
      if (kB) o->b[t][rank] = b;
      if (kC) o->c[t][rank] = c;
    }
  }
  row_barrier(parts);
  const auto row = [&](auto word, const u64 (&of)[kSliceParts]) {  // (by every warp: a loop over the blocks takes longer)
    using W = typename decltype(word)::OfBlocks;
    return W::warp(lane < parts ? of[lane & (kSliceParts - 1)] : W::none);
  };
  Words w = {row(A(), x.a[t]), 0, 0};
  if (kB) w.b = row(B(), x.b[t]);
  if (kC) w.c = row(C(), x.c[t]);
  return w;
}

// How a row is cut up: as few blocks as `most` bytes of shared memory each allow (16 at most: what does not fit is read again where it is wanted), or more where
// all of them still have their places side by side (two a multiprocessor; of clusters of 8 and 16 there are places for 32 and 12 or so, since one lies in a
// group of 16 to 20 multiprocessors, and for 15 and 7 with a multiprocessor for each block), down to a vector a thread.  cluster: the blocks are one (a power of two).
struct SlicePlan {
  int parts, share, seg, res, sms;
  size_t smem;
};
// (a whole row for one block)
inline void plan_row(int vocab, int dtype, int warps, int* share, int* seg) {
  const int E = dtype == COS_DTYPE_F32 ? 4 : 8;
  *share = static_cast<int>((static_cast<long long>(vocab) + 2 * (E - 1)) / E);
  *seg = (*share + 32 * warps - 1) / (32 * warps) * 32;
}
cudaError_t slice_plan(int device, int rows, int vocab, int dtype, int most, bool cluster, SlicePlan* plan);

// Errors of the calls without a context (the text of cos_verify_last_error(NULL)).
cos_status call_failed(cos_status st, const char* what);
cos_status call_failed(const char* what, cudaError_t e);

// Whether rows that a call writes share an entry with rows that it reads, other than being the same ones (strides in entries of `bytes`; in: 0 for one row for all).
inline bool overlap(const void* in, long long stride_in, const void* out, long long stride_out, int rows, int vocab, int bytes) {
  const long long row = static_cast<long long>(vocab) * bytes, a = reinterpret_cast<long long>(in), b = reinterpret_cast<long long>(out), sa = stride_in * bytes, sb = stride_out * bytes;
  if (a == b) return rows > 1 && sa != sb;
  if (rows == 1) return a < b + row && b < a + row;
  if (b >= a + (rows - 1) * sa + row || a >= b + (rows - 1) * sb + row) return false;
  if (sa != sb) return true;
  const long long apart = ((b - a) % sa + sa) % sa;  // columns of one buffer
  return apart < row || apart > sa - row;
}

// log2(e) / T of a temperature in (0, 1e300), in 32 bits and as that number in 64.  Never 0 (at any temperature -inf is infinitely far, and 0 times it is not a number): 2^-149 from T = 2e45 on, at
// which differences of any two logits come to less than 5e-7.  Subnormal numbers are put together from their bits, since a thread may flush them.
struct Exponent {
  float c;
  double value;
};
inline Exponent exponent_of(double temperature) {
  const double c = fmin(1.4426950408889634 / temperature, 3e38);
  if (c >= FLT_MIN) return {static_cast<float>(c), static_cast<double>(static_cast<float>(c))};
  const unsigned units = static_cast<unsigned>(fmax(c * 0x1p149 + 0.5, 1.0));
  Exponent e = {0.0f, units * 0x1p-149};
  memcpy(&e.c, &units, sizeof(units));
  return e;
}

// The device of a call, made current for its duration.
struct OnDevice {
  int before = -1;
  cudaError_t error;
  explicit OnDevice(int device) {
    error = cudaGetDevice(&before);
    if (error == cudaSuccess && before != device) error = cudaSetDevice(device);
    if (error != cudaSuccess || before == device) before = -1;
  }
  ~OnDevice() {
    if (before >= 0) (void)cudaSetDevice(before);
  }
};

// most: of shared memory, that the kernel is ever launched with (the attribute is the kernel's, and calls of other threads may come between it and the launch: they all set the same)
template <class P>
cudaError_t slice_launch(void (*fn)(P), const P& p, int blocks, int parts, size_t smem, size_t most, cudaStream_t stream, int threads = kSliceThreads) {
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most));
  if (e == cudaSuccess && parts > 8) e = cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(static_cast<unsigned>(blocks), 1, 1);
  lc.blockDim = dim3(static_cast<unsigned>(threads), 1, 1);
  lc.dynamicSmemBytes = smem;
  lc.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = static_cast<unsigned>(parts);
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = parts > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&lc, fn, p);
}

}  // namespace cosv

#endif  // COS_SLICE_CUH
