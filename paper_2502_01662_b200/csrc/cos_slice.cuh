// A row of logits on a cluster of blocks: each block holds a slice of it in shared memory and sweeps it as often as it has to, and the
// blocks exchange what they found.
//
// A slice is a range of the row's 16-byte vectors, counted from the 16-byte boundary at or before the row's first entry, so every vector inside
// the row is one aligned load wherever the row starts; entries of the first and the last vector that are not the row's read as -inf.  A warp has a
// contiguous part of the slice and a lane every 32nd vector of it, the same in every sweep, so sweeps need no barrier between them.
#ifndef COS_SLICE_CUH
#define COS_SLICE_CUH

#include "cos_common.cuh"
#include "cos_draft.h"

namespace cosv {

constexpr int kSliceThreads = 512, kSliceWarps = kSliceThreads / 32, kSliceParts = 16;  // threads of a block, most blocks of a row
typedef unsigned long long u64;

template <int DT>
struct RowSlice {
  static constexpr int E = Elem<DT>::E;
  const char* base;  // the boundary
  int off, V;        // entries between it and the row, entries of the row
  int v0, nv;        // the slice's vectors
  int begin, end;    // this warp's part of them
  uint4* kept;       // the first `res` are here
  int res;

  // part of `parts` vectors each, parts / 16 warps' worth (a multiple of 32)
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

  // Brings the warp's part here; f(values) sees every vector on the way.
  template <class F>
  __device__ __forceinline__ void load(F&& f) const {
    constexpr int kAhead = 4;
    const int lane = threadIdx.x & 31;
    for (int i = begin + lane; i < end; i += 32 * kAhead) {
      uint4 r[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) r[k] = i + 32 * k < end ? fetch(i + 32 * k) : neg_inf_vector<DT>();
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (i + 32 * k < end && i + 32 * k < res) kept[i + 32 * k] = r[k];
        float v[E];
        Elem<DT>::unpack(r[k], v);
        f(v);
      }
    }
  }
  // f(token of the first entry, values) for every vector of this lane.
  template <class F>
  __device__ __forceinline__ void sweep(F&& f) const {
    for (int i = begin + (threadIdx.x & 31); i < end; i += 32) {
      const uint4 r = at(i);
      float v[E];
      Elem<DT>::unpack(r, v);
      f(token(i), v);
    }
  }
};

// ------------------------------------------------------------------------------------
// the cluster
// ------------------------------------------------------------------------------------
__device__ __forceinline__ void cluster_barrier_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void row_barrier(int parts) {
  if (parts > 1) {
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

__device__ __forceinline__ float max_nan(float a, float b) {  // NaN where one is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Two words from every block of the row.  Used in turns: a block may write the next exchange while another still reads this one, not the one after
// (the barrier of the next one is between them).
struct Exchange {
  u64 a[2][kSliceParts], b[2][kSliceParts];
  u64 warp_a[kSliceWarps], warp_b[kSliceWarps];
};

struct Words {
  u64 a, b;
};
// Both words reduced over the row (fa, fb: of two words), the same in every thread.  `turn` counts the exchanges of the kernel.  Every block has
// started (the caller has waited once for the cluster) and all threads come here.
template <class FA, class FB>
__device__ __forceinline__ Words exchange(Exchange& x, int& turn, int parts, int rank, u64 a, u64 b, FA&& fa, FB&& fb) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a = fa(a, __shfl_xor_sync(0xffffffffu, a, d));
    b = fb(b, __shfl_xor_sync(0xffffffffu, b, d));
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = turn & 1;
  ++turn;
  if (lane == 0) {
    x.warp_a[warp] = a;
    x.warp_b[warp] = b;
  }
  __syncthreads();
  if (warp == 0) {
    a = x.warp_a[lane & (kSliceWarps - 1)];
    b = x.warp_b[lane & (kSliceWarps - 1)];
#pragma unroll
    for (int d = kSliceWarps / 2; d > 0; d >>= 1) {
      a = fa(a, __shfl_xor_sync(0xffffffffu, a, d));
      b = fb(b, __shfl_xor_sync(0xffffffffu, b, d));
    }
    if (parts == 1) {
      if (lane == 0) {
        x.a[t][0] = a;
        x.b[t][0] = b;
      }
    } else if (lane < parts) {
      *of_rank(&x.a[t][rank], lane) = a;
      *of_rank(&x.b[t][rank], lane) = b;
    }
  }
  row_barrier(parts);
  Words w = {x.a[t][0], x.b[t][0]};
  for (int r = 1; r < parts; ++r) {
    w.a = fa(w.a, x.a[t][r]);
    w.b = fb(w.b, x.b[t][r]);
  }
  return w;
}

// How many of `rows` rows' blocks: the fewest that fill the device twice over, within what a slice's shared memory and its least size allow.
struct SlicePlan {
  int parts, share, seg, res;
  size_t smem;
};
cudaError_t slice_plan(int device, int rows, int vocab, int dtype, SlicePlan* plan);

// Errors of the calls without a context (the text of cos_verify_last_error(NULL)).
cos_status call_failed(cos_status st, const char* what);
cos_status call_failed(const char* what, cudaError_t e);

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

template <class P>
cudaError_t slice_launch(void (*fn)(P), const P& p, int blocks, int parts, size_t smem, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e == cudaSuccess && parts > 8) e = cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(static_cast<unsigned>(blocks), 1, 1);
  lc.blockDim = dim3(kSliceThreads, 1, 1);
  lc.dynamicSmemBytes = smem;
  lc.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = static_cast<unsigned>(parts);
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = parts > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&lc, fn, p);
}

}  // namespace cosv

#endif  // COS_SLICE_CUH
