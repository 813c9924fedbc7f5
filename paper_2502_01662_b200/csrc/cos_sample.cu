// Drawing a token from a row of logits at a temperature, after top-k, top-p and min-p, and listing the largest logits of a row: one launch, a
// cluster of blocks a row (cos_slice.cuh).
//
// Mathematics.  In order of (logit down, index up) every one of the three limits keeps a beginning of the line, so what is kept is the tokens at or
// above one of them; a token's place in the line is one 64-bit number (`place_of`).  The limit is found by a histogram of 2048 bins, linear in the
// logit below the maximum: the bin in which the k-th token lies, or the one in which the sum of the weights reaches p, then (usually a handful of tokens)
// the places in that bin against each other.  A bin of more than kCandidates is cut into 2048 ranges of places, again until few are left: places
// are 64 bits and no two are alike, so this ends after at most six histograms, for any number of equal logits.
//
// Weights are exp2 of 64-bit arguments, from a table of 2^(j/64) and the power series of 2^r for |r| <= 1/128 (the fifth term is below 4e-14), rounded to
// whole multiples of 2^-scale and summed as integers: a token is drawn where a border of the cumulative sums lies next to u, and 32-bit sums are off by more
// than the weight of a token there.  Integers make sums independent of their order, so atomics and the split over blocks change nothing.
#include "cos_slice.cuh"

namespace cosv {
namespace {

constexpr int kBins = 2048, kCandidates = 512, kTopCandidates = COS_TOP_MAX + 512;

struct Common {  // of both kernels
  const void* logits;
  long long stride;
  int V, parts, share, seg, res;
};

struct SampleParams {
  Common c;
  const float* u;
  float T, p, min_p;
  int k;
  const float *row_T, *row_p, *row_min_p;
  const int* row_k;
  int* tokens;
  float* prob;
  int* kept;
  unsigned* status;
  char* filtered;
  long long stride_filtered;
};

struct TopParams {
  Common c;
  int k;
  float T;
  float* values;
  int* ids;
  float* lse;
};

// A float as an unsigned integer of the same order (equal zeros), and back.
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned u = __float_as_uint(v + 0.0f);
  return u ^ (static_cast<unsigned>(static_cast<int>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(unsigned k) { return __uint_as_float(k ^ ((k & 0x80000000u) ? 0x80000000u : 0xffffffffu)); }
// A token's place in the line: the larger the earlier.
__device__ __forceinline__ u64 place_of(float v, int token) { return static_cast<u64>(ordered(v)) << 32 | (0xffffffffu - static_cast<unsigned>(token)); }
__device__ __forceinline__ float logit_at(u64 place) { return unordered(static_cast<unsigned>(place >> 32)); }
__device__ __forceinline__ int token_at(u64 place) { return static_cast<int>(0xffffffffu - static_cast<unsigned>(place)); }

// exp((l - m) / T) in units of 2^-scale.
struct Weight {
  double m, c;       // the row's largest logit, log2(e) / T
  const double* table;  // 2^(j / 64)
  int scale;
  __device__ __forceinline__ double of(float l) const {  // not rounded to the unit; l is finite
    constexpr double kRound = 105553116266496.0;         // 1.5 * 2^46: sums with it are multiples of 2^-6
    const double t = fmax((static_cast<double>(l) - m) * c, -900.0);
    const double k = t + kRound;
    const double r = t - (k - kRound);
    const int n = __double2loint(k);
    double e = fma(0.009618129107628477, r, 0.05550410866482158);  // ln(2)^i / i!
    e = fma(e, r, 0.2402265069591007);
    e = fma(e, r, 0.6931471805599453);
    e = fma(e, r, 1.0);
    e *= table[n & 63];
    return __hiloint2double(__double2hiint(e) + (((n >> 6) + scale) << 20), __double2loint(e));
  }
  static __device__ __forceinline__ u64 whole(double w) {  // w <= 2^46
    return static_cast<u64>(__double_as_longlong(w + 4503599627370496.0)) & 0xfffffffffffffull;
  }
};

struct Found {
  u64 before_count, before_mass, count;
  int bin, there;
};

template <int kList, int kMasses>
struct Histogram {
  unsigned count[kBins], mass_lo[kBins], mass_hi[kBins];
  u64 list[kList];    // this block's candidates
  u64 merged[kList];  // the row's
  u64 mass[kMasses];
  u64 scan_count[kSliceWarps], scan_mass[kSliceWarps];
  int listed, pad[3];
  Found found[2];
};

using SampleShared = Histogram<kCandidates, kCandidates>;
using TopShared = Histogram<kTopCandidates, 2>;
static_assert(sizeof(SampleShared) % 16 == 0 && sizeof(TopShared) % 16 == 0, "the slice lies behind it");

// The bins of this block's share of the row's histogram, four a thread at most, with what lies before them in the line.
struct Bins {
  int first, n;  // this thread's
  u64 count[4], mass[4], before_count, before_mass;
  u64 all_count, all_mass;  // of the row
};

template <class H>
__device__ __forceinline__ void clear_bins(H& h, bool masses) {
  for (int i = threadIdx.x; i < kBins; i += kSliceThreads) {
    h.count[i] = 0;
    if (masses) h.mass_lo[i] = h.mass_hi[i] = 0;
  }
  __syncthreads();
}

template <class H>
__device__ __forceinline__ void add_to_bin(H& h, int bin, bool masses, u64 w) {
  atomicAdd(&h.count[bin], 1u);
  if (masses) {  // 64 bits in two words: whoever makes the low one overflow carries
    const unsigned lo = static_cast<unsigned>(w);
    const unsigned was = atomicAdd(&h.mass_lo[bin], lo);
    const unsigned hi = static_cast<unsigned>(w >> 32) + (was + lo < was ? 1u : 0u);
    if (hi) atomicAdd(&h.mass_hi[bin], hi);
  }
}

struct Add {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a + b; }
};
struct Max {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a > b ? a : b; }
};
struct Min {
  __device__ __forceinline__ u64 operator()(u64 a, u64 b) const { return a < b ? a : b; }
};

// Behind the sweep that filled the blocks' bins: the sums over the blocks, in order.  The bins may be cleared afterwards.
template <class H>
__device__ __forceinline__ void merge_bins(H& h, Exchange& x, int& turn, int parts, int rank, bool masses, Bins& b) {
  row_barrier(parts);
  const int own = kBins / parts, each = own > kSliceThreads ? own / kSliceThreads : 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  b.n = tid * each < own ? each : 0;
  b.first = rank * own + tid * each;
  u64 count = 0, mass = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    b.count[q] = b.mass[q] = 0;
    if (q < b.n) {
      if (parts == 1) {
        b.count[q] = h.count[b.first + q];
        if (masses) b.mass[q] = static_cast<u64>(h.mass_hi[b.first + q]) << 32;
        if (masses) b.mass[q] += h.mass_lo[b.first + q];
      } else {
#pragma unroll 4
        for (int r = 0; r < parts; ++r) {
          const H* o = of_rank(&h, r);
          b.count[q] += o->count[b.first + q];
          if (masses) b.mass[q] += (static_cast<u64>(o->mass_hi[b.first + q]) << 32) + o->mass_lo[b.first + q];
        }
      }
    }
    count += b.count[q];
    mass += b.mass[q];
  }
  // exclusive scan over the block
  u64 sc = count, sm = mass;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u64 c = __shfl_up_sync(0xffffffffu, sc, d), m = __shfl_up_sync(0xffffffffu, sm, d);
    if (lane >= d) {
      sc += c;
      sm += m;
    }
  }
  if (lane == 31) {
    h.scan_count[warp] = sc;
    h.scan_mass[warp] = sm;
  }
  const int t = turn & 1;
  exchange(x, turn, parts, rank, count, mass, Add(), Add());  // (its barriers are this scan's too)
  sc -= count;
  sm -= mass;
  for (int w = 0; w < warp; ++w) {
    sc += h.scan_count[w];
    sm += h.scan_mass[w];
  }
  b.all_count = b.all_mass = 0;
  for (int r = 0; r < parts; ++r) {
    if (r < rank) {
      sc += x.a[t][r];
      sm += x.b[t][r];
    }
    b.all_count += x.a[t][r];
    b.all_mass += x.b[t][r];
  }
  b.before_count = sc;
  b.before_mass = sm;
}

// The bin in which the `target`-th token (by_mass: unit of mass) lies; 1 <= target <= what the row has.  `slot`: used in turns.
template <class H>
__device__ __forceinline__ Found locate(H& h, const Bins& b, int parts, bool by_mass, u64 target, int slot) {
  u64 c = b.before_count, m = b.before_mass;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const u64 at = by_mass ? m : c, here = by_mass ? b.mass[q] : b.count[q];
    if (q < b.n && at < target && target <= at + here) {
      const Found f = {c, m, b.count[q], b.first + q, 1};
      if (parts == 1)
        h.found[slot] = f;
      else
        for (int r = 0; r < parts; ++r) *of_rank(&h.found[slot], r) = f;
    }
    c += b.count[q];
    m += b.mass[q];
  }
  row_barrier(parts);
  return h.found[slot];
}

// The places of the tokens that `in` holds, all of them to every block of the row: h.merged[0 .. n).  There are no more than the list has room for.
template <class H, class S, class In>
__device__ __forceinline__ int gather(H& h, Exchange& x, int& turn, int parts, int rank, const S& s, In&& in) {
  if (threadIdx.x == 0) h.listed = 0;
  __syncthreads();
  s.sweep([&](int token, const auto& v) {
#pragma unroll
    for (int e = 0; e < S::E; ++e)
      if (in(v[e], token + e)) h.list[atomicAdd(&h.listed, 1)] = place_of(v[e], token + e);
  });
  __syncthreads();
  const int mine = h.listed, t = turn & 1;
  exchange(x, turn, parts, rank, threadIdx.x == 0 ? mine : 0, 0, Add(), Add());
  int n = 0;
  for (int r = 0; r < parts; ++r) n += static_cast<int>(x.a[t][r]);
  for (int i = threadIdx.x; i < n; i += kSliceThreads) {
    int r = 0, j = i;
    while (j >= static_cast<int>(x.a[t][r])) j -= static_cast<int>(x.a[t][r++]);
    h.merged[i] = parts == 1 ? h.list[j] : *of_rank(&h.list[j], r);
  }
  __syncthreads();
  return n;
}

// Where in the line a bin's tokens lie, cut down until no more than `most` of them are left.
struct Range {
  u64 lo, hi;  // places, inclusive
  u64 before_count, before_mass, count;
};
template <class H, class S, class In>
__device__ __forceinline__ Range narrow(H& h, Exchange& x, int& turn, int& slot, int parts, int rank, const S& s, const Weight* w, bool by_mass, u64 target, const Found& f, u64 most, In&& in) {
  Range g = {~0ull, 0, f.before_count, f.before_mass, f.count};
  s.sweep([&](int token, const auto& v) {
#pragma unroll
    for (int e = 0; e < S::E; ++e)
      if (in(v[e], token + e)) {
        const u64 at = place_of(v[e], token + e);
        g.lo = at < g.lo ? at : g.lo;
        g.hi = at > g.hi ? at : g.hi;
      }
  });
  const Words ends = exchange(x, turn, parts, rank, g.lo, g.hi, Min(), Max());
  g.lo = ends.a;
  g.hi = ends.b;
  while (g.count > most) {
    const int bits = 64 - __clzll(static_cast<long long>(g.hi - g.lo)), shift = bits > 11 ? bits - 11 : 0;
    clear_bins(h, by_mass);
    s.sweep([&](int token, const auto& v) {
#pragma unroll
      for (int e = 0; e < S::E; ++e) {
        const u64 at = place_of(v[e], token + e);
        if (v[e] > -INFINITY && token + e >= 0 && at >= g.lo && at <= g.hi)
          add_to_bin(h, static_cast<int>((g.hi - at) >> shift), by_mass, by_mass ? Weight::whole(w->of(v[e])) : 0);
      }
    });
    Bins b;
    merge_bins(h, x, turn, parts, rank, by_mass, b);
    const Found sub = locate(h, b, parts, by_mass, target - (by_mass ? g.before_mass : g.before_count), slot);
    slot ^= 1;
    g.before_count += sub.before_count;
    g.before_mass += sub.before_mass;
    g.count = sub.count;
    const u64 top = g.hi - (static_cast<u64>(sub.bin) << shift), low = top - ((1ull << shift) - 1);
    g.hi = top;
    g.lo = low > g.lo && low <= top ? low : g.lo;
  }
  return g;
}

// The last place of the line that is kept, by count (the first `target` tokens) or by mass (while what lies before is below `target`), given the bin that
// `target` falls into; and the mass up to and with it.
struct Limit {
  u64 place, mass;
};
template <class H, class S, class In>
__device__ __forceinline__ Limit limit_in(H& h, Exchange& x, int& turn, int& slot, int parts, int rank, const S& s, const Weight& w, bool by_mass, bool masses, u64 target, const Found& f, In&& in) {
  Range g = {0, 0, f.before_count, f.before_mass, f.count};
  int n;
  if (f.count <= kCandidates) {
    n = gather(h, x, turn, parts, rank, s, in);
  } else {
    g = narrow(h, x, turn, slot, parts, rank, s, &w, by_mass, target, f, kCandidates, in);
    // (masses before a range found by counts are not known: they are summed up where they are wanted)
    n = gather(h, x, turn, parts, rank, s, [&](float v, int token) {
      const u64 at = place_of(v, token);
      return v > -INFINITY && token >= 0 && at >= g.lo && at <= g.hi;
    });
    if (masses && !by_mass) {
      u64 sum = 0;
      s.sweep([&](int token, const auto& v) {
#pragma unroll
        for (int e = 0; e < S::E; ++e)
          if (v[e] > -INFINITY && token + e >= 0 && place_of(v[e], token + e) > g.hi) sum += Weight::whole(w.of(v[e]));
      });
      g.before_mass = exchange(x, turn, parts, rank, sum, 0, Add(), Add()).a;
    }
  }
  const int i = threadIdx.x;  // (kCandidates == kSliceThreads)
  const u64 mine = i < n ? h.merged[i] : 0;
  const u64 weight = i < n && masses ? Weight::whole(w.of(logit_at(mine))) : 0;
  h.mass[i] = weight;
  __syncthreads();
  u64 rank_of = g.before_count, mass = g.before_mass;
  for (int j = 0; j < n; ++j)
    if (h.merged[j] > mine) {
      ++rank_of;
      mass += h.mass[j];
    }
  // the tokens of the list that are kept: their last place, and the largest sum with one of them
  const bool kept = i < n && (by_mass ? mass < target : rank_of < target);
  u64 last = kept ? mine : ~0ull, sum = kept ? mass + weight : 0;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    last = Min()(last, __shfl_xor_sync(0xffffffffu, last, d));
    sum = Max()(sum, __shfl_xor_sync(0xffffffffu, sum, d));
  }
  if ((i & 31) == 0) {
    h.scan_count[i >> 5] = last;
    h.scan_mass[i >> 5] = sum;
  }
  __syncthreads();
  Limit l = {~0ull, 0};
  for (int k = 0; k < kSliceWarps; ++k) {
    l.place = Min()(l.place, h.scan_count[k]);
    l.mass = Max()(l.mass, h.scan_mass[k]);
  }
  __syncthreads();
  return l;
}

// The row's entries that f(value, token) keeps, -inf in place of the others.
template <int DT, class F>
__device__ __forceinline__ void write_filtered(const RowSlice<DT>& s, char* row, F&& f) {
  constexpr int E = Elem<DT>::E, B = Elem<DT>::bytes;
  const unsigned none = DT == COS_DTYPE_F32 ? 0xff800000u : (DT == COS_DTYPE_BF16 ? 0xff80u : 0xfc00u);
  const int lane = threadIdx.x & 31;
  const bool whole = static_cast<int>(reinterpret_cast<unsigned long long>(row) & 15) / B == s.off;
  for (int i = s.begin + lane; i < s.end; i += 32) {
    uint4 r = s.at(i);
    float v[E];
    Elem<DT>::unpack(r, v);
    const int x = s.token(i);
    unsigned* w = reinterpret_cast<unsigned*>(&r);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (!f(v[e], x + e)) {
        if (DT == COS_DTYPE_F32)
          w[e] = none;
        else
          w[e >> 1] = (e & 1) ? ((w[e >> 1] & 0xffffu) | none << 16) : ((w[e >> 1] & 0xffff0000u) | none);
      }
    char* at = row + static_cast<long long>(x) * B;
    if (whole && x >= 0 && x <= s.V - E) {
      *reinterpret_cast<uint4*>(at) = r;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (x + e >= 0 && x + e < s.V) {
          if (DT == COS_DTYPE_F32)
            reinterpret_cast<unsigned*>(at)[e] = w[e];
          else
            reinterpret_cast<unsigned short*>(at)[e] = static_cast<unsigned short>((e & 1) ? w[e >> 1] >> 16 : w[e >> 1]);
        }
    }
  }
}

// The largest entry (NaN where there is one) of the row, brought here on the way.
template <int DT>
__device__ __forceinline__ float load_max(const RowSlice<DT>& s, Exchange& x, int& turn, int parts, int rank) {
  float m = -INFINITY;
  s.load([&](const float (&v)[RowSlice<DT>::E]) {
#pragma unroll
    for (int e = 0; e < RowSlice<DT>::E; ++e) m = max_nan(m, v[e]);
  });
  if (parts > 1) cluster_barrier_wait();  // (every block of the row has started)
  const auto larger = [](u64 a, u64 b) {
    return static_cast<u64>(__float_as_uint(max_nan(__uint_as_float(static_cast<unsigned>(a)), __uint_as_float(static_cast<unsigned>(b)))));
  };
  return __uint_as_float(static_cast<unsigned>(exchange(x, turn, parts, rank, __float_as_uint(m), 0, larger, Max()).a));
}

template <int DT>
__global__ void __launch_bounds__(kSliceThreads, 2) cos_sample_kernel(const SampleParams p) {
  extern __shared__ uint4 smem[];
  SampleShared& h = *reinterpret_cast<SampleShared*>(smem);
  __shared__ Exchange x;
  __shared__ double table[64];
  const int parts = p.c.parts, rank = blockIdx.x % parts, row = blockIdx.x / parts, tid = threadIdx.x;
  if (parts > 1) cluster_barrier_arrive();
  int turn = 0, slot = 0;
  if (tid < 64) table[tid] = exp2(static_cast<double>(tid) / 64.0);
  RowSlice<DT> s;
  s.init(static_cast<const char*>(p.c.logits) + static_cast<long long>(row) * p.c.stride * Elem<DT>::bytes, p.c.V, rank, p.c.share, p.c.seg, smem + sizeof(h) / 16, p.c.res);
  const float T = p.row_T ? p.row_T[row] : p.T;
  const float m = load_max(s, x, turn, parts, rank);
  char* const filtered = p.filtered ? p.filtered + static_cast<long long>(row) * p.stride_filtered * Elem<DT>::bytes : nullptr;

  if (!(m > -INFINITY && m < INFINITY) || !(T >= 0.0f)) {
    if (rank == 0 && tid == 0) {
      p.tokens[row] = -1;
      if (p.prob) p.prob[row] = __int_as_float(0x7fc00000);
      if (p.kept) p.kept[row] = 0;
      if (p.status) p.status[row] = COS_ROW_NONFINITE;
    }
    if (filtered) write_filtered<DT>(s, filtered, [](float, int) { return true; });
    return;
  }

  if (T == 0.0f) {
    u64 first = ~0ull;
    s.sweep([&](int token, const auto& v) {
#pragma unroll
      for (int e = 0; e < RowSlice<DT>::E; ++e)
        if (v[e] == m && static_cast<u64>(token + e) < first) first = static_cast<u64>(token + e);
    });
    const int token = static_cast<int>(exchange(x, turn, parts, rank, first, 0, Min(), Max()).a);
    if (rank == 0 && tid == 0) {
      p.tokens[row] = token;
      if (p.prob) p.prob[row] = 1.0f;
      if (p.kept) p.kept[row] = 1;
      if (p.status) p.status[row] = 0;
    }
    if (filtered) write_filtered<DT>(s, filtered, [&](float, int t) { return t == token; });
    return;
  }

  int k = p.row_k ? p.row_k[row] : p.k;
  if (k <= 0 || k > p.c.V) k = p.c.V;
  const float top_p = p.row_p ? p.row_p[row] : p.p, min_raw = p.row_min_p ? p.row_min_p[row] : p.min_p;
  const bool by_p = top_p < 1.0f;
  Weight w = {static_cast<double>(m), 1.4426950408889634 / static_cast<double>(T), table, min(46, 63 - (32 - __clz(p.c.V - 1)))};
  const double least = ldexp(min_raw > 0.0f ? fmin(static_cast<double>(min_raw), 1.0) : 0.0, w.scale);

  // the last place that is kept; nothing at -inf is
  u64 last = static_cast<u64>(ordered(-INFINITY) + 1) << 32;
  if (k < p.c.V || by_p) {
    // bins of 1/32 of a power of two of the weight where sums of weights are wanted, else of 1/64 of a logit
    const float per = by_p ? fminf(46.166241f / T, 1e30f) : 64.0f;
    const auto bin_of = [&](float v) { return min(static_cast<int>((m - v) * per), kBins - 1); };
    clear_bins(h, by_p);
    s.sweep([&](int, const auto& v) {
#pragma unroll
      for (int e = 0; e < RowSlice<DT>::E; ++e)
        if (v[e] > -INFINITY) add_to_bin(h, bin_of(v[e]), by_p, by_p ? Weight::whole(w.of(v[e])) : 0);
    });
    Bins b;
    merge_bins(h, x, turn, parts, rank, by_p, b);
    u64 mass = b.all_mass;
    if (static_cast<u64>(k) < b.all_count) {
      const Found f = locate(h, b, parts, false, k, slot);
      slot ^= 1;
      const Limit l = limit_in(h, x, turn, slot, parts, rank, s, w, false, by_p, k, f, [&](float v, int) { return v > -INFINITY && bin_of(v) == f.bin; });
      last = l.place;
      mass = l.mass;
    }
    if (by_p) {
      const double want = ceil(static_cast<double>(fmaxf(top_p, 0.0f)) * static_cast<double>(mass));
      u64 target = want < 1.0 ? 1 : static_cast<u64>(want);  // (the first one is kept in any case; NaN counts as no limit above)
      if (target < mass) {
        const Found f = locate(h, b, parts, true, target, slot);
        slot ^= 1;
        const Limit l = limit_in(h, x, turn, slot, parts, rank, s, w, true, true, target, f, [&](float v, int) { return v > -INFINITY && bin_of(v) == f.bin; });
        last = Max()(last, l.place);
      }
    }
  }

  // what is kept, in order of the index
  const auto keeps = [&](float v, int token) { return place_of(v, token) >= last && v > -INFINITY; };
  u64 mine = 0, kept = 0;
  s.sweep([&](int token, const auto& v) {
#pragma unroll
    for (int e = 0; e < RowSlice<DT>::E; ++e)
      if (keeps(v[e], token + e)) {
        const double we = w.of(v[e]);
        if (we >= least) {
          mine += Weight::whole(we);
          ++kept;
        }
      }
  });
  const int t = turn & 1;
  const Words all = exchange(x, turn, parts, rank, mine, kept, Add(), Add());
  const double u = static_cast<double>(p.u[row]);
  const double want = ceil(fmin(fmax(u, 0.0), 1.0) * static_cast<double>(all.a));
  const u64 target = want >= static_cast<double>(all.a) ? all.a : (want < 1.0 ? 1 : static_cast<u64>(want));
  u64 before = 0;
  for (int r = 0; r < rank; ++r) before += x.a[t][r];
  if (before < target && target <= before + x.a[t][rank]) {
    const int lane = tid & 31, warp = tid >> 5;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
    if (lane == 0) h.scan_mass[warp] = mine;
    __syncthreads();
    for (int i = 0; i < warp; ++i) before += h.scan_mass[i];
    if (before < target && target <= before + mine) {  // this warp has it
      const int steps = (s.end - s.begin + 31) / 32;
      for (int q = 0; q < steps; ++q) {
        const int i = s.begin + q * 32 + lane;
        const uint4 r = i < s.end ? s.at(i) : neg_inf_vector<DT>();
        float v[RowSlice<DT>::E];
        Elem<DT>::unpack(r, v);
        const int token = s.token(i);
        u64 sum = 0;
#pragma unroll
        for (int e = 0; e < RowSlice<DT>::E; ++e)
          if (keeps(v[e], token + e)) {
            const double we = w.of(v[e]);
            if (we >= least) sum += Weight::whole(we);
          }
        u64 up = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const u64 o = __shfl_up_sync(0xffffffffu, up, d);
          if (lane >= d) up += o;
        }
        const unsigned reached = __ballot_sync(0xffffffffu, before + up >= target);
        if (reached) {
          if (lane == __ffs(reached) - 1) {
            u64 at = before + up - sum;
            bool open = true;
#pragma unroll
            for (int e = 0; e < RowSlice<DT>::E; ++e)
              if (open && keeps(v[e], token + e)) {
                const double we = w.of(v[e]);
                if (we >= least) at += Weight::whole(we);
                if (we >= least && at >= target) {
                  open = false;
                  p.tokens[row] = token + e;
                  if (p.prob) p.prob[row] = static_cast<float>(we / static_cast<double>(all.a));
                }
              }
          }
          break;
        }
        before += __shfl_sync(0xffffffffu, up, 31);
      }
    }
  }
  if (rank == 0 && tid == 0) {
    if (p.kept) p.kept[row] = static_cast<int>(all.b);
    if (p.status) p.status[row] = 0;
  }
  if (filtered) {
    // (the weight is at the minimum or above it: tested by it where the two are close, since the logits of the type are)
    write_filtered<DT>(s, filtered, [&](float v, int token) { return keeps(v, token) && (least == 0.0 || w.of(v) >= least); });
  }
}

template <int DT>
__global__ void __launch_bounds__(kSliceThreads, 2) cos_top_kernel(const TopParams p) {
  extern __shared__ uint4 smem[];
  TopShared& h = *reinterpret_cast<TopShared*>(smem);
  __shared__ Exchange x;
  const int parts = p.c.parts, rank = blockIdx.x % parts, row = blockIdx.x / parts, tid = threadIdx.x;
  if (parts > 1) cluster_barrier_arrive();
  int turn = 0, slot = 0;
  RowSlice<DT> s;
  s.init(static_cast<const char*>(p.c.logits) + static_cast<long long>(row) * p.c.stride * Elem<DT>::bytes, p.c.V, rank, p.c.share, p.c.seg, smem + sizeof(h) / 16, p.c.res);
  const float m = load_max(s, x, turn, parts, rank);
  float* const values = p.values + static_cast<long long>(row) * p.k;
  int* const ids = p.ids + static_cast<long long>(row) * p.k;
  if (!(m > -INFINITY && m < INFINITY)) {
    if (rank == 0) {
      for (int i = tid; i < p.k; i += kSliceThreads) {
        values[i] = -INFINITY;
        ids[i] = -1;
      }
      if (tid == 0) p.lse[row] = m == -INFINITY ? -INFINITY : __int_as_float(0x7fc00000);
    }
    return;
  }
  const auto bin_of = [&](float v) { return min(static_cast<int>((m - v) * 64.0f), kBins - 1); };
  const float c = fminf(static_cast<float>(1.4426950408889634 / static_cast<double>(p.T)), 3e38f);
  clear_bins(h, false);
  double sum = 0.0;
  s.sweep([&](int, const auto& v) {
    float part = 0.0f;  // (of a vector: eight terms of at most 1)
#pragma unroll
    for (int e = 0; e < RowSlice<DT>::E; ++e)
      if (v[e] > -INFINITY) {
        part += ex2_approx((v[e] - m) * c);
        add_to_bin(h, bin_of(v[e]), false, 0);
      }
    sum += static_cast<double>(part);
  });
  const auto add = [](u64 a, u64 b) {
    return static_cast<u64>(__double_as_longlong(__longlong_as_double(static_cast<long long>(a)) + __longlong_as_double(static_cast<long long>(b))));
  };
  const Words sums = exchange(x, turn, parts, rank, static_cast<u64>(__double_as_longlong(sum)), 0, add, Max());
  if (rank == 0 && tid == 0)
    p.lse[row] = static_cast<float>(static_cast<double>(m) / static_cast<double>(p.T) + log(__longlong_as_double(static_cast<long long>(sums.a))));
  Bins b;
  merge_bins(h, x, turn, parts, rank, false, b);
  int n;
  if (static_cast<u64>(p.k) < b.all_count) {
    const Found f = locate(h, b, parts, false, p.k, slot);
    slot ^= 1;
    if (f.before_count + f.count <= kTopCandidates) {
      n = gather(h, x, turn, parts, rank, s, [&](float v, int) { return v > -INFINITY && bin_of(v) <= f.bin; });
    } else {
      const Range g = narrow(h, x, turn, slot, parts, rank, s, static_cast<const Weight*>(nullptr), false, p.k, f, kTopCandidates - COS_TOP_MAX,
                             [&](float v, int) { return v > -INFINITY && bin_of(v) == f.bin; });
      n = gather(h, x, turn, parts, rank, s, [&](float v, int token) { return v > -INFINITY && token >= 0 && place_of(v, token) >= g.lo; });
    }
  } else {
    n = gather(h, x, turn, parts, rank, s, [&](float v, int) { return v > -INFINITY; });
  }
  for (int i = rank * kSliceThreads + tid; i < n; i += parts * kSliceThreads) {
    const u64 mine = h.merged[i];
    int at = 0;
    for (int j = 0; j < n; ++j) at += h.merged[j] > mine;
    if (at < p.k) {
      values[at] = logit_at(mine);
      ids[at] = token_at(mine);
    }
  }
  if (rank == 0)
    for (int i = n + tid; i < p.k; i += kSliceThreads) {
      values[i] = -INFINITY;
      ids[i] = -1;
    }
  row_barrier(parts);  // (no block leaves while another reads its list)
}

// What the host can see of the rows that both calls take.
cos_status check_rows(const void* logits, long long stride, int rows, int vocab, int dtype) {
  if (!logits) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (rows < 1 || vocab < 1 || vocab > 0x7ffffff0) return call_failed(COS_ERR_INVALID_ARG, "rows and vocab must be positive");
  if (dtype < COS_DTYPE_F32 || dtype > COS_DTYPE_F16) return call_failed(COS_ERR_INVALID_ARG, "unknown dtype");
  if (rows > 1 && stride < vocab) return call_failed(COS_ERR_INVALID_ARG, "rows overlap: stride_row is less than vocab");
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == COS_DTYPE_F32 ? 4 : 2)) return call_failed(COS_ERR_ALIGNMENT, "logits pointer not aligned to its element type");
  return COS_OK;
}

template <class P, class F>
cos_status launch_rows(P& p, int rows, int vocab, int dtype, int device, size_t shared, cudaStream_t stream, F&& kernel_of) {
  OnDevice on(device);
  if (on.error != cudaSuccess) return call_failed("cudaSetDevice", on.error);
  SlicePlan plan;
  cudaError_t e = slice_plan(device, rows, vocab, dtype, &plan);
  if (e != cudaSuccess) return call_failed("device query", e);
  if (static_cast<long long>(rows) * plan.parts > 0x7fffffffll) return call_failed(COS_ERR_UNSUPPORTED, "too many rows for one launch");
  p.c.V = vocab;
  p.c.parts = plan.parts;
  p.c.share = plan.share;
  p.c.seg = plan.seg;
  p.c.res = plan.res;
  e = slice_launch(kernel_of(dtype), p, rows * plan.parts, plan.parts, shared + plan.smem, stream);
  return e == cudaSuccess ? COS_OK : call_failed("launch", e);
}

bool misaligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

}  // namespace

cudaError_t slice_plan(int device, int rows, int vocab, int dtype, SlicePlan* plan) {
  int sms = 0;
  const cudaError_t e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (e != cudaSuccess) return e;
  constexpr long long kMostKept = 64 * 1024 / 16;  // vectors: two blocks of a multiprocessor have room for that beside their histograms
  const int E = dtype == COS_DTYPE_F32 ? 4 : 8;
  const long long all = (static_cast<long long>(vocab) + 2 * (E - 1)) / E;
  int parts = 1;
  while (parts < kSliceParts && ((all + parts - 1) / parts > kMostKept || (static_cast<long long>(rows) * parts < 2 * sms && all / parts >= 512))) parts *= 2;
  plan->parts = parts;
  plan->share = static_cast<int>((all + parts - 1) / parts);
  plan->seg = static_cast<int>((plan->share + 32 * kSliceWarps - 1) / (32 * kSliceWarps) * 32);
  plan->res = static_cast<int>(plan->share < kMostKept ? plan->share : kMostKept);
  plan->smem = static_cast<size_t>(plan->res) * 16;
  return cudaSuccess;
}

}  // namespace cosv

using namespace cosv;

extern "C" cos_status cos_sample(const cos_sample_args* a, void* cuda_stream) {
  if (!a) return call_failed(COS_ERR_INVALID_ARG, "null argument");
  const cos_status st = check_rows(a->logits, a->stride_row, a->rows, a->vocab, a->dtype);
  if (st != COS_OK) return st;
  if (!a->uniforms || !a->tokens) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (!a->row_temperature && !(a->temperature >= 0.0f)) return call_failed(COS_ERR_INVALID_ARG, "temperature must be >= 0");
  if (!a->row_top_p && !(a->top_p > 0.0f)) return call_failed(COS_ERR_INVALID_ARG, "top_p must be > 0");
  if (!a->row_min_p && !(a->min_p >= 0.0f && a->min_p <= 1.0f)) return call_failed(COS_ERR_INVALID_ARG, "min_p must be in [0, 1]");
  for (const void* q : {static_cast<const void*>(a->uniforms), static_cast<const void*>(a->row_temperature), static_cast<const void*>(a->row_top_k), static_cast<const void*>(a->row_top_p),
                        static_cast<const void*>(a->row_min_p), static_cast<const void*>(a->tokens), static_cast<const void*>(a->prob), static_cast<const void*>(a->kept),
                        static_cast<const void*>(a->row_status)})
    if (misaligned4(q)) return call_failed(COS_ERR_ALIGNMENT, "an int32/float pointer is not 4-byte aligned");
  if (a->filtered) {
    if (reinterpret_cast<uintptr_t>(a->filtered) % (a->dtype == COS_DTYPE_F32 ? 4 : 2)) return call_failed(COS_ERR_ALIGNMENT, "filtered pointer not aligned to its element type");
    if (a->rows > 1 && a->stride_filtered < a->vocab) return call_failed(COS_ERR_INVALID_ARG, "rows overlap: stride_filtered is less than vocab");
    if (a->filtered == a->logits && a->rows > 1 && a->stride_filtered != a->stride_row) return call_failed(COS_ERR_INVALID_ARG, "filtered in place needs the stride of the logits");
  }
  SampleParams p = {};
  p.c.logits = a->logits;
  p.c.stride = a->stride_row;
  p.u = a->uniforms;
  p.T = a->temperature;
  p.k = a->top_k;
  p.p = a->top_p;
  p.min_p = a->min_p;
  p.row_T = a->row_temperature;
  p.row_k = a->row_top_k;
  p.row_p = a->row_top_p;
  p.row_min_p = a->row_min_p;
  p.tokens = a->tokens;
  p.prob = a->prob;
  p.kept = a->kept;
  p.status = a->row_status;
  p.filtered = static_cast<char*>(a->filtered);
  p.stride_filtered = a->stride_filtered;
  return launch_rows(p, a->rows, a->vocab, a->dtype, a->device, sizeof(SampleShared), static_cast<cudaStream_t>(cuda_stream), [](int dt) {
    return dt == COS_DTYPE_F32 ? cos_sample_kernel<COS_DTYPE_F32> : (dt == COS_DTYPE_BF16 ? cos_sample_kernel<COS_DTYPE_BF16> : cos_sample_kernel<COS_DTYPE_F16>);
  });
}

extern "C" cos_status cos_top_logits(const cos_top_args* a, void* cuda_stream) {
  if (!a) return call_failed(COS_ERR_INVALID_ARG, "null argument");
  const cos_status st = check_rows(a->logits, a->stride_row, a->rows, a->vocab, a->dtype);
  if (st != COS_OK) return st;
  if (!a->values || !a->ids || !a->lse) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (misaligned4(a->values) || misaligned4(a->ids) || misaligned4(a->lse)) return call_failed(COS_ERR_ALIGNMENT, "an int32/float pointer is not 4-byte aligned");
  if (a->k < 1 || a->k > COS_TOP_MAX || a->k > a->vocab) return call_failed(COS_ERR_INVALID_ARG, "k must be in [1, min(COS_TOP_MAX, vocab)]");
  if (!(a->temperature > 0.0f)) return call_failed(COS_ERR_INVALID_ARG, "temperature must be > 0");
  TopParams p = {};
  p.c.logits = a->logits;
  p.c.stride = a->stride_row;
  p.k = a->k;
  p.T = a->temperature;
  p.values = a->values;
  p.ids = a->ids;
  p.lse = a->lse;
  return launch_rows(p, a->rows, a->vocab, a->dtype, a->device, sizeof(TopShared), static_cast<cudaStream_t>(cuda_stream), [](int dt) {
    return dt == COS_DTYPE_F32 ? cos_top_kernel<COS_DTYPE_F32> : (dt == COS_DTYPE_BF16 ? cos_top_kernel<COS_DTYPE_BF16> : cos_top_kernel<COS_DTYPE_F16>);
  });
}
