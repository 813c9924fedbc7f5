// Drawing a token from a row of logits at a temperature, after top-k, top-p and min-p, and listing the largest logits of a row: one launch, a
// cluster of blocks a row (cos_slice.cuh).
//
// Mathematics.  In order of (logit down, index up) every one of the three limits keeps a beginning of the line, so what is kept is the tokens at or
// above one of them.  A token's place in the line is one 64-bit number (`place_of`).
//
// The head of the line is found without sorting or counting tokens: of 512 groups of tokens (the same for all blocks; 1024 where a block has the row for itself) each block gets the largest logit; the
// k-th largest of these is at most the k-th largest logit, and little below it (k of 512 groups are taken up by some -512 ln(1 - k/512) tokens: 53 for k = 50).
// The few tokens from there on are compared with one another, and where the limits lie among them the row is done (top-k up to kHeadMost; top-p whose tokens
// are among the first few hundred).  Else a histogram of 1024 bins, linear in the logit below the maximum, says in which bin a limit lies, and the places in
// that bin are compared; a bin of more than kCandidates is cut into 1024 ranges of places, again until few are left: places are 64 bits and no two are alike,
// so this ends after at most seven histograms, for any number of equal logits.
//
// Weights are exp2 of 64-bit arguments (2^-36 of the largest and less: of 32-bit ones, off by 2^-17 of themselves), from a table of 2^(j/512) and the power
// series of 2^r for |r| <= 2^-10 (the fourth term is below 1e-14), rounded to whole multiples of 2^-scale and summed as integers: a token is drawn where a
// border of the cumulative sums lies next to u, and 32-bit sums are off by more than the weight of a token there.  Integers make sums independent of their
// order, so atomics and the split over blocks change nothing.
//
// Bound by latency, not bytes: a draw from one row of 151936 bf16 under top-k and top-p takes 8.7 us, three exchanges over 16 blocks (1.3 us each) among them; 64 x 256000 bf16 drawn from
// whole 33 us (1 TB/s; two waves of clusters, issue slots half busy); 32 x 128256 bf16 with a flat nucleus among them 42 us, the time of
// the rows that take the general path.  A block for each row, in registers: top 64 of 512 x 128256 bf16 38.5 us, 3.4 TB/s, 20 us at the copy rate (four rows on some multiprocessors, three on others).
#include <float.h>

#include "cos_slice.cuh"

namespace cosv {
namespace {

constexpr int kBins = 1024, kBinBits = 10, kCandidates = 512, kTopCandidates = COS_TOP_MAX + 512;
// the largest k that a list of that size is used for
template <int kList>
constexpr int kMost = kList == kTopCandidates ? COS_TOP_MAX : 288;
constexpr int kMostKept = 64 * 1024;  // bytes of a slice: two blocks of a multiprocessor have room for that beside what they share
// A block of so few entries counts those of a bin, and adds up their places in it (in eighths), in one word.
constexpr int kPackedEntries = 16384, kPackedShift = 17;
constexpr int kFew = 128;
constexpr int kHeadMost = kMost<kCandidates>, kHeadGuess = 96;  // the largest top-k that the head is tried for; the k it is tried with for a top-p alone
static_assert(kCandidates == kSliceThreads, "a thread for each");

struct Common {  // of both kernels
  const void* logits;
  long long stride;
  int V, parts, shift, share, seg, res;  // parts: 2^shift
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
  double inv_T;
  float scale;  // log2(e) / T
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

constexpr int kTable = 512;
constexpr double kNear = 36.0;  // powers of two

// How many entries are above -inf.
template <int DT>
__device__ __forceinline__ unsigned finite_entries(const uint4& r) {
  unsigned low;
  if constexpr (DT == COS_DTYPE_F32) {
    low = __float_as_uint(fminf(fminf(__uint_as_float(r.x), __uint_as_float(r.y)), fminf(__uint_as_float(r.z), __uint_as_float(r.w))));
  } else if constexpr (DT == COS_DTYPE_BF16) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&r);
    const __nv_bfloat162 m = __hmin2(__hmin2(h[0], h[1]), __hmin2(h[2], h[3]));
    low = *reinterpret_cast<const unsigned*>(&m);
  } else {
    const __half2* h = reinterpret_cast<const __half2*>(&r);
    const __half2 m = __hmin2(__hmin2(h[0], h[1]), __hmin2(h[2], h[3]));
    low = *reinterpret_cast<const unsigned*>(&m);
  }
  const uint4 m = make_uint4(low, 0, 0, 0);
  if (fminf(entry<DT>(m, 0), DT == COS_DTYPE_F32 ? INFINITY : entry<DT>(m, 1)) > -INFINITY) return Elem<DT>::E;
  unsigned n = 0;
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; ++e) n += entry<DT>(r, e) > -INFINITY;
  return n;
}

// exp((l - m) / T) in whole multiples of 2^-scale.
template <int DT>
struct Weight {
  float half, c32x2;    // half the row's largest logit (differences of halves do not overflow), twice log2(e) / T
  float near_from;      // logits from here on go by 64 bits
  double m64, c;        // the logit, log2(e) / T
  const double* table;  // 2^(j / 512) in units
  int scale;
  __device__ __forceinline__ void init(float m, float T, int V, const double* table_) {
    half = 0.5f * m;
    m64 = static_cast<double>(m);
    c = 1.4426950408889634 / static_cast<double>(T);
    c32x2 = fmaxf(fminf(static_cast<float>(2.0 * c), 3e38f), 1e-37f);  // (-inf is infinitely far at any temperature)
    near_from = fmaxf(static_cast<float>(m64 - kNear / c), -FLT_MAX);
    table = table_;
    scale = scale_of(V);
  }
  static __device__ __forceinline__ int scale_of(int V) { return min(46, 63 - (32 - __clz(V - 1))); }
  // 2^(i / 512) units
  __device__ __forceinline__ double power(int i) const {
    const double e = table[i & (kTable - 1)];
    return __hiloint2double(__double2hiint(e) + (i >> 9 << 20), __double2loint(e));
  }
  // Not rounded to the unit; l is at most 2^40 units of the temperature below the largest.
  __device__ __forceinline__ double exact(float l) const {
    constexpr double kRound = 13194139533312.0;  // 1.5 * 2^43: sums with it are multiples of 2^-9
    const double d = static_cast<double>(l) - m64;
    const double k = fma(d, c, kRound);
    const double r = fma(d, c, kRound - k);
    const int n = __double2loint(k);
    double e = fma(0.05550410866482158, r, 0.2402265069591007);  // ln(2)^i / i!
    e = fma(e, r, 0.6931471805599453);
    e = fma(e, r, 1.0);
    e *= table[n & (kTable - 1)];
    return __hiloint2double(__double2hiint(e) + (n >> 9 << 20), __double2loint(e));
  }
  // l >= near_from; at most 2^46: the rounded number's bits, with kUnits above them
  static constexpr u64 kUnits = 0x4330000000000000ull;
  __device__ __forceinline__ u64 near_bits(float l) const { return static_cast<u64>(__double_as_longlong(exact(l) + 4503599627370496.0)); }
  __device__ __forceinline__ u64 near(float l) const { return near_bits(l) - kUnits; }
  __device__ __forceinline__ unsigned far(float l) const {  // l < near_from: at most 2^10 (else some number)
    return __float_as_uint(ex2_approx(fmaf(fmaf(-0.5f, l, half), -c32x2, static_cast<float>(scale))) + 8388608.0f) - 0x4b000000u;
  }
  // l is not +inf or NaN; 0 for -inf.
  __device__ __forceinline__ u64 of(float l) const { return l >= near_from ? near(l) : far(l); }
  // The sum of far() of all entries of a vector, modulo 2^32.
  __device__ __forceinline__ unsigned far_vector(const uint4& r) const {
    f32x2 x[Elem<DT>::E / 2];
    unpack_pairs<DT>(r, x);
    const f32x2 minus_half = pack2(-0.5f, -0.5f), h = pack2(half, half), c = pack2(-c32x2, -c32x2), unit = pack2(static_cast<float>(scale), static_cast<float>(scale)), whole = pack2(8388608.0f, 8388608.0f);
    unsigned sum = 0;
#pragma unroll
    for (int k = 0; k < Elem<DT>::E / 2; ++k) {
      const f32x2 a = fma2(fma2(x[k], minus_half, h), c, unit);
      const f32x2 w = add2(pack2(ex2_approx(lo2(a)), ex2_approx(hi2(a))), whole);
      sum += __float_as_uint(lo2(w)) + __float_as_uint(hi2(w));
    }
    return sum - static_cast<unsigned>(Elem<DT>::E) * 0x4b000000u;
  }
  // The near entries of a vector that `head` has bits of (two under way), and what far() made of them.
  __device__ __forceinline__ u64 near_ones(const uint4& r, unsigned head, unsigned& as_far) const {
    u64 sum = 0;
    while (head) {
      const int a = __ffs(head) - 1;
      head &= head - 1;
      const bool two = head != 0;
      const int b = two ? __ffs(head) - 1 : a;
      head &= head - 1;
      const float va = pick(r, a), vb = pick(r, b);
      const u64 wa = near(va), wb = near(vb);
      sum += wa + (two ? wb : 0ull);
      as_far += far(va) + (two ? far(vb) : 0u);
    }
    return sum;
  }
  // Sum over the entries of a vector that keep(value, token) holds of.
  template <class K>
  __device__ __forceinline__ u64 of_vector(const uint4& r, int token, K&& keep) const {
    unsigned kept = 0, close = 0;
#pragma unroll
    for (int e = 0; e < Elem<DT>::E; ++e) {
      const float v = entry<DT>(r, e);
      kept |= static_cast<unsigned>(keep(v, token + e)) << e;
      close |= static_cast<unsigned>(v >= near_from) << e;
    }
    return of_some(r, kept, close);
  }
  // ... that `kept` has bits of, `close` of the near ones.
  __device__ __forceinline__ u64 of_some(const uint4& r, unsigned kept, unsigned close) const {
    unsigned unused = 0;
    u64 sum = near_ones(r, kept & close, unused);
    for (unsigned e = kept & ~close; e; e &= e - 1) sum += far(pick(r, __ffs(e) - 1));
    return sum;
  }
  // Sum over all entries of a vector.
  __device__ __forceinline__ u64 of_entries(const uint4& r) const {
    unsigned head = 0, as_far = 0;
#pragma unroll
    for (int e = 0; e < Elem<DT>::E; ++e) head |= static_cast<unsigned>(entry<DT>(r, e) >= near_from) << e;
    const u64 sum = near_ones(r, head, as_far);
    return sum + static_cast<unsigned>(far_vector(r) - as_far);  // (modulo 2^32)
  }
  // Sum over all entries of this lane.  Vectors far below the largest go by 32 bits; those with near entries in a second pass, in which every lane goes from one of its own to
  // the next (few where the tail is long): the near ones by 64-bit instructions, the others by 32 bits with all of the vector, modulo 2^32, from which what that makes
  // of the near ones is taken off again.
  __device__ __forceinline__ u64 of_all(const RowSlice<DT>& s, unsigned& finite) const {
    const int first = s.begin + (threadIdx.x & 31);
    u64 sum = 0;
    unsigned tail = 0;
    for (int block = first; block < s.end; block += 32 * 32) {  // (a bit for each of 32 vectors)
      unsigned any = 0;
      const int end = min(s.end, block + 32 * 32);
#pragma unroll 2
      for (int i = block, bit = 0; i < end; i += 32, ++bit) {
        const uint4 r = s.at(i);
        RunningMax<DT> top;
        top.add(r);
        finite += finite_entries<DT>(r);
        const bool close = top.value() >= near_from;
        if (!close) tail += far_vector(r);
        any |= static_cast<unsigned>(close) << bit;
      }
      for (; any; any &= any - 1) {
        const uint4 r = s.at(block + 32 * (__ffs(any) - 1));
        unsigned head = 0, as_far = 0;
#pragma unroll
        for (int e = 0; e < Elem<DT>::E; ++e) head |= static_cast<unsigned>(entry<DT>(r, e) >= near_from) << e;
        if (head == (1u << Elem<DT>::E) - 1) {
          u64 bits = 0;
#pragma unroll
          for (int e = 0; e < Elem<DT>::E; ++e) bits += near_bits(entry<DT>(r, e));
          sum += bits - Elem<DT>::E * kUnits;
        } else {
          sum += near_ones(r, head, as_far);
          tail += far_vector(r) - as_far;
        }
      }
    }
    return sum + tail;
  }
  static __device__ __forceinline__ float pick(const uint4& r, int e) {
    const int i = DT == COS_DTYPE_F32 ? e : e >> 1;
    const unsigned lo = (i & 1) ? r.y : r.x, hi = (i & 1) ? r.w : r.z, w = (i & 2) ? hi : lo;
    if (DT == COS_DTYPE_F32) return __uint_as_float(w);
    const unsigned h = (e & 1) ? w >> 16 : w & 0xffffu;
    if (DT == COS_DTYPE_BF16) return __uint_as_float(h << 16);
    return __half2float(__ushort_as_half(static_cast<unsigned short>(h)));
  }
};

struct Found {
  u64 before_count, before_mass, count;
  int bin, pad;
};

template <int kList>
struct Shared {
  unsigned count[kBins], lo[kBins], hi[kBins];
  u64 list[kList];             // this block's candidates
  u64 merged[kList];           // the row's
  u64 order[kFew];             // ... sorted, where they are few
  float group[kSliceThreads];  // the largest logit of each group of the row
  u64 scan_count[kSliceWarps], scan_mass[kSliceWarps];
  Found found[2];
  u64 word[2];
  unsigned steps[64];
  int listed, hits, pad[2];
};
using SampleShared = Shared<kCandidates>;
static_assert(sizeof(SampleShared) % 16 == 0 && sizeof(Shared<kTopCandidates>) % 16 == 0, "the slice lies behind it");

constexpr int kBinsEach = kBins / kSliceThreads;
static_assert(kBinsEach == 2, "a thread reads two bins at once");
// The row's histogram: a thread's bins, with what lies before them in the line.
struct Bins {
  u64 count[kBinsEach], mass[kBinsEach], before_count, before_mass;
  u64 all_count, all_mass;
};

// What is the same for every step of a row.
template <class H>
struct Row {
  H& h;
  Exchange& x;
  int parts, rank, turn, slot;
};

template <class H>
__device__ __forceinline__ void clear_bins(H& h) {
  for (int i = threadIdx.x; i < kBins; i += kSliceThreads) h.count[i] = h.lo[i] = h.hi[i] = 0;
}

// Behind the sweep that filled the blocks' bins and a barrier of the row: the sums over the blocks, in order, with mass_of(bin, count, lo, hi) for a bin, of the first `bins`.  Every block reads the bins of all
// of them (64 KB over 16 blocks at 10 bytes a clock), which takes less than a share for each and telling one another.  Bins may be cleared behind the next barrier of the row.
template <class H, class M>
__device__ __forceinline__ void merge_bins(Row<H>& w, int bins, bool masses, bool wide, bool packed, Bins& b, M&& mass_of) {
  constexpr int kAtOnce = 4;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, first = tid * kBinsEach;
  unsigned n[2] = {0, 0}, hi[2] = {0, 0};
  u64 lo[2] = {0, 0};
  const auto add = [&](const uint2& c, const uint2& l, const uint2& h) {
    constexpr unsigned kPlaces = (1u << kPackedShift) - 1;
    n[0] += packed ? c.x >> kPackedShift : c.x;
    n[1] += packed ? c.y >> kPackedShift : c.y;
    lo[0] += packed ? c.x & kPlaces : l.x;
    lo[1] += packed ? c.y & kPlaces : l.y;
    hi[0] += h.x;
    hi[1] += h.y;
  };
  const auto two = [&](const unsigned (&of)[kBins]) { return *reinterpret_cast<const uint2*>(&of[first]); };
  const uint2 none = make_uint2(0, 0);
  if (first >= bins) {
  } else if (w.parts == 1) {
    add(two(w.h.count), masses && !packed ? two(w.h.lo) : none, wide ? two(w.h.hi) : none);
  } else {
    for (int r0 = 0; r0 < w.parts; r0 += kAtOnce) {  // (so many blocks' under way at once, a block again where there are fewer)
      uint2 c[kAtOnce], l[kAtOnce], h[kAtOnce];
#pragma unroll
      for (int r = 0; r < kAtOnce; ++r) {
        const H* o = of_rank(&w.h, min(r0 + r, w.parts - 1));
        c[r] = two(o->count);
        l[r] = masses && !packed ? two(o->lo) : none;
        h[r] = wide ? two(o->hi) : none;
      }
#pragma unroll
      for (int r = 0; r < kAtOnce; ++r)
        if (r0 + r < w.parts) add(c[r], l[r], h[r]);
    }
  }
  u64 count = 0, mass = 0;
#pragma unroll
  for (int q = 0; q < kBinsEach; ++q) {
    b.count[q] = n[q];
    b.mass[q] = masses && first < bins ? mass_of(first + q, n[q], lo[q], hi[q]) : 0;
    count += b.count[q];
    mass += b.mass[q];
  }
  u64 sc = count, sm = mass;  // exclusive scan over the block
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const u64 c = __shfl_up_sync(0xffffffffu, sc, d), m = __shfl_up_sync(0xffffffffu, sm, d);
    if (lane >= d) {
      sc += c;
      sm += m;
    }
  }
  if (lane == 31) {
    w.h.scan_count[warp] = sc;
    w.h.scan_mass[warp] = sm;
  }
  __syncthreads();
  // (what the warps before this one have, and all of them: by every warp at once)
  const u64 ac = lane < kSliceWarps ? w.h.scan_count[lane & (kSliceWarps - 1)] : 0, am = lane < kSliceWarps ? w.h.scan_mass[lane & (kSliceWarps - 1)] : 0;
  b.before_count = sc - count + Add::warp(lane < warp ? ac : 0);
  b.before_mass = sm - mass + Add::warp(lane < warp ? am : 0);
  b.all_count = Add::warp(ac);
  b.all_mass = Add::warp(am);
}

// The bin in which the `target`-th token (by_mass: unit of mass) lies; 1 <= target <= what the row has.
template <class H>
__device__ __forceinline__ Found locate(Row<H>& w, const Bins& b, bool by_mass, u64 target) {
  const int slot = w.slot;
  w.slot ^= 1;
  u64 c = b.before_count, m = b.before_mass;
#pragma unroll
  for (int q = 0; q < kBinsEach; ++q) {
    const u64 at = by_mass ? m : c, here = by_mass ? b.mass[q] : b.count[q];
    if (at < target && target <= at + here) w.h.found[slot] = {c, m, b.count[q], static_cast<int>(threadIdx.x) * kBinsEach + q, 0};  // (one thread)
    c += b.count[q];
    m += b.mass[q];
  }
  __syncthreads();
  return w.h.found[slot];
}

// Lists a candidate of this block (as many as there is room for).
template <class H>
__device__ __forceinline__ void list(H& h, float v, int token) {
  const int at = atomicAdd(&h.listed, 1);
  if (at < static_cast<int>(sizeof(h.list) / sizeof(u64))) h.list[at] = place_of(v, token);
}
// ... those of a vector from a logit on; a bit for each.
template <int DT, class H>
__device__ __forceinline__ unsigned list_from(H& h, float from, int token, const uint4& r) {
  RunningMax<DT> top;
  top.add(r);
  if (!(top.value() >= from)) return 0;
  unsigned in = 0;
#pragma unroll
  for (int e = 0; e < Elem<DT>::E; ++e) {
    const float v = entry<DT>(r, e);
    in |= static_cast<unsigned>((v >= from) & (v > -INFINITY)) << e;
  }
  if (in == 0) return 0;
  int at = atomicAdd(&h.listed, __popc(in));
  for (unsigned left = in; left; left &= left - 1, ++at)
    if (at < static_cast<int>(sizeof(h.list) / sizeof(u64))) {
      const int e = __ffs(left) - 1;
      h.list[at] = place_of(Weight<DT>::pick(r, e), token + e);
    }
  return in;
}
// Behind the sweep that listed them (h.listed was 0): how many candidates the row has, and the sums over the row of `sum` and of the lanes' masses of what
// they listed.
struct Taken {
  u64 n, sum, listed;
};
template <class Sum = Nothing, class Listed = Nothing, class H>
__device__ __forceinline__ Taken taken(Row<H>& w, u64 sum = 0, u64 listed = 0) {
  __syncthreads();
  const Words all = exchange<OfFirst, Sum, Listed>(w.x, w.turn, w.parts, w.rank, static_cast<u64>(w.h.listed), sum, listed);
  if (threadIdx.x == 0) w.h.listed = 0;  // (for the next one: behind a barrier of the row, and ahead of one of the block)
  return {all.a, all.b, all.c};
}
// ... and the candidates of all blocks, n of them, to this one: right behind take().
template <class H>
__device__ __forceinline__ void merge_lists(Row<H>& w, int n) {
  const int t = (w.turn - 1) & 1;
  for (int i = threadIdx.x; i < n; i += kSliceThreads) {
    if (w.parts == 1) {
      w.h.merged[i] = w.h.list[i];
      continue;
    }
    int r = 0, j = i, before = 0;
#pragma unroll
    for (int q = 0; q < kSliceParts - 1; ++q)
      if (q < w.parts - 1) {
        before += static_cast<int>(w.x.a[t][q]);
        if (i >= before) {
          r = q + 1;
          j = i - before;
        }
      }
    w.h.merged[i] = *of_rank(&w.h.list[j], r);
  }
}

// Where in the line a bin's tokens lie, cut down until no more than `most` of them are left.
struct Range {
  u64 lo, hi;  // places, inclusive
  u64 before_count, before_mass, count;
};
template <class H, class S, class W, class In>
__device__ __forceinline__ Range narrow(Row<H>& w, const S& s, W&& weight, bool by_mass, u64 target, Range g, u64 most, In&& in) {
  u64 lo = ~0ull, hi = 0;
  s.entries([&](int token, float v) {
    if (v > -INFINITY && in(v)) {
      const u64 at = place_of(v, token);
      lo = at < lo ? at : lo;
      hi = at > hi ? at : hi;
    }
  });
  const Words ends = exchange<Min, Max>(w.x, w.turn, w.parts, w.rank, lo, hi);
  g.lo = ends.a;
  g.hi = ends.b;
  while (g.count > most) {
    const int bits = 64 - __clzll(static_cast<long long>(g.hi - g.lo)), shift = bits > kBinBits ? bits - kBinBits : 0;
    row_barrier(w.parts);  // (the bins have been read by all blocks)
    clear_bins(w.h);
    __syncthreads();
    s.entries([&](int token, float v) {
      const u64 at = place_of(v, token);
      if (v > -INFINITY && at >= g.lo && at <= g.hi) {
        const int bin = static_cast<int>((g.hi - at) >> shift);
        atomicAdd(&w.h.count[bin], 1u);
        if (by_mass) {  // 64 bits in two words: whoever makes the low one overflow carries
          const u64 m = weight(v);
          const unsigned was = atomicAdd(&w.h.lo[bin], static_cast<unsigned>(m));
          const unsigned up = static_cast<unsigned>(m >> 32) + (was + static_cast<unsigned>(m) < was ? 1u : 0u);
          if (up) atomicAdd(&w.h.hi[bin], up);
        }
      }
    });
    row_barrier(w.parts);
    Bins b;
    merge_bins(w, kBins, by_mass, by_mass, false, b, [](int, unsigned, u64 lo, unsigned hi) { return (static_cast<u64>(hi) << 32) + lo; });
    const Found sub = locate(w, b, by_mass, target - (by_mass ? g.before_mass : g.before_count));
    g.before_count += sub.before_count;
    g.before_mass += sub.before_mass;
    g.count = sub.count;
    const u64 top = g.hi - (static_cast<u64>(sub.bin) << shift), low = top - ((1ull << shift) - 1);
    g.hi = top;
    g.lo = low > g.lo && low <= top ? low : g.lo;
  }
  return g;
}

// Sums of the first n threads' words before this one, in order of the threads, and over all of them; the other warps only come along.
struct Scan {
  u64 before, all;
};
template <class H>
__device__ __forceinline__ Scan block_scan(H& h, int n, u64 mine) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (n + 31) >> 5;
  u64 up = mine;
  if (warp < warps) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const u64 o = __shfl_up_sync(0xffffffffu, up, d);
      if (lane >= d) up += o;
    }
    if (lane == 31) h.scan_mass[warp] = up;
  }
  __syncthreads();
  Scan s = {up - mine, 0};
  for (int i = 0; i < warps; ++i) {
    const u64 o = h.scan_mass[i];
    if (i < warp) s.before += o;
    s.all += o;
  }
  __syncthreads();
  return s;
}

// The first n threads' words, no two alike, in falling order (the other threads bring 0): thread i gets the i-th.  Few of them by counting, each by several lanes,
// how many are larger; more of them by a bitonic network.
template <class H>
__device__ __forceinline__ u64 sorted(H& h, int n, u64 v) {
  const int i = threadIdx.x;
  if (n <= kFew) {
    if (i < n) h.merged[i] = v;
    __syncthreads();
    const int wide = n > 1 ? 32 - __clz(n - 1) : 0, split = 9 - wide > 5 ? 5 : 9 - wide, lanes = 1 << split;  // 2^wide >= n candidates, 2^split lanes for each
    const int of = i >> split;
    const u64 mine = of < n ? h.merged[of] : 0;
    int larger = 0;
#pragma unroll 4
    for (int j = i & (lanes - 1); j < n; j += lanes) larger += h.merged[j] > mine;
    for (int d = 1; d < lanes; d *= 2) larger += __shfl_xor_sync(0xffffffffu, larger, d);
    if (of < n && (i & (lanes - 1)) == 0) h.order[larger] = mine;
    __syncthreads();
    return i < n ? h.order[i] : 0;
  }
  const auto step = [&](u64 o, bool up) { return up ? Max::two(v, o) : Min::two(v, o); };
#pragma unroll
  for (int block = 2; block <= 32; block *= 2)
#pragma unroll
    for (int stride = block / 2; stride > 0; stride /= 2) v = step(__shfl_xor_sync(0xffffffffu, v, stride), ((i & stride) == 0) == ((i & block) == 0));
#pragma unroll 1
  for (int block = 64; block < 2 * n; block *= 2) {
#pragma unroll 1
    for (int stride = block >> 1; stride >= 32; stride >>= 1) {
      __syncthreads();
      h.merged[i] = v;
      __syncthreads();
      v = step(h.merged[i ^ stride], ((i & stride) == 0) == ((i & block) == 0));
    }
#pragma unroll
    for (int stride = 16; stride > 0; stride /= 2) v = step(__shfl_xor_sync(0xffffffffu, v, stride), ((i & stride) == 0) == ((i & block) == 0));
  }
  return v;
}

// The n candidates of the row in order, one a thread: right behind taken().
template <class H>
__device__ __forceinline__ u64 in_order(Row<H>& w, int n) {
  merge_lists(w, n);
  return sorted(w.h, n, static_cast<int>(threadIdx.x) < n ? w.h.merged[threadIdx.x] : 0);  // (which this thread wrote)
}
// The place of the last thread of which `kept` holds: of the first ones, in order.
template <class H>
__device__ __forceinline__ u64 last_of(H& h, bool kept, u64 place) {
  const int n = __syncthreads_count(kept);
  if (static_cast<int>(threadIdx.x) == n - 1) h.word[0] = place;
  __syncthreads();
  const u64 at = h.word[0];
  __syncthreads();
  return at;
}

// The last place of the line that is kept by count: the first `target` tokens.
template <class H, class S, class W, class BinOf>
__device__ __forceinline__ u64 limit_by_count(Row<H>& w, const S& s, W&& weight, u64 target, const Found& f, BinOf&& bin_of) {
  Range g = {0, ~0ull, f.before_count, 0, f.count};
  if (f.count > kCandidates) g = narrow(w, s, weight, false, target, g, kCandidates, [&](float v) { return bin_of(v) == f.bin; });
  s.entries([&](int token, float v) {
    if (v > -INFINITY && bin_of(v) == f.bin) {
      const u64 at = place_of(v, token);
      if (at >= g.lo && at <= g.hi) list(w.h, v, token);
    }
  });
  const int n = static_cast<int>(taken(w).n);
  const u64 place = in_order(w, n);
  return last_of(w.h, static_cast<int>(threadIdx.x) < n && g.before_count + threadIdx.x < target, place);
}

// What a thread has weighed of the row on the way to a limit: the mass and number of its tokens before the limit's bin.  The block's tokens of that bin are in its list, `listed` of them (-1: not
// all, or nothing was weighed).
struct Weighed {
  u64 mass;
  int n, listed;
};
// ... and by mass: those before which less than `target` lies, 1 <= target <= the mass of the row.  b: the row's bins, whose masses are estimates; bin_at: a
// logit's bin before it is cut to a whole number.
template <int DT, class H, class BinAt>
__device__ __forceinline__ u64 limit_by_mass(Row<H>& w, const RowSlice<DT>& s, const Weight<DT>& weight, u64 target, const Bins& b, int bins, BinAt&& bin_at, Weighed& done) {
  const auto weigh = [&](float v) { return weight.of(v); };
  Found f = locate(w, b, true, Max::two(1, Min::two(target, b.all_mass)));
  Range g;
  int n;
  for (;;) {  // the estimates are good to 1e-4: the bin is this one or one next to it
    const auto in = [&](float v) { return min(static_cast<int>(bin_at(v)), bins - 1) == f.bin; };
    const float lo = static_cast<float>(f.bin), hi = lo + 1.0f;
    const bool last_bin = f.bin == bins - 1;
    const bool few = f.count <= kCandidates;
    u64 above = 0, inside = 0;
    int n_above = 0;
    s.raw([&](int token, const uint4& r) {
      RunningMax<DT> top;
      top.add(r);
      if (!(bin_at(top.value()) < hi) && !last_bin) return;  // (all of it lies behind the bin)
      unsigned before = 0, here = 0, close = 0;
#pragma unroll
      for (int e = 0; e < Elem<DT>::E; ++e) {
        const float v = entry<DT>(r, e), at = bin_at(v);
        before |= static_cast<unsigned>(at < lo) << e;
        here |= static_cast<unsigned>((at >= lo) & ((at < hi) | last_bin) & (v > -INFINITY)) << e;
        close |= static_cast<unsigned>(v >= weight.near_from) << e;
      }
      above += weight.of_some(r, before, close);
      n_above += __popc(before);
      for (; here; here &= here - 1) {
        const int e = __ffs(here) - 1;
        const float v = Weight<DT>::pick(r, e);
        inside += weigh(v);
        if (few) list(w.h, v, token + e);
      }
    });
    const Taken got = taken<Add, Add>(w, above, inside);
    g = {0, ~0ull, f.before_count, got.sum, f.count};
    n = static_cast<int>(got.n);
    if (target <= got.sum && f.before_count > 0) {
      f = locate(w, b, false, f.before_count);
    } else if (target > got.sum + got.listed && f.before_count + f.count < b.all_count) {
      f = locate(w, b, false, f.before_count + f.count + 1);
    } else if (few) {
      done = {above, n_above, w.parts > 1 ? static_cast<int>(w.x.a[(w.turn - 1) & 1][w.rank]) : n};
      break;
    } else {
      g = narrow(w, s, weigh, true, target, g, kCandidates, in);
      s.entries([&](int token, float v) {
        const u64 at = place_of(v, token);
        if (v > -INFINITY && at >= g.lo && at <= g.hi) list(w.h, v, token);
      });
      n = static_cast<int>(taken(w).n);
      break;
    }
  }
  const u64 place = in_order(w, n);
  const bool there = static_cast<int>(threadIdx.x) < n;
  const Scan up = block_scan(w.h, n, there ? weigh(logit_at(place)) : 0ull);
  return last_of(w.h, there && g.before_mass + up.before < target, place);
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

// Behind start(): the row's largest entry (NaN where there is one), the smallest of its 512 groups' largest ones that are above -inf (the largest, where none is),
// this lane's and this thread's group's.
struct Groups {
  float largest, smallest, own, group;
};
// largest and smallest from every thread's: `top` the largest of its groups, `low` the smallest above -inf (or -inf).
template <class H>
__device__ __forceinline__ void group_range(H& h, Groups& g, float top, float low) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const unsigned hi = __reduce_max_sync(0xffffffffu, top != top ? 0xffffffffu : ordered(top));  // (NaN above all)
  const unsigned lo = __reduce_min_sync(0xffffffffu, low == -INFINITY ? 0xffffffffu : ordered(low));
  if (lane == 0) {
    h.scan_count[warp] = hi;
    h.scan_mass[warp] = lo;
  }
  __syncthreads();
  const unsigned all = __reduce_max_sync(0xffffffffu, static_cast<unsigned>(h.scan_count[lane & (kSliceWarps - 1)]));
  const unsigned least = __reduce_min_sync(0xffffffffu, static_cast<unsigned>(h.scan_mass[lane & (kSliceWarps - 1)]));
  g.largest = all == 0xffffffffu ? __int_as_float(0x7fc00000) : unordered(all);
  g.smallest = least == 0xffffffffu ? g.largest : unordered(least);
}  // (the two arrays are written next behind a barrier of the block)
template <int DT, class H>
__device__ __forceinline__ Groups group_max(Row<H>& w, const RowSlice<DT>& s) {
  const int tid = threadIdx.x, lane = tid & 31;
  Groups g;
  s.finish();
  RunningMax<DT> here;
  s.raw([&](int, const uint4& r) { here.add(r); });
  float m = here.value();
  g.own = m;
  for (int d = 1; d < w.parts; d <<= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, d));
  if (w.parts > 1) {
    cluster_barrier_wait();  // (every block of the row has started)
    const int to = tid & (w.parts - 1);
    *of_rank(&w.h.group[(w.rank * kSliceThreads + tid) / w.parts], to) = m;
  } else {
    w.h.group[tid] = m;
  }
  row_barrier(w.parts);
  g.group = w.h.group[tid];
  group_range(w.h, g, g.group, g.group);
  return g;
}

// A logit that at least k of the groups reach, the largest one up to 1/64 of the range that the groups' largest logits span; -inf where fewer groups have a token.
// own: this thread's groups.  h.steps is 0, and is again.
template <class H, int N>
__device__ __forceinline__ float reached_by(H& h, const Groups& g, const float (&own)[N], int k) {
  const int tid = threadIdx.x, lane = tid & 31;
  const float span = g.largest - g.smallest, per = 64.0f / span;  // (span: overflows to inf for logits further apart than floats go: all in the first step)
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (own[i] > -INFINITY) atomicAdd(&h.steps[min(static_cast<int>((g.largest - own[i]) * per), 63)], 1u);
  __syncthreads();
  const unsigned a = h.steps[2 * lane], b = h.steps[2 * lane + 1];
  unsigned up = a + b;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const unsigned o = __shfl_up_sync(0xffffffffu, up, d);
    if (lane >= d) up += o;
  }
  const unsigned enough = __ballot_sync(0xffffffffu, up >= static_cast<unsigned>(k));
  const int first = enough ? __ffs(enough) - 1 : 31;
  const bool lower = __shfl_sync(0xffffffffu, up - b, first) >= static_cast<unsigned>(k);
  const int step = 2 * first + (lower ? 1 : 2);
  __syncthreads();
  if (tid < 64) h.steps[tid] = 0;
  if (!enough) return -INFINITY;
  if (step >= 64 || !(span > 0.0f && span < INFINITY)) return g.smallest;
  // (a hundredth of a step for the rounding of the steps)
  return __double2float_rd(static_cast<double>(g.largest) - (static_cast<double>(step) + 0.01) * static_cast<double>(span) / 64.0);
}

// A row that a block has for itself and that stays in memory: two groups a thread, halves of its vectors.
constexpr int kOwnGroups = 2;
__device__ __forceinline__ int group_span(const Common& c) { return (c.seg / 32 + kOwnGroups - 1) / kOwnGroups * 32; }  // vectors of a warp's groups of one half
// The largest logits of the thread's groups, from one pass over the row; f(four vectors, the largest of them) on the way.
template <int DT, class H, class F>
__device__ __forceinline__ Groups stream_groups(H& h, const RowSlice<DT>& s, const Common& c, float (&own)[kOwnGroups], F&& f) {
  const int half = group_span(c);
#pragma unroll
  for (int g = 0; g < kOwnGroups; ++g) {
    RunningMax<DT> group;
    s.stream(s.begin + (threadIdx.x & 31) + g * half, min(s.end, s.begin + (g + 1) * half), [&](const uint4 (&r)[4]) {
      RunningMax<DT> top;
#pragma unroll
      for (int k = 0; k < 4; ++k) top.add(r[k]);
      group.add(top);
      f(r, top);
    });
    own[g] = group.value();
  }
  Groups groups;
  groups.own = max_nan(own[0], own[1]);
  groups.group = 0.0f;
  group_range(h, groups, groups.own, own[0] == -INFINITY ? own[1] : own[1] == -INFINITY ? own[0] : fminf(own[0], own[1]));
  return groups;
}
// ... and f(token of the first entry, vector) for the vectors of the groups that reach a logit: those groups are dealt out over the warps, whose lanes read a group's vectors side by side.
// (Once a launch: h.hits is 0; h.group is free.)
template <int DT, class H, class F>
__device__ __forceinline__ void in_groups(H& h, const RowSlice<DT>& s, const Common& c, const float (&own)[kOwnGroups], float from, F&& f) {
  const int tid = threadIdx.x, half = group_span(c);
  unsigned short* const hit = reinterpret_cast<unsigned short*>(h.group);
  static_assert(sizeof(h.group) >= kOwnGroups * kSliceThreads * sizeof(unsigned short), "a place for every group");
#pragma unroll
  for (int g = 0; g < kOwnGroups; ++g)
    if (own[g] >= from) hit[atomicAdd(&h.hits, 1)] = static_cast<unsigned short>(tid * kOwnGroups + g);
  __syncthreads();
  const int hits = h.hits;
  for (int q = tid >> 5; q < hits; q += kSliceWarps) {
    const int thread = hit[q] / kOwnGroups, g = hit[q] % kOwnGroups;
    const int begin = min(s.nv, (thread >> 5) * c.seg), end = min(min(s.nv, begin + c.seg), begin + (g + 1) * half);
    for (int i = begin + g * half + (thread & 31) + 32 * (tid & 31); i < end; i += 32 * 32) f(s.token(i), s.fetch(i));
  }
}

// kStream: a block for each row, which stays in memory (a temperature of 0, or a top-k that the head is tried for).
template <int DT, bool kStream>
__global__ void __launch_bounds__(kSliceThreads, 2) cos_sample_kernel(const SampleParams p) {
  extern __shared__ uint4 smem[];
  SampleShared& h = *reinterpret_cast<SampleShared*>(smem);
  __shared__ Exchange x;
  __shared__ double table[kTable];
  const int parts = kStream ? 1 : p.c.parts, rank = kStream ? 0 : blockIdx.x & (parts - 1), row = kStream ? blockIdx.x : blockIdx.x >> p.c.shift, tid = threadIdx.x;
  if (parts > 1) cluster_barrier_arrive();
  wait_for_inputs();
  let_next_launch();
  RowSlice<DT> s;
  s.init(static_cast<const char*>(p.c.logits) + static_cast<long long>(row) * p.c.stride * Elem<DT>::bytes, p.c.V, rank, p.c.share, p.c.seg, smem + sizeof(h) / 16, kStream ? 0 : p.c.res);
  if (!kStream) s.start();
  const float T = p.row_T ? p.row_T[row] : p.T;
  int k = p.row_k ? p.row_k[row] : p.k;
  const float top_p = p.row_p ? p.row_p[row] : p.p, min_p = p.row_min_p ? p.row_min_p[row] : p.min_p;
  const double u = fmin(fmax(static_cast<double>(p.u[row]), 0.0), 1.0);  // (NaN: 0)
  char* const filtered = p.filtered ? p.filtered + static_cast<long long>(row) * p.stride_filtered * Elem<DT>::bytes : nullptr;
  table[tid] = exp2(static_cast<double>(tid) / kTable + Weight<DT>::scale_of(p.c.V));
  clear_bins(h);
  if (tid < 64) h.steps[tid] = 0;
  if (tid == 0) h.listed = h.hits = 0;
  Row<SampleShared> w = {h, x, parts, rank, 0, 0};
  Groups groups;
  float of_groups[kOwnGroups];
  if constexpr (kStream)
    groups = stream_groups<DT>(h, s, p.c, of_groups, [](const uint4 (&)[4], const RunningMax<DT>&) {});
  else
    groups = group_max(w, s);
  const float m = groups.largest, own = groups.own;

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
    const auto look = [&](int token, const uint4& r) {
#pragma unroll
      for (int e = 0; e < Elem<DT>::E; ++e)
        if (entry<DT>(r, e) == m) first = Min::two(first, static_cast<u64>(token + e));
    };
    if constexpr (kStream)
      in_groups<DT>(h, s, p.c, of_groups, m, look);
    else if (own == m)
      s.raw(look);
    const int token = static_cast<int>(exchange<Min>(x, w.turn, parts, rank, first).a);
    if (rank == 0 && tid == 0) {
      p.tokens[row] = token;
      if (p.prob) p.prob[row] = 1.0f;
      if (p.kept) p.kept[row] = 1;
      if (p.status) p.status[row] = 0;
    }
    if (filtered) write_filtered<DT>(s, filtered, [&](float, int t) { return t == token; });
    return;
  }

  if (k <= 0 || k > p.c.V) k = p.c.V;
  const bool by_k = k < p.c.V, by_p = top_p < 1.0f;
  Weight<DT> weight;
  weight.init(m, T, p.c.V, table);
  const auto weigh = [&](float v) { return weight.of(v); };
  // min-p as a logit: w >= min_p where l >= m + T ln(min_p); at a T without an end every token weighs 1
  const float least = min_p > 0.0f && T < INFINITY ? __double2float_ru(fma(static_cast<double>(T), log(fmin(static_cast<double>(min_p), 1.0)), static_cast<double>(m))) : -INFINITY;
  const auto share_of = [&](u64 mass) {  // of top-p: at least a unit, so that the first token is kept
    const double want = ceil(static_cast<double>(fmaxf(top_p, 0.0f)) * static_cast<double>(mass));
    return want < 1.0 ? 1ull : static_cast<u64>(want);
  };
  const auto drawn = [&](u64 mass) {  // the unit of mass that u falls on
    const double want = ceil(u * static_cast<double>(mass));
    return want >= static_cast<double>(mass) ? mass : (want < 1.0 ? 1ull : static_cast<u64>(want));
  };

  const u64 everything = place_of(-FLT_MAX, 0x7fffffff);
  u64 last = everything;  // the last place that is kept; nothing at -inf is
  Weighed done = {0, 0, -1};
  if (by_k || by_p) {
    u64 total = 0;  // what top-p is a part of
    if (!by_k || k <= kHeadMost) {
      float from;
      if constexpr (kStream)
        from = reached_by(h, groups, of_groups, by_k ? k : min(kHeadGuess, p.c.V));
      else
        from = reached_by(h, groups, {groups.group}, by_k ? k : min(kHeadGuess, p.c.V));
      u64 sum = 0, mass = 0;
      unsigned unused = 0;
      if (!by_k) sum = weight.of_all(s, unused);
      if (kStream && by_k) {
        in_groups<DT>(h, s, p.c, of_groups, from, [&](int token, const uint4& r) { list_from<DT>(h, from, token, r); });
      } else if (own >= from) {
        s.raw([&](int token, const uint4& r) {
          const unsigned in = list_from<DT>(h, from, token, r);
          if (!by_k)
            for (unsigned e = in; e; e &= e - 1) mass += weigh(Weight<DT>::pick(r, __ffs(e) - 1));
        });
      }
      const Taken got = taken<Add, Add>(w, sum, mass);
      total = got.sum;
      const u64 part = by_k ? 0 : share_of(total);
      if (got.n <= kCandidates && got.listed >= part) {  // the limits lie among these
        const int n = static_cast<int>(got.n);
        const u64 place = in_order(w, n);
        const bool there = tid < n && tid < k;
        const float logit = logit_at(place);
        const u64 mine = there ? weigh(logit) : 0;
        const Scan up = block_scan(h, n, mine);
        const u64 target = by_k ? (by_p ? share_of(up.all) : ~0ull) : part;
        const bool kept = there && up.before < target && logit >= least;
        const int count = __syncthreads_count(kept);
        if (tid == count - 1) {
          h.word[0] = place;
          h.word[1] = up.before + mine;
        }
        __syncthreads();
        last = h.word[0];
        const u64 all = h.word[1];
        if (rank == 0) {
          // in order of the index
          const u64 by_token = sorted(h, count, kept ? ~(static_cast<u64>(token_at(place)) << 32 | place >> 32) : 0);
          const bool of_these = tid < count;
          const float l = unordered(~static_cast<unsigned>(by_token));
          const u64 weighs = of_these ? weigh(l) : 0, goal = drawn(all);
          const u64 before = block_scan(h, count, weighs).before;
          if (of_these && before < goal && goal <= before + weighs) {
            p.tokens[row] = static_cast<int>(~static_cast<unsigned>(by_token >> 32));
            if (p.prob) p.prob[row] = static_cast<float>(weight.exact(l) / static_cast<double>(all));
          }
          if (tid == 0) {
            if (p.kept) p.kept[row] = count;
            if (p.status) p.status[row] = 0;
          }
        }
        if (filtered) write_filtered<DT>(s, filtered, [&](float v, int token) { return v > -INFINITY && place_of(v, token) >= last; });
        row_barrier(parts);  // (no block leaves while another reads its list)
        return;
      }
    }
    // Bins of 1/64 of a logit for a top-k alone, of 1/32 of a power of two of the weight for both (twice that where there are 512).  For a top-p alone they reach as far as its limit may lie: all logits
    // whose weight is below (1 - p) / vocab of the total have less than (1 - p) of it together, and are left out.
    // 512 bins over 16 blocks, whose bins take 7000 clocks to read otherwise; not for rows so long that the limit's bin would then hold more than the list does (256000 of N(0, 2.5^2) at p = 0.9:
    // some rows 56 us).
    const int bins = parts > 8 && p.c.V <= 320 * kCandidates ? kBins / 2 : kBins;
    bool cut = false;
    float per_unit = static_cast<float>(bins / 32);
    if (by_p && !by_k) {
      const double at = (1.0 - static_cast<double>(fmaxf(top_p, 0.0f))) * static_cast<double>(total) / p.c.V;  // that weight, in units
      cut = at >= 16.0;                                                                                      // (far from the rounding to units)
      if (cut) per_unit = static_cast<float>(bins - 2) / fmaxf(static_cast<float>(weight.scale) - log2f(static_cast<float>(at)) + 0.1f, 0.01f);
    }
    const float per_half = by_p ? fminf(per_unit * weight.c32x2, 1e30f) : static_cast<float>(bins / 8);
    const auto bin_at = [&](float v) { return fmaf(-0.5f, v, weight.half) * per_half; };
    const auto bin_of = [&](float v) { return min(static_cast<int>(bin_at(v)), bins - 1); };
    const bool packed = by_p && p.c.share <= kPackedEntries / Elem<DT>::E;
    s.raw([&](int, const uint4& r) {
#pragma unroll
      for (int e = 0; e < Elem<DT>::E; ++e) {
        const float v = entry<DT>(r, e);
        const int eighths = static_cast<int>(bin_at(v) * 8.0f), bin = eighths >> 3;
        if (v > -INFINITY && (bin < bins - 1 || !cut)) {
          const unsigned part = by_p && bin < bins - 1 ? eighths & 7 : 0;
          atomicAdd(&h.count[min(bin, bins - 1)], packed ? 1u << kPackedShift | part : 1u);
          if (!packed && part) atomicAdd(&h.lo[bin], part);
        }
      }
    });
    row_barrier(parts);
    Bins b;
    // the weights of a bin, from the places of its tokens in it (in eighths), up to the curvature of exp2 over it (1e-4)
    const float eighth = (1.0f - exp2f(-1.0f / per_unit)) * 0.125f;
    const double unit = weight.power(0);
    merge_bins(w, bins, by_p, false, packed, b, [&](int bin, unsigned count, u64 eighths, unsigned) {
      const float part = static_cast<float>(count) - eighth * (static_cast<float>(eighths) + 0.5f * static_cast<float>(count));
      return bin == bins - 1 ? 0ull : static_cast<u64>(unit * static_cast<double>(part * exp2f(static_cast<float>(-bin) / per_unit)));
    });
    if (by_k && static_cast<u64>(k) < b.all_count) {
      const Found f = locate(w, b, false, k);
      last = limit_by_count(w, s, weigh, k, f, bin_of);
    }
    if (by_p) {
      if (by_k) {
        u64 mine = 0;
        s.raw([&](int token, const uint4& r) {
          mine += weight.of_vector(r, token, [&](float v, int t) { return (v > -INFINITY) & (place_of(v, t) >= last); });
        });
        total = exchange<Add>(x, w.turn, parts, rank, mine).a;
      }
      const u64 target = share_of(total);
      if (target < total) last = limit_by_mass<DT>(w, s, weight, target, b, bins, bin_at, done);  // (among the first k: less than all of what they weigh lies before it)
    }
  }

  // what is kept, in order of the index
  const float last_logit = logit_at(last), bound = fmaxf(least, last_logit);
  const int last_token = least > last_logit ? 0x7fffffff : token_at(last);
  const auto keeps = [&](float v, int token) { return (v > bound) | ((v == bound) & (token <= last_token)); };
  u64 mine = 0;
  unsigned kept = 0;
  const bool every = last == everything && bound == last_logit;
  if (every) {
    mine = weight.of_all(s, kept);
  } else if (done.listed >= 0 && bound == last_logit) {  // weighed already, but for those of the limit's bin: a sweep less (5300 clocks for 8 blocks' 128256 tokens, all near)
    const int warp = tid >> 5;
    if (tid < kSliceWarps) h.scan_count[tid] = h.scan_mass[tid] = 0;
    __syncthreads();
    for (int i = tid; i < done.listed; i += kSliceThreads) {
      const u64 place = h.list[i];
      if (place < last) continue;
      const int of = s.warp_of(token_at(place), p.c.seg);
      atomicAdd(&h.scan_mass[of], weigh(logit_at(place)));
      atomicAdd(&h.scan_count[of], 1ull);
    }
    __syncthreads();
    mine = done.mass;
    kept = done.n;
    if ((tid & 31) == 0) {
      mine += h.scan_mass[warp];
      kept += static_cast<unsigned>(h.scan_count[warp]);
    }
  } else if (own >= bound) {
    s.raw([&](int token, const uint4& r) {
      RunningMax<DT> top;
      top.add(r);
      if (!(top.value() >= bound)) return;
      mine += weight.of_vector(r, token, keeps);
#pragma unroll
      for (int e = 0; e < Elem<DT>::E; ++e) kept += keeps(entry<DT>(r, e), token + e);
    });
  }
  const int t = w.turn & 1;
  const Words all = exchange<Add, Add>(x, w.turn, parts, rank, mine, kept);
  const u64 goal = drawn(all.a);
  u64 before = 0;
  for (int r = 0; r < rank; ++r) before += x.a[t][r];
  if (before < goal && goal <= before + x.a[t][rank]) {
    const int lane = tid & 31, warp = tid >> 5;
    mine = Add::warp(mine);
    if (lane == 0) h.scan_mass[warp] = mine;
    __syncthreads();
    for (int i = 0; i < warp; ++i) before += h.scan_mass[i];
    if (before < goal && goal <= before + mine) {  // this warp has it
      for (int at = s.begin; at < s.end; at += 32) {
        const int i = at + lane;
        const uint4 r = i < s.end ? s.at(i) : neg_inf_vector<DT>();
        const int token = s.token(i);
        const u64 sum = every ? weight.of_entries(r) : weight.of_vector(r, token, keeps);
        u64 up = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const u64 o = __shfl_up_sync(0xffffffffu, up, d);
          if (lane >= d) up += o;
        }
        const unsigned reached = __ballot_sync(0xffffffffu, before + up >= goal);
        if (reached) {  // a lane for each entry of that vector
          const int src = __ffs(reached) - 1;
          before += __shfl_sync(0xffffffffu, up - sum, src);
          const uint4 v4 = make_uint4(__shfl_sync(0xffffffffu, r.x, src), __shfl_sync(0xffffffffu, r.y, src), __shfl_sync(0xffffffffu, r.z, src), __shfl_sync(0xffffffffu, r.w, src));
          const int x0 = __shfl_sync(0xffffffffu, token, src) + lane;
          const float v = Weight<DT>::pick(v4, lane & (RowSlice<DT>::E - 1));
          const u64 own_weight = lane < RowSlice<DT>::E && keeps(v, x0) ? weigh(v) : 0;
          u64 to = own_weight;
#pragma unroll
          for (int d = 1; d < RowSlice<DT>::E; d <<= 1) {
            const u64 o = __shfl_up_sync(0xffffffffu, to, d);
            if (lane >= d) to += o;
          }
          const unsigned there = __ballot_sync(0xffffffffu, before + to >= goal);
          if (lane == __ffs(there) - 1) {
            p.tokens[row] = x0;
            if (p.prob) p.prob[row] = static_cast<float>(weight.exact(v) / static_cast<double>(all.a));
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
  if (filtered) write_filtered<DT>(s, filtered, keeps);
}

// kStream: a block for each row, which goes by in registers; what has candidates in it is read again.
template <int DT, int kList, bool kStream>
__global__ void __launch_bounds__(kSliceThreads, 2) cos_top_kernel(const TopParams p) {
  extern __shared__ uint4 smem[];
  Shared<kList>& h = *reinterpret_cast<Shared<kList>*>(smem);
  __shared__ Exchange x;
  const int parts = kStream ? 1 : p.c.parts, rank = kStream ? 0 : blockIdx.x & (parts - 1), row = kStream ? blockIdx.x : blockIdx.x >> p.c.shift, tid = threadIdx.x;
  if (parts > 1) cluster_barrier_arrive();
  wait_for_inputs();
  let_next_launch();
  RowSlice<DT> s;
  s.init(static_cast<const char*>(p.c.logits) + static_cast<long long>(row) * p.c.stride * Elem<DT>::bytes, p.c.V, rank, p.c.share, p.c.seg, smem + sizeof(h) / 16, p.c.res);
  if (tid < 64) h.steps[tid] = 0;
  if (tid == 0) h.listed = h.hits = 0;
  Row<Shared<kList>> w = {h, x, parts, rank, 0, 0};
  const float c = p.scale;
  Groups groups;
  float own[kStream ? kOwnGroups : 1], mine;  // the largest of this thread's groups, and of them
  double sum = 0.0;
  if constexpr (kStream) {
    RunningSum<DT> part;
    groups = stream_groups<DT>(h, s, p.c, own, [&](const uint4 (&r)[4], const RunningMax<DT>& top) { part.add(r, top, c); });
    mine = part.m;
    sum = part.z;
  } else {
    s.start();
    groups = group_max(w, s);
    own[0] = groups.group;
    mine = groups.own;
  }
  const float m = groups.largest;
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
  if constexpr (kStream) {
    if (mine != -INFINITY) sum *= static_cast<double>(ex2_approx((mine - m) * c));
  } else {
    const f32x2 minus_m = pack2(-m, -m), cc = pack2(c, c);
    s.raw([&](int, const uint4& r) { sum += static_cast<double>(sum_exp2<DT>(r, minus_m, cc)); });
  }
  int n = kList + 1;
  if (p.k <= kHeadMost) {
    const float from = reached_by(h, groups, own, p.k);
    if constexpr (kStream) {
      in_groups<DT>(h, s, p.c, own, from, [&](int token, const uint4& r) { list_from<DT>(h, from, token, r); });
    } else if (mine >= from) {
      s.raw([&](int token, const uint4& r) { list_from<DT>(h, from, token, r); });
    }
    const Taken got = taken<AddDouble>(w, bits_of(sum));
    n = static_cast<int>(got.n);
    sum = double_of(got.sum);
  } else {
    sum = double_of(exchange<AddDouble>(x, w.turn, parts, rank, bits_of(sum)).a);
  }
  if (rank == 0 && tid == 0) p.lse[row] = static_cast<float>(static_cast<double>(m) * p.inv_T + log(sum));
  if (n > kList) {
    const auto bin_of = [&](float v) { return min(static_cast<int>(fmaf(-0.5f, v, 0.5f * m) * 128.0f), kBins - 1); };
    clear_bins(h);
    __syncthreads();
    s.entries([&](int, float v) {
      if (v > -INFINITY) atomicAdd(&h.count[bin_of(v)], 1u);
    });
    row_barrier(parts);
    Bins b;
    merge_bins(w, kBins, false, false, false, b, [](int, unsigned, u64, unsigned) { return 0ull; });
    u64 from = 0;  // of places
    if (static_cast<u64>(p.k) < b.all_count) {
      const Found f = locate(w, b, false, p.k);
      Range g = {0, 0, f.before_count, 0, f.count};
      // (what lies before the bin is less than k, and kList holds as many and the rest)
      if (f.before_count + f.count > kList) {
        g = narrow(w, s, [](float) { return 0ull; }, false, p.k, g, kList - kMost<kList>, [&](float v) { return bin_of(v) == f.bin; });
        from = g.lo;
        s.entries([&](int token, float v) {
          if (v > -INFINITY && place_of(v, token) >= from) list(h, v, token);
        });
      } else {
        s.entries([&](int token, float v) {
          if (v > -INFINITY && bin_of(v) <= f.bin) list(h, v, token);
        });
      }
    } else {
      s.entries([&](int token, float v) {
        if (v > -INFINITY) list(h, v, token);
      });
    }
    n = static_cast<int>(taken(w).n);
  }
  merge_lists(w, n);
  __syncthreads();
  // every block compares its share of the candidates with all of them, a candidate by as many lanes as there are
  const int each = (n + parts - 1) / parts, end = min(n, (rank + 1) * each);
  int lanes = 1;
  while (lanes < 32 && 2 * lanes * each <= kSliceThreads) lanes *= 2;
  for (int first = rank * each; first < end; first += kSliceThreads / lanes) {  // (the same for all lanes of a warp)
    const int i = first + tid / lanes;
    const u64 mine = i < end ? h.merged[i] : 0;
    int at = 0;
    if (i < end) {
#pragma unroll 4
      for (int j = tid & (lanes - 1); j < n; j += lanes) at += h.merged[j] > mine;
    }
    for (int d = 1; d < lanes; d *= 2) at += __shfl_xor_sync(0xffffffffu, at, d);
    if (i < end && (tid & (lanes - 1)) == 0 && at < p.k) {
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
  if (rows > 1 && stride < vocab && stride != 0) return call_failed(COS_ERR_INVALID_ARG, "rows overlap: stride_row is less than vocab");
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == COS_DTYPE_F32 ? 4 : 2)) return call_failed(COS_ERR_ALIGNMENT, "logits pointer not aligned to its element type");
  return COS_OK;
}

// A block for each row where there are rows enough, and too long for a block's shared memory: no exchanges, and one wave where clusters take several.  Rows from which on (us, clusters / a block
// a row, logits drawn from N(0, 2.5^2)):
//   top logits, k <= 64     48   64 of 48 x 128256 bf16 13.5 / 13.2, of 32 rows 9.9 / 12.7, of 100 21.0 / 13.0
//   top logits, more        80   288 of 80 x 256000 bf16 42.6 / 32.6, of 64 rows 32.5 / 32.4, of 64 x 128256 23.4 / 28.6 (their groups are read again in turns)
//   a draw, k <= 64         16   64 of 16 x 128256 bf16 11.5 / 11.0, of 8 x 256000 (k = 50) 11.8 / 12.1, of 100 x 128256 26.5 / 11.7
//   a draw, more            40   200 of 40 x 128256 bf16 22.3 / 20.2, of 32 rows 19.7 / 20.7, of 100 33.9 / 20.9
//   the largest logit       16   16 x 128256 bf16 5.0 / 4.6, 100 rows 13.2 / 4.8, 64 x 32000 4.7 / 3.3; not for shorter rows (256 x 16000 4.2 / 5.2)
// Rows whose limit lies among so many equal logits that the list does not hold them are swept again from memory, which a block alone does longer than a cluster (128256 bf16, a row of three values, one row less /
// as many rows: a draw of 64 at 16 rows 40 / 229, of 200 at 40 rows 101 / 232, top 64 at 48 rows 54 / 144, top 288 at 80 rows 84 / 149; bf16 of uniform numbers, a few dozen of each value: 12 / 20, 67 / 160, 16 / 23,
// 112 / 200).  The host cannot see it, and logits of models are not like that.
bool own_blocks(int rows, int vocab, int dtype, int from, int longer_than = kMostKept) { return rows >= from && static_cast<long long>(vocab) * (dtype == COS_DTYPE_F32 ? 4 : 2) > longer_than; }

template <class P, class F>
cos_status launch_rows(P& p, int rows, int vocab, int dtype, int device, size_t shared, bool whole, cudaStream_t stream, F&& kernel_of) {
  OnDevice on(device);
  if (on.error != cudaSuccess) return call_failed("cudaSetDevice", on.error);
  SlicePlan plan;
  cudaError_t e = slice_plan(device, rows, vocab, dtype, kMostKept, true, &plan);
  if (e != cudaSuccess) return call_failed("device query", e);
  if (static_cast<long long>(rows) * plan.parts > 0x7fffffffll) return call_failed(COS_ERR_UNSUPPORTED, "too many rows for one launch");
  if (whole) {  // a block for each row, which stays in memory
    plan.parts = 1;
    plan.res = 0;
    plan.smem = 0;
    plan_row(vocab, dtype, kSliceWarps, &plan.share, &plan.seg);
  }
  p.c.V = vocab;
  p.c.parts = plan.parts;
  p.c.shift = __builtin_ctz(plan.parts);
  p.c.share = plan.share;
  p.c.seg = plan.seg;
  p.c.res = plan.res;
  e = slice_launch(kernel_of(dtype), p, rows * plan.parts, plan.parts, shared + plan.smem, shared + kMostKept, stream);
  return e == cudaSuccess ? COS_OK : call_failed("launch", e);
}

bool misaligned4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 != 0; }

}  // namespace

cudaError_t slice_plan(int device, int rows, int vocab, int dtype, int most, bool cluster, SlicePlan* plan) {
  const cudaError_t e = cudaDeviceGetAttribute(&plan->sms, cudaDevAttrMultiProcessorCount, device);
  if (e != cudaSuccess) return e;
  const int E = dtype == COS_DTYPE_F32 ? 4 : 8, kept = most / 16;
  const long long all = (static_cast<long long>(vocab) + 2 * (E - 1)) / E;
  long long parts = 1;
  while ((parts < kSliceParts || !cluster) && (all + parts - 1) / parts > kept) parts *= 2;
  // Places for blocks of rows in 2, 4, 8, 16.  Blocks in eights and sixteens that share a multiprocessor pay where slices are long only (us, of 12 rows in eights / sixteens: top 256 of 32000 fp32
  // 7.2 / 8.7, p = 0.9 18.7 / 21.9, drawn from 256000 bf16 18.2 / 14.7; of 24 rows in fours / eights: k = 50 of 32000 bf16 8.6 / 10.4, drawn from 128256 bf16 18.3 / 15.3).
  const auto places = [&](long long blocks) -> long long {
    const bool longer = all / (blocks / 2) * 16 > (blocks == 8 ? 24 : 48) * 1024;
    return blocks < 8 ? 2 * plan->sms : blocks == 8 ? (longer ? 256 : 120) : (longer ? 192 : 112);
  };
  for (long long blocks = 2; blocks <= kSliceParts; blocks *= 2)
    if (parts == blocks / 2 && all / parts >= kSliceThreads && rows * blocks <= places(blocks)) parts = blocks;
  plan->parts = static_cast<int>(parts);
  plan->share = static_cast<int>((all + parts - 1) / parts);
  plan->seg = static_cast<int>((plan->share + 32 * kSliceWarps - 1) / (32 * kSliceWarps) * 32);
  plan->res = plan->share < kept ? plan->share : kept;
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
    if (overlap(a->logits, a->stride_row, a->filtered, a->stride_filtered, a->rows, a->vocab, a->dtype == COS_DTYPE_F32 ? 4 : 2))
      return call_failed(COS_ERR_INVALID_ARG, "filtered overlaps the logits (in place: the same address and stride)");
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
  const auto call = [&](auto stream) {
    constexpr bool kStream = decltype(stream)::value;
    return launch_rows(p, a->rows, a->vocab, a->dtype, a->device, sizeof(SampleShared), kStream, static_cast<cudaStream_t>(cuda_stream), [](int dt) {
      return dt == COS_DTYPE_F32 ? cos_sample_kernel<COS_DTYPE_F32, kStream> : (dt == COS_DTYPE_BF16 ? cos_sample_kernel<COS_DTYPE_BF16, kStream> : cos_sample_kernel<COS_DTYPE_F16, kStream>);
    });
  };
  // A block for each row where the host knows that the rows are done with their heads or maxima.
  const bool largest = !a->row_temperature && a->temperature == 0.0f;
  const bool head = !a->row_temperature && !largest && !a->row_top_k && a->top_k > 0 && a->top_k <= kHeadMost && a->top_k < a->vocab;
  const bool own = (largest && own_blocks(a->rows, a->vocab, a->dtype, 16, kMostKept / 2)) || (head && own_blocks(a->rows, a->vocab, a->dtype, a->top_k <= 64 ? 16 : 40));
  return own ? call(std::true_type()) : call(std::false_type());
}

extern "C" cos_status cos_top_logits(const cos_top_args* a, void* cuda_stream) {
  if (!a) return call_failed(COS_ERR_INVALID_ARG, "null argument");
  const cos_status st = check_rows(a->logits, a->stride_row, a->rows, a->vocab, a->dtype);
  if (st != COS_OK) return st;
  if (!a->values || !a->ids || !a->lse) return call_failed(COS_ERR_INVALID_ARG, "null device pointer");
  if (misaligned4(a->values) || misaligned4(a->ids) || misaligned4(a->lse)) return call_failed(COS_ERR_ALIGNMENT, "an int32/float pointer is not 4-byte aligned");
  if (a->k < 1 || a->k > COS_TOP_MAX || a->k > a->vocab) return call_failed(COS_ERR_INVALID_ARG, "k must be in [1, min(COS_TOP_MAX, vocab)]");
  if (!(a->temperature > 1e-300 && a->temperature < 1e300)) return call_failed(COS_ERR_INVALID_ARG, "temperature must be finite and > 0 (1e-300 to 1e300)");
  TopParams p = {};
  p.c.logits = a->logits;
  p.c.stride = a->stride_row;
  p.k = a->k;
  p.inv_T = 1.0 / a->temperature;
  p.scale = exponent_of(a->temperature).c;
  p.values = a->values;
  p.ids = a->ids;
  p.lse = a->lse;
  const auto call = [&](auto list, auto stream) {
    constexpr int kList = decltype(list)::value;
    constexpr bool kStream = decltype(stream)::value;
    return launch_rows(p, a->rows, a->vocab, a->dtype, a->device, sizeof(Shared<kList>), kStream, static_cast<cudaStream_t>(cuda_stream), [](int dt) {
      return dt == COS_DTYPE_F32 ? cos_top_kernel<COS_DTYPE_F32, kList, kStream> : (dt == COS_DTYPE_BF16 ? cos_top_kernel<COS_DTYPE_BF16, kList, kStream> : cos_top_kernel<COS_DTYPE_F16, kList, kStream>);
    });
  };
  using Few = std::integral_constant<int, kCandidates>;
  if (a->k > kMost<kCandidates>) return call(std::integral_constant<int, kTopCandidates>(), std::false_type());
  return own_blocks(a->rows, a->vocab, a->dtype, a->k <= 64 ? 48 : 80) ? call(Few(), std::true_type()) : call(Few(), std::false_type());
}
