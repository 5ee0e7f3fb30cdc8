// The next token of each row of logits by temperature, top-k, top-p and min-p
// (nacl_sample).
//
// Two launches and one pass over the logits.  sample_slices_kernel reads slices
// of a row (kSlice tokens, whatever the batch, so that a row's sums and its
// result do not depend on it) and sorts what can matter into bins of an eighth of
// a power of two of the weight: bin(x) = floor(8 x log2(e) / temperature), the
// same grid for every slice and without the row's maximum.  A bin holds the
// count of its tokens and the sum of their weights over the bin's lower edge,
// both as integers, so that the order of the atomics does not show.
// sample_finish_kernel joins a row's slices, finds the bin in which the kept
// tokens end, reads the row again only for the tokens down to that bin, sorts
// those and draws.

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

constexpr int kSliceThreads = 512;
constexpr int kSlicePer = 16;                            // tokens per thread
constexpr int kSlice = kSliceThreads * kSlicePer;        // tokens per slice
constexpr int kBins = 256;                               // 32 powers of two below a slice's largest
constexpr int kMaxSlices = (NACL_MAX_V + kSlice - 1) / kSlice;
constexpr int kFinishThreads = 1024;
constexpr int kList = 4096;                              // tokens that the finish sorts
constexpr float kUnit = 0x1p22f;                         // a weight over its bin's edge, in units
constexpr int kCountShift = 43;                          // of a bin word: count above, weight units below
constexpr float kMaxBin = 0x1p20f;                       // bins beyond are too coarse to use
static_assert(NACL_MAX_V < (1 << (64 - kCountShift)) && NACL_MAX_V * 1.1 * 0x1p22 < 0x1p43, "bin words");

// What a slice leaves for the finish, followed by its bins.
struct SliceInfo {
  float max;     // largest logit
  int top;       // its bin (the slice's bins go down from it)
  int n_bins;    // bins filled; -1: the logits are beyond the grid
  int left;      // top-k: a token above -infinity lies below the bins
  double rest;   // weights outside the bins over the largest one's
};

struct Settings {
  float scale;   // log2(e) / temperature
  int k;         // 0: no limit
  float p;       // >= 1: no limit
  float m;       // 0: no limit
};
__device__ __forceinline__ Settings settings_of(const SampleLaunch& a, int n) {
  Settings s;
  const float t = a.temperature ? a.temperature[n] : 1.f;
  s.p = a.top_p ? a.top_p[n] : 1.f;
  s.m = a.min_p ? a.min_p[n] : 0.f;
  s.k = a.top_k ? a.top_k[n] : 0;
  if (s.p != s.p) s.p = 1.f;
  s.m = s.m > 0.f ? fminf(s.m, 1.f) : 0.f;
  if (s.k <= 0 || s.k >= a.V) s.k = 0;
  s.scale = 1.44269504f / t;
  const bool greedy = !(t > 0.f);
  if (greedy) s.scale = 1.44269504f;
  if (greedy || s.p <= 0.f) {
    s.k = 1;
    s.p = 1.f;
    s.m = 0.f;
  }
  return s;
}

__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : x + 0.f; }  // -0 counts as 0

template <typename T>
__device__ __forceinline__ float logit(const T* p, int64_t i) {
  return clean((float)p[i]);
}

__device__ __forceinline__ float bin_of(float x, float scale) { return floorf(x * (8.f * scale)); }
// A weight over its bin's lower edge, in [1, 2^(1/8)] or so; the product is
// exact in the FMA, so only the scale's rounding shows, as in a temperature.
__device__ __forceinline__ float over_edge(float x, float scale, float bin) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(x, scale, -0.125f * bin));
}

// kSlicePer logits of a thread: runs of 8, kSliceThreads * 8 apart.
template <typename T>
__device__ __forceinline__ void load_slice(const T* row, int V, int i0, int tid, float (&x)[kSlicePer]) {
#pragma unroll
  for (int e = 0; e < kSlicePer / 8; ++e) {
    const int i = i0 + (e * kSliceThreads + tid) * 8;
    T raw[8];
    if (i + 8 <= V) {
      __builtin_memcpy(raw, row + i, sizeof(raw));
#pragma unroll
      for (int c = 0; c < 8; ++c) x[8 * e + c] = clean((float)raw[c]);
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) x[8 * e + c] = i + c < V ? logit(row, i + c) : -INFINITY;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kSliceThreads) void sample_slices_kernel(SampleLaunch a, int n_slices) {
  __shared__ unsigned long long bins[kBins];
  __shared__ uint32_t tops[kBins];
  __shared__ float wmax[kSliceThreads / 64];
  __shared__ double wrest[kSliceThreads / 64];
  __shared__ int need;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int slice = blockIdx.x, n = blockIdx.y;
  const Settings s = settings_of(a, n);
  const T* row = reinterpret_cast<const T*>(a.logits) + (int64_t)n * a.stride;

  float x[kSlicePer];
  load_slice(row, a.V, slice * kSlice, tid, x);
  if (tid < kBins) {
    bins[tid] = 0;
    tops[tid] = 0;
  }
  float tmax = x[0];
#pragma unroll
  for (int i = 1; i < kSlicePer; ++i) tmax = fmaxf(tmax, x[i]);
  float mx = tmax;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) mx = fmaxf(mx, __shfl_xor(mx, d));
  if (lane == 0) wmax[wave] = mx;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSliceThreads / 64; ++w) mx = fmaxf(mx, wmax[w]);

  char* out = static_cast<char*>(a.ws) + ((int64_t)n * n_slices + slice) * (sizeof(SliceInfo) + kBins * 8);
  SliceInfo* info = reinterpret_cast<SliceInfo*>(out);
  const float top = bin_of(mx, s.scale);
  // All hidden, or beyond the grid (infinite and NaN products among that).
  if (mx == -INFINITY || !(__builtin_fabsf(top) < kMaxBin) || s.scale < 0x1p-60f) {
    if (tid == 0) *info = SliceInfo{mx, 0, mx == -INFINITY ? 0 : -1, 0, 0.0};
    return;
  }

  // How many bins can matter.  Top-k: the row's k-th largest is not below the
  // slice's, and that not below the k-th largest of the threads' maxima.  Top-p:
  // the tokens from the last kept one down weigh at least (1 - p) of the sum, so
  // the last kept one weighs at least (1 - p) / V of it, which is not below the
  // slice's largest weight.  Min-p: the row's largest is not below the slice's.
  int n_bins = 0;
  if (s.k > 0) {
    n_bins = kBins;
    if (s.k <= kSliceThreads) {
      const float j = top - bin_of(tmax, s.scale);
      if (j < kBins) atomicAdd(&tops[(int)j], 1u);
      __syncthreads();
      if (wave == 0) {
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += c[i] = tops[4 * lane + i];
        uint32_t before = sum;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const uint32_t y = __shfl_up(before, d);
          if (lane >= d) before += y;
        }
        before -= sum;
        int at = kBins;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          before += c[i];
          if (before >= (uint32_t)s.k) at = min(at, 4 * lane + i + 1);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) at = min(at, __shfl_xor(at, d));
        if (lane == 0) need = at;
      }
      __syncthreads();
      n_bins = need;
    }
  } else if (s.p < 1.f) {
    n_bins = min(kBins, (int)(8.f * log2f((float)a.V / (1.f - s.p))) + 3);
  } else if (s.m > 0.f) {
    n_bins = (int)fminf((float)kBins, -8.f * log2f(s.m) + 3.f);
  }

  float rest = 0.f;
  bool left = false;
  const bool with_rest = s.k == 0 && (s.p < 1.f || s.m == 0.f);
  if (n_bins > 0) {
    const float n_binsf = (float)n_bins;
#pragma unroll
    for (int i = 0; i < kSlicePer; ++i) {
      const float b = bin_of(x[i], s.scale), j = top - b;
      if (j < n_binsf)
        atomicAdd(&bins[(int)j], (1ull << kCountShift) + (uint32_t)rintf(over_edge(x[i], s.scale, b) * kUnit));
      else if (with_rest)
        rest += __builtin_amdgcn_exp2f((x[i] - mx) * s.scale);
      else
        left = left || x[i] > -INFINITY;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kSlicePer; ++i) rest += x[i] == mx ? 1.f : __builtin_amdgcn_exp2f((x[i] - mx) * s.scale);
  }
  double total = rest;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d);
  if (lane == 0) wrest[wave] = total;
  const int any_left = __syncthreads_or(left);
  if (tid == 0) {
    total = 0.0;
    for (int w = 0; w < kSliceThreads / 64; ++w) total += wrest[w];
    *info = SliceInfo{mx, (int)top, n_bins, any_left, total};
  }
  if (tid < n_bins) reinterpret_cast<unsigned long long*>(info + 1)[tid] = bins[tid];
}

// Exclusive sums in thread order and the sum of all, by a fixed tree.
template <typename U>
__device__ U block_scan(U x, U* total, U* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  U s = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const U y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  U before = __shfl_up(s, 1);
  if (lane == 0) before = 0;
  __syncthreads();
  if (lane == 63) tmp[wave] = s;
  __syncthreads();
  U base = 0, all = 0;
  for (int w = 0; w < kFinishThreads / 64; ++w) {
    if (w < wave) base += tmp[w];
    all += tmp[w];
  }
  *total = all;
  return base + before;
}

// Sorts n words of LDS (a power of two) in falling order.
__device__ void sort_falling(uint64_t* v, int n) {
  for (int size = 2; size <= n; size *= 2)
    for (int step = size / 2; step > 0; step /= 2) {
      __syncthreads();
      for (int i = threadIdx.x; i < n / 2; i += kFinishThreads) {
        const int lo = (i / step) * 2 * step + (i % step), hi = lo + step;
        const uint64_t x = v[lo], y = v[hi];
        const bool falling = (lo & size) == 0;
        if ((x < y) == falling) {
          v[lo] = y;
          v[hi] = x;
        }
      }
    }
  __syncthreads();
}

__device__ __forceinline__ double pow2(double x) { return exp2(x); }

struct FinishShared {
  uint64_t list[kList];
  double value[kList];
  double tmp[kFinishThreads / 64];
  uint64_t tmpu[kFinishThreads / 64];
  unsigned long long bins[kBins];
  uint32_t hist[kBins];
  SliceInfo info[kMaxSlices];
  double slice_w[kMaxSlices];
  uint32_t wanted[kMaxSlices / 32];
  int pick[4];
  uint64_t picku[2];
};

// Order of tokens as falling words: larger logits first, then lower indexes.
__device__ __forceinline__ uint64_t word_of(float x, uint32_t i) { return (uint64_t)float_order_key(x) << 32 | (uint32_t)~i; }
__device__ __forceinline__ float float_of_key(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key);
}

// Which tokens are kept: those whose word is at least `last` and logit at least
// `least`.
struct Kept {
  uint64_t last;
  double least;
  __device__ __forceinline__ bool operator()(float x, uint32_t i) const {
    return x > -INFINITY && word_of(x, i) >= last && (double)x >= least;
  }
};

__device__ __forceinline__ void answer(const SampleLaunch& a, int n, int token, double p) {
  a.tokens[n] = token;
  if (a.logprobs) a.logprobs[n] = token < 0 ? -INFINITY : (float)log(p);
}

// The draw among the kept tokens of [i0, i1), whose weights start at `before`
// and of which the one is wanted at which the sum passes `at`.  A thread takes a
// run of tokens; of a sum that falls short by rounding, the last token.
template <typename T, class W>
__device__ void draw_in(const SampleLaunch& a, int n, const T* row, int i0, int i1, double at, double total, const Kept& kept,
                        const W& weight, FinishShared& sh) {
  const int per = (i1 - i0 + kFinishThreads - 1) / kFinishThreads;
  const int lo = min(i1, i0 + (int)threadIdx.x * per), hi = min(i1, lo + per);
  double sum = 0.0;
  int last = -1;
  for (int i = lo; i < hi; ++i) {
    const float x = logit(row, i);
    const double w = kept(x, i) ? weight(x) : 0.0;
    sum += w;
    if (w > 0.0) last = i;
  }
  double all;
  const double before = block_scan(sum, &all, sh.tmp);
  if (threadIdx.x == 0) sh.pick[0] = -1;
  __syncthreads();
  if (last >= 0) atomicMax(&sh.pick[0], last);
  if (threadIdx.x == 0) sh.pick[1] = 0x7FFFFFFF;
  __syncthreads();
  if (before + sum > at && sum > 0.0) {  // the first such thread's first such token
    double cum = before;
    for (int i = lo; i < hi; ++i) {
      const float x = logit(row, i);
      const double w = kept(x, i) ? weight(x) : 0.0;
      cum += w;
      if (w > 0.0 && cum > at) {
        atomicMin(&sh.pick[1], i);
        break;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const int token = sh.pick[1] == 0x7FFFFFFF ? sh.pick[0] : sh.pick[1];
    answer(a, n, token, token < 0 ? 0.0 : weight(logit(row, token)) / total);
  }
}

// Any row, slowly: the last kept token by a search over the words' range that
// narrows it 256-fold a pass, then the draw over the whole row.  For logits
// beyond the grid, and where more than kList tokens share the last bin.
template <typename T>
__device__ void finish_any(const SampleLaunch& a, int n, const Settings& s, const T* row, float mx, FinishShared& sh) {
  const int tid = threadIdx.x, V = a.V;
  const float scale = s.scale;
  // Weights in units of 2^-43 of the largest: 2^20 of them fit a word.
  auto units = [=](float x) -> uint64_t {
    if (x == mx) return 1ull << 43;
    if (x == -INFINITY) return 0;
    return (uint64_t)rintf(__builtin_amdgcn_exp2f((x - mx) * scale) * 0x1p43f);
  };
  auto weight = [=](float x) -> double { return (double)units(x); };
  uint64_t sum = 0, count = 0, total, seen;
  for (int i = tid; i < V; i += kFinishThreads) {
    const float x = logit(row, i);
    sum += units(x);
    count += x > -INFINITY;
  }
  block_scan(sum, &total, sh.tmpu);
  block_scan(count, &seen, sh.tmpu);
  uint64_t last = 0;
  double least = -INFINITY;
  if (s.m > 0.f && scale > 0.f) least = mx < INFINITY ? (double)mx + log2((double)s.m) / (double)scale : (double)mx;
  for (int by_weight = 0; by_weight < 2; ++by_weight) {
    uint64_t want;
    if (by_weight) {
      if (s.p >= 1.f) break;
      want = max((uint64_t)1, (uint64_t)ceil((double)s.p * (double)total));
    } else {
      if (s.k == 0 || (uint64_t)s.k >= seen) continue;
      want = s.k;
    }
    // Words in [lo, hi]; `above` of the count or the weight lies past hi.
    uint64_t lo = word_of(-INFINITY, 0) + 1, hi = ~0ull, above = 0;
    for (int pass = 0; pass < 8 && lo < hi; ++pass) {  // 8 bits a pass
      const int shift = max(0, 64 - 8 - __builtin_clzll(hi - lo));
      __syncthreads();
      for (int i = tid; i < kBins; i += kFinishThreads) sh.bins[i] = 0;
      __syncthreads();
      for (int i = tid; i < V; i += kFinishThreads) {
        const float x = logit(row, i);
        const uint64_t w = word_of(x, i);
        if (x > -INFINITY && w >= lo && w <= hi && w >= last)
          atomicAdd(&sh.bins[(w - lo) >> shift], (unsigned long long)(by_weight ? units(x) : 1));
      }
      __syncthreads();
      // Bins from the top, a thread each.
      uint64_t all;
      const uint64_t mine = tid < kBins ? sh.bins[kBins - 1 - tid] : 0;
      const uint64_t before = above + block_scan(mine, &all, sh.tmpu);
      if (tid < kBins && before < want && before + mine >= want) {
        sh.pick[0] = kBins - 1 - tid;
        sh.picku[0] = before;
      }
      if (tid == 0 && above + all < want) {  // not reached: everything
        sh.pick[0] = 0;
        sh.picku[0] = above + all;
      }
      __syncthreads();
      const uint64_t base = lo + ((uint64_t)sh.pick[0] << shift);
      const uint64_t width = ((uint64_t)1 << shift) - 1;
      if (hi - base > width) hi = base + width;
      lo = base;
      above = sh.picku[0];
      __syncthreads();
    }
    last = max(last, lo);
    if (!by_weight && s.p < 1.f) {
      sum = 0;
      for (int i = tid; i < V; i += kFinishThreads) {
        const float x = logit(row, i);
        if (word_of(x, i) >= last) sum += units(x);
      }
      block_scan(sum, &total, sh.tmpu);
    }
  }
  const Kept kept{last, least};
  double part = 0.0, all;
  for (int i = tid; i < V; i += kFinishThreads) {
    const float x = logit(row, i);
    if (kept(x, i)) part += weight(x);
  }
  block_scan(part, &all, sh.tmp);
  const float u = a.u[n];
  const double at = u > 0.f ? (double)u * all : 0.0;
  draw_in(a, n, row, 0, V, at, all, kept, weight, sh);
}

template <typename T>
__global__ __launch_bounds__(kFinishThreads) void sample_finish_kernel(SampleLaunch a, int n_slices) {
  __shared__ FinishShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = blockIdx.x, V = a.V;
  const Settings s = settings_of(a, n);
  const T* row = reinterpret_cast<const T*>(a.logits) + (int64_t)n * a.stride;
  constexpr int64_t kStep = sizeof(SliceInfo) + kBins * 8;
  const char* in = static_cast<const char*>(a.ws) + (int64_t)n * n_slices * kStep;
  auto bins_of = [&](int i) { return reinterpret_cast<const unsigned long long*>(in + i * kStep + sizeof(SliceInfo)); };

  for (int i = tid; i < n_slices; i += kFinishThreads) sh.info[i] = *reinterpret_cast<const SliceInfo*>(in + i * kStep);
  for (int i = tid; i < kMaxSlices / 32; i += kFinishThreads) sh.wanted[i] = 0;
  if (tid < 4) sh.pick[tid] = kBins;
  __syncthreads();
  float mx = -INFINITY;
  int top = -0x7FFFFFFF;
  bool beyond = false, left = false;
  for (int i = 0; i < n_slices; ++i) {
    mx = fmaxf(mx, sh.info[i].max);
    left = left || sh.info[i].left;
    if (sh.info[i].n_bins < 0) beyond = true;
    else if (sh.info[i].max > -INFINITY) top = max(top, sh.info[i].top);
  }
  if (mx == -INFINITY) {
    if (tid == 0) answer(a, n, -1, 0.0);
    return;
  }
  if (beyond) {
    finish_any(a, n, s, row, mx, sh);
    return;
  }
  const float scale = s.scale;
  const float u = a.u[n];
  // A weight relative to the edge of the row's top bin.
  auto weight = [=](float x) -> double {
    const float b = bin_of(x, scale);
    return rintf(over_edge(x, scale, b) * kUnit) * pow2(((double)b - top) * 0.125);
  };

  if (s.k == 0 && s.p >= 1.f && s.m == 0.f) {
    // Everything is kept: the slice by the slices' sums, then the token.
    double w = tid < n_slices && sh.info[tid].max > -INFINITY
                   ? sh.info[tid].rest * pow2(((double)sh.info[tid].max - (double)mx) * (double)scale)
                   : 0.0;
    double all;
    const double before = block_scan(w, &all, sh.tmp);
    const double at = u > 0.f ? fmin((double)u * all, all) : 0.0;
    if (tid == 0) sh.pick[0] = -1, sh.pick[1] = 0x7FFFFFFF;
    __syncthreads();
    if (w > 0.0) atomicMax(&sh.pick[0], tid);
    if (w > 0.0 && before + w > at) atomicMin(&sh.pick[1], tid);
    __syncthreads();
    const int slice = sh.pick[1] == 0x7FFFFFFF ? sh.pick[0] : sh.pick[1];
    if (tid == slice) sh.value[0] = before;
    __syncthreads();
    const double start = sh.value[0];
    auto plain = [=](float x) -> double {
      return x == mx ? 1.0 : pow2(((double)x - (double)mx) * (double)scale);
    };
    draw_in(a, n, row, slice * kSlice, min(V, (slice + 1) * kSlice), at - start, all, Kept{0, -INFINITY}, plain, sh);
    return;
  }

  // The row's bins, and the first one (from the top) at which the kept tokens
  // have ended for sure: `end`.
  uint64_t units = 0, count = 0;
  if (tid < kBins) {
    for (int i = 0; i < n_slices; ++i) {
      if (sh.info[i].max == -INFINITY) continue;
      const int j = tid - (top - sh.info[i].top);
      if (j >= 0 && j < sh.info[i].n_bins) {
        const uint64_t x = bins_of(i)[j];
        count += x >> kCountShift;
        units += x & ((1ull << kCountShift) - 1);
      }
    }
  }
  const double here = (double)units * pow2(-0.125 * tid);
  uint64_t all_c;
  double all_w;
  const uint64_t before_c = block_scan(count, &all_c, sh.tmpu);
  const double before_w = block_scan(here, &all_w, sh.tmp);
  double least = -INFINITY;
  if (s.m > 0.f) least = (double)mx + log2((double)s.m) / (double)scale;
  double target = 0.0;
  if (s.k > 0) {
    if (tid < kBins && before_c < (uint64_t)s.k && before_c + count >= (uint64_t)s.k) sh.pick[0] = tid;
  } else if (s.p < 1.f) {
    // The sum of everything: the bins and the slices' rests.
    double rest = tid < n_slices && sh.info[tid].max > -INFINITY
                      ? sh.info[tid].rest * kUnit * pow2((double)sh.info[tid].max * (double)scale - 0.125 * top)
                      : 0.0;
    double all_rest;
    block_scan(rest, &all_rest, sh.tmp);
    target = (double)s.p * (all_w + all_rest);
    if (tid < kBins && before_w < target && before_w + here >= target) sh.pick[0] = tid;
  }
  if (tid == 0 && s.m > 0.f) {
    const double j = (double)top - (double)bin_of((float)least, scale);
    if (j < kBins) sh.pick[1] = (int)j;
  }
  __syncthreads();
  int end = sh.pick[0];
  if (s.k == 0) end = min(end, sh.pick[1]);
  else if (all_c < (uint64_t)s.k && !left) end = kBins - 1;  // fewer than k tokens: all of them
  if (end == kBins) {  // below the bins
    finish_any(a, n, s, row, mx, sh);
    return;
  }
  // Tokens down to `end`, or the last bin's alone if those are too many.
  if (tid == end) {
    sh.picku[0] = before_c + count;
    sh.picku[1] = before_c;
    sh.value[0] = before_w;
  }
  __syncthreads();
  const uint64_t down_to = sh.picku[0], in_last = down_to - sh.picku[1];
  const bool whole = down_to <= kList;
  if (!whole && (in_last > kList || s.k > 0)) {
    finish_any(a, n, s, row, mx, sh);
    return;
  }
  const double above = whole ? 0.0 : sh.value[0];
  const int from = whole ? 0 : end;
  __syncthreads();
  if (tid == 0) sh.pick[2] = 0;
  // Slices with such tokens.
  for (int i = wave; i < n_slices; i += kFinishThreads / 64) {
    if (sh.info[i].max == -INFINITY) continue;
    const int off = top - sh.info[i].top;
    bool any = false;
    for (int j = from + lane; j <= end; j += 64) any = any || (j - off >= 0 && j - off < sh.info[i].n_bins && bins_of(i)[j - off]);
    if (__any(any) && lane == 0) atomicOr(&sh.wanted[i / 32], 1u << (i % 32));
  }
  __syncthreads();
  const float first = (float)top - from, lastb = (float)top - end;
  for (int i = wave; i < n_slices * (kSlice / 512); i += kFinishThreads / 64) {
    const int slice = i / (kSlice / 512);
    if (!(sh.wanted[slice / 32] >> (slice % 32) & 1)) continue;
    const int at = i * 512 + lane * 8;
    T raw[8];
    float x[8];
    if (at + 8 <= V) {
      __builtin_memcpy(raw, row + at, sizeof(raw));
#pragma unroll
      for (int c = 0; c < 8; ++c) x[c] = clean((float)raw[c]);
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) x[c] = at + c < V ? logit(row, at + c) : -INFINITY;
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const float b = bin_of(x[c], scale);
      if (b <= first && b >= lastb) {
        const int slot = atomicAdd(&sh.pick[2], 1);
        if (slot < kList) sh.list[slot] = word_of(x[c], at + c);
      }
    }
  }
  __syncthreads();
  const int m = min(sh.pick[2], kList);
  int padded = 64;
  while (padded < m) padded *= 2;
  for (int i = m + tid; i < padded; i += kFinishThreads) sh.list[i] = 0;
  sort_falling(sh.list, padded);

  // The kept ones among them, in falling order; a thread takes a run.
  const int per = (padded + kFinishThreads - 1) / kFinishThreads;
  const int lo = min(m, tid * per), hi = min(m, lo + per);
  double sum = 0.0;
  for (int i = lo; i < hi; ++i) {
    const double w = weight(float_of_key((uint32_t)(sh.list[i] >> 32)));
    sh.value[i] = w;
    if (s.k == 0 || i < s.k) sum += w;
  }
  double sum_k;
  const double before = above + block_scan(sum, &sum_k, sh.tmp);
  if (s.k > 0) target = (double)s.p * sum_k;
  double cum = before, kept_sum = 0.0;
  int n_kept = 0;
  for (int i = lo; i < hi; ++i) {
    const bool by_k = s.k == 0 || i < s.k;
    const bool by_p = s.p >= 1.f || cum < target || (i == 0 && above == 0.0);
    const bool by_m = (double)float_of_key((uint32_t)(sh.list[i] >> 32)) >= least;
    cum += sh.value[i];
    if (!(by_k && by_p && by_m)) break;  // each holds for a leading part
    ++n_kept;
    kept_sum += sh.value[i];
  }
  uint64_t n_all;
  block_scan((uint64_t)n_kept, &n_all, sh.tmpu);
  double total;
  block_scan(kept_sum, &total, sh.tmp);
  total += above;
  const double at = u > 0.f ? fmin((double)u, 1.0) * total : 0.0;

  if (whole) {
    // In order of index: the words become (index, place).
    const int keep = (int)n_all;
    int size = 64;
    while (size < keep) size *= 2;
    uint64_t mine[kList / kFinishThreads];
#pragma unroll
    for (int c = 0; c < kList / kFinishThreads; ++c) {
      const int i = tid + c * kFinishThreads;
      mine[c] = i < keep ? (sh.list[i] << 32) | (uint32_t)(sh.list[i] >> 32) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kList / kFinishThreads; ++c) {
      const int i = tid + c * kFinishThreads;
      if (i < size) sh.list[i] = mine[c];
    }
    sort_falling(sh.list, size);  // ~index falls: indexes rise
    const int pr = (size + kFinishThreads - 1) / kFinishThreads;
    const int l0 = min(keep, tid * pr), l1 = min(keep, l0 + pr);
    double part = 0.0, all;
    int last = -1;
    for (int i = l0; i < l1; ++i) {
      const double w = weight(float_of_key((uint32_t)sh.list[i]));
      sh.value[i] = w;
      part += w;
      if (w > 0.0) last = i;
    }
    const double b0 = block_scan(part, &all, sh.tmp);
    if (tid == 0) sh.pick[0] = -1, sh.pick[1] = 0x7FFFFFFF;
    __syncthreads();
    if (last >= 0) atomicMax(&sh.pick[0], last);
    if (part > 0.0 && b0 + part > at) {
      double c = b0;
      for (int i = l0; i < l1; ++i) {
        c += sh.value[i];
        if (sh.value[i] > 0.0 && c > at) {
          atomicMin(&sh.pick[1], i);
          break;
        }
      }
    }
    __syncthreads();
    if (tid == 0) {
      const int i = sh.pick[1] == 0x7FFFFFFF ? sh.pick[0] : sh.pick[1];
      answer(a, n, (int)~(uint32_t)(sh.list[i] >> 32), sh.value[i] / total);
    }
    return;
  }

  // Many kept tokens: the slice by the kept weight of each, then the token.
  __syncthreads();
  if (tid == 0) sh.picku[0] = n_all ? sh.list[n_all - 1] : ~0ull;
  __syncthreads();
  // No token of the last bin kept: those above it, whose words are larger than
  // any of the bin's.
  const uint64_t last = n_all ? sh.picku[0] : sh.list[0] + 1;
  const Kept kept{last, least};
  __syncthreads();
  for (int i = tid; i < n_slices; i += kFinishThreads) sh.slice_w[i] = 0.0;
  for (int i = wave; i < n_slices; i += kFinishThreads / 64) {
    if (sh.info[i].max == -INFINITY) continue;
    const int off = top - sh.info[i].top;
    double w = 0.0;
    for (int j = lane; j < end; j += 64)
      if (j - off >= 0 && j - off < sh.info[i].n_bins)
        w += (double)(bins_of(i)[j - off] & ((1ull << kCountShift) - 1)) * pow2(-0.125 * j);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) w += __shfl_xor(w, d);
    double extra = 0.0;
    for (uint32_t j = lane; j < (uint32_t)n_all; j += 64)
      if ((int)(~(uint32_t)sh.list[j] / kSlice) == i) extra += sh.value[j];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) extra += __shfl_xor(extra, d);
    if (lane == 0) sh.slice_w[i] = w + extra;
  }
  __syncthreads();
  const double w = tid < n_slices ? sh.slice_w[tid] : 0.0;
  double all;
  const double b0 = block_scan(w, &all, sh.tmp);
  if (tid == 0) sh.pick[0] = -1, sh.pick[1] = 0x7FFFFFFF;
  __syncthreads();
  if (w > 0.0) atomicMax(&sh.pick[0], tid);
  if (w > 0.0 && b0 + w > at) atomicMin(&sh.pick[1], tid);
  __syncthreads();
  const int slice = sh.pick[1] == 0x7FFFFFFF ? sh.pick[0] : sh.pick[1];
  if (tid == slice) sh.value[0] = b0;
  __syncthreads();
  const double start = sh.value[0];
  draw_in(a, n, row, slice * kSlice, min(V, (slice + 1) * kSlice), at - start, total, kept, weight, sh);
}

}  // namespace

size_t sample_workspace(int N, int V, int) {
  return (size_t)N * ((V + kSlice - 1) / kSlice) * (sizeof(SliceInfo) + kBins * 8);
}

hipError_t launch_sample(const SampleLaunch& a, int dtype, hipStream_t stream) {
  const int n_slices = (a.V + kSlice - 1) / kSlice;
  const dim3 grid((unsigned)n_slices, (unsigned)a.N);
  if (dtype == NACL_F32) {
    sample_slices_kernel<float><<<grid, kSliceThreads, 0, stream>>>(a, n_slices);
    if (hipError_t e = hipGetLastError()) return e;
    sample_finish_kernel<float><<<a.N, kFinishThreads, 0, stream>>>(a, n_slices);
  } else {
    sample_slices_kernel<__bf16><<<grid, kSliceThreads, 0, stream>>>(a, n_slices);
    if (hipError_t e = hipGetLastError()) return e;
    sample_finish_kernel<__bf16><<<a.N, kFinishThreads, 0, stream>>>(a, n_slices);
  }
  return hipGetLastError();
}

}  // namespace nacl
