// The next token of each row of logits by temperature, top-k, top-p and min-p
// (nacl_sample).
//
// Two launches and one pass over the logits.  sample_slices_kernel reads slices
// of a row (their size depends on V alone, so that a row's sums and its result do
// not depend on the batch) and sorts what can matter into bins of an eighth of a
// power of two of the weight: bin(x) = floor(8 x log2(e) / temperature), the same
// grid for every slice and without the row's maximum.  A bin holds the count of
// its tokens and the sum of their weights over the bin's lower edge, both as
// integers, so that the order of the atomics does not show; where few tokens are
// binned the slice lists them too.  sample_finish_kernel, a work-group per row,
// joins the slices, finds the bin in which the kept tokens end, collects the
// tokens of that bin (from the lists, or from the slices that have some) or, if
// they are few, all down to it, sorts them and draws.

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

constexpr int kSliceThreads = 512;
constexpr int kMinSlice = kSliceThreads * 16;            // tokens per slice: 16 or 32 per thread
constexpr int kBins = 256;                               // 32 powers of two below a slice's largest
constexpr int kMaxSlices = NACL_MAX_V / (2 * kMinSlice);
constexpr int kFinishThreads = 1024;
constexpr int kList = kFinishThreads;                    // tokens that the finish sorts, one per thread
constexpr int kWide = 6144;                              // tokens of a bin that it holds
constexpr int kKeep = 128;                               // tokens that a slice lists
constexpr float kUnit = 0x1p22f;                         // a weight over its bin's edge, in units: rounded by 2^-23
                                                         // of it as an fp32 exponential is, so that sums of
                                                         // integers need no order (log-probabilities good to 1.4e-7)
constexpr int kCountShift = 43;                          // of a bin word: count above, weight units below
constexpr uint64_t kUnitMask = ((uint64_t)1 << kCountShift) - 1;
constexpr int kFaint = 1024;                             // top-k: as many tokens below the bins (2^-32 of the
                                                         // largest each) weigh less than one unit, 2^-22 of it
constexpr float kMaxBin = 0x1p20f;                       // bins beyond are too coarse to use
static_assert(NACL_MAX_V < (1 << (64 - kCountShift)) && NACL_MAX_V * 1.1 * 0x1p22 < 0x1p43, "bin words");

// Long vocabularies take longer slices: a work-group then has more in flight, and
// the finish joins fewer (256 x 131072, top-k 50 47.7 us, by short slices 54.3; top-p
// 0.9 79.4 and 82.2).  Short ones need the work-groups (1 x 32000, top-p 0.9 30.5 us,
// by long slices 33.9; 32 x 50257 37.3 and 40.5).
constexpr int slice_of(int V) { return V > 65536 ? 2 * kMinSlice : kMinSlice; }
static_assert(65536 / kMinSlice <= kMaxSlices, "slices");

// What a slice leaves for the finish: this, then its bins, then its list.
struct SliceInfo {
  float max;     // largest logit
  int top;       // its bin (the slice's bins go down from it)
  int n_bins;    // bins filled; -1: the logits are beyond the grid
  int left;      // top-k: a token above -infinity lies below the bins
  double rest;   // weights outside the bins over the largest one's
  int n_list;    // tokens in the bins, as words; -1: too many for the list
  int first;     // top-k of 1: the first token of the largest logit
};
constexpr int kSliceBytes = sizeof(SliceInfo) + (kBins + kKeep) * 8;

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

// Order of tokens as falling words: larger logits first, then lower indexes.
__device__ __forceinline__ uint64_t word_of(float x, uint32_t i) { return (uint64_t)float_order_key(x) << 32 | (uint32_t)~i; }
__device__ __forceinline__ float float_of_key(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key);
}

// 8 E logits of a thread: runs of 8, `apart` tokens from one to the next, in
// range below `end`.
template <typename T, int E>
__device__ __forceinline__ void load_run(const T* row, int i0, int apart, int end, float (&x)[8 * E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = i0 + e * apart;
    T raw[8];
    if (i + 8 <= end) {
      __builtin_memcpy(raw, row + i, sizeof(raw));
#pragma unroll
      for (int c = 0; c < 8; ++c) x[8 * e + c] = clean((float)raw[c]);
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) x[8 * e + c] = i + c < end ? logit(row, i + c) : -INFINITY;
    }
  }
}

// 256 x 131072 bf16 in 32 us (67 MB: 2.1 TB/s): vector instructions bound it, about
// 21 per token (half of the issue slots) besides the LDS atomics of the binned tokens.
// 1 x 32000: 5 us, the launch and the chain of loads, maximum, bins and sums.
template <typename T, int E>
__global__ __launch_bounds__(kSliceThreads) void sample_slices_kernel(SampleLaunch a, int n_slices) {
  constexpr int kPer = 8 * E, kSlice = kSliceThreads * kPer;
  __shared__ unsigned long long bins[kBins];
  __shared__ uint64_t list[kKeep];
  __shared__ uint32_t tops[kBins];
  __shared__ float wmax[kSliceThreads / 64];
  __shared__ double wrest[kSliceThreads / 64];
  __shared__ int need, listed;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int slice = blockIdx.x, n = blockIdx.y;
  const T* row = reinterpret_cast<const T*>(a.logits) + (int64_t)n * a.stride;

  float x[kPer];
  const int i0 = slice * kSlice + 8 * tid;
  load_run<T, E>(row, i0, kSliceThreads * 8, a.V, x);
  const Settings s = settings_of(a, n);
  if (tid < kBins) {
    bins[tid] = 0;
    tops[tid] = 0;
  }
  if (tid == 0) {
    listed = 0;
    need = 0x7FFFFFFF;
  }
  float tmax = x[0];
#pragma unroll
  for (int i = 1; i < kPer; ++i) tmax = fmaxf(tmax, x[i]);
  float mx = tmax;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) mx = fmaxf(mx, __shfl_xor(mx, d));
  if (lane == 0) wmax[wave] = mx;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSliceThreads / 64; ++w) mx = fmaxf(mx, wmax[w]);

  SliceInfo* info = reinterpret_cast<SliceInfo*>(static_cast<char*>(a.ws) + ((int64_t)n * n_slices + slice) * kSliceBytes);
  if (s.k == 1) {
    // No bins: the first of the largest (1 x 32000 6.2 us, by bins 19.1; 256 x
    // 131072 19.7 and 41.0).
    int at = 0x7FFFFFFF;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i)
      if (x[i] == mx) at = i0 + (i / 8) * kSliceThreads * 8 + i % 8;
    if (at != 0x7FFFFFFF) atomicMin(&need, at);
    __syncthreads();
    if (tid == 0) *info = SliceInfo{mx, 0, 0, 0, 0.0, 0, need};
    return;
  }
  const float top = bin_of(mx, s.scale);
  // All hidden, or beyond the grid (infinite and NaN products among that).
  if (mx == -INFINITY || !(__builtin_fabsf(top) < kMaxBin) || s.scale < 0x1p-60f) {
    if (tid == 0) *info = SliceInfo{mx, 0, mx == -INFINITY ? 0 : -1, 0, 0.0, 0, 0};
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
  if (n_bins > 0) {
    const bool with_rest = s.k == 0 && s.p < 1.f;
    const float n_binsf = (float)n_bins;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float b = bin_of(x[i], s.scale), j = top - b;
      if (j < n_binsf) {
        atomicAdd(&bins[(int)j], (1ull << kCountShift) + (uint32_t)rintf(over_edge(x[i], s.scale, b) * kUnit));
        if (listed <= kKeep) {  // a count past kKeep says that there are more
          const int at = atomicAdd(&listed, 1);
          if (at < kKeep) list[at] = word_of(x[i], i0 + (i / 8) * kSliceThreads * 8 + i % 8);
        }
      } else if (with_rest) {
        rest += __builtin_amdgcn_exp2f((x[i] - mx) * s.scale);
      } else {
        left = left || x[i] > -INFINITY;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) rest += __builtin_amdgcn_exp2f((x[i] - mx) * s.scale);
  }
  double total = rest;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d);
  if (lane == 0) wrest[wave] = total;
  const int any_left = __syncthreads_or(left);
  if (tid == 0) {
    total = 0.0;
    for (int w = 0; w < kSliceThreads / 64; ++w) total += wrest[w];
    *info = SliceInfo{mx, (int)top, n_bins, any_left, total, n_bins > 0 && listed <= kKeep ? listed : -1, 0};
  }
  unsigned long long* words = reinterpret_cast<unsigned long long*>(info + 1);
  if (tid < n_bins) words[tid] = bins[tid];
  if (tid < min(listed, kKeep)) words[kBins + tid] = list[tid];
}

// One work-group and a long chain of steps: what counts in the finish is latency,
// so lanes exchange by DPP and permlane moves (a few cycles) and not through LDS
// (over a hundred).

template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint32_t dpp(uint32_t old, uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS = 0xF, typename U>
__device__ __forceinline__ U dpp64(U x) {  // lanes without a source: 0
  const uint64_t v = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(U, (uint64_t)dpp<CTRL, ROWS>(0, (uint32_t)(v >> 32)) << 32 | dpp<CTRL, ROWS>(0, (uint32_t)v));
}
// Inclusive sums over the wave: rows of 16 by shifts, then the last lane of row
// 0 to row 1 and of row 2 to row 3, then of row 1 to rows 2 and 3.
template <typename U>
__device__ __forceinline__ U wave_scan(U x) {
  x += dpp64<0x111>(x);
  x += dpp64<0x112>(x);
  x += dpp64<0x114>(x);
  x += dpp64<0x118>(x);
  x += dpp64<0x142, 0xA>(x);
  x += dpp64<0x143, 0xC>(x);
  return x;
}
// The value of lane ^ J.
template <int J>
__device__ __forceinline__ uint32_t swap_lanes(uint32_t x) {
  if constexpr (J == 1) return dpp<0xB1>(x, x);
  if constexpr (J == 2) return dpp<0x4E>(x, x);
  if constexpr (J == 4) {
    const uint32_t y = dpp<0x141>(x, x);  // lane ^ 7
    return dpp<0x1B>(y, y);               // lane ^ 3
  }
  if constexpr (J == 8) return dpp<0x128>(x, x);
  if constexpr (J == 16) {
    auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? a[0] : a[1];
  }
  if constexpr (J == 32) {
    auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return threadIdx.x & 32 ? a[0] : a[1];
  }
}

// Exclusive sums in thread order and the sum of all, by a fixed tree.
template <typename U>
__device__ __forceinline__ U block_scan(U x, U* total, U* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const U s = wave_scan(x);
  __syncthreads();
  if (lane == 63) tmp[wave] = s;
  __syncthreads();
  const U t = tmp[lane & 15], sums = wave_scan(lane < 16 ? t : U(0));  // of the 16 waves
  auto of = [&](int i) {
    const uint64_t v = __builtin_bit_cast(uint64_t, sums);
    return __builtin_bit_cast(U, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32 |
                                     (uint32_t)__builtin_amdgcn_readlane((int)v, i));
  };
  *total = of(15);
  return (wave ? of(__builtin_amdgcn_readfirstlane(wave) - 1) : U(0)) + (s - x);
}

// One step of a sort: words J threads apart are put in order, those of a run of
// `size` threads falling where the run's number is even.
template <int J>
__device__ __forceinline__ void sort_step(uint64_t& v, int size, uint64_t* tmp) {
  const int tid = threadIdx.x;
  uint64_t other;
  if constexpr (J >= 64) {
    __syncthreads();
    tmp[tid] = v;
    __syncthreads();
    other = tmp[tid ^ J];
  } else {
    other = (uint64_t)swap_lanes<J>((uint32_t)(v >> 32)) << 32 | swap_lanes<J>((uint32_t)v);
  }
  const bool larger = ((tid & J) == 0) == ((tid & size) == 0);
  if ((other > v) == larger) v = other;
}
// Sorts words in falling order, one per thread, those of the first `n` threads
// (a power of two from 64 on; every thread takes part, the waves past them only
// in the barriers).
__device__ __noinline__ uint64_t sort_falling(uint64_t v, int n, uint64_t* tmp) {
  const bool mine = (int)(threadIdx.x & ~63u) < n;
#pragma unroll 1
  for (int size = 2; size <= n; size *= 2) {
    if (size >= 1024) sort_step<512>(v, size, tmp);
    if (size >= 512) sort_step<256>(v, size, tmp);
    if (size >= 256) sort_step<128>(v, size, tmp);
    if (size >= 128) sort_step<64>(v, size, tmp);
    if (!mine) continue;
    if (size >= 64) sort_step<32>(v, size, tmp);
    if (size >= 32) sort_step<16>(v, size, tmp);
    if (size >= 16) sort_step<8>(v, size, tmp);
    if (size >= 8) sort_step<4>(v, size, tmp);
    if (size >= 4) sort_step<2>(v, size, tmp);
    sort_step<1>(v, size, tmp);
  }
  __syncthreads();
  return v;
}

// 2^(-j / 8); root: of j from 0 to 7.
__device__ __forceinline__ double eighths(const double* root, int j) { return ldexp(root[j & 7], -(j >> 3)); }
// (Made of instructions: a table in memory would cost the first reader of its page
// some microseconds.)
__device__ __forceinline__ double root_of(int j) {
  constexpr double kRoot[8] = {1.0,
                               0.91700404320467123174,
                               0.84089641525371454303,
                               0.77110541270397041180,
                               0.70710678118654752440,
                               0.64841977732550483297,
                               0.59460355750136053336,
                               0.54525386633262882702};
  double r = kRoot[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) r = j == i ? kRoot[i] : r;
  return r;
}

struct FinishShared {
  uint64_t list[kList], wide[kWide];
  double root[8];
  double tmp[kFinishThreads / 64];
  uint64_t tmpu[kFinishThreads / 64];
  unsigned long long bins[kBins];          // finish_any: a pass's; otherwise the row's
  uint64_t before_c[kBins + 1];            // tokens above each bin, and their weight
  double before_w[kBins + 1];
  SliceInfo info[kMaxSlices];
  double slice_w[kMaxSlices];
  unsigned long long extra[kMaxSlices];    // units of a slice's tokens of the last bin above the list's
  int pick[4];
  int first[kFinishThreads / 64], last[kFinishThreads / 64];
  uint64_t picku;
  double pickd;
};

// Which tokens are kept: those whose word is at least `last` and logit at least
// `least`.
struct Kept {
  uint64_t last;
  float least;
  __device__ __forceinline__ bool operator()(float x, uint32_t i) const {
    return x > -INFINITY && word_of(x, i) >= last && x >= least;
  }
};
// The smallest logit that min-p keeps.
__device__ __forceinline__ float least_of(const Settings& s, float mx) {
  if (!(s.m > 0.f) || !(s.scale > 0.f)) return -INFINITY;
  if (mx == INFINITY) return mx;
  const double limit = (double)mx + log2((double)s.m) / (double)s.scale;
  const float x = (float)limit;
  return (double)x < limit ? float_of_key(float_order_key(x) + 1) : x;
}

__device__ __noinline__ void answer(int32_t* token_at, float* logprob_at, int token, double p) {
  *token_at = token;
  // (close to 1 by what is missing from it)
  if (logprob_at) *logprob_at = token < 0 ? -INFINITY : p > 0.5 ? log1pf((float)(p - 1.0)) : logf((float)p);
}
__device__ __forceinline__ void answer(const SampleLaunch& a, int n, int token, double p) {
  answer(a.tokens + n, a.logprobs ? a.logprobs + n : nullptr, token, p);
}

// Threads' candidates in order: the first at which the running sum, `before` plus
// the thread's `sum`, passes `at`; of a sum that falls short by rounding, the last
// thread with a weight.
__device__ __forceinline__ int pick_thread(double before, double sum, double at, FinishShared& sh) {
  const int wave = threadIdx.x >> 6;
  const uint64_t with = __ballot(sum > 0.0), past = __ballot(sum > 0.0 && before + sum > at);
  if ((threadIdx.x & 63) == 0) {
    sh.first[wave] = past ? 64 * wave + __builtin_ctzll(past) : 0x7FFFFFFF;
    sh.last[wave] = with ? 64 * wave + 63 - __builtin_clzll(with) : -1;
  }
  __syncthreads();
  int first = 0x7FFFFFFF, last = -1;
#pragma unroll
  for (int w = 0; w < kFinishThreads / 64; ++w) {
    first = min(first, sh.first[w]);
    last = max(last, sh.last[w]);
  }
  __syncthreads();
  return first == 0x7FFFFFFF ? last : first;
}

// A number of the caller's, at most the largest below 1 (at 1 the rounding of the
// sum would decide); a NaN stays one.
__device__ __forceinline__ float below_one(float u) { return u < 0x1.fffffep-1f ? u : u >= 1.f ? 0x1.fffffep-1f : u; }

// The draw among the kept tokens of a slice, of which the one is wanted at which
// the sum of the weights passes `at`.  A thread takes a run of 8 E tokens.
template <typename T, int E, class W>
__device__ void draw_slice(const SampleLaunch& a, int n, const T* row, int slice, double at, double total, const Kept& kept,
                           const W& weight, FinishShared& sh) {
  constexpr int kPer = 8 * E;
  const int lo = (slice * kFinishThreads + (int)threadIdx.x) * kPer;
  float x[kPer];
  load_run<T, E>(row, lo, 8, a.V, x);
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (kept(x[i], lo + i)) sum += weight(x[i]);
  double all;
  const double before = block_scan(sum, &all, sh.tmp);
  // That thread's tokens again, a lane each.
  const int thread = max(0, pick_thread(before, sum, at, sh));
  if ((int)threadIdx.x == thread) sh.pickd = before;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  const int lane = threadIdx.x, i = (slice * kFinishThreads + thread) * kPer + lane;
  const float y = lane < kPer && i < a.V ? logit(row, i) : -INFINITY;
  const double w = kept(y, i) ? weight(y) : 0.0;
  double cum = w;
#pragma unroll
  for (int d = 1; d < kPer; d *= 2) {
    const double z = __shfl_up(cum, d);
    if (lane >= d) cum += z;
  }
  const uint64_t with = __ballot(w > 0.0), past = __ballot(w > 0.0 && sh.pickd + cum > at);
  if (lane == (past ? __builtin_ctzll(past) : 63 - __builtin_clzll(with | 1))) answer(a, n, i, w / total);
}

// Any row, slowly: the last kept token by a search over the words' range that
// narrows it 256-fold a pass, then the draw over the whole row.  For logits
// beyond the grid, and where the slices' bins do not suffice (a top-k or top-p that
// ends below them).
template <typename T>
__device__ void finish_any(const SampleLaunch& a, int n, const Settings& s, const T* row, float mx, float least, FinishShared& sh) {
  const int tid = threadIdx.x, V = a.V;
  const float scale = s.scale;
  // Weights in units of 2^-43 of the largest: 2^20 of them fit a word.
  auto units = [=](float x) -> uint64_t {
    if (x == mx) return 1ull << 43;
    if (x == -INFINITY || mx == INFINITY) return 0;  // (an infinite temperature's 0 times infinity: NaN)
    return (uint64_t)rintf(__builtin_amdgcn_exp2f((x - mx) * scale) * 0x1p43f);
  };
  auto weight = [=](float x) -> double { return (double)units(x); };
  // Calls f(logit, index) for every token (and with -infinity past the last).
  auto every = [&](auto f) {
    for (int i0 = tid * 8; i0 < V; i0 += kFinishThreads * 8) {
      float x[8];
      load_run<T, 1>(row, i0, 0, V, x);
#pragma unroll
      for (int c = 0; c < 8; ++c) f(x[c], (uint32_t)(i0 + c));
    }
  };
  uint64_t sum = 0, count = 0, total, seen;
  every([&](float x, uint32_t) {
    sum += units(x);
    count += x > -INFINITY;
  });
  block_scan(sum, &total, sh.tmpu);
  block_scan(count, &seen, sh.tmpu);
  uint64_t last = 0;
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
      every([&](float x, uint32_t i) {
        const uint64_t w = word_of(x, i);
        if (x > -INFINITY && w >= lo && w <= hi && w >= last)
          atomicAdd(&sh.bins[(w - lo) >> shift], (unsigned long long)(by_weight ? units(x) : 1));
      });
      __syncthreads();
      // Bins from the top, a thread each.
      uint64_t all;
      const uint64_t mine = tid < kBins ? sh.bins[kBins - 1 - tid] : 0;
      const uint64_t before = above + block_scan(mine, &all, sh.tmpu);
      if (tid < kBins && before < want && before + mine >= want) {
        sh.pick[0] = kBins - 1 - tid;
        sh.picku = before;
      }
      if (tid == 0 && above + all < want) {  // not reached: everything
        sh.pick[0] = 0;
        sh.picku = above + all;
      }
      __syncthreads();
      const uint64_t base = lo + ((uint64_t)sh.pick[0] << shift);
      const uint64_t width = ((uint64_t)1 << shift) - 1;
      if (hi - base > width) hi = base + width;
      lo = base;
      above = sh.picku;
      __syncthreads();
    }
    last = max(last, lo);
    if (!by_weight && s.p < 1.f) {
      sum = 0;
      every([&](float x, uint32_t i) {
        if (word_of(x, i) >= last) sum += units(x);
      });
      block_scan(sum, &total, sh.tmpu);
    }
  }
  const Kept kept{last, least};
  const int per = (V + kFinishThreads - 1) / kFinishThreads;
  const int i0 = min(V, tid * per), i1 = min(V, i0 + per);
  double part = 0.0, all;
  for (int i = i0; i < i1; ++i) {
    const float x = logit(row, i);
    if (kept(x, i)) part += weight(x);
  }
  const double before = block_scan(part, &all, sh.tmp);
  const float u = below_one(a.u[n]);
  const double at = u > 0.f ? (double)u * all : 0.0;
  if (tid == pick_thread(before, part, at, sh)) {
    double cum = before, w_of = 0.0;
    int token = -1;
    for (int i = i0; i < i1; ++i) {
      const float x = logit(row, i);
      const double w = kept(x, i) ? weight(x) : 0.0;
      if (w > 0.0 && (token < 0 || cum <= at)) {
        token = i;
        w_of = w;
      }
      cum += w;
    }
    answer(a, n, token, w_of / all);
  }
}

// A row from its slices' bins; false where they do not suffice.
template <typename T, int E>
__device__ __forceinline__ bool finish_bins(const SampleLaunch& a, int n, int n_slices, const Settings& s, const T* row, const char* in,
                                            float mx, float least, int top, bool left, bool unlisted, FinishShared& sh) {
  constexpr int kSlice = kFinishThreads * 8 * E;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float u = below_one(a.u[n]);
  auto words_of = [&](int i) { return reinterpret_cast<const unsigned long long*>(in + i * kSliceBytes + sizeof(SliceInfo)); };
  const float scale = s.scale;
  auto logit_of = [](uint64_t w) { return float_of_key((uint32_t)(w >> 32)); };
  // A weight relative to the edge of the row's top bin, in units.
  auto weight = [&](float x) -> double {
    const float b = bin_of(x, scale);
    return (double)rintf(over_edge(x, scale, b) * kUnit) * eighths(sh.root, top - (int)b);
  };
  // Each slice's weight outside its bins, relative to the row's largest (of a
  // slice whose tokens' fp32 weights may all be 0: nothing).
  auto rest_of = [&](int i) -> double {
    if (i >= n_slices || sh.info[i].max == -INFINITY) return 0.0;
    const double x = ((double)sh.info[i].max - (double)mx) * (double)scale;
    return x < -120.0 ? 0.0 : sh.info[i].rest * exp2(x);
  };

  if (s.k == 0 && s.p >= 1.f && s.m == 0.f) {
    // Everything is kept: the slice by the slices' sums, then the token.
    const double w = rest_of(tid);
    double all;
    const double before = block_scan(w, &all, sh.tmp);
    const double at = u > 0.f ? (double)u * all : 0.0;
    const int slice = pick_thread(before, w, at, sh);
    if (tid == slice) sh.pickd = before;
    __syncthreads();
    auto plain = [=](float x) -> double { return (double)__builtin_amdgcn_exp2f((x - mx) * scale); };
    draw_slice<T, E>(a, n, row, slice, at - sh.pickd, all, Kept{0, -INFINITY}, plain, sh);
    return true;
  }

  // The row's bins.
  uint64_t units = 0, count = 0, under = 0;  // (`under` the row's bins: a slice's lower ones)
  if (tid < kBins) {
    for (int i = 0; i < n_slices; ++i) {
      const SliceInfo& f = sh.info[i];
      const int j = tid - (top - f.top);
      if (f.max > -INFINITY && j >= 0 && j < f.n_bins) {
        const uint64_t x = words_of(i)[j];
        count += x >> kCountShift;
        units += x & kUnitMask;
      }
      if (f.max > -INFINITY && j + kBins >= 0 && j + kBins < f.n_bins) under += words_of(i)[j + kBins] & kUnitMask;
    }
  }
  const double here = (double)units * eighths(sh.root, tid < kBins ? tid : 0);
  uint64_t all_c;
  double all_w;
  const uint64_t before_c = block_scan(count, &all_c, sh.tmpu);
  const double before_w = block_scan(here, &all_w, sh.tmp);
  if (tid < kBins) {
    sh.before_c[tid] = before_c;
    sh.before_w[tid] = before_w;
    if (tid == kBins - 1) {
      sh.before_c[kBins] = all_c;
      sh.before_w[kBins] = all_w;
    }
  }
  double target = INFINITY;
  if (s.k == 0 && s.p < 1.f) {
    // Of the sum of everything: the bins and the slices' rests.
    double all_rest;
    block_scan(rest_of(tid) * (kUnit * exp2((double)mx * (double)scale - 0.125 * top)) + (double)under * eighths(sh.root, (tid & 255) + kBins),
               &all_rest, sh.tmp);
    target = (double)s.p * (all_w + all_rest);
  }
  __syncthreads();
  // The first bin, from the top, down to which the top k lie (or the top-p
  // target) and the min-p limit's: the kept tokens end at `end`.
  if (tid < kBins) {
    const bool by_k = s.k > 0 && before_c < (uint64_t)s.k && sh.before_c[tid + 1] >= (uint64_t)s.k;
    const bool by_p = s.k == 0 && s.p < 1.f && before_w < target && sh.before_w[tid + 1] >= target;
    if (by_k || by_p) sh.pick[0] = tid;
  }
  if (tid == 0 && s.m > 0.f) {
    const float j = (float)top - bin_of(least, scale);
    if (j < kBins) sh.pick[1] = (int)j;
  }
  __syncthreads();
  int end = sh.pick[0];
  if (s.k == 0) end = min(end, sh.pick[1]);
  else if (all_c < (uint64_t)s.k && (!left || s.k <= kFaint)) end = kBins - 1;  // fewer than k tokens, or faint ones
  if (end >= kBins) return false;  // below the bins

  // The smallest logit of bin b (counted from the grid's origin) or a higher one:
  // a few steps around the quotient, a lane each.  (Bin 0 begins below 0, where the
  // product vanishes: at half of the smallest denormal.)
  auto first_of = [&](float b) {
    const float q = b == 0.f ? -0x1p-149f / (16.f * scale) : b / (8.f * scale);
    const float x = float_of_key(float_order_key(q) - 24 + lane);
    const uint64_t in = __ballot(bin_of(x, scale) >= b) | 1ull << 63;
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), __builtin_ctzll(in)));
  };
  // Calls f(word) for the tokens in bins from .. to, from the slices' lists
  // or, of slices that have such tokens and no list, from the logits.
  auto visit = [&](int from, int to, auto f) {
    const float first = (float)(top - from), last = (float)(top - to);
    for (int i = wave; i < n_slices; i += kFinishThreads / 64) {
      for (int c = lane; c < sh.info[i].n_list; c += 64) {
        const uint64_t w = words_of(i)[kBins + c];
        const float b = bin_of(logit_of(w), scale);
        if (b <= first && b >= last) f(w);
      }
    }
    if (unlisted) {
      // The bins' range as one of logits: one conversion and two comparisons each,
      // which bound this.
      const float lo = first_of(last), hi = first_of(first + 1.f);
      auto inside = [&](float x) { return x >= lo && x < hi; };
      constexpr int kBatch = 8 / (int)sizeof(T);  // runs of 8 in flight per thread
      const int n_runs = n_slices * E;
      for (int c0 = 0; c0 < n_runs; c0 += kBatch) {
        T raw[kBatch][8];
        uint32_t runs = 0, mask = 0;
        auto start = [&](int b) { return ((c0 + b) * kFinishThreads + tid) * 8; };
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const int slice = (c0 + b) / E;
          if (slice < n_slices) {
            const SliceInfo& g = sh.info[slice];
            const int off = top - g.top;
            if (g.max > -INFINITY && g.n_list < 0 && to >= off && from - off < g.n_bins) runs |= 1u << b;
          }
          if (runs >> b & 1 && start(b) + 8 <= a.V) __builtin_memcpy(raw[b], row + start(b), sizeof(raw[b]));
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
          if (runs >> b & 1) {
            if (start(b) + 8 <= a.V) {
              bool any = false;
#pragma unroll
              for (int c = 0; c < 8; ++c) any |= inside((float)raw[b][c]);
              if (__any(any)) {
#pragma unroll
                for (int c = 0; c < 8; ++c) mask |= inside((float)raw[b][c]) ? 1u << (8 * b + c) : 0u;
              }
            } else {
              for (int c = 0; start(b) + c < a.V; ++c) mask |= inside(logit(row, start(b) + c)) ? 1u << (8 * b + c) : 0u;
            }
          }
        for (; mask; mask &= mask - 1) {  // few
          const int c = __builtin_ctz(mask), i = start(c / 8) + c % 8;
          f(word_of(logit(row, i), (uint32_t)i));
        }
      }
    }
    __syncthreads();
  };
  auto slice_index = [](uint64_t word) { return (int)(~(uint32_t)word / kSlice); };
  auto units_of = [=](uint64_t word) {
    const float x = logit_of(word);
    return (uint32_t)rintf(over_edge(x, scale, bin_of(x, scale)) * kUnit);
  };

  // All kept tokens, if few, or those at the end of the last bin, above which
  // `above` tokens of weight `above_w` are kept; and each one's weight.  With a
  // top-p limit on the top k in two steps: the top k's sum, then the bin in which
  // a part of it is reached.
  const bool whole = sh.before_c[end + 1] <= kList;
  uint64_t v = 0, above = 0;
  double w = 0.0, above_w = 0.0, sum;
  for (bool sum_k = s.k > 0 && s.p < 1.f;; sum_k = false) {
    if (!sum_k && !whole && s.k > 0) {
      __syncthreads();
      if (tid == 0) sh.pick[0] = end;
      __syncthreads();
      if (tid < end && sh.before_w[tid] < target && sh.before_w[tid + 1] >= target) sh.pick[0] = tid;
      __syncthreads();
      end = min(end, min(sh.pick[0], sh.pick[1]));
    }
    const int first = whole ? 0 : end;
    above = sh.before_c[first];
    above_w = sh.before_w[first];
    uint64_t n_here = sh.before_c[end + 1] - above;
    // Too many for the list: the part of the bin in which the kept tokens end, by
    // the bins' way of search over the words, 256 parts a pass, on the logits
    // until the bin's tokens fit the work-group's memory.
    bool held = false;
    int n_held = 0;
    // (the bin's edges, wider by what their rounding may be)
    const float b = (float)(top - end);
    uint64_t lo = (uint64_t)(float_order_key(b == 0.f ? -0x1p-60f : b / (8.f * scale)) - 16) << 32;
    uint64_t hi = (uint64_t)(float_order_key((b + 1.f) / (8.f * scale)) + 16) << 32;
    uint64_t w_lo = 0, w_hi = ~(uint64_t)0;
    __syncthreads();
    if (tid < kMaxSlices) sh.extra[tid] = 0;
    for (int pass = 0; pass < 10; ++pass) {
      const bool fits = n_here <= kWide;
      if (held && n_here <= kList) break;
      const int shift = max(0, 64 - 8 - __builtin_clzll((hi - lo) | 255));
      auto part_of = [&](uint64_t x) { return x < lo ? 0 : x > hi ? kBins - 1 : min(kBins - 1, (int)((x - lo) >> shift)); };
      auto count_in = [&](uint64_t word) {
        if (word >= w_lo && word <= w_hi) atomicAdd(&sh.bins[part_of(word)], (1ull << kCountShift) + units_of(word));
      };
      __syncthreads();
      if (tid < kBins) sh.bins[tid] = 0;
      if (tid == 0) {
        sh.pick[0] = kBins - 1;
        sh.pick[2] = 0;
      }
      __syncthreads();
      if (held) {
        for (int i = tid; i < n_held; i += kFinishThreads) count_in(sh.wide[i]);
        __syncthreads();
      } else {
        visit(first, end, [&](uint64_t word) {
          if (!fits) {
            count_in(word);
          } else if (word > w_hi) {
            atomicAdd(&sh.extra[slice_index(word)], (unsigned long long)units_of(word));
          } else if (word >= w_lo) {
            const int at = atomicAdd(&sh.pick[2], 1);
            if (at < kWide) sh.wide[at] = word;
          }
        });
        if (fits) {
          n_held = min(sh.pick[2], kWide);
          held = true;
          continue;
        }
      }
      const uint64_t mine = tid < kBins ? sh.bins[kBins - 1 - tid] : 0;  // from the top
      uint64_t all;
      const uint64_t before = block_scan(mine, &all, sh.tmpu);
      auto c_of = [&](uint64_t x) { return above + (x >> kCountShift); };
      auto w_of = [&](uint64_t x) { return above_w + (double)(x & kUnitMask) * eighths(sh.root, end); };
      if (tid < kBins) {
        const bool by_k = s.k > 0 && c_of(before) < (uint64_t)s.k && c_of(before + mine) >= (uint64_t)s.k;
        const bool by_p = !sum_k && w_of(before) < target && w_of(before + mine) >= target;
        const bool by_m = !sum_k && s.m > 0.f && sh.pick[1] == end && tid == kBins - 1 - part_of((uint64_t)float_order_key(least) << 32);
        if (by_k || by_p || by_m) atomicMin(&sh.pick[0], tid);
      }
      __syncthreads();
      const int at = sh.pick[0];
      if (tid == at) {
        sh.picku = before;
        sh.pickd = (double)(mine >> kCountShift);
      }
      __syncthreads();
      above = c_of(sh.picku);
      above_w = w_of(sh.picku);
      n_here = (uint64_t)sh.pickd;
      const int part = kBins - 1 - at;
      const uint64_t p_lo = lo + ((uint64_t)part << shift), p_hi = p_lo + (((uint64_t)1 << shift) - 1);
      if (part > 0) w_lo = max(w_lo, p_lo);
      if (part < kBins - 1) w_hi = p_hi < w_hi ? p_hi : w_hi;
      lo = max(w_lo, lo);
      hi = w_hi < hi ? w_hi : hi;
    }
    // (Eight passes reach a single word; a bin's tokens outside the edges' margin
    // above would not be narrowed.)
    if (!held || n_here > kList) return false;
    // Those of the range, one per thread in falling order (0 past their number).
    int m = n_held;
    if (n_held > kList) {
      __syncthreads();
      if (tid == 0) sh.pick[2] = 0;
      __syncthreads();
      for (int i = tid; i < n_held; i += kFinishThreads) {
        const uint64_t word = sh.wide[i];
        if (word > w_hi) {
          atomicAdd(&sh.extra[slice_index(word)], (unsigned long long)units_of(word));
        } else if (word >= w_lo) {
          const int at = atomicAdd(&sh.pick[2], 1);
          if (at < kList) sh.list[at] = word;
        }
      }
      __syncthreads();
      m = min(sh.pick[2], kList);
    }
    v = tid < m ? (n_held > kList ? sh.list : sh.wide)[tid] : 0;
    int size = 64;
    while (size < m) size *= 2;
    __syncthreads();
    v = sort_falling(v, size, sh.list);
    w = v ? weight(logit_of(v)) : 0.0;
    if (!sum_k) break;
    block_scan(above + tid < (uint64_t)s.k ? w : 0.0, &sum, sh.tmp);
    target = (double)s.p * (above_w + sum);
    if (whole) break;
  }
  bool keep = v != 0 && (s.k == 0 || above + tid < (uint64_t)s.k);
  const double before = above_w + block_scan(keep ? w : 0.0, &sum, sh.tmp);
  keep = keep && (before < target || (tid == 0 && above == 0)) && logit_of(v) >= least;
  const int n_kept = __syncthreads_count(keep);  // they come first
  if (tid == max(n_kept - 1, 0)) sh.pickd = n_kept ? before + w : above_w;
  __syncthreads();
  const double total = sh.pickd;
  const double at = u > 0.f ? (double)u * total : 0.0;

  if (whole) {
    // In order of index (the words turned round).
    int size = 64;
    while (size < n_kept) size *= 2;
    v = sort_falling(keep ? v << 32 | v >> 32 : 0, size, sh.list);
    w = v ? weight(float_of_key((uint32_t)v)) : 0.0;
    const double b0 = block_scan(w, &sum, sh.tmp);
    if (tid == pick_thread(b0, w, at, sh)) answer(a, n, (int)~(uint32_t)(v >> 32), w / total);
    return true;
  }

  // The slice by the kept weight of each, then the token.  If no token of the
  // last bin is kept, the words of those above it are larger than any of the bin's.
  sh.list[tid] = keep ? v : 0;
  if (tid == (n_kept ? n_kept - 1 : 0)) sh.picku = n_kept ? v : v + 1;
  __syncthreads();
  const Kept kept{sh.picku, least};
  for (int i = wave; i < n_slices; i += kFinishThreads / 64) {
    const SliceInfo& f = sh.info[i];
    const int off = top - f.top;
    double part = 0.0;
    if (f.max > -INFINITY) {
      for (int j = lane; j < end; j += 64)
        if (j - off >= 0 && j - off < f.n_bins) part += (double)(words_of(i)[j - off] & kUnitMask) * eighths(sh.root, j);
      if (lane == 0) part += (double)sh.extra[i] * eighths(sh.root, end);
      for (int j = lane; j < n_kept; j += 64)
        if (slice_index(sh.list[j]) == i) part += weight(logit_of(sh.list[j]));
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) part += __shfl_xor(part, d);
    if (lane == 0) sh.slice_w[i] = part;
  }
  __syncthreads();
  const double part = tid < n_slices ? sh.slice_w[tid] : 0.0;
  const double b0 = block_scan(part, &sum, sh.tmp);
  const int slice = pick_thread(b0, part, at, sh);
  if (tid == slice) sh.pickd = b0;
  __syncthreads();
  draw_slice<T, E>(a, n, row, slice, at - sh.pickd, total, kept, weight, sh);
  return true;
}

// A work-group per row, so a chain of dependent steps over some kilobytes bounds it:
// 14 us for 1 x 32000 with top-k, top-p and a temperature, 47 for 256 x 131072 bf16,
// where one work-group per CU waits for the rows whose last bin holds more tokens
// than a slice lists (their logits are read again, 24 MB in all).
template <typename T, int E>
__global__ __launch_bounds__(kFinishThreads) void sample_finish_kernel(SampleLaunch a, int n_slices) {
  __shared__ FinishShared sh;
  const int tid = threadIdx.x, n = blockIdx.x;
  const Settings s = settings_of(a, n);
  const T* row = reinterpret_cast<const T*>(a.logits) + (int64_t)n * a.stride;
  const char* in = static_cast<const char*>(a.ws) + (int64_t)n * n_slices * kSliceBytes;
  if (tid < n_slices) sh.info[tid] = *reinterpret_cast<const SliceInfo*>(in + tid * kSliceBytes);
  if (tid < 4) sh.pick[tid] = kBins;
  if (tid < 8) sh.root[tid] = root_of(tid);
  __syncthreads();
  float mx = -INFINITY;
  int top = -0x7FFFFFFF;
  bool beyond = false, left = false, unlisted = false;
  for (int i = 0; i < n_slices; ++i) {
    const SliceInfo& f = sh.info[i];
    mx = fmaxf(mx, f.max);
    left = left || f.left;
    unlisted = unlisted || f.n_list < 0;
    beyond = beyond || f.n_bins < 0;
    if (f.n_bins >= 0 && f.max > -INFINITY) top = max(top, f.top);
  }
  if (mx == -INFINITY) {
    if (tid == 0) answer(a, n, -1, 0.0);
    return;
  }
  if (s.k == 1) {
    if (tid == 0) {
      int i = 0;
      while (sh.info[i].max != mx) ++i;
      answer(a, n, sh.info[i].first, 1.0);
    }
    return;
  }
  for (int i = 0; i < n_slices; ++i)  // a slice's lower bins may lie below the row's
    left = left || (sh.info[i].max > -INFINITY && top - sh.info[i].top + sh.info[i].n_bins > kBins);
  const float least = least_of(s, mx);
  if (!beyond && finish_bins<T, E>(a, n, n_slices, s, row, in, mx, least, top, left, unlisted, sh)) return;
  finish_any(a, n, s, row, mx, least, sh);
}

}  // namespace

size_t sample_workspace(int N, int V) { return (size_t)N * ((V + slice_of(V) - 1) / slice_of(V)) * kSliceBytes; }

hipError_t launch_sample(const SampleLaunch& a, int dtype, hipStream_t stream) {
  const int slice = slice_of(a.V), n_slices = (a.V + slice - 1) / slice;
  auto run = [&](auto slices, auto finish) {
    slices<<<dim3((unsigned)n_slices, (unsigned)a.N), kSliceThreads, 0, stream>>>(a, n_slices);
    if (hipError_t e = hipGetLastError()) return e;
    finish<<<a.N, kFinishThreads, 0, stream>>>(a, n_slices);
    return hipGetLastError();
  };
  static_assert(kFinishThreads == 2 * kSliceThreads, "a slice in the finish");
  const bool large = slice > kMinSlice;
  if (dtype == NACL_F32)
    return large ? run(sample_slices_kernel<float, 4>, sample_finish_kernel<float, 2>)
                 : run(sample_slices_kernel<float, 2>, sample_finish_kernel<float, 1>);
  return large ? run(sample_slices_kernel<__bf16, 4>, sample_finish_kernel<__bf16, 2>)
               : run(sample_slices_kernel<__bf16, 2>, sample_finish_kernel<__bf16, 1>);
}

}  // namespace nacl
