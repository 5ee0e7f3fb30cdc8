// The best continuations of every group's beams (nacl_beam_select).
//
//   value(w, v) = score_w + x_wv - ln sum_v exp x_wv
//
// Within a beam the order of the values is that of the logits, so a work-group
// reads a slice of a row once: its maximum, the sum of its exponentials and its K
// largest logits, in order.  A second launch, a work-group per group, joins the
// slices' sums to the rows' normalisers and picks the K best of the lists.
//
// The K largest of n numbers are found by a threshold: the K-th largest of some
// of them (of the threads' maxima, of the lists' heads) is no larger than the
// K-th largest of all, and few pass it.  Keys are unsigned with the numbers' order,
// 0 for nothing.
//
// 32 groups of 8 beams, 131072 tokens each (67 MB of bf16), 16 wanted: slices 16.4 us (4.1
// TB/s; vector and scalar instructions bound them, some 300 and 150 a wave), finish 6.5 us
// (slices of 4096 tokens 21.6 + 8.2); 64 wanted: 22.5 + 10.2; 4 beams of 32000 tokens 4.4 + 4.3
// us, one chain of loads and barriers each.

#include <type_traits>

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxK = 64;
// Keys that may reach a bound before it is looked for more closely: each costs a
// place in a list, each round of the search some 100 cycles.
__host__ __device__ constexpr int most_of(int K) { return K + K / 4 + 2; }

__device__ __forceinline__ float of_order_key(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}
__device__ __forceinline__ uint64_t order_key(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return (b >> 63) ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double of_order_key(uint64_t k) {
  return __builtin_bit_cast(double, (k >> 63) ? k & ~(1ull << 63) : ~k);
}

// x of the lane N further in its row of 16, cyclically.
template <int N>
__device__ __forceinline__ double row_turn(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, 0x120 + N, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), 0x120 + N, 0xF, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// The wave's maximum and sum in lane 63, by row shifts and broadcasts.
template <int CTRL, int ROWS>
__device__ __forceinline__ float shifted(float x, float none) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), CTRL, ROWS, 0xF, false));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double shifted(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ float last_max(float x) {
  x = fmaxf(x, shifted<0x111, 0xF>(x, -INFINITY));
  x = fmaxf(x, shifted<0x112, 0xF>(x, -INFINITY));
  x = fmaxf(x, shifted<0x114, 0xF>(x, -INFINITY));
  x = fmaxf(x, shifted<0x118, 0xF>(x, -INFINITY));
  x = fmaxf(x, shifted<0x142, 0xA>(x, -INFINITY));
  return fmaxf(x, shifted<0x143, 0xC>(x, -INFINITY));
}
__device__ __forceinline__ double last_sum(double x) {
  x += shifted<0x111, 0xF>(x);
  x += shifted<0x112, 0xF>(x);
  x += shifted<0x114, 0xF>(x);
  x += shifted<0x118, 0xF>(x);
  x += shifted<0x142, 0xA>(x);
  return x + shifted<0x143, 0xC>(x);
}

// A bound that at least `want` of the wave's keys (N per lane) reach and at most
// `most` of them, unless more are equal to it; 1 where fewer than `want` are not 0.
// It is looked for downwards from the largest key, top, in steps that grow from
// `step`, then between the last two: a handful of rounds where the step is of the
// size of the keys' distances, twice the key's bits at most.  `reach`: how many keys
// reach it.  Every wave with the same keys gets the same bound.
template <int N, typename K>
__device__ __forceinline__ K bound_of(const K (&key)[N], K top, K step, int want, int most, int& reach) {
  if (top == 0) {
    reach = 0;
    return 1;
  }
  K lo = 0, hi = 0, d = min(step, (K)(top - 1));  // distances: too few keys are nearer than lo
  for (;;) {
    reach = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) reach += (int)__popcll(__ballot(key[i] >= top - d));
    if (reach >= want) {
      if (reach <= most || d == lo) break;
      hi = d;
      d = lo + (d - lo) / 2;
    } else {
      if (d == top - 1) break;
      lo = d + 1;
      d = hi ? lo + (hi - lo) / 2 : d > (top - 1) / 4 ? top - 1 : 4 * d + 3;
    }
  }
  return top - d;
}

// ---------------------------------------------------------------------------
// Slices.  A thread takes kPer tokens as pieces of 16 bytes, at any alignment of the
// row, so that a row's result depends on its logits alone (equal beams tie).

template <typename T>
struct Piece;
template <>
struct Piece<__bf16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void load(const __bf16* p, float (&x)[8]) {
    typedef uint32_t words __attribute__((ext_vector_type(4), aligned(2)));
    const words w = *reinterpret_cast<const words*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};
template <>
struct Piece<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void load(const float* p, float (&x)[4]) {
    typedef float words __attribute__((ext_vector_type(4), aligned(4)));
    const words w = *reinterpret_cast<const words*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = w[i];
  }
};

constexpr uint32_t kLeast = 0x00800000u;  // key of the lowest finite number
constexpr float kLog2e = 1.44269504f;

// kPer tokens per thread, a.K at most kTop (so that eight work-groups fit a CU where
// few are looked for).
template <typename T, int kPer, int kTop>
__global__ __launch_bounds__(kThreads, kTop < kMaxK ? 8 : 6) void beam_slices_kernel(BeamLaunch a) {
  using P = Piece<T>;
  constexpr int kPieces = kPer / P::kN, kSlice = kPer * kThreads;
  // Threads whose maxima reach the bound, their logits, and those of them that reach it.
  __shared__ int chosen[most_of(kTop)];
  __shared__ f32x4 held[most_of(kTop) * kPer / 4];
  __shared__ uint16_t places[most_of(kTop) * kPer];  // in held
  __shared__ uint64_t list[kThreads];
  __shared__ uint32_t maxima[kThreads];
  __shared__ uint32_t bounds[2];
  __shared__ float wave_max[kThreads / 64];
  __shared__ double wave_sum[kThreads / 64];
  __shared__ int n_chosen, found, n_reach;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.y, slice = blockIdx.x;
  if (a.ended && a.ended[row]) return;  // its one continuation needs no logits
  const T* x0 = reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.stride;
  const int first = slice * kSlice;
  auto token = [&](int u, int i) { return first + (u * kThreads + tid) * P::kN + i; };

  float x[kPieces][P::kN];
  if (first + kSlice <= a.V) {
#pragma unroll
    for (int u = 0; u < kPieces; ++u) P::load(x0 + token(u, 0), x[u]);
  } else {
    // What lies past the row's end is -infinity.  A piece of which that is a part is
    // loaded by elements, after the whole ones are under way together (in the place
    // of the others, the row's first).
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
      if (a.V >= P::kN) P::load(x0 + (token(u, 0) + P::kN <= a.V ? token(u, 0) : 0), x[u]);
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
      if (token(u, 0) + P::kN <= a.V) continue;
#pragma unroll
      for (int i = 0; i < P::kN; ++i) x[u][i] = -INFINITY;
      if (token(u, 0) >= a.V) continue;
#pragma unroll
      for (int i = 0; i < P::kN; ++i)
        if (token(u, i) < a.V) x[u][i] = (float)x0[token(u, i)];
    }
  }
  if (tid == 0) found = n_chosen = 0;

  // The thread's maximum and its exponentials' sum against it, of kPer terms in
  // fp32, as powers of two of x log2(e) - c with c = m log2(e) rounded, from which the
  // sum is freed afterwards (c's own rounding, in front of all terms alike).
  float m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int u = 0; u < kPieces; ++u)
#pragma unroll
    for (int i = 0; i < P::kN; i += 2) asm("v_max3_f32 %0, %0, %1, %2" : "+v"(m) : "v"(x[u][i]), "v"(x[u][i + 1]));
  const float c = m * kLog2e;
#pragma unroll
  for (int u = 0; u < kPieces; ++u)
#pragma unroll
    for (int i = 0; i < P::kN; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[u][i], kLog2e, -c));
  sum *= __builtin_amdgcn_exp2f(-__builtin_fmaf(m, kLog2e, -c));
  if (!(sum == sum && __builtin_fabsf(m) < 0x1p20f)) {
    // A NaN among the logits, no finite maximum, or one next to which c's rounding
    // is not small.  A NaN counts as -infinity; infinite logits share a row, one
    // each, and the others are nothing beside them.
    m = -INFINITY;
    sum = 0.f;
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
      for (int i = 0; i < P::kN; ++i) m = x[u][i] > m ? x[u][i] : m;
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
      for (int i = 0; i < P::kN; ++i) {
        const float e = x[u][i] == m ? 1.f : __builtin_amdgcn_exp2f((x[u][i] - m) * kLog2e);
        sum += m > -INFINITY && x[u][i] == x[u][i] ? e : 0.f;
      }
  }
  const uint32_t mine = m == -INFINITY ? 0 : float_order_key(m + 0.f);  // (-0 is 0)
  maxima[tid] = mine;
  const float wm = last_max(m);
  if (lane == 63) wave_max[wave] = wm;
  __syncthreads();
  float top = wave_max[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) top = fmaxf(top, wave_max[i]);
  // The sums are joined in fp64.
  const double s = last_sum((double)(m == top ? sum : sum * __builtin_amdgcn_exp2f((m - top) * kLog2e)));
  if (lane == 63) wave_sum[wave] = s;

  // The bound of the threads' maxima, by one wave, as the others' instructions count
  // too; logits of a language model are a few units apart there, 2^20 steps each.
  const int most = most_of(a.K);
  uint32_t key[kThreads / 64];
  if (wave == 0) {
    int reach;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) key[i] = maxima[lane + 64 * i];
    const uint32_t x = bound_of(key, top == -INFINITY ? 0 : float_order_key(top + 0.f), 1u << 20, a.K, most, reach);
    if (lane == 0) {
      bounds[0] = x;
      n_reach = reach;
    }
  }
  __syncthreads();
  const uint32_t bound = bounds[0];
  uint32_t tie = 0;  // of the logits equal to the bound, those whose ~token reaches it
  const int64_t slot = (int64_t)row * a.S + slice;
  if (tid == 0) {
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) t += wave_sum[i];
    a.sums[2 * slot] = (double)top;
    a.sums[2 * slot + 1] = t;
  }
  bool take = mine >= bound;
  if (n_reach > most) {
    // Equal maxima: the threads with the first tokens among them count.
    uint32_t k = mine > bound ? ~0u : 0;
    if (mine == bound) {
#pragma unroll
      for (int u = kPieces - 1; u >= 0; --u)
#pragma unroll
        for (int i = P::kN - 1; i >= 0; --i)
          if (x[u][i] == m) k = ~(uint32_t)token(u, i);
    }
    maxima[tid] = k;
    __syncthreads();
    if (wave == 0) {
      int reach;
#pragma unroll
      for (int i = 0; i < kThreads / 64; ++i) key[i] = maxima[lane + 64 * i];
      const uint32_t x = bound_of(key, ~0u, 1u << 12, a.K, a.K, reach);
      if (lane == 0) bounds[1] = x;
    }
    __syncthreads();
    tie = bounds[1];
    take = k >= tie;
  }
  // Their logits to all threads, which look for those that reach it.
  if (take) {
    const int at = atomicAdd(&n_chosen, 1);
    chosen[at] = tid;
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
      for (int i = 0; i < P::kN; i += 4)
        held[(at * kPer + u * P::kN + i) / 4] = f32x4{x[u][i], x[u][i + 1], x[u][i + 2], x[u][i + 3]};
  }
  __syncthreads();
  // Logit i of held, as its key and ~token.
  auto entry = [&](int i) {
    const int e = i % kPer, at = first + (e / P::kN * kThreads + chosen[i / kPer]) * P::kN + e % P::kN;
    return (uint64_t)float_order_key(reinterpret_cast<const float*>(held)[i] + 0.f) << 32 | ~(uint32_t)at;
  };
  const float least = of_order_key(max(bound, kLeast));
  for (int i = tid; i < n_chosen * kPer; i += kThreads) {
    const float v = reinterpret_cast<const float*>(held)[i];
    if (v > least || (v == least && (uint32_t)entry(i) >= tie)) places[atomicAdd(&found, 1)] = (uint16_t)i;
  }
  __syncthreads();
  const int n = found;
  uint64_t* out = a.keys + slot * a.K;
  if (n <= kThreads) {
    const uint64_t k = tid < n ? entry(places[tid]) : 0;
    list[tid] = k;
    __syncthreads();
    if (tid < n) {
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += list[j] > k;
      if (rank < a.K) out[rank] = k;
    }
  } else {  // few threads hold most of the largest
    for (int i = tid; i < n; i += kThreads) {
      const uint64_t k = entry(places[i]);
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += entry(places[j]) > k;
      if (rank < a.K) out[rank] = k;
    }
  }
  for (int i = n + tid; i < a.K; i += kThreads) out[i] = 0;
}

// ---------------------------------------------------------------------------
// A group's lists: list l holds the K largest logits of slice l mod S of beam l / S.

enum Mode { kNone, kLogits, kInfinite, kEnded };

constexpr int kHeads = kBeamLists / kThreads;  // of a thread, at most
constexpr int kGroup = 16;                     // lanes per beam

// Where a continuation comes from, larger for those that come first among equal values: by
// beam, within it by logit, then by token.  (A beam's values may be equal where its
// logits are not: next to a large score their differences are lost in fp64.)  Bits 52 ..
// 57 hold the beam, 20 .. 51 the logit's key, the others the token.
constexpr uint64_t kPlace = 1ull << 58;        // of every continuation: 0 is none
__device__ __forceinline__ uint64_t place_of(int w, uint32_t logit, uint32_t inverse_token) {
  return kPlace | (uint64_t)(kMaxK - 1 - w) << 52 | (uint64_t)logit << 20 | (inverse_token & 0xFFFFFu);
}
__device__ __forceinline__ int beam_at(uint64_t place) { return kMaxK - 1 - (int)(place >> 52 & (kMaxK - 1)); }
__device__ __forceinline__ int token_at(uint64_t place) { return (int)(~(uint32_t)place & 0xFFFFFu); }

__global__ __launch_bounds__(kThreads) void beam_finish_kernel(BeamLaunch a) {
  // A logit's value is (x - tops) + shift (kEnded, kInfinite: shift): a difference
  // that is exact next to a top of any size, then numbers of the values' size.
  __shared__ double tops[kMaxK], shift[kMaxK];
  __shared__ int mode[kMaxK];
  // What reaches the bound, its values and their places; before that, the lists' first ones.
  __shared__ uint64_t list[kMaxK * kMaxK], list_at[kMaxK * kMaxK];
  uint64_t* head = list;
  uint64_t* head_at = list_at;
  __shared__ uint64_t best;
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63;
  const int group = blockIdx.x;
  if (tid == 0) {
    best = 0;
    found = 0;
  }
  __syncthreads();
  const int lists = a.W * a.S;
  const uint64_t* keys = a.keys + (int64_t)group * lists * a.K;

  // The lists' first `kept` entries, on their way while the normalisers are made.
  // The bound is looked for among the first R of a list, about four times as many as
  // are wanted, so that it is near theirs.
  const int enough = max(1, (4 * a.K + lists - 1) / lists);
  const int kept = min(min(a.K, kBeamLists / lists), max(4, 4 * enough)), n_kept = lists * kept;
  const int R = min(kept, enough), heads = lists * R;
  uint64_t raw[kHeads];
#pragma unroll
  for (int c = 0; c < kHeads; ++c) {
    const int i = tid + c * kThreads;
    raw[c] = i < n_kept ? keys[(int64_t)(i / kept) * a.K + i % kept] : 0;
  }

  // The beams' normalisers, kGroup lanes per beam.
  for (int w0 = 0; w0 < a.W; w0 += kThreads / kGroup) {
    const int w = w0 + tid / kGroup, sub = tid % kGroup;
    const int64_t row = (int64_t)group * a.W + w;
    const bool there = w < a.W;
    double top = -INFINITY, sum = 0.0, score = 0.0;
    bool ended = false;
    if (there) {
      // (Of a beam that has ended, whatever the sums hold is not used.)
      const double2* sums = reinterpret_cast<const double2*>(a.sums) + row * a.S;
      double2 next = sub < a.S ? sums[sub] : double2{-INFINITY, 0.0};
      score = (double)a.scores[row];
      ended = a.ended && a.ended[row];
      for (int s = sub; s < a.S; s += kGroup) {
        const double2 x = next;  // maximum, sum
        if (s + kGroup < a.S) next = sums[s + kGroup];
        if (x.x == top) {
          sum += x.x == -INFINITY ? 0.0 : x.y;
        } else if (x.x > top) {
          sum = x.y + (x.x == INFINITY ? 0.0 : sum * exp(top - x.x));
          top = x.x;
        } else if (top != INFINITY) {
          sum += x.y * exp(x.x - top);
        }
      }
    }
    double all = top;
    all = fmax(all, row_turn<8>(all));
    all = fmax(all, row_turn<4>(all));
    all = fmax(all, row_turn<2>(all));
    all = fmax(all, row_turn<1>(all));
    if (top != all) sum = all == INFINITY ? 0.0 : sum * exp(top - all);
    sum += row_turn<8>(sum);
    sum += row_turn<4>(sum);
    sum += row_turn<2>(sum);
    sum += row_turn<1>(sum);
    if (there && sub == 0) {
      const bool finite = fabs(score) < INFINITY;
      mode[w] = !finite || (!ended && all == -INFINITY) ? kNone : ended ? kEnded : all == INFINITY ? kInfinite : kLogits;
      tops[w] = all;
      shift[w] = (ended ? score : score - log(sum)) + 0.0;  // (-0 is 0)
      // The beam's best value: that of its largest logit.
      if (mode[w] != kNone) atomicMax((unsigned long long*)&best, (unsigned long long)order_key(shift[w]));
    }
  }
  __syncthreads();

  // Entry r of list l, whose key is k: its value and its place, beam and token.
  auto entry = [&](int l, int r, uint64_t k, uint64_t& at) -> uint64_t {
    const int w = l / a.S, kind = mode[w];
    if (kind == kNone) return 0;
    at = place_of(w, 0, ~(uint32_t)a.end_token);
    if (kind == kEnded) return l == w * a.S && r == 0 ? order_key(shift[w]) : 0;
    if (!k) return 0;
    at = place_of(w, (uint32_t)(k >> 32), (uint32_t)k);
    const float x = of_order_key((uint32_t)(k >> 32));
    if (kind == kInfinite) return x == INFINITY ? order_key(shift[w]) : 0;
    return order_key(((double)x - tops[w]) + shift[w]);
  };
  uint64_t mine[kHeads], mine_at[kHeads];
#pragma unroll
  for (int c = 0; c < kHeads; ++c) {
    const int i = tid + c * kThreads;
    mine[c] = mine_at[c] = 0;
    if (i >= n_kept) break;
    mine[c] = entry(i / kept, i % kept, raw[c], mine_at[c]);
    head[i] = mine[c];
    head_at[i] = mine_at[c];
  }
  __syncthreads();
  const uint64_t top = best;

  // The bound of the heads (of equal values the largest places).  Values are a few
  // units apart, 2^48 steps each.  (The list holds what follows `most` heads.)
  uint64_t bound = 1;
  uint64_t tie = 0;
  const int most = R > 1 || most_of(a.K) * a.K <= kMaxK * kMaxK ? most_of(a.K) : a.K;
  auto search = [&](auto n_c) {
    constexpr int N = decltype(n_c)::value;
    uint64_t k[N], at[N];
    int reach;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = 64 * i + lane, from = x / R * kept + x % R;
      k[i] = x < heads ? head[from] : 0;
      at[i] = x < heads ? head_at[from] : 0;
    }
    bound = bound_of(k, top, (uint64_t)1 << 48, a.K, most, reach);
    if (reach > most) {
      uint64_t t[N];
#pragma unroll
      for (int i = 0; i < N; ++i) t[i] = k[i] > bound ? 2 * kPlace - 1 : k[i] == bound ? at[i] : 0;
      tie = bound_of(t, 2 * kPlace - 1, (uint64_t)1 << 52, a.K, a.K, reach);
    }
  };
  if (heads <= 64) search(std::integral_constant<int, 1>{});
  else if (heads <= kThreads) search(std::integral_constant<int, kThreads / 64>{});
  else search(std::integral_constant<int, kBeamLists / 64>{});

  // What reaches it, and of the lists whose entries here all do, what follows.
  __syncthreads();
  auto reaches = [&](uint64_t v, uint64_t at) { return v > bound || (v == bound && at >= tie); };
  auto add = [&](uint64_t v, uint64_t at) {
    const int i = atomicAdd(&found, 1);
    list[i] = v;
    list_at[i] = at;
  };
#pragma unroll
  for (int c = 0; c < kHeads; ++c) {
    const int i = tid + c * kThreads;
    if (i >= n_kept) break;
    if (!reaches(mine[c], mine_at[c])) continue;
    add(mine[c], mine_at[c]);
    if (i % kept != kept - 1) continue;
    for (int r = kept; r < a.K; ++r) {
      uint64_t at = 0;
      const uint64_t v = entry(i / kept, r, keys[(int64_t)(i / kept) * a.K + r], at);
      if (!reaches(v, at)) break;
      add(v, at);
    }
  }
  __syncthreads();
  // Eight lanes rank one of them.
  const int n = found;
  for (int i = tid / 8; i < n; i += kThreads / 8) {
    const uint64_t v = list[i], at = list_at[i];
    int rank = 0;
#pragma unroll 4
    for (int j = tid % 8; j < n; j += 8) {
      const uint64_t v2 = list[j], at2 = list_at[j];
      rank += (int)((v2 > v) | ((v2 == v) & (at2 > at)));
    }
#pragma unroll
    for (int x = 1; x < 8; x *= 2) rank += __shfl_xor(rank, x);
    if (rank < a.K && tid % 8 == 0) {
      const int64_t to = (int64_t)group * a.K + rank;
      a.parents[to] = beam_at(at);
      a.tokens[to] = token_at(at);
      a.out[to] = (float)of_order_key(v);
    }
  }
  for (int i = n + tid; i < a.K; i += kThreads) {
    const int64_t to = (int64_t)group * a.K + i;
    a.parents[to] = a.tokens[to] = -1;
    a.out[to] = -INFINITY;
  }
}

}  // namespace

hipError_t launch_beam(const BeamLaunch& a, int dtype, hipStream_t stream) {
  const dim3 grid((unsigned)a.S, (unsigned)(a.B * a.W));
  auto run = [&](auto kernel) { kernel<<<grid, kThreads, 0, stream>>>(a); };
  constexpr int kSmall = kBeamSmallSlice / kThreads, kLarge = kBeamSlice / kThreads, kFew = 16;
  if (a.slice == kBeamSmallSlice) {
    if (dtype == NACL_F32) run(beam_slices_kernel<float, kSmall, kMaxK>);
    else run(beam_slices_kernel<__bf16, kSmall, kMaxK>);
  } else if (a.K <= kFew) {
    if (dtype == NACL_F32) run(beam_slices_kernel<float, kLarge, kFew>);
    else run(beam_slices_kernel<__bf16, kLarge, kFew>);
  } else {
    if (dtype == NACL_F32) run(beam_slices_kernel<float, kLarge, kMaxK>);
    else run(beam_slices_kernel<__bf16, kLarge, kMaxK>);
  }
  if (hipError_t e = hipGetLastError()) return e;
  beam_finish_kernel<<<a.B, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace nacl
