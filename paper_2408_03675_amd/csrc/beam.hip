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

#include <type_traits>

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = kBeamSlice / kThreads;  // tokens per thread of a slice
constexpr int kMaxK = 64;

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

// A bound that at least `want` of the wave's keys (N per lane) reach, at most
// `most` of them unless more are equal; 1 where fewer than `want` are not 0.
// Every wave that calls it with the same keys gets the same bound.
template <int N, typename K>
__device__ __forceinline__ K bound_of(const K (&key)[N], int want, int most) {
  K bound = 0;
  for (int bit = 8 * (int)sizeof(K) - 1; bit >= 0; --bit) {
    const K trial = bound | (K)1 << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += (int)__popcll(__ballot(key[i] >= trial));
    if (n >= want) {
      bound = trial;
      if (n <= most) break;
    }
  }
  return bound ? bound : 1;
}
template <int N, typename K>
__device__ __forceinline__ int count_of(const K (&key)[N], K bound) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) n += (int)__popcll(__ballot(key[i] >= bound));
  return n;
}

// ---------------------------------------------------------------------------
// Slices.  A thread takes kPer tokens as 16-byte pieces; the piece's place is its
// address's, so that rows of any alignment are read by aligned loads (the row's
// first and last pieces by elements).

template <typename T>
struct Piece;
template <>
struct Piece<__bf16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void load(const __bf16* p, float (&x)[8]) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
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
    const f32x4 w = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = w[i];
  }
};

constexpr uint32_t kLeast = 0x00800000u;  // key of the lowest finite number

template <typename T>
__global__ __launch_bounds__(kThreads) void beam_slices_kernel(BeamLaunch a) {
  using P = Piece<T>;
  constexpr int kPieces = kPer / P::kN;
  // Logits that reach the bound: at most K threads hold them.
  __shared__ uint64_t list[kMaxK * kPer];
  __shared__ uint32_t maxima[kThreads];
  __shared__ float wave_max[kThreads / 64];
  __shared__ double wave_sum[kThreads / 64];
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.y, slice = blockIdx.x;
  if (a.ended && a.ended[row]) return;  // its one continuation needs no logits
  const T* x0 = reinterpret_cast<const T*>(a.logits) + (int64_t)row * a.stride;
  const int head = (int)(((uintptr_t)x0 & 15) / sizeof(T));  // tokens by which the pieces start before the row
  const int first = slice * kBeamSlice - head;

  // NaN and what lies outside the row are -infinity, -0 is 0.
  float x[kPieces][P::kN];
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    const int at = first + (u * kThreads + tid) * P::kN;
    if (at >= 0 && at + P::kN <= a.V) {
      P::load(x0 + at, x[u]);
    } else {
#pragma unroll
      for (int i = 0; i < P::kN; ++i) x[u][i] = (uint32_t)(at + i) < (uint32_t)a.V ? (float)x0[at + i] : -INFINITY;
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int u = 0; u < kPieces; ++u)
#pragma unroll
    for (int i = 0; i < P::kN; ++i) {
      x[u][i] = x[u][i] == x[u][i] ? x[u][i] + 0.f : -INFINITY;
      m = fmaxf(m, x[u][i]);
    }
  if (tid == 0) found = 0;
  maxima[tid] = m == -INFINITY ? 0 : float_order_key(m);

  // The slice's maximum and its exponentials' sum against it, each thread's sum
  // of kPer in fp32 against its own maximum, those in fp64.  Infinite logits share
  // a row, so they count as one each and the others as nothing.
  float sum = 0.f;
#pragma unroll
  for (int u = 0; u < kPieces; ++u)
#pragma unroll
    for (int i = 0; i < P::kN; ++i)
      sum += m == INFINITY ? (x[u][i] == INFINITY ? 1.f : 0.f)
                           : __builtin_amdgcn_exp2f((x[u][i] - (m == -INFINITY ? 0.f : m)) * 1.44269504f);
  float wm = m;
#pragma unroll
  for (int i = 1; i < 64; i *= 2) wm = fmaxf(wm, __shfl_xor(wm, i));
  if (lane == 0) wave_max[wave] = wm;
  __syncthreads();
  float top = wave_max[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) top = fmaxf(top, wave_max[i]);
  double s = m == top ? (double)sum : (double)sum * __builtin_amdgcn_exp2f((m - top) * 1.44269504f);
  if (top == -INFINITY) s = 0.0;
#pragma unroll
  for (int i = 1; i < 64; i *= 2) s += __shfl_xor(s, i);
  if (lane == 0) wave_sum[wave] = s;

  // The bound: the K-th largest of the threads' maxima or a little less.  Where
  // more threads reach it, equal maxima do, and those with the first tokens count.
  uint32_t key[kThreads / 64];
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) key[i] = maxima[lane + 64 * i];
  const uint32_t bound = bound_of(key, a.K, a.K);
  uint32_t tie = 0;  // of the logits equal to the bound, those whose ~token reaches it
  const int reach = count_of(key, bound);
  __syncthreads();  // the maxima are read
  const int64_t slot = (int64_t)row * a.S + slice;
  if (tid == 0) {
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) t += wave_sum[i];
    a.sums[2 * slot] = (double)top;
    a.sums[2 * slot + 1] = t;
  }
  const uint32_t mine = m == -INFINITY ? 0 : float_order_key(m);
  if (reach > a.K) {
    uint32_t k = mine > bound ? ~0u : 0;
    if (mine == bound) {
#pragma unroll
      for (int u = kPieces - 1; u >= 0; --u)
#pragma unroll
        for (int i = P::kN - 1; i >= 0; --i)
          if (x[u][i] == m) k = ~(uint32_t)(first + (u * kThreads + tid) * P::kN + i);
    }
    maxima[tid] = k;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) key[i] = maxima[lane + 64 * i];
    tie = bound_of(key, a.K, a.K);
  }
  if (mine >= bound) {
#pragma unroll
    for (int u = 0; u < kPieces; ++u)
#pragma unroll
      for (int i = 0; i < P::kN; ++i) {
        const uint32_t k = float_order_key(x[u][i]), t = ~(uint32_t)(first + (u * kThreads + tid) * P::kN + i);
        if (k >= kLeast && (k > bound || (k == bound && t >= tie))) list[atomicAdd(&found, 1)] = (uint64_t)k << 32 | t;
      }
  }
  __syncthreads();
  const int n = found;
  uint64_t* out = a.keys + slot * a.K;
  for (int i = tid; i < n; i += kThreads) {
    const uint64_t k = list[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += list[j] > k;
    if (rank < a.K) out[rank] = k;
  }
  for (int i = n + tid; i < a.K; i += kThreads) out[i] = 0;
}

// ---------------------------------------------------------------------------
// A group's lists: list l holds the K largest logits of slice l mod S of beam l / S.

enum Mode { kNone, kLogits, kInfinite, kEnded };

__global__ __launch_bounds__(kThreads) void beam_finish_kernel(BeamLaunch a) {
  // A logit's value is (x - tops) + shift (kEnded, kInfinite: shift): a difference
  // that is exact next to a top of any size, then numbers of the values' size.
  __shared__ double tops[kMaxK], shift[kMaxK];
  __shared__ int mode[kMaxK];
  __shared__ uint64_t head[kBeamLists];  // the lists' first values
  __shared__ uint32_t head_at[kBeamLists];
  __shared__ uint64_t list[kMaxK * kMaxK];
  __shared__ uint32_t list_at[kMaxK * kMaxK];
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int group = blockIdx.x;

  // The beams' normalisers, a wave per beam.
  for (int w = wave; w < a.W; w += kThreads / 64) {
    const int64_t row = (int64_t)group * a.W + w;
    const double score = (double)a.scores[row];
    const bool ended = a.ended && a.ended[row];
    double top = -INFINITY, sum = 0.0;
    if (!ended) {
      const double* sums = a.sums + 2 * row * a.S;
      for (int s = lane; s < a.S; s += 64) top = fmax(top, sums[2 * s]);
#pragma unroll
      for (int i = 1; i < 64; i *= 2) top = fmax(top, __shfl_xor(top, i));
      for (int s = lane; s < a.S; s += 64) {
        const double m = sums[2 * s];
        if (m == top) sum += sums[2 * s + 1];
        else if (m != -INFINITY && top != INFINITY) sum += sums[2 * s + 1] * exp(m - top);
      }
#pragma unroll
      for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i);
    }
    if (lane == 0) {
      const bool finite = fabs(score) < INFINITY;
      mode[w] = !finite || (!ended && top == -INFINITY) ? kNone : ended ? kEnded : top == INFINITY ? kInfinite : kLogits;
      tops[w] = top;
      shift[w] = ended ? score : score - log(sum);
    }
  }
  if (tid == 0) found = 0;
  __syncthreads();

  const int lists = a.W * a.S;
  const uint64_t* keys = a.keys + (int64_t)group * lists * a.K;
  // Entry r of list l: its value and its place, beam and token.
  auto entry = [&](int l, int r, uint32_t& at) -> uint64_t {
    const int w = l / a.S, kind = mode[w];
    if (kind == kNone) return 0;
    at = (uint32_t)w << 20 | (uint32_t)a.end_token;
    if (kind == kEnded) return l == w * a.S && r == 0 ? order_key(shift[w]) : 0;
    const uint64_t k = keys[(int64_t)l * a.K + r];
    if (!k) return 0;
    at = (uint32_t)w << 20 | ~(uint32_t)k;
    const float x = of_order_key((uint32_t)(k >> 32));
    if (kind == kInfinite) return x == INFINITY ? order_key(shift[w]) : 0;
    return order_key(((double)x - tops[w]) + shift[w]);
  };
  // The lists' first R entries, and the bound that K of them reach (of equal
  // values the first places).
  const int R = min(a.K, kBeamLists / lists), heads = lists * R;
  for (int i = tid; i < kBeamLists; i += kThreads) {
    uint32_t at = 0;
    head[i] = i < heads ? entry(i / R, i % R, at) : 0;
    head_at[i] = at;
  }
  __syncthreads();
  uint64_t bound = 1;
  uint32_t tie = 0;
  auto search = [&](auto n_c) {
    constexpr int N = decltype(n_c)::value;
    uint64_t k[N];
#pragma unroll
    for (int i = 0; i < N; ++i) k[i] = head[64 * i + lane];
    bound = bound_of(k, a.K, a.K);
    if (count_of(k, bound) > a.K) {
      uint32_t t[N];
#pragma unroll
      for (int i = 0; i < N; ++i) t[i] = k[i] > bound ? ~0u : k[i] == bound ? ~head_at[64 * i + lane] : 0;
      tie = bound_of(t, a.K, a.K);
    }
  };
  if (heads <= 64) search(std::integral_constant<int, 1>{});
  else if (heads <= 256) search(std::integral_constant<int, 4>{});
  else search(std::integral_constant<int, 16>{});

  // What reaches it: K of the heads at most, and of their lists what follows.
  auto reaches = [&](uint64_t v, uint32_t at) { return v > bound || (v == bound && ~at >= tie); };
  auto add = [&](uint64_t v, uint32_t at) {
    const int i = atomicAdd(&found, 1);
    list[i] = v;
    list_at[i] = at;
  };
  for (int i = tid; i < heads; i += kThreads) {
    if (!reaches(head[i], head_at[i])) continue;
    add(head[i], head_at[i]);
    if (i % R != R - 1) continue;
    for (int r = R; r < a.K; ++r) {
      uint32_t at = 0;
      const uint64_t v = entry(i / R, r, at);
      if (!reaches(v, at)) break;
      add(v, at);
    }
  }
  __syncthreads();
  const int n = found;
  for (int i = tid; i < n; i += kThreads) {
    const uint64_t v = list[i];
    const uint32_t at = list_at[i];
    int rank = 0;
    for (int j = 0; j < n; ++j) rank += list[j] > v || (list[j] == v && list_at[j] < at);
    if (rank < a.K) {
      const int64_t to = (int64_t)group * a.K + rank;
      a.parents[to] = (int)(at >> 20);
      a.tokens[to] = (int)(at & 0xFFFFFu);
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
  if (dtype == NACL_F32) beam_slices_kernel<float><<<grid, kThreads, 0, stream>>>(a);
  else beam_slices_kernel<__bf16><<<grid, kThreads, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError()) return e;
  beam_finish_kernel<<<a.B, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace nacl
