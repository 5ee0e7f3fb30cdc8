// The next token of each row of logits by temperature, top-k, top-p and min-p
// (nacl_sample).

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

constexpr int kSampleThreads = 1024;

template <typename T>
__device__ __forceinline__ float logit(const T* p, int64_t i) {
  const float x = (float)p[i];
  return x != x ? -INFINITY : x + 0.f;  // -0 counts as 0
}

// A row's weights: exp((x - max) / temperature) and in units of 2^-43.
struct Weight {
  float max, scale;  // scale: log2(e) / temperature
  __device__ __forceinline__ float of(float x) const {
    if (x == max) return 1.f;
    if (x == -INFINITY) return 0.f;
    return __builtin_amdgcn_exp2f((x - max) * scale);
  }
  __device__ __forceinline__ uint64_t units(float x) const { return (uint64_t)rintf(of(x) * 0x1p43f); }
};

// Sums over the block and exclusive prefix sums in thread order.
__device__ uint64_t block_scan(uint64_t x, uint64_t* total, uint64_t* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t s = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  __syncthreads();
  if (lane == 63) tmp[wave] = s;
  __syncthreads();
  uint64_t before = 0, all = 0;
  for (int w = 0; w < kSampleThreads / 64; ++w) {
    if (w < wave) before += tmp[w];
    all += tmp[w];
  }
  *total = all;
  return before + s - x;
}

template <typename T>
__global__ __launch_bounds__(kSampleThreads) void sample_kernel(SampleLaunch a) {
  __shared__ uint64_t tmp[kSampleThreads / 64], hw[256];
  __shared__ uint32_t hc[256], pick[4];
  __shared__ float wmax[kSampleThreads / 64];
  __shared__ uint64_t above_w;
  const int tid = threadIdx.x, n = blockIdx.x, V = a.V;
  const T* row = reinterpret_cast<const T*>(a.logits) + (int64_t)n * a.stride;

  float mx = -INFINITY;
  for (int i = tid; i < V; i += kSampleThreads) mx = fmaxf(mx, logit(row, i));
#pragma unroll
  for (int d = 1; d < 64; d *= 2) mx = fmaxf(mx, __shfl_xor(mx, d));
  if ((tid & 63) == 0) wmax[tid >> 6] = mx;
  __syncthreads();
  for (int w = 0; w < kSampleThreads / 64; ++w) mx = fmaxf(mx, wmax[w]);
  if (mx == -INFINITY) {
    if (tid == 0) {
      a.tokens[n] = -1;
      if (a.logprobs) a.logprobs[n] = -INFINITY;
    }
    return;
  }
  const float temperature = a.temperature ? a.temperature[n] : 1.f;
  const bool greedy = !(temperature > 0.f);
  const Weight w{mx, greedy ? 1.f : 1.44269504f / temperature};
  int k = greedy ? 1 : a.top_k ? a.top_k[n] : 0;
  if (k <= 0 || k > V) k = V;
  const float top_p = a.top_p ? a.top_p[n] : 1.f;
  float min_p = a.min_p ? a.min_p[n] : 0.f;
  min_p = min_p > 0.f ? fminf(min_p, 1.f) : 0.f;

  // The last kept key and how many of its tokens, by a radix search over the
  // order-preserving bits: for the count k, then for the weight.
  uint32_t last = 0, ties = 0;
  uint64_t sum_k = 0;
  for (int by_weight = 0; by_weight < 2; ++by_weight) {
    uint64_t want = k;
    if (by_weight) {
      if (top_p >= 1.f || top_p != top_p) break;
      want = top_p > 0.f ? (uint64_t)ceil((double)top_p * (double)sum_k) : 1;
    } else if (k == V) {
      last = 0;
      ties = V;
      uint64_t s = 0;
      for (int i = tid; i < V; i += kSampleThreads) s += w.units(logit(row, i));
      block_scan(s, &sum_k, tmp);
      continue;
    }
    uint32_t prefix = 0;
    uint64_t above_c = 0, above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < 256) hc[tid] = 0, hw[tid] = 0;
      __syncthreads();
      for (int i = tid; i < V; i += kSampleThreads) {
        const float x = logit(row, i);
        const uint32_t key = float_order_key(x);
        if (shift < 24 && (key >> (shift + 8)) != prefix) continue;
        atomicAdd(&hc[(key >> shift) & 255], 1u);
        atomicAdd((unsigned long long*)&hw[(key >> shift) & 255], (unsigned long long)w.units(x));
      }
      __syncthreads();
      if (tid == 0) {
        int bin = 255;
        uint64_t c = above_c, s = above;
        for (; bin > 0; --bin) {
          if ((by_weight ? s + hw[bin] : c + hc[bin]) >= want) break;
          c += hc[bin];
          s += hw[bin];
        }
        pick[0] = bin;
        pick[1] = (uint32_t)c;
        pick[2] = hc[bin];
        above_w = s;
      }
      __syncthreads();
      prefix = prefix << 8 | pick[0];
      above_c = pick[1];
      above = above_w;
    }
    // prefix is the whole key; all of its tokens weigh the same.
    const uint32_t here = pick[2];
    const uint64_t each = hw[prefix & 255] / (here ? here : 1);
    uint32_t r;
    if (by_weight) {
      r = each ? (uint32_t)((want - above + each - 1) / each) : 1;
      if (prefix < last || (prefix == last && r > ties)) break;  // the top k end first
    } else {
      r = k - (uint32_t)above_c;
      sum_k = above + r * each;
    }
    last = prefix;
    ties = r;
  }

  // The draw: each thread a run of the vocabulary.
  const int seg = (V + kSampleThreads - 1) / kSampleThreads;
  const int i0 = min(V, tid * seg), i1 = min(V, i0 + seg);
  uint64_t c = 0, total;
  for (int i = i0; i < i1; ++i) c += float_order_key(logit(row, i)) == last;
  const uint64_t tie0 = block_scan(c, &total, tmp);
  auto kept = [&](int i, uint64_t& tie) -> uint64_t {
    const float x = logit(row, i);
    const uint32_t key = float_order_key(x);
    if (key < last || (key == last && tie++ >= ties) || !(w.of(x) >= min_p)) return 0;
    return w.units(x);
  };
  uint64_t s = 0, tie = tie0;
  for (int i = i0; i < i1; ++i) s += kept(i, tie);
  const uint64_t before = block_scan(s, &total, tmp);
  const float u = a.u[n];
  const uint64_t r = u > 0.f ? (uint64_t)fmin((double)u * (double)total, (double)(total - 1)) : 0;
  if (r >= before && r < before + s) {
    uint64_t cum = before;
    tie = tie0;
    for (int i = i0; i < i1; ++i) {
      const uint64_t x = kept(i, tie);
      cum += x;
      if (cum > r) {
        a.tokens[n] = i;
        if (a.logprobs) a.logprobs[n] = (float)log((double)x / (double)total);
        break;
      }
    }
  }
}

}  // namespace

size_t sample_workspace(int, int, int) { return 0; }

hipError_t launch_sample(const SampleLaunch& a, int dtype, hipStream_t stream) {
  if (dtype == NACL_F32) sample_kernel<float><<<a.N, kSampleThreads, 0, stream>>>(a);
  else sample_kernel<__bf16><<<a.N, kSampleThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace nacl
