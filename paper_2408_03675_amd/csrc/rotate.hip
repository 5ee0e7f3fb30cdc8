// Queries and keys of new tokens, normalised per head and rotated by position,
// into the cache (nacl_rotate_append) or its pages (nacl_paged_append).

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotHeads = 2;  // heads in flight per wave

// 16 entries of a head per lane, as two runs of 8.
template <typename T>
struct Rot16;

template <>
struct Rot16<__bf16> {
  u32x4 w[2];
  __device__ __forceinline__ void load(const __bf16* p, int o0, int o1) {
    w[0] = *reinterpret_cast<const u32x4*>(p + o0);
    w[1] = *reinterpret_cast<const u32x4*>(p + o1);
  }
  __device__ __forceinline__ void store(__bf16* p, int o0, int o1) const {
    __builtin_nontemporal_store(w[0], reinterpret_cast<u32x4*>(p + o0));
    __builtin_nontemporal_store(w[1], reinterpret_cast<u32x4*>(p + o1));
  }
  __device__ __forceinline__ void get(float (&x)[16]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[2 * i] = __uint_as_float(w[i >> 2][i & 3] << 16);
      x[2 * i + 1] = __uint_as_float(w[i >> 2][i & 3] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[16]) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      bf16x8 t;
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = (__bf16)x[8 * e + i];
      w[e] = __builtin_bit_cast(u32x4, t);
    }
  }
};

template <>
struct Rot16<float> {
  f32x4 w[4];
  __device__ __forceinline__ void load(const float* p, int o0, int o1) {
    w[0] = *reinterpret_cast<const f32x4*>(p + o0);
    w[1] = *reinterpret_cast<const f32x4*>(p + o0 + 4);
    w[2] = *reinterpret_cast<const f32x4*>(p + o1);
    w[3] = *reinterpret_cast<const f32x4*>(p + o1 + 4);
  }
  __device__ __forceinline__ void store(float* p, int o0, int o1) const {
    __builtin_nontemporal_store(w[0], reinterpret_cast<f32x4*>(p + o0));
    __builtin_nontemporal_store(w[1], reinterpret_cast<f32x4*>(p + o0 + 4));
    __builtin_nontemporal_store(w[2], reinterpret_cast<f32x4*>(p + o1));
    __builtin_nontemporal_store(w[3], reinterpret_cast<f32x4*>(p + o1 + 4));
  }
  __device__ __forceinline__ void get(float (&x)[16]) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = w[i >> 2][i & 3];
  }
  __device__ __forceinline__ void set(const float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i >> 2][i & 3] = x[i];
  }
};

// D / 16 lanes hold one token's head, lane j of them the 16 entries that pairs
// 8 j .. 8 j + 7 rotate: entries 8 j .. and rot/2 + 8 j .. where a pair is half
// the rotated entries apart, entries 16 j .. 16 j + 15 where pairs are
// neighbours (and past the rotated entries).  So a pair lies in one lane, every
// access is 16 bytes, and a wave takes 1024 / D consecutive tokens of the batch
// through a run of heads with the tokens' cosines and sines in registers.
// Memory bounds it; the angles cost a fp64 product and one sincospi per pair and
// token, shared by the run.  Stores are non-temporal and two heads are in flight:
// 32768 tokens of 32 + 2 x 32 heads of 128 310 us (5.2 TB/s; a copy of 1 GiB
// reaches 5.15), with plain stores 347, with four heads 331; 2 x 12345 tokens of
// 32 + 2 x 8 heads from one projection's output 123 us (4.9 TB/s), plain 138; fp32,
// 16384 tokens of 32 + 2 x 32 heads 333 us (4.8 TB/s).  Neighbours as pairs put a lane's
// 16 entries side by side, so that an instruction stores 16 bytes of every 32 (bf16,
// 16384 tokens of 32 + 2 x 8 heads 87 us, 4.6 TB/s) or of every 64 (fp32, 8192 tokens
// of them 229 us, 1.8 TB/s; halves 79 us, 5.1 TB/s).
template <typename T, int D>
__global__ __launch_bounds__(kRotThreads) void rotate_append_kernel(RotateLaunch a) {
  constexpr int kLanes = D / 16, kTokens = 64 / kLanes;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int j = lane % kLanes;
  const int64_t tok = ((int64_t)blockIdx.x * (kRotThreads / 64) + wave) * kTokens + lane / kLanes;
  if (tok >= (int64_t)a.B * a.T) return;  // whole groups of kLanes lanes leave together
  const int b = (int)(tok / a.T), t = (int)(tok - (int64_t)b * a.T);
  if (a.n_new && t >= a.n_new[b]) return;
  // The token's place: a row of its sequence's cache, or of the page that its slot lies in.
  int64_t row, owner = b;
  bool in_cache;
  if (a.slots) {
    const int slot = a.slots[tok];
    in_cache = slot >= 0 && slot < a.n_pages * a.page;
    owner = slot / a.page;
    row = slot - owner * a.page;
  } else {
    row = (int64_t)a.row0 + (a.lens ? a.lens[b] : 0) + t;
    in_cache = row >= 0 && row < a.L;
  }

  const bool rotated = 16 * j < a.rot;
  const bool halves = rotated && !a.interleaved;
  const int o0 = halves ? 8 * j : 16 * j;
  const int o1 = halves ? a.rot / 2 + 8 * j : 16 * j + 8;

  const int Hq = a.H * a.G, n_heads = Hq + 2 * a.H;
  const int h0 = blockIdx.y * a.heads_per_run, h1 = min(n_heads, h0 + a.heads_per_run);

  // Cosine and sine of the lane's 8 pairs.  The turn's fraction is taken in
  // fp64: in fp32 a position of 2^20 would leave an angle good to 2^-4.  Of the
  // fraction the fp32 sine and cosine do: errors of 3.6e-8 of the outputs' size.
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = 1.f, sn[i] = 0.f;
  if (rotated && h0 < Hq + a.H) {
    const double pos = (double)a.pos[(int64_t)b * a.pos_stride + t];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double turn = pos * (double)a.inv_freq[8 * j + i] * 0.15915494309189533577;
      sincospif((float)(2.0 * (turn - rint(turn))), &sn[i], &cs[i]);
    }
  }
  float wt[16];
  int wt_of = -1;  // which weights wt holds

  const T* q = reinterpret_cast<const T*>(a.q) + (int64_t)b * a.qs[0] + (int64_t)t * a.qs[2];
  const T* kn = reinterpret_cast<const T*>(a.k_new) + (int64_t)b * a.kns[0] + (int64_t)t * a.kns[2];
  const T* vn = reinterpret_cast<const T*>(a.v_new) + (int64_t)b * a.vns[0] + (int64_t)t * a.vns[2];
  T* qo = reinterpret_cast<T*>(a.q_out) + (int64_t)b * a.qos[0] + (int64_t)t * a.qos[2];
  T* kc = reinterpret_cast<T*>(a.k) + owner * a.ks[0] + row * a.ks[2];
  T* vc = reinterpret_cast<T*>(a.v) + owner * a.vs[0] + row * a.vs[2];

  for (int hb = h0; hb < h1; hb += kRotHeads) {
    Rot16<T> x[kRotHeads];
#pragma unroll
    for (int e = 0; e < kRotHeads; ++e) {
      const int h = hb + e;
      if (h >= h1) break;
      const T* src = h < Hq ? q + h * a.qs[1] : h < Hq + a.H ? kn + (h - Hq) * a.kns[1] : vn + (h - Hq - a.H) * a.vns[1];
      x[e].load(src, o0, o1);
    }
#pragma unroll
    for (int e = 0; e < kRotHeads; ++e) {
      const int h = hb + e;
      if (h >= h1) break;
      if (h >= Hq + a.H) {  // a value: as it is
        if (in_cache) x[e].store(vc + (h - Hq - a.H) * a.vs[1], o0, o1);
        continue;
      }
      const int of = h < Hq ? 0 : 1;
      const T* weight = reinterpret_cast<const T*>(of ? a.k_weight : a.q_weight);
      float y[16];
      x[e].get(y);
      if (weight) {
        if (wt_of != of) {
          Rot16<T> w;
          w.load(weight, o0, o1);
          w.get(wt);
          wt_of = of;
        }
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) ss = fmaf(y[i], y[i], ss);
#pragma unroll
        for (int m = 1; m < kLanes; m *= 2) ss += __shfl_xor(ss, m);
        const float inv = 1.f / sqrtf(ss * (1.f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = y[i] * inv * wt[i];
      }
      float z[16];
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          z[2 * i] = y[2 * i] * cs[i] - y[2 * i + 1] * sn[i];
          z[2 * i + 1] = y[2 * i + 1] * cs[i] + y[2 * i] * sn[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          z[i] = y[i] * cs[i] - y[8 + i] * sn[i];
          z[8 + i] = y[8 + i] * cs[i] + y[i] * sn[i];
        }
      }
      if (!rotated) {  // an infinity times a sine of 0 would be NaN
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = y[i];
      }
      x[e].set(z);
      if (h < Hq)
        x[e].store(qo + h * a.qos[1], o0, o1);
      else if (in_cache)
        x[e].store(kc + (h - Hq) * a.ks[1], o0, o1);
    }
  }
}

}  // namespace

hipError_t launch_rotate_append(RotateLaunch a, int dtype, int D, int cus, hipStream_t stream) {
  const int tokens = (kRotThreads / 64) * 1024 / D;  // per work-group
  const int64_t groups = ((int64_t)a.B * a.T + tokens - 1) / tokens;
  const int heads = (a.G + 2) * a.H;
  // Runs of heads short enough that four work-groups per CU are there: 1024
  // single tokens 7.8 us, for eight 9.0; 2048 tokens 11.1 and 12.1.
  const int64_t want = (4 * (int64_t)cus + groups - 1) / groups;
  int runs = (int)(want < 1 ? 1 : want > heads ? heads : want);
  a.heads_per_run = (heads + runs - 1) / runs;
  runs = (heads + a.heads_per_run - 1) / a.heads_per_run;
  const dim3 grid((unsigned)groups, (unsigned)runs);
  if (dtype == NACL_F32) {
    if (D == 64) rotate_append_kernel<float, 64><<<grid, kRotThreads, 0, stream>>>(a);
    else rotate_append_kernel<float, 128><<<grid, kRotThreads, 0, stream>>>(a);
  } else {
    if (D == 64) rotate_append_kernel<__bf16, 64><<<grid, kRotThreads, 0, stream>>>(a);
    else rotate_append_kernel<__bf16, 128><<<grid, kRotThreads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace nacl
