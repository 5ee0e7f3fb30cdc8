// Attention of a decoding step: the new tokens' queries against their own
// sequence's cache and against a prefix that a group of sequences shares
// (nacl_prefix_attention).
//
// The rows that read the same K and V are taken together: for the prefix the
// queries of every sequence, query head and token of a group (rows of one K/V
// head: ((i * G) + e) * T + t for sequence i of the group), for the own cache
// those of one sequence ((t * G) + e, so that a block's causal limits rise).
// A work-group takes a block of rows and a chunk of keys, its waves the chunk's
// tiles in turn, each with a softmax of its own (running maximum and sum); the
// waves' results are joined in LDS and either are the output (one chunk in all)
// or go to the workspace, where merge_kernel joins a row's chunks.

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

constexpr int kStreamWaves = 4;
constexpr int kStreamThreads = 64 * kStreamWaves;
constexpr int kRsrcWord3 = 0x00020000;

__device__ __forceinline__ float group_max(float x) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float group_sum(float x) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Own cache rows that query token t of sequence b sees.
__device__ __forceinline__ int own_limit(const PrefixLaunch& a, int b, int t) {
  if (a.n_new && t >= a.n_new[b]) return 0;
  const int64_t n = (int64_t)a.row0 + (a.lens ? a.lens[b] : 0) + t + 1;
  return (int)(n < 0 ? 0 : n > a.L ? a.L : n);
}
__device__ __forceinline__ int prefix_len(const PrefixLaunch& a, int group) {
  const int n = a.plens ? a.plens[group] : a.Lp;
  return n < 0 ? 0 : n > a.Lp ? a.Lp : n;
}
// The last of tokens t0 .. t1 that is not padding (none: t0 - 1).
__device__ __forceinline__ int last_real(const PrefixLaunch& a, int b, int t0, int t1) {
  if (!a.n_new) return t1;
  return max(t0 - 1, min(t1, a.n_new[b] - 1));
}
// Keys per chunk where n keys are shared out to at most n_split chunks.
__device__ __forceinline__ int chunk_of(int n, int n_split) {
  const int c = (n + n_split - 1) / n_split;
  return max(kPrefixMinChunk, (c + 31) & ~31);
}

// A query row of a block: its (sequence, query head, token), the keys it sees.
struct RowAt {
  int b, hq, t, limit;
};
__device__ __forceinline__ RowAt row_at(const PrefixLaunch& a, bool prefix, int owner, int h, int row) {
  RowAt r;
  if (prefix) {
    const int per = a.G * a.T;
    const int i = row / per, u = row - i * per;
    r.b = owner * a.per_group + i;
    r.hq = h * a.G + u / a.T;
    r.t = u % a.T;
    r.limit = a.n_new && r.t >= a.n_new[r.b] ? 0 : prefix_len(a, owner);
  } else {
    r.b = owner;
    r.t = row / a.G;
    r.hq = h * a.G + row % a.G;
    r.limit = own_limit(a, owner, r.t);
  }
  return r;
}

// K, V and Q fragments by type.  Lane (g, r) = (lane / 16, lane mod 16).
//
// S^T = K Q^T, keys as MFMA rows: the lane holds logits of query r (keys 4 g ..
// 4 g + 3 of each block of 16), so its softmax statistics are scalars.  O^T +=
// V^T P^T with P straight from those registers: the contraction runs over the
// keys in the order the lanes hold them, and row r of O^T's tile dt is entry
// kDt r + dt of the head, so that a lane loads kDt neighbouring entries of each
// of its keys and holds kDt * 4 neighbouring entries of its query's output.
template <typename T, int D>
struct Frag;

// v_mfma_f32_16x16x32_bf16: 32 keys a tile; the value product's operand needs a
// lane's 8 keys of one entry side by side, by v_perm_b32 from the rows loaded.
template <int D>
struct Frag<__bf16, D> {
  static constexpr int kKeys = 32, kDt = D / 16, kKb = D / 32;
  bf16x8 kf[2][kKb];
  uint32_t vw[8][kDt / 2];  // key (4 g + i of block e: 4 e + i), entries kDt r ..

  struct Query {
    bf16x8 f[kKb];
    __device__ __forceinline__ void load(const __bf16* row, int g) {
#pragma unroll
      for (int kb = 0; kb < kKb; ++kb)
        f[kb] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(row + 32 * kb + 8 * g));
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
      for (int kb = 0; kb < kKb; ++kb) f[kb] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
    }
  };

  __device__ __forceinline__ void load_k(__amdgpu_buffer_rsrc_t rsrc, uint32_t row_bytes, int key0, int g, int r) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int kb = 0; kb < kKb; ++kb)
        kf[e][kb] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(
                                                   rsrc, (uint32_t)(key0 + 16 * e + r) * row_bytes + 64 * kb + 16 * g, 0, 0));
  }
  __device__ __forceinline__ void load_v(__amdgpu_buffer_rsrc_t rsrc, uint32_t row_bytes, int key0, int g, int r) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t at = (uint32_t)(key0 + 16 * e + 4 * g + i) * row_bytes + (uint32_t)r * (2 * kDt);
        if constexpr (kDt == 8) {
          const u32x4 w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0));
#pragma unroll
          for (int c = 0; c < 4; ++c) vw[4 * e + i][c] = w[c];
        } else {
          const auto w = __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, 0, 0);
#pragma unroll
          for (int c = 0; c < 2; ++c) vw[4 * e + i][c] = w[c];
        }
      }
  }
  // Logits of the tile: s[e][i] of key 16 e + 4 g + i.
  __device__ __forceinline__ void logits(const Query& q, f32x4 (&s)[2]) const {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < kKb; ++kb) t = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[e][kb], q.f[kb], t, 0, 0, 0);
      s[e] = t;
    }
  }
  // V^T's fragment of tile dt: entry kDt r + dt of the lane's 8 keys.
  __device__ __forceinline__ bf16x8 vfrag(int dt) const {
    u32x4 w;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      w[c] = __builtin_amdgcn_perm(vw[2 * c + 1][dt >> 1], vw[2 * c][dt >> 1], (dt & 1) ? 0x07060302u : 0x05040100u);
    return __builtin_bit_cast(bf16x8, w);
  }
  template <int R>
  __device__ __forceinline__ void value(const f32x4 (&p)[R][2], f32x4 (&acc)[R][kDt]) const {
    bf16x8 pf[R];
#pragma unroll
    for (int q = 0; q < R; ++q)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) pf[q][4 * e + i] = (__bf16)p[q][e][i];
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) {
      const bf16x8 vf = vfrag(dt);
#pragma unroll
      for (int q = 0; q < R; ++q) acc[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[q], acc[q][dt], 0, 0, 0);
    }
  }
  // Whether a value of the lane's key (e, i) is infinite or NaN; dropping it.
  __device__ __forceinline__ bool odd(int e, int i) const {
    bool x = false;
#pragma unroll
    for (int c = 0; c < kDt / 2; ++c) {
      const uint32_t w = vw[4 * e + i][c];
      x |= (w & 0x7F800000u) == 0x7F800000u || (w & 0x7F80u) == 0x7F80u;
    }
    return x;
  }
  __device__ __forceinline__ void drop(int e, int i) {
#pragma unroll
    for (int c = 0; c < kDt / 2; ++c) vw[4 * e + i][c] = 0;
  }
};

// v_mfma_f32_16x16x4_f32: 16 keys a tile (one block), everything as loaded.
template <int D>
struct Frag<float, D> {
  static constexpr int kKeys = 16, kDt = D / 16, kC = D / 16;
  f32x4 kf[kC];
  float vw[4][kDt];

  struct Query {
    f32x4 f[kC];
    __device__ __forceinline__ void load(const float* row, int g) {
#pragma unroll
      for (int c = 0; c < kC; ++c) f[c] = *reinterpret_cast<const f32x4*>(row + 16 * c + 4 * g);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
      for (int c = 0; c < kC; ++c) f[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };

  __device__ __forceinline__ void load_k(__amdgpu_buffer_rsrc_t rsrc, uint32_t row_bytes, int key0, int g, int r) {
#pragma unroll
    for (int c = 0; c < kC; ++c)
      kf[c] = __builtin_bit_cast(
          f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (uint32_t)(key0 + r) * row_bytes + 64 * c + 16 * g, 0, 0));
  }
  __device__ __forceinline__ void load_v(__amdgpu_buffer_rsrc_t rsrc, uint32_t row_bytes, int key0, int g, int r) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < kDt / 4; ++c) {
        const f32x4 w = __builtin_bit_cast(
            f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       rsrc, (uint32_t)(key0 + 4 * g + i) * row_bytes + (uint32_t)(r * kDt + 4 * c) * 4, 0, 0));
#pragma unroll
        for (int x = 0; x < 4; ++x) vw[i][4 * c + x] = w[x];
      }
  }
  __device__ __forceinline__ void logits(const Query& q, f32x4 (&s)[1]) const {
    f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) t = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c][i], q.f[c][i], t, 0, 0, 0);
    s[0] = t;
  }
  template <int R>
  __device__ __forceinline__ void value(const f32x4 (&p)[R][1], f32x4 (&acc)[R][kDt]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
        for (int q = 0; q < R; ++q)
          acc[q][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(vw[i][dt], p[q][0][i], acc[q][dt], 0, 0, 0);
  }
  __device__ __forceinline__ bool odd(int, int i) const {
    bool x = false;
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) x |= !(__builtin_fabsf(vw[i][dt]) < INFINITY);
    return x;
  }
  __device__ __forceinline__ void drop(int, int i) {
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) vw[i][dt] = 0.f;
  }
};

template <typename T>
__device__ __forceinline__ T to_out(float x) {
  return (T)x;
}

// One block of 16 R rows by one chunk of keys; see above.
template <typename T, int D, int R>
__global__ __launch_bounds__(kStreamThreads, 2) void prefix_stream_kernel(PrefixLaunch a) {
  using F = Frag<T, D>;
  constexpr int kE = F::kKeys / 16, kDt = F::kDt;
  constexpr int kRows = 16 * R;
  constexpr int kPad = 4;  // floats after each row in LDS: lanes of one column hit distinct banks
  __shared__ float so[kStreamWaves][kRows][D + kPad];
  __shared__ float sm[kStreamWaves][kRows], sl[kStreamWaves][kRows];

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = lane >> 4, r = lane & 15;

  // The item: prefix items first (the longer ones), then the sequences' own.
  int item = blockIdx.x;
  const bool prefix = item < a.prefix_items;
  if (!prefix) item -= a.prefix_items;
  const int n_split = prefix ? a.prefix_split : a.own_split;
  const int n_blocks = prefix ? a.prefix_blocks : a.own_blocks;
  const int n_rows = prefix ? a.per_group * a.G * a.T : a.G * a.T;
  const int split = item % n_split;
  item /= n_split;
  const int block = item % n_blocks;
  item /= n_blocks;
  const int h = item % a.H, owner = item / a.H;
  const int row0 = block * kRows, row1 = min(n_rows, row0 + kRows);

  // Keys of the block: those its last real row sees.
  int n;
  if (prefix) {
    n = prefix_len(a, owner);
  } else {
    const int t0 = row0 / a.G, t1 = last_real(a, owner, t0, (row1 - 1) / a.G);
    n = t1 < t0 ? 0 : own_limit(a, owner, t1);
  }
  const int chunk = chunk_of(n, n_split);
  const int key_lo = split * chunk, key_hi = min(n, key_lo + chunk);
  if (key_lo >= key_hi && !(a.direct && split == 0)) return;

  typename F::Query qf[R];
  int limit[R];
  bool plain = true;  // every row of the block sees every key of the chunk
#pragma unroll
  for (int q = 0; q < R; ++q) {
    const int row = row0 + 16 * q + r;
    limit[q] = 0;
    qf[q].zero();
    if (row < row1) {
      const RowAt x = row_at(a, prefix, owner, h, row);
      limit[q] = x.limit;
      qf[q].load(reinterpret_cast<const T*>(a.q) + (int64_t)x.b * a.qs[0] + (int64_t)x.hq * a.qs[1] + (int64_t)x.t * a.qs[2],
                 g);
    }
    plain = plain && (row >= row1 || limit[q] >= key_hi);
  }
  plain = __all(plain);

  const int64_t* ks = prefix ? a.pks : a.ks;
  const int64_t* vs = prefix ? a.pvs : a.vs;
  const T* kh = reinterpret_cast<const T*>(prefix ? a.pk : a.k) + (int64_t)owner * ks[0] + (int64_t)h * ks[1];
  const T* vh = reinterpret_cast<const T*>(prefix ? a.pv : a.v) + (int64_t)owner * vs[0] + (int64_t)h * vs[1];
  const uint32_t krow = (uint32_t)ks[2] * sizeof(T), vrow = (uint32_t)vs[2] * sizeof(T);
  // Rows at or past the chunk's end read as zeros.
  const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(kh), (short)0,
                                                                      (int)((uint32_t)key_hi * krow), kRsrcWord3);
  const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(vh), (short)0,
                                                                      (int)((uint32_t)key_hi * vrow), kRsrcWord3);

  f32x4 acc[R][kDt];
  float m[R], l[R];
#pragma unroll
  for (int q = 0; q < R; ++q) {
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) acc[q][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[q] = -INFINITY;
    l[q] = 0.f;
  }

  F f;
  int key0 = key_lo + wave * F::kKeys;
  if (key0 < key_hi) {
    f.load_k(kr, krow, key0, g, r);
    f.load_v(vr, vrow, key0, g, r);
  }
  for (; key0 < key_hi; key0 += kStreamWaves * F::kKeys) {
    f32x4 s[R][kE];
#pragma unroll
    for (int q = 0; q < R; ++q) f.logits(qf[q], s[q]);
    const int next = key0 + kStreamWaves * F::kKeys;
    if (next < key_hi) f.load_k(kr, krow, next, g, r);
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (!plain || key0 + F::kKeys > key_hi) {
        const int lim = min(limit[q], key_hi) - key0 - 4 * g;
#pragma unroll
        for (int e = 0; e < kE; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * e + i >= lim) s[q][e][i] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < kE; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[q][e][i]);
      mx = group_max(mx);
      const float mn = fmaxf(m[q], mx * a.c2);
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float alpha = __builtin_amdgcn_exp2f(m[q] - ref);
      m[q] = mn;
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < kE; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[q][e][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[q][e][i], a.c2, -ref));
          sum += s[q][e][i];
        }
      l[q] = l[q] * alpha + sum;
      if (__ballot(alpha != 1.f)) {
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt) acc[q][dt] *= alpha;
      }
    }
    if (!plain) {
      // Some rows do not see all keys.  A hidden key has probability 0, which
      // times an infinite or NaN value would still be NaN: where there is such a
      // value, the product is taken row by row of the causal order, each with
      // the keys it sees.
      bool odd = false;
#pragma unroll
      for (int e = 0; e < kE; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) odd = odd || f.odd(e, i);
      if (__any(odd)) {
        int from = 0;  // rows with this limit or less are done
        while (true) {
          int lim = 0x7FFFFFFF;  // the smallest limit left
#pragma unroll
          for (int q = 0; q < R; ++q)
            if (limit[q] > from) lim = min(lim, limit[q]);
#pragma unroll
          for (int x = 1; x < 16; x *= 2) lim = min(lim, __shfl_xor(lim, x));
          if (lim == 0x7FFFFFFF) break;
          F part = f;
          f32x4 p[R][kE];
#pragma unroll
          for (int q = 0; q < R; ++q)
#pragma unroll
            for (int e = 0; e < kE; ++e)
#pragma unroll
              for (int i = 0; i < 4; ++i) p[q][e][i] = limit[q] == lim ? s[q][e][i] : 0.f;
#pragma unroll
          for (int e = 0; e < kE; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + 16 * e + 4 * g + i >= lim) part.drop(e, i);
          f32x4 add[R][kDt];
#pragma unroll
          for (int q = 0; q < R; ++q)
#pragma unroll
            for (int dt = 0; dt < kDt; ++dt) add[q][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
          part.template value<R>(p, add);
#pragma unroll
          for (int q = 0; q < R; ++q)
            if (limit[q] == lim) {
#pragma unroll
              for (int dt = 0; dt < kDt; ++dt) acc[q][dt] += add[q][dt];
            }
          from = lim;
        }
        if (next < key_hi) f.load_v(vr, vrow, next, g, r);
        continue;
      }
    }
    f.template value<R>(s, acc);
    if (next < key_hi) f.load_v(vr, vrow, next, g, r);
  }

  // Join the waves: rows in LDS, each thread a run of entries of one row.
#pragma unroll
  for (int q = 0; q < R; ++q) {
    const float lq = group_sum(l[q]);
    if (g == 0) {
      sm[wave][16 * q + r] = m[q];
      sl[wave][16 * q + r] = lq;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int dt = 0; dt < kDt; dt += 4)
        *reinterpret_cast<f32x4*>(&so[wave][16 * q + r][kDt * (4 * g + i) + dt]) =
            f32x4{acc[q][dt][i], acc[q][dt + 1][i], acc[q][dt + 2][i], acc[q][dt + 3][i]};
  }
  __syncthreads();
  constexpr int kPer = 8;  // entries per thread
  for (int u = tid; u < (row1 - row0) * (D / kPer); u += kStreamThreads) {
    const int lr = u / (D / kPer), d0 = (u % (D / kPer)) * kPer;
    float mt = -INFINITY;
#pragma unroll
    for (int w = 0; w < kStreamWaves; ++w) mt = fmaxf(mt, sm[w][lr]);
    const float ref = mt == -INFINITY ? 0.f : mt;
    float lt = 0.f, o[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] = 0.f;
#pragma unroll
    for (int w = 0; w < kStreamWaves; ++w) {
      const float c = __builtin_amdgcn_exp2f(sm[w][lr] - ref);
      lt += c * sl[w][lr];
#pragma unroll
      for (int i = 0; i < kPer; ++i) o[i] += c * so[w][lr][d0 + i];
    }
    const RowAt x = row_at(a, prefix, owner, h, row0 + lr);
    const int64_t at = ((int64_t)x.b * a.H * a.G + x.hq) * a.T + x.t;
    if (a.direct) {
      const float inv = lt == 0.f ? 0.f : 1.f / lt;
      T* dst = reinterpret_cast<T*>(a.out) + at * D + d0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) dst[i] = (T)(o[i] * inv);
      if (a.lse && d0 == 0) a.lse[at] = lt == 0.f ? -INFINITY : (mt + log2f(lt)) * 0.69314718055994531f;
    } else {
      const int64_t slot = at * (a.prefix_split + a.own_split) + (prefix ? split : a.prefix_split + split);
      float* dst = a.part_o + slot * D + d0;
#pragma unroll
      for (int i = 0; i < kPer; i += 4) *reinterpret_cast<f32x4*>(dst + i) = f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
      if (d0 == 0) a.part_ml[slot] = float2{mt, lt};
    }
  }
}

// A row's chunks joined: one wave per row.
template <typename T, int D>
__global__ __launch_bounds__(256) void prefix_merge_kernel(PrefixLaunch a) {
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int Hq = a.H * a.G;
  if (row >= (int64_t)a.B * Hq * a.T) return;
  const int t = (int)(row % a.T);
  const int64_t bh = row / a.T;
  const int b = (int)(bh / Hq), e = (int)(bh % Hq) % a.G;
  // The chunks that the row's blocks made.
  int np = 0, no = 0;
  if (!(a.n_new && t >= a.n_new[b])) {
    if (a.Lp) {
      const int n = prefix_len(a, b / a.per_group), c = chunk_of(n, a.prefix_split);
      np = (n + c - 1) / c;
    }
    const int r0 = (t * a.G + e) / a.block_rows * a.block_rows, r1 = min(a.G * a.T, r0 + a.block_rows);
    const int n = own_limit(a, b, last_real(a, b, r0 / a.G, (r1 - 1) / a.G)), c = chunk_of(n, a.own_split);
    no = (n + c - 1) / c;
  }
  const int64_t base = row * (a.prefix_split + a.own_split);
  const int total = np + no;
  auto slot = [&](int i) { return base + (i < np ? i : a.prefix_split + i - np); };
  float m = -INFINITY;
  for (int i = lane; i < total; i += 64) m = fmaxf(m, a.part_ml[slot(i)].x);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f, o[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) o[i] = 0.f;
  for (int i = 0; i < total; ++i) {
    const float2 ml = a.part_ml[slot(i)];
    const float c = __builtin_amdgcn_exp2f(ml.x - ref);
    l += c * ml.y;
#pragma unroll
    for (int x = 0; x < kPer; ++x) o[x] += c * a.part_o[slot(i) * D + kPer * lane + x];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* dst = reinterpret_cast<T*>(a.out) + row * D + kPer * lane;
#pragma unroll
  for (int x = 0; x < kPer; ++x) dst[x] = (T)(o[x] * inv);
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

template <typename T, int D>
hipError_t launch_t(const PrefixLaunch& a, hipStream_t stream) {
  const int64_t items = (int64_t)a.prefix_items + a.own_items;
  if (a.block_rows == 16) prefix_stream_kernel<T, D, 1><<<(unsigned)items, kStreamThreads, 0, stream>>>(a);
  else prefix_stream_kernel<T, D, 2><<<(unsigned)items, kStreamThreads, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError()) return e;
  if (!a.direct) {
    const int64_t rows = (int64_t)a.B * a.H * a.G * a.T;
    prefix_merge_kernel<T, D><<<(unsigned)((rows + 3) / 4), 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefix(const PrefixLaunch& a, int dtype, int D, hipStream_t stream) {
  if (dtype == NACL_F32) return D == 64 ? launch_t<float, 64>(a, stream) : launch_t<float, 128>(a, stream);
  return D == 64 ? launch_t<__bf16, 64>(a, stream) : launch_t<__bf16, 128>(a, stream);
}

}  // namespace nacl
