// Attention of a decoding step: the new tokens' queries against their own
// sequence's cache and against a prefix that a group of sequences shares
// (nacl_prefix_attention), or against their sequence's pages
// (nacl_paged_attention).
//
// The rows that read the same K and V are taken together: for the prefix the
// queries of every sequence, query head and token of a group (rows of one K/V
// head: ((i * G) + e) * T + t for sequence i of the group), for the own cache
// those of one sequence ((t * G) + e, so that a block's causal limits rise).
// A work-group takes a block of rows and a chunk of keys (of pages: blocks of keys that lie
// as many blocks apart as there are splits), its waves the chunk's tiles in turn, each
// with a softmax of its own (running maximum and sum); the waves' results are joined in
// LDS and either are the output (one chunk in all) or go to the workspace, where
// prefix_merge_kernel joins a row's chunks.

#include <type_traits>

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kTileRows = kPrefixTileRows, kWideRows = kPrefixWideRows, kTileKeys = 64;
constexpr int kMergeBatch = 8;
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

// Of pages, split i of n_split takes the blocks of so many keys i, i + n_split, i + 2 n_split, ...
// of those there are: blocks that its waves read at once (tiles: two of them).
template <typename T>
constexpr int kPagedBlock = sizeof(T) == 2 ? 128 : 64;

// A query row of a block: its (sequence, query head, token), the keys it sees
// (of padding, anything: its results are not taken).
struct RowAt {
  int b, hq, t, limit;
};
__device__ __forceinline__ bool padding(const PrefixLaunch& a, const RowAt& x) { return a.n_new && x.t >= a.n_new[x.b]; }
__device__ __forceinline__ RowAt row_at(const PrefixLaunch& a, bool prefix, int owner, int h, int row) {
  RowAt r;
  if (prefix) {
    const int per = a.G * a.T;
    const int i = row / per, u = row - i * per;
    r.b = owner * a.per_group + i;
    r.hq = h * a.G + u / a.T;
    r.t = u % a.T;
    r.limit = prefix_len(a, owner);
  } else {
    r.b = owner;
    r.t = a.T == 1 ? 0 : row / a.G;
    r.hq = h * a.G + row - r.t * a.G;
    r.limit = own_limit(a, owner, r.t);
  }
  return r;
}

// How a kernel's own caches are laid out: rows of a head behind each other, or pages;
// pools that span less than 4 GiB (kPagedNear) are addressed as such rows are, by
// buffer descriptors with 32-bit byte offsets: half the lane moves, and three
// work-groups of 16 rows fit a CU's registers (by 64-bit addresses two; calls of 32 caches of
// up to 600 rows 13.8 us and 15.4, of 2 x 2000 tokens 132 and 141, of 32 caches of up to 8256
// 137 and 136, of 3 of up to 131072 226 and 224).
enum Layout { kRows, kPagedNear, kPagedFar };
constexpr uint32_t kNowhere = 0xFFFFF000u;  // a byte offset past every near pool: loads give zeros

// Keys key0 .. key0 + N - 1 of a paged cache: lane i looks key key0 + i mod N up,
// a tile ahead of the loads that need it, and gives its rows' places to the
// lanes that load them.
template <int N, Layout LAYOUT>
struct PageTile {
  using Place = std::conditional_t<LAYOUT == kPagedFar, int64_t, uint32_t>;  // far: elements; near: bytes
  int page = 0, row = 0, key = 0;
  Place k = 0, v = 0;  // the key's row in the pools
  uint64_t ok = 0;     // bit i: key key0 + i is there

  // (A product with 2^32 / page, rounded down, is at most one short of j / page.)
  static __device__ __forceinline__ int entry_of(const PrefixLaunch& a, int j) {
    const int e = (int)__umulhi((uint32_t)j, a.page_inv);
    return j - e * a.page >= a.page ? e + 1 : e;
  }
  __device__ __forceinline__ void lookup(const PrefixLaunch& a, const int32_t* table, int key0, int lane) {
    key = key0 + (lane & (N - 1));
    const int j = min(key, a.L - 1), e = entry_of(a, j);
    row = j - e * a.page;
    page = table[e];
  }
  // What lies past key_hi or in a page outside the pool is hidden, and loaded from
  // nowhere (far: from the pool's first row).
  template <typename T>
  __device__ __forceinline__ void resolve(const PrefixLaunch& a, int key_hi) {
    const bool there = key < key_hi && (uint32_t)page < (uint32_t)a.n_pages;
    ok = __ballot(there);
    if constexpr (N < 64) ok &= (1ull << N) - 1;
    if constexpr (LAYOUT == kPagedFar) {
      k = there ? (int64_t)page * a.ks[0] + (int64_t)row * a.ks[2] : 0;
      v = there ? (int64_t)page * a.vs[0] + (int64_t)row * a.vs[2] : 0;
    } else {
      k = there ? ((uint32_t)page * (uint32_t)a.ks[0] + (uint32_t)row * (uint32_t)a.ks[2]) * (uint32_t)sizeof(T) : kNowhere;
      v = there ? ((uint32_t)page * (uint32_t)a.vs[0] + (uint32_t)row * (uint32_t)a.vs[2]) * (uint32_t)sizeof(T) : kNowhere;
    }
  }
  static constexpr uint64_t kAll = N < 64 ? (1ull << (N & 63)) - 1 : ~0ull;
};
__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) {
  return (uint32_t)__builtin_amdgcn_ds_bpermute(4 * lane, (int)x);
}
__device__ __forceinline__ int64_t from_lane(int64_t x, int lane) {
  return (int64_t)((uint64_t)from_lane((uint32_t)(x >> 32), lane) << 32 | from_lane((uint32_t)x, lane));
}

// What a head's K or V rows are loaded from: a descriptor and the bytes per row
// (kRows), a descriptor (kPagedNear), an address (kPagedFar).
template <typename T, Layout LAYOUT>
struct Head {
  __amdgpu_buffer_rsrc_t rsrc;
  uint32_t row_bytes = 0;
  const T* at = nullptr;
  // 16 or 8 bytes, `bytes` from the start of row `key` (kRows) or from a place.
  template <int BYTES, typename Where>
  __device__ __forceinline__ auto load(Where where, uint32_t bytes) const {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    using W = std::conditional_t<BYTES == 16, u32x4, u32x2>;
    if constexpr (LAYOUT == kPagedFar) {
      return *reinterpret_cast<const W*>(reinterpret_cast<const char*>(at + where) + bytes);
    } else {
      const uint32_t off = (LAYOUT == kRows ? (uint32_t)where * row_bytes : (uint32_t)where) + bytes;
      if constexpr (BYTES == 16) return __builtin_bit_cast(W, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, 0, 0));
      else return __builtin_bit_cast(W, __builtin_amdgcn_raw_buffer_load_b64(rsrc, off, 0, 0));
    }
  }
};

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

  // key(i): where key i of the tile lies.
  template <typename H, typename Key>
  __device__ __forceinline__ void load_k(const H& head, Key key, int g, int r) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const auto at = key(16 * e + r);
#pragma unroll
      for (int kb = 0; kb < kKb; ++kb) kf[e][kb] = __builtin_bit_cast(bf16x8, head.template load<16>(at, 64 * kb + 16 * g));
    }
  }
  template <typename H, typename Key>
  __device__ __forceinline__ void load_v(const H& head, Key key, int g, int r) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const auto w = head.template load<2 * kDt>(key(16 * e + 4 * g + i), (uint32_t)r * (2 * kDt));
#pragma unroll
        for (int c = 0; c < kDt / 2; ++c) vw[4 * e + i][c] = w[c];
      }
  }
  __device__ __forceinline__ void zero_v(int e, int i) {
#pragma unroll
    for (int c = 0; c < kDt / 2; ++c) vw[4 * e + i][c] = 0;
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
  // acc += V^T P^T.  The probabilities as two bf16, the nearest and the nearest of
  // what is left (2^-17 of them at most is lost): the second product costs nothing
  // where K and V come from memory, and the output's error against 64 bits is its
  // own rounding's (1.6e-3 of its size; 2.1e-3 with one bf16).
  template <int R>
  __device__ __forceinline__ void value(const f32x4 (&p)[R][2], f32x4 (&acc)[R][kDt]) const {
    bf16x8 hi[R], lo[R];
#pragma unroll
    for (int q = 0; q < R; ++q)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          hi[q][4 * e + i] = (__bf16)p[q][e][i];
          lo[q][4 * e + i] = (__bf16)(p[q][e][i] - (float)hi[q][4 * e + i]);
        }
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) {
      const bf16x8 vf = vfrag(dt);
#pragma unroll
      for (int q = 0; q < R; ++q) {
        acc[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, hi[q], acc[q][dt], 0, 0, 0);
        acc[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lo[q], acc[q][dt], 0, 0, 0);
      }
    }
  }
  // Whether a value of the lane's key (e, i) is infinite or NaN.
  __device__ __forceinline__ bool odd(int e, int i) const {
    bool x = false;
#pragma unroll
    for (int c = 0; c < kDt / 2; ++c) {
      const uint32_t w = vw[4 * e + i][c];
      x |= (w & 0x7F800000u) == 0x7F800000u || (w & 0x7F80u) == 0x7F80u;
    }
    return x;
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

  template <typename H, typename Key>
  __device__ __forceinline__ void load_k(const H& head, Key key, int g, int r) {
    const auto at = key(r);
#pragma unroll
    for (int c = 0; c < kC; ++c) kf[c] = __builtin_bit_cast(f32x4, head.template load<16>(at, 64 * c + 16 * g));
  }
  template <typename H, typename Key>
  __device__ __forceinline__ void load_v(const H& head, Key key, int g, int r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto at = key(4 * g + i);
#pragma unroll
      for (int c = 0; c < kDt / 4; ++c) {
        const f32x4 w = __builtin_bit_cast(f32x4, head.template load<16>(at, (uint32_t)(r * kDt + 4 * c) * 4));
#pragma unroll
        for (int x = 0; x < 4; ++x) vw[i][4 * c + x] = w[x];
      }
    }
  }
  __device__ __forceinline__ void zero_v(int, int i) {
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt) vw[i][dt] = 0.f;
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
};

// A work-group's share: a block of rows and a chunk of the keys they read.
struct Item {
  bool prefix;
  int owner, h, row0, row1;      // group or sequence, K/V head, rows of it
  int split, key_lo, key_hi;
  __device__ __forceinline__ bool nothing(const PrefixLaunch& a) const { return key_lo >= key_hi && !(a.direct && split == 0); }
};
__device__ __forceinline__ Item item_of(const PrefixLaunch& a, bool prefix, int i, int block, int rows) {
  Item it;
  it.prefix = prefix;
  const int n_split = prefix ? a.prefix_split : a.own_split;
  const int n_rows = prefix ? a.per_group * a.G * a.T : a.G * a.T;
  it.split = i % n_split;
  i /= n_split;
  it.h = i % a.H;
  it.owner = i / a.H;
  it.row0 = block * rows;
  it.row1 = min(n_rows, it.row0 + rows);
  // Keys of the block: those its last real row sees.
  int n;
  if (prefix) {
    n = prefix_len(a, it.owner);
  } else {
    const int t0 = it.row0 / a.G, t1 = last_real(a, it.owner, t0, (it.row1 - 1) / a.G);
    n = t1 < t0 ? 0 : own_limit(a, it.owner, t1);
  }
  const int chunk = chunk_of(n, n_split);
  it.key_lo = it.split * chunk;
  it.key_hi = min(n, it.key_lo + chunk);
  return it;
}

// A paged work-group's share.  Its first key depends on the split alone, so that the first
// page is looked up while the lengths are loaded (32 caches of up to 600 rows 13.8 us, with
// chunks that the lengths place 17.4), and all splits that there are blocks for are at
// work, however much wider than the sequence its table is (8 of 4000 rows under a table of
// 131072 29 us, by chunks of a fixed number of keys 100; under one of 4000 27.5 and 28).
template <typename T>
__device__ __forceinline__ Item paged_item(const PrefixLaunch& a, int rows, int unit, int block) {
  Item it;
  it.prefix = false;
  if (a.own_blocks == 1) {
    it.split = blockIdx.x;
    it.h = blockIdx.y;
    it.owner = blockIdx.z;
  } else {
    it.split = unit % a.own_split;
    unit /= a.own_split;
    it.h = unit % a.H;
    it.owner = unit / a.H;
  }
  it.row0 = block * rows;
  it.row1 = min(a.G * a.T, it.row0 + rows);
  it.key_lo = it.split * kPagedBlock<T>;
  return it;
}
__device__ __forceinline__ void paged_limit(const PrefixLaunch& a, Item& it) {
  int t0 = 0, t1 = 0;
  if (a.T > 1) {
    t0 = it.row0 / a.G;
    t1 = (it.row1 - 1) / a.G;
  }
  t1 = last_real(a, it.owner, t0, t1);
  it.key_hi = t1 < t0 ? 0 : own_limit(a, it.owner, t1);
}

// One head's K or V rows below the item's last key (what lies past them reads as
// zeros), or its pool.
template <typename T, Layout LAYOUT>
__device__ __forceinline__ Head<T, LAYOUT> head_of(const PrefixLaunch& a, const Item& it, const void* base, const int64_t (&st)[3]) {
  Head<T, LAYOUT> x;
  T* p = reinterpret_cast<T*>(const_cast<void*>(base)) + (int64_t)it.h * st[1];
  if constexpr (LAYOUT == kRows) {
    p += (int64_t)it.owner * st[0];
    x.row_bytes = (uint32_t)st[2] * sizeof(T);
    x.rsrc = __builtin_amdgcn_make_buffer_rsrc(p, (short)0, (int)((uint32_t)it.key_hi * x.row_bytes), kRsrcWord3);
  } else if constexpr (LAYOUT == kPagedNear) {
    x.rsrc = __builtin_amdgcn_make_buffer_rsrc(p, (short)0, (int)kNowhere, kRsrcWord3);
  } else {
    x.at = p;
  }
  return x;
}
template <typename T>
__device__ __forceinline__ const T* query_of(const PrefixLaunch& a, const RowAt& x) {
  return reinterpret_cast<const T*>(a.q) + (int64_t)x.b * a.qs[0] + (int64_t)x.hq * a.qs[1] + (int64_t)x.t * a.qs[2];
}

// Takes N neighbouring entries from d0 of a row's unnormalised output, with its
// maximum (base 2) and sum, to the output or the workspace.
template <typename T, int D, int N>
__device__ __forceinline__ void put(const PrefixLaunch& a, const Item& it, const RowAt& x, float m, float l, int d0,
                                    const float (&o)[N]) {
  const int64_t at = ((int64_t)x.b * a.H * a.G + x.hq) * a.T + x.t;
  if (a.direct) {
    const bool empty = l == 0.f || padding(a, x);
    const float inv = 1.f / l;
    T* dst = reinterpret_cast<T*>(a.out) + at * D + d0;
#pragma unroll
    for (int i = 0; i < N; ++i) dst[i] = (T)(empty ? 0.f : o[i] * inv);
    if (a.lse && d0 == 0) a.lse[at] = empty ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  } else {
    const int64_t slot = at * (a.prefix_split + a.own_split) + (it.prefix ? it.split : a.prefix_split + it.split);
    float* dst = a.part_o + slot * D + d0;
    if constexpr (N % 4 == 0) {
#pragma unroll
      for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4*>(dst + i) = f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) dst[i] = o[i];
    }
    if (d0 == 0) a.part_ml[slot] = float2{m, l};
  }
}

// An item one row after the other, reading the keys that the row sees and no
// others: for chunks of which some rows see a part and in which a value is
// infinite or NaN.  The matrix products above give a hidden key the probability
// 0, which times such a value would still be NaN.  A wave per row: 64 keys at a
// time, a lane each for the logits, then each lane D / 64 entries of the output.
template <typename T, int D, Layout LAYOUT>
__device__ __forceinline__ void odd_item(const PrefixLaunch& a, const Item& it) {
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t* ks = it.prefix ? a.pks : a.ks;
  const int64_t* vs = it.prefix ? a.pvs : a.vs;
  const int64_t owner = (LAYOUT != kRows) ? 0 : it.owner;
  const T* kh = reinterpret_cast<const T*>(it.prefix ? a.pk : a.k) + owner * ks[0] + (int64_t)it.h * ks[1];
  const T* vh = reinterpret_cast<const T*>(it.prefix ? a.pv : a.v) + owner * vs[0] + (int64_t)it.h * vs[1];
  // Key j's place; whether it is there.
  auto place = [&](int j, const int64_t* st, int64_t& at) {
    at = (int64_t)j * st[2];
    if constexpr (LAYOUT != kRows) {
      const int e = PageTile<64, kPagedFar>::entry_of(a, j), page = a.table[(int64_t)it.owner * a.table_stride + e];
      if ((uint32_t)page >= (uint32_t)a.n_pages) return false;
      at = (int64_t)page * st[0] + (int64_t)(j - e * a.page) * st[2];
    }
    return true;
  };
  for (int row = it.row0 + (threadIdx.x >> 6); row < it.row1; row += blockDim.x >> 6) {
    const RowAt x = row_at(a, it.prefix, it.owner, it.h, row);
    const T* q = query_of<T>(a, x);
    const int end = min(x.limit, it.key_hi);
    float m = -INFINITY, l = 0.f, o[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] = 0.f;
    auto keys = [&](int key0, int end) {
      float s = -INFINITY;
      int64_t at;
      const bool there = key0 + lane < end && place(key0 + lane, ks, at);
      if (there) {
        s = 0.f;
        const T* k = kh + at;
        for (int d = 0; d < D; ++d) s = __builtin_fmaf((float)k[d], (float)q[d], s);
      }
      float mn = s;
#pragma unroll
      for (int i = 1; i < 64; i *= 2) mn = fmaxf(mn, __shfl_xor(mn, i));
      mn = fmaxf(m, mn * a.c2);
      const float ref = mn == -INFINITY ? 0.f : mn;
      const float alpha = __builtin_amdgcn_exp2f(m - ref);
      m = mn;
      const float p = there ? __builtin_amdgcn_exp2f(__builtin_fmaf(s, a.c2, -ref)) : 0.f;
      l = l * alpha + p;
#pragma unroll
      for (int i = 0; i < kPer; ++i) o[i] *= alpha;
      for (int j = 0; j < min(64, end - key0); ++j) {
        const float pj = __shfl(p, j);
        if (!place(key0 + j, vs, at)) continue;
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[i] = __builtin_fmaf(pj, (float)vh[at + kPer * lane + i], o[i]);
      }
    };
    if constexpr (LAYOUT == kRows) {
      for (int key0 = it.key_lo; key0 < end; key0 += 64) keys(key0, end);
    } else {
      for (int block = it.key_lo; block < end; block += a.own_split * kPagedBlock<T>)
        for (int key0 = block; key0 < min(end, block + kPagedBlock<T>); key0 += 64) keys(key0, end);
    }
#pragma unroll
    for (int i = 1; i < 64; i *= 2) l += __shfl_xor(l, i);
    put<T, D, kPer>(a, it, x, m, l, kPer * lane, o);
  }
}

// ---------------------------------------------------------------------------
// Few rows: 16 R per work-group, whose waves take the chunk's tiles in turn,
// each with a softmax of its own; K and V go from memory to the fragments' registers.
// Memory bounds it: 32 ragged caches of up to 8256 rows, 8 heads, 4 query heads each,
// 690 MB in 137 us at best, 147 on average (5.0 and 4.7 TB/s; reads alone of as many
// bytes reach 5.9); 8 sequences over a prefix of 6553 rows and up to 576 of their own,
// 32 heads, 158 MB in 27 us (5.9 TB/s); fp32, 32 caches of 4128 rows, 1.08 GB in a call
// of 191 us (5.7 TB/s).  One token over 2112 rows: 5.6 to 6 us, one load latency after
// the other.

template <int D, int R>
struct StreamShared {
  static constexpr int kPad = 4;  // floats after each row: lanes of one column hit distinct banks
  float o[kWaves][16 * R][D + kPad];
  float m[kWaves][16 * R], l[kWaves][16 * R];
};

template <typename T, int D, int R, Layout LAYOUT>
__device__ __forceinline__ void stream_item(const PrefixLaunch& a, const Item& it, StreamShared<D, R>& sh,
                                            PageTile<Frag<T, D>::kKeys, LAYOUT> pages = {}) {
  using F = Frag<T, D>;
  constexpr int kE = F::kKeys / 16, kDt = F::kDt;
  static_assert(kPagedBlock<T> == kWaves * F::kKeys);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = lane >> 4, r = lane & 15;
  const int key_lo = it.key_lo, key_hi = it.key_hi;
  const int step = (LAYOUT != kRows) ? a.own_split * kPagedBlock<T> : kWaves * F::kKeys;

  typename F::Query qf[R];
  int limit[R];
  bool plain = true;  // every row of the block sees every key of the item
#pragma unroll
  for (int q = 0; q < R; ++q) {
    const int row = it.row0 + 16 * q + r;
    limit[q] = key_hi;
    qf[q].zero();
    if (row < it.row1) {
      const RowAt x = row_at(a, it.prefix, it.owner, it.h, row);
      limit[q] = min(x.limit, key_hi);
      qf[q].load(query_of<T>(a, x), g);
    }
    plain = plain && limit[q] >= key_hi;
  }
  plain = __all(plain);
  const int least = __builtin_amdgcn_readfirstlane(limit[0]);  // (pages: the first row sees the fewest)

  const Head<T, LAYOUT> kh = head_of<T, LAYOUT>(a, it, it.prefix ? a.pk : a.k, it.prefix ? a.pks : a.ks);
  const Head<T, LAYOUT> vh = head_of<T, LAYOUT>(a, it, it.prefix ? a.pv : a.v, it.prefix ? a.pvs : a.vs);
  const int32_t* table = (LAYOUT != kRows) ? a.table + (int64_t)it.owner * a.table_stride : nullptr;

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
  auto load_k = [&](int key) {
    if constexpr (LAYOUT != kRows) {
      pages.template resolve<T>(a, key_hi);
      f.load_k(kh, [&](int i) { return from_lane(pages.k, i); }, g, r);
      pages.lookup(a, table, key + step, lane);
    } else {
      f.load_k(kh, [&](int i) { return key + i; }, g, r);
    }
  };
  auto load_v = [&](int key) {
    if constexpr (LAYOUT != kRows) f.load_v(vh, [&](int i) { return from_lane(pages.v, i); }, g, r);
    else f.load_v(vh, [&](int i) { return key + i; }, g, r);
  };
  bool odd = false;  // an infinite or NaN value beside which some rows do not see all keys
  int key0 = key_lo + wave * F::kKeys;
  if (key0 < key_hi) {
    load_k(key0);
    load_v(key0);
  }
  for (; key0 < key_hi; key0 += step) {
    f32x4 s[R][kE];
#pragma unroll
    for (int q = 0; q < R; ++q) f.logits(qf[q], s[q]);
    const int next = key0 + step;
    const bool seen = plain || ((LAYOUT != kRows) && key0 + F::kKeys <= least);  // the tile, by every row
    const uint32_t ok = (uint32_t)pages.ok;  // of this tile
    const bool whole = (LAYOUT != kRows) ? ok == (uint32_t)pages.kAll : key0 + F::kKeys <= key_hi;
    if (next < key_hi) load_k(next);
#pragma unroll
    for (int q = 0; q < R; ++q) {
      if (!seen || !whole) {
        const int lim = limit[q] - key0 - 4 * g;
        const uint32_t mine = ok >> (4 * g);  // the lane's keys
#pragma unroll
        for (int e = 0; e < kE; ++e)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * e + i >= lim || ((LAYOUT != kRows) && !(mine >> (16 * e + i) & 1))) s[q][e][i] = -INFINITY;
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
    if (LAYOUT == kPagedFar && !whole) {
#pragma unroll
      for (int e = 0; e < kE; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(ok >> (16 * e + 4 * g + i) & 1)) f.zero_v(e, i);
    }
    if (!seen) {
#pragma unroll
      for (int e = 0; e < kE; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i) odd = odd || f.odd(e, i);
    }
    f.template value<R>(s, acc);
    if (next < key_hi) load_v(next);
  }

  if (!plain && __syncthreads_or(odd)) {
    odd_item<T, D, LAYOUT>(a, it);
    return;
  }

  // Join the waves: rows in LDS, each thread a run of entries of one row.
#pragma unroll
  for (int q = 0; q < R; ++q) {
    const float lq = group_sum(l[q]);
    if (g == 0) {
      sh.m[wave][16 * q + r] = m[q];
      sh.l[wave][16 * q + r] = lq;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int dt = 0; dt < kDt; dt += 4)
        *reinterpret_cast<f32x4*>(&sh.o[wave][16 * q + r][kDt * (4 * g + i) + dt]) =
            f32x4{acc[q][dt][i], acc[q][dt + 1][i], acc[q][dt + 2][i], acc[q][dt + 3][i]};
  }
  __syncthreads();
  constexpr int kPer = 8;  // entries per thread
  for (int u = tid; u < (it.row1 - it.row0) * (D / kPer); u += kThreads) {
    const int lr = u / (D / kPer), d0 = (u % (D / kPer)) * kPer;
    float mt = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mt = fmaxf(mt, sh.m[w][lr]);
    const float ref = mt == -INFINITY ? 0.f : mt;
    float lt = 0.f, o[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float c = __builtin_amdgcn_exp2f(sh.m[w][lr] - ref);
      lt += c * sh.l[w][lr];
#pragma unroll
      for (int i = 0; i < kPer; ++i) o[i] += c * sh.o[w][lr][d0 + i];
    }
    put<T, D, kPer>(a, it, row_at(a, it.prefix, it.owner, it.h, it.row0 + lr), mt, lt, d0, o);
  }
}

// ---------------------------------------------------------------------------
// Many rows (bf16): 32 per wave, 128 or 256 per work-group, whose waves share tiles of
// 64 keys in LDS (two of each of K and V, one barrier per tile; the next tile's
// rows wait in registers while the one in hand is used).  v_mfma_f32_32x32x16_bf16
// with the roles as above: lane (hl, n) = (lane / 32, lane mod 32) holds logits of
// query n, keys 8 (i / 4) + 4 hl + i mod 4, and the output's entries likewise.
// V stays in rows and is read transposed (ds_read_b64_tr_b16).
// 512 rows of 8 heads to 26214 keys: 67.5 us (0.82 PFLOP/s; a large product of the
// library 1.21).  The matrix cores are busy for 0.35 of the cycles (the LDS for 0.22,
// without conflicts); the softmax between the two products takes about as many, and two
// waves per SIMD that meet at each tile's barrier overlap the two in part.

typedef float f32x16 __attribute__((ext_vector_type(16)));

// The exponentials' reference is the row's exact maximum so far, so that the largest
// probability is 1, which bf16 holds without error.  (A reference that follows once
// it is passed by 2^8 spares most rescales: 512 rows of 8 heads to 26214 keys 80.0 us
// instead of 83.6, but with logits of standard deviation 1 / 2 / 3 an error of 2.26 /
// 2.10 / 1.94e-3 of the output's size instead of 2.14 / 1.75 / 1.68e-3; the output's
// own rounding is 1.66e-3.  The probabilities as two bf16 reach that at 101.0 us; one,
// as in the prefill's attention, is what matrix cores as busy as here are worth.)
constexpr int kAhead = 2;

template <int D>
struct TileShared {
  unsigned char k[2][kTileKeys * D * 2], v[2][kTileKeys * D * 2];
};

template <int D, int ROWS, Layout LAYOUT>
__device__ __forceinline__ void tile_item(const PrefixLaunch& a, const Item& it, TileShared<D>& sh,
                                          PageTile<kTileKeys, LAYOUT> pages = {}) {
  constexpr int kRowBytes = D * 2, kChunks = kRowBytes / 16;
  constexpr int kC = D / 16, kDt = D / 32;
  constexpr int kThreads = 2 * ROWS;
  constexpr int kUnits = kTileKeys * kChunks / kThreads;  // 16-byte pieces of a tile per thread
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int hl = lane >> 5, n = lane & 31;
  const int key_lo = it.key_lo, key_hi = it.key_hi;

  bf16x8 qf[kC];
  int limit = key_hi;
  const int row = it.row0 + 32 * wave + n;
  const bool real = row < it.row1;
  RowAt at{};
  if (real) {
    at = row_at(a, it.prefix, it.owner, it.h, row);
    limit = min(at.limit, key_hi);
  }
#pragma unroll
  for (int c = 0; c < kC; ++c)
    qf[c] = real ? __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(query_of<__bf16>(a, at) + 16 * c + 8 * hl))
                 : __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
  const bool plain = __all(limit >= key_hi);
  const int least = __builtin_amdgcn_readfirstlane(limit);  // (pages: the wave's first row sees the fewest)
  static_assert(kPagedBlock<__bf16> == 2 * kTileKeys);
  const int step = (LAYOUT != kRows) ? a.own_split * kPagedBlock<__bf16> : 2 * kTileKeys;
  const bool idle = it.row0 + 32 * wave >= it.row1;  // no row in this wave

  const Head<__bf16, LAYOUT> kh = head_of<__bf16, LAYOUT>(a, it, it.prefix ? a.pk : a.k, it.prefix ? a.pks : a.ks);
  const Head<__bf16, LAYOUT> vh = head_of<__bf16, LAYOUT>(a, it, it.prefix ? a.pv : a.v, it.prefix ? a.pvs : a.vs);
  const int32_t* table = (LAYOUT != kRows) ? a.table + (int64_t)it.owner * a.table_stride : nullptr;

  // Pieces of 16 bytes are permuted by row: the 16 rows of a K fragment's half and
  // the four rows by four pieces of a V fragment's fall on all 64 banks (two rows of
  // D = 64 share a line of banks).  No conflicts, which were 0.29 of the LDS's busy
  // cycles with V permuted within 128 bytes.
  auto kswz = [](int key) { return kChunks == 16 ? key & 15 : (key >> 1) & 7; };
  auto vswz = [](int key) { return kChunks == 16 ? (key & 3) << 2 : (key & 2) << 1; };
  const bool causal = !it.prefix && a.T > 1;
  bool odd = false;  // as for few rows
  u32x4 kreg[kUnits], vreg[kUnits];
  auto load = [&](int key0, int after) {  // the tile after it
    if constexpr (LAYOUT != kRows) pages.template resolve<__bf16>(a, key_hi);
    auto piece = [&](const Head<__bf16, LAYOUT>& head, auto place, int u) {
      const int p = tid + kThreads * u, key = p / kChunks;
      const uint32_t bytes = (uint32_t)(p % kChunks) * 16;
      if constexpr (LAYOUT != kRows) return head.template load<16>(from_lane(place, key), bytes);
      else return head.template load<16>(key0 + key, bytes);
    };
#pragma unroll
    for (int u = 0; u < kUnits; ++u) kreg[u] = piece(kh, pages.k, u);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) vreg[u] = piece(vh, pages.v, u);
    if constexpr (LAYOUT == kPagedFar) {
      if (pages.ok != pages.kAll) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
          if (!(pages.ok >> ((tid + kThreads * u) / kChunks) & 1)) vreg[u] = u32x4{0, 0, 0, 0};
      }
    }
    if constexpr (LAYOUT != kRows) pages.lookup(a, table, after, lane);
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int p = tid + kThreads * u, r = p / kChunks, x = p % kChunks;
      *reinterpret_cast<u32x4*>(sh.k[buf] + r * kRowBytes + ((x ^ kswz(r)) * 16)) = kreg[u];
      *reinterpret_cast<u32x4*>(sh.v[buf] + r * kRowBytes + ((x ^ vswz(r)) * 16)) = vreg[u];
      if (causal) {
#pragma unroll
        for (int c = 0; c < 4; ++c) odd = odd || (vreg[u][c] & 0x7F800000u) == 0x7F800000u || (vreg[u][c] & 0x7F80u) == 0x7F80u;
      }
    }
  };
  // K fragment (keys 32 kt + n, entries 16 c + 8 hl ..), V^T fragment (entries 32
  // dt + n, the keys that the lane's logits of step ks hold).
  auto kfrag = [&](int buf, int kt, int c) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(sh.k[buf] + (32 * kt + n) * kRowBytes +
                                                                      (((2 * c + hl) ^ kswz(n)) * 16)));
  };
  const int i16 = lane & 15, vkey = 4 * hl + (i16 >> 2);
  uint32_t va[kDt];
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt)
    va[dt] = (uint32_t)(vkey * kRowBytes + (((4 * dt + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ vswz(vkey)) * 16) +
                        (i16 & 1) * 8);
  auto vfrag = [&](int buf, int ks, int dt) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    const unsigned char* p = sh.v[buf] + va[dt] + ks * 16 * kRowBytes;
    union {
      s16x4 h[2];
      bf16x8 v;
    } u;
    u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
    u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 8 * kRowBytes));
    return u.v;
  };

  f32x16 acc[kDt];
#pragma unroll
  for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;
  float m = -INFINITY, l = 0.f;

  if (key_lo < key_hi) {
    load(key_lo, key_lo + kTileKeys);
    store(0);
  }
  auto tile = [&](auto buf_c, int key0, int next, int after) {
    constexpr int buf = decltype(buf_c)::value;
    __syncthreads();
    const uint64_t ok = pages.ok;  // of this tile
    const bool seen = plain || ((LAYOUT != kRows) && key0 + kTileKeys <= least);
    const bool whole = (LAYOUT != kRows) ? ok == pages.kAll : key0 + kTileKeys <= key_hi;
    if (next < key_hi) load(next, after);
    if (!idle) {
      f32x16 s[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
      // K's fragments are read kAhead steps (of two MFMAs) before their use, and
      // fenced there: left alone, each pair is read right before it.
      bf16x8 kf[kAhead + 1][2];
#pragma unroll
      for (int c = 0; c < kC + kAhead; ++c) {
        if (c < kC) {
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) kf[c % (kAhead + 1)][kt] = kfrag(buf, kt, c);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (c >= kAhead) {
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
            s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[(c - kAhead) % (kAhead + 1)][kt], qf[c - kAhead], s[kt], 0, 0, 0);
        }
      }
      if (!seen || !whole) {
        asm volatile("");  // a branch: the comparisons cost as much as the exponentials' FMAs
        const int lim = limit - key0 - 4 * hl;
        const uint32_t mine[2] = {(uint32_t)(hl ? ok >> 4 : ok), (uint32_t)((hl ? ok >> 4 : ok) >> 32)};  // the lane's keys
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (32 * kt + 8 * (i / 4) + i % 4 >= lim || ((LAYOUT != kRows) && !(mine[kt] >> (8 * (i / 4) + i % 4) & 1)))
              s[kt][i] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kt][i]);
      auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * a.c2;
      if (__any(mx > m)) {
        const float mn = fmaxf(m, mx);
        const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= alpha;
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      float sum[2] = {0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[kt][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][i], a.c2, -ref));
          sum[i & 1] += s[kt][i];
        }
      l += sum[0] + sum[1];
      bf16x8 pf[4];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int i = 0; i < 8; ++i) pf[ks][i] = (__bf16)s[ks / 2][8 * (ks % 2) + i];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int dt = 0; dt < kDt; ++dt)
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vfrag(buf, ks, dt), pf[ks], acc[dt], 0, 0, 0);
    }
    if (next < key_hi) store(buf ^ 1);
  };
  for (int key0 = key_lo; key0 < key_hi; key0 += step) {
    tile(std::integral_constant<int, 0>{}, key0, key0 + kTileKeys, key0 + step);
    if (key0 + kTileKeys < key_hi) tile(std::integral_constant<int, 1>{}, key0 + kTileKeys, key0 + step, key0 + step + kTileKeys);
  }

  if (causal && __syncthreads_or(odd)) {
    odd_item<__bf16, D, LAYOUT>(a, it);
    return;
  }
  auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  if (real) {
#pragma unroll
    for (int dt = 0; dt < kDt; ++dt)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float o[4] = {acc[dt][i], acc[dt][i + 1], acc[dt][i + 2], acc[dt][i + 3]};
        put<__bf16, D, 4>(a, it, at, m, l, 32 * dt + 2 * i + 4 * hl, o);
      }
  }
}

// What takes the prefix's items and the own caches' (rows per work-group: 16,
// 32, 128 or 256).  The prefix's come first: they are the longer ones.
template <typename T, int D, int ROWS, Layout LAYOUT>
struct Part {
  using Shared = StreamShared<D, ROWS / 16>;
  using Pages = PageTile<Frag<T, D>::kKeys, LAYOUT>;
  static constexpr int kWaveKeys = Frag<T, D>::kKeys;  // by which a wave's first key lies after the one's before
  static __device__ __forceinline__ void run(const PrefixLaunch& a, const Item& it, Shared& sh, const Pages& pages = {}) {
    stream_item<T, D, ROWS / 16, LAYOUT>(a, it, sh, pages);
  }
};
template <int D, Layout LAYOUT>
struct Part<__bf16, D, kTileRows, LAYOUT> {
  using Shared = TileShared<D>;
  using Pages = PageTile<kTileKeys, LAYOUT>;
  static constexpr int kWaveKeys = 0;
  static __device__ __forceinline__ void run(const PrefixLaunch& a, const Item& it, Shared& sh, const Pages& pages = {}) {
    tile_item<D, kTileRows, LAYOUT>(a, it, sh, pages);
  }
};
template <int D>
struct Part<__bf16, D, kWideRows, kRows> {
  using Shared = TileShared<D>;
  static __device__ __forceinline__ void run(const PrefixLaunch& a, const Item& it, Shared& sh) {
    tile_item<D, kWideRows, kRows>(a, it, sh);
  }
};
constexpr int threads_of(int rows) { return rows >= kTileRows ? 2 * rows : kThreads; }

// (0: none of them in this launch, so that the code of the other alone is there.)
template <typename T, int D, int PREFIX, int OWN, Layout LAYOUT = kRows, int WAVES = LAYOUT == kPagedNear && OWN == 16 ? 3 : 2>
__global__ __launch_bounds__(threads_of(PREFIX > OWN ? PREFIX : OWN), WAVES) void prefix_kernel(PrefixLaunch a) {
  using P = Part<T, D, PREFIX ? PREFIX : OWN, LAYOUT>;
  using O = Part<T, D, OWN ? OWN : PREFIX, LAYOUT>;
  union Shared {
    typename P::Shared p;
    typename O::Shared o;
  };
  __shared__ __attribute__((aligned(16))) unsigned char smem[sizeof(Shared)];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  if constexpr (LAYOUT != kRows) {
    const int blocks = a.own_blocks, slot = blockIdx.x >> 3;
    const int unit = blocks == 1 ? 0 : (slot / blocks) * 8 + (blockIdx.x & 7);
    if (unit >= a.own_units) return;
    Item it = paged_item<T>(a, OWN, unit, blocks == 1 ? 0 : slot % blocks);
    typename O::Pages pages;
    pages.lookup(a, a.table + (int64_t)it.owner * a.table_stride, it.key_lo + (int)(threadIdx.x >> 6) * O::kWaveKeys, threadIdx.x & 63);
    paged_limit(a, it);
    if (!it.nothing(a)) O::run(a, it, sh.o, pages);
    return;
  }
  // Work-groups are dealt to the 8 XCDs in turn.  The row blocks that read the
  // same chunk of K and V follow each other on one XCD, whose L2 they share; the
  // prefix's chunks come first.
  const int xcd = blockIdx.x & 7;
  int slot = blockIdx.x >> 3;
  const bool prefix = OWN == 0 || (PREFIX != 0 && slot < a.prefix_slots);
  if (PREFIX && !prefix) slot -= a.prefix_slots;
  const int blocks = prefix ? a.prefix_blocks : a.own_blocks;
  const int unit = (slot / blocks) * 8 + xcd;
  if (unit >= (prefix ? a.prefix_units : a.own_units)) return;
  const Item it = item_of(a, prefix, unit, slot % blocks, prefix ? PREFIX : OWN);
  if (it.nothing(a)) return;
  if constexpr (PREFIX == OWN || PREFIX == 0 || OWN == 0) {
    O::run(a, it, sh.o);
  } else {
    if (prefix) P::run(a, it, sh.p);
    else O::run(a, it, sh.o);
  }
}

// A row's chunks joined (the workspace's bytes bound it: 4096 rows of 17 chunks 36 MB,
// written and read back by way of the caches), W waves per row: D / 4 lanes take a
// chunk's output, the others the next chunks', and all loads of up to kBatch chunks a
// lane are under way together.  One wave where that takes all chunks or the rows fill the chip
// (4096 rows of 17 chunks: 9.6 us, by four waves a row 12.8; of 2560 rows of 43 chunks
// the whole call 45.7 and 45.7), otherwise four (32 rows of 128 chunks: the whole call
// 99 us, by one wave 105).
template <typename T, int D, int W>
__global__ __launch_bounds__(kThreads) void prefix_merge_kernel(PrefixLaunch a) {
  constexpr int kPer = D / 4, kSlots = 64 / kPer, kBatch = kMergeBatch;
  __shared__ float so[W][D], sm[W], sl[W];
  const int lane = threadIdx.x & 63, d0 = (lane % kPer) * 4, mine = lane / kPer;
  const int wave = threadIdx.x >> 6;
  const int64_t row = W == 1 ? (int64_t)blockIdx.x * kWaves + wave : (int64_t)blockIdx.x;
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
    const int r0 = (t * a.G + e) / a.own_rows * a.own_rows, r1 = min(a.G * a.T, r0 + a.own_rows);
    const int n = own_limit(a, b, last_real(a, b, r0 / a.G, (r1 - 1) / a.G)), c = a.page ? kPagedBlock<T> : chunk_of(n, a.own_split);
    no = min((n + c - 1) / c, a.own_split);
  }
  const int64_t base = row * (a.prefix_split + a.own_split);
  const int total = np + no;
  auto slot = [&](int i) { return base + (i < np ? i : a.prefix_split + i - np); };
  f32x4 w[kBatch], o = {0.f, 0.f, 0.f, 0.f};
  float2 ml[kBatch];
  float m = -INFINITY, l = 0.f;
  for (int i0 = W == 1 ? 0 : wave * kBatch * kSlots; i0 < total; i0 += W * kBatch * kSlots) {
    float mx = m;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int i = i0 + u * kSlots + mine;
      ml[u] = float2{-INFINITY, 0.f};
      w[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (i < total) {
        ml[u] = a.part_ml[slot(i)];
        w[u] = *reinterpret_cast<const f32x4*>(a.part_o + slot(i) * D + d0);
      }
      mx = fmaxf(mx, ml[u].x);
    }
    const float ref = mx == -INFINITY ? 0.f : mx;  // of the lane's chunks
    const float alpha = __builtin_amdgcn_exp2f(m - ref);
    l *= alpha;
    o *= alpha;
    m = mx;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const float c = __builtin_amdgcn_exp2f(ml[u].x - ref);
      l += c * ml[u].y;
      o += c * w[u];
    }
  }
  // The lanes of the same entries.
#pragma unroll
  for (int x = kPer; x < 64; x *= 2) {
    const float m2 = __shfl_xor(m, x), l2 = __shfl_xor(l, x), mx = fmaxf(m, m2), ref = mx == -INFINITY ? 0.f : mx;
    const float c = __builtin_amdgcn_exp2f(m - ref), c2 = __builtin_amdgcn_exp2f(m2 - ref);
    l = c * l + c2 * l2;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = c * o[i] + c2 * __shfl_xor(o[i], x);
    m = mx;
  }
  if constexpr (W > 1) {
    if (mine == 0) *reinterpret_cast<f32x4*>(&so[wave][d0]) = o;
    if (lane == 0) {
      sm[wave] = m;
      sl[wave] = l;
    }
    __syncthreads();
    if (wave) return;
    m = -INFINITY;
#pragma unroll
    for (int i = 0; i < W; ++i) m = fmaxf(m, sm[i]);
    const float ref = m == -INFINITY ? 0.f : m;
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float c = __builtin_amdgcn_exp2f(sm[i] - ref);
      l += c * sl[i];
      o += c * *reinterpret_cast<const f32x4*>(&so[i][d0]);
    }
  }
  if (mine) return;
  const float inv = 1.f / l;
  T* dst = reinterpret_cast<T*>(a.out) + row * D + d0;
  // (A row without weight may hold 0 times an infinite value.)
#pragma unroll
  for (int i = 0; i < 4; ++i) dst[i] = (T)(l == 0.f ? 0.f : o[i] * inv);
  if (a.lse && lane == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

template <typename T, int D>
hipError_t launch_merge(const PrefixLaunch& a, hipStream_t stream) {
  if (a.direct) return hipSuccess;
  const int64_t rows = (int64_t)a.B * a.H * a.G * a.T;
  if (rows > 2048 || a.prefix_split + a.own_split <= kMergeBatch * (256 / D))
    prefix_merge_kernel<T, D, 1><<<(unsigned)((rows + kWaves - 1) / kWaves), kThreads, 0, stream>>>(a);
  else
    prefix_merge_kernel<T, D, kWaves><<<(unsigned)rows, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_paged_t(const PrefixLaunch& a, hipStream_t stream) {
  // (One row block: no two work-groups read the same keys, and the grid spares the divisions.)
  const dim3 groups = a.own_blocks == 1 ? dim3(a.own_split, a.H, a.B) : dim3(8u * (unsigned)a.own_slots);
  auto run = [&](auto layout) {
    constexpr Layout kLayout = decltype(layout)::value;
    if (a.own_rows == 16) prefix_kernel<T, D, 0, 16, kLayout><<<groups, kThreads, 0, stream>>>(a);
    else if (a.own_rows == 32) prefix_kernel<T, D, 0, 32, kLayout><<<groups, kThreads, 0, stream>>>(a);
    else if constexpr (std::is_same_v<T, __bf16>) prefix_kernel<T, D, 0, kTileRows, kLayout><<<groups, kThreads, 0, stream>>>(a);
  };
  if (a.near) run(std::integral_constant<Layout, kPagedNear>{});
  else run(std::integral_constant<Layout, kPagedFar>{});
  if (hipError_t e = hipGetLastError()) return e;
  return launch_merge<T, D>(a, stream);
}

template <typename T, int D>
hipError_t launch_t(const PrefixLaunch& a, hipStream_t stream) {
  PrefixLaunch own = a;
  auto run = [&](auto kernel, const PrefixLaunch& x, int threads = kThreads) {
    kernel<<<8u * (unsigned)(x.prefix_slots + x.own_slots), threads, 0, stream>>>(x);
  };
  if constexpr (std::is_same_v<T, __bf16>) {
    // The prefix's tiles have a launch of their own, so that the own caches'
    // chunks, which wait for memory, run at their own occupancy.  (Both in one,
    // alternating: 142 us for 512 rows of 8 heads to 26214 keys beside 64 caches of
    // 576 rows; the caches' last 119.)
    if (a.prefix_slots && a.prefix_rows >= kTileRows) {
      PrefixLaunch prefix = a;
      prefix.own_slots = 0;
      if (a.prefix_rows == kTileRows) run(prefix_kernel<T, D, kTileRows, 0>, prefix);
      else run(prefix_kernel<T, D, kWideRows, 0>, prefix, threads_of(kWideRows));
      if (hipError_t e = hipGetLastError()) return e;
      own.prefix_slots = 0;
    }
    if (a.own_rows == kTileRows) run(prefix_kernel<T, D, 0, kTileRows>, own);
  }
  if (a.own_rows == 32) run(prefix_kernel<T, D, 32, 32>, own);
  else if (a.own_rows == 16 && own.prefix_slots && a.prefix_rows == 32) run(prefix_kernel<T, D, 32, 16>, own);
  else if (a.own_rows == 16) run(prefix_kernel<T, D, 16, 16>, own);
  if (hipError_t e = hipGetLastError()) return e;
  return launch_merge<T, D>(a, stream);
}

}  // namespace

hipError_t launch_prefix(const PrefixLaunch& a, int dtype, int D, hipStream_t stream) {
  if (dtype == NACL_F32) return D == 64 ? launch_t<float, 64>(a, stream) : launch_t<float, 128>(a, stream);
  return D == 64 ? launch_t<__bf16, 64>(a, stream) : launch_t<__bf16, 128>(a, stream);
}

hipError_t launch_paged(const PrefixLaunch& a, int dtype, int D, hipStream_t stream) {
  if (dtype == NACL_F32) return D == 64 ? launch_paged_t<float, 64>(a, stream) : launch_paged_t<float, 128>(a, stream);
  return D == 64 ? launch_paged_t<__bf16, 64>(a, stream) : launch_paged_t<__bf16, 128>(a, stream);
}

}  // namespace nacl
