// Validation that the decoding step's entry points share, and the plan of its
// attention (host side).
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <utility>

#include "../../include/nacl.h"
#include "internal.h"

namespace nacl {

constexpr int kPlanCus = 256;  // compute units the launches are planned for
constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline int elt_bytes(int dtype) { return dtype == NACL_F32 ? 4 : 2; }
inline int q_group_of(const nacl_problem* p) { return p->q_group > 1 ? p->q_group : 1; }

// Bytes [lo, hi) that a strided tensor of n[0] x n[1] x n[2] rows of D spans.
struct Extent {
  uintptr_t lo = 0, hi = 0;
  Extent(const void* base, const int64_t st[3], int64_t n0, int64_t n1, int64_t n2, int64_t D, int eb) {
    lo = (uintptr_t)base;
    hi = lo + (uintptr_t)((n0 - 1) * st[0] + (n1 - 1) * st[1] + (n2 - 1) * st[2] + D) * eb;
  }
  Extent(const void* base, uintptr_t bytes) : lo((uintptr_t)base), hi((uintptr_t)base + bytes) {}
  bool meets(const Extent& o) const { return lo < o.hi && o.lo < hi; }
};

inline int check_strides(const char* name, const int64_t st[3], int eb) {
  for (int i = 0; i < 3; ++i) {
    if (st[i] < 0) return fail_status(NACL_ERR_INVALID_ARG, "%s[%d] < 0", name, i);
    if (st[i] > ((int64_t)1 << 40)) return fail_status(NACL_ERR_UNSUPPORTED, "%s[%d] exceeds 2^40", name, i);
    if ((st[i] * eb) % 16)
      return fail_status(NACL_ERR_INVALID_ARG, "%s[%d] * element size must be a multiple of 16 bytes", name, i);
  }
  return NACL_OK;
}

// The problem and the parts of a step that both calls read.
inline int check_step(const nacl_problem* p, const nacl_step* s) {
  int st = validate_problem(p);
  if (st) return st;
  if (!s) return fail_status(NACL_ERR_INVALID_ARG, "step is NULL");
  if (s->T < 1) return fail_status(NACL_ERR_INVALID_ARG, "T must be >= 1 (got %d)", s->T);
  if (s->T > NACL_MAX_L) return fail_status(NACL_ERR_UNSUPPORTED, "T = %d exceeds %d", s->T, NACL_MAX_L);
  if (s->row0 < 0) return fail_status(NACL_ERR_INVALID_ARG, "row0 must be >= 0 (got %d)", s->row0);
  if ((int64_t)p->B * s->T >= (int64_t)1 << 28)
    return fail_status(NACL_ERR_UNSUPPORTED, "B * T reaches 2^28");
  if (!aligned(s->lens, 4) || !aligned(s->n_new, 4))
    return fail_status(NACL_ERR_INVALID_ARG, "lens and n_new must be 4-byte aligned");
  return check_strides("the step's q_stride", s->q_stride, elt_bytes(p->dtype));
}

// How the attention's rows and keys are shared out.  It depends on sizes only:
// the lengths are on the device, where each row block's keys are dealt to at
// most n_split chunks.
struct Plan {
  int per_group = 1, Lp = 0;
  int prefix_rows = 16, own_rows = 16;
  int prefix_blocks = 0, prefix_split = 0, own_blocks = 0, own_split = 0;
  int64_t prefix_units = 0, prefix_slots = 0, own_units = 0, own_slots = 0, rows = 0;
  bool direct = false;
  size_t ml = 0, total = 0;  // byte offset of part_ml, workspace bytes
};

inline Plan plan_of(const nacl_problem* p, const nacl_step* s, const nacl_prefix* x) {
  Plan a;
  const int G = q_group_of(p);
  const int groups = x ? x->G : 1;
  a.per_group = p->B / groups;
  a.Lp = x ? x->L : 0;
  a.rows = (int64_t)p->B * p->H * G * s->T;
  const int64_t own_rows = (int64_t)G * s->T, prefix_rows = own_rows * a.per_group;
  auto block = [&](int64_t rows) {
    return rows <= 16 ? 16 : rows <= 32 || p->dtype == NACL_F32 ? 32 : kPrefixTileRows;
  };
  a.own_rows = block(own_rows);
  a.prefix_rows = x ? block(prefix_rows) : a.own_rows;
  // Of a prefix 256 rows share a tile where there are as many: half the reads per
  // row (8 heads, 26214 keys: 512 rows 89 us, by tiles of 128 97, 2048 rows 246 and
  // 271, 256 rows 54 and 58, 160 rows 43 and 48).  Not of the own caches, whose work-groups are fewer (4 caches of
  // 4096 rows, 8 heads, 256 rows: 54 us, by 256 rows 83).
  if (x && a.prefix_rows == kPrefixTileRows && prefix_rows > kPrefixTileRows) a.prefix_rows = kPrefixWideRows;
  auto up = [](int64_t n, int64_t d) { return (n + d - 1) / d; };
  a.own_blocks = (int)up(own_rows, a.own_rows);
  a.prefix_blocks = x ? (int)up(prefix_rows, a.prefix_rows) : 0;
  const int64_t own_blocks = (int64_t)p->B * p->H * a.own_blocks, prefix_blocks = (int64_t)groups * p->H * a.prefix_blocks;
  // Chunks of about the same number of keys in both, as many as run together: three
  // work-groups per CU of 16 rows (32 caches of 8256 rows: 188 us, two 207, four 197), two of
  // 32 (3 caches of 5000 rows, 8 heads: 21.5 us, one 25; fp32, 32 rows of 8 heads to 8000 keys
  // beside 32 caches of 2000: 135 and 158) and of 16 beside a prefix read by tiles (whole
  // calls with 40 caches of 300 rows: 35.8 us, three 37.0, one 36.6; 16 of 4000: 80.1, 81.3,
  // 79.7; 48 of 1500: 63.0, 62.3, 70.0; 64 of 2000 and 128 of 1000 within 0.3 %), four
  // of 128, as causal blocks differ in length (512 tokens, 64 query heads over 8192 rows: 207
  // us, three 227).  Where most keys are a bf16 prefix's, one: fewer partial outputs to write
  // and join (32 rows of 8 heads to 26214 keys: 26 us, two 30, three 35; 8 sequences, 32
  // heads, a prefix of 6553 rows and 576 of their own: 33 us, three 35.5; but 32 caches of
  // 4000 rows beside 8 prefixes of 2000: 123 us, three 115).  A prefix read by tiles has
  // chunks of its own, one per CU (128 rows of 8 heads to 26214 keys: 40 us, two per CU 45; 64
  // rows 34.5 and 37) of at least 256 keys (128 rows of one head to 26214: 23 us, with 128
  // keys 26, with 512 26).
  const bool tiles = x && a.prefix_rows >= kPrefixTileRows;
  const int64_t own_keys = own_blocks * p->L, prefix_keys = prefix_blocks * a.Lp;
  const int64_t keys = own_keys + (tiles ? 0 : prefix_keys);
  const bool mostly_prefix = !tiles && p->dtype == NACL_BF16 && prefix_keys >= own_keys;
  const int per_cu = a.own_rows == kPrefixTileRows ? 4 : mostly_prefix ? 1 : tiles || a.own_rows == 32 || a.prefix_rows == 32 ? 2 : 3;
  const int64_t chunk = std::max<int64_t>(kPrefixMinChunk, up(keys, per_cu * kPlanCus));
  a.own_split = (int)up(p->L, chunk);
  a.prefix_split = (int)up(a.Lp, tiles ? std::max<int64_t>(256, up(prefix_keys, kPlanCus)) : chunk);
  a.own_units = (int64_t)p->B * p->H * a.own_split;
  a.prefix_units = x ? (int64_t)groups * p->H * a.prefix_split : 0;
  a.own_slots = up(a.own_units, 8) * a.own_blocks;
  a.prefix_slots = up(a.prefix_units, 8) * a.prefix_blocks;
  a.direct = !x && a.own_split == 1;
  const size_t slots = a.direct ? 0 : (size_t)a.rows * (a.own_split + a.prefix_split);
  a.ml = align_up(slots * p->D * sizeof(float));
  a.total = a.ml + align_up(std::max<size_t>(slots * sizeof(float2), 1));
  return a;
}

inline int check_planned(const Plan& a) {
  if (a.rows >= (int64_t)1 << 26) return fail_status(NACL_ERR_UNSUPPORTED, "B * H * q_group * T reaches 2^26");
  if (8 * (a.own_slots + a.prefix_slots) >= (int64_t)1 << 24)
    return fail_status(NACL_ERR_UNSUPPORTED, "%lld work-groups, at most 2^24", (long long)(8 * (a.own_slots + a.prefix_slots)));
  return NACL_OK;
}

inline int check_workspace(const void* ws, size_t ws_bytes, size_t need) {
  if (ws_bytes < need) return fail_status(NACL_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
  if (!ws) return fail_status(NACL_ERR_WORKSPACE, "workspace is NULL");
  if (!aligned(ws, kAlign)) return fail_status(NACL_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return NACL_OK;
}

// The table of a paged cache (not whether it is there).
inline int check_pages(const nacl_problem* p, const nacl_pages* x) {
  if (!x) return fail_status(NACL_ERR_INVALID_ARG, "pages are NULL");
  if (x->n_pages < 1 || x->page < 1 || x->entries < 1)
    return fail_status(NACL_ERR_INVALID_ARG, "n_pages, page and entries must be >= 1 (got %d, %d, %d)", x->n_pages, x->page, x->entries);
  if (x->entries > 1 << 20) return fail_status(NACL_ERR_UNSUPPORTED, "entries = %d exceeds 2^20", x->entries);
  if ((int64_t)x->n_pages * x->page >= (int64_t)1 << 31)
    return fail_status(NACL_ERR_UNSUPPORTED, "n_pages * page reaches 2^31");
  if (x->table_stride < x->entries) return fail_status(NACL_ERR_INVALID_ARG, "table_stride must be at least entries");
  if (x->table_stride > ((int64_t)1 << 32)) return fail_status(NACL_ERR_UNSUPPORTED, "table_stride exceeds 2^32");
  return aligned(x->table, 4) ? (int)NACL_OK : fail_status(NACL_ERR_INVALID_ARG, "the table must be 4-byte aligned");
}

// Its pools.
inline int check_pool(const nacl_problem* p, const nacl_pages* x) {
  const int eb = elt_bytes(p->dtype);
  if (!x->k || !x->v) return fail_status(NACL_ERR_INVALID_ARG, "the pages' k and v must be non-NULL");
  if (!aligned(x->k, 16) || !aligned(x->v, 16)) return fail_status(NACL_ERR_INVALID_ARG, "the pages' k and v must be 16-byte aligned");
  if (int st = check_strides("the pages' k_stride", x->k_stride, eb)) return st;
  if (int st = check_strides("the pages' v_stride", x->v_stride, eb)) return st;
  if (std::max(x->k_stride[0], x->v_stride[0]) > ((int64_t)1 << 56) / x->n_pages)
    return fail_status(NACL_ERR_UNSUPPORTED, "the pools span more than 2^56 elements");
  return NACL_OK;
}
inline Extent pool_extent(const nacl_problem* p, const nacl_pages* x, const void* base, const int64_t st[3]) {
  return Extent(base, st, x->n_pages, p->H, x->page, p->D, elt_bytes(p->dtype));
}

// That no two rows of the pools, which are written, lie at one place.
inline int check_pool_apart(const nacl_problem* p, const nacl_pages* x) {
  const int eb = elt_bytes(p->dtype);
  const bool same = std::equal(x->k_stride, x->k_stride + 3, x->v_stride);
  const uintptr_t k = (uintptr_t)x->k, v = (uintptr_t)x->v;
  const int64_t gap = (int64_t)((k < v ? v - k : k - v) / eb);
  bool apart = !pool_extent(p, x, x->k, x->k_stride).meets(pool_extent(p, x, x->v, x->v_stride));
  for (const int64_t* st : {x->k_stride, x->v_stride}) {
    // From the innermost dimension on, each steps over what those inside it span; K
    // and V of one buffer lie apart where V's span fits beside K's into a step.
    std::pair<int64_t, int64_t> dims[3] = {{st[0], x->n_pages}, {st[1], p->H}, {st[2], x->page}};
    std::sort(dims, dims + 3);
    int64_t span = p->D;
    for (const auto& [step, n] : dims) {
      if (n == 1) continue;
      if (step < span) return fail_status(NACL_ERR_INVALID_ARG, "rows of the pools overlap");
      apart = apart || (same && gap >= span && gap + span <= step);
      span += (n - 1) * step;
    }
  }
  return apart ? (int)NACL_OK : fail_status(NACL_ERR_INVALID_ARG, "K and V overlap");
}

inline int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? (int)NACL_OK : fail_status(NACL_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace nacl
