// C ABI of the decoding step between two evictions: argument validation,
// the attention's plan and workspace, and the launches.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/nacl.h"
#include "internal.h"

namespace {

using nacl::fail_status;

constexpr int kPlanCus = 256;  // compute units the launches are planned for
constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int elt_bytes(int dtype) { return dtype == NACL_F32 ? 4 : 2; }
int q_group_of(const nacl_problem* p) { return p->q_group > 1 ? p->q_group : 1; }

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

int check_strides(const char* name, const int64_t st[3], int eb) {
  for (int i = 0; i < 3; ++i) {
    if (st[i] < 0) return fail_status(NACL_ERR_INVALID_ARG, "%s[%d] < 0", name, i);
    if (st[i] > ((int64_t)1 << 40)) return fail_status(NACL_ERR_UNSUPPORTED, "%s[%d] exceeds 2^40", name, i);
    if ((st[i] * eb) % 16)
      return fail_status(NACL_ERR_INVALID_ARG, "%s[%d] * element size must be a multiple of 16 bytes", name, i);
  }
  return NACL_OK;
}

// The problem and the parts of a step that both calls read.
int check_step(const nacl_problem* p, const nacl_step* s) {
  int st = nacl::validate_problem(p);
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

int check_prefix(const nacl_problem* p, const nacl_prefix* x) {
  if (!x) return NACL_OK;
  if (x->G < 1 || p->B % x->G)
    return fail_status(NACL_ERR_INVALID_ARG, "the prefix's groups must divide B = %d (got %d)", p->B, x->G);
  if (x->L < 1) return fail_status(NACL_ERR_INVALID_ARG, "the prefix's L must be >= 1 (got %d)", x->L);
  if (x->L > NACL_MAX_L) return fail_status(NACL_ERR_UNSUPPORTED, "the prefix's L = %d exceeds %d", x->L, NACL_MAX_L);
  const int eb = elt_bytes(p->dtype);
  if (int st = check_strides("the prefix's k_stride", x->k_stride, eb)) return st;
  return check_strides("the prefix's v_stride", x->v_stride, eb);
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

Plan plan_of(const nacl_problem* p, const nacl_step* s, const nacl_prefix* x) {
  Plan a;
  const int G = q_group_of(p);
  const int groups = x ? x->G : 1;
  a.per_group = p->B / groups;
  a.Lp = x ? x->L : 0;
  a.rows = (int64_t)p->B * p->H * G * s->T;
  const int64_t own_rows = (int64_t)G * s->T, prefix_rows = own_rows * a.per_group;
  auto block = [&](int64_t rows) {
    return rows <= 16 ? 16 : rows <= 32 || p->dtype == NACL_F32 ? 32 : nacl::kPrefixTileRows;
  };
  a.own_rows = block(own_rows);
  a.prefix_rows = x ? block(prefix_rows) : a.own_rows;
  // Of a prefix 256 rows share a tile where there are as many: half the reads per
  // row (8 heads, 26214 keys: 512 rows 89 us, by tiles of 128 97, 2048 rows 246 and
  // 271, 256 rows 54 and 58, 160 rows 43 and 48).  Not of the own caches, whose work-groups are fewer (4 caches of
  // 4096 rows, 8 heads, 256 rows: 54 us, by 256 rows 83).
  if (x && a.prefix_rows == nacl::kPrefixTileRows && prefix_rows > nacl::kPrefixTileRows) a.prefix_rows = nacl::kPrefixWideRows;
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
  const bool tiles = x && a.prefix_rows >= nacl::kPrefixTileRows;
  const int64_t own_keys = own_blocks * p->L, prefix_keys = prefix_blocks * a.Lp;
  const int64_t keys = own_keys + (tiles ? 0 : prefix_keys);
  const bool mostly_prefix = !tiles && p->dtype == NACL_BF16 && prefix_keys >= own_keys;
  const int per_cu = a.own_rows == nacl::kPrefixTileRows ? 4 : mostly_prefix ? 1 : tiles || a.own_rows == 32 || a.prefix_rows == 32 ? 2 : 3;
  const int64_t chunk = std::max<int64_t>(nacl::kPrefixMinChunk, up(keys, per_cu * kPlanCus));
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

int check_planned(const Plan& a) {
  if (a.rows >= (int64_t)1 << 26) return fail_status(NACL_ERR_UNSUPPORTED, "B * H * q_group * T reaches 2^26");
  if (8 * (a.own_slots + a.prefix_slots) >= (int64_t)1 << 24)
    return fail_status(NACL_ERR_UNSUPPORTED, "%lld work-groups, at most 2^24", (long long)(8 * (a.own_slots + a.prefix_slots)));
  return NACL_OK;
}

int check_draw(const nacl_draw* d) {
  if (!d) return fail_status(NACL_ERR_INVALID_ARG, "settings are NULL");
  if (d->N < 1 || d->V < 1) return fail_status(NACL_ERR_INVALID_ARG, "N and V must be >= 1 (got %d, %d)", d->N, d->V);
  if (d->N > 65535) return fail_status(NACL_ERR_UNSUPPORTED, "N = %d exceeds 65535", d->N);
  if (d->V > NACL_MAX_V) return fail_status(NACL_ERR_UNSUPPORTED, "V = %d exceeds %d", d->V, NACL_MAX_V);
  if (d->dtype != NACL_F32 && d->dtype != NACL_BF16) return fail_status(NACL_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
  if (d->stride < d->V) return fail_status(NACL_ERR_INVALID_ARG, "the row stride must be at least V");
  if (d->stride > ((int64_t)1 << 40)) return fail_status(NACL_ERR_UNSUPPORTED, "the row stride exceeds 2^40");
  if (!aligned(d->temperature, 4) || !aligned(d->top_k, 4) || !aligned(d->top_p, 4) || !aligned(d->min_p, 4))
    return fail_status(NACL_ERR_INVALID_ARG, "the settings' arrays must be 4-byte aligned");
  return NACL_OK;
}

int check_workspace(const void* ws, size_t ws_bytes, size_t need) {
  if (ws_bytes < need) return fail_status(NACL_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", ws_bytes, need);
  if (!ws) return fail_status(NACL_ERR_WORKSPACE, "workspace is NULL");
  if (!aligned(ws, kAlign)) return fail_status(NACL_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return NACL_OK;
}

int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? (int)NACL_OK : fail_status(NACL_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace

extern "C" {

int nacl_rotate_append(const nacl_problem* p, const nacl_step* s, const nacl_rotation* r, const int32_t* positions,
                       const void* q_new, const void* k_new, const void* v_new, void* q_out, void* k, void* v,
                       void* stream) {
  nacl::clear_detail();
  int st = check_step(p, s);
  if (st) return st;
  const int eb = elt_bytes(p->dtype), G = q_group_of(p);
  if ((st = check_strides("the step's k_stride", s->k_stride, eb))) return st;
  if ((st = check_strides("the step's v_stride", s->v_stride, eb))) return st;
  if ((st = check_strides("the step's q_out_stride", s->q_out_stride, eb))) return st;
  if (!r) return fail_status(NACL_ERR_INVALID_ARG, "rotation is NULL");
  if (r->rot < 0 || r->rot > p->D) return fail_status(NACL_ERR_INVALID_ARG, "rot must lie in [0, D] (got %d)", r->rot);
  if (r->rot % 16) return fail_status(NACL_ERR_UNSUPPORTED, "rot must be a multiple of 16 (got %d)", r->rot);
  if (!(std::isfinite(r->eps) && r->eps >= 0.f)) return fail_status(NACL_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (r->pos_stride < 0 || (r->pos_stride > 0 && r->pos_stride < s->T))
    return fail_status(NACL_ERR_INVALID_ARG, "pos_stride must be 0 or at least T");
  if (r->rot && (!r->inv_freq || !positions))
    return fail_status(NACL_ERR_INVALID_ARG, "a rotation needs inv_freq and positions");
  if (!aligned(r->inv_freq, 4) || !aligned(positions, 4))
    return fail_status(NACL_ERR_INVALID_ARG, "inv_freq and positions must be 4-byte aligned");
  if (!q_new || !k_new || !v_new || !q_out || !k || !v)
    return fail_status(NACL_ERR_INVALID_ARG, "q_new, k_new, v_new, q_out, k and v must be non-NULL");
  for (const void* t : {q_new, k_new, v_new, (const void*)q_out, (const void*)k, (const void*)v, r->q_weight, r->k_weight})
    if (!aligned(t, 16)) return fail_status(NACL_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
  // What is written: q_out (or q_new itself), K and V.
  const int Hq = p->H * G;
  const Extent kc(k, p->k_stride, p->B, p->H, p->L, p->D, eb), vc(v, p->v_stride, p->B, p->H, p->L, p->D, eb);
  const Extent qn(q_new, s->q_stride, p->B, Hq, s->T, p->D, eb), kn(k_new, s->k_stride, p->B, p->H, s->T, p->D, eb);
  const Extent vn(v_new, s->v_stride, p->B, p->H, s->T, p->D, eb);
  const Extent qo(q_out, s->q_out_stride, p->B, Hq, s->T, p->D, eb);
  if (kc.meets(vc)) return fail_status(NACL_ERR_INVALID_ARG, "K and V overlap");
  for (const Extent* t : {&qn, &kn, &vn, &qo})
    if (t->meets(kc) || t->meets(vc)) return fail_status(NACL_ERR_INVALID_ARG, "the new tokens or q_out overlap the cache");
  const bool in_place = q_out == q_new;
  if (in_place) {
    if (q_new == k_new || q_new == v_new)
      return fail_status(NACL_ERR_INVALID_ARG, "in place (q_out == q_new), k_new and v_new must lie elsewhere");
    for (int i = 0; i < 3; ++i)
      if (s->q_out_stride[i] != s->q_stride[i])
        return fail_status(NACL_ERR_INVALID_ARG, "in place (q_out == q_new), q_out_stride must be q_stride");
  } else if (qo.meets(qn) || qo.meets(kn) || qo.meets(vn)) {
    return fail_status(NACL_ERR_INVALID_ARG, "q_out overlaps the new tokens");
  }
  // Rows of what is written lie apart.
  const int64_t dims[3] = {p->B, Hq, s->T};
  for (int i = 0; i < 3; ++i)
    if (dims[i] > 1 && s->q_out_stride[i] < p->D)
      return fail_status(NACL_ERR_INVALID_ARG, "q_out_stride[%d] must be at least D", i);
  const int64_t cache_dims[3] = {p->B, p->H, p->L};
  for (int i = 0; i < 3; ++i)
    if (cache_dims[i] > 1 && (p->k_stride[i] < p->D || p->v_stride[i] < p->D))
      return fail_status(NACL_ERR_INVALID_ARG, "K and V need strides of at least D (k_stride, v_stride [%d])", i);
  nacl::RotateLaunch a{};
  a.B = p->B;
  a.H = p->H;
  a.G = G;
  a.T = s->T;
  a.L = p->L;
  a.row0 = s->row0;
  a.rot = r->rot;
  a.interleaved = r->interleaved != 0;
  a.eps = r->eps;
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = s->q_stride[i];
    a.kns[i] = s->k_stride[i];
    a.vns[i] = s->v_stride[i];
    a.qos[i] = s->q_out_stride[i];
    a.ks[i] = p->k_stride[i];
    a.vs[i] = p->v_stride[i];
  }
  a.pos_stride = r->pos_stride;
  a.lens = s->lens;
  a.n_new = s->n_new;
  a.pos = positions;
  a.inv_freq = r->inv_freq;
  a.q_weight = r->q_weight;
  a.k_weight = r->k_weight;
  a.q = q_new;
  a.k_new = k_new;
  a.v_new = v_new;
  a.q_out = q_out;
  a.k = k;
  a.v = v;
  return launched(nacl::launch_rotate_append(a, p->dtype, p->D, kPlanCus, static_cast<hipStream_t>(stream)), "rotate kernel");
}

size_t nacl_prefix_workspace_bytes(const nacl_problem* p, const nacl_step* s, const nacl_prefix* x) {
  nacl::clear_detail();
  if (check_step(p, s) != NACL_OK || check_prefix(p, x) != NACL_OK) return 0;
  const Plan a = plan_of(p, s, x);
  return check_planned(a) == NACL_OK ? a.total : 0;
}

int nacl_prefix_attention(const nacl_problem* p, const nacl_step* s, const nacl_prefix* x, const void* q,
                          const void* k, const void* v, void* out, float* lse, void* ws, size_t ws_bytes,
                          void* stream) {
  nacl::clear_detail();
  int st = check_step(p, s);
  if (st) return st;
  if ((st = check_prefix(p, x))) return st;
  const int eb = elt_bytes(p->dtype), G = q_group_of(p);
  if (!q || !k || !v || !out) return fail_status(NACL_ERR_INVALID_ARG, "q, k, v and out must be non-NULL");
  if (x && (!x->k || !x->v)) return fail_status(NACL_ERR_INVALID_ARG, "the prefix's k and v must be non-NULL");
  for (const void* t : {q, k, v, (const void*)out, x ? x->k : nullptr, x ? x->v : nullptr})
    if (!aligned(t, 16)) return fail_status(NACL_ERR_INVALID_ARG, "q, k, v, out and the prefix must be 16-byte aligned");
  if (!aligned(lse, 4) || (x && !aligned(x->lens, 4)))
    return fail_status(NACL_ERR_INVALID_ARG, "lse and the prefix's lens must be 4-byte aligned");
  // A head's rows are addressed through buffer descriptors with 32-bit byte
  // offsets, up to 127 rows past the last: below 2^32 with these limits.
  const int64_t row_strides[4] = {p->k_stride[2], p->v_stride[2], x ? x->k_stride[2] : p->D, x ? x->v_stride[2] : p->D};
  for (int i = 0; i < 4; ++i) {
    const int64_t bytes = row_strides[i] * eb, n = i < 2 ? p->L : x ? x->L : 1;
    if (row_strides[i] < p->D) return fail_status(NACL_ERR_INVALID_ARG, "K and V need row strides of at least D");
    if (n * bytes >= (int64_t)1 << 31 || bytes >= (int64_t)1 << 24)
      return fail_status(NACL_ERR_UNSUPPORTED, "one head's rows span 2 GiB or more, or one row 16 MiB");
  }
  const Plan plan = plan_of(p, s, x);
  if ((st = check_planned(plan))) return st;
  if ((st = check_workspace(ws, ws_bytes, plan.total))) return st;
  const int64_t out_row[3] = {(int64_t)p->H * G * s->T * p->D, (int64_t)s->T * p->D, p->D};
  const Extent eo(out, out_row, p->B, p->H * G, s->T, p->D, eb), el(lse, lse ? (uintptr_t)plan.rows * 4 : 0);
  const Extent ew(ws, plan.total);
  const Extent in[3] = {Extent(q, s->q_stride, p->B, p->H * G, s->T, p->D, eb),
                        Extent(k, p->k_stride, p->B, p->H, p->L, p->D, eb),
                        Extent(v, p->v_stride, p->B, p->H, p->L, p->D, eb)};
  const Extent* written[3] = {&eo, &el, &ew};
  for (int i = 0; i < 3; ++i) {
    if (written[i]->lo == written[i]->hi) continue;
    bool bad = false;
    for (const Extent& t : in) bad = bad || written[i]->meets(t);
    if (x)
      bad = bad || written[i]->meets(Extent(x->k, x->k_stride, x->G, p->H, x->L, p->D, eb)) ||
            written[i]->meets(Extent(x->v, x->v_stride, x->G, p->H, x->L, p->D, eb));
    for (int j = 0; j < i; ++j) bad = bad || (written[j]->lo < written[j]->hi && written[i]->meets(*written[j]));
    if (bad) return fail_status(NACL_ERR_INVALID_ARG, "out, lse or the workspace overlap an input or each other");
  }
  nacl::PrefixLaunch a{};
  a.B = p->B;
  a.H = p->H;
  a.G = G;
  a.T = s->T;
  a.L = p->L;
  a.row0 = s->row0;
  a.Lp = plan.Lp;
  a.per_group = plan.per_group;
  a.prefix_rows = plan.prefix_rows;
  a.own_rows = plan.own_rows;
  a.prefix_blocks = plan.prefix_blocks;
  a.prefix_split = plan.prefix_split;
  a.prefix_units = (int)plan.prefix_units;
  a.prefix_slots = (int)plan.prefix_slots;
  a.own_blocks = plan.own_blocks;
  a.own_split = plan.own_split;
  a.own_units = (int)plan.own_units;
  a.own_slots = (int)plan.own_slots;
  a.direct = plan.direct ? 1 : 0;
  a.c2 = (float)((double)p->sm_scale * 1.4426950408889634);
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = s->q_stride[i];
    a.ks[i] = p->k_stride[i];
    a.vs[i] = p->v_stride[i];
    a.pks[i] = x ? x->k_stride[i] : 0;
    a.pvs[i] = x ? x->v_stride[i] : 0;
  }
  a.lens = s->lens;
  a.n_new = s->n_new;
  a.plens = x ? x->lens : nullptr;
  a.q = q;
  a.k = k;
  a.v = v;
  a.pk = x ? x->k : nullptr;
  a.pv = x ? x->v : nullptr;
  a.out = out;
  a.lse = lse;
  a.part_o = reinterpret_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + plan.ml);
  return launched(nacl::launch_prefix(a, p->dtype, p->D, static_cast<hipStream_t>(stream)), "prefix attention kernels");
}

size_t nacl_sample_workspace_bytes(const nacl_draw* d) {
  nacl::clear_detail();
  if (check_draw(d) != NACL_OK) return 0;
  return align_up(std::max<size_t>(nacl::sample_workspace(d->N, d->V), 1));
}

int nacl_sample(const nacl_draw* d, const void* logits, const float* u, int32_t* tokens, float* logprobs, void* ws,
                size_t ws_bytes, void* stream) {
  nacl::clear_detail();
  int st = check_draw(d);
  if (st) return st;
  if (!logits || !u || !tokens) return fail_status(NACL_ERR_INVALID_ARG, "logits, u and tokens must be non-NULL");
  const int eb = elt_bytes(d->dtype);
  if (!aligned(logits, eb) || !aligned(u, 4) || !aligned(tokens, 4) || !aligned(logprobs, 4))
    return fail_status(NACL_ERR_INVALID_ARG, "logits must be aligned to their elements, u, tokens and logprobs to 4 bytes");
  const size_t need = nacl_sample_workspace_bytes(d);
  if ((st = check_workspace(ws, ws_bytes, need))) return st;
  const uintptr_t n4 = (uintptr_t)d->N * 4;
  const Extent el(logits, ((uintptr_t)(d->N - 1) * d->stride + d->V) * eb), eu(u, n4);
  const Extent written[3] = {Extent(tokens, n4), Extent(logprobs, logprobs ? n4 : 0), Extent(ws, need)};
  const void* arrays[4] = {d->temperature, d->top_k, d->top_p, d->min_p};
  for (int i = 0; i < 3; ++i) {
    if (written[i].lo == written[i].hi) continue;
    bool bad = written[i].meets(el) || written[i].meets(eu);
    for (const void* t : arrays) bad = bad || (t && written[i].meets(Extent(t, n4)));
    for (int j = 0; j < i; ++j) bad = bad || (written[j].lo < written[j].hi && written[i].meets(written[j]));
    if (bad) return fail_status(NACL_ERR_INVALID_ARG, "tokens, logprobs or the workspace overlap an input or each other");
  }
  nacl::SampleLaunch a{};
  a.N = d->N;
  a.V = d->V;
  a.stride = d->stride;
  a.temperature = d->temperature;
  a.top_k = d->top_k;
  a.top_p = d->top_p;
  a.min_p = d->min_p;
  a.logits = logits;
  a.u = u;
  a.tokens = tokens;
  a.logprobs = logprobs;
  a.ws = ws;
  return launched(nacl::launch_sample(a, d->dtype, static_cast<hipStream_t>(stream)), "sample kernel");
}

}  // extern "C"
