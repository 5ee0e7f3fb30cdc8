// C ABI of decoding over a paged cache and of beam search: argument validation and
// the launches (nacl_paged_append is beside nacl_rotate_append).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>

#include "../../include/nacl.h"
#include "internal.h"
#include "step_common.h"

namespace {

using namespace nacl;

// How a step's attention over pages is shared out, by sizes alone: blocks of rows
// as for own caches, and splits that take a sequence's blocks of keys in turn, so that all
// of them are at work however short the sequence is beside its table.
struct PagedPlan {
  int L = 0, rows = 16, blocks = 0, split = 0;
  int64_t units = 0, slots = 0, all_rows = 0;
  bool direct = false;
  size_t ml = 0, total = 0;  // byte offset of part_ml, workspace bytes
};
PagedPlan paged_plan(const nacl_problem* p, const nacl_step* s, const nacl_pages* x) {
  PagedPlan a;
  const int G = q_group_of(p);
  a.L = (int)std::min<int64_t>(p->L, (int64_t)x->entries * x->page);
  const int64_t own = (int64_t)G * s->T;
  a.all_rows = (int64_t)p->B * p->H * own;
  // Up to 128 rows by 32, whose blocks read the same keys one after the other on one
  // XCD (64 rows, 8 heads, 16000 keys: 25.7 us, as half a tile of 128 rows 27.4; 128 rows,
  // 8000 keys: 24.8 and 26.6; but 32000 keys 52.7 and 44.1).
  a.rows = own <= 16 ? 16 : own <= kPrefixTileRows || p->dtype == NACL_F32 ? 32 : kPrefixTileRows;
  auto up = [](int64_t n, int64_t d) { return (n + d - 1) / d; };
  a.blocks = (int)up(own, a.rows);
  const int64_t keys = (int64_t)p->B * p->H * a.blocks * a.L;
  // Six work-groups of 16 rows per CU if every sequence were as long as its table, two rounds
  // of the three that run together (calls of 32 caches of up to 8256 rows, the mean over
  // lengths: 138 us, three 140, five 140; of 3 caches of up to 131072 rows 228, 219, 238; of 32
  // with lengths from 0 on 122, 127, 124), two of more (4 caches of 8000 rows, 32 rows: 31.7
  // us, three 35, four 38; 512 tokens of 32 heads over 8192 rows 106, 121, 117).
  const int per_cu = a.rows == 16 ? 6 : 2;
  const int64_t chunk = std::max<int64_t>(kPrefixMinChunk, up(keys, per_cu * kPlanCus));
  a.split = (int)up(a.L, up(chunk, kPrefixMinChunk) * kPrefixMinChunk);
  a.units = (int64_t)p->B * p->H * a.split;
  a.slots = up(a.units, 8) * a.blocks;
  a.direct = a.split == 1;
  const size_t parts = a.direct ? 0 : (size_t)a.all_rows * a.split;
  a.ml = align_up(parts * p->D * sizeof(float));
  a.total = a.ml + align_up(std::max<size_t>(parts * sizeof(float2), 1));
  return a;
}
int check_planned(const PagedPlan& a) {
  if (a.all_rows >= (int64_t)1 << 26) return fail_status(NACL_ERR_UNSUPPORTED, "B * H * q_group * T reaches 2^26");
  if (8 * a.slots >= (int64_t)1 << 24)
    return fail_status(NACL_ERR_UNSUPPORTED, "%lld work-groups, at most 2^24", (long long)(8 * a.slots));
  return NACL_OK;
}

// Whether one of the written extents meets another or one of those read.
bool overlap(std::initializer_list<Extent> written, std::initializer_list<Extent> read) {
  for (const Extent* a = written.begin(); a != written.end(); ++a) {
    if (a->lo == a->hi) continue;
    for (const Extent* b = written.begin(); b != a; ++b)
      if (b->lo != b->hi && a->meets(*b)) return true;
    for (const Extent& b : read)
      if (b.lo != b.hi && a->meets(b)) return true;
  }
  return false;
}
// n int32 or fp32 numbers (none where there is no array).
Extent words(const void* base, int64_t n) { return Extent(base, base ? (uintptr_t)n * 4 : 0); }
Extent table_extent(const void* base, int64_t stride, int64_t B, int64_t entries) {
  return words(base, (B - 1) * stride + entries);
}

// Small slices where large ones leave compute units without one and the small ones'
// lists are still a few (4 beams of 32000 tokens: the kernels 4.7 + 4.6 us, by large ones
// 6.2 + 4.2; 8 of 131072, whose small slices are 512: 5.7 + 9.4 and 6.8 + 6.7).
int beam_slice(const nacl_beams* d) {
  auto slices = [&](int n) { return ((int64_t)d->V + n - 1) / n; };
  const bool small = d->B * d->W * slices(kBeamSlice) < kPlanCus && d->W * slices(kBeamSmallSlice) <= kBeamLists / 4;
  return small ? kBeamSmallSlice : kBeamSlice;
}
int beam_slices(const nacl_beams* d) { return (d->V + beam_slice(d) - 1) / beam_slice(d); }

int check_beams(const nacl_beams* d) {
  if (!d) return fail_status(NACL_ERR_INVALID_ARG, "beams are NULL");
  if (d->B < 1 || d->W < 1 || d->V < 1 || d->K < 1)
    return fail_status(NACL_ERR_INVALID_ARG, "B, W, V and K must be >= 1 (got %d, %d, %d, %d)", d->B, d->W, d->V, d->K);
  if (d->W > NACL_MAX_W || d->K > NACL_MAX_W) return fail_status(NACL_ERR_UNSUPPORTED, "W or K exceeds %d", NACL_MAX_W);
  if ((int64_t)d->B * d->W > 65535) return fail_status(NACL_ERR_UNSUPPORTED, "B * W exceeds 65535");
  if (d->V > NACL_MAX_V) return fail_status(NACL_ERR_UNSUPPORTED, "V = %d exceeds %d", d->V, NACL_MAX_V);
  if ((int64_t)d->W * beam_slices(d) > kBeamLists)
    return fail_status(NACL_ERR_UNSUPPORTED, "a group of %d beams of %d slices, at most %d in all", d->W, beam_slices(d), kBeamLists);
  if (d->dtype != NACL_F32 && d->dtype != NACL_BF16) return fail_status(NACL_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
  if (d->stride < d->V) return fail_status(NACL_ERR_INVALID_ARG, "the row stride must be at least V");
  if (d->stride > ((int64_t)1 << 40)) return fail_status(NACL_ERR_UNSUPPORTED, "the row stride exceeds 2^40");
  if (d->ended && (d->end_token < 0 || d->end_token >= d->V))
    return fail_status(NACL_ERR_INVALID_ARG, "end_token must lie in [0, V) (got %d)", d->end_token);
  if (!aligned(d->ended, 4)) return fail_status(NACL_ERR_INVALID_ARG, "ended must be 4-byte aligned");
  return NACL_OK;
}
size_t beam_key_bytes(const nacl_beams* d) {
  return align_up((size_t)d->B * d->W * beam_slices(d) * d->K * sizeof(uint64_t));
}

}  // namespace

extern "C" {

int nacl_pages_assign(const nacl_problem* p, const nacl_step* s, const nacl_pages* x, const int32_t* held,
                      const int32_t* shared, int32_t* free, const int32_t* n_free, int32_t* held_out,
                      int32_t* n_free_out, int32_t* slots, int32_t* missing, void* stream) {
  nacl::clear_detail();
  int st = check_step(p, s);
  if (st) return st;
  if ((st = check_pages(p, x))) return st;
  if (!x->table || !held || !free || !n_free || !held_out || !n_free_out || !slots)
    return fail_status(NACL_ERR_INVALID_ARG, "table, held, free, n_free, held_out, n_free_out and slots must be non-NULL");
  for (const void* t : {(const void*)held, (const void*)shared, (const void*)free, (const void*)n_free, (const void*)held_out,
                        (const void*)n_free_out, (const void*)slots, (const void*)missing})
    if (!aligned(t, 4)) return fail_status(NACL_ERR_INVALID_ARG, "arrays must be 4-byte aligned");
  const int64_t B = p->B;
  if (overlap({table_extent(x->table, x->table_stride, B, x->entries), words(free, x->n_pages), words(held_out, B),
               words(n_free_out, 1), words(slots, B * s->T), words(missing, 1)},
              {words(s->lens, B), words(s->n_new, B), words(shared, B), words(held == held_out ? nullptr : held, B),
               words(n_free == n_free_out ? nullptr : n_free, 1)}))
    return fail_status(NACL_ERR_INVALID_ARG, "what is written overlaps an input or another output");
  nacl::AssignLaunch a{};
  a.B = p->B;
  a.T = s->T;
  a.L = p->L;
  a.row0 = s->row0;
  a.page = x->page;
  a.n_pages = x->n_pages;
  a.entries = x->entries;
  a.table_stride = x->table_stride;
  a.lens = s->lens;
  a.n_new = s->n_new;
  a.shared = shared;
  a.held = held;
  a.n_free = n_free;
  a.table = x->table;
  a.free = free;
  a.held_out = held_out;
  a.n_free_out = n_free_out;
  a.slots = slots;
  a.missing = missing;
  return launched(nacl::launch_assign(a, kPlanCus, static_cast<hipStream_t>(stream)), "page kernels");
}

size_t nacl_paged_workspace_bytes(const nacl_problem* p, const nacl_step* s, const nacl_pages* x) {
  nacl::clear_detail();
  if (check_step(p, s) != NACL_OK || check_pages(p, x) != NACL_OK) return 0;
  const PagedPlan a = paged_plan(p, s, x);
  return check_planned(a) == NACL_OK ? a.total : 0;
}

int nacl_paged_attention(const nacl_problem* p, const nacl_step* s, const nacl_pages* x, const void* q, void* out,
                         float* lse, void* ws, size_t ws_bytes, void* stream) {
  nacl::clear_detail();
  int st = check_step(p, s);
  if (st) return st;
  if ((st = check_pages(p, x)) || (st = check_pool(p, x))) return st;
  const int eb = elt_bytes(p->dtype), G = q_group_of(p);
  if (!q || !out || !x->table) return fail_status(NACL_ERR_INVALID_ARG, "q, out and the table must be non-NULL");
  if (!aligned(q, 16) || !aligned(out, 16)) return fail_status(NACL_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
  if (!aligned(lse, 4)) return fail_status(NACL_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  const PagedPlan plan = paged_plan(p, s, x);
  if ((st = check_planned(plan))) return st;
  if ((st = check_workspace(ws, ws_bytes, plan.total))) return st;
  if (overlap({Extent(out, (uintptr_t)plan.all_rows * p->D * eb), words(lse, plan.all_rows), Extent(ws, plan.total)},
              {Extent(q, s->q_stride, p->B, p->H * G, s->T, p->D, eb), pool_extent(p, x, x->k, x->k_stride),
               pool_extent(p, x, x->v, x->v_stride), table_extent(x->table, x->table_stride, p->B, x->entries),
               words(s->lens, p->B), words(s->n_new, p->B)}))
    return fail_status(NACL_ERR_INVALID_ARG, "out, lse or the workspace overlap an input or each other");
  nacl::PrefixLaunch a{};
  a.B = p->B;
  a.H = p->H;
  a.G = G;
  a.T = s->T;
  a.L = plan.L;
  a.row0 = s->row0;
  a.per_group = p->B;
  a.own_rows = plan.rows;
  a.own_blocks = plan.blocks;
  a.own_split = plan.split;
  a.own_units = (int)plan.units;
  a.own_slots = (int)plan.slots;
  a.direct = plan.direct ? 1 : 0;
  a.c2 = (float)((double)p->sm_scale * 1.4426950408889634);
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = s->q_stride[i];
    a.ks[i] = x->k_stride[i];
    a.vs[i] = x->v_stride[i];
  }
  a.lens = s->lens;
  a.n_new = s->n_new;
  a.q = q;
  a.k = x->k;
  a.v = x->v;
  a.out = out;
  a.lse = lse;
  a.part_o = reinterpret_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + plan.ml);
  a.table = x->table;
  a.table_stride = x->table_stride;
  a.page = x->page;
  a.n_pages = x->n_pages;
  a.page_inv = ~0u / (uint32_t)x->page;
  auto span = [&](const int64_t st[3]) { return ((x->n_pages - 1) * st[0] + (x->page - 1) * st[2] + p->D) * eb; };
  a.near = std::max(span(x->k_stride), span(x->v_stride)) <= kPagedNearBytes;
  return launched(nacl::launch_paged(a, p->dtype, p->D, static_cast<hipStream_t>(stream)), "paged attention kernels");
}

size_t nacl_beam_workspace_bytes(const nacl_beams* d) {
  nacl::clear_detail();
  if (check_beams(d) != NACL_OK) return 0;
  return beam_key_bytes(d) + align_up((size_t)d->B * d->W * beam_slices(d) * 2 * sizeof(double));
}

int nacl_beam_select(const nacl_beams* d, const void* logits, const float* scores, int32_t* parents,
                     int32_t* tokens, float* out, void* ws, size_t ws_bytes, void* stream) {
  nacl::clear_detail();
  int st = check_beams(d);
  if (st) return st;
  if (!logits || !scores || !parents || !tokens || !out)
    return fail_status(NACL_ERR_INVALID_ARG, "logits, scores, parents, tokens and out must be non-NULL");
  const int eb = elt_bytes(d->dtype);
  if (!aligned(logits, eb) || !aligned(scores, 4) || !aligned(parents, 4) || !aligned(tokens, 4) || !aligned(out, 4))
    return fail_status(NACL_ERR_INVALID_ARG, "logits must be aligned to their elements, the other arrays to 4 bytes");
  const size_t need = nacl_beam_workspace_bytes(d);
  if ((st = check_workspace(ws, ws_bytes, need))) return st;
  const int64_t rows = (int64_t)d->B * d->W, n = (int64_t)d->B * d->K;
  if (overlap({words(parents, n), words(tokens, n), words(out, n), Extent(ws, need)},
              {Extent(logits, (uintptr_t)((rows - 1) * d->stride + d->V) * eb), words(scores, rows), words(d->ended, rows)}))
    return fail_status(NACL_ERR_INVALID_ARG, "parents, tokens, out or the workspace overlap an input or each other");
  nacl::BeamLaunch a{};
  a.B = d->B;
  a.W = d->W;
  a.V = d->V;
  a.K = d->K;
  a.slice = beam_slice(d);
  a.S = beam_slices(d);
  a.stride = d->stride;
  a.logits = logits;
  a.scores = scores;
  a.ended = d->ended;
  a.end_token = d->ended ? d->end_token : 0;
  a.parents = parents;
  a.tokens = tokens;
  a.out = out;
  a.keys = reinterpret_cast<uint64_t*>(ws);
  a.sums = reinterpret_cast<double*>(static_cast<char*>(ws) + beam_key_bytes(d));
  return launched(nacl::launch_beam(a, d->dtype, static_cast<hipStream_t>(stream)), "beam kernels");
}

int nacl_beam_reorder(const nacl_problem* p, const nacl_pages* x, int32_t W, const int32_t* parents,
                      const int32_t* lens, const int32_t* held, int32_t* table_out, int64_t out_stride,
                      int32_t* lens_out, int32_t* held_out, void* stream) {
  nacl::clear_detail();
  int st = validate_problem(p);
  if (st) return st;
  if ((st = check_pages(p, x)) || (st = check_pool(p, x)) || (st = check_pool_apart(p, x))) return st;
  if (W < 1 || p->B % W) return fail_status(NACL_ERR_INVALID_ARG, "the beams W must divide B = %d (got %d)", p->B, W);
  if (W > NACL_MAX_W) return fail_status(NACL_ERR_UNSUPPORTED, "W = %d exceeds %d", W, NACL_MAX_W);
  if (out_stride < x->entries) return fail_status(NACL_ERR_INVALID_ARG, "out_stride must be at least entries");
  if (out_stride > ((int64_t)1 << 32)) return fail_status(NACL_ERR_UNSUPPORTED, "out_stride exceeds 2^32");
  if (!x->table || !parents || !lens || !table_out || !lens_out)
    return fail_status(NACL_ERR_INVALID_ARG, "the table, parents, lens, table_out and lens_out must be non-NULL");
  if (!held != !held_out) return fail_status(NACL_ERR_INVALID_ARG, "held and held_out are given together");
  for (const void* t : {(const void*)parents, (const void*)lens, (const void*)held, (const void*)table_out, (const void*)lens_out,
                        (const void*)held_out})
    if (!aligned(t, 4)) return fail_status(NACL_ERR_INVALID_ARG, "arrays must be 4-byte aligned");
  const int64_t B = p->B;
  const Extent kc = pool_extent(p, x, x->k, x->k_stride), vc = pool_extent(p, x, x->v, x->v_stride);
  const std::initializer_list<Extent> read = {table_extent(x->table, x->table_stride, B, x->entries), words(parents, B),
                                              words(lens, B), words(held, B)};
  const Extent to = table_extent(table_out, out_stride, B, x->entries);
  // (The pools may be interleaved, which check_pool_apart looks at.)
  if (overlap({to, words(lens_out, B), words(held_out, B), kc}, read) ||
      overlap({to, words(lens_out, B), words(held_out, B), vc}, read))
    return fail_status(NACL_ERR_INVALID_ARG, "what is written overlaps an input or another output");
  nacl::ReorderLaunch a{};
  a.groups = p->B / W;
  a.W = W;
  a.H = p->H;
  a.L = p->L;
  a.page = x->page;
  a.n_pages = x->n_pages;
  a.entries = x->entries;
  a.table_stride = x->table_stride;
  a.out_stride = out_stride;
  for (int i = 0; i < 3; ++i) {
    a.ks[i] = x->k_stride[i];
    a.vs[i] = x->v_stride[i];
  }
  a.table = x->table;
  a.parents = parents;
  a.lens = lens;
  a.held = held;
  a.table_out = table_out;
  a.lens_out = lens_out;
  a.held_out = held_out;
  a.k = x->k;
  a.v = x->v;
  return launched(nacl::launch_reorder(a, p->dtype, p->D, kPlanCus, static_cast<hipStream_t>(stream)), "reorder kernel");
}

}  // extern "C"
