// Page tables of a paged cache: pages for a step's new tokens and the slots that
// they take (nacl_pages_assign), and the tables and rows of beams that go on from
// other beams (nacl_beam_reorder).

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

// ---------------------------------------------------------------------------
// nacl_pages_assign.  One work-group takes the sequences 1024 at a time: the
// pages to give back and to take are counted per sequence, a scan over the
// sequences gives each its run of the stack, and the pages themselves are moved
// by all threads together, a thread finding its page's sequence in the scanned
// counts (a sequence that ended gives hundreds back, most take none).

constexpr int kAssignThreads = 1024;
constexpr int kAssignSlots = 16384;  // slots that the same launch writes

// The rows that sequence b holds before and after the step.
__device__ __forceinline__ int64_t rows_before(const AssignLaunch& a, int b) {
  return (int64_t)a.row0 + (a.lens ? a.lens[b] : 0);
}
__device__ __forceinline__ int new_of(const AssignLaunch& a, int b) {
  return a.n_new ? max(0, min(a.T, a.n_new[b])) : a.T;
}
__device__ __forceinline__ int pages_wanted(const AssignLaunch& a, int b) {
  int64_t rows = rows_before(a, b) + new_of(a, b);
  rows = rows < 0 ? 0 : rows > a.L ? a.L : rows;
  return (int)min((int64_t)a.entries, (rows + a.page - 1) / a.page);
}
__device__ __forceinline__ int pages_held(const AssignLaunch& a, int b) { return max(0, min(a.entries, a.held[b])); }

// The slot of token t of sequence b, whose pages are in place.
__device__ __forceinline__ int slot_of(const AssignLaunch& a, int b, int t) {
  const int64_t row = rows_before(a, b) + t;
  if (t >= new_of(a, b) || row < 0 || row >= a.L) return -1;
  const int entry = (int)row / a.page;
  if (entry >= a.held_out[b]) return -1;
  const int page = a.table[(int64_t)b * a.table_stride + entry];
  return (uint32_t)page < (uint32_t)a.n_pages ? page * a.page + (int)row % a.page : -1;
}

// Sums of x over the threads up to and with this one, and over all.
__device__ __forceinline__ int64_t scan(int64_t x, int64_t* waves, int64_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    const int64_t y = __shfl_up(x, i);
    if (lane >= i) x += y;
  }
  __syncthreads();  // the last call's sums are read
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  int64_t before = 0;
  all = 0;
  for (int i = 0; i < (int)(blockDim.x >> 6); ++i) {
    if (i < wave) before += waves[i];
    all += waves[i];
  }
  return x + before;
}

// The first of n ascending sums that exceeds i.
__device__ __forceinline__ int owner_of(const int64_t* sums, int n, int64_t i) {
  int lo = 0;
  for (int step = kAssignThreads / 2; step; step /= 2)
    if (lo + step <= n && sums[lo + step - 1] <= i) lo += step;
  return lo;
}

__global__ __launch_bounds__(kAssignThreads) void assign_kernel(AssignLaunch a, int with_slots) {
  __shared__ int64_t sums[kAssignThreads], waves[kAssignThreads / 64];
  __shared__ int first[kAssignThreads];  // of each sequence's entries that change hands
  __shared__ int64_t granted_all;
  const int tid = threadIdx.x;
  const int64_t in_stack = max(0, min(a.n_pages, a.n_free[0]));

  // Pages back to the stack: entries [max(wanted, shared), held).
  int64_t given = 0;
  for (int b0 = 0; b0 < a.B; b0 += kAssignThreads) {
    const int b = b0 + tid, n = min(kAssignThreads, a.B - b0);
    int gives = 0, from = 0;
    if (tid < n) {
      from = max(pages_wanted(a, b), a.shared ? a.shared[b] : 0);
      gives = max(0, pages_held(a, b) - from);
    }
    int64_t all;
    const int64_t upto = scan(gives, waves, all);
    sums[tid] = upto;
    first[tid] = from;
    __syncthreads();
    for (int64_t i = tid; i < all; i += kAssignThreads) {
      const int s = owner_of(sums, n, i);
      const int entry = first[s] + (int)(i - (s ? sums[s - 1] : 0));
      const int64_t at = in_stack + given + i;
      if (at < a.n_pages) a.free[at] = a.table[(int64_t)(b0 + s) * a.table_stride + entry];
    }
    given += all;
    __syncthreads();
  }
  const int64_t stack = min((int64_t)a.n_pages, in_stack + given);

  // Pages off the stack's top, as long as it lasts: entries [held, wanted).
  int64_t asked = 0, taken = 0;
  for (int b0 = 0; b0 < a.B; b0 += kAssignThreads) {
    const int b = b0 + tid, n = min(kAssignThreads, a.B - b0);
    int takes = 0, held = 0, wanted = 0;
    if (tid < n) {
      wanted = pages_wanted(a, b);
      held = pages_held(a, b);
      takes = max(0, wanted - held);
    }
    int64_t all;
    const int64_t upto = scan(takes, waves, all);
    const bool granted = asked + upto <= stack;
    sums[tid] = upto;
    first[tid] = held;
    if (tid == 0) granted_all = 0;
    __syncthreads();
    // (Sums rise, so those who get theirs come first: the last of them has all.)
    const bool next_granted = tid + 1 < n && asked + sums[tid + 1] <= stack;
    if (tid < n && granted && !next_granted) granted_all = upto;
    if (tid < n) a.held_out[b] = takes && !granted ? held : wanted;
    __syncthreads();
    for (int64_t i = tid; i < granted_all; i += kAssignThreads) {
      const int s = owner_of(sums, n, i);
      const int entry = first[s] + (int)(i - (s ? sums[s - 1] : 0));
      a.table[(int64_t)(b0 + s) * a.table_stride + entry] = a.free[stack - 1 - taken - i];
    }
    asked += all;
    taken += granted_all;
    __syncthreads();
  }
  if (tid == 0) {
    a.n_free_out[0] = (int)(stack - taken);
    if (a.missing) a.missing[0] = (int)min((int64_t)INT32_MAX, max((int64_t)0, asked - stack));
  }
  if (with_slots)
    for (int i = tid; i < a.B * a.T; i += kAssignThreads) a.slots[i] = slot_of(a, i / a.T, i % a.T);
}

__global__ __launch_bounds__(256) void slots_kernel(AssignLaunch a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < (int64_t)a.B * a.T) a.slots[i] = slot_of(a, (int)(i / a.T), (int)(i % a.T));
}

// ---------------------------------------------------------------------------
// nacl_beam_reorder.  A wave works out its group: lane i is beam i.

constexpr int kReorderThreads = 256;

struct Beams {
  int parent;       // -1: none
  bool first;       // the first beam of its parent, whose pages it takes over
  int takes;        // the beam whose table row it takes
  uint64_t copies;  // the beams that copy rows: those after the first of a parent
};
__device__ __forceinline__ Beams beams_of(const ReorderLaunch& a, int group) {
  const int lane = threadIdx.x & 63;
  Beams x;
  x.parent = lane < a.W ? a.parents[(int64_t)group * a.W + lane] : -1;
  if ((uint32_t)x.parent >= (uint32_t)a.W) x.parent = -1;
  uint64_t has_child = 0, firsts = 0;
  for (int i = 0; i < a.W; ++i) {
    const int p = __builtin_amdgcn_readlane(x.parent, i);
    if (p >= 0 && !(has_child >> p & 1)) {
      has_child |= 1ull << p;
      firsts |= 1ull << i;
    }
  }
  const uint64_t all = a.W == 64 ? ~0ull : (1ull << a.W) - 1, below = (1ull << lane) - 1;
  x.first = firsts >> lane & 1;
  x.takes = x.parent;
  uint64_t spare = all & ~has_child;
  x.copies = __ballot(lane < a.W && !x.first && x.parent >= 0);
  if (!x.first && lane < a.W) {
    // The others take the rows of beams without a child, in order.
    for (int rank = __popcll(all & ~firsts & below); rank; --rank) spare &= spare - 1;
    x.takes = __ffsll((unsigned long long)spare) - 1;
  }
  return x;
}

// Strides are in 16-byte pieces here, of which a row has VEC.
template <int VEC>
__global__ __launch_bounds__(kReorderThreads) void reorder_kernel(ReorderLaunch a) {
  constexpr int kBatch = 4;  // pieces of K and of V that a thread has under way
  const int group = blockIdx.x / a.wgs, wg = blockIdx.x % a.wgs;
  const int lane = threadIdx.x & 63, base = group * a.W;
  const Beams x = beams_of(a, group);
  // Rows that the beam holds afterwards: its parent's, as far as its pages go.
  int len = 0;
  if (lane < a.W && x.parent >= 0) {
    const int held = a.held ? max(0, min(a.entries, a.held[base + x.takes])) : a.entries;
    len = (int)max((int64_t)0, min((int64_t)min(a.lens[base + x.parent], a.L), (int64_t)held * a.page));
  }
  // The tables.
  for (int i = wg; i < a.W; i += a.wgs) {
    const int32_t* from = a.table + (int64_t)(base + __builtin_amdgcn_readlane(x.takes, i)) * a.table_stride;
    int32_t* to = a.table_out + (int64_t)(base + i) * a.out_stride;
    for (int e = threadIdx.x; e < a.entries; e += kReorderThreads) to[e] = from[e];
    if ((int)threadIdx.x == i) {
      a.lens_out[base + i] = len;
      if (a.held_out) a.held_out[base + i] = a.held[base + x.takes];
    }
  }
  // The rows of those that copy: a page and a run of heads at a time.
  const int runs = (a.H + a.heads_per_item - 1) / a.heads_per_item;
  u32x4* k = reinterpret_cast<u32x4*>(a.k);
  u32x4* v = reinterpret_cast<u32x4*>(a.v);
  int item = wg;
  for (uint64_t left = x.copies; left; left &= left - 1) {
    const int i = __ffsll((unsigned long long)left) - 1;
    const int n = __builtin_amdgcn_readlane(len, i);
    const int32_t* to_row = a.table + (int64_t)(base + __builtin_amdgcn_readlane(x.takes, i)) * a.table_stride;
    const int32_t* of_row = a.table + (int64_t)(base + __builtin_amdgcn_readlane(x.parent, i)) * a.table_stride;
    const int items = (n + a.page - 1) / a.page * runs;
    for (; item < items; item += a.wgs) {
      const int e = item / runs, h0 = item % runs * a.heads_per_item;
      const int to = to_row[e], of = of_row[e];
      if (to == of || (uint32_t)to >= (uint32_t)a.n_pages || (uint32_t)of >= (uint32_t)a.n_pages) continue;
      const int rows = min(a.page, n - e * a.page), heads = min(a.heads_per_item, a.H - h0);
      const int pieces = heads * rows * VEC;
      for (int u0 = threadIdx.x; u0 < pieces; u0 += kBatch * kReorderThreads) {
        u32x4 kx[kBatch], vx[kBatch];
        int64_t ka[kBatch], va[kBatch];
#pragma unroll
        for (int c = 0; c < kBatch; ++c) {
          const int u = u0 + c * kReorderThreads;
          if (u >= pieces) break;
          const int y = u / VEC, h = h0 + y / rows, row = y % rows;
          ka[c] = h * a.ks[1] + row * a.ks[2] + u % VEC;
          va[c] = h * a.vs[1] + row * a.vs[2] + u % VEC;
          kx[c] = k[of * a.ks[0] + ka[c]];
          vx[c] = v[of * a.vs[0] + va[c]];
        }
#pragma unroll
        for (int c = 0; c < kBatch; ++c) {
          if (u0 + c * kReorderThreads >= pieces) break;
          k[to * a.ks[0] + ka[c]] = kx[c];
          v[to * a.vs[0] + va[c]] = vx[c];
        }
      }
    }
    item -= items;
  }
}

}  // namespace

hipError_t launch_assign(const AssignLaunch& a, hipStream_t stream) {
  const int64_t slots = (int64_t)a.B * a.T;
  const bool with_slots = slots <= kAssignSlots;
  assign_kernel<<<1, kAssignThreads, 0, stream>>>(a, with_slots);
  if (hipError_t e = hipGetLastError()) return e;
  if (!with_slots) slots_kernel<<<(unsigned)((slots + 255) / 256), 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_reorder(ReorderLaunch a, int dtype, int D, int cus, hipStream_t stream) {
  const int vec = D * (dtype == NACL_F32 ? 4 : 2) / 16;
  for (int i = 0; i < 3; ++i) {
    a.ks[i] = a.ks[i] * vec / D;
    a.vs[i] = a.vs[i] * vec / D;
  }
  // About 2048 pieces of K and of V per item.
  const int64_t per_head = (int64_t)a.page * vec;
  a.heads_per_item = (int)(per_head >= 2048 ? 1 : (2048 / per_head < a.H ? 2048 / per_head : a.H));
  const int64_t most = ((int64_t)a.entries * a.W) * ((a.H + a.heads_per_item - 1) / a.heads_per_item);
  int64_t wgs = (8 * cus + a.groups - 1) / a.groups;
  if (wgs > most) wgs = most;
  a.wgs = (int)wgs;
  const unsigned grid = (unsigned)(wgs * a.groups);
  if (vec == 8) reorder_kernel<8><<<grid, kReorderThreads, 0, stream>>>(a);
  else if (vec == 16) reorder_kernel<16><<<grid, kReorderThreads, 0, stream>>>(a);
  else reorder_kernel<32><<<grid, kReorderThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace nacl
