// Page tables of a paged cache: pages for a step's new tokens and the slots that
// they take (nacl_pages_assign), and the tables and rows of beams that go on from
// other beams (nacl_beam_reorder).

#include "device_common.h"
#include "internal.h"

namespace nacl {

namespace {

// ---------------------------------------------------------------------------
// nacl_pages_assign.  A thread per sequence counts the pages that it gives back or
// takes; a scan over the sequences gives each its run of the stack.  The pages are
// moved by all threads together, a thread finding its page's sequence in the
// scanned counts (a sequence that ended gives hundreds back, most take none).
// Latency bounds it, the lengths' loads, the scan, the pages' loads one after the other: 64
// sequences of one token 4.9 us, 256 that take up to 2048 tokens while 64 end (10000 pages,
// 524288 slots of 4 bytes) 9.6 us; in place, by one work-group and a second launch for the
// slots, 14.9 together.  1500 sequences of one token 15.5 us, 4000 of eight 28.8.

constexpr int kAssignSeqs = 1024;     // sequences of a work-group

// What sequence b holds before the step, what it is to get.
struct Sequence {
  int64_t rows;       // before
  int fresh;          // new tokens
  int held, wanted;   // pages
  int keeps;          // entries below do not go back
};
__device__ __forceinline__ Sequence sequence(const AssignLaunch& a, int b) {
  Sequence s;
  const int shared = a.shared ? a.shared[b] : 0, held = a.held[b];
  s.rows = (int64_t)a.row0 + (a.lens ? a.lens[b] : 0);
  s.fresh = a.n_new ? max(0, min(a.T, a.n_new[b])) : a.T;
  const int64_t after = max((int64_t)0, min(s.rows + s.fresh, (int64_t)a.L));
  s.wanted = (int)min((int64_t)a.entries, (after + a.page - 1) / a.page);
  s.held = max(0, min(a.entries, held));
  s.keeps = max(s.wanted, shared);
  return s;
}
__device__ __forceinline__ int stack_of(const AssignLaunch& a) { return max(0, min(a.n_pages, a.n_free[0])); }
__device__ __forceinline__ int in_pool(const AssignLaunch& a, int page, int row) {
  return (uint32_t)page < (uint32_t)a.n_pages ? page * a.page + row % a.page : -1;
}

// Sums over the wave's lanes up to and with this one.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return x;
}

// The first of n ascending sums that exceeds i.
template <int N>
__device__ __forceinline__ int owner_of(const int* sums, int n, int i) {
  int lo = 0;
  for (int step = N / 2; step; step /= 2)
    if (lo + step <= n && sums[lo + step - 1] <= i) lo += step;
  return lo;
}

// The sequences [b0, b0 + n) of a step, n at most N: their counts and scanned sums
// (of at most 1024 times 2^20 pages).
template <int N>
struct Counts {
  int gives[N], takes[N];  // sums up to and with each
  int first[N];            // entry of the first page that changes hands
  int waves[2][N / 64];
  int granted;             // sum of the takes that the stack has pages for

  // all_gives, all_takes: of all n; the caller has the threads meet before the sums
  // are read.
  __device__ __forceinline__ void count(const Sequence& s, int n, int& all_gives, int& all_takes) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int g = tid < n ? max(0, s.held - s.keeps) : 0, t = tid < n ? max(0, s.wanted - s.held) : 0;
    int gs = wave_scan(g), ts = wave_scan(t);
    if (lane == 63) {
      waves[0][wave] = gs;
      waves[1][wave] = ts;
    }
    if (tid == 0) granted = 0;
    __syncthreads();
    all_gives = all_takes = 0;
#pragma unroll
    for (int i = 0; i < N / 64; ++i) {
      const int x = waves[0][i], y = waves[1][i];
      gs += i < wave ? x : 0;
      ts += i < wave ? y : 0;
      all_gives += x;
      all_takes += y;
    }
    gives[tid] = gs;
    takes[tid] = ts;
    first[tid] = g ? s.keeps : s.held;
  }
  __device__ __forceinline__ int before(const int* sums, int i) const { return i ? sums[i - 1] : 0; }
};

// All sequences by one work-group (N threads, B <= N), or by several that all count
// and share the pages and the slots out.  What one of them reads, none writes: pages
// below the stack's top stay where they are in the stack, and those that came back
// are read where they came from.
template <int N>
__global__ __launch_bounds__(N) void assign_kernel(AssignLaunch a, int with_slots) {
  __shared__ Counts<N> c;
  __shared__ int64_t rows[N];
  __shared__ int fresh[N], held[N], held_after[N];
  const int tid = threadIdx.x;
  const int in_stack = stack_of(a);
  const Sequence s = sequence(a, min(tid, a.B - 1));
  int given, asked;
  c.count(s, a.B, given, asked);
  const int stack = (int)min((int64_t)a.n_pages, (int64_t)in_stack + given);
  const int upto = c.takes[tid];  // (the thread's own)
  const bool takes = s.wanted > s.held, granted = upto <= stack;
  const int after = takes && !granted ? s.held : s.wanted;
  // (The sums rise, so those that get theirs come first.)
  if (tid < a.B && takes && granted) atomicMax(&c.granted, upto);
  rows[tid] = s.rows;
  fresh[tid] = s.fresh;
  held[tid] = s.held;
  held_after[tid] = after;
  __syncthreads();
  // The stack's page at a place.
  auto page_at = [&](int place) {
    if (place < in_stack) return a.free[place];
    const int i = place - in_stack, b = owner_of<N>(c.gives, a.B, i);
    return a.table[(int64_t)b * a.table_stride + c.first[b] + i - c.before(c.gives, b)];
  };
  // The page of an entry of sequence b below held_after[b].
  auto page_of = [&](int b, int entry) {
    return entry < held[b] ? a.table[(int64_t)b * a.table_stride + entry]
                           : page_at(stack - 1 - (c.before(c.takes, b) + entry - held[b]));
  };
  const int wg = blockIdx.x, wgs = gridDim.x;
  if (wg == 0) {
    if (tid < a.B) a.held_out[tid] = after;
    if (tid == 0) {
      a.n_free_out[0] = stack - c.granted;
      if (a.missing) a.missing[0] = max(0, asked - stack);
    }
  }
  for (int i = wg * N + tid; i < stack - in_stack; i += wgs * N) a.free[in_stack + i] = page_at(in_stack + i);
  for (int i = wg * N + tid; i < c.granted; i += wgs * N) {
    const int b = owner_of<N>(c.takes, a.B, i);
    a.table[(int64_t)b * a.table_stride + c.first[b] + i - c.before(c.takes, b)] = page_at(stack - 1 - i);
  }
  if (!with_slots) return;
  if (a.T < 64) {
    const int n = a.B * a.T;
    for (int i = wg * N + tid; i < n; i += wgs * N) {
      const int b = i / a.T, t = i - b * a.T;
      const int64_t row = rows[b] + t;
      const bool there = t < fresh[b] && row >= 0 && row < a.L && (int)row / a.page < held_after[b];
      a.slots[i] = there ? in_pool(a, page_of(b, (int)row / a.page), (int)row) : -1;
    }
    return;
  }
  // A wave takes 64 tokens, whose entries are looked up by a lane each.
  const int runs = (a.T + 63) / 64, lane = tid & 63;
  for (int u = wg * (N / 64) + (tid >> 6); u < a.B * runs; u += wgs * (N / 64)) {
    const int b = u / runs, t = (u - b * runs) * 64 + lane;
    const int64_t row = rows[b] + t;
    const bool there = t < fresh[b] && row >= 0 && row < a.L && (int)row / a.page < held_after[b];
    const uint64_t some = __ballot(there);
    int slot = -1;
    if (some) {
      const int entry = there ? (int)row / a.page : 0;
      const int e0 = __builtin_amdgcn_readlane(entry, __ffsll((unsigned long long)some) - 1);
      const int e1 = __builtin_amdgcn_readlane(entry, 63 - __clzll((long long)some));
      const int page = e0 + lane <= e1 ? page_of(b, e0 + lane) : -1;
      const int mine = __shfl(page, entry - e0);
      if (there) slot = in_pool(a, mine, (int)row);
    }
    if (t < a.T) a.slots[(int64_t)b * a.T + t] = slot;
  }
}

// More sequences, by one work-group, kAssignSeqs at a time: all pages back, then
// pages off the stack.
__global__ __launch_bounds__(kAssignSeqs) void assign_many_kernel(AssignLaunch a) {
  __shared__ Counts<kAssignSeqs> c;
  const int tid = threadIdx.x;
  const int64_t in_stack = stack_of(a);
  int64_t given = 0;
  for (int b0 = 0; b0 < a.B; b0 += kAssignSeqs) {
    const int n = min(kAssignSeqs, a.B - b0);
    int gives, takes;
    c.count(sequence(a, b0 + min(tid, n - 1)), n, gives, takes);
    __syncthreads();
    for (int i = tid; i < gives; i += kAssignSeqs) {
      const int b = owner_of<kAssignSeqs>(c.gives, n, i);
      const int64_t place = in_stack + given + i;
      if (place < a.n_pages)
        a.free[place] = a.table[(int64_t)(b0 + b) * a.table_stride + c.first[b] + i - c.before(c.gives, b)];
    }
    given += gives;
    __syncthreads();
  }
  const int64_t stack = min((int64_t)a.n_pages, in_stack + given);
  int64_t asked = 0, taken = 0;
  for (int b0 = 0; b0 < a.B; b0 += kAssignSeqs) {
    const int n = min(kAssignSeqs, a.B - b0);
    const Sequence s = sequence(a, b0 + min(tid, n - 1));
    int gives, all;
    c.count(s, n, gives, all);
    const bool takes = s.wanted > s.held, granted = asked + c.takes[tid] <= stack;
    if (tid < n && takes && granted) atomicMax(&c.granted, c.takes[tid]);
    if (tid < n) a.held_out[b0 + tid] = takes && !granted ? s.held : s.wanted;
    __syncthreads();
    for (int i = tid; i < c.granted; i += kAssignSeqs) {
      const int b = owner_of<kAssignSeqs>(c.takes, n, i);
      a.table[(int64_t)(b0 + b) * a.table_stride + c.first[b] + i - c.before(c.takes, b)] = a.free[stack - 1 - taken - i];
    }
    asked += all;
    taken += c.granted;
    __syncthreads();
  }
  if (tid == 0) {
    a.n_free_out[0] = (int)(stack - taken);
    if (a.missing) a.missing[0] = (int)min((int64_t)INT32_MAX, max((int64_t)0, asked - stack));
  }
}

// The slots, of tables and held_out in place.
__global__ __launch_bounds__(256) void slots_kernel(AssignLaunch a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)a.B * a.T) return;
  const int b = (int)(i / a.T), t = (int)(i - (int64_t)b * a.T);
  const int64_t row = (int64_t)a.row0 + (a.lens ? a.lens[b] : 0) + t;
  const int fresh = a.n_new ? min(a.T, a.n_new[b]) : a.T;
  int slot = -1;
  if (t < fresh && row >= 0 && row < a.L && (int)row / a.page < a.held_out[b])
    slot = in_pool(a, a.table[(int64_t)b * a.table_stride + (int)row / a.page], (int)row);
  a.slots[i] = slot;
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

// Memory bounds the copies: 16 groups of 8 beams, three of which copy up to 576 rows of
// 8 heads of 128 (174 MB read and written) in 35 us (4.9 TB/s; a copy of 1 GiB reaches
// 5.0).  Items of 2048 pieces leave the groups' work-groups uneven loads (43 us), plain
// stores take 39 us.  Strides are in 16-byte pieces here, of which a row has VEC.
template <int VEC>
__global__ __launch_bounds__(kReorderThreads) void reorder_kernel(ReorderLaunch a) {
  constexpr int kBatch = 4;  // pieces of K and of V that a thread has under way
  const int group = blockIdx.x / a.wgs, wg = blockIdx.x % a.wgs;
  const int lane = threadIdx.x & 63, base = group * a.W;
  const Beams x = beams_of(a, group);
  // Rows that the beam holds afterwards: its parent's, as far as the parent's pages go
  // and its own.
  int len = 0;
  if (lane < a.W && x.parent >= 0) {
    const int held = a.held ? max(0, min(a.entries, min(a.held[base + x.takes], a.held[base + x.parent]))) : a.entries;
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
          __builtin_nontemporal_store(kx[c], k + to * a.ks[0] + ka[c]);
          __builtin_nontemporal_store(vx[c], v + to * a.vs[0] + va[c]);
        }
      }
    }
    item -= items;
  }
}

}  // namespace

hipError_t launch_assign(const AssignLaunch& a, int cus, hipStream_t stream) {
  const int64_t slots = (int64_t)a.B * a.T;
  // (In place, held and n_free are not there to be read by other work-groups.)
  const bool in_place = a.held_out == a.held || a.n_free_out == a.n_free;
  if (a.B <= kAssignSeqs) {
    // (In place all threads of the one work-group move pages: the 256 sequences above 14.9
    // us, by 256 threads 31.5; 64 of one token 5.5 and 6.3.)
    const int n = a.B <= 256 && !in_place ? 256 : kAssignSeqs;
    // A work-group takes a slot per thread, and up to 32 pages per thread if
    // every page of the tables changes hands.
    const bool with_slots = !in_place || slots <= 4 * n;
    const int64_t by_slots = (slots + n - 1) / n, by_pages = ((int64_t)a.B * a.entries + 32 * n - 1) / (32 * n);
    const int64_t wgs = in_place ? 1 : by_slots > by_pages ? by_slots : by_pages;
    const unsigned grid = (unsigned)(wgs > 2 * cus ? 2 * cus : wgs);
    if (n == 256) assign_kernel<256><<<grid, 256, 0, stream>>>(a, with_slots);
    else assign_kernel<kAssignSeqs><<<grid, kAssignSeqs, 0, stream>>>(a, with_slots);
    if (with_slots) return hipGetLastError();
  } else {
    assign_many_kernel<<<1, kAssignSeqs, 0, stream>>>(a);
  }
  if (hipError_t e = hipGetLastError()) return e;
  slots_kernel<<<(unsigned)((slots + 255) / 256), 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_reorder(ReorderLaunch a, int dtype, int D, int cus, hipStream_t stream) {
  const int vec = D * (dtype == NACL_F32 ? 4 : 2) / 16;
  for (int i = 0; i < 3; ++i) {
    a.ks[i] = a.ks[i] * vec / D;
    a.vs[i] = a.vs[i] * vec / D;
  }
  // About 512 pieces of K and of V per item, so that the few beams that copy are spread
  // over all compute units.
  const int64_t per_head = (int64_t)a.page * vec;
  a.heads_per_item = (int)(per_head >= 512 ? 1 : (512 / per_head < a.H ? 512 / per_head : a.H));
  const int64_t most = ((int64_t)a.entries * a.W) * ((a.H + a.heads_per_item - 1) / a.heads_per_item);
  // Six work-groups per CU, which run together (four beams of one prompt 4.7 us, by eight 5.4;
  // 12 of 16 beams that copy 500 rows of 32 heads 21.5 and 23.5; 4 of 8 beams of 16 groups, 512 rows
  // of 4 heads of 64, 9.9 and 10.8).
  int64_t wgs = (6 * cus + a.groups - 1) / a.groups;
  if (wgs > most) wgs = most;
  a.wgs = (int)wgs;
  const unsigned grid = (unsigned)(wgs * a.groups);
  if (vec == 8) reorder_kernel<8><<<grid, kReorderThreads, 0, stream>>>(a);
  else if (vec == 16) reorder_kernel<16><<<grid, kReorderThreads, 0, stream>>>(a);
  else reorder_kernel<32><<<grid, kReorderThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace nacl
