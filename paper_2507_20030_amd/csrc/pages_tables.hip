// Pages that several sequences hold: sequences that take over others' beginnings, lengths of a step with copies on write, pages moved together, pages copied.
//
// refs[p] counts the sequences that hold page p, each at the same place of its row (what shares a page shares all pages before it).  A page goes back on the
// stack when its last holder gives it up.  Several give up the same page at once: they meet, in a hash table in LDS or, in small tables, in refs itself, and the
// last of them in the order that the call defines takes all off the count.  Sums over the threads place what goes on the stack: nothing depends on the order
// in which atomics arrive.
#include <algorithm>

#include "pages.h"

namespace iwdft {

namespace {

constexpr int kWave = kLanes;

// Atomics on refs are those of one workgroup (a page is held at one place, which one workgroup looks after), in its L2: read past the L1.
__device__ __forceinline__ int32_t refs_now(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void refs_add(int32_t* p, int x) { __hip_atomic_fetch_add(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void refs_least(int32_t* p, int x) { __hip_atomic_fetch_min(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void refs_set(int32_t* p, int x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void all_here() {  // what the workgroup has written, in memory too, is there for all of it; its atomics have arrived
  __threadfence_block();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

__device__ __forceinline__ bool is_page(const SharedTables& t, int p) { return (uint32_t)p < (uint32_t)t.n_pages; }
__device__ __forceinline__ int length_of(const SharedTables& t, int b) { return min(max(t.lens[b], 0), t.max_pages << t.logP); }
__device__ __forceinline__ int last_not_above(const int32_t* v, int n, int x) {  // largest i < n with v[i] <= x (v ascending, v[0] <= x)
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (v[m] <= x) lo = m;
    else hi = m;
  }
  return lo;
}
template <int THREADS>
__device__ __forceinline__ int sum_before(int x, int* all, long long (*lds)[1]) {  // of small numbers
  const int in[1] = {x};
  long long before[1], sum[1];
  sums_before<THREADS>(in, before, sum, lds);
  *all = (int)sum[0];
  return (int)before[0];
}

// ------------------------------------------------------------------------------------------------ lengths of a step
constexpr int kSmallTable = 8192;  // entries of a small table
constexpr int kGiven = 4;          // entries of a thread that are given up at a time
// One workgroup, a thread for each sequence: a chain of loads, sums and stores, 5.0 us for 16 samples that leave their shared page.  What large tables give up takes more threads
// than they have sequences, which only wait while the others sum.  With the tables' copy that comes before it in the timed step (2.2 us): 256 sequences that bring a token each 12.9 us with
// 256 threads, 18.4 with 1024 that all sum, 14.9 so (the launch alone 10.7 and, so, 12.4); 7840 pages given up, most of them shared, and 806 taken, with the slots' launch, 51.7, 37.0, 32.0.
// What a table could hold decides, since lengths are on the device.  With atomics on refs in place of the hash table 49, in three passes over the entries 111.
// A sequence whose last page has room, and which others hold, leaves that page before it grows: it gets a new one and
// an entry in copies.  Where all holders leave in this call, the last of them stays.  It is held to the pages that are left as those before it
// are: had one of them been refused, the page would still be shared.
template <int THREADS, int ROWS>
__global__ __launch_bounds__(THREADS) void pages_grow_kernel(GrowArgs a) {
  constexpr int kGivenSlots = 2 * kGiven * THREADS;
  __shared__ long long lds1[THREADS / kWave][1], lds2[ROWS / kWave][2], totals[2];
  __shared__ struct {
    int32_t page[kGivenSlots], last[kGivenSlots], count[kGivenSlots];
  } given;
  __shared__ int32_t base[ROWS], first[ROWS], back[ROWS];
  __shared__ __attribute__((aligned(16))) int32_t open[ROWS];
  const SharedTables& t = a.t;
  const int b = threadIdx.x, P = 1 << t.logP, most = t.max_pages << t.logP;
  const bool mine = b < t.batch;
  const auto sums_of_rows = [&](const int(&x)[2], long long(&before)[2], long long(&all)[2]) {  // other waves wait
    if (b < ROWS) {
      sums_before<ROWS>(x, before, all, lds2);
    } else {
      __syncthreads();
      __syncthreads();
    }
  };
  const int count = min(max(t.free[0], 0), t.n_pages);
  int have = 0, want = 0;
  if (mine) {
    have = length_of(t, b);
    const int w = a.want[b];
    want = w < 0 || w > most ? have : w;
  }
  const int had = page_count(have, t.logP), get = page_count(want, t.logP);
  int32_t* const row = t.table + (int64_t)b * t.max_pages;

  const bool up = mine && want > have;
  int last = -1;
  if (up && (have & (P - 1))) {
    last = row[had - 1];
    last = is_page(t, last) ? last : -1;
  }

  // pages that are given up, from the last one of the last sequence on; by how many
  const int given_up[2] = {max(had - get, 0), had > get ? 1 : 0};
  long long gone_before[2], gone_all[2];
  sums_of_rows(given_up, gone_before, gone_all);
  if (b == 0) totals[0] = gone_all[0], totals[1] = gone_all[1];
  __syncthreads();
  const int gone = (int)totals[0], givers = (int)totals[1];
  int released = 0;
  if (gone > 0) {
    // those that give something up, side by side: base, the first place that goes, who it is
    if (had > get) base[gone_before[1]] = (int)gone_before[0], first[gone_before[1]] = get, back[gone_before[1]] = b;
    __syncthreads();
    // Batch by batch: a page that two batches give up goes with the second.  Givers of a page meet in a hash table; the last of them in this order counts all off.
    for (int e0 = 0; e0 < gone; e0 += kGiven * THREADS) {
      for (int i = b; i < kGivenSlots; i += THREADS) given.page[i] = -1, given.last[i] = -1, given.count[i] = 0;
      __syncthreads();
      int page[kGiven], slot[kGiven], left[kGiven];
      int o = gone - 1 - e0 - kGiven * b, s = o >= 0 ? last_not_above(base, givers, o) : 0;
#pragma unroll
      for (int i = 0; i < kGiven; ++i, --o) {
        if (o >= 0 && o < base[s]) --s;
        const int p = o >= 0 ? t.table[(int64_t)back[s] * t.max_pages + min(first[s] + o - base[s], t.max_pages - 1)] : -1;
        page[i] = is_page(t, p) ? p : -1;
      }
#pragma unroll
      for (int i = 0; i < kGiven; ++i) {
        slot[i] = -1;
        if (page[i] < 0) continue;
        uint32_t at = ((uint32_t)page[i] * 2654435769u) >> 8;
        for (;; ++at) {  // there are twice as many slots as entries
          at &= kGivenSlots - 1;
          const int was = atomicCAS(&given.page[at], -1, page[i]);
          if (was == -1 || was == page[i]) break;
        }
        slot[i] = (int)at;
        atomicMax(&given.last[at], kGiven * b + i), atomicAdd(&given.count[at], 1);
      }
      __syncthreads();
      int n, goes = 0;
#pragma unroll
      for (int i = 0; i < kGiven; ++i) {
        left[i] = 1;
        if (slot[i] >= 0 && given.last[slot[i]] == kGiven * b + i) left[i] = t.refs[page[i]] - given.count[slot[i]];
        else slot[i] = -1;
      }
#pragma unroll
      for (int i = 0; i < kGiven; ++i) {
        if (slot[i] >= 0) t.refs[page[i]] = max(left[i], 0);
        goes += left[i] <= 0;
      }
      int to = count + released + sum_before<THREADS>(goes, &n, lds1);
#pragma unroll
      for (int i = 0; i < kGiven; ++i)
        if (left[i] <= 0) {
          if (to < t.n_pages) t.free[1 + to] = page[i];
          ++to;
        }
      released += n;
      all_here();
    }
    released = min(released, t.n_pages - count);
  }

  // who has to leave a shared page
  const int holders = last >= 0 ? t.refs[last] : 0;
  const bool shared = holders > 1;
  bool leave = shared;
  if (b < ROWS) open[b] = shared ? last : -1;
  if (__syncthreads_or(shared)) {
    if (shared) {
      int n = 0, after = 0;  // those who share the page and leave it; behind this one
#pragma unroll 8
      for (int c = 0; c < t.batch; c += 4) {
        const int4 o = *(const int4*)(open + c);
        const int is[4] = {o.x == last, o.y == last, o.z == last, o.w == last};
#pragma unroll
        for (int k = 0; k < 4; ++k) n += is[k], after += c + k > b ? is[k] : 0;
      }
      leave = n < holders || after > 0;
    }
  }
  const int x[2] = {up ? get - had + (leave ? 1 : 0) : 0, up ? want - have : 0};
  long long before[2] = {0, 0}, all[2];
  sums_of_rows(x, before, all);
  const bool ok = up && before[1] + x[1] <= a.n_slots && ((x[0] == 0 && !shared) || before[0] + x[0] <= (long long)count + released);
  leave = leave && ok;
  const int in[2] = {ok ? x[0] : 0, ok ? x[1] : 0};
  long long in_before[2], in_all[2];
  sums_of_rows(in, in_before, in_all);
  if (b < ROWS) base[b] = (int)in_before[0], first[b] = leave ? had - 1 : had, back[b] = leave ? last : -1;
  if (b == 0) totals[0] = in_all[0], totals[1] = in_all[1];
  __syncthreads();
  const int taken = (int)totals[0], total = (int)totals[1], top = count + released - 1;
  for (int o = b; o < taken; o += THREADS) {  // pages from the top of the stack
    const int s = last_not_above(base, ROWS, o), i = o - base[s], was = back[s];
    const int p = t.free[1 + max(top - o, 0)];
    t.table[(int64_t)s * t.max_pages + first[s] + i] = p;
    if (is_page(t, p)) refs_set(t.refs + p, 1);
    if (i == 0 && was >= 0) {
      refs_add(t.refs + was, -1);
      ((int2*)a.copies)[s] = make_int2(was, p);
    }
  }
  if (mine) {
    if (!leave) ((int2*)a.copies)[b] = make_int2(-1, -1);
    a.starts[b] = (int)in_before[1];
    t.lens[b] = ok || want < have ? want : have;
  }
  if (b == 0) {
    a.starts[t.batch] = total;
    t.free[0] = count + released - taken;
  }
  if (a.n_slots > kResizeOneSlots) return;  // pages_slots_kernel
  __syncthreads();  // base has been read
  if (b < ROWS) base[b] = (int)in_before[1], first[b] = have;
  all_here();
  for (int i = b; i < a.n_slots; i += THREADS) {
    int slot = -1;
    if (i < total) {
      const int s = last_not_above(base, min(ROWS, t.batch), i), pos = first[s] + i - base[s];
      const int p = t.table[(int64_t)s * t.max_pages + (pos >> t.logP)];
      if (is_page(t, p)) slot = (p << t.logP) + (pos & (P - 1));
    }
    a.slots[i] = slot;
  }
}

// Many slots: after the tables have been brought up to date.
__global__ __launch_bounds__(256) void pages_slots_kernel(GrowArgs a) {
  __shared__ int32_t starts[kSharedBatch + 1], lens[kSharedBatch];
  const SharedTables& t = a.t;
  for (int b = threadIdx.x; b <= t.batch; b += 256) {
    starts[b] = a.starts[b];
    if (b < t.batch) lens[b] = t.lens[b];
  }
  __syncthreads();
  const int total = starts[t.batch];
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.n_slots; i += (int64_t)gridDim.x * 256) {
    int slot = -1;
    if (i < total) {
      const int s = last_not_above(starts, t.batch, (int)i), pos = lens[s] - (starts[s + 1] - (int)i);
      const int p = t.table[(int64_t)s * t.max_pages + (pos >> t.logP)];
      if (is_page(t, p)) slot = (p << t.logP) + (pos & ((1 << t.logP) - 1));
    }
    a.slots[i] = slot;
  }
}

// ------------------------------------------------------------------------------------------------ forking
// Every row takes its parent's entries, all at once: whoever has a place reads it of all rows and then writes.  A page is held at one place, so those who leave
// and enter it meet there.
struct ForkRows {
  int32_t parent[kSharedBatch], had[kSharedBatch], get[kSharedBatch], len[kSharedBatch];
};
template <int THREADS>
__device__ __forceinline__ void fork_rows(const ForkArgs& a, ForkRows& r) {
  for (int b = threadIdx.x; b < a.t.batch; b += THREADS) {
    int p = a.parent[b];
    p = (uint32_t)p < (uint32_t)a.t.batch ? p : b;
    const int keep = a.keep ? a.keep[b] : -1, len = length_of(a.t, p), n = keep < 0 ? len : min(keep, len);
    r.parent[b] = p, r.len[b] = n, r.had[b] = page_count(length_of(a.t, b), a.t.logP), r.get[b] = page_count(n, a.t.logP);
  }
}

// Small tables, all of them in LDS; left in place of an entry that is given up: the page where it goes back on the stack, else -1.
template <int THREADS>
__device__ __forceinline__ void fork_places(const ForkArgs& a, const ForkRows& r, int32_t* lds) {
  const SharedTables& t = a.t;
  const int n = t.max_pages, all = t.batch * n;
  const auto each = [&](auto use) {  // neighbouring threads: neighbouring places
    for (int i = threadIdx.x; i < all; i += THREADS) {
      const int b = (int)((uint32_t)i / (uint32_t)n);
      use(i, b, i - b * n);
    }
  };
  each([&](int i, int b, int j) { lds[i] = j < r.had[b] ? t.table[(int64_t)b * t.max_pages + j] : -1; });
  __syncthreads();
  const auto now_of = [&](int b, int j) { return j < r.get[b] ? lds[r.parent[b] * n + j] : -1; };
  each([&](int i, int b, int j) {
    const int old = lds[i], now = now_of(b, j);
    if (j < r.get[b]) t.table[(int64_t)b * t.max_pages + j] = now;
    if (old == now) return;
    if (is_page(t, now)) refs_add(t.refs + now, 1);
    if (is_page(t, old)) refs_add(t.refs + old, -1);
  });
  all_here();
  const auto left = [&](int b, int j, int old) { return j < r.had[b] && is_page(t, old) && old != now_of(b, j); };
  each([&](int i, int b, int j) {
    if (left(b, j, lds[i]) && refs_now(t.refs + lds[i]) <= 0) refs_least(t.refs + lds[i], b - t.batch);
  });
  all_here();
  each([&](int i, int b, int j) {
    if (j >= r.had[b]) return;
    const int old = lds[i];
    const bool goes = is_page(t, old) && refs_now(t.refs + old) == b - t.batch;  // it has left it: nobody else's entry is looked at
    if (goes) refs_set(t.refs + old, 0);
    lds[i] = goes ? old : -1;
  });
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void pages_fork_one_kernel(ForkArgs a) {
  __shared__ ForkRows r;
  __shared__ int32_t entries[kSmallTable];
  __shared__ long long lds1[THREADS / kWave][1];
  const SharedTables& t = a.t;
  fork_rows<THREADS>(a, r);
  __syncthreads();
  const int n = t.max_pages, all = t.batch * n;
  fork_places<THREADS>(a, r, entries);
  const int count = min(max(t.free[0], 0), t.n_pages);
  __syncthreads();
  int released = 0;
  for (int e0 = 0; e0 < all; e0 += THREADS) {
    const int i = all - 1 - e0 - (int)threadIdx.x, b = i >= 0 ? (int)((uint32_t)i / (uint32_t)n) : 0;
    const int p = i >= 0 && i - b * n < r.had[b] ? entries[i] : -1;
    int m;
    const int at = released + sum_before<THREADS>(p >= 0 ? 1 : 0, &m, lds1);
    if (p >= 0 && count + at < t.n_pages) t.free[1 + count + at] = p;
    released += m;
  }
  for (int b = threadIdx.x; b < t.batch; b += THREADS) t.lens[b] = r.len[b];
  if (threadIdx.x == 0) t.free[0] = min(count + released, t.n_pages);
}

// Large tables: a wave for each place.  What leaves and what enters meets in a hash table in LDS, so that refs are read and written once, by the first of those who
// leave a page or, where nobody does, of those who enter it.  256 rows of 550 places: 10.2 us, and 5.6 for the stack; with atomics on refs, by workgroups of 8192 entries each, 78.
// scratch: the stack's count, the most pages of a row, new lengths [batch], bits of the rows whose entry is given back [places][words], those pages [batch][max_pages]
struct ForkScratch {
  int32_t *head, *lens;
  unsigned long long* bits;
  int32_t* drops;
  int words;
  __device__ __host__ ForkScratch(int32_t* p, int batch, int max_pages) {
    words = (batch + kWave - 1) / kWave;
    bits = (unsigned long long*)p, head = p + 2 * (int64_t)words * max_pages, lens = head + 2, drops = lens + batch;
  }
};
template <int EACH, int WAVES>
__global__ __launch_bounds__(WAVES* kWave) void pages_fork_kernel(ForkArgs a) {
  constexpr int kRows = EACH * kWave, kSlots = 4 * kRows;  // up to two pages of a row
  __shared__ int32_t column[WAVES][kRows], keys[WAVES][kSlots], sums[WAVES][kSlots], firsts[WAVES][kSlots];
  const SharedTables& t = a.t;
  const ForkScratch w(a.scratch, t.batch, t.max_pages);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, j = blockIdx.x * WAVES + wave;
  if (j >= t.max_pages) return;
  const auto in_wave = [] {  // LDS that the lanes of a wave exchange
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  int parent[EACH], had[EACH], get[EACH], len[EACH], most = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int x = lane + kWave * i;
    parent[i] = x, had[i] = get[i] = len[i] = 0;
    if (x < t.batch) {
      const int p = a.parent[x], keep = a.keep ? a.keep[x] : -1;
      parent[i] = (uint32_t)p < (uint32_t)t.batch ? p : x;
      const int n = length_of(t, parent[i]);
      len[i] = keep < 0 ? n : min(keep, n), had[i] = page_count(length_of(t, x), t.logP), get[i] = page_count(len[i], t.logP);
      most = max(most, max(had[i], get[i]));
    }
  }
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) most = max(most, __shfl_xor(most, d));
  if (j == 0) {
    if (lane == 0) w.head[0] = t.free[0], w.head[1] = most;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (lane + kWave * i < t.batch) w.lens[lane + kWave * i] = len[i];
  }
  if (j >= most) return;
#pragma unroll
  for (int i = 0; i < EACH; ++i) column[wave][lane + kWave * i] = j < had[i] ? t.table[(int64_t)(lane + kWave * i) * t.max_pages + j] : -1;
  for (int i = lane; i < kSlots; i += kWave) keys[wave][i] = -1, sums[wave][i] = 0, firsts[wave][i] = 2 * kRows;
  in_wave();
  int out[EACH], in[EACH], leaves[EACH], enters[EACH];  // pages; their slots, -1: none
  const auto slot_of = [&](int page) {
    uint32_t s = ((uint32_t)page * 2654435769u) >> 8;
    for (;; ++s) {  // there are twice as many slots as pages
      s &= kSlots - 1;
      const int was = atomicCAS(&keys[wave][s], -1, page);
      if (was == -1 || was == page) return (int)s;
    }
  };
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int x = lane + kWave * i;
    out[i] = column[wave][x], in[i] = j < get[i] ? column[wave][parent[i]] : -1, leaves[i] = enters[i] = -1;
    if (out[i] == in[i]) continue;
    if (is_page(t, out[i])) {
      leaves[i] = slot_of(out[i]);
      atomicAdd(&sums[wave][leaves[i]], -1), atomicMin(&firsts[wave][leaves[i]], x);
    }
    if (is_page(t, in[i])) {
      enters[i] = slot_of(in[i]);
      atomicAdd(&sums[wave][enters[i]], 1), atomicMin(&firsts[wave][enters[i]], kRows + x);
    }
  }
  in_wave();
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int x = lane + kWave * i;
    bool goes = false;
    if (leaves[i] >= 0 && firsts[wave][leaves[i]] == x) {
      const int left = t.refs[out[i]] + sums[wave][leaves[i]];
      goes = left <= 0;
      t.refs[out[i]] = max(left, 0);
    }
    if (enters[i] >= 0 && firsts[wave][enters[i]] == kRows + x) t.refs[in[i]] = (int)min((long long)t.refs[in[i]] + sums[wave][enters[i]], 0x7fffffffll);
    if (j < get[i] && (out[i] != in[i] || j >= had[i])) t.table[(int64_t)x * t.max_pages + j] = in[i];
    if (goes) w.drops[(int64_t)x * t.max_pages + j] = out[i];
    const unsigned long long m = __ballot(goes);
    if (lane == 0 && i < w.words) w.bits[(int64_t)j * w.words + i] = m;
  }
}
// A workgroup for each row: behind what the rows after it give back.
__global__ __launch_bounds__(256) void pages_fork_free_kernel(ForkArgs a) {
  __shared__ long long lds1[256 / kWave][1];
  const SharedTables& t = a.t;
  const ForkScratch w(a.scratch, t.batch, t.max_pages);
  const int b = blockIdx.x, word = b / kWave, count = min(max(w.head[0], 0), t.n_pages), most = w.head[1];
  const unsigned long long bit = 1ull << (b % kWave);
  if (threadIdx.x == 0) t.lens[b] = w.lens[b];
  bool any = false;
  for (int j = threadIdx.x; j < most; j += 256) any |= (w.bits[(int64_t)j * w.words + word] & bit) != 0;
  if (!__syncthreads_or(any) && b) return;
  int before = 0, all, own = 0;
  for (int j = threadIdx.x; j < most; j += 256)
    for (int i = word; i < w.words; ++i) {
      const unsigned long long m = w.bits[(int64_t)j * w.words + i];
      before += __popcll(i == word ? m & ~(bit | (bit - 1)) : m);
      if (i == word) own += (m & bit) != 0;
    }
  sum_before<256>(before, &all, lds1);
  int released = all, n;
  sum_before<256>(own, &n, lds1);
  if (b == 0 && threadIdx.x == 0) t.free[0] = min(count + released + n, t.n_pages);
  for (int e0 = 0; n && e0 < most; e0 += 256) {
    const int j = most - 1 - e0 - (int)threadIdx.x;
    const bool goes = j >= 0 && (w.bits[(int64_t)j * w.words + word] & bit);
    int m;
    const int at = count + released + sum_before<256>(goes ? 1 : 0, &m, lds1);
    if (goes && at < t.n_pages) t.free[1 + at] = w.drops[(int64_t)b * t.max_pages + j];
    released += m;
  }
}

// ------------------------------------------------------------------------------------------------ compacting
// The i-th highest held page goes to the i-th lowest free place, while that is below it.  One workgroup: 17000 pages 103 us with a thread for each word of bits, 16 with a lane for
// each page; 240 pages and their table 5.1.  Held pages as bits, 64 to a word; ranks are sums of their counts.
// With h held pages and m moves, what becomes of a page follows from the held pages before it alone:
//   held, h - 1 - (held before) =: i < m         moves to the i-th lowest free place
//   free, (free before) < m                      is that place
//   otherwise free, or moving                    lies on the stack: free pages below it when all is done = free before - m, plus held before - (h - m) where positive
// scratch: which move a page is [n_pages], the lowest page that moves, how many move, and, of a large pool, the bits
constexpr int kCompactThreads = 1024, kCompactWords = 2048;  // words in LDS
__device__ __forceinline__ int32_t* compact_head(const CompactArgs& a) { return a.scratch + a.t.n_pages; }
// Counts and entries after the moves, by thread `at` of `step`: a page from the lowest that moves on, if held, moves.
__device__ __forceinline__ void compact_refs(const CompactArgs& a, int moved, int at, int step) {
  for (int i = at; i < moved; i += step) {
    const int2 m = ((const int2*)a.moves)[i];
    a.t.refs[m.y] = a.t.refs[m.x], a.t.refs[m.x] = 0;
  }
}
__device__ __forceinline__ void compact_row(const CompactArgs& a, int moved, int lowest, int b, int at, int step) {
  const SharedTables& t = a.t;
  const int n = page_count(length_of(t, b), t.logP);
  for (int j = at; j < n; j += step) {
    int32_t* entry = t.table + (int64_t)b * t.max_pages + j;
    const int p = *entry;
    if (p < lowest || p >= t.n_pages) continue;
    const int i = a.scratch[p];
    if ((uint32_t)i < (uint32_t)moved) *entry = a.moves[2 * i + 1];  // always, unless the page is counted as free
  }
}

// ONE: the table, which is small, too.
template <bool LDS, bool ONE>
__global__ __launch_bounds__(kCompactThreads) void pages_compact_kernel(CompactArgs a) {
  __shared__ long long lds1[kCompactThreads / kWave][1];
  __shared__ unsigned long long kept[LDS ? kCompactWords : 1];
  __shared__ int32_t base[kCompactThreads], found[2];
  const SharedTables& t = a.t;
  constexpr int kWaves = kCompactThreads / kWave;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, words = (t.n_pages + kWave - 1) / kWave;
  int32_t *move = a.scratch, *head = compact_head(a);
  unsigned long long* bits = LDS ? kept : (unsigned long long*)(((uintptr_t)(head + 2) + 7) & ~(uintptr_t)7);
  const unsigned long long below = (1ull << lane) - 1;
  int held = 0;
  {
    int mine = 0;
#pragma unroll 8
    for (int w = wave; w < words; w += kWaves) {
      const int p = w * kWave + lane;
      const unsigned long long m = __ballot(p < t.n_pages && t.refs[p] > 0);
      if (lane == 0) bits[w] = m, mine += __popcll(m);
    }
    sum_before<kCompactThreads>(mine, &held, lds1);
  }
  all_here();
  // held pages from `held` on, which is as many as free places below
  int above = 0;
  {
    int mine = 0;
    for (int w = held / kWave + threadIdx.x; w < words; w += kCompactThreads) mine += __popcll(w == held / kWave ? bits[w] & ~((1ull << (held % kWave)) - 1) : bits[w]);
    sum_before<kCompactThreads>(mine, &above, lds1);
  }
  const int moved = min(above, a.n_moves);
  if (threadIdx.x == 0) found[0] = t.n_pages;
  int before = 0;
  for (int w0 = 0; w0 < words; w0 += kCompactThreads) {
    int n;
    const int at = before + sum_before<kCompactThreads>(w0 + threadIdx.x < words ? __popcll(bits[w0 + threadIdx.x]) : 0, &n, lds1);
    base[threadIdx.x] = at;
    __syncthreads();
    before += n;
#pragma unroll 4
    for (int w = w0 + wave; w < min(words, w0 + kCompactThreads); w += kWaves) {
      const unsigned long long m = bits[w];
      const int p = w * kWave + lane, held_before = base[w - w0] + __popcll(m & below), free_before = p - held_before;
      if (p >= t.n_pages) continue;
      const bool is_held = m >> lane & 1;
      const int i = held - 1 - held_before;
      if (is_held && i < moved) {
        move[p] = i, a.moves[2 * i] = p;
        if (i == moved - 1) found[0] = p;
      }
      if (!is_held && free_before < moved) a.moves[2 * free_before + 1] = p;
      if (is_held ? i < moved : free_before >= moved) t.free[t.n_pages - held - (free_before - moved) - max(held_before - (held - moved), 0)] = p;
    }
    __syncthreads();
  }
  for (int64_t i = moved + threadIdx.x; i < a.n_moves; i += kCompactThreads) ((int2*)a.moves)[i] = make_int2(-1, -1);
  const int lowest = found[0];
  if (threadIdx.x == 0) head[0] = lowest, head[1] = moved, t.free[0] = t.n_pages - held;
  if (!ONE || moved == 0) return;
  all_here();
  compact_refs(a, moved, threadIdx.x, kCompactThreads);
  for (int b = wave; b < t.batch; b += kWaves) compact_row(a, moved, lowest, b, lane, kWave);
}
__global__ __launch_bounds__(256) void pages_compact_table_kernel(CompactArgs a) {
  const int lowest = compact_head(a)[0], moved = compact_head(a)[1], at = blockIdx.x * 256 + threadIdx.x, step = gridDim.x * 256;
  if (moved == 0) return;
  if ((int)blockIdx.y < a.t.batch) compact_row(a, moved, lowest, blockIdx.y, at, step);
  else compact_refs(a, moved, at, step);
}

// ------------------------------------------------------------------------------------------------ copying
// A workgroup copies EACH 16-byte words a thread of a page of one layer, or what a page has less; the first one the exponents too.  Bound by memory.  What is written is not read
// again soon: with stores that go through the caches 33 MB (16 pages from 4, 32 layers) take 21.1 us, so 7.4.  What is read may be, by copies of the same
// page: past the caches 33 MB take 12.7 us, and 165 MB 54 for 48.  Beyond what the last cache holds that turns: 330 MB 105 us past it in pieces of 4 KB (in pieces of
// 8 108), 116 through it; 1.25 GB 397 and 447, 6.3 TB/s.
// How many of a list are to be copied is on the device; a workgroup whose pair is not there ends at once, and 1000 of those take 0.37 us: 256 rows of 32 layers of 64 KB, as a step of growth
// has them, 49 us.  2048 workgroups that read the list and take turns (4.2 us then) copy 33 MB in 9.1 us for 7.4 and 1.25 GB in 485 to 552 for 399: loads wait for older stores, and what runs
// at a time lies apart.  Larger pieces: 16 KB 8.2 and 434, 64 KB 9.4 and 473.
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
constexpr int64_t kCachedCopies = 256 << 20;
template <int EACH, bool PAST>
__global__ __launch_bounds__(256) void pages_copy_kernel(Pages from, Pages to, int layer0, int n, const int32_t* copies, int pieces, int64_t piece0) {
  constexpr int64_t kBytes = EACH * 256 * 16;
  const int64_t piece = piece0 + (int)(blockIdx.x % (uint32_t)pieces);
  const int rest = (int)(blockIdx.x / (uint32_t)pieces), layer = layer0 + rest / n;
  const int2 c = ((const int2*)copies)[rest % n];
  if ((uint32_t)c.x >= (uint32_t)from.n_pages || (uint32_t)c.y >= (uint32_t)to.n_pages) return;
  const int64_t source = page_head(from, layer, c.x, 0), target = page_head(to, layer, c.y, 0), bytes = (int64_t)from.H << (from.logP + 8);
  const uint4v* s = (const uint4v*)(page_values(from, source) + piece * kBytes);
  uint4v* d = (uint4v*)(page_values(to, target) + piece * kBytes);
  const int words = (int)(min(kBytes, bytes - piece * kBytes) / 16);
  uint4v x[EACH];
#pragma unroll
  for (int k = 0; k < EACH; ++k)
    if (k * 256 + (int)threadIdx.x < words) x[k] = PAST ? __builtin_nontemporal_load(s + k * 256 + threadIdx.x) : s[k * 256 + threadIdx.x];
#pragma unroll
  for (int k = 0; k < EACH; ++k)
    if (k * 256 + (int)threadIdx.x < words) __builtin_nontemporal_store(x[k], d + k * 256 + threadIdx.x);
  if (piece == 0)
    for (int h = threadIdx.x; h < from.H; h += 256) ((int2*)to.exponents)[target + h] = ((const int2*)from.exponents)[source + h];
}
int64_t page_bytes(const Pages& S) { return (int64_t)S.H << (S.logP + 8); }
bool copies_past(const Pages& S, int n_layers, int n) { return (double)page_bytes(S) * n_layers * n > (double)kCachedCopies; }

bool fork_in_one(int batch, int max_pages) { return (int64_t)batch * max_pages <= kSmallTable; }

}  // namespace

size_t pages_fork_bytes(int batch, int max_pages) {
  if (fork_in_one(batch, max_pages)) return 0;
  const ForkScratch w(nullptr, batch, max_pages);
  return (size_t)((const char*)(w.drops + (int64_t)batch * max_pages) - (const char*)nullptr);
}
size_t pages_compact_bytes(int n_pages) { return sizeof(int32_t) * ((size_t)n_pages + 4) + sizeof(long long) * (((size_t)n_pages + 63) / 64 + 1); }

hipError_t launch_pages_grow(const GrowArgs& a, hipStream_t st) {
  if (a.t.batch <= 256 && (int64_t)a.t.batch * a.t.max_pages <= kSmallTable) pages_grow_kernel<256, 256><<<1, 256, 0, st>>>(a);
  else if (a.t.batch <= 256) pages_grow_kernel<kSharedBatch, 256><<<1, kSharedBatch, 0, st>>>(a);
  else pages_grow_kernel<kSharedBatch, kSharedBatch><<<1, kSharedBatch, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_slots <= kResizeOneSlots) return e;
  pages_slots_kernel<<<(unsigned)std::min(1024, (a.n_slots + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const ForkArgs& a, hipStream_t st) {
  if (fork_in_one(a.t.batch, a.t.max_pages)) {
    pages_fork_one_kernel<kSharedBatch><<<1, kSharedBatch, 0, st>>>(a);
    return hipGetLastError();
  }
  const auto grid = [&](int waves) { return (unsigned)((a.t.max_pages + waves - 1) / waves); };
  if (a.t.batch <= kWave) pages_fork_kernel<1, 4><<<grid(4), 4 * kWave, 0, st>>>(a);
  else if (a.t.batch <= 4 * kWave) pages_fork_kernel<4, 4><<<grid(4), 4 * kWave, 0, st>>>(a);
  else pages_fork_kernel<16, 1><<<grid(1), kWave, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  pages_fork_free_kernel<<<a.t.batch, 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const CompactArgs& a, hipStream_t st) {
  const bool lds = a.t.n_pages <= kCompactWords * kWave, one = lds && (int64_t)a.t.batch * a.t.max_pages <= kSmallTable;
  if (one) pages_compact_kernel<true, true><<<1, kCompactThreads, 0, st>>>(a);
  else if (lds) pages_compact_kernel<true, false><<<1, kCompactThreads, 0, st>>>(a);
  else pages_compact_kernel<false, false><<<1, kCompactThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || one) return e;
  pages_compact_table_kernel<<<dim3((unsigned)std::min(16, (a.t.max_pages + 255) / 256), (unsigned)a.t.batch + 1), 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const Pages& from, const Pages& to, int layer, int n_layers, const int32_t* copies, int n, hipStream_t st) {
  const bool past = copies_past(from, n_layers, n);
  const int64_t size = past ? 4096 : 8192, pieces = (page_bytes(from) + size - 1) / size;
  // One launch, unless that were too many threads: of 64 GiB of a list's pages each then.  A list is as long as it may have to be, and is never too long: tables
  // have changed by the time it is here.
  constexpr int64_t kMost = kMostUnits / 4;  // workgroups
  const int64_t each_pieces = std::min(pieces, kMost), each_copies = std::min<int64_t>(n, kMost / each_pieces), each_layers = std::min<int64_t>(n_layers, kMost / (each_pieces * each_copies));
  for (int64_t l = 0; l < n_layers; l += each_layers)
    for (int64_t c = 0; c < n; c += each_copies)
      for (int64_t p = 0; p < pieces; p += each_pieces) {
        const int here = (int)std::min(pieces - p, each_pieces), some = (int)std::min<int64_t>(n - c, each_copies), layers = (int)std::min<int64_t>(n_layers - l, each_layers);
        const unsigned grid = (unsigned)((int64_t)here * some * layers);
        if (past) pages_copy_kernel<1, true><<<grid, 256, 0, st>>>(from, to, layer + (int)l, some, copies + 2 * c, here, p);
        else pages_copy_kernel<2, false><<<grid, 256, 0, st>>>(from, to, layer + (int)l, some, copies + 2 * c, here, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
  return hipSuccess;
}

}  // namespace iwdft
