// Pages that several sequences hold: sequences that take over others' beginnings, lengths of a step with copies on write, pages moved together, pages copied.
//
// refs[p] counts the sequences that hold page p, each at the same place of its row (what shares a page shares all pages before it).  A page goes back on the
// stack when its last holder gives it up.  Several threads give up the same page at once, so the order on the stack is settled in three steps: all count down; of a page
// that has come to 0 the givers leave the smallest of their places in refs, as a negative number; who finds its own there pushes the page.
// Sums over the threads place the pushes: nothing depends on the order in which atomics arrive.
#include <algorithm>

#include "pages.h"

namespace iwdft {

namespace {

constexpr int kWave = kLanes;

// refs are changed by atomics, which the L2 carries out: read past the L1.
__device__ __forceinline__ int32_t refs_now(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void refs_add(int32_t* p, int x) { __hip_atomic_fetch_add(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void refs_least(int32_t* p, int x) { __hip_atomic_fetch_min(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void refs_set(int32_t* p, int x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
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
// One workgroup, a thread for each sequence.  A sequence whose last page has room, and which others hold, leaves that page before it grows: it gets a new one and
// an entry in copies.  Where all holders leave in this call, the last of them stays.  It is held to the pages that are left as those before it
// are: had one of them been refused, the page would still be shared.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void pages_grow_kernel(GrowArgs a) {
  __shared__ long long lds1[THREADS / kWave][1], lds2[THREADS / kWave][2];
  __shared__ int32_t base[THREADS + 1], first[THREADS], open[THREADS], back[THREADS];
  const SharedTables& t = a.t;
  const int b = threadIdx.x, P = 1 << t.logP, most = t.max_pages << t.logP;
  const bool mine = b < t.batch;
  const int count = min(max(t.free[0], 0), t.n_pages);
  int have = 0, want = 0;
  if (mine) {
    have = length_of(t, b);
    const int w = a.want[b];
    want = w < 0 || w > most ? have : w;
  }
  const int had = page_count(have, t.logP), get = page_count(want, t.logP);
  int32_t* const row = t.table + (int64_t)b * t.max_pages;

  // pages that are given up, from the last one of the last sequence on
  int gone = 0, released = 0;
  const int gone_before = sum_before<THREADS>(max(had - get, 0), &gone, lds1);
  if (gone > 0) {
    base[b] = gone_before, first[b] = get;
    __syncthreads();
    const auto entry = [&](int o) {
      const int s = last_not_above(base, THREADS, o), j = first[s] + o - base[s];
      const int p = t.table[(int64_t)s * t.max_pages + min(j, t.max_pages - 1)];
      return is_page(t, p) ? p : -1;
    };
    for (int o = b; o < gone; o += THREADS)
      if (const int p = entry(o); p >= 0) refs_add(t.refs + p, -1);
    all_here();
    for (int o = b; o < gone; o += THREADS)
      if (const int p = entry(o); p >= 0 && refs_now(t.refs + p) <= 0) refs_least(t.refs + p, o - gone);
    all_here();
    for (int e0 = 0; e0 < gone; e0 += THREADS) {
      const int o = gone - 1 - e0 - b, p = o >= 0 ? entry(o) : -1;
      const bool goes = p >= 0 && refs_now(t.refs + p) == o - gone;
      int n;
      const int at = released + sum_before<THREADS>(goes ? 1 : 0, &n, lds1);
      if (goes) {
        if (count + at < t.n_pages) t.free[1 + count + at] = p;
        refs_set(t.refs + p, 0);
      }
      released += n;
    }
    released = min(released, t.n_pages - count);
    all_here();
  }

  // who has to leave a shared page
  const bool up = mine && want > have;
  int last = -1;
  if (up && (have & (P - 1))) {
    last = row[had - 1];
    last = is_page(t, last) ? last : -1;
  }
  const int holders = last >= 0 ? refs_now(t.refs + last) : 0;
  const bool shared = holders > 1;
  bool leave = shared;
  open[b] = shared ? last : -1;
  if (__syncthreads_or(shared)) {
    if (shared) {
      int n = 0, after = 0;
      for (int c = 0; c < t.batch; ++c) {
        n += open[c] == last;
        after += c > b && open[c] == last;
      }
      leave = n < holders || after > 0;
    }
  }
  const int x[2] = {up ? get - had + (leave ? 1 : 0) : 0, up ? want - have : 0};
  long long before[2], all[2];
  sums_before<THREADS>(x, before, all, lds2);
  const bool ok = up && before[1] + x[1] <= a.n_slots && ((x[0] == 0 && !shared) || before[0] + x[0] <= (long long)count + released);
  leave = leave && ok;
  const int in[2] = {ok ? x[0] : 0, ok ? x[1] : 0};
  long long in_before[2], in_all[2];
  sums_before<THREADS>(in, in_before, in_all, lds2);
  const int taken = (int)in_all[0], total = (int)in_all[1], top = count + released - 1;

  base[b] = (int)in_before[0], first[b] = leave ? had - 1 : had, back[b] = leave ? last : -1;
  __syncthreads();
  for (int o = b; o < taken; o += THREADS) {  // pages from the top of the stack
    const int s = last_not_above(base, THREADS, o), i = o - base[s], was = back[s];
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
  base[b] = (int)in_before[1], first[b] = have;
  all_here();
  for (int i = b; i < a.n_slots; i += THREADS) {
    int slot = -1;
    if (i < total) {
      const int s = last_not_above(base, min(THREADS, t.batch), i), pos = first[s] + i - base[s];
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
// Every row takes its parent's entries, all at once: a workgroup has some places of all rows, reads them whole and then writes.  A page is held at one place, so
// who gives it up meets in one workgroup.
constexpr int kForkEntries = 8192;  // in LDS
constexpr int kForkGroups = 64;     // workgroups: each leaves a count for every row

struct ForkRows {
  int32_t parent[kSharedBatch], had[kSharedBatch], get[kSharedBatch], len[kSharedBatch];
};
template <int THREADS>
__device__ __forceinline__ int fork_rows(const ForkArgs& a, ForkRows& r) {  // returns the most pages of a row, before or after
  int most = 0;
  for (int b = threadIdx.x; b < a.t.batch; b += THREADS) {
    int p = a.parent[b];
    p = (uint32_t)p < (uint32_t)a.t.batch ? p : b;
    const int keep = a.keep ? a.keep[b] : -1, len = length_of(a.t, p), n = keep < 0 ? len : min(keep, len);
    r.parent[b] = p, r.len[b] = n, r.had[b] = page_count(length_of(a.t, b), a.t.logP), r.get[b] = page_count(n, a.t.logP);
    most = max(most, max(r.had[b], r.get[b]));
  }
  return most;
}

// Places [j0, j0 + n) of all rows; drop(b, j, page) for every entry that a row had: page where it goes back on the stack, else -1.
template <int THREADS, class Drop>
__device__ __forceinline__ void fork_places(const ForkArgs& a, const ForkRows& r, int32_t* lds, int j0, int n, Drop drop) {
  const SharedTables& t = a.t;
  const int all = t.batch * n;
  const auto each = [&](auto use) {  // neighbouring threads: neighbouring places
    for (int i = threadIdx.x; i < all; i += THREADS) {
      const int b = (int)((uint32_t)i / (uint32_t)n), j = j0 + i - b * n;
      use(i, b, j);
    }
  };
  each([&](int i, int b, int j) { lds[i] = j < r.had[b] ? t.table[(int64_t)b * t.max_pages + j] : -1; });
  __syncthreads();
  const auto now_of = [&](int b, int j) { return j < r.get[b] ? lds[r.parent[b] * n + j - j0] : -1; };
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
    const bool goes = is_page(t, old) && refs_now(t.refs + old) == b - t.batch;  // it has left it; drop may write where lds[i] is
    if (goes) refs_set(t.refs + old, 0);
    drop(b, j, goes ? old : -1);
  });
}

// Small tables: one launch.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void pages_fork_one_kernel(ForkArgs a) {
  __shared__ ForkRows r;
  __shared__ int32_t entries[kForkEntries];
  __shared__ long long lds1[THREADS / kWave][1];
  const SharedTables& t = a.t;
  fork_rows<THREADS>(a, r);
  __syncthreads();
  const int n = t.max_pages, all = t.batch * n;
  fork_places<THREADS>(a, r, entries, 0, n, [&](int b, int j, int page) { entries[b * n + j] = page; });
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

// scratch: new lengths [batch], pages given back [kForkGroups][batch], of every entry the page that is given back [batch][max_pages], the stack's count
__global__ __launch_bounds__(256) void pages_fork_kernel(ForkArgs a) {
  __shared__ ForkRows r;
  __shared__ int32_t entries[kForkEntries], gone[kSharedBatch], most;
  const SharedTables& t = a.t;
  if (threadIdx.x == 0) most = 0;
  __syncthreads();
  atomicMax(&most, fork_rows<256>(a, r));
  for (int b = threadIdx.x; b < t.batch; b += 256) gone[b] = 0;
  __syncthreads();
  int32_t *lens = a.scratch, *counts = lens + t.batch + (int64_t)blockIdx.x * t.batch, *drops = a.scratch + (int64_t)t.batch * (1 + kForkGroups);
  const int n = min(64, kForkEntries / t.batch);
  for (int64_t j0 = (int64_t)blockIdx.x * n; j0 < most; j0 += (int64_t)gridDim.x * n) {
    fork_places<256>(a, r, entries, (int)j0, min(n, t.max_pages - (int)j0), [&](int b, int j, int page) {
      drops[(int64_t)b * t.max_pages + j] = page;
      if (page >= 0) atomicAdd(&gone[b], 1);
    });
    __syncthreads();
  }
  for (int b = threadIdx.x; b < t.batch; b += 256) {
    counts[b] = gone[b];
    if (blockIdx.x == 0) lens[b] = r.len[b];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) drops[(int64_t)t.batch * t.max_pages] = t.free[0];
}
// A workgroup for each row: behind what the rows after it give back.
__global__ __launch_bounds__(256) void pages_fork_free_kernel(ForkArgs a, int groups) {
  __shared__ long long lds1[256 / kWave][1], lds2[256 / kWave][2];
  const SharedTables& t = a.t;
  const int32_t *lens = a.scratch, *counts = lens + t.batch, *drops = a.scratch + (int64_t)t.batch * (1 + kForkGroups);
  const int b = blockIdx.x, had = page_count(length_of(t, b), t.logP);
  const int count = min(max(drops[(int64_t)t.batch * t.max_pages], 0), t.n_pages);
  int x[2] = {0, 0};
  for (int i = threadIdx.x; i < groups * t.batch; i += 256) {
    const int c = i % t.batch;
    x[0] += c > b ? counts[i] : 0, x[1] += c == b ? counts[i] : 0;
  }
  long long before[2], all[2];
  sums_before<256>(x, before, all, lds2);
  int released = (int)all[0];
  const int own = (int)all[1];
  for (int e0 = 0; own && e0 < had; e0 += 256) {
    const int j = had - 1 - e0 - (int)threadIdx.x, p = j >= 0 ? drops[(int64_t)b * t.max_pages + j] : -1;
    int m;
    const int at = released + sum_before<256>(p >= 0 ? 1 : 0, &m, lds1);
    if (p >= 0 && count + at < t.n_pages) t.free[1 + count + at] = p;
    released += m;
  }
  __syncthreads();  // the length has been read
  if (threadIdx.x == 0) {
    t.lens[b] = lens[b];
    if (b == 0) t.free[0] = (int)min((long long)count + all[0] + own, (long long)t.n_pages);
  }
}

// ------------------------------------------------------------------------------------------------ compacting
// The i-th highest held page goes to the i-th lowest free place, while that is below it.  Held pages as bits, 64 to a word; ranks are sums of their counts.
// scratch: where each page that moves goes [n_pages], the lowest page that moves, how many, bits [2 * words]
constexpr int kCompactThreads = 1024;
__global__ __launch_bounds__(kCompactThreads) void pages_compact_kernel(CompactArgs a) {
  __shared__ long long lds1[kCompactThreads / kWave][1];
  const SharedTables& t = a.t;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, words = (t.n_pages + kWave - 1) / kWave;
  int32_t *to = a.scratch, *head = to + t.n_pages;
  unsigned long long* bits = (unsigned long long*)(((uintptr_t)(head + 2) + 7) & ~(uintptr_t)7);
  const auto word_mask = [&](int w) { return w == words - 1 && (t.n_pages & 63) ? (1ull << (t.n_pages & 63)) - 1 : ~0ull; };
  for (int w = wave; w < words; w += kCompactThreads / kWave) {
    const int p = w * kWave + lane;
    const unsigned long long m = __ballot(p < t.n_pages && t.refs[p] > 0);
    if (lane == 0) bits[w] = m;
  }
  for (int i = threadIdx.x; i < a.n_moves; i += kCompactThreads) ((int2*)a.moves)[i] = make_int2(-1, -1);
  all_here();
  int held = 0;
  for (int w0 = 0; w0 < words; w0 += kCompactThreads) {
    const int w = w0 + threadIdx.x;
    int n;
    sum_before<kCompactThreads>(w < words ? __popcll(bits[w]) : 0, &n, lds1);
    held += n;
  }
  // held pages from `held` on and free places below: as many of each
  int below = 0;  // held pages before the word
  for (int w0 = 0; w0 < words; w0 += kCompactThreads) {
    const int w = w0 + threadIdx.x;
    const unsigned long long m = w < words ? bits[w] : 0;
    int n, before = below + sum_before<kCompactThreads>(__popcll(m), &n, lds1);
    below += n;
    if (w >= words) continue;
    unsigned long long rest = m;
    int rank = held - 1 - before;  // from the highest held page on
    for (; rest; rest &= rest - 1, --rank) {
      const int p = w * kWave + __builtin_ctzll(rest);
      if (p >= held && rank < a.n_moves) a.moves[2 * rank] = p;
    }
    rest = ~m & word_mask(w);
    int place = w * kWave - before;  // free places before the word
    for (; rest; rest &= rest - 1, ++place) {
      const int p = w * kWave + __builtin_ctzll(rest);
      if (p < held && place < a.n_moves) a.moves[2 * place + 1] = p;
    }
  }
  all_here();
  int lowest = t.n_pages, moved = 0;
  for (int i0 = 0; i0 < a.n_moves; i0 += kCompactThreads) {
    const int i = i0 + threadIdx.x;
    const int2 m = i < a.n_moves ? ((const int2*)a.moves)[i] : make_int2(-1, -1);
    if (m.x >= 0) {
      to[m.x] = m.y, lowest = m.x;
      t.refs[m.y] = t.refs[m.x], t.refs[m.x] = 0;
      atomicAnd(&bits[m.x / kWave], ~(1ull << (m.x % kWave)));
      atomicOr(&bits[m.y / kWave], 1ull << (m.y % kWave));
    }
    int n;
    sum_before<kCompactThreads>(m.x >= 0 ? 1 : 0, &n, lds1);
    moved += n;
  }
  all_here();
  if (threadIdx.x == 0) head[1] = moved, t.free[0] = t.n_pages - held;
  if (moved ? lowest == a.moves[2 * (moved - 1)] : threadIdx.x == 0) head[0] = lowest;
  int free_before = 0;
  for (int w0 = 0; w0 < words; w0 += kCompactThreads) {  // free pages, the lowest on top
    const int w = w0 + threadIdx.x;
    unsigned long long m = 0;
    if (w < words) m = ~__hip_atomic_load(&bits[w], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & word_mask(w);
    int n, rank = free_before + sum_before<kCompactThreads>(__popcll(m), &n, lds1);
    free_before += n;
    for (; m; m &= m - 1, ++rank) t.free[t.n_pages - held - rank] = w * kWave + __builtin_ctzll(m);
  }
}
// The pages that move are the highest ones held: an entry from the lowest of them on is one of them.
__global__ __launch_bounds__(256) void pages_compact_table_kernel(CompactArgs a) {
  const SharedTables& t = a.t;
  const int32_t *to = a.scratch, *head = to + t.n_pages;
  const int lowest = head[0], b = blockIdx.y, n = page_count(length_of(t, b), t.logP);
  if (head[1] == 0) return;
  for (int j = blockIdx.x * 256 + threadIdx.x; j < n; j += gridDim.x * 256) {
    int32_t* at = t.table + (int64_t)b * t.max_pages + j;
    const int p = *at;
    if (p >= lowest && p < t.n_pages) *at = to[p];
  }
}

// ------------------------------------------------------------------------------------------------ copying
// A workgroup copies 16 KB of a page of one layer, or what a page has less; the first one the exponents too.
constexpr int kCopyBytes = 16384;
__global__ __launch_bounds__(256) void pages_copy_kernel(Pages from, Pages to, int layer0, int n, const int32_t* copies, int pieces, int64_t units) {
  const int64_t unit = blockIdx.x;
  if (unit >= units) return;
  const int piece = (int)(unit % pieces);
  const int64_t rest = unit / pieces;
  const int i = (int)(rest % n), layer = layer0 + (int)(rest / n);
  const int2 c = ((const int2*)copies)[i];
  if ((uint32_t)c.x >= (uint32_t)from.n_pages || (uint32_t)c.y >= (uint32_t)to.n_pages) return;
  const int64_t source = page_head(from, layer, c.x, 0), target = page_head(to, layer, c.y, 0), bytes = (int64_t)from.H << (from.logP + 8);
  const uint4* s = (const uint4*)(page_values(from, source) + (int64_t)piece * kCopyBytes);
  uint4* d = (uint4*)(page_values(to, target) + (int64_t)piece * kCopyBytes);
  const int words = (int)(min((int64_t)kCopyBytes, bytes - (int64_t)piece * kCopyBytes) / 16);
  uint4 x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k * 256 + (int)threadIdx.x < words) x[k] = s[k * 256 + threadIdx.x];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k * 256 + (int)threadIdx.x < words) d[k * 256 + threadIdx.x] = x[k];
  if (piece == 0)
    for (int h = threadIdx.x; h < from.H; h += 256) ((int2*)to.exponents)[target + h] = ((const int2*)from.exponents)[source + h];
}
int64_t copy_pieces(const Pages& S) { return (((int64_t)S.H << (S.logP + 8)) + kCopyBytes - 1) / kCopyBytes; }

bool fork_in_one(int batch, int max_pages) { return (int64_t)batch * max_pages <= kForkEntries; }

}  // namespace

size_t pages_fork_bytes(int batch, int max_pages) {
  return fork_in_one(batch, max_pages) ? 0 : sizeof(int32_t) * ((size_t)batch * (1 + kForkGroups + (size_t)max_pages) + 1);
}
size_t pages_compact_bytes(int n_pages) { return sizeof(int32_t) * ((size_t)n_pages + 4) + sizeof(long long) * (((size_t)n_pages + 63) / 64 + 1); }

hipError_t launch_pages_grow(const GrowArgs& a, hipStream_t st) {
  if (a.t.batch <= 256) pages_grow_kernel<256><<<1, 256, 0, st>>>(a);
  else pages_grow_kernel<kSharedBatch><<<1, kSharedBatch, 0, st>>>(a);
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
  const int n = std::min(64, kForkEntries / a.t.batch), groups = std::min(kForkGroups, (a.t.max_pages + n - 1) / n);
  pages_fork_kernel<<<groups, 256, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  pages_fork_free_kernel<<<a.t.batch, 256, 0, st>>>(a, groups);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const CompactArgs& a, hipStream_t st) {
  pages_compact_kernel<<<1, kCompactThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.t.batch == 0) return e;
  pages_compact_table_kernel<<<dim3((unsigned)std::min(16, (a.t.max_pages + 255) / 256), (unsigned)a.t.batch), 256, 0, st>>>(a);
  return hipGetLastError();
}

int64_t pages_copy_units(const Pages& S, int n_layers, int n) { return copy_pieces(S) * n_layers * n; }
hipError_t launch_pages_copy(const Pages& from, const Pages& to, int layer, int n_layers, const int32_t* copies, int n, hipStream_t st) {
  const int64_t units = pages_copy_units(from, n_layers, n);
  pages_copy_kernel<<<(unsigned)units, 256, 0, st>>>(from, to, layer, n, copies, (int)copy_pieces(from), units);
  return hipGetLastError();
}

}  // namespace iwdft
