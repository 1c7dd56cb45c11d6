// Attention over pages that sequences share: every page is read once for all sequences that hold it.
//
// A run is a range of places in the table and the sequences that hold the same pages there, as many as there are and the same ones from its first place to
// its last.  The rows of all of them -- (new token, query head of the KV head) -- go through the run's tokens together: blocks of rows and parts of
// tokens, as pages_rows.h has them.  A row's runs follow each other along its sequence, so its softmax is joined from their parts:
//   m = max m_i,  o = sum 2^(m_i - m) o_i / sum 2^(m_i - m) l_i.
// Who shares what is read off the table, whatever brought it about: the plan.  It is made once a step, for all layers:
//   1. for every place the sequences that hold the same page there, named by the first of them; where a set begins, ends or changes;
//   2. the runs, cut into parts of about the same work, and where their rows, parts and sums lie;
//   3. for every run its rows, for every sequence its runs, for every workgroup what it does.
// Tables without an order in what they share -- pages at several places, sets that change at every place -- have more runs than the plan holds; then nothing is
// shared, and the result is the same.
#include "pages_rows.h"

namespace iwdft {

namespace {

// ------------------------------------------------------------------------------------------------ the plan
constexpr int kPlaces = 4;         // of a wave in the first launch
// Parts of a call: two workgroups on each CU, as iwdft_pages_attn has them; a second one from parts of 8 tiles (few rows 16) on.  64 requests of 480 rows over 32768 tokens:
// many_rows with 256 parts 145 us, 512 130, 1024 141.
constexpr int kSharedParts = 512;
// Runs of up to so many rows go to few_rows, in blocks of 32 (fp32 16), the others to many_rows.  us, plan included, with up to 64 / up to 128 there (bf16, 8 heads): 60 rows over 65536
// tokens 71.5 / 72.6 (with up to 32 75.2; fp32 100 / 99, 132); 92 rows over 65536 78 / 97; 120 over 8192 48.6 / 45.1, over 32768 63.0 / 70.2, over 131072 128 / 184.
constexpr int kSharedFew = 64;
constexpr int kPlanMark = 0x49574446;
constexpr int kFlat = kWave;  // parts of a row that are listed for it

struct PlanHead {
  int32_t mark, n_layers, H, G, logP, max_pages, batch, n_tokens, n_sink, n_recent, few_rows;
  int32_t n_runs, many, few, slots, unshared;  // items of each kind; rows of sums of a (layer, head)
};
struct Run {
  int32_t leader, from, to, tokens;  // whose row of the table, places, new tokens of all its sequences
  int32_t mem, item, np, slot;       // first entry of the rows, first item, parts, first row of sums
};
struct Item {
  int32_t leader, from, to, mem;
  int32_t row0, rows, part, np;
  int32_t slot, unused[3];
};
static_assert(sizeof(PlanHead) == 64 && sizeof(Run) == 32 && sizeof(Item) == 48, "");

struct PlanSizes {
  int places, chunks, events, chain;
  int64_t mem, items, slots;
};
// Rows of sums of all (layer, head) that a call has room for, four for each row and what cutting adds to few: every row goes through them, one with a single part too.
int64_t most_slots(const Pages& S, int n_layers, int n_tokens) {
  const int64_t rows = (int64_t)n_tokens * S.G;
  return (2 * kSharedParts + 64) * std::min<int64_t>(128, (rows + 15) / 16 * 16) + 4 * rows * n_layers * S.H;
}
PlanSizes sizes_of(const Pages& S, int n_layers, int batch, int n_tokens) {
  PlanSizes z;
  z.places = (S.max_pages + kPlaces - 1) / kPlaces * kPlaces;
  z.chunks = z.places / kPlaces;
  z.events = 3 * batch;
  z.chain = std::min(S.max_pages, z.events);
  z.mem = n_tokens + std::min<int64_t>((int64_t)n_tokens * std::min(S.max_pages, batch), 1 << 20);
  z.slots = most_slots(S, n_layers, n_tokens) / ((int64_t)n_layers * S.H);
  z.items = std::min(z.mem * S.G / 16 + z.events + 2 * (2 * kSharedParts + 64), z.slots);  // each has a row of sums
  return z;
}
struct Plan {
  PlanHead* head;
  Item* items;
  Run* runs;
  int4* chain;       // [sequence][chain]: first row of sums, parts, rows of a part
  int2* mem;         // (row of q, position)
  int4* events;      // [chunk][events]: sequence and place; of the set that begins with it there, new tokens (-1: none does) and the least position of one
  uint16_t* names;   // [sequence][places]: the first sequence that holds the same page there
  int32_t *counts, *chained;  // events of a chunk; runs of a sequence
  int4* owner;                // of a row of q: its sequence (-1: none), which of its new tokens it is, its parts
  int32_t* flat;              // [row of q][kFlat]: the first row of sums of each of its parts, where they are no more
};
template <class Take>
void lay_out(const PlanSizes& z, int batch, int n_tokens, Plan* p, Take take) {
  p->head = (PlanHead*)take(sizeof(PlanHead));
  p->items = (Item*)take(z.items * sizeof(Item));
  p->runs = (Run*)take(z.events * sizeof(Run));
  p->chain = (int4*)take((size_t)batch * z.chain * sizeof(int4));
  p->mem = (int2*)take(z.mem * sizeof(int2));
  p->events = (int4*)take((size_t)z.chunks * z.events * sizeof(int4));
  p->names = (uint16_t*)take((size_t)batch * z.places * sizeof(uint16_t));
  p->counts = (int32_t*)take(z.chunks * sizeof(int32_t));
  p->chained = (int32_t*)take(batch * sizeof(int32_t));
  p->owner = (int4*)take(n_tokens * sizeof(int4));
  p->flat = (int32_t*)take((size_t)n_tokens * kFlat * sizeof(int32_t));
}

struct PlanArgs {
  Pages S;
  int32_t n_layers, batch, n_tokens, n_sink, n_recent, few_rows;
  const int32_t *starts, *table, *lens;
  PlanSizes z;
  Plan p;
};
struct News {
  int len, first, n;  // tokens, first new one (row of q), new ones
};
__device__ __forceinline__ News news_of(const PlanArgs& a, int b) {
  News s;
  s.len = min(max(a.lens[b], 0), a.S.max_pages << a.S.logP);
  s.first = min(max(a.starts[b], 0), a.n_tokens);
  s.n = min(max(a.starts[b + 1], s.first), a.n_tokens) - s.first;
  return s;
}
__device__ __forceinline__ int pages_of_news(const PlanArgs& a, const News& s) { return s.n ? page_count(s.len, a.S.logP) : 0; }  // who brings nothing is not asked
__device__ __forceinline__ void in_wave() {  // LDS that the lanes of a wave exchange
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wave has kPlaces places, and looks at the one before them; its lanes have the sequences in turn.  Equal pages meet in a hash table in LDS: one look-up for each
// sequence, whoever shares with whom.  A chain of loads and five rounds through LDS: 16 sequences of 272 pages 4.6 us, 64 of 528 6.2, 256 of 144 13.
template <int EACH, int WAVES>
__global__ __launch_bounds__(WAVES* kWave) void plan_sets_kernel(PlanArgs a) {
  constexpr int kRows = EACH * kWave, kSlots = 2 * kRows;
  __shared__ int32_t keys[WAVES][kSlots], firsts[WAVES][kSlots], tokens[WAVES][kRows], least[WAVES][kRows], changes[WAVES][kRows];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, chunk = blockIdx.x * WAVES + wave, c0 = chunk * kPlaces;
  for (int64_t t = (int64_t)blockIdx.x * (WAVES * kWave) + threadIdx.x; t < a.n_tokens; t += (int64_t)gridDim.x * (WAVES * kWave)) a.p.owner[t] = make_int4(-1, 0, 0, 0);
  if (chunk >= a.z.chunks) return;
  int pages[EACH], news[EACH], begin[EACH], most = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int x = lane + kWave * i;
    const News s = x < a.batch ? news_of(a, x) : News{0, 0, 0};
    pages[i] = pages_of_news(a, s), news[i] = s.n, begin[i] = s.len - s.n, most = max(most, pages[i]);
  }
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) most = max(most, __shfl_xor(most, d));
  int n = 0;
  if (c0 < most) {
    int prev[EACH], entry[EACH][kPlaces + 1];  // pages of the places, the one before them first
    uint32_t name[EACH][kPlaces / 2];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      prev[i] = -2;
#pragma unroll
      for (int c = 0; c < kPlaces / 2; ++c) name[i][c] = 0xffffffffu;
      const int32_t* at = a.table + (int64_t)(lane + kWave * i) * a.S.max_pages + c0;
#pragma unroll
      for (int c = 0; c <= kPlaces; ++c) entry[i][c] = c0 + c - 1 >= 0 && c0 + c - 1 < pages[i] ? at[c - 1] : -1;
    }
#pragma unroll
    for (int cc = -1; cc < kPlaces; ++cc) {
      const int c = c0 + cc;
      if (c < 0 || c >= most) continue;
      for (int i = lane; i < kSlots; i += kWave) keys[wave][i] = -1, firsts[wave][i] = kRows;
      for (int i = lane; i < kRows; i += kWave) tokens[wave][i] = 0, least[wave][i] = 0x7fffffff, changes[wave][i] = 0;
      in_wave();
      int cur[EACH], at[EACH];
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        const int x = lane + kWave * i;
        cur[i] = -1, at[i] = -1;
        if (c < pages[i]) {
          const int page = entry[i][cc + 1];
          cur[i] = x;  // a page that is not there is shared with nobody
          if ((uint32_t)page < (uint32_t)a.S.n_pages) {
            uint32_t s = ((uint32_t)page * 2654435769u) >> 8;
            for (;; ++s) {  // there are twice as many slots as sequences
              s &= kSlots - 1;
              const int was = atomicCAS(&keys[wave][s], -1, page);
              if (was == -1 || was == page) break;
            }
            atomicMin(&firsts[wave][s], x);
            at[i] = (int)s;
          }
        }
      }
      in_wave();
#pragma unroll
      for (int i = 0; i < EACH; ++i)
        if (at[i] >= 0) cur[i] = firsts[wave][at[i]];
      if (cc >= 0) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
          if (cur[i] == prev[i]) continue;
          if (cur[i] >= 0) changes[wave][cur[i]] = 1;
          if (prev[i] >= 0) changes[wave][prev[i]] = 1;
        }
        in_wave();
#pragma unroll
        for (int i = 0; i < EACH; ++i)
          if (cur[i] >= 0 && changes[wave][cur[i]]) atomicAdd(&tokens[wave][cur[i]], news[i]), atomicMin(&least[wave][cur[i]], begin[i]);
        in_wave();
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
          const int x = lane + kWave * i;
          const bool leads = cur[i] == x, event = changes[wave][x] && (leads || (prev[i] == x && cur[i] >= 0));  // where its row ends is known
          const unsigned long long m = __ballot(event);
          const int to = n + __popcll(m & ((1ull << lane) - 1));
          if (event && to < a.z.events) a.p.events[(int64_t)chunk * a.z.events + to] = make_int4(x | cc << 16, leads ? tokens[wave][x] : -1, least[wave][x], 0);
          n += __popcll(m);
          name[i][cc / 2] = cc % 2 ? (name[i][cc / 2] & 0xffffu) | (uint32_t)cur[i] << 16 : (name[i][cc / 2] & 0xffff0000u) | ((uint32_t)cur[i] & 0xffffu);
        }
        in_wave();
      }
#pragma unroll
      for (int i = 0; i < EACH; ++i) prev[i] = cur[i];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int x = lane + kWave * i;
      if (x < a.batch) *(uint2*)(a.p.names + (int64_t)x * a.z.places + c0) = make_uint2(name[i][0], name[i][1]);
    }
  }
  if (lane == 0) a.p.counts[chunk] = n;
}

// Tokens of a run that rows from position p on see: the work is shared out by it.
__device__ __forceinline__ int tokens_seen(const PlanArgs& a, int t0, int t1, int p) {
  if (!a.n_recent) return t1 - t0;
  const int near = max(t1 - max(t0, max(p, 0) - min(a.n_recent, max(p, 0))), 0), sinks = max(min(t1, a.n_sink) - t0, 0);
  return min(near + sinks, t1 - t0);
}

// One workgroup: the runs from the events, which lie in the order of their places.  Sums over 16 waves cost more than a few turns of 4: up to 256 sequences 256 threads (us with the
// attention, 256 / 1024: 256 sequences with 16 beginnings 87 / 95, 100 nested ones 49 / 55; 1000 sequences with 40 beginnings 209 / 134).  16 sequences 7 us, 64 8.  (All three launches
// in one, for tables of 128 pages: 29 us with the attention, 25 so; every load would wait for the one workgroup's own.)
constexpr int kGoesBack = 1 << 30;  // more than rows; starts that ascend have no more new tokens than there are rows
template <int THREADS, int BATCH>
__global__ __launch_bounds__(THREADS) void plan_share_kernel(PlanArgs a) {
  static_assert(BATCH <= THREADS, "");
  constexpr int kEvents = 3 * BATCH;  // where a set begins or ends; sequences that fork have fewer than 3 each
  __shared__ __attribute__((aligned(16))) int32_t leader[kEvents], from[kEvents];
  __shared__ int32_t news[kEvents], tiles[kEvents], least[kEvents], base[THREADS];
  __shared__ long long lds2[THREADS / kWave][2], lds4[THREADS / kWave][4];
  __shared__ float lds_f[THREADS / kWave][4];
  __shared__ int32_t longest[THREADS / kWave];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const float slices = (float)(a.n_layers * a.S.H);
  int n = 0, chunks = a.z.chunks;
  bool unshared = false;
  for (int c0 = 0; c0 < chunks; c0 += THREADS) {
    const int c = c0 + tid, mine = c < chunks ? a.p.counts[c] : 0;
    int x[2] = {mine, 0};
    if (c0 == 0) {
      int most = 0;
      for (int b = tid; b < a.batch; b += THREADS) {
        const News s = news_of(a, b);
        x[1] += a.starts[b + 1] < a.starts[b] ? kGoesBack : s.n, most = max(most, pages_of_news(a, s));  // one sequence a thread
      }
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) most = max(most, __shfl_xor(most, d));
      if (lane == 0) longest[wave] = most;
    }
    long long before[2], all[2];
    sums_before<THREADS>(x, before, all, lds2);
    if (c0 == 0) {  // of a wide table only what sequences have
      int most = 0;
#pragma unroll
      for (int w = 0; w < THREADS / kWave; ++w) most = max(most, longest[w]);
      chunks = min(chunks, (most + kPlaces - 1) / kPlaces);
    }
    if (c0 == 0 && all[1] > a.n_tokens) {  // starts that go back: where rows would belong to several sequences nothing is done
      bool twice = false;
      for (int b = tid; b < a.batch; b += THREADS) {
        const News s = news_of(a, b);
        for (int y = 0; y < b && s.n; ++y) {
          const News o = news_of(a, y);
          twice |= s.first < o.first + o.n && o.first < s.first + s.n && o.n;
        }
      }
      if (__syncthreads_or(twice)) {
        if (tid == 0) *a.p.head = PlanHead{};
        return;
      }
    }
    unshared = __syncthreads_or(mine > a.z.events) || n + all[0] > a.z.events;
    if (unshared) break;
    base[tid] = (int)before[0];
    __syncthreads();
    for (int e = tid; e < (int)all[0]; e += THREADS) {
      int lo = 0, hi = THREADS;  // largest with base <= e
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (base[m] <= e) lo = m;
        else hi = m;
      }
      const int4 v = a.p.events[(int64_t)(c0 + lo) * a.z.events + e - base[lo]];
      leader[n + e] = v.x & 0xffff, from[n + e] = (c0 + lo) * kPlaces + (v.x >> 16), news[n + e] = v.y, least[n + e] = v.z;
    }
    n += (int)all[0];
    __syncthreads();
  }
  for (;; unshared = true) {
    if (unshared) {
      __syncthreads();
      n = a.batch;
      for (int i = tid; i < n; i += THREADS) leader[i] = i, from[i] = 0, news[i] = news_of(a, i).n, least[i] = news_of(a, i).len - news[i];
      __syncthreads();
    }
    const auto end_of = [&](int i) {  // where its leader's next event is, or its row ends
      const int mine = leader[i];
      int end = pages_of_news(a, news_of(a, mine));
      if (unshared) return end;
#pragma unroll 4
      for (int k = i / 4 * 4; k < n; k += 4) {
        const int4 l = *(const int4*)(leader + k), f = *(const int4*)(from + k);
        const auto next = [&](int c, int lead, int at) { end = k + c > i && k + c < n && lead == mine ? min(end, at) : end; };
        next(0, l.x, f.x), next(1, l.y, f.y), next(2, l.z, f.z), next(3, l.w, f.w);
      }
      return end;
    };
    const auto rows_of = [&](int i) { return max(news[i], 0) * a.S.G; };
    const auto is_many = [&](int rows) { return rows > kSharedFew; };
    const auto blocks_of = [&](int rows) { return is_many(rows) ? (rows + Many::rows - 1) / Many::rows : (rows + a.few_rows - 1) / a.few_rows; };
    float sums[4] = {0.f, 0.f, 0.f, 0.f};  // tiles times blocks and blocks, of the few and of the many
    int to = 0;
    for (int i = tid; i < n; i += THREADS) {
      const int rows = rows_of(i), tile = is_many(rows) ? Many::tile : Few<1>::tile;
      to = end_of(i);
      const int seen = tokens_seen(a, from[i] << a.S.logP, to << a.S.logP, least[i]);
      tiles[i] = to > from[i] && rows ? max((seen + tile - 1) / tile, 1) : 0;
      const float blocks = tiles[i] ? (float)blocks_of(rows) : 0.f;
      const bool many = is_many(rows);
      sums[0] += many ? 0.f : blocks * (float)tiles[i], sums[1] += many ? 0.f : blocks;
      sums[2] += many ? blocks * (float)tiles[i] : 0.f, sums[3] += many ? blocks : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) sums[k] += __shfl_xor(sums[k], d);
      if (lane == 0) lds_f[wave][k] = sums[k];
    }
    __syncthreads();
    float per[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float sum = 0.f, blocks = 0.f;
#pragma unroll
      for (int w = 0; w < THREADS / kWave; ++w) sum += lds_f[w][2 * k], blocks += lds_f[w][2 * k + 1];
      sum *= slices, blocks *= slices;
      const float alone = fminf(ceilf(sum / (float)kCus), (float)(k ? Many::pair : Few<1>::pair));
      per[k] = fminf(fmaxf(fmaxf((float)kLeastTiles, alone), ceilf(sum / fmaxf((float)kSharedParts - blocks, 0.5f * kSharedParts))), 1e9f);
    }
    // where everything lies, items of the many first; longer parts where the sums of all of them would not fit
    struct Place {
      int np;
      long long mem, many, few, slot;
    };
    long long sum[4];  // rows, items of the many and of the few, rows of sums
    const auto places = [&](int i, long long (&done)[4]) {  // of run i of this thread, behind `done`
      const bool there = i < n && tiles[i];
      const int rows = there ? rows_of(i) : 0;
      const bool many = is_many(rows);
      const int np = there ? max(1, (int)ceilf((float)tiles[i] / (many ? per[1] : per[0]))) : 0;
      const int items = (int)min((long long)blocks_of(rows) * np, 0x3fffffffll);
      const int x[4] = {there ? news[i] : 0, many ? items : 0, many ? 0 : items, (int)min((long long)rows * np, 0x7fffffffll)};
      long long before[4], all[4];
      sums_before<THREADS>(x, before, all, lds4);
      const Place p{np, done[0] + before[0], done[1] + before[1], done[2] + before[2], done[3] + before[3]};
#pragma unroll
      for (int c = 0; c < 4; ++c) done[c] += all[c];
      return p;
    };
    Place p{};
    for (;;) {
      sum[0] = sum[1] = sum[2] = sum[3] = 0;
      for (int i0 = 0; i0 < n; i0 += THREADS) p = places(i0 + tid, sum);
      if ((sum[3] <= a.z.slots && sum[1] + sum[2] <= a.z.items) || per[0] > 1e8f) break;
      per[0] *= 2.f, per[1] *= 2.f;
    }
    if (!unshared && (sum[3] > a.z.slots || sum[1] + sum[2] > a.z.items || sum[0] > a.z.mem)) continue;
    long long done[4] = {0, 0, 0, 0};
    for (int i0 = 0; i0 < n; i0 += THREADS) {
      const int i = i0 + tid;
      if (n > THREADS) p = places(i, done), to = i < n ? end_of(i) : 0;
      if (i < n) {
        const bool many = is_many(rows_of(i));
        a.p.runs[i] = Run{leader[i], from[i], p.np ? to : from[i], p.np ? news[i] : 0, (int)p.mem, (int)(many ? p.many : sum[1] + p.few), p.np, (int)p.slot};
      }
    }
    if (tid == 0)
      *a.p.head = PlanHead{kPlanMark, a.n_layers, a.S.H, a.S.G, a.S.logP, a.S.max_pages, a.batch, a.n_tokens, a.n_sink, a.n_recent, a.few_rows,
                           n, (int)sum[1], (int)sum[2], (int)sum[3], unshared ? 1 : 0};
    return;
  }
}

// The first row of sums of part `part` of a row's runs, a lane for each run: x of the run that it is in -- which is how many end before it --, y parts of z rows; to: their sums.
__device__ __forceinline__ int part_slot(int4 run, int to, int runs, int part) {
  int which = 0;
  for (int c = 0; c < runs; ++c) which += __builtin_amdgcn_readlane(to, c) <= part;
  which = min(which, kWave - 1);
  return __shfl(run.x, which) + (part - (__shfl(to, which) - __shfl(run.y, which))) * __shfl(run.z, which);
}

// A wave for each sequence: its runs, in order, its rows in them and their parts.  A wave for each run: its items.  16 sequences 5 us, 12 with forty runs 9, 256 10.
__global__ __launch_bounds__(256) void plan_rows_kernel(PlanArgs a) {
  const int lane = threadIdx.x % kWave, unit = blockIdx.x * 4 + threadIdx.x / kWave;
  const PlanHead& head = *a.p.head;
  if (head.mark != kPlanMark) return;  // whose rows they are is not defined
  const int n = head.n_runs;
  const bool unshared = head.unshared != 0;
  const auto holds = [&](int x, const News& s, const Run& r) {
    return s.n > 0 && r.from < page_count(s.len, a.S.logP) && (unshared ? r.leader == x : (int)a.p.names[(int64_t)x * a.z.places + r.from] == r.leader);
  };
  if (unit < a.batch) {
    const int x = unit;
    const News s = news_of(a, x);
    int k = 0;
    for (int i0 = 0; i0 < n && s.n; i0 += kWave) {
      const int i = i0 + lane;
      const Run mine = i < n ? a.p.runs[i] : Run{};
      const bool member = mine.tokens > 0 && holds(x, s, mine);
      const unsigned long long in = __ballot(member);
      // its rows begin behind those of the sequences before it: a lane for each run, or for each sequence
      int before = 0;
      const bool each_run = !unshared && __popcll(in) * ((x + kWave - 1) / kWave) > x / 4;
      if (each_run && member) {
#pragma unroll 4
        for (int y = 0; y < x; ++y) {
          const News o = news_of(a, y);
          before += holds(y, o, mine) ? o.n : 0;
        }
      }
      for (unsigned long long rest = in; rest && !each_run && !unshared; rest &= rest - 1) {
        const int l = __builtin_ctzll(rest);
        Run r{};
        r.leader = __builtin_amdgcn_readlane(mine.leader, l), r.from = __builtin_amdgcn_readlane(mine.from, l);
        int sum = 0;
        for (int y = lane; y < x; y += kWave) {
          const News o = news_of(a, y);
          sum += holds(y, o, r) ? o.n : 0;
        }
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) sum += __shfl_xor(sum, d);
        before = lane == l ? sum : before;
      }
      const int at = k + __popcll(in & ((1ull << lane) - 1));
      if (member && at < a.z.chain) a.p.chain[(int64_t)x * a.z.chain + at] = make_int4(mine.slot + before * a.S.G, mine.np, mine.tokens * a.S.G, 0);
      if (s.n <= 4) {
        for (int t = 0; t < s.n; ++t)
          if (member && mine.mem + before + t < a.z.mem) a.p.mem[mine.mem + before + t] = make_int2(s.first + t, s.len - s.n + t);
      } else {
        for (unsigned long long rest = in; rest; rest &= rest - 1) {
          const int l = __builtin_ctzll(rest), to = __builtin_amdgcn_readlane(mine.mem + before, l);
          for (int t = lane; t < s.n; t += kWave)
            if (to + t < a.z.mem) a.p.mem[to + t] = make_int2(s.first + t, s.len - s.n + t);
        }
      }
      k += __popcll(in);
    }
    // all parts of its rows, run by run: a lane for each.  The lanes read what others of their wave have just stored.
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int4 run = lane < min(k, a.z.chain) ? a.p.chain[(int64_t)x * a.z.chain + lane] : make_int4(0, 0, 0, 0);
    const int to = scan(run.y), parts = k > kFlat ? kFlat + 1 : last_lane(to);
    const int first = part_slot(run, to, min(k, kFlat), lane);
    for (int t = 0; t < s.n && parts <= kFlat; ++t)
      if (lane < parts) a.p.flat[(int64_t)(s.first + t) * kFlat + lane] = first + t * a.S.G;
    for (int t = lane; t < s.n; t += kWave) a.p.owner[s.first + t] = make_int4(x, t, parts, 0);
    if (lane == 0) a.p.chained[x] = min(k, a.z.chain);
  } else {
    const int waves = gridDim.x * 4 - a.batch;
    for (int i = unit - a.batch; i < n; i += waves) {
      const Run r = a.p.runs[i];
      const int rows = r.tokens * a.S.G, size = rows > kSharedFew ? Many::rows : a.few_rows, blocks = (rows + size - 1) / size;
      for (int k = lane; k < blocks * r.np; k += kWave) {
        if (r.item + k >= a.z.items) break;
        const int part = k / blocks, block = blocks - 1 - (k - part * blocks), row0 = block * size;  // blocks that read the same tokens side by side
        a.p.items[r.item + k] = Item{r.leader, r.from, r.to, r.mem, row0, min(size, rows - row0), part, r.np, r.slot + part * rows + row0, {0, 0, 0}};
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ attention
struct SharedAttn {
  PagesAttn a;
  Plan p;
  PlanSizes z;
  int32_t few_rows;
  float* part;
  float2* stat;
};
__device__ __forceinline__ bool is_for(const PlanHead& h, const SharedAttn& s) {
  const PagesAttn& a = s.a;
  return h.mark == kPlanMark && h.n_layers == a.n_layers && h.H == a.S.H && h.G == a.S.G && h.logP == a.S.logP && h.max_pages == a.S.max_pages && h.batch == a.batch &&
         h.n_tokens == a.n_tokens && h.n_sink == a.n_sink && h.n_recent == a.n_recent && h.few_rows == s.few_rows;
}

// The items of one kind: see pages_rows.h for what the kernels ask.  A short part is a chain: plan, item, rows (0.5 us), table and first tokens (0.9), queries (2), four tiles for each
// wave (5.5, vector work as much as waiting: a second tile ahead is slower), sums through LDS (1.5 to 2).  Long parts of many rows run at what the products and conversions of
// many_rows reach: two workgroups of 128 rows on a CU 1.28 us a tile of 64 tokens each, 840 TFLOP/s.  (The kinds taking turns on the CUs, a workgroup of each, gains nothing: 130 us for 127.)
class Items {
 public:
  static constexpr bool looks_up = true;
  __device__ __forceinline__ float* part() const { return s.part; }
  __device__ __forceinline__ float2* stat() const { return s.stat; }

  __device__ __forceinline__ Items(const SharedAttn& s, bool many, int lane)
      : s(s), lane(lane), first(many ? 0 : s.p.head->many), n(many ? s.p.head->many : s.p.head->few), slots(s.p.head->slots),
        slices((uint32_t)(s.a.n_layers * s.a.S.H)) {}

  struct Block {
    const int32_t* table;
    int layer, h, rows, p_lo, p_hi, from_lo, hi, part, np, last_page, base, last_token, mem, row0, lh, slot;
    static constexpr bool whole = false;
    __device__ __forceinline__ int from_hi(const PagesAttn& a) const { return window_from(a, hi); }
  };
  __device__ __forceinline__ uint32_t count() const { return (uint32_t)n * slices; }
  __device__ __forceinline__ Block block(uint32_t x) const {
    const PagesAttn& a = s.a;
    const int4* at = (const int4*)(s.p.items + first + x / slices);
    const int4 u = at[0], v = at[1], w = at[2];
    Block k;
    k.lh = (int)(x % slices), k.layer = (int)((uint32_t)k.lh / (uint32_t)a.S.H), k.h = k.lh - k.layer * a.S.H;
    const auto uni = [](int y) { return __builtin_amdgcn_readfirstlane(y); };
    k.table = a.table + (int64_t)uni(u.x) * a.S.max_pages, k.base = uni(u.y) << a.S.logP, k.last_page = uni(u.z) - 1, k.last_token = (uni(u.z) << a.S.logP) - 1;
    k.mem = uni(u.w), k.row0 = uni(v.x), k.rows = uni(v.y), k.part = uni(v.z), k.np = uni(v.w), k.slot = uni(w.x);
    int lo = 0x7fffffff, hi = -1;
    for (int r = lane; r < k.rows; r += kWave) {
      const int p = max(s.p.mem[k.mem + (int)((uint32_t)(k.row0 + r) / (uint32_t)a.S.G)].y, -1);
      lo = min(lo, p), hi = max(hi, p);
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) lo = min(lo, __shfl_xor(lo, d)), hi = max(hi, __shfl_xor(hi, d));
    lo = uni(lo), hi = uni(hi);
    k.from_lo = window_from(a, lo), k.hi = hi, k.p_lo = min(lo, k.last_token), k.p_hi = min(hi, k.last_token);
    return k;
  }
  __device__ __forceinline__ RowAt row(const Block& k, int r) const {
    const PagesAttn& a = s.a;
    const uint32_t m = (uint32_t)(k.row0 + min(r, k.rows - 1)), G = (uint32_t)a.S.G;
    const int token = (int)(m / G);
    const int2 at = s.p.mem[k.mem + token];
    const int pos = max(at.y, -1);
    return RowAt{((int64_t)k.layer * a.n_tokens + at.x) * (a.S.H * a.S.G) + k.h * a.S.G + (int)(m - (uint32_t)token * G), min(pos, k.last_token), window_from(a, pos)};
  }
  __device__ __forceinline__ WaveRows wave_rows(const Block& k, int wave) const { return WaveRows{32 * wave < k.rows ? k.p_hi : -1, k.from_lo}; }
  __device__ __forceinline__ int64_t slot(const Block& k) const { return (int64_t)k.lh * slots + k.slot; }

 private:
  const SharedAttn& s;
  int lane, first, n, slots;
  uint32_t slices;
};

template <bool BF16, int R, bool MANY>
__global__ __launch_bounds__(kWaves* kWave, BF16 ? 2 : (R == 1 && !MANY ? 2 : 1)) void shared_attn_kernel(SharedAttn s) {
  if (!is_for(*s.p.head, s)) return;
  uint32_t x = blockIdx.x;
  if constexpr (MANY) {
    const uint32_t n = many_rows<BF16>(s.a, Items(s, true, threadIdx.x % kWave), x, gridDim.x);
    if (x < n) x += (n - x + gridDim.x - 1) / gridDim.x * gridDim.x;  // its next turn
    x -= n;
  }
  if constexpr (R > 0) few_rows<BF16, R, kWaves>(s.a, Items(s, false, threadIdx.x % kWave), x, gridDim.x);
}

// A row's parts: the plan lists where the sums of up to 64 of them are; of more they are found from its runs, a lane for each.  A lane for each part reads its reference, then all
// sums are on their way at once.  Bound by loads that wait for each other: 480 rows of 17 parts 5.8 us (6.7 with the runs looked up for every row); beams of twenty runs, 17 MB, 9.8
// (run by run and part by part, each rescaling the last, 15.5).
// Few rows: a workgroup for each, its waves share the parts.  Many: a wave for each (3840 rows of 17 parts, 34 MB: 14.9 and 11.4 us; 2048 rows 7.2 and 7.9; 736 rows of beams
// 10.3 and 20); all of these have 17 to 20 parts a row.
constexpr int64_t kManyShared = 2048;
template <bool BF16>
__global__ __launch_bounds__(kWaves* kWave) void shared_join_kernel(SharedAttn s, int64_t all, int many) {
  __shared__ float2 sums[kWaves][kWave], stats[kWaves];
  const PagesAttn& a = s.a;
  const bool fits = is_for(*s.p.head, s);  // looked at together with the row, whose loads do not wait for it
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), slots = s.p.head->slots, G = a.S.G;
  const uint32_t row_heads = (uint32_t)(a.n_tokens * G);
  for (uint32_t x = many ? blockIdx.x * kWaves + wave : blockIdx.x; x < (uint32_t)all; x += gridDim.x * (many ? kWaves : 1)) {
    const int lh = (int)(x / row_heads), r = (int)(x - (uint32_t)lh * row_heads), token = (int)((uint32_t)r / (uint32_t)G);
    const int4 owner = s.p.owner[token];
    const int listed = s.p.flat[(int64_t)token * kFlat + lane];
    const int b = __builtin_amdgcn_readfirstlane(owner.x), listed_parts = __builtin_amdgcn_readfirstlane(owner.z);
    if (!fits || b < 0) continue;  // behind the last sequence
    float m = -FLT_MAX, l = 0.f;
    float2 o = make_float2(0.f, 0.f);
    const auto add = [&](float top, float2 v, float sum, float half) {  // half: 2^(half of the reference's distance)
      const float up = fmaxf(m, top), f = __builtin_amdgcn_exp2f(0.5f * (m - up));
      o.x = o.x * (f * f) + v.x * (half * half), o.y = o.y * (f * f) + v.y * (half * half), l = l * f * f + sum * half * half, m = up;
    };
    const auto add_parts = [&](int64_t at, int here) {  // a lane for each
      const float2 st = lane < here ? s.stat[at] : make_float2(-FLT_MAX, 0.f);
      float top = st.x;
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
      const float up = fmaxf(m, top), g = __builtin_amdgcn_exp2f(0.5f * (st.x - up)), f = __builtin_amdgcn_exp2f(0.5f * (m - up));
      float sum = st.y * g * g;  // a denominator's share may need both factors
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) sum += __shfl_xor(sum, d);
      l = l * f * f + sum, o.x *= f * f, o.y *= f * f, m = up;
#pragma unroll 8
      for (int c = 0; c < here; ++c) {
        const int64_t row = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)at, c) | (int64_t)__builtin_amdgcn_readlane((int)(at >> 32), c) << 32;
        const float2 v = *(const float2*)(s.part + row * kHeadDim + 2 * lane);
        const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(g), c)), ww = w * w;
        o.x += v.x * ww, o.y += v.y * ww;
      }
    };
    const auto share = [&](int parts, auto slot_of) {  // those of this wave
      const int size = many ? kWave : min(kWave, (parts + kWaves - 1) / kWaves);
      for (int p0 = many ? 0 : wave * size; p0 < parts; p0 += size * (many ? 1 : kWaves)) add_parts((int64_t)lh * slots + (r - token * G) + slot_of(p0 + lane), min(parts - p0, size));
    };
    if (listed_parts <= kFlat) {
      share(listed_parts, [&](int part) { return __shfl(listed, min(part, kWave - 1)); });
    } else {
      const int n = s.p.chained[b];
      for (int i0 = 0; i0 < n; i0 += kWave) {
        const int4 run = i0 + lane < n ? s.p.chain[(int64_t)b * s.z.chain + i0 + lane] : make_int4(0, 0, 0, 0);
        const int to = scan(run.y);
        share(last_lane(to), [&](int part) { return part_slot(run, to, min(n - i0, kWave), part) + owner.y * G; });
      }
    }
    if (!many) {
      sums[wave][lane] = o;
      if (lane == 0) stats[wave] = make_float2(m, l);
      __syncthreads();
      m = -FLT_MAX, l = 0.f, o = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kWaves; ++i) add(stats[i].x, sums[i][lane], stats[i].y, __builtin_amdgcn_exp2f(0.5f * (stats[i].x - fmaxf(m, stats[i].x))));
      __syncthreads();
      if (wave) continue;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int layer = (int)((uint32_t)lh / (uint32_t)a.S.H), h = lh - layer * a.S.H;
    const int64_t to = (((int64_t)layer * a.n_tokens + token) * (a.S.H * G) + h * G + r - token * G) * kHeadDim + 2 * lane;
    if constexpr (BF16) *(uint32_t*)((uint16_t*)a.out + to) = (uint32_t)f32_to_bf16(result<true>(o.x, inv)) | (uint32_t)f32_to_bf16(result<true>(o.y, inv)) << 16;
    else *(float2*)((float*)a.out + to) = make_float2(result<false>(o.x, inv), result<false>(o.y, inv));
  }
}

int few_rows_of(const Pages& S, int n_tokens, bool bf16) { return bf16 && (int64_t)n_tokens * S.G > 16 ? 32 : 16; }

Plan plan_at(const PlanSizes& z, int batch, int n_tokens, void* at) {
  Plan p;
  size_t done = 0;
  lay_out(z, batch, n_tokens, &p, [&](size_t bytes) {
    char* here = (char*)at + done;
    done += (bytes + 255) / 256 * 256;
    return here;
  });
  return p;
}

template <bool BF16, int R, bool MANY>
hipError_t launch_shared(const SharedAttn& s, hipStream_t st) {
  const int64_t lh = (int64_t)s.a.n_layers * s.a.S.H, rows = (int64_t)s.a.n_tokens * s.a.S.G;
  const int64_t grid = (MANY ? 2 : 1) * kSharedParts + lh * (2 * s.a.batch + rows / 32);
  shared_attn_kernel<BF16, R, MANY><<<(unsigned)std::min<int64_t>(grid, 1 << 20), kWaves * kWave, 0, st>>>(s);
  return hipGetLastError();
}

}  // namespace

size_t pages_plan_bytes(const Pages& S, int n_layers, int batch, int n_tokens) {
  Plan p;
  size_t done = 0;
  lay_out(sizes_of(S, n_layers, batch, n_tokens), batch, n_tokens, &p, [&](size_t bytes) {
    done += (bytes + 255) / 256 * 256;
    return (void*)nullptr;
  });
  return done;
}
size_t pages_shared_bytes(const Pages& S, int n_layers, int batch, int n_tokens) {
  return batch == 0 || n_tokens == 0 ? 0 : (size_t)most_slots(S, n_layers, n_tokens) * (kHeadDim * sizeof(float) + sizeof(float2));
}

hipError_t launch_pages_plan(const PagesAttn& g, bool bf16, void* plan, hipStream_t st) {
  PlanArgs a{g.S, g.n_layers, g.batch, g.n_tokens, g.n_sink, g.n_recent, few_rows_of(g.S, g.n_tokens, bf16), g.starts, g.table, g.lens, {}, {}};
  a.z = sizes_of(g.S, g.n_layers, g.batch, g.n_tokens);
  a.p = plan_at(a.z, g.batch, g.n_tokens, plan);
  const auto grid = [&](int waves) { return (unsigned)((a.z.chunks + waves - 1) / waves); };
  if (g.batch <= kWave) plan_sets_kernel<1, 4><<<grid(4), 4 * kWave, 0, st>>>(a);
  else if (g.batch <= 4 * kWave) plan_sets_kernel<4, 4><<<grid(4), 4 * kWave, 0, st>>>(a);
  else plan_sets_kernel<16, 2><<<grid(2), 2 * kWave, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (g.batch <= kWave) plan_share_kernel<256, kWave><<<1, 256, 0, st>>>(a);
  else if (g.batch <= 4 * kWave) plan_share_kernel<256, 4 * kWave><<<1, 256, 0, st>>>(a);
  else plan_share_kernel<1024, kSharedBatch><<<1, 1024, 0, st>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  plan_rows_kernel<<<(unsigned)((2 * g.batch + 64 + 3) / 4), 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_pages_shared(const PagesAttn& g, bool bf16, const void* plan, void* ws, hipStream_t st) {
  SharedAttn s{};
  s.a = g, s.z = sizes_of(g.S, g.n_layers, g.batch, g.n_tokens), s.p = plan_at(s.z, g.batch, g.n_tokens, (void*)plan);
  s.few_rows = few_rows_of(g.S, g.n_tokens, bf16);
  s.part = (float*)ws, s.stat = (float2*)(s.part + most_slots(g.S, g.n_layers, g.n_tokens) * kHeadDim);
  const int64_t rows = (int64_t)g.n_tokens * g.S.G;
  hipError_t e;
  if (bf16) e = rows <= 16 ? launch_shared<true, 1, false>(s, st) : rows <= kSharedFew ? launch_shared<true, 2, false>(s, st) : launch_shared<true, 2, true>(s, st);
  else {
    e = rows > kSharedFew ? launch_shared<false, 0, true>(s, st) : hipSuccess;
    if (e == hipSuccess) e = launch_shared<false, 1, false>(s, st);
  }
  if (e != hipSuccess) return e;
  const int64_t all = rows * g.n_layers * g.S.H;
  const bool many = all > kManyShared;
  const unsigned grid = (unsigned)std::min<int64_t>(many ? (all + kWaves - 1) / kWaves : all, 4096);
  if (bf16) shared_join_kernel<true><<<grid, kWaves * kWave, 0, st>>>(s, all, many);
  else shared_join_kernel<false><<<grid, kWaves * kWave, 0, st>>>(s, all, many);
  return hipGetLastError();
}

}  // namespace iwdft
