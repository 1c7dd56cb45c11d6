// Attention of new tokens over the 8-bit pages of their sequences: the kernels of pages_rows.h with each sequence's own rows and tokens.
#include "pages_rows.h"

namespace iwdft {

namespace {

// ------------------------------------------------------------------------------------------------ sharing out the work
// A block is `rows` consecutive (new token, query head of the KV head) pairs of a sequence; its tokens are cut into parts, one workgroup each, such that
// all parts of a call hold about the same number of tiles and, up to parts / 2 blocks, there are about `parts` of them: two workgroups on each CU (more would run
// alone in the end: 16 contexts of 4096 to 16384 tokens 90 us, with the blocks' last, shorter parts counted in 78, 71 with what is below).  More blocks make more parts, and
// the two kinds of rows count for themselves.  Lengths live on the device, so every wave works out the shares by itself, 64 sequences at a time: the launch only has to be large enough.
// The kernels that leave a SIMD one wave (64 rows in bf16, 32 rows and prompts in fp32) run 256 workgroups at a time, so 512 parts are two rounds there; us with 512 / 256:
// one sequence of 65536 tokens and 48 rows 70 / 58, in fp32 20 rows 57 / 49; four of up to 16384 and 48 rows 28 / 33, 800 rows over 32768 in fp32 297 / 314, 4096 tokens' prompt 355 / 355.
// Short parts cost more in the join than the second workgroup on a CU gains: one token over 8192 tokens of 8 heads 14.3 us with parts of 4 tiles, 11.6 with 8,
// over 16000 17.3 with 8 and 15.1 with 16.
constexpr float kMostBlocks = 1100000000.f;  // 2^30 rows have fewer: starts that overlap, whose counts would not fit; such a call does nothing
constexpr int kFewRows = 64;  // sequences of up to so many rows go to few_rows, where a call may have both

struct Seq {
  int len, first, nq, rows, tiles;  // tokens, first new token (row of q), new tokens, rows of all blocks, most tiles of a block
};
struct Shares {
  int tiles;       // of a part
  int parts;       // of all sequences, for one (layer, KV head)
  int split;       // ... of blocks that are cut
  int split_rows;  // rows of sequences whose blocks are cut
};
// The sequence that holds entry y of a numbering that gives every sequence some entries: its index, y's place in it, its blocks' parts, and how
// many parts of cut blocks the sequences before it have.
struct Place {
  int b, at, before, np;
  Seq s;
};

__device__ __forceinline__ float scan(float x) {
  const auto add = [](float y, int z) { return y + __int_as_float(z); };
  x = add(x, from_lane<0x111, 0xf>(__float_as_int(x))), x = add(x, from_lane<0x112, 0xf>(__float_as_int(x)));
  x = add(x, from_lane<0x114, 0xf>(__float_as_int(x))), x = add(x, from_lane<0x118, 0xf>(__float_as_int(x)));
  x = add(x, from_lane<0x142, 0xa>(__float_as_int(x)));
  return add(x, from_lane<0x143, 0xc>(__float_as_int(x)));
}

template <class Geo>
class Schedule {
 public:
  Shares w;

  __device__ __forceinline__ Schedule(const PagesAttn& args, const PagesRows& which, int lane) : a(args), which(which), lane(lane), head(load(lane)) {
    float sum = 0.f, all_blocks = 0.f;  // every wave adds in the same order: all agree
    each([&](int, const Seq& s) {
      const float n = (float)blocks(s.rows);
      sum += (float)s.tiles * n, all_blocks += n;
    });
    const float slices = (float)(a.n_layers * a.S.H);
    sum = __int_as_float(last_lane(__float_as_int(scan(sum)))) * slices;
    all_blocks = __int_as_float(last_lane(__float_as_int(scan(all_blocks)))) * slices;
    const float alone = fminf(ceilf(sum / (float)kCus), (float)Geo::pair);
    w.tiles = which.part ? (int)fminf(fmaxf(fmaxf((float)kLeastTiles, alone), ceilf(sum / fmaxf((float)Geo::parts - all_blocks, 0.5f * (float)Geo::parts))), 1e9f) : 0x7fffffff;
    int n = 0, cut = 0, cut_rows = 0;
    each([&](int, const Seq& s) {
      const int np = parts(s), all = np * blocks(s.rows);
      n += all;
      if (np > 1) cut += all, cut_rows += s.rows;
    });
    w.parts = last_lane(scan(n)), w.split = last_lane(scan(cut)), w.split_rows = last_lane(scan(cut_rows));
    if (all_blocks > kMostBlocks) w.parts = w.split = w.split_rows = 0;
  }

  static __device__ __forceinline__ int blocks(int rows) { return (rows + Geo::rows - 1) / Geo::rows; }
  __device__ __forceinline__ int parts(const Seq& s) const { return s.nq ? max(1, (int)(((uint32_t)s.tiles + (uint32_t)w.tiles - 1u) / (uint32_t)w.tiles)) : 0; }

  template <class Count>
  __device__ __forceinline__ Place find(int y, Count count) const {
    int done = 0, cut = 0;
    for (int b0 = 0;; b0 += kWave) {
      const Seq s = b0 == 0 && kHold ? head : load(b0 + lane);
      const int np = parts(s), n = count(s, np), c = np > 1 ? np * blocks(s.rows) : 0, in = scan(n), cin = scan(c);
      const unsigned long long m = __ballot(y < done + in);
      if (m || b0 + kWave >= a.batch) {  // always found: y is below the sum of all counts
        const int src = m ? __builtin_ctzll(m) : 0;
        const auto uni = [&](int x) { return __builtin_amdgcn_readlane(x, src); };
        return Place{b0 + src, y - done - uni(in - n), cut + uni(cin - c), uni(np), {uni(s.len), uni(s.first), uni(s.nq), uni(s.rows), uni(s.tiles)}};
      }
      done += last_lane(in), cut += last_lane(cin);
    }
  }

 private:
  const PagesAttn& a;
  const PagesRows& which;
  int lane;
  // The lane's sequence of the first 64; read again by the kernel of 64 rows, which has no registers left (12 tokens over 65536: 71.1 us with it held, 68.6 so).
  static constexpr bool kHold = Geo::rows != 64;
  Seq head;

  template <class Do>
  __device__ __forceinline__ void each(Do use) const {
    use(0, head);
    for (int b0 = kWave; b0 < a.batch; b0 += kWave) use(b0, load(b0 + lane));
  }

  __device__ __forceinline__ Seq load(int b) const {
    Seq s{0, 0, 0, 0, 0};
    if (b >= a.batch) return s;
    s.len = min(max(a.lens[b], 0), a.S.max_pages << a.S.logP);
    s.first = min(max(a.starts[b], 0), a.n_tokens);
    s.nq = min(max(a.starts[b + 1], s.first), a.n_tokens) - s.first;
    s.rows = s.nq * a.S.G;
    if (s.rows <= which.over || s.rows > which.to) s.nq = s.rows = 0;
    s.tiles = (s.len + Geo::tile - 1) / Geo::tile;
    if (a.n_recent) {
      const int sink = (min(a.n_sink, s.len) + Geo::tile - 1) / Geo::tile;
      const uint32_t span = (uint32_t)a.n_recent + (uint32_t)(min(s.nq, Geo::rows / a.S.G + 2) + 2 * Geo::tile);
      s.tiles = min(s.tiles, sink + (int)(span / (uint32_t)Geo::tile));
    }
    return s;
  }
};

// Blocks of a sequence's rows over its tokens.
template <class Geo>
class Sequences {
 public:
  static constexpr bool looks_up = false;
  __device__ __forceinline__ Sequences(const PagesAttn& a, const PagesRows& which, int lane) : a(a), which(which), plan(a, which, lane) {}
  __device__ __forceinline__ float* part() const { return which.part; }
  __device__ __forceinline__ float2* stat() const { return which.stat; }

  struct Block {
    static constexpr int base = 0;
    const int32_t* table;
    int layer, h, rows, p_lo, p_hi, from_lo, part, np, last_page, lh, slot, row0, first, before;
    bool whole;
    __device__ __forceinline__ int from_hi(const PagesAttn& a) const { return window_from(a, max(p_hi, -1)); }
  };
  __device__ __forceinline__ uint32_t count() const { return (uint32_t)plan.w.parts * slices(); }
  __device__ __forceinline__ Block block(uint32_t x) const {
    Block k;
    k.lh = (int)(x % slices());  // workgroups are dealt to the XCDs in turn: with 8 heads each reads one head's pages
    const Place at = plan.find((int)(x / slices()), [](const Seq& s, int np) { return np * Schedule<Geo>::blocks(s.rows); });
    const Seq& s = at.s;
    const int turn = (int)((uint32_t)at.at / (uint32_t)at.np), block = plan.blocks(s.rows) - 1 - turn;  // the longest first
    k.part = at.at - turn * at.np, k.np = at.np, k.whole = at.np == 1;
    k.layer = (int)((uint32_t)k.lh / (uint32_t)a.S.H), k.h = k.lh - k.layer * a.S.H;
    const uint32_t G = (uint32_t)a.S.G;
    k.row0 = block * Geo::rows, k.rows = min(s.rows - k.row0, Geo::rows);
    k.first = s.first, k.before = s.len - s.nq;  // position of the sequence's first new token
    k.p_lo = k.before + (int)((uint32_t)k.row0 / G), k.p_hi = k.before + (int)((uint32_t)(k.row0 + k.rows - 1) / G);
    k.from_lo = window_from(a, max(k.p_lo, -1));
    k.table = a.table + (int64_t)at.b * a.S.max_pages, k.last_page = max(page_count(s.len, a.S.logP) - 1, 0);
    k.slot = at.before + at.at;
    return k;
  }
  __device__ __forceinline__ RowAt row(const Block& k, int r) const {
    const uint32_t n = (uint32_t)(k.row0 + r), G = (uint32_t)a.S.G;  // of the sequence's rows
    const int token = (int)(n / G), pos = max(k.before + token, -1);
    return RowAt{((int64_t)k.layer * a.n_tokens + k.first + token) * (a.S.H * a.S.G) + k.h * a.S.G + (int)(n - (uint32_t)token * G), pos, window_from(a, pos)};
  }
  __device__ __forceinline__ WaveRows wave_rows(const Block& k, int wave) const {
    const int lo = k.before + (k.row0 + 32 * wave) / a.S.G;
    return WaveRows{32 * wave < k.rows ? k.before + (k.row0 + min(32 * wave + 32, k.rows) - 1) / a.S.G : -1, window_from(a, max(lo, -1))};
  }
  __device__ __forceinline__ int64_t slot(const Block& k) const { return ((int64_t)k.lh * plan.w.split + k.slot) * Geo::rows; }

 private:
  const PagesAttn& a;
  const PagesRows& which;
  const Schedule<Geo> plan;
  __device__ __forceinline__ uint32_t slices() const { return (uint32_t)(a.n_layers * a.S.H); }
};

// ------------------------------------------------------------------------------------------------ joining the parts
// Rows whose tokens were shared out.  Few of them: a workgroup for each, its waves take the parts in turn.  Many: a wave for each.
constexpr uint32_t kManyJoined = 4096;
template <bool BF16, class Geo>
__device__ __forceinline__ void join_rows(const PagesAttn& a, const PagesRows& which, uint32_t block_id) {
  constexpr int BR = Geo::rows;
  __shared__ float2 sums[kWaves][kWave], stats[kWaves];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const Schedule<Geo> plan(a, which, lane);
  const uint32_t slices = (uint32_t)(a.n_layers * a.S.H), all = (uint32_t)plan.w.split_rows * slices;
  const bool many = all > kManyJoined;
  const uint32_t step = many ? which.join_grid * kWaves : which.join_grid;
  for (uint32_t x = many ? block_id * kWaves + wave : block_id; x < all; x += step) {
    const int lh = (int)(x / (uint32_t)plan.w.split_rows);
    const Place at = plan.find((int)(x - (uint32_t)lh * (uint32_t)plan.w.split_rows), [](const Seq& s, int np) { return np > 1 ? s.rows : 0; });
    const int r = at.at, block = r / BR;
    const int64_t slot = (int64_t)lh * plan.w.split + at.before + (plan.blocks(at.s.rows) - 1 - block) * at.np;
    const float2* stat = which.stat + slot * BR + (r - block * BR);
    const float* part = which.part + (slot * BR + (r - block * BR)) * kHeadDim + 2 * lane;
    const int k0 = many ? 0 : wave, dk = many ? 1 : kWaves;
    float m = -FLT_MAX, l = 0.f;
    float2 o = make_float2(0.f, 0.f);
    const auto add = [&](float2 st, float2 v) {  // (reference, sum of weights), sum
      const float up = fmaxf(m, st.x), f = __builtin_amdgcn_exp2f(0.5f * (m - up)), g = __builtin_amdgcn_exp2f(0.5f * (st.x - up));
      o.x = o.x * (f * f) + v.x * (g * g), o.y = o.y * (f * f) + v.y * (g * g), l = l * f * f + st.y * g * g, m = up;
    };
#pragma unroll 8
    for (int k = k0; k < at.np; k += dk) add(stat[(int64_t)k * BR], *(const float2*)(part + (int64_t)k * BR * kHeadDim));
    if (!many) {
      sums[wave][lane] = o;
      if (lane == 0) stats[wave] = make_float2(m, l);
      __syncthreads();
      m = -FLT_MAX, l = 0.f, o = make_float2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kWaves; ++i) add(stats[i], sums[i][lane]);
      __syncthreads();
      if (wave) continue;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int layer = (int)((uint32_t)lh / (uint32_t)a.S.H), h = lh - layer * a.S.H, G = a.S.G, token = (int)((uint32_t)r / (uint32_t)G);
    const int64_t base = (((int64_t)layer * a.n_tokens + at.s.first + token) * (a.S.H * G) + h * G + r - token * G) * kHeadDim + 2 * lane;
    if constexpr (BF16) *(uint32_t*)((uint16_t*)a.out + base) = (uint32_t)f32_to_bf16(result<true>(o.x, inv)) | (uint32_t)f32_to_bf16(result<true>(o.y, inv)) << 16;
    else *(float2*)((float*)a.out + base) = make_float2(result<false>(o.x, inv), result<false>(o.y, inv));
  }
}

// ------------------------------------------------------------------------------------------------ launches
// R: row tiles of few_rows (0: none), MANY: many_rows too.  A call that may have both kinds of sequences is one launch, the blocks of many rows first: the
// others fill what these leave free in the end.  (Prompts of 791 and 630 tokens beside five single ones, windows: four launches 206 us, one and a join 181; 150 with what is below, 163 since scores are fp16 products.)
template <bool BF16, int R, bool MANY>
__global__ __launch_bounds__(kWaves* kWave, BF16 ? (R <= 2 ? 2 : 1) : (R == 1 && !MANY ? 2 : 1)) void pages_attn_kernel(PagesAttn a) {
  uint32_t x = blockIdx.x;
  if constexpr (MANY) {
    const uint32_t n = many_rows<BF16>(a, Sequences<Many>(a, a.many, threadIdx.x % kWave), x, gridDim.x);
    if (x < n) x += (n - x + gridDim.x - 1) / gridDim.x * gridDim.x;  // its next turn
    x -= n;
  }
  if constexpr (R > 0) few_rows<BF16, R, kWaves>(a, Sequences<Few<R>>(a, a.few, threadIdx.x % kWave), x, gridDim.x);
}
// Tables of up to kShortTiles tiles: blocks are not cut, so nothing is to be joined; twice the waves share their tiles.  One sequence, 8 heads, us with parts
// and a join / so: fp32, 100 tokens 7.9 / 6.3, 500 9.1 / 9.2, 1000 9.4 / 12.2; bf16, 4 query heads, 500 9.3 / 8.7, 1000 9.6 / 11.0 (a workgroup cannot
// draw more than 50 KB a microsecond); 8 sequences of 1000 11.2 / 12.0, 64 29.0 / 30.3.
constexpr int kShortTiles = 17, kShortWaves = 8;
template <bool BF16, int R>
__global__ __launch_bounds__(kShortWaves* kWave, 2) void pages_short_kernel(PagesAttn a) {
  few_rows<BF16, R, kShortWaves>(a, Sequences<Few<R>>(a, a.few, threadIdx.x % kWave), blockIdx.x, gridDim.x);
}
template <bool BF16, int R, bool MANY>
__global__ __launch_bounds__(kWaves* kWave) void pages_join_kernel(PagesAttn a) {
  if constexpr (R > 0)
    if (!MANY || blockIdx.x < a.few.join_grid) return join_rows<BF16, Few<R>>(a, a.few, blockIdx.x);
  if constexpr (MANY) join_rows<BF16, Many>(a, a.many, blockIdx.x - a.few.join_grid);
}

// Parts of cut blocks: a block of more than w.tiles tiles has fewer than 2 tiles / w.tiles of them, all blocks together `parts` times w.tiles tiles (rounding: + 64).
template <class Geo>
constexpr int64_t kMostCut = 2 * Geo::parts + 64;
template <class Geo>
constexpr size_t kPartsBytes = (size_t)kMostCut<Geo> * Geo::rows * (kHeadDim * sizeof(float) + sizeof(float2));

// What a call launches.  A sequence's rows are known on the device only; what the sizes exclude is not launched.
struct Launches {
  int few = 0;        // row tiles of few_rows' blocks, 0: none
  bool many = false;  // many_rows
  bool cut = false;   // blocks may be cut into parts
  size_t few_bytes = 0, bytes = 0;  // of the workspace
};
int few_tiles(int64_t usual, bool bf16, bool many) { return usual <= 16 ? 1 : usual <= 32 || !bf16 || many ? 2 : 4; }
size_t few_bytes(int tiles) { return tiles == 1 ? kPartsBytes<Few<1>> : tiles == 2 ? kPartsBytes<Few<2>> : tiles == 4 ? kPartsBytes<Few<4>> : 0; }
bool may_cut(const Pages& S) { return ((int64_t)S.max_pages << S.logP) > (int64_t)kShortTiles * 32; }
Launches launches_of(const Pages& S, int batch, int n_tokens, bool bf16) {
  Launches n;
  const int64_t rows = (int64_t)n_tokens * S.G, average = S.G * (((int64_t)n_tokens + batch - 1) / batch);
  // About one token for each row of the table, idle ones among them: few_rows alone, whoever brings more.  (500 tokens of one sequence of 8192, 4 query heads, and
  // 250 idle rows 191 us, with 248 idle ones, where many_rows takes them, 144, with none 118; 250 tokens beside 255 single ones 312, these alone 220.)
  n.many = rows > kFewRows && n_tokens >= 2 * (int64_t)batch;
  if (!n.many || batch > 1) n.few = few_tiles(average > kFewRows ? S.G : average, bf16, n.many);  // beside prompts: single tokens
  n.cut = may_cut(S);
  if (n.cut) {
    n.few_bytes = few_bytes(n.few);
    n.bytes = n.few_bytes + (n.many ? kPartsBytes<Many> : 0);
  }
  return n;
}

template <class Geo>
PagesRows rows_of(const PagesAttn& a, int over, int to, char* ws) {
  const int64_t lh = (int64_t)a.n_layers * a.S.H, blocks = (int64_t)a.n_tokens * a.S.G / Geo::rows + a.batch;
  PagesRows r{};
  r.over = over, r.to = to;
  r.grid = (uint32_t)std::min<int64_t>(Geo::parts + lh * blocks, 1 << 20);
  if (ws) {
    r.join_grid = (uint32_t)std::min<int64_t>(lh * a.n_tokens * a.S.G, 2048);
    r.part = (float*)ws;
    r.stat = (float2*)(r.part + kMostCut<Geo> * Geo::rows * kHeadDim);
  }
  return r;
}

template <bool BF16, int R>
hipError_t launch_short(const PagesAttn& a, hipStream_t st) {
  pages_short_kernel<BF16, R><<<a.few.grid, kShortWaves * kWave, 0, st>>>(a);
  return hipGetLastError();
}
template <bool BF16, int R, bool MANY>
hipError_t launch(const PagesAttn& a, hipStream_t st) {
  pages_attn_kernel<BF16, R, MANY><<<a.few.grid + a.many.grid, kWaves * kWave, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  const uint32_t join = a.few.join_grid + a.many.join_grid;
  if (e != hipSuccess || !join) return e;
  pages_join_kernel<BF16, R, MANY><<<join, kWaves * kWave, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t pages_attn_bytes(const Pages& S, int batch, int n_tokens, bool bf16) {
  return batch == 0 || n_tokens == 0 ? 0 : launches_of(S, batch, n_tokens, bf16).bytes;
}
// The largest row tiles that few_rows takes in any of these calls, and many_rows, which one sequence with all rows takes.
size_t pages_attn_most_bytes(const Pages& S, int batch, int n_tokens, bool bf16) {
  if (batch == 0 || n_tokens == 0 || !may_cut(S)) return 0;
  const int64_t rows = (int64_t)n_tokens * S.G;
  return few_bytes(few_tiles(std::max<int64_t>(S.G, std::min<int64_t>(rows, kFewRows)), bf16, false)) + (rows > kFewRows ? kPartsBytes<Many> : 0);
}

hipError_t launch_pages_attn(PagesAttn a, bool bf16, void* ws, hipStream_t st) {
  const Launches n = launches_of(a.S, a.batch, a.n_tokens, bf16);
  char* at = n.bytes ? (char*)ws : nullptr;
  constexpr int kAny = 0x7fffffff;
  const int few_to = n.many ? kFewRows : kAny;
  if (n.few) a.few = n.few == 1 ? rows_of<Few<1>>(a, 0, few_to, at) : n.few == 2 ? rows_of<Few<2>>(a, 0, few_to, at) : rows_of<Few<4>>(a, 0, few_to, at);
  if (n.many) a.many = rows_of<Many>(a, n.few ? kFewRows : 0, kAny, at ? at + n.few_bytes : nullptr);
  if (bf16) {
    if (n.many) return n.few == 0 ? launch<true, 0, true>(a, st) : n.few == 1 ? launch<true, 1, true>(a, st) : launch<true, 2, true>(a, st);
    if (!n.cut && n.few <= 2) return n.few == 1 ? launch_short<true, 1>(a, st) : launch_short<true, 2>(a, st);
    return n.few == 1 ? launch<true, 1, false>(a, st) : n.few == 2 ? launch<true, 2, false>(a, st) : launch<true, 4, false>(a, st);
  }
  // fp32: many_rows takes twice the registers; together few_rows would have half of the waves
  if (n.many) {
    PagesAttn b = a;
    b.few = PagesRows{};
    const hipError_t e = launch<false, 0, true>(b, st);
    if (e != hipSuccess || !n.few) return e;
    a.many = PagesRows{};
  }
  if (!n.cut && n.few == 1) return launch_short<false, 1>(a, st);
  return n.few == 1 ? launch<false, 1, false>(a, st) : launch<false, 2, false>(a, st);
}

}  // namespace iwdft
