// Attention of new tokens over the 8-bit pages of their sequences.
//
//   o_t = sum_j p_j v_j,  p = softmax_j (scale q_t k_j),  over the tokens j that t sees.
//
// All products run on the matrix cores.  What keeps them exact:
//  * q k: fp16, which holds e4m3 exactly.  A row of q is multiplied by the power of two that brings its largest value to [2^14, 2^15); a bf16 number is exact in
//    fp16 down to 2^-31 of that value, a smaller one errs by 2^-39 of it; fp32 queries are the sum of two fp16 parts (22 bits).  (The block-scaled products of e4m3 bytes
//    need no conversions and make prompts 8 % faster, but one of them loses what is 2^14 times smaller than the largest product of its group: a score's sum errs by up to
//    2^-12 of sum |q k|, 2^-15 in the mean, with fp16 products by 2^-22 and 2^-25.)
//  * p v: fp16.
//  * the pages' exponents: that of K enters the score's factor; that of V joins the exponent of the weight.  With s_j the score times log2 e and
//    eV_j the exponent of j's page, the weights in the sum are P_j = 2^(s_j + eV_j - m), m a running bound of s_j + eV_j, and the
//    denominator is sum 2^(s_j - m) = sum P_j 2^-eV_j.  So no weight overflows fp16 or loses bits because its page is small.
//  * the denominator where pages are far apart: of a page 2^130 smaller than another P_j is nothing in fp32, and 2^(s_j - m) may still be all of the
//    denominator.  From the first tile with a page of |eV| > kNear on, a wave sums 2^(s_j - s), s the largest of them, and scales it by 2^(s - m).  m is then no
//    less than any s_j + eV_j: the denominator lies between 2^-120 and 2^100 times the number of tokens, and is held 2^-4 times as large.
//  * P_j is rounded to fp16 (11 bits; bf16 results have 8), for fp32 to two parts; the denominator and all sums are fp32.
// The sums hold 2^lift P_j.  m grows where an exponent passes it by more than `slack`; 2^lift P_j <= 2^(slack + lift) < 65504 then.  bf16: lift 6,
// slack 8, few rescalings.  fp32: lift 15, slack 0: fp16 ends at 2^-25, so weights err by 2^-40 of the largest one at least, and a page's
// values, whose sizes are up to 2^18 apart, by 2^-22 of what they add up to.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "pages.h"

namespace iwdft {

namespace {

constexpr int kWave = 64;
constexpr int kWaves = 4;
template <bool BF16>
struct Weights {
  static constexpr float lift = BF16 ? 6.f : 15.f, slack = BF16 ? 8.f : 0.f;
  static constexpr int down = (int)lift + 4;   // what the sums are larger than 2^4 times the denominator by
  static constexpr float unit = 1.f / (float)(1 << down);
};
constexpr int kQTop = 14;  // rows of q: largest value in [2^kQTop, 2^(kQTop + 1))
constexpr int kNear = 32;
// x * 2^d.  In two factors: 2^d may be out of range where the product is not.
__device__ __forceinline__ float times_power(float x, float d) {
  const float k = ceilf(fmaxf(d, -1000.f));
  return ldexpf(x * __builtin_amdgcn_exp2f(d - k), (int)k);
}
// Sum of 2^((x[j] - m) - d), j < 8; top: the largest x.  (x and m may be so large that m + d would be m.)
__device__ __forceinline__ float sum_of_powers(const float* x, float top, float m, float d) {
  const float t = fmaxf(top, -FLT_MAX);
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum += __builtin_amdgcn_exp2f(x[j] - t);
  return times_power(sum, (t - m) - d);
}

// ------------------------------------------------------------------------------------------------ sharing out the work
// A block is `rows` consecutive (new token, query head of the KV head) pairs of a sequence; its tokens are cut into parts, one workgroup each, such that
// all parts of a call hold about the same number of tiles and, up to parts / 2 blocks, there are about `parts` of them: two workgroups on each CU (more would run
// alone in the end: 16 contexts of 4096 to 16384 tokens 90 us, with the blocks' last, shorter parts counted in 78, 71 with what is below).  More blocks make more parts, and
// the two kinds of rows count for themselves.  Lengths live on the device, so every wave works out the shares by itself, 64 sequences at a time: the launch only has to be large enough.
// The kernels that leave a SIMD one wave (64 rows in bf16, 32 rows and prompts in fp32) run 256 workgroups at a time, so 512 parts are two rounds there; us with 512 / 256:
// one sequence of 65536 tokens and 48 rows 70 / 58, in fp32 20 rows 57 / 49; four of up to 16384 and 48 rows 28 / 33, 800 rows over 32768 in fp32 297 / 314, 4096 tokens' prompt 355 / 355.
// Short parts cost more in the join than the second workgroup on a CU gains: one token over 8192 tokens of 8 heads 14.3 us with parts of 4 tiles, 11.6 with 8,
// over 16000 17.3 with 8 and 15.1 with 16.
constexpr int kLeastTiles = 4, kCus = 256;
constexpr float kMostBlocks = 1100000000.f;  // 2^30 rows have fewer: starts that overlap, whose counts would not fit; such a call does nothing
constexpr int kFewRows = 64;  // sequences of up to so many rows go to few_rows, where a call may have both

template <int ROWS, int TOKENS, int PARTS, int PAIR>
struct Geometry {
  static constexpr int rows = ROWS, tile = TOKENS, parts = PARTS;  // of a block; of a tile; of a call
  static constexpr int pair = PAIR;  // a second workgroup on a CU from parts of so many tiles on: more parts are more to join
};
template <int R>
using Few = Geometry<16 * R, 32, 512, 16>;
using Many = Geometry<128, 64, 512, 8>;

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
      const Seq s = b0 == 0 ? head : load(b0 + lane);
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
  Seq head;  // the lane's sequence of the first 64

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

// Tiles of part k of n: as even as they can be.
struct Share {
  int from, to;
};
__device__ __forceinline__ Share share_of(int tiles, int k, int n) {
  const int each = (int)((uint32_t)tiles / (uint32_t)n), more = tiles - each * n;
  return Share{k * each + min(k, more), (k + 1) * each + min(k + 1, more)};
}

// ------------------------------------------------------------------------------------------------ operands
__device__ __forceinline__ half2v e4m3_halves(uint32_t w, bool high) {
  return high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false);
}
// Eight bytes as an operand.
__device__ __forceinline__ half8 operand(uint32_t lo, uint32_t hi) {
  const half2v a = e4m3_halves(lo, false), b = e4m3_halves(lo, true), c = e4m3_halves(hi, false), d = e4m3_halves(hi, true);
  return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {  // 1 in every byte that is NaN (0x7f, 0xff)
  return (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
}
template <int PARTS>
__device__ __forceinline__ void to_halves(const float* x, half8* parts) {  // x[8] as PARTS fp16 numbers that add up to it
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    float rest = x[c];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const _Float16 h = (_Float16)rest;
      parts[p][c] = h;
      rest -= (float)h;
    }
  }
}
__device__ __forceinline__ float max_over_16s(float x) {  // over lanes that differ in their upper two bits
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

template <bool BF16>
__device__ __forceinline__ void load_channels(const void* p, int64_t i, float* f) {  // 16 channels
  if constexpr (BF16) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint4 w = ((const uint4*)((const uint16_t*)p + i))[h];
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int c = 0; c < 4; ++c) f[8 * h + 2 * c] = __uint_as_float(u[c] << 16), f[8 * h + 2 * c + 1] = __uint_as_float(u[c] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const float4 x = ((const float4*)((const float*)p + i))[h];
      f[4 * h] = x.x, f[4 * h + 1] = x.y, f[4 * h + 2] = x.z, f[4 * h + 3] = x.w;
    }
  }
}

template <bool BF16>
__device__ __forceinline__ float result(float sum, float inv) { return sum * Weights<BF16>::unit * inv; }  // inv: of the denominator as it is held
template <bool BF16>
__device__ __forceinline__ void store8(void* p, int64_t i, const float* y, float inv) {  // 8 channels
  if constexpr (BF16) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (uint32_t)f32_to_bf16(result<true>(y[2 * j], inv)) | (uint32_t)f32_to_bf16(result<true>(y[2 * j + 1], inv)) << 16;
    *(uint4*)((uint16_t*)p + i) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; j += 4)
      *(float4*)((float*)p + i + j) = make_float4(result<false>(y[j], inv), result<false>(y[j + 1], inv), result<false>(y[j + 2], inv), result<false>(y[j + 3], inv));
  }
}

// A row at position p sees the tokens (from, p] and those below sink.
__device__ __forceinline__ int window_from(const PagesAttn& a, int p) { return a.n_recent ? max(p - a.n_recent, -1) : -1; }  // p >= -1, n_recent >= 0: no overflow
// ... as one bit for each of the eight tokens from j0 on.  (Bits in a register, not a comparison's mask for each token: those would push the loops' own scalars out.)
__device__ __forceinline__ uint32_t seen_bits(int j0, int from, int to, int sink) {
  const auto below = [&](int n) { return (1u << min(max(n, 0), 8)) - 1u; };
  return below(to + 1 - j0) & (~below(from + 1 - j0) | below(sink - j0));
}
__device__ __forceinline__ uint32_t bytes_of_bits(uint32_t four) { return (four & 15u) * 0x00204081u & 0x01010101u; }  // 1 in the byte of every bit
__device__ __forceinline__ float seen_or_none(float x, uint32_t bits, int j) {  // -infinity unless bit j is set
  const uint32_t keep = (uint32_t)((int32_t)(bits << (31 - j)) >> 31);
  return __uint_as_float((__float_as_uint(x) & keep) | (0xff800000u & ~keep));
}

// Tiles that a block's rows see: those of the sinks, then the others.
struct Span {
  int sinks, skip, n;
  __device__ __forceinline__ int tile(int i) const { return i < sinks ? i : i + skip; }
};
template <int kTile>
__device__ __forceinline__ Span span_of(const PagesAttn& a, int p_lo, int p_hi) {  // positions of the block's first and last token
  Span s{0, 0, 0};
  if (p_hi < 0) return s;
  const int end = p_hi / kTile + 1;
  int from = 0;
  if (a.n_recent) {
    from = (window_from(a, max(p_lo, -1)) + 1) / kTile;
    s.sinks = a.n_sink > 0 ? min((min(a.n_sink, p_hi + 1) + kTile - 1) / kTile, end) : 0;
  }
  s.skip = max(from - s.sinks, 0);
  s.n = max(end - s.skip, s.sinks);
  return s;
}

// One row tile of 16 query rows: lane l holds row l % 16.
template <int PARTS>
struct Rows {
  half8 q[4][PARTS];  // [chunk of 16 channels oct + 4 (c / 2)][8 of them: c % 2]
  floatx4 o[8];   // [16-byte load of V][channel of the pair]: row l % 16, channels 32 (i / 2) + 8 (l / 16) + 2 c + i % 2
  float m, l;
  int pos, from, eq;
};

// ------------------------------------------------------------------------------------------------ few rows
// A workgroup has a part of the tokens of one block of 16 R rows; its W waves take the tiles in turn and join their sums in the end.  A tile of 32
// tokens is 8 KB, eight 16-byte loads a lane, the next one's on their way while this one is multiplied (two or three ahead are no faster): S^T = K Q^T leaves lane l
// with row l % 16 and the 8 tokens of octet l / 16, which is how O^T = V^T P^T wants them, so nothing moves between lanes but the maximum.
// Bound by memory where there is much of it, by the chain lengths -> table -> tokens -> sums where there is little: the first tile is on its
// way before q is looked at.
template <bool BF16, int R, int W>
__device__ __forceinline__ void few_rows(const PagesAttn& a, uint32_t x0, uint32_t step) {
  using Geo = Few<R>;
  constexpr int PARTS = BF16 ? 1 : 2, BR = Geo::rows, kTile = Geo::tile;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int row = lane & 15, oct = lane >> 4;
  __shared__ __attribute__((aligned(16))) float join[W][16][kHeadDim + 4];
  __shared__ float2 join_stat[W][16];

  const Schedule<Geo> plan(a, a.few, lane);
  const uint32_t slices = (uint32_t)(a.n_layers * a.S.H), all = (uint32_t)plan.w.parts * slices;
  for (uint32_t x = x0; x < all; x += step) {
    const int lh = (int)(x % slices);  // workgroups are dealt to the XCDs in turn: with 8 heads each reads one head's pages
    const Place at = plan.find((int)(x / slices), [](const Seq& s, int np) { return np * Schedule<Geo>::blocks(s.rows); });
    const Seq s = at.s;
    const int turn = (int)((uint32_t)at.at / (uint32_t)at.np), part = at.at - turn * at.np, block = plan.blocks(s.rows) - 1 - turn;
    const int layer = (int)((uint32_t)lh / (uint32_t)a.S.H), h = lh - layer * a.S.H, G = a.S.G;
    const int row0 = block * BR, rows = min(s.rows - row0, BR);
    const int before = s.len - s.nq;  // position of the sequence's first new token
    const int p_lo = before + (int)((uint32_t)row0 / (uint32_t)G), p_hi = before + (int)((uint32_t)(row0 + rows - 1) / (uint32_t)G);
    const Span span = span_of<kTile>(a, p_lo, p_hi);
    const Share mine = share_of(span.n, part, at.np);
    const int n_rt = (rows + 15) / 16;
    const int sink = a.n_recent ? a.n_sink : 0, all_from = window_from(a, max(p_lo, -1));

    // pages of a lane's octets: that of its K row and that of its tokens in V and in the scores
    const int32_t* table = a.table + (int64_t)at.b * a.S.max_pages;
    const int last_page = max(page_count(s.len, a.S.logP) - 1, 0), in_page = (1 << a.S.logP) - 1;
    const int k_oct = row >> 2, k_tok = 8 * k_oct + (row & 3);
    struct Ids {
      int k, v;
    };
    const auto pages_at = [&](int i) {
      const int t = span.tile(i) * kTile;
      return Ids{table[min((t + 8 * k_oct) >> a.S.logP, last_page)], table[min((t + 8 * oct) >> a.S.logP, last_page)]};
    };
    struct Data {
      uint4 k[2][2], v[4];
      int2 e;
      bool bad;
    };
    const auto load_tile = [&](int i, Ids id) {
      Data d;
      const int t = span.tile(i) * kTile;
      d.bad = id.v < 0 || id.v >= a.S.n_pages;
      const int kp = id.k < 0 || id.k >= a.S.n_pages ? 0 : id.k, vp = d.bad ? 0 : id.v;
      const int64_t vh = page_head(a.S, a.layer + layer, vp, h);
      const uint8_t* kb = page_values(a.S, page_head(a.S, a.layer + layer, kp, h)) + ((t + k_tok) & in_page) * kHeadDim + 16 * oct;
      const uint8_t* vb = page_values(a.S, vh) + ((size_t)kHeadDim << a.S.logP) + ((t + 8 * oct) & in_page) * kHeadDim + 16 * row;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int p = 0; p < 2; ++p) d.k[u][p] = *(const uint4*)(kb + u * 4 * kHeadDim + 64 * p);
#pragma unroll
      for (int p = 0; p < 4; ++p) d.v[p] = *(const uint4*)(vb + 256 * p);
      d.e = *(const int2*)(a.S.exponents + 2 * vh);
      return d;
    };
    const int first = mine.from + wave;
    Ids id{0, 0};
    Data next{};
    if (first < mine.to) {
      next = load_tile(first, pages_at(first));
      if (first + W < mine.to) id = pages_at(first + W);
    }

    Rows<PARTS> rt[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      Rows<PARTS>& z = rt[r];
      const uint32_t n = (uint32_t)(row0 + 16 * r + row);  // of the sequence's rows
      const int token = (int)(n / (uint32_t)G);
      const bool have = 16 * r + row < rows;
      z.pos = have ? max(before + token, -1) : -1, z.from = window_from(a, z.pos);
      z.m = -FLT_MAX, z.l = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) z.o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
      float f[2][16];
      float top = 0.f;
      if (have) {
        const int64_t base = (((int64_t)layer * a.n_tokens + s.first + token) * (a.S.H * G) + h * G + (int)(n - (uint32_t)token * (uint32_t)G)) * kHeadDim;
#pragma unroll
        for (int p = 0; p < 2; ++p) load_channels<BF16>(a.q, base + 64 * p + 16 * oct, f[p]);
      } else {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int c = 0; c < 16; ++c) f[p][c] = 0.f;
      }
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int c = 0; c < 16; ++c) top = fmaxf(top, fabsf(f[p][c]));
      top = max_over_16s(top);
      z.eq = max((int)(__float_as_uint(top) >> 23) - 127, kLeastExponent);
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int c = 0; c < 16; ++c) f[p][c] = ldexpf(f[p][c], kQTop - z.eq);
#pragma unroll
      for (int c = 0; c < 4; ++c) to_halves<PARTS>(f[c / 2] + 8 * (c % 2), z.q[c]);
    }

    int near = kNear;  // -1 from the first far page on
    for (int i = first; i < mine.to; i += W) {
      Data d = next;
      if (i + W < mine.to) {
        next = load_tile(i + W, id);
        if (i + 2 * W < mine.to) id = pages_at(i + 2 * W);
      }
      const int t0 = span.tile(i) * kTile, t1 = t0 + kTile - 1, j0 = t0 + 8 * oct;
      // whether every row sees the whole tile
      const bool edge = t1 > p_lo || (t1 >= sink && t0 <= window_from(a, p_hi)) || __any(d.bad);
      bool poison = false;
      if (edge) {  // tokens that no row sees may hold anything
        const uint32_t any = d.bad ? 0u : seen_bits(j0, all_from, p_hi, sink), keep[2] = {bytes_of_bits(any) * 0xffu, bytes_of_bits(any >> 4) * 0xffu};
        uint32_t nans = 0;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          d.v[p].x &= keep[0], d.v[p].y &= keep[1], d.v[p].z &= keep[0], d.v[p].w &= keep[1];
          nans |= nan_bytes(d.v[p].x) | nan_bytes(d.v[p].y) | nan_bytes(d.v[p].z) | nan_bytes(d.v[p].w);
        }
        poison = __any(nans != 0);
      }

      half8 kf[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int p = 0; p < 2; ++p) kf[u][2 * p] = operand(d.k[u][p].x, d.k[u][p].y), kf[u][2 * p + 1] = operand(d.k[u][p].z, d.k[u][p].w);
      const float ev = (float)d.e.y;
      const bool far = __builtin_expect(__any(abs(d.e.y) > near), 0);
      near = far ? -1 : near;
      const float slack = far ? -__builtin_inff() : Weights<BF16>::slack;
      const int shift = far ? -1000 : -d.e.y - Weights<BF16>::down;  // of the weights' sum; far: it comes another way
      half8 pw[R][PARTS];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r >= n_rt) continue;
        Rows<PARTS>& z = rt[r];
        float sc[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          floatx4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[u][c], z.q[c][p], acc, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < 4; ++j) sc[4 * u + j] = acc[j];
        }
        const float factor = ldexpf(a.scale, z.eq - kQTop + d.e.x);
#pragma unroll
        for (int j = 0; j < 8; ++j) sc[j] = sc[j] * factor + ev;
        if (edge) {
          const uint32_t bits = d.bad ? 0u : seen_bits(j0, z.from, z.pos, sink);
#pragma unroll
          for (int j = 0; j < 8; ++j) sc[j] = seen_or_none(sc[j], bits, j);
        }
        float top = sc[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, sc[j]);
        if (__any(top > z.m + slack)) {
          const float up = fmaxf(z.m, max_over_16s(top)), fade = __builtin_amdgcn_exp2f(z.m - up);
          if (__builtin_expect(far, 0)) z.l = times_power(z.l, z.m - up) + sum_of_powers(sc, top, up, ev + 4.f);
          else z.l *= fade;
          z.m = up;
#pragma unroll
          for (int c = 0; c < 8; ++c) z.o[c] *= fade;
        }
        float y[8], sum = 0.f;
        const float ref = z.m - Weights<BF16>::lift;
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = __builtin_amdgcn_exp2f(sc[j] - ref), sum += y[j];
        z.l += ldexpf(sum, shift);
        to_halves<PARTS>(y, pw[r]);
      }
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        uint4 v = d.v[p];
        if (__builtin_expect(poison, 0)) {  // NaN where only some rows may see it: taken out here, brought back to those rows
          const uint32_t n[4] = {nan_bytes(v.x), nan_bytes(v.y), nan_bytes(v.z), nan_bytes(v.w)};
          v.x &= ~(n[0] * 0xffu), v.y &= ~(n[1] * 0xffu), v.z &= ~(n[2] * 0xffu), v.w &= ~(n[3] * 0xffu);
          const half8 bad[2] = {operand(n[0] * 0x38u, n[1] * 0x38u), operand(n[2] * 0x38u, n[3] * 0x38u)};  // 0x38: 1
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const uint32_t bits = d.bad ? 0u : seen_bits(j0, rt[r].from, rt[r].pos, sink);
            const half8 one = operand(bytes_of_bits(bits) * 0x38u, bytes_of_bits(bits >> 4) * 0x38u);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(bad[c], one, floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
              for (int j = 0; j < 4; ++j) rt[r].o[2 * p + c][j] += hit[j] > 0.f ? __builtin_nanf("") : 0.f;
            }
          }
        }
        const half8 v0 = operand(v.x, v.y), v1 = operand(v.z, v.w);
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (r >= n_rt) continue;
#pragma unroll
          for (int u = PARTS - 1; u >= 0; --u) {
            rt[r].o[2 * p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pw[r][u], rt[r].o[2 * p], 0, 0, 0);
            rt[r].o[2 * p + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pw[r][u], rt[r].o[2 * p + 1], 0, 0, 0);
          }
        }
      }
    }

    // the four waves' sums of 16 rows at a time, then 8 channels of a row to each thread
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r >= n_rt) continue;
      Rows<PARTS>& z = rt[r];
      z.l += __shfl_xor(z.l, 16);
      z.l += __shfl_xor(z.l, 32);
      if (r) __syncthreads();
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float* to = join[wave][row] + 32 * p + 8 * oct;
        *(float4*)to = make_float4(z.o[2 * p][0], z.o[2 * p + 1][0], z.o[2 * p][1], z.o[2 * p + 1][1]);
        *(float4*)(to + 4) = make_float4(z.o[2 * p][2], z.o[2 * p + 1][2], z.o[2 * p][3], z.o[2 * p + 1][3]);
      }
      if (oct == 0) join_stat[wave][row] = make_float2(z.m, z.l);
      __syncthreads();
      if (threadIdx.x >= 256) continue;
      const int jr = threadIdx.x >> 4, jc = 8 * (threadIdx.x & 15);
      float2 st[W];
#pragma unroll
      for (int v = 0; v < W; ++v) st[v] = join_stat[v][jr];
      float m = st[0].x;
#pragma unroll
      for (int v = 1; v < W; ++v) m = fmaxf(m, st[v].x);
      float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, l = 0.f;
#pragma unroll
      for (int v = 0; v < W; ++v) {
        const float half = __builtin_amdgcn_exp2f(0.5f * (st[v].x - m)), fade = half * half;  // the denominator's share may need both factors
        const float4 lo = *(const float4*)(join[v][jr] + jc), hi = *(const float4*)(join[v][jr] + jc + 4);
        l += st[v].y * half * half;
        y[0] += lo.x * fade, y[1] += lo.y * fade, y[2] += lo.z * fade, y[3] += lo.w * fade;
        y[4] += hi.x * fade, y[5] += hi.y * fade, y[6] += hi.z * fade, y[7] += hi.w * fade;
      }
      if (16 * r + jr >= rows) continue;
      if (at.np == 1) {
        const uint32_t n = (uint32_t)(row0 + 16 * r + jr);
        const int token = (int)(n / (uint32_t)G);
        store8<BF16>(a.out, (((int64_t)layer * a.n_tokens + s.first + token) * (a.S.H * G) + h * G + (int)(n - (uint32_t)token * (uint32_t)G)) * kHeadDim + jc, y,
                     l == 0.f ? 0.f : 1.f / l);
      } else {
        const int64_t slot = (int64_t)lh * plan.w.split + at.before + at.at;
        float* to = a.few.part + (slot * BR + 16 * r + jr) * kHeadDim + jc;
        *(float4*)to = make_float4(y[0], y[1], y[2], y[3]), *(float4*)(to + 4) = make_float4(y[4], y[5], y[6], y[7]);
        if (jc == 0) a.few.stat[slot * BR + 16 * r + jr] = make_float2(m, l);
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------ many rows
// Prompts: four waves of 32 rows share tiles of 64 tokens that go through LDS as bytes, the next tile's loads in flight while this one is multiplied; a wave
// turns the bytes into operands itself (128 conversions per 32 products of 32 cycles; K as fp16 in LDS: a prompt of 8000 tokens 1 % faster, a mixed call 40 % slower, whose CUs then hold one workgroup).
// S^T = K Q^T leaves lane l with row l % 32 and tokens 16 t + 8 (l / 32) + j, the operand of O^T = V^T P^T.  K's 16-byte chunks are
// swizzled by their token so that the eight lanes of a bank group read eight different ones.
template <bool BF16>
__device__ __forceinline__ uint32_t many_rows(const PagesAttn& a, uint32_t x0, uint32_t step) {  // returns the workgroups' number
  using Geo = Many;
  constexpr int PARTS = BF16 ? 1 : 2, BR = Geo::rows, kTile = Geo::tile, kHalf = 32;
  constexpr float kLift = Weights<BF16>::lift;
  static_assert(BR == 32 * kWaves && kTile == 2 * kHalf, "");
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int row = lane & 31, grp = lane >> 5;
  __shared__ __attribute__((aligned(16))) uint8_t kbuf[2][kTile * kHeadDim], vbuf[2][kTile * kHeadDim];
  __shared__ float4 meta[2][kTile / 16];  // of the pages of 16 tokens each: scale 2^(eK - kQTop), eV, 2^-eV in the denominator's unit, infinity where |eV| > kNear

  const Schedule<Geo> plan(a, a.many, lane);
  const uint32_t slices = (uint32_t)(a.n_layers * a.S.H), all = (uint32_t)plan.w.parts * slices;
  for (uint32_t x = x0; x < all; x += step) {
    const int lh = (int)(x % slices);
    const Place at = plan.find((int)(x / slices), [](const Seq& s, int np) { return np * Schedule<Geo>::blocks(s.rows); });
    const Seq s = at.s;
    const int turn = (int)((uint32_t)at.at / (uint32_t)at.np), part = at.at - turn * at.np, block = plan.blocks(s.rows) - 1 - turn;  // the longest first
    const int layer = (int)((uint32_t)lh / (uint32_t)a.S.H), h = lh - layer * a.S.H, G = a.S.G;
    const int row0 = block * BR, rows = min(s.rows - row0, BR), before = s.len - s.nq;
    const int p_lo = before + (int)((uint32_t)row0 / (uint32_t)G), p_hi = before + (int)((uint32_t)(row0 + rows - 1) / (uint32_t)G);
    const Span span = span_of<kTile>(a, p_lo, p_hi);
    const Share share = share_of(span.n, part, at.np);
    const int t_from = share.from, t_to = share.to;

    const uint32_t mine = (uint32_t)(row0 + 32 * wave + row);  // of the sequence's rows
    const int token = (int)(mine / (uint32_t)G);
    const bool have = 32 * wave + row < rows;
    const int pos = have ? max(before + token, -1) : -1;
    const bool any_row = 32 * wave < rows;
    const int w_lo = before + (row0 + 32 * wave) / G, w_hi = any_row ? before + (row0 + min(32 * wave + 32, rows) - 1) / G : -1;  // positions of the wave's rows
    const int sink = a.n_recent ? a.n_sink : 0, from = window_from(a, pos), w_from = window_from(a, max(w_lo, -1));
    const int64_t out_at = (((int64_t)layer * a.n_tokens + s.first + token) * (a.S.H * G) + h * G + (int)(mine - (uint32_t)token * (uint32_t)G)) * kHeadDim;

    half8 q[8][PARTS];  // [chunk of 16 channels 2 (c / 2) + grp][8 of them: c % 2]
    int eq;
    {
      float f[4][16], top = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (have) load_channels<BF16>(a.q, out_at + 32 * c + 16 * grp, f[c]);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (!have) f[c][j] = 0.f;
          top = fmaxf(top, fabsf(f[c][j]));
        }
      }
      top = fmaxf(top, __shfl_xor(top, 32));
      eq = max((int)(__float_as_uint(top) >> 23) - 127, kLeastExponent);
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int j = 0; j < 16; ++j) f[c][j] = ldexpf(f[c][j], kQTop - eq);
#pragma unroll
      for (int c = 0; c < 8; ++c) to_halves<PARTS>(f[c / 2] + 8 * (c % 2), q[c]);
    }
    const float q_scale = ldexpf(1.f, eq);
    floatx16 o[4];  // rows 8 (i / 4) + 4 grp + i % 4 =: u of channel tile c: channel 64 (c / 2) + 2 u + c % 2
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
    float m = -FLT_MAX, l = 0.f;
    float most = kLift + Weights<BF16>::slack;  // -infinity from the first far page on

    // a wave brings 16 tokens of a tile, which are in one page; that page is looked up a tile earlier
    const int32_t* table = a.table + (int64_t)at.b * a.S.max_pages;
    const int last_page = max(page_count(s.len, a.S.logP) - 1, 0), in_page = (1 << a.S.logP) - 1;
    const int64_t slice = (int64_t)(a.layer + layer) * a.S.n_pages * a.S.H + h;
    const uint8_t* const slice_values = a.S.values + (slice << (a.S.logP + 8));
    const int2* const slice_exponents = (const int2*)a.S.exponents + slice;
    int next_page = 0;
    uint4 nk[2], nv[2];
    int2 ne;
    bool none;
    const auto find_tile = [&](int i) { next_page = table[min((span.tile(i) * kTile + 16 * wave) >> a.S.logP, last_page)]; };
    const auto load_tile = [&](int i) {
      const int t = span.tile(i) * kTile + 16 * wave;
      int page = __builtin_amdgcn_readfirstlane(next_page);
      none = (uint32_t)page >= (uint32_t)a.S.n_pages;
      page = none ? 0 : page;
      const int64_t head = (int64_t)page * a.S.H;
      const uint8_t* from = slice_values + (head << (a.S.logP + 8)) + (t & in_page) * kHeadDim;
      nk[0] = ((const uint4*)from)[lane], nk[1] = ((const uint4*)from)[kWave + lane];
      from += (size_t)kHeadDim << a.S.logP;
      nv[0] = ((const uint4*)from)[lane], nv[1] = ((const uint4*)from)[kWave + lane];
      ne = slice_exponents[head];
    };
    const auto store_tile = [&](int b) {
      float4 e = make_float4(ldexpf(a.scale, ne.x - kQTop), (float)ne.y, ldexpf(1.f, -ne.y - Weights<BF16>::down), abs(ne.y) > kNear ? __builtin_inff() : -__builtin_inff());
      if (none) {  // a page that is not there: scores of -infinity, weights and values of 0
        nk[0] = nk[1] = nv[0] = nv[1] = make_uint4(0, 0, 0, 0);
        e = make_float4(0.f, -__builtin_inff(), 0.f, -__builtin_inff());
      }
      const int tok = lane >> 3, ch = lane & 7;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        ((uint4*)kbuf[b])[(16 * wave + kOct * u + tok) * 8 + (ch ^ ((tok & 3) | u << 2))] = nk[u];
        ((uint4*)vbuf[b])[64 * (2 * wave + u) + lane] = nv[u];
      }
      if (lane == 0) meta[b][wave] = e;
    };
    if (t_from < t_to) {
      find_tile(t_from);
      load_tile(t_from);
      store_tile(0);
      if (t_from + 1 < t_to) find_tile(t_from + 1);
    }
    __syncthreads();
    // K row of this lane in a half: token 16 (row / 16) + 8 ((row / 4) % 2) + 4 ((row / 8) % 2) + row % 4
    const int k_tok = 16 * (row >> 4) + 8 * ((row >> 2) & 1) + 4 * ((row >> 3) & 1) + (row & 3), k_swz = (row & 3) | ((row >> 2) & 1) << 2;
    // EDGE: some row of the block may not see all of the tile
    const auto step = [&](int i, auto kEdge) {
      constexpr bool EDGE = decltype(kEdge)::value;
      const int b = (i - t_from) & 1;
      if (i + 1 < t_to) load_tile(i + 1);
      if (i + 2 < t_to) find_tile(i + 2);
      const int t0 = span.tile(i) * kTile;
      if (!EDGE || t0 <= w_hi) {  // else behind all of the wave's rows
        floatx16 acc[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[u][j] = 0.f;
        const auto chunk = [&](int u, int c) { return ((const uint4*)kbuf[b])[(kHalf * u + k_tok) * 8 + ((2 * c + grp) ^ k_swz)]; };
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint4 kw[2] = {chunk(0, c), chunk(1, c)};
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
              for (int u = 0; u < 2; ++u)
                acc[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(i ? operand(kw[u].z, kw[u].w) : operand(kw[u].x, kw[u].y), q[2 * c + i][p], acc[u], 0, 0, 0);
        }
        const int base = t0 + 8 * grp;  // tokens of the lane: base + 16 t + j
        float inv[4], far = -__builtin_inff();
        float sc[32];  // exponents of the weights as they enter the sums: relative to m - lift
        const bool unset = m == -FLT_MAX;  // the row has seen nothing: relative to 0
        const float ref = (unset ? 0.f : m) - kLift;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float4 e = meta[b][t];
          const float factor = e.x * q_scale, shift = e.y - ref;
          inv[t] = e.z, far = fmaxf(far, e.w);
#pragma unroll
          for (int j = 0; j < 8; ++j) sc[8 * t + j] = acc[t / 2][8 * (t % 2) + j] * factor + shift;
        }
        if constexpr (EDGE) {
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const uint32_t bits = seen_bits(base + 16 * t, from, pos, sink);
#pragma unroll
            for (int j = 0; j < 8; ++j) sc[8 * t + j] = seen_or_none(sc[8 * t + j], bits, j);
          }
        }
        float top = sc[0];
#pragma unroll
        for (int j = 1; j < 32; ++j) top = fmaxf(top, sc[j]);
        if (__any(fmaxf(top, far) > (unset ? -FLT_MAX : most))) {
          top = fmaxf(top, __shfl_xor(top, 32));
          const bool first = unset && top >= -FLT_MAX;
          const float up = unset ? (first ? top - kLift : 0.f) : fmaxf(top - kLift, 0.f), fade = unset ? 1.f : __builtin_amdgcn_exp2f(-up);
          m = first ? up : m + up, l = times_power(l, unset ? 0.f : -up);
#pragma unroll
          for (int j = 0; j < 32; ++j) sc[j] -= up;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[c][j] *= fade;
          if (__builtin_expect(__any(far > 0.f || most < 0.f), 0)) {
            most = -__builtin_inff();
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const float ev = meta[b][t].y;
              float s = sc[8 * t];
#pragma unroll
              for (int j = 1; j < 8; ++j) s = fmaxf(s, sc[8 * t + j]);
              l += sum_of_powers(sc + 8 * t, s, 0.f, fmaxf(ev, -FLT_MAX) + (float)Weights<BF16>::down);
              inv[t] = 0.f;  // not again below
            }
          }
        }
        half8 pw[4][PARTS];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float y[8], sum = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = __builtin_amdgcn_exp2f(sc[8 * t + j]);
          to_halves<PARTS>(y, pw[t]);
#pragma unroll
          for (int j = 0; j < 8; ++j) sum += y[j];  // not of the rounded weights: where V's pages are far apart, those of a small page may all be 0 in fp16
          l += sum * inv[t];
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uint4 v[2];
#pragma unroll
          for (int p = 0; p < 2; ++p) v[p] = ((const uint4*)vbuf[b])[(2 * t + grp) * 64 + 32 * p + row];
          if constexpr (EDGE) {  // tokens that no row sees may hold anything; NaN that only some rows see is brought back to those
            const uint32_t any = seen_bits(base + 16 * t, w_from, w_hi, sink), keep[2] = {bytes_of_bits(any) * 0xffu, bytes_of_bits(any >> 4) * 0xffu};
            uint32_t nans = 0;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              v[p].x &= keep[0], v[p].y &= keep[1], v[p].z &= keep[0], v[p].w &= keep[1];
              nans |= nan_bytes(v[p].x) | nan_bytes(v[p].y) | nan_bytes(v[p].z) | nan_bytes(v[p].w);
            }
            if (__builtin_expect(__any(nans != 0), 0)) {
              const uint32_t bits = seen_bits(base + 16 * t, from, pos, sink);
              const half8 one = operand(bytes_of_bits(bits) * 0x38u, bytes_of_bits(bits >> 4) * 0x38u);
#pragma unroll
              for (int p = 0; p < 2; ++p) {
                const uint32_t n[4] = {nan_bytes(v[p].x), nan_bytes(v[p].y), nan_bytes(v[p].z), nan_bytes(v[p].w)};
                v[p].x &= ~(n[0] * 0xffu), v[p].y &= ~(n[1] * 0xffu), v[p].z &= ~(n[2] * 0xffu), v[p].w &= ~(n[3] * 0xffu);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  floatx16 hit;
#pragma unroll
                  for (int j = 0; j < 16; ++j) hit[j] = 0.f;
                  hit = __builtin_amdgcn_mfma_f32_32x32x16_f16(operand(n[2 * c] * 0x38u, n[2 * c + 1] * 0x38u), one, hit, 0, 0, 0);  // 0x38: 1
#pragma unroll
                  for (int j = 0; j < 16; ++j) o[2 * p + c][j] += hit[j] > 0.f ? __builtin_nanf("") : 0.f;
                }
              }
            }
          }
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const half8 v0 = operand(v[p].x, v[p].y), v1 = operand(v[p].z, v[p].w);
#pragma unroll
            for (int u = PARTS - 1; u >= 0; --u) {
              o[2 * p] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v0, pw[t][u], o[2 * p], 0, 0, 0);
              o[2 * p + 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v1, pw[t][u], o[2 * p + 1], 0, 0, 0);
            }
          }
        }
      }
      if (i + 1 < t_to) store_tile(b ^ 1);
      __syncthreads();
    };
    // The tiles that every row sees whole lie side by side, between the sinks and the window's left border and the diagonal.
    const int full_from = max(t_from, a.n_recent ? max((window_from(a, p_hi) + kTile) / kTile - span.skip, span.sinks) : 0);
    const int full_to = min(t_to, (p_lo + 1) / kTile - span.skip);
    int i = t_from;
    for (const int to = min(full_from, t_to); i < to; ++i) step(i, std::true_type{});
    for (; i < full_to; ++i) step(i, std::false_type{});
    for (; i < t_to; ++i) step(i, std::true_type{});

    l += __shfl_xor(l, 32);
    if (have) {
      const bool whole = at.np == 1;
      const int64_t slot = (int64_t)lh * plan.w.split + at.before + at.at;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      float* to = a.many.part + (slot * BR + 32 * wave + row) * kHeadDim;
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int r = 0; r < 4; ++r) {  // 8 channels side by side
          const int c0 = 64 * p + 16 * r + 8 * grp;
          float y[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) y[2 * j] = o[2 * p][4 * r + j], y[2 * j + 1] = o[2 * p + 1][4 * r + j];
          if (whole) {
            store8<BF16>(a.out, out_at + c0, y, inv);
          } else {
            *(float4*)(to + c0) = make_float4(y[0], y[1], y[2], y[3]), *(float4*)(to + c0 + 4) = make_float4(y[4], y[5], y[6], y[7]);
          }
        }
      if (!whole && grp == 0) a.many.stat[slot * BR + 32 * wave + row] = make_float2(m, l);
    }
  }
  return all;
}

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
    const uint32_t n = many_rows<BF16>(a, x, gridDim.x);
    if (x < n) x += (n - x + gridDim.x - 1) / gridDim.x * gridDim.x;  // its next turn
    x -= n;
  }
  if constexpr (R > 0) few_rows<BF16, R, kWaves>(a, x, gridDim.x);
}
// Tables of up to kShortTiles tiles: blocks are not cut, so nothing is to be joined; twice the waves share their tiles.  One sequence, 8 heads, us with parts
// and a join / so: fp32, 100 tokens 7.9 / 6.3, 500 9.1 / 9.2, 1000 9.4 / 12.2; bf16, 4 query heads, 500 9.3 / 8.7, 1000 9.6 / 11.0 (a workgroup cannot
// draw more than 50 KB a microsecond); 8 sequences of 1000 11.2 / 12.0, 64 29.0 / 30.3.
constexpr int kShortTiles = 17, kShortWaves = 8;
template <bool BF16, int R>
__global__ __launch_bounds__(kShortWaves* kWave, 2) void pages_short_kernel(PagesAttn a) {
  few_rows<BF16, R, kShortWaves>(a, blockIdx.x, gridDim.x);
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
