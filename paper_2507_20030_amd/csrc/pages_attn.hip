// Attention of new tokens over the 8-bit pages of their sequences.
//
//   o_t = sum_j p_j v_j,  p = softmax_j (scale q_t k_j),  over the tokens j that t sees.
//
// All products run on the matrix cores.  What keeps them exact:
//  * q k in bf16 calls: K goes in as the bytes it is stored as.  A bf16 number has 8 significant bits and is the sum of two e4m3 numbers of 4: the
//    nearest one and the rest, 32 times as large, which the instruction scales back.  A row of q is multiplied by the power of two that
//    brings its largest value to [2^7, 2^8); down to 2^-14 of that value the sum is exact, smaller ones err by 2^-22 of it.  Two products of
//    bytes take as long as one of fp16, and nothing has to be converted.
//  * q k in fp32 calls: fp16, which holds e4m3 exactly; q, its largest value in [2^14, 2^15), as the sum of two fp16 parts (22 bits).
//  * p v: fp16.
//  * the pages' exponents: that of K enters the score's factor; that of V joins the exponent of the weight.  With s_j the score times log2 e and
//    eV_j the exponent of j's page, the weights in the sum are P_j = 2^(s_j + eV_j - m), m a running bound of s_j + eV_j, and the
//    denominator is sum 2^(s_j - m) = sum P_j 2^-eV_j.  So no weight overflows fp16 or loses bits because its page is small.
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
  static constexpr int q_top = BF16 ? 7 : 14;  // rows of q: largest value in [2^q_top, 2^(q_top + 1))
};

// ------------------------------------------------------------------------------------------------ sharing out the work
// A block is `rows` consecutive (new token, query head of the KV head) pairs of a sequence; its tokens are cut into parts, one workgroup each, such that
// all parts of a call hold about the same number of tiles and there are about kParts of them.  Lengths live on the device, so every wave
// works out the shares by itself (64 sequences at a time): the launch only has to be large enough.
constexpr int kParts = 512;
constexpr int kLeastTiles = 4;
constexpr int kFewRows = 64;  // sequences of up to so many rows go to pages_few_kernel, where a call has both

template <int ROWS, int TOKENS>
struct Geometry {
  static constexpr int rows = ROWS, tile = TOKENS;  // of a block; of a tile
};
template <int R>
using Few = Geometry<16 * R, 32>;
using Many = Geometry<128, 64>;

struct Seq {
  int len, first, nq, rows, tiles;  // tokens, first new token (row of q), new tokens, rows of all blocks, most tiles of a block
};

template <class Geo>
__device__ __forceinline__ Seq seq_of(const PagesAttn& a, int b) {
  constexpr int BR = Geo::rows, kTile = Geo::tile;
  Seq s;
  s.len = min(max(a.lens[b], 0), a.S.max_pages << a.S.logP);
  s.first = min(max(a.starts[b], 0), a.n_tokens);
  s.nq = min(max(a.starts[b + 1], s.first), a.n_tokens) - s.first;
  s.rows = s.nq * a.S.G;
  if (s.rows <= a.rows_over || s.rows > a.rows_to) s.nq = s.rows = 0;
  s.tiles = (s.len + kTile - 1) / kTile;
  if (a.n_recent) {
    const int sink = (min(a.n_sink, s.len) + kTile - 1) / kTile;
    const int64_t span = (int64_t)a.n_recent + min(s.nq, BR / a.S.G + 2) + 2 * kTile;
    s.tiles = (int)min((int64_t)s.tiles, sink + span / kTile);
  }
  return s;
}

__device__ __forceinline__ int blocks_of(int rows, int BR) { return (rows + BR - 1) / BR; }

struct Shares {
  int tiles;  // of a part
  int parts;  // of all sequences, for one (layer, KV head)
  int split;  // ... of blocks that are cut
  int split_rows;  // rows of sequences whose blocks are cut
};
__device__ __forceinline__ int parts_of(const Seq& s, int tiles) { return s.nq ? max(1, (s.tiles + tiles - 1) / tiles) : 0; }

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

template <class Geo>
__device__ Shares shares_of(const PagesAttn& a, int lane) {
  float sum = 0.f;  // every wave adds in the same order: all agree
  for (int b0 = 0; b0 < a.batch; b0 += kWave)
    if (b0 + lane < a.batch) {
      const Seq s = seq_of<Geo>(a, b0 + lane);
      sum += (float)s.tiles * (float)blocks_of(s.rows, Geo::rows);
    }
  sum = wave_sum(sum) * (float)(a.n_layers * a.S.H);
  Shares w;
  w.tiles = max(kLeastTiles, (int)fminf(ceilf(sum / (float)kParts), 1e9f));
  w.parts = w.split = w.split_rows = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kWave)
    if (b0 + lane < a.batch) {
      const Seq s = seq_of<Geo>(a, b0 + lane);
      const int np = parts_of(s, w.tiles), n = np * blocks_of(s.rows, Geo::rows);
      w.parts += n;
      if (np > 1) w.split += n, w.split_rows += s.rows;
    }
  w.parts = wave_sum(w.parts), w.split = wave_sum(w.split), w.split_rows = wave_sum(w.split_rows);
  return w;
}

// The sequence that holds entry y of a numbering that gives every sequence count(its Seq, its parts) entries: its index, y's place in it, and how many
// parts of cut blocks the sequences before it have.
struct Place {
  int b, at, before, np;
  Seq s;
};
template <class Geo, class Count>
__device__ Place place_of(const PagesAttn& a, const Shares& w, int y, int lane, Count count) {
  int done = 0, cut = 0;
  for (int b0 = 0;; b0 += kWave) {
    Seq s{0, 0, 0, 0, 0};
    int np = 0, n = 0, c = 0;
    if (b0 + lane < a.batch) {
      s = seq_of<Geo>(a, b0 + lane);
      np = parts_of(s, w.tiles);
      n = count(s, np);
      c = np > 1 ? np * blocks_of(s.rows, Geo::rows) : 0;
    }
    int in = n, cin = c;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const int u = __shfl_up(in, d), v = __shfl_up(cin, d);
      if (lane >= d) in += u, cin += v;
    }
    const unsigned long long m = __ballot(y < done + in);
    if (m || b0 + kWave >= a.batch) {  // always found: y is below the sum of all counts
      const int src = m ? __builtin_ctzll(m) : 0;
      const auto uni = [&](int x) { return __builtin_amdgcn_readlane(x, src); };
      Place p;
      p.b = b0 + src, p.at = y - done - uni(in - n), p.before = cut + uni(cin - c), p.np = uni(np);
      p.s.len = uni(s.len), p.s.first = uni(s.first), p.s.nq = uni(s.nq), p.s.rows = uni(s.rows), p.s.tiles = uni(s.tiles);
      return p;
    }
    done += __builtin_amdgcn_readlane(in, kWave - 1), cut += __builtin_amdgcn_readlane(cin, kWave - 1);
  }
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
template <int N, int PARTS>
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
// 16 values as bytes hi + 2^-5 lo; what is not finite becomes NaN.
typedef int intx8 __attribute__((ext_vector_type(8)));
constexpr int kOne = 0x7f7f7f7f, kThirtySecond = 0x7a7a7a7a;  // scales of the matrix instructions: 2^0, 2^-5
__device__ __forceinline__ void to_bytes(const float* x, int* hi, int* lo) {
#pragma unroll
  for (int c = 0; c < 16; c += 4) {
    float y[4], back[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = fabsf(x[c + j]) <= (float)kE4m3Max ? x[c + j] : __builtin_nanf("");
    hi[c / 4] = (int)floats_e4m3(y);
    e4m3_floats((uint32_t)hi[c / 4], back);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = 32.f * (y[j] - back[j]);
    lo[c / 4] = (int)floats_e4m3(y);
  }
}
__device__ __forceinline__ intx8 operand8(uint4 a, uint4 b) { return intx8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w}; }
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

// A row at position p sees the tokens (from, p] and those below sink.
__device__ __forceinline__ int window_from(const PagesAttn& a, int p) { return a.n_recent ? max(p - a.n_recent, -1) : -1; }  // p >= -1, n_recent >= 0: no overflow
__device__ __forceinline__ bool sees(int t, int from, int to, int sink) { return (t <= to) & ((t > from) | (t < sink)); }

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
    from = (int)(max((int64_t)0, (int64_t)p_lo - a.n_recent + 1) / kTile);
    s.sinks = a.n_sink > 0 ? min((min(a.n_sink, p_hi + 1) + kTile - 1) / kTile, end) : 0;
  }
  s.skip = max(from - s.sinks, 0);
  s.n = max(end - s.skip, s.sinks);
  return s;
}

// One row tile of 16 query rows: lane l holds row l % 16.
template <int PARTS>
struct Rows {
  half8 q[PARTS == 1 ? 1 : 4][PARTS];  // fp32: [chunk of 16 channels oct + 4 (c / 2)][8 of them: c % 2]
  intx8 q8[2];                         // bf16: both chunks, hi and lo
  floatx4 o[8];   // [16-byte load of V][channel of the pair]: row l % 16, channels 32 (i / 2) + 8 (l / 16) + 2 c + i % 2
  float m, l, factor;
  int pos, from, eq;
};

// ------------------------------------------------------------------------------------------------ few rows
// A workgroup has a part of the tokens of one block of 16 R rows; its four waves take the tiles in turn and join their sums in the end.  A tile of 32
// tokens is 8 KB, eight 16-byte loads a lane, the next one's in flight while this one is multiplied: S^T = K Q^T leaves lane l
// with row l % 16 and the 8 tokens of octet l / 16, which is how O^T = V^T P^T wants them, so nothing moves between lanes but the maximum.
template <bool BF16, int R>
__global__ __launch_bounds__(kWaves* kWave) void pages_few_kernel(PagesAttn a) {
  using Geo = Few<R>;
  constexpr int PARTS = BF16 ? 1 : 2, BR = Geo::rows, kTile = Geo::tile, kQTop = Weights<BF16>::q_top;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int row = lane & 15, oct = lane >> 4;
  __shared__ __attribute__((aligned(16))) float join[2][BR][kHeadDim + 4];
  __shared__ float2 join_stat[2][BR];

  const Shares w = shares_of<Geo>(a, lane);
  const int64_t all = (int64_t)w.parts * a.n_layers * a.S.H;
  for (int64_t x = blockIdx.x; x < all; x += gridDim.x) {
    const int lh = (int)(x % (a.n_layers * a.S.H));  // workgroups are dealt to the XCDs in turn: with 8 heads each reads one head's pages
    const Place at = place_of<Geo>(a, w, (int)(x / (a.n_layers * a.S.H)), lane, [](const Seq& s, int np) { return np * blocks_of(s.rows, Geo::rows); });
    const Seq s = at.s;
    const int block = blocks_of(s.rows, BR) - 1 - at.at / at.np, part = at.at % at.np, layer = lh / a.S.H, h = lh % a.S.H, G = a.S.G;
    const int row0 = block * BR, rows = min(s.rows - row0, BR);
    const int before = s.len - s.nq;  // position of the sequence's first new token
    const int p_lo = before + row0 / G, p_hi = before + (row0 + rows - 1) / G;
    const Span span = span_of<kTile>(a, p_lo, p_hi);
    const int t_from = (int)((int64_t)span.n * part / at.np), t_to = (int)((int64_t)span.n * (part + 1) / at.np);
    const int n_rt = (rows + 15) / 16;
    const int sink = a.n_recent ? a.n_sink : 0, all_from = window_from(a, max(p_lo, -1));

    Rows<PARTS> rt[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      Rows<PARTS>& z = rt[r];
      const int mine = row0 + 16 * r + row;
      const bool have = 16 * r + row < rows;
      z.pos = have ? max(before + mine / G, -1) : -1, z.from = window_from(a, z.pos);
      z.m = -FLT_MAX, z.l = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) z.o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
      float f[2][16];
      float top = 0.f;
      if (have) {
        const int64_t base = (((int64_t)layer * a.n_tokens + s.first + mine / G) * (a.S.H * G) + h * G + mine % G) * kHeadDim;
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
      if constexpr (BF16) {
        int hi[8], lo[8];
        to_bytes(f[0], hi, lo), to_bytes(f[1], hi + 4, lo + 4);
#pragma unroll
        for (int c = 0; c < 8; ++c) z.q8[0][c] = hi[c], z.q8[1][c] = lo[c];
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) to_halves<8, PARTS>(f[c / 2] + 8 * (c % 2), z.q[c]);
      }
    }

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

    const int first = t_from + wave;
    Ids id{0, 0};
    Data next{};
    if (first < t_to) {
      next = load_tile(first, pages_at(first));
      if (first + kWaves < t_to) id = pages_at(first + kWaves);
    }
    for (int i = first; i < t_to; i += kWaves) {
      Data d = next;
      if (i + kWaves < t_to) {
        next = load_tile(i + kWaves, id);
        if (i + 2 * kWaves < t_to) id = pages_at(i + 2 * kWaves);
      }
      const int t0 = span.tile(i) * kTile, t1 = t0 + kTile - 1, j0 = t0 + 8 * oct;
      // whether every row sees the whole tile
      const bool edge = t1 > p_lo || (t1 >= sink && t0 <= window_from(a, p_hi)) || __any(d.bad);
      bool poison = false;
      if (edge) {  // tokens that no row sees may hold anything
        uint32_t keep[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int t = j0 + j;
          const bool seen = !d.bad & sees(t, all_from, p_hi, sink);
          keep[j / 4] |= seen ? 0xffu << (8 * (j % 4)) : 0u;
        }
        uint32_t nans = 0;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          d.v[p].x &= keep[0], d.v[p].y &= keep[1], d.v[p].z &= keep[0], d.v[p].w &= keep[1];
          nans |= nan_bytes(d.v[p].x) | nan_bytes(d.v[p].y) | nan_bytes(d.v[p].z) | nan_bytes(d.v[p].w);
        }
        poison = __any(nans != 0);
      }

      half8 kf[2][BF16 ? 1 : 4];
      if constexpr (!BF16)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int p = 0; p < 2; ++p) kf[u][2 * p] = operand(d.k[u][p].x, d.k[u][p].y), kf[u][2 * p + 1] = operand(d.k[u][p].z, d.k[u][p].w);
      const float ev = (float)d.e.y;
      half8 pw[R][PARTS], ones[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r >= n_rt) continue;
        Rows<PARTS>& z = rt[r];
        float sc[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          floatx4 acc{0.f, 0.f, 0.f, 0.f};
          if constexpr (BF16) {
            const intx8 k8 = operand8(d.k[u][0], d.k[u][1]);
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k8, z.q8[1], acc, 0, 0, 0, kOne, 0, kThirtySecond);
            acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k8, z.q8[0], acc, 0, 0, 0, kOne, 0, kOne);
          } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int p = PARTS - 1; p >= 0; --p) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[u][c], z.q[c][p], acc, 0, 0, 0);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) sc[4 * u + j] = acc[j];
        }
        const float factor = ldexpf(a.scale, z.eq - kQTop + d.e.x);
#pragma unroll
        for (int j = 0; j < 8; ++j) sc[j] = sc[j] * factor + ev;
        if (edge) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int t = j0 + j;
            const bool seen = !d.bad & sees(t, z.from, z.pos, sink);
            ones[r][j] = seen ? (_Float16)1.f : (_Float16)0.f;
            sc[j] = seen ? sc[j] : -__builtin_inff();
          }
        }
        float top = sc[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, sc[j]);
        if (__any(top > z.m + Weights<BF16>::slack)) {
          top = fmaxf(z.m, max_over_16s(top));
          const float fade = __builtin_amdgcn_exp2f(z.m - top);
          z.m = top, z.l *= fade;
#pragma unroll
          for (int c = 0; c < 8; ++c) z.o[c] *= fade;
        }
        float y[8], sum = 0.f;
        const float ref = z.m - Weights<BF16>::lift;
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = __builtin_amdgcn_exp2f(sc[j] - ref), sum += y[j];
        z.l += ldexpf(sum, -d.e.y);
        to_halves<8, PARTS>(y, pw[r]);
      }
      half8 vf[8];
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        uint4 v = d.v[p];
        if (poison) {  // NaN where only some rows may see it: taken out here, brought back to those rows
          const uint32_t n[4] = {nan_bytes(v.x), nan_bytes(v.y), nan_bytes(v.z), nan_bytes(v.w)};
          v.x &= ~(n[0] * 0xffu), v.y &= ~(n[1] * 0xffu), v.z &= ~(n[2] * 0xffu), v.w &= ~(n[3] * 0xffu);
          const half8 bad[2] = {operand(n[0] * 0x38u, n[1] * 0x38u), operand(n[2] * 0x38u, n[3] * 0x38u)};  // 0x38: 1
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if (r >= n_rt) continue;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const floatx4 hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(bad[c], ones[r], floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (hit[j] > 0.f) rt[r].o[2 * p + c][j] = __builtin_nanf("");
            }
          }
        }
        vf[2 * p] = operand(v.x, v.y), vf[2 * p + 1] = operand(v.z, v.w);
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r >= n_rt) continue;
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p) rt[r].o[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[c], pw[r][p], rt[r].o[c], 0, 0, 0);
      }
    }

    // the four waves' sums: 2 and 3 to 0 and 1, then 1 to 0
#pragma unroll
    for (int r = 0; r < R; ++r) {
      rt[r].l += __shfl_xor(rt[r].l, 16);
      rt[r].l += __shfl_xor(rt[r].l, 32);
    }
#pragma unroll
    for (int from = 2; from >= 1; --from) {
      __syncthreads();
      if (wave >= from && wave < 2 * from)
#pragma unroll
        for (int r = 0; r < R; ++r) {
          float* at_row = join[wave - from][16 * r + row] + 8 * oct;
#pragma unroll
          for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) at_row[32 * (c / 2) + 2 * j + c % 2] = rt[r].o[c][j];
          if (oct == 0) join_stat[wave - from][16 * r + row] = make_float2(rt[r].m, rt[r].l);
        }
      __syncthreads();
      if (wave < from)
#pragma unroll
        for (int r = 0; r < R; ++r) {
          Rows<PARTS>& z = rt[r];
          const float* at_row = join[wave][16 * r + row] + 8 * oct;
          const float2 st = join_stat[wave][16 * r + row];
          const float m = fmaxf(z.m, st.x), f0 = __builtin_amdgcn_exp2f(z.m - m), f1 = __builtin_amdgcn_exp2f(st.x - m);
          z.m = m, z.l = z.l * f0 + st.y * f1;
#pragma unroll
          for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) z.o[c][j] = z.o[c][j] * f0 + at_row[32 * (c / 2) + 2 * j + c % 2] * f1;
        }
    }
    if (wave == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const Rows<PARTS>& z = rt[r];
        if (16 * r + row >= rows) continue;
        if (at.np == 1) {
          const int mine = row0 + 16 * r + row;
          const int64_t base = (((int64_t)layer * a.n_tokens + s.first + mine / G) * (a.S.H * G) + h * G + mine % G) * kHeadDim + 8 * oct;
          const float inv = z.l == 0.f ? 0.f : 1.f / z.l;
#pragma unroll
          for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) store_kv<BF16>(a.out, base + 32 * (c / 2) + 2 * j + c % 2, z.o[c][j] * inv);
        } else {
          const int64_t slot = (int64_t)lh * w.split + at.before + at.at;
          float* to = a.part + (slot * BR + 16 * r + row) * kHeadDim + 8 * oct;
#pragma unroll
          for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) to[32 * (c / 2) + 2 * j + c % 2] = z.o[c][j];
          if (oct == 0) a.stat[slot * BR + 16 * r + row] = make_float2(z.m, z.l);
        }
      }
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------ many rows
// Prompts: four waves of 32 rows share tiles of 64 tokens that go through LDS as bytes, the next tile's loads in flight while this one is multiplied; a wave
// turns the bytes into operands itself (32 conversions per 8 products of 32 cycles; fp16 in LDS would need the LDS's whole bandwidth).
// S^T = K Q^T leaves lane l with row l % 32 and tokens 16 t + 8 (l / 32) + j, the operand of O^T = V^T P^T.  K's 16-byte chunks are
// swizzled by their token so that the eight lanes of a bank group read eight different ones.
template <bool BF16>
__global__ __launch_bounds__(kWaves* kWave, BF16 ? 2 : 1) void pages_many_kernel(PagesAttn a) {
  using Geo = Many;
  constexpr int PARTS = BF16 ? 1 : 2, BR = Geo::rows, kTile = Geo::tile, kHalf = 32, kQTop = Weights<BF16>::q_top;
  constexpr float kLift = Weights<BF16>::lift;
  static_assert(BR == 32 * kWaves && kTile == 2 * kHalf, "");
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int row = lane & 31, grp = lane >> 5;
  __shared__ __attribute__((aligned(16))) uint8_t kbuf[2][kTile * kHeadDim], vbuf[2][kTile * kHeadDim];
  __shared__ float4 meta[2][kTile / kOct];  // of the octets' pages: scale 2^(eK - kQTop), eV, 2^-eV

  const Shares w = shares_of<Geo>(a, lane);
  const int64_t all = (int64_t)w.parts * a.n_layers * a.S.H;
  for (int64_t x = blockIdx.x; x < all; x += gridDim.x) {
    const int lh = (int)(x % (a.n_layers * a.S.H));
    const Place at = place_of<Geo>(a, w, (int)(x / (a.n_layers * a.S.H)), lane, [](const Seq& s, int np) { return np * blocks_of(s.rows, BR); });
    const Seq s = at.s;
    const int block = blocks_of(s.rows, BR) - 1 - at.at / at.np, part = at.at % at.np, layer = lh / a.S.H, h = lh % a.S.H, G = a.S.G;
    const int row0 = block * BR, rows = min(s.rows - row0, BR), before = s.len - s.nq;
    const int p_lo = before + row0 / G, p_hi = before + (row0 + rows - 1) / G;
    const Span span = span_of<kTile>(a, p_lo, p_hi);
    const int t_from = (int)((int64_t)span.n * part / at.np), t_to = (int)((int64_t)span.n * (part + 1) / at.np);

    const int mine = row0 + 32 * wave + row;  // of the sequence's rows
    const bool have = 32 * wave + row < rows;
    const int pos = have ? max(before + mine / G, -1) : -1;
    const bool any_row = 32 * wave < rows;
    const int w_lo = before + (row0 + 32 * wave) / G, w_hi = any_row ? before + (row0 + min(32 * wave + 32, rows) - 1) / G : -1;  // positions of the wave's rows
    const int sink = a.n_recent ? a.n_sink : 0, from = window_from(a, pos), w_from = window_from(a, max(w_lo, -1));
    const int64_t out_at = (((int64_t)layer * a.n_tokens + s.first + mine / G) * (a.S.H * G) + h * G + mine % G) * kHeadDim;

    half8 q[BF16 ? 1 : 8][PARTS];  // fp32: [chunk of 16 channels 2 (c / 2) + grp][8 of them: c % 2]
    intx8 q8[2][2];                // bf16: [two chunks][hi, lo]
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
      if constexpr (BF16) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          int hi[8], lo[8];
          to_bytes(f[2 * c], hi, lo), to_bytes(f[2 * c + 1], hi + 4, lo + 4);
#pragma unroll
          for (int j = 0; j < 8; ++j) q8[c][0][j] = hi[j], q8[c][1][j] = lo[j];
        }
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c) to_halves<8, PARTS>(f[c / 2] + 8 * (c % 2), q[c]);
      }
    }
    const float q_scale = ldexpf(1.f, eq);
    floatx16 o[4];  // rows 8 (i / 4) + 4 grp + i % 4 =: u of channel tile c: channel 64 (c / 2) + 2 u + c % 2
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
    float m = -FLT_MAX, l = 0.f;

    // a wave brings octets wave and wave + 4 of a tile; their pages are looked up a tile earlier
    const int32_t* table = a.table + (int64_t)at.b * a.S.max_pages;
    const int last_page = max(page_count(s.len, a.S.logP) - 1, 0), in_page = (1 << a.S.logP) - 1;
    int next_page[2] = {0, 0};
    uint4 nk[2], nv[2];
    int2 ne[2];
    bool none[2];
    const auto find_tile = [&](int i) {
#pragma unroll
      for (int u = 0; u < 2; ++u) next_page[u] = table[min((span.tile(i) * kTile + kOct * (wave + kWaves * u)) >> a.S.logP, last_page)];
    };
    const auto load_tile = [&](int i) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int t = span.tile(i) * kTile + kOct * (wave + kWaves * u);
        int page = __builtin_amdgcn_readfirstlane(next_page[u]);
        none[u] = page < 0 || page >= a.S.n_pages;
        page = none[u] ? 0 : page;
        const int64_t ph = page_head(a.S, a.layer + layer, page, h);
        const uint8_t* at_k = page_values(a.S, ph) + (t & in_page) * kHeadDim;
        nk[u] = ((const uint4*)at_k)[lane];
        nv[u] = ((const uint4*)(at_k + ((size_t)kHeadDim << a.S.logP)))[lane];
        ne[u] = *(const int2*)(a.S.exponents + 2 * ph);
      }
    };
    const auto store_tile = [&](int b) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float4 e = make_float4(ldexpf(a.scale, ne[u].x - kQTop), (float)ne[u].y, ldexpf(1.f, -ne[u].y), 0.f);
        if (none[u]) {  // a page that is not there: scores of -infinity, weights and values of 0
          nk[u] = nv[u] = make_uint4(0, 0, 0, 0);
          e = make_float4(0.f, -__builtin_inff(), 0.f, 0.f);
        }
        const int oc = wave + kWaves * u, tok = lane >> 3, ch = lane & 7;
        ((uint4*)kbuf[b])[(kOct * oc + tok) * 8 + (ch ^ ((tok & 3) | ((oc & 1) << 2)))] = nk[u];
        ((uint4*)vbuf[b])[64 * oc + lane] = nv[u];
        if (lane == 0) meta[b][oc] = e;
      }
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
        if constexpr (BF16) {
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const intx8 k8 = operand8(chunk(u, 2 * c), chunk(u, 2 * c + 1));
              acc[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k8, q8[c][1], acc[u], 0, 0, 0, kOne, 0, kThirtySecond);
              acc[u] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k8, q8[c][0], acc[u], 0, 0, 0, kOne, 0, kOne);
            }
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint4 kw = chunk(u, c);
              const half8 k0 = operand(kw.x, kw.y), k1 = operand(kw.z, kw.w);
#pragma unroll
              for (int p = PARTS - 1; p >= 0; --p) {
                acc[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k0, q[2 * c][p], acc[u], 0, 0, 0);
                acc[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k1, q[2 * c + 1][p], acc[u], 0, 0, 0);
              }
            }
        }
        const int base = t0 + 8 * grp;  // tokens of the lane: base + 16 t + j
        float inv[4];
        float sc[32];  // exponents of the weights as they enter the sums: relative to m - lift
        const bool unset = m == -FLT_MAX;  // the row has seen nothing: relative to 0
        const float ref = (unset ? 0.f : m) - kLift;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float4 e = meta[b][2 * t + grp];
          const float factor = e.x * q_scale, shift = e.y - ref;
          inv[t] = e.z;
#pragma unroll
          for (int j = 0; j < 8; ++j) sc[8 * t + j] = acc[t / 2][8 * (t % 2) + j] * factor + shift;
        }
        if constexpr (EDGE) {
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < 8; ++j) sc[8 * t + j] = sees(base + 16 * t + j, from, pos, sink) ? sc[8 * t + j] : -__builtin_inff();
        }
        float top = sc[0];
#pragma unroll
        for (int j = 1; j < 32; ++j) top = fmaxf(top, sc[j]);
        if (__any(top > (unset ? -FLT_MAX : kLift + Weights<BF16>::slack))) {
          top = fmaxf(top, __shfl_xor(top, 32));
          const bool first = unset && top >= -FLT_MAX;
          const float up = unset ? (first ? top - kLift : 0.f) : fmaxf(top - kLift, 0.f), fade = unset ? 1.f : __builtin_amdgcn_exp2f(-up);
          m = first ? up : m + up, l *= fade;
#pragma unroll
          for (int j = 0; j < 32; ++j) sc[j] -= up;
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[c][j] *= fade;
        }
        half8 pw[4][PARTS];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float y[8], sum = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = __builtin_amdgcn_exp2f(sc[8 * t + j]);
          to_halves<8, PARTS>(y, pw[t]);
          if constexpr (PARTS == 1) {  // of the rounded weights: half the instructions, and they add up to 1
#pragma unroll
            for (int j = 0; j < 8; j += 2) sum = __builtin_amdgcn_fdot2(half2v{pw[t][0][j], pw[t][0][j + 1]}, half2v{(_Float16)1.f, (_Float16)1.f}, sum, false);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += y[j];
          }
          l += sum * inv[t];
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          uint4 v[2];
#pragma unroll
          for (int p = 0; p < 2; ++p) v[p] = ((const uint4*)vbuf[b])[(2 * t + grp) * 64 + 32 * p + row];
          if constexpr (EDGE) {  // tokens that no row sees may hold anything; NaN that only some rows see is brought back to those
            uint32_t keep[2] = {0, 0}, nans = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) keep[j / 4] |= sees(base + 16 * t + j, w_from, w_hi, sink) ? 0xffu << (8 * (j % 4)) : 0u;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              v[p].x &= keep[0], v[p].y &= keep[1], v[p].z &= keep[0], v[p].w &= keep[1];
              nans |= nan_bytes(v[p].x) | nan_bytes(v[p].y) | nan_bytes(v[p].z) | nan_bytes(v[p].w);
            }
            if (__builtin_expect(__any(nans != 0), 0)) {
              half8 one;
#pragma unroll
              for (int j = 0; j < 8; ++j) one[j] = sees(base + 16 * t + j, from, pos, sink) ? (_Float16)1.f : (_Float16)0.f;
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
      const int64_t slot = (int64_t)lh * w.split + at.before + at.at;
      const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
      float* to = a.part + (slot * BR + 32 * wave + row) * kHeadDim;
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int r = 0; r < 4; ++r) {  // 8 channels side by side
          const int c0 = 64 * p + 16 * r + 8 * grp;
          float y[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) y[2 * j] = o[2 * p][4 * r + j] * inv, y[2 * j + 1] = o[2 * p + 1][4 * r + j] * inv;
          if (whole) {
#pragma unroll
            for (int j = 0; j < 8; ++j) store_kv<BF16>(a.out, out_at + c0 + j, y[j]);
          } else {
            *(float4*)(to + c0) = make_float4(y[0], y[1], y[2], y[3]), *(float4*)(to + c0 + 4) = make_float4(y[4], y[5], y[6], y[7]);
          }
        }
      if (!whole && grp == 0) a.stat[slot * BR + 32 * wave + row] = make_float2(m, l);
    }
  }
}

// Rows whose tokens were shared out: one workgroup per row, its waves take the parts in turn.
template <bool BF16, class Geo>
__global__ __launch_bounds__(kWaves* kWave) void pages_join_kernel(PagesAttn a) {
  constexpr int BR = Geo::rows;
  __shared__ float2 sums[kWaves][kWave];
  __shared__ float dens[kWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const Shares w = shares_of<Geo>(a, lane);
  const int64_t all = (int64_t)w.split_rows * a.n_layers * a.S.H;
  for (int64_t x = blockIdx.x; x < all; x += gridDim.x) {
    const int lh = (int)(x / w.split_rows);
    const Place at = place_of<Geo>(a, w, (int)(x % w.split_rows), lane, [](const Seq& s, int np) { return np > 1 ? s.rows : 0; });
    const int r = at.at, G = a.S.G;
    const int64_t slot = (int64_t)lh * w.split + at.before + (int64_t)(blocks_of(at.s.rows, BR) - 1 - r / BR) * at.np;
    const float2* stat = a.stat + slot * BR + r % BR;
    const float* part = a.part + (slot * BR + r % BR) * kHeadDim + 2 * lane;
    float m = -FLT_MAX;
    for (int k = lane; k < at.np; k += kWave) m = fmaxf(m, stat[(int64_t)k * BR].x);
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    float2 o = make_float2(0.f, 0.f);
    float l = 0.f;
    for (int k = wave; k < at.np; k += kWaves) {
      const float2 st = stat[(int64_t)k * BR], v = *(const float2*)(part + (int64_t)k * BR * kHeadDim);
      const float f = __builtin_amdgcn_exp2f(st.x - m);
      o.x += v.x * f, o.y += v.y * f, l += st.y * f;
    }
    sums[wave][lane] = o;
    if (lane == 0) dens[wave] = l;
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int i = 1; i < kWaves; ++i) o.x += sums[i][lane].x, o.y += sums[i][lane].y, l += dens[i];
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int layer = lh / a.S.H, h = lh % a.S.H;
      const int64_t base = (((int64_t)layer * a.n_tokens + at.s.first + r / G) * (a.S.H * G) + h * G + r % G) * kHeadDim + 2 * lane;
      store_kv<BF16>(a.out, base, o.x * inv), store_kv<BF16>(a.out, base + 1, o.y * inv);
    }
    __syncthreads();
  }
}

// Parts of cut blocks: a block of more than w.tiles tiles has fewer than 2 tiles / w.tiles of them, all blocks together kParts w.tiles tiles (rounding: + 64).
constexpr int64_t kMostCut = 2 * kParts + 64;

// What a call launches.  A sequence's rows are known on the device only; what the sizes exclude is not launched.
struct Launches {
  int few = 0;        // row tiles of pages_few_kernel's blocks, 0: not launched
  bool many = false;  // pages_many_kernel
  size_t few_bytes = 0, bytes = 0;  // of the workspace
};
Launches launches_of(const Pages& S, int batch, int n_tokens, bool bf16) {
  Launches n;
  const int64_t rows = (int64_t)n_tokens * S.G, average = S.G * (((int64_t)n_tokens + batch - 1) / batch);
  n.many = rows > kFewRows;
  if (!n.many || batch > 1) {
    const int64_t usual = std::min<int64_t>(average > kFewRows ? S.G : average, kFewRows);  // beside prompts: single tokens
    n.few = usual <= 16 ? 1 : usual <= 32 || !bf16 ? 2 : 4;
  }
  const auto part = [](int64_t block) { return (size_t)kMostCut * (size_t)block * (kHeadDim * sizeof(float) + sizeof(float2)); };
  const int64_t most = ((int64_t)S.max_pages << S.logP) / 32 + 1;  // tiles of a sequence
  if (most > kLeastTiles) {                                       // else no block is ever cut
    n.few_bytes = n.few ? part(16 * n.few) : 0;
    n.bytes = n.few_bytes + (n.many ? part(Many::rows) : 0);
  }
  return n;
}

template <class Geo, class Kernel, class Join>
hipError_t launch_blocks(PagesAttn a, Kernel kernel, Join join, char* ws, hipStream_t st) {
  a.part = (float*)ws;
  a.stat = ws ? (float2*)(a.part + kMostCut * Geo::rows * kHeadDim) : nullptr;
  const int64_t lh = (int64_t)a.n_layers * a.S.H, blocks = (int64_t)a.n_tokens * a.S.G / Geo::rows + a.batch;
  kernel<<<(unsigned)std::min<int64_t>(kParts + lh * blocks, 1 << 20), kWaves * kWave, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !ws) return e;
  join<<<(unsigned)std::min<int64_t>(lh * a.n_tokens * a.S.G, 2048), kWaves * kWave, 0, st>>>(a);
  return hipGetLastError();
}

template <bool BF16, int R>
hipError_t launch_few(const PagesAttn& a, char* ws, hipStream_t st) {
  return launch_blocks<Few<R>>(a, pages_few_kernel<BF16, R>, pages_join_kernel<BF16, Few<R>>, ws, st);
}
template <bool BF16>
hipError_t launch_many(const PagesAttn& a, char* ws, hipStream_t st) {
  return launch_blocks<Many>(a, pages_many_kernel<BF16>, pages_join_kernel<BF16, Many>, ws, st);
}

}  // namespace

size_t pages_attn_bytes(const Pages& S, int batch, int n_tokens, bool bf16) {
  return batch == 0 || n_tokens == 0 ? 0 : launches_of(S, batch, n_tokens, bf16).bytes;
}

hipError_t launch_pages_attn(PagesAttn a, bool bf16, void* ws, hipStream_t st) {
  const Launches n = launches_of(a.S, a.batch, a.n_tokens, bf16);
  char* few = n.bytes ? (char*)ws : nullptr;
  a.rows_to = 0x7fffffff;
  if (n.many) {  // the longer work first
    a.rows_over = n.few ? kFewRows : 0;
    char* many = n.bytes ? (char*)ws + n.few_bytes : nullptr;
    const hipError_t e = bf16 ? launch_many<true>(a, many, st) : launch_many<false>(a, many, st);
    if (e != hipSuccess || !n.few) return e;
    a.rows_to = kFewRows;
  }
  a.rows_over = 0;
  if (bf16) return n.few == 1 ? launch_few<true, 1>(a, few, st) : n.few == 2 ? launch_few<true, 2>(a, few, st) : launch_few<true, 4>(a, few, st);
  return n.few == 1 ? launch_few<false, 1>(a, few, st) : launch_few<false, 2>(a, few, st);
}

}  // namespace iwdft
