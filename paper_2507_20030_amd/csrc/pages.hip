// The 8-bit paged cache: block tables and slot maps from lengths, new tokens into the pages, the pages' tokens back.
#include <algorithm>

#include "pages.h"

namespace iwdft {

namespace {

constexpr int kWave = 64;

// ------------------------------------------------------------------------------------------------ block tables
// free[0] pages lie on a stack, free[1 ..]; a call gives back R pages and takes A.  With V = (stack, R given back) and its top at the end, page i that is
// taken is V[count + R - 1 - i], and where fewer are taken than given back the first R - A of the latter are pushed.  The stack is
// either read or written, never both, so nothing has to be ordered.  Pages are given back from the last one of the last sequence on:
// a call that undoes another one leaves the stack as it was.
struct ResizeState {
  int count, released, taken, total;  // total: new tokens
};

struct Change {
  int have, want;  // want: have where the sequence stays or cannot be so long
};
__device__ __forceinline__ Change change_of(const ResizeArgs& a, int b) {
  const int most = a.max_pages << a.logP;
  Change c;
  c.have = min(max(a.lens[b], 0), most);
  const int w = a.want[b];
  c.want = w < 0 || w > most ? c.have : w;
  return c;
}

// What a thread of the filling kernel looks up.
struct Fill {
  const int32_t *have, *now, *need, *gone, *starts;  // per sequence: old length, new one, new pages of those before, pages given back before
  ResizeState s;
};

__device__ __forceinline__ int last_not_above(const int32_t* v, int n, int x) {  // largest i < n with v[i] <= x (v ascending, v[0] <= x)
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (v[m] <= x) lo = m;
    else hi = m;
  }
  return lo;
}

// k-th page that is given back.
__device__ __forceinline__ int released_page(const ResizeArgs& a, const Fill& f, int k) {
  const int ord = f.s.released - 1 - k, b = last_not_above(f.gone, a.batch, ord);
  const int j = page_count(f.now[b], a.logP) + ord - f.gone[b];
  return (uint32_t)j < (uint32_t)a.max_pages ? a.table[(int64_t)b * a.max_pages + j] : -1;  // always, unless lengths are damaged
}

__device__ void resize_fill(const ResizeArgs& a, const Fill& f, int at, int step) {
  const int P = 1 << a.logP;
  for (int64_t t0 = at; t0 < a.n_slots; t0 += step) {
    const int t = (int)t0;
    int slot = -1;
    if (t < f.s.total) {
      const int b = last_not_above(f.starts, a.batch, t);
      const int have = f.have[b], had = page_count(have, a.logP), pos = have + t - f.starts[b], j = pos >> a.logP;
      int32_t* row = a.table + (int64_t)b * a.max_pages;
      int page;
      if (j < had) {
        page = row[j];
      } else {
        const int v = f.s.count + f.s.released - 1 - (f.need[b] + j - had);
        page = v < f.s.count ? a.free[1 + v] : released_page(a, f, v - f.s.count);
        if ((pos & (P - 1)) == 0) row[j] = page;
      }
      if (page >= 0 && page < a.n_pages) slot = (page << a.logP) + (pos & (P - 1));
    }
    a.slots[t] = slot;
  }
  const int push = min(f.s.released - f.s.taken, a.n_pages - f.s.count);
  for (int64_t k = at; k < push; k += step) a.free[1 + f.s.count + (int)k] = released_page(a, f, (int)k);
}

// ONE: up to kResizeOneBatch sequences and kResizeOneSlots slots, everything in this launch.  A decode step's call is the chain of loads, sums and
// stores of one workgroup.  Otherwise resize_fill_kernel follows.  THREADS: 256 sequences, 5.6 us with 1024 threads, whose 16 waves join their sums, 2.2 with 256.
template <bool ONE, int THREADS>
__global__ __launch_bounds__(THREADS) void resize_kernel(ResizeArgs a) {
  __shared__ long long lds3[THREADS / kWave][3], lds2[THREADS / kWave][2], lds1[THREADS / kWave][1];
  __shared__ int32_t keep[ONE ? 4 * kResizeOneBatch : 1];
  int32_t *have = ONE ? keep : a.scratch + 4, *need = have + (ONE ? kResizeOneBatch : a.batch), *gone = need + (ONE ? kResizeOneBatch : a.batch);
  int32_t* starts = ONE ? gone + kResizeOneBatch : a.starts;
  const int tid = threadIdx.x;
  const int count = min(max(a.free[0], 0), a.n_pages);
  const auto pages_gone = [&](const Change& c) { return max(0, page_count(c.have, a.logP) - page_count(c.want, a.logP)); };

  long long given = 0;  // pages given back by all: they serve this call too
  if (!ONE && a.batch > THREADS)
    for (int b0 = 0; b0 < a.batch; b0 += THREADS) {
      const int b = b0 + tid, x[1] = {b < a.batch ? pages_gone(change_of(a, b)) : 0};
      long long before[1], all[1];
      sums_before<THREADS>(x, before, all, lds1);
      given += all[0];
    }

  long long asked = 0, fresh = 0, back = 0;
  int taken = 0, total = 0, released = 0;
  for (int b0 = 0; b0 < a.batch; b0 += THREADS) {
    const int b = b0 + tid;
    Change c{0, 0};
    if (b < a.batch) c = change_of(a, b);
    const bool up = c.want > c.have;
    const int x[3] = {pages_gone(c), up ? page_count(c.want, a.logP) - page_count(c.have, a.logP) : 0, up ? c.want - c.have : 0};
    long long before[3], all[3];
    sums_before<THREADS>(x, before, all, lds3);
    released = (int)min(a.batch > THREADS ? given : all[0], (long long)a.n_pages);  // more only if two sequences held the same page
    const long long pages_to = asked + before[1] + x[1], tokens_to = fresh + before[2] + x[2];
    const bool ok = up && tokens_to <= a.n_slots && (x[1] == 0 || pages_to <= (long long)count + released);
    const int in[2] = {ok ? x[1] : 0, ok ? x[2] : 0};
    long long in_before[2], in_all[2];
    sums_before<THREADS>(in, in_before, in_all, lds2);
    if (b < a.batch) {
      have[b] = c.have;
      need[b] = (int)min(pages_to - x[1], (long long)0x7fffffff);  // of admitted sequences: whoever asked before them got it
      gone[b] = (int)min(back + before[0], (long long)0x7fffffff);
      starts[b] = total + (int)in_before[1];
      if (ONE) a.starts[b] = starts[b];
      a.lens[b] = ok || c.want < c.have ? c.want : c.have;
    }
    asked += all[1], fresh += all[2], back += all[0], taken += (int)in_all[0], total += (int)in_all[1];
  }
  if (tid == 0) {
    a.starts[a.batch] = total;
    a.free[0] = min(count + released - taken, a.n_pages);
    if (!ONE) a.scratch[0] = count, a.scratch[1] = released, a.scratch[2] = taken, a.scratch[3] = total;
  }
  if constexpr (ONE) {
    __threadfence_block();
    __syncthreads();
    resize_fill(a, Fill{have, a.lens, need, gone, starts, {count, released, taken, total}}, tid, THREADS);
  }
}

// Up to 64 sequences: the sums are one wave's scans, then everybody fills.  Tokens and pages of a sequence are cut to what passes the slots anyway (a new page
// has a new token), so that 32 bits hold the sums.  A decode step of 16 sequences: 6.8 us with the scans of 16 waves above, 1.9 with these.
__global__ __launch_bounds__(256) void resize_wave_kernel(ResizeArgs a) {
  __shared__ int32_t keep[5][kResizeWaveBatch];
  __shared__ ResizeState state;
  if (threadIdx.x < kWave) {
    const int b = threadIdx.x;
    const int count = min(max(a.free[0], 0), a.n_pages);
    Change c{0, 0};
    if (b < a.batch) c = change_of(a, b);
    const int had = page_count(c.have, a.logP), get = page_count(c.want, a.logP);
    const int gone = max(0, had - get), gone_to = scan(gone), released = min(max(last_lane(gone_to), 0), a.n_pages);
    const bool up = c.want > c.have;
    const int tokens = up ? min(c.want - c.have, kResizeOneSlots + 1) : 0, pages = up ? min(get - had, kResizeOneSlots + 1) : 0;
    const int tokens_to = scan(tokens), pages_to = scan(pages);
    const bool ok = up && tokens_to <= a.n_slots && (pages == 0 || pages_to <= count + released);
    const int in = ok ? pages : 0, fresh = ok ? tokens : 0, taken = last_lane(scan(in)), fresh_to = scan(fresh), total = last_lane(fresh_to);
    const int now = ok || c.want < c.have ? c.want : c.have;
    keep[0][b] = c.have, keep[1][b] = now, keep[2][b] = pages_to - pages, keep[3][b] = gone_to - gone, keep[4][b] = fresh_to - fresh;
    if (b < a.batch) a.starts[b] = fresh_to - fresh, a.lens[b] = now;
    if (b == 0) {
      a.starts[a.batch] = total;
      a.free[0] = min(count + released - taken, a.n_pages);
      state = ResizeState{count, released, taken, total};
    }
  }
  __syncthreads();
  resize_fill(a, Fill{keep[0], keep[1], keep[2], keep[3], keep[4], state}, threadIdx.x, 256);
}

// Every slot looks its sequence up, in LDS where the sequences fit (256 sequences, 387346 slots: 5.9 us with eight dependent loads from memory, 5.2 with the starts in LDS,
// 4.8 with what is looked up there beside them).
__global__ __launch_bounds__(256) void resize_fill_kernel(ResizeArgs a) {
  __shared__ int32_t keep[3][kResizeOneBatch];
  const int32_t* s = a.scratch;
  Fill f{s + 4, a.lens, s + 4 + a.batch, s + 4 + 2 * a.batch, a.starts, {s[0], s[1], s[2], s[3]}};
  if (a.batch <= kResizeOneBatch) {
    for (int b = threadIdx.x; b < a.batch; b += 256) keep[0][b] = f.have[b], keep[1][b] = f.need[b], keep[2][b] = f.starts[b];
    f.have = keep[0], f.need = keep[1], f.starts = keep[2];
    __syncthreads();
  }
  resize_fill(a, f, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

// ------------------------------------------------------------------------------------------------ writing
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));

// 8 tokens of one head as a lane stores them.  K: token lane / 8, channels 16 (lane % 8) ..; V: channels 2 lane, 2 lane + 1 of every token.
template <bool BF16, bool V>
struct Octet {
  uint32_t w[BF16 ? 8 : 16];

  __device__ __forceinline__ void load(const void* x, int64_t row0, int64_t row_step, int first, int n) {  // tokens [first, n) of the run; the rest is 0
    const int lane = threadIdx.x % kWave;
    constexpr int kElem = BF16 ? 2 : 4;
#pragma unroll
    for (int i = 0; i < (BF16 ? 8 : 16); ++i) w[i] = 0;
    if constexpr (!V) {
      const int t = first + lane / 8;
      if (t >= 0 && t < n) {
        const uint4* p = (const uint4*)((const char*)x + (row0 + t * row_step + 16 * (lane % 8)) * kElem);
#pragma unroll
        for (int i = 0; i < (BF16 ? 2 : 4); ++i) {
          const uint4 v = p[i];
          w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < kOct; ++j) {
        const int t = first + j;
        if (t < 0 || t >= n) continue;
        const char* p = (const char*)x + (row0 + t * row_step + 2 * lane) * kElem;
        if constexpr (BF16) {
          w[j] = *(const uint32_t*)p;
        } else {
          const uint2 v = *(const uint2*)p;
          w[2 * j] = v.x, w[2 * j + 1] = v.y;
        }
      }
    }
  }
  __device__ __forceinline__ float value(int i) const {  // K: channel i; V: channel i % 2 of token i / 2
    if constexpr (BF16) return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    else return __uint_as_float(w[i]);
  }
  // Magnitudes compare like their bits: largest |x| as a float's bits, NaN and infinities (kInf and more) among them, or without them.
  static constexpr uint32_t kInf = 0x7f800000u;
  __device__ __forceinline__ uint32_t top() const {
    if constexpr (BF16) {
      ushort2v t{0, 0};
#pragma unroll
      for (int i = 0; i < 8; ++i) t = __builtin_elementwise_max(t, __builtin_bit_cast(ushort2v, w[i] & 0x7fff7fffu));
      return (uint32_t)max(t[0], t[1]) << 16;
    } else {
      uint32_t t = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) t = max(t, w[i] & 0x7fffffffu);
      return t;
    }
  }
  __device__ __forceinline__ uint32_t finite_top() const {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t u = __float_as_uint(value(i)) & 0x7fffffffu;
      t = u < kInf && u > t ? u : t;
    }
    return t;
  }
  // in the page's order, times scale = 2^-e, which brings every finite value to 448 at most
  __device__ __forceinline__ void bytes(float scale, bool finite, uint32_t* out) const {
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) f[V ? 8 * (i % 2) + i / 2 : i] = value(i) * scale;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = finite ? floats_e4m3_in_range(f + 4 * i) : floats_e4m3(f + 4 * i);
  }
};

// A run -- new tokens that follow each other in one page -- is one wave's work for each head and tensor: its largest value, the page's exponent, the
// values, and no two waves meet.  Up to kHeld octets stay in registers, all on their way at a time; a longer run (pages of 128) is read twice, the
// second time from the caches.  Bound by memory: 30675 tokens of 8 heads, bf16 (126 MB read, 63 written):
// 78 us with every run read twice, 256 bytes at a time, 50 held in registers, 43 with integer maxima.
// old: the page's exponent, used from its second token on; returns the new one.  Old values are only touched where it grows; of an octet of V that
// holds other tokens too the bytes of those stay.
constexpr int kHeld = 8;
template <bool BF16, bool V>
__device__ int write_run(const Pages& S, int64_t ph, const void* x, int64_t row0, int64_t row_step, int offset, int n, int old) {
  const int lane = threadIdx.x % kWave;
  const int o0 = offset / kOct, octets = (offset + n + kOct - 1) / kOct - o0;
  Octet<BF16, V> held[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
    if (k < octets) held[k].load(x, row0, row_step, (o0 + k) * kOct - offset, n);
  const auto over = [&](auto top_of) {  // the octets, then the lanes
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (k < octets) top = max(top, top_of(held[k]));
    for (int k = kHeld; k < octets; ++k) {
      Octet<BF16, V> more;
      more.load(x, row0, row_step, (o0 + k) * kOct - offset, n);
      top = max(top, top_of(more));
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    return top;
  };
  uint32_t top = over([](const Octet<BF16, V>& y) { return y.top(); });
  const bool finite = __builtin_amdgcn_readfirstlane((int)top) < (int)Octet<BF16, V>::kInf;
  if (!finite) top = over([](const Octet<BF16, V>& y) { return y.finite_top(); });  // NaN and infinities do not set the scale
  int e = e4m3_exponent(__uint_as_float(top)), grown = 0;
  if (offset > 0) {
    grown = max(0, e - old);
    e = max(e, old);
  }
  const float scale = ldexpf(1.f, -e);
  if (lane == 0) S.exponents[2 * ph + (V ? 1 : 0)] = e;
  uint8_t* base = page_values(S, ph) + (V ? (size_t)kHeadDim << S.logP : 0);

  const auto rescaled = [&](uint32_t w) {
    float f[4];
    e4m3_floats(w, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = ldexpf(f[j], -grown);
    return floats_e4m3(f);
  };
  const auto store = [&](const Octet<BF16, V>& oct, int o) {
    uint4* at = (uint4*)(base + o * kOct * kHeadDim) + lane;
    uint32_t now[4];
    oct.bytes(scale, finite, now);
    if constexpr (!V) {
      const int row = o * kOct + lane / 8;
      if (row < offset && grown) {
        const uint4 w = *at;
        now[0] = rescaled(w.x), now[1] = rescaled(w.y), now[2] = rescaled(w.z), now[3] = rescaled(w.w);
      }
      if (row >= offset + n || (row < offset && !grown)) return;
    } else if (o * kOct < offset || (o + 1) * kOct > offset + n) {
      const uint4 was4 = *at;
      const uint32_t was[4] = {was4.x, was4.y, was4.z, was4.w};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t after = 0, before = 0;  // bytes of tokens behind the run and in front of it
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int row = o * kOct + 4 * (w & 1) + j;
          if (row < offset) before |= 0xffu << (8 * j);
          else if (row >= offset + n) after |= 0xffu << (8 * j);
        }
        now[w] = (now[w] & ~(after | before)) | ((grown ? rescaled(was[w]) : was[w]) & before) | (was[w] & after);
      }
    }
    *at = make_uint4(now[0], now[1], now[2], now[3]);
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
    if (k < octets) store(held[k], o0 + k);
  for (int k = kHeld; k < octets; ++k) {
    Octet<BF16, V> more;
    more.load(x, row0, row_step, (o0 + k) * kOct - offset, n);
    store(more, o0 + k);
  }
  if (grown)  // octets of old tokens only
    for (int o = 0; o < o0; ++o) {
      uint4* at = (uint4*)(base + o * kOct * kHeadDim) + lane;
      const uint4 w = *at;
      *at = make_uint4(rescaled(w.x), rescaled(w.y), rescaled(w.z), rescaled(w.w));
    }
  return e;
}

// The nearest row with a slot, from `row` on in steps of DIR (1 or -1); outside [0, n): none.  512 rows a turn, for rows that pad a batch.
template <int DIR>
__device__ __forceinline__ int row_with_slot(const int32_t* slots, int row, int n, int top) {
  const int lane = threadIdx.x % kWave;
  for (; row >= 0 && row < n; row += DIR * 8 * kWave) {
    unsigned long long m[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t r = row + (int64_t)DIR * (j * kWave + lane);
      const int s = r >= 0 && r < n ? slots[r] : -1;
      m[j] = __ballot(s >= 0 && s < top);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (m[j]) return row + DIR * (j * kWave + __builtin_ctzll(m[j]));
    if (DIR > 0 && row > n - 8 * kWave) break;
  }
  return -1;
}

// One wave per (segment of the slots, layer, head, tensor): the runs that begin in its segment.  Rows without a slot inside a page's new tokens do not
// end the wave's work: what follows is a second run of the same page, after the first.
template <bool BF16>
__global__ __launch_bounds__(256) void pages_write_kernel(Pages S, int layer0, int n_layers, const void* k, const void* v, const int32_t* slots, int n_tokens,
                                                          int segment, int64_t units) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  if (unit >= units) return;
  const int lane = threadIdx.x % kWave, P = 1 << S.logP;
  const int which = (int)(unit & 1), h = (int)((unit >> 1) % S.H);
  const int64_t rest = (unit >> 1) / S.H;
  const int layer = (int)(rest % n_layers);
  const int t0 = (int)(rest / n_layers) * segment, top = S.n_pages << S.logP;
  const int t = t0 + lane;
  int slot = -1, prev = -2;
  if (lane < segment && t < n_tokens) {
    slot = slots[t];
    if (t > 0) prev = slots[t - 1];
  }
  const bool in = slot >= 0 && slot < top;
  const bool follows = in && (slot & (P - 1)) != 0 && prev + 1 == slot;
  unsigned long long leads = __ballot(in && !follows);
  unsigned long long unsure = __ballot(in && (slot & (P - 1)) != 0 && t > 0 && (prev < 0 || prev >= top));
  while (unsure) {  // behind rows without a slot
    const int at = __builtin_ctzll(unsure), r = row_with_slot<-1>(slots, t0 + at - 1, n_tokens, top);
    if (r >= 0 && slots[r] + 1 == __builtin_amdgcn_readlane(slot, at)) leads &= ~(1ull << at);
    unsure &= unsure - 1;
  }
  while (leads) {
    const int first = __builtin_ctzll(leads);
    leads &= leads - 1;
    int start = __builtin_amdgcn_readlane(slot, first), t1 = t0 + first, e = 0;
    const int64_t ph = page_head(S, layer0 + layer, start >> S.logP, h);
    const int64_t row_step = (int64_t)S.H * kHeadDim;
    if (start & (P - 1)) e = S.exponents[2 * ph + which];
    for (;;) {
      const int offset = start & (P - 1), most = min(P - offset, n_tokens - t1);
      int n = 0;  // length of the run: up to 128
      for (int c = 0; c < most; c += kWave) {
        const int i = c + lane;
        const bool same = i < most && slots[t1 + i] == start + i;
        const unsigned long long m = ~__ballot(same);
        const int got = m ? __builtin_ctzll(m) : kWave;
        n += got;
        if (got < kWave) break;
      }
      const int64_t row0 = ((int64_t)layer * n_tokens + t1) * row_step + h * kHeadDim;
      if (which) e = write_run<BF16, true>(S, ph, v, row0, row_step, offset, n, e);
      else e = write_run<BF16, false>(S, ph, k, row0, row_step, offset, n, e);
      if (offset + n == P || t1 + n >= n_tokens) break;
      const int after = slots[t1 + n];
      if (after >= 0 && after < top) break;
      t1 = row_with_slot<1>(slots, t1 + n, n_tokens, top);
      if (t1 < 0 || slots[t1] != start + n) break;
      start += n;
    }
  }
}

// ------------------------------------------------------------------------------------------------ reading
template <bool BF16>
__device__ __forceinline__ void store2(void* p, int64_t i, float x, float y) {
  if constexpr (BF16) *(uint32_t*)((uint16_t*)p + i) = (uint32_t)f32_to_bf16(x) | (uint32_t)f32_to_bf16(y) << 16;
  else *(float2*)((float*)p + i) = make_float2(x, y);
}

// One wave per octet of tokens of a sequence and head, K and V.  Bound by what it writes.
template <bool BF16>
__global__ __launch_bounds__(256) void pages_read_kernel(Pages S, int layer0, int batch, int n, const int32_t* table, const int32_t* lens, void* K, void* V,
                                                         int64_t units) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
  if (unit >= units) return;
  const int lane = threadIdx.x % kWave, octets = (n + kOct - 1) / kOct;
  const int o = (int)(unit % octets);
  int64_t rest = unit / octets;
  const int h = (int)(rest % S.H);
  rest /= S.H;
  const int b = (int)(rest % batch), layer = (int)(rest / batch);
  const int len = min(max(lens[b], 0), S.max_pages << S.logP);
  const int t0 = o * kOct;
  uint4 k = make_uint4(0, 0, 0, 0), v = k;
  int ek = 0, ev = 0, there = min(len - t0, kOct);  // tokens of the octet
  if (there > 0) {
    const int page = table[(int64_t)b * S.max_pages + (t0 >> S.logP)];
    if (page < 0 || page >= S.n_pages) {
      there = 0;
    } else {
      const int64_t ph = page_head(S, layer0 + layer, page, h);
      const uint8_t* at = page_values(S, ph) + (t0 & ((1 << S.logP) - 1)) * kHeadDim;
      k = ((const uint4*)at)[lane], v = ((const uint4*)(at + ((size_t)kHeadDim << S.logP)))[lane];
      ek = S.exponents[2 * ph], ev = S.exponents[2 * ph + 1];
    }
  }
  const int64_t row = ((((int64_t)layer * batch + b) * S.H + h) * n + t0) * kHeadDim;
  float f[16];
  e4m3_floats(k.x, f), e4m3_floats(k.y, f + 4), e4m3_floats(k.z, f + 8), e4m3_floats(k.w, f + 12);
  const int mine = lane / 8;
  if (K && t0 + mine < n) {
#pragma unroll
    for (int c = 0; c < 16; ++c) f[c] = mine < there ? ldexpf(f[c], ek) : 0.f;
    const int64_t to = row + mine * kHeadDim + 16 * (lane % 8);
    if constexpr (BF16) {
      uint32_t w[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) w[c] = (uint32_t)f32_to_bf16(f[2 * c]) | (uint32_t)f32_to_bf16(f[2 * c + 1]) << 16;
      uint4* p = (uint4*)((uint16_t*)K + to);
      p[0] = make_uint4(w[0], w[1], w[2], w[3]), p[1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
#pragma unroll
      for (int c = 0; c < 16; c += 4) *(float4*)((float*)K + to + c) = make_float4(f[c], f[c + 1], f[c + 2], f[c + 3]);
    }
  }
  if (V) {
    e4m3_floats(v.x, f), e4m3_floats(v.y, f + 4), e4m3_floats(v.z, f + 8), e4m3_floats(v.w, f + 12);
#pragma unroll
    for (int j = 0; j < kOct; ++j)
      if (t0 + j < n) store2<BF16>(V, row + j * kHeadDim + 2 * lane, j < there ? ldexpf(f[j], ev) : 0.f, j < there ? ldexpf(f[8 + j], ev) : 0.f);
  }
}

}  // namespace

hipError_t launch_pages_resize(const ResizeArgs& a, hipStream_t st) {
  if (!a.scratch && a.batch <= kResizeWaveBatch) {
    resize_wave_kernel<<<1, 256, 0, st>>>(a);
    return hipGetLastError();
  }
  const bool small = a.batch <= kResizeSmallThreads;
  if (!a.scratch) {
    if (small) resize_kernel<true, kResizeSmallThreads><<<1, kResizeSmallThreads, 0, st>>>(a);
    else resize_kernel<true, kResizeThreads><<<1, kResizeThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  if (small) resize_kernel<false, kResizeSmallThreads><<<1, kResizeSmallThreads, 0, st>>>(a);
  else resize_kernel<false, kResizeThreads><<<1, kResizeThreads, 0, st>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t items = std::max<int64_t>(a.n_slots, (int64_t)a.batch * 16);
  resize_fill_kernel<<<(unsigned)std::min<int64_t>(1024, (items + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError();
}

namespace {
// as many waves as fill the chip, each with up to a page of tokens, which is one run of a prompt
int write_segment(const Pages& S, int n_layers, int n_tokens) {
  return (int)std::max<int64_t>(1, std::min<int64_t>({kWave, (int64_t)1 << S.logP, n_tokens * ((int64_t)n_layers * S.H * 2) / 8192}));
}
}  // namespace
int64_t pages_write_units(const Pages& S, int n_layers, int n_tokens) {
  const int segment = write_segment(S, n_layers, n_tokens);
  return ((int64_t)n_tokens + segment - 1) / segment * n_layers * S.H * 2;
}
int64_t pages_read_units(const Pages& S, int n_layers, int batch, int n) { return ((int64_t)n + kOct - 1) / kOct * S.H * batch * n_layers; }

hipError_t launch_pages_write(const Pages& S, int layer, int n_layers, bool bf16, const void* k, const void* v, const int32_t* slots, int n_tokens,
                              hipStream_t st) {
  const int segment = write_segment(S, n_layers, n_tokens);
  const int64_t units = pages_write_units(S, n_layers, n_tokens);
  const unsigned grid = (unsigned)((units + 3) / 4);
  if (bf16) pages_write_kernel<true><<<grid, 256, 0, st>>>(S, layer, n_layers, k, v, slots, n_tokens, segment, units);
  else pages_write_kernel<false><<<grid, 256, 0, st>>>(S, layer, n_layers, k, v, slots, n_tokens, segment, units);
  return hipGetLastError();
}

hipError_t launch_pages_read(const Pages& S, int layer, int n_layers, bool bf16, const int32_t* table, const int32_t* lens, int batch, int n, void* K, void* V,
                             hipStream_t st) {
  const int64_t units = pages_read_units(S, n_layers, batch, n);
  const unsigned grid = (unsigned)((units + 3) / 4);
  if (bf16) pages_read_kernel<true><<<grid, 256, 0, st>>>(S, layer, batch, n, table, lens, K, V, units);
  else pages_read_kernel<false><<<grid, 256, 0, st>>>(S, layer, batch, n, table, lens, K, V, units);
  return hipGetLastError();
}

}  // namespace iwdft
