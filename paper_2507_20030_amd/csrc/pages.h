// The 8-bit paged cache: layout and conversions shared by its kernels (pages.hip, pages_attn.hip, pages_tables.hip, pages_shared.hip).
//
// Exact tokens of requests that are not (yet) in the frequency domain, P to a page, as OCP e4m3 with one power-of-two scale for each page,
// KV head and tensor.  A power of two loses nothing: x 2^-e is exact, so a stored value is off by one rounding to four significant bits
// (at most 2^-4 of its size, 2^-10 2^e near zero), and a page whose exponent grows keeps its values except where they leave the
// normal range of e4m3.  Layout of one page's head, 256 P bytes:
//     K [token][channel]                as a row goes into the matrix instruction: 16 bytes are 16 channels of a token
//     V [token / 8][channel][token % 8] 8 bytes are the 8 tokens of one operand register pair, so that p V needs no transposition
#pragma once
#include "common.h"

namespace iwdft {

constexpr int kOct = 8;                  // tokens of V that sit side by side
constexpr int kLeastExponent = -100;     // values below 2^-110 count as 0
constexpr int kE4m3Max = 448;

struct Pages {
  int32_t n_pages, H, G, logP, max_pages;
  uint8_t* values;     // [layer][page][head][K, V][P * 128]
  int32_t* exponents;  // [layer][page][head][K, V]
};

__device__ __forceinline__ int64_t page_head(const Pages& S, int layer, int page, int h) {
  return ((int64_t)layer * S.n_pages + page) * S.H + h;
}
__device__ __forceinline__ uint8_t* page_values(const Pages& S, int64_t ph) { return S.values + (ph << (S.logP + 8)); }
__device__ __forceinline__ int page_count(int n, int logP) { return (n + (1 << logP) - 1) >> logP; }

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

// Four bytes of e4m3 (one register) as floats.
__device__ __forceinline__ void e4m3_floats(uint32_t w, float* f) {
  const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  f[0] = lo[0], f[1] = lo[1], f[2] = hi[0], f[3] = hi[1];
}
// Nearest e4m3 of four floats, ties to even; beyond 448 (infinities) 448, NaN stays NaN.
__device__ __forceinline__ float e4m3_range(float x) { return x != x ? x : fminf(fmaxf(x, -(float)kE4m3Max), (float)kE4m3Max); }
__device__ __forceinline__ uint32_t floats_e4m3_in_range(const float* f) {  // |f| <= 448
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
}
__device__ __forceinline__ uint32_t floats_e4m3(const float* f) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(f[0]), e4m3_range(f[1]), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(f[2]), e4m3_range(f[3]), w, true);
}

// Smallest e >= kLeastExponent with a <= 448 * 2^e = 1.75 * 2^(e + 8); a finite, >= 0.
__device__ __forceinline__ int e4m3_exponent(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < kLeastExponent ? kLeastExponent : e;  // below 2^-126 as well
}

// Inclusive sums over the lanes of a wave, within rows of 16 and then across them.
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_lane(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int scan(int x) {
  x += from_lane<0x111, 0xf>(x), x += from_lane<0x112, 0xf>(x), x += from_lane<0x114, 0xf>(x), x += from_lane<0x118, 0xf>(x);
  x += from_lane<0x142, 0xa>(x);
  return x + from_lane<0x143, 0xc>(x);
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

constexpr int kLanes = 64;
// Sums of N numbers >= 0 over the threads before this one and over all threads of the workgroup; every thread calls it.  In two halves of 16 bits, whose sums over
// a wave fit 32.
template <int THREADS, int N>
__device__ __forceinline__ void sums_before(const int (&x)[N], long long (&before)[N], long long (&all)[N], long long (*lds)[N]) {
  const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int lo = scan(x[i] & 0xffff), hi = scan((int)((uint32_t)x[i] >> 16));
    before[i] = ((long long)hi << 16) + lo;
  }
  __syncthreads();  // the last call's sums have been read
  if (lane == kLanes - 1)
#pragma unroll
    for (int i = 0; i < N; ++i) lds[wave][i] = before[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    long long sum = 0, mine = 0;
#pragma unroll 4
    for (int w = 0; w < THREADS / kLanes; ++w) {
      mine = w == wave ? sum : mine;
      sum += lds[w][i];
    }
    before[i] += mine - x[i], all[i] = sum;
  }
}

struct ResizeArgs {
  const int32_t* want;
  int32_t batch, logP, max_pages, n_pages, n_slots;
  int32_t *table, *lens, *free, *starts, *slots;
  int32_t* scratch;  // 4 + 3 * batch ints, or null where one workgroup does it all
};
constexpr int kResizeThreads = 1024, kResizeSmallThreads = 256;  // up to so many sequences: fewer waves, whose sums are joined sooner
// One launch, without scratch, up to so many sequences and slots; one wave's scans up to kResizeWaveBatch sequences.
constexpr int kResizeOneBatch = 1024, kResizeOneSlots = 2048, kResizeWaveBatch = 64;
hipError_t launch_pages_resize(const ResizeArgs& a, hipStream_t st);

// Pages that sequences share (pages_tables.hip).
constexpr int kSharedBatch = 1024;  // sequences: a thread for each
struct SharedTables {
  int32_t batch, logP, max_pages, n_pages;
  int32_t *table, *lens, *free, *refs;
};
struct GrowArgs {
  SharedTables t;
  const int32_t* want;
  int32_t n_slots;
  int32_t *starts, *slots, *copies;
};
struct ForkArgs {
  SharedTables t;
  const int32_t *parent, *keep;
  int32_t* scratch;  // null: one launch
};
struct CompactArgs {
  SharedTables t;
  int32_t *moves, n_moves;
  int32_t* scratch;
};
size_t pages_fork_bytes(int batch, int max_pages);
size_t pages_compact_bytes(int n_pages);
hipError_t launch_pages_grow(const GrowArgs& a, hipStream_t st);
hipError_t launch_pages_fork(const ForkArgs& a, hipStream_t st);
hipError_t launch_pages_compact(const CompactArgs& a, hipStream_t st);
hipError_t launch_pages_copy(const Pages& from, const Pages& to, int layer, int n_layers, const int32_t* copies, int n, hipStream_t st);

constexpr int64_t kMostUnits = ((int64_t)1 << 26) - 4;  // waves of a launch: 2^32 threads are too many
int64_t pages_write_units(const Pages& S, int n_layers, int n_tokens);
int64_t pages_read_units(const Pages& S, int n_layers, int batch, int n);
hipError_t launch_pages_write(const Pages& S, int layer, int n_layers, bool bf16, const void* k, const void* v, const int32_t* slots, int n_tokens,
                              hipStream_t st);
hipError_t launch_pages_read(const Pages& S, int layer, int n_layers, bool bf16, const int32_t* table, const int32_t* lens, int batch, int n, void* K,
                             void* V, hipStream_t st);

// The sequences of one kind of blocks.
struct PagesRows {
  int32_t over, to;          // rows (new tokens times query heads of a KV head): more than `over`, up to `to`
  uint32_t grid, join_grid;  // workgroups
  float* part;   // [slot][rows of a block][128]: sums of a part of the tokens
  float2* stat;  // [slot][rows of a block]: (reference of the exponents, sum of weights)
};
struct PagesAttn {
  Pages S;
  int32_t layer, n_layers, batch, n_tokens, n_sink, n_recent;
  float scale;  // of the scores, times log2 e
  const void* q;
  void* out;
  const int32_t *starts, *table, *lens;
  PagesRows few, many;
};
size_t pages_attn_bytes(const Pages& S, int batch, int n_tokens, bool bf16);       // of a call of these sizes
size_t pages_attn_most_bytes(const Pages& S, int batch, int n_tokens, bool bf16);  // of any call of up to these sizes
hipError_t launch_pages_attn(PagesAttn a, bool bf16, void* ws, hipStream_t st);

// Attention over pages that sequences share (pages_shared.hip); of the arguments the plan takes all but the pool, q and out.
size_t pages_plan_bytes(const Pages& S, int n_layers, int batch, int n_tokens);
size_t pages_shared_bytes(const Pages& S, int n_layers, int batch, int n_tokens);
hipError_t launch_pages_plan(const PagesAttn& a, bool bf16, void* plan, hipStream_t st);
hipError_t launch_pages_shared(const PagesAttn& a, bool bf16, const void* plan, void* ws, hipStream_t st);

}  // namespace iwdft
