// The paged cache of a pruned context: rotation of new queries and keys by their positions with the
// append of keys and values (bf16 pages, or e4m3 codes with a power-of-two scale for each page and
// head), and the attention of new tokens over the cached ones.
#include <math.h>

#include <new>
#include <type_traits>
#include <vector>

#include "pace_internal.h"

namespace pace {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8]) {
  x[0] = bf16_lo(u.x); x[1] = bf16_hi(u.x); x[2] = bf16_lo(u.y); x[3] = bf16_hi(u.y);
  x[4] = bf16_lo(u.z); x[5] = bf16_hi(u.z); x[6] = bf16_lo(u.w); x[7] = bf16_hi(u.w);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                    pack_bf16x2(x[6], x[7]));
}

// ---------------------------------------------------------------- append
// The cache as the kernels see it.
struct Pool {
  void *k, *v;
  float *k_scale, *v_scale;
  const int32_t* table;      // [B, max_pages]
  int num_pages, max_pages, heads, page, shift;
};

struct AppendParams {
  const uint16_t *q, *k, *v;
  long long qs, ks, vs;      // elements between rows
  const int32_t *rows, *cu, *ctx, *pos;
  const float* freq;
  uint16_t* q_out;
  Pool pool;
  int n_src, n_new, max_new, B, Hq;
  int end0, end1;            // frequencies [0, end0) turn by axis 0, [end0, end1) by axis 1, the rest by axis 2
  int tokens, tiles;         // append_rows: tokens per workgroup, workgroups per sequence
  int pages;                 // append_pages: pages a sequence may write
};

// cos and sin of positions[axis(f)][src] * freq[f].  The product is formed in 64 bits and reduced to a
// fraction of a turn there (a position of 2^20 leaves an error under 1e-10 turns), so the single-precision
// functions see at most half a turn.
__device__ __forceinline__ f32x2 turn(const AppendParams& p, int src, int f) {
  if (p.pos == nullptr) return f32x2{1.f, 0.f};
  const int axis = (f >= p.end0) + (f >= p.end1);
  double t = static_cast<double>(p.pos[static_cast<long long>(axis) * p.n_src + src]) *
             static_cast<double>(p.freq[f]) * 0.15915494309189535;
  t -= rint(t);
  f32x2 r;
  float s, c;
  sincospif(2.f * static_cast<float>(t), &s, &c);
  r.x = c;
  r.y = s;
  return r;
}

__device__ __forceinline__ void rotate8(float (&a)[8], float (&b)[8], const f32x2* cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = a[i], y = b[i], c = cs[i].x, s = cs[i].y;
    a[i] = x * c - y * s;
    b[i] = y * c + x * s;
  }
}

// The rows of sequence b's new tokens: its first row and how many there are.
__device__ __forceinline__ int new_tokens(const AppendParams& p, int b, int* first) {
  const int r0 = p.cu[b];
  int n = p.cu[b + 1] - r0;
  n = n > p.max_new ? p.max_new : n;
  *first = r0;
  if (r0 < 0) return 0;
  return n > p.n_new - r0 ? p.n_new - r0 : n;
}

constexpr int kAppendThreads = 256;
constexpr int kAppendTokens = 8;   // most tokens per workgroup

// Queries, and keys and values of bf16 pages.  A workgroup takes some tokens of one sequence: their
// angles' cos and sin go to LDS once (all heads share them), then every thread moves 16 values of one
// head (8 of each half, so that a pair meets in one thread) per step.  Short calls are one chain of loads (offsets,
// source row, position, table entry, values) behind a launch: one token 3.3 us.
template <int D, bool KV>
__device__ __forceinline__ void append_rows(const AppendParams& p, int block) {
  constexpr int HALF = D / 2, CH = D / 16;
  __shared__ f32x2 cs[kAppendTokens * HALF];
  __shared__ int src_of[kAppendTokens];
  const int b = block / p.tiles, t0 = (block % p.tiles) * p.tokens;
  int r0;
  const int n = new_tokens(p, b, &r0);
  const int here = n - t0 < p.tokens ? n - t0 : p.tokens;
  if (here <= 0) return;
  if (threadIdx.x < here) {
    const int r = r0 + t0 + threadIdx.x;
    const int s = p.rows ? p.rows[r] : r;
    src_of[threadIdx.x] = s >= 0 && s < p.n_src ? s : -1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < here * HALF; i += kAppendThreads) {
    const int s = src_of[i / HALF];
    if (s >= 0) cs[i] = turn(p, s, i % HALF);
  }
  __syncthreads();
  const int hq = p.q ? p.Hq : 0, heads = hq + (KV ? 2 * p.pool.heads : 0);
  for (int i = threadIdx.x; i < here * heads * CH; i += kAppendThreads) {
    const int c = i % CH, h = i / CH % heads, t = i / (CH * heads);
    const int src = src_of[t];
    if (src < 0) continue;
    const uint16_t* from;
    uint16_t* to;
    if (h < hq) {
      from = p.q + src * p.qs + h * D;
      to = p.q_out + (static_cast<long long>(r0 + t0 + t) * p.Hq + h) * D;
    } else {
      const bool val = h - hq >= p.pool.heads;
      const int hk = val ? h - hq - p.pool.heads : h - hq;
      const long long place = static_cast<long long>(p.ctx[b]) + t0 + t;
      const long long pi = place >> p.pool.shift;
      if (place < 0 || pi >= p.pool.max_pages) continue;
      const int pg = p.pool.table[static_cast<long long>(b) * p.pool.max_pages + pi];
      if (pg < 0 || pg >= p.pool.num_pages) continue;
      from = val ? p.v + src * p.vs + hk * D : p.k + src * p.ks + hk * D;
      to = static_cast<uint16_t*>(val ? p.pool.v : p.pool.k) +
           ((static_cast<long long>(pg) * p.pool.heads + hk) * p.pool.page + (place & (p.pool.page - 1))) * D;
    }
    uint4 lo = *reinterpret_cast<const uint4*>(from + 8 * c);
    uint4 hi = *reinterpret_cast<const uint4*>(from + HALF + 8 * c);
    if (p.pos != nullptr && h < hq + p.pool.heads) {
      float a[8], d[8];
      unpack8(lo, a);
      unpack8(hi, d);
      rotate8(a, d, &cs[t * HALF + 8 * c]);
      lo = pack8(a);
      hi = pack8(d);
    }
    *reinterpret_cast<uint4*>(to + 8 * c) = lo;
    *reinterpret_cast<uint4*>(to + HALF + 8 * c) = hi;
  }
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }

// Four floats to e4m3, nearest even; infinities become NaN (what the conversion makes of them otherwise depends on a
// mode bit).  Magnitudes are at most 448.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  const float nan = __uint_as_float(0x7fc00000u);
  a = finite(a) ? a : nan;
  b = finite(b) ? b : nan;
  c = finite(c) ? c : nan;
  d = finite(d) ? d : nan;
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return static_cast<uint32_t>(r);
}
__device__ __forceinline__ void from_e4m3(uint32_t u, float (&x)[4]) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), false);
  const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(u), true);
  x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}

// The least power of two s >= 2^-120 with top <= 448 s.  448 = 1.75 * 2^8.
__device__ __forceinline__ float page_scale(float top) {
  const uint32_t u = __float_as_uint(top);
  int e = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  e = e < -120 ? -120 : e;
  return __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}

// Keys or values of 8-bit pages: one workgroup owns one (sequence, page, head) of k or v, so the page's
// scale needs no atomics and one launch is enough.  The new values stay in registers between the
// maximum and the store.  With the queries' rows beside it bound by memory: 10,677 tokens, 28/4 heads of 128, move 186 MB
// in 43.5 us (4.3 TB/s; a copy of them takes 33.8); one token of each of 64 sequences takes 5.4 us.
template <int D, int ITEMS>
__device__ __forceinline__ void append_pages(const AppendParams& p, int block) {
  constexpr int HALF = D / 2, CH = D / 16;
  __shared__ float red[kAppendThreads / 64];
  int id = block;
  const bool val = id & 1;
  id >>= 1;
  const int h = id % p.pool.heads;
  id /= p.pool.heads;
  const int b = id / p.pages, j = id % p.pages;
  int r0;
  const int n = new_tokens(p, b, &r0), ctx = p.ctx[b], P = p.pool.page;
  if (ctx < 0) return;
  const long long pi = (ctx >> p.pool.shift) + j, start = pi << p.pool.shift;
  const long long lo = ctx > start ? ctx : start;
  const long long end = static_cast<long long>(ctx) + n < start + P ? static_cast<long long>(ctx) + n : start + P;
  if (lo >= end || pi >= p.pool.max_pages) return;
  const int pg = p.pool.table[static_cast<long long>(b) * p.pool.max_pages + pi];
  if (pg < 0 || pg >= p.pool.num_pages) return;
  const int held = static_cast<int>(lo - start), count = static_cast<int>(end - lo);
  const int row0 = r0 + static_cast<int>(lo - ctx);
  const long long ph = static_cast<long long>(pg) * p.pool.heads + h;
  uint8_t* codes = static_cast<uint8_t*>(val ? p.pool.v : p.pool.k) + ph * P * D;
  float* scale = (val ? p.pool.v_scale : p.pool.k_scale) + ph;

  float x[ITEMS][2][8];
  bool there[ITEMS];
  float top = 0.f;
#pragma unroll
  for (int it = 0; it < ITEMS; ++it) {
    const int i = it * kAppendThreads + threadIdx.x, t = i / CH, c = i % CH;
    there[it] = false;
    if (t < count) {
      const int src = p.rows ? p.rows[row0 + t] : row0 + t;
      if (src >= 0 && src < p.n_src) {
        there[it] = true;
        const uint16_t* from = (val ? p.v + src * p.vs : p.k + src * p.ks) + h * D + 8 * c;
        unpack8(*reinterpret_cast<const uint4*>(from), x[it][0]);
        unpack8(*reinterpret_cast<const uint4*>(from + HALF), x[it][1]);
        if (!val && p.pos != nullptr) {
          f32x2 cs[8];
#pragma unroll
          for (int f = 0; f < 8; ++f) cs[f] = turn(p, src, 8 * c + f);
          rotate8(x[it][0], x[it][1], cs);
        }
#pragma unroll
        for (int f = 0; f < 8; ++f) {
          const float a = fabsf(x[it][0][f]), d = fabsf(x[it][1][f]);
          top = fmaxf(top, finite(a) ? a : 0.f);
          top = fmaxf(top, finite(d) ? d : 0.f);
        }
      }
    }
  }
  const float old = held ? *scale : 0.f;
  top = block_reduce<1>(top, red);
  const float s = fmaxf(old, page_scale(top));
  __syncthreads();                                  // every thread has read the old scale
  if (threadIdx.x == 0) *scale = s;
  if (held && s != old) {
    const float f = old / s;
    for (int i = threadIdx.x; i < held * (D / 16); i += kAppendThreads) {
      uint4 u = *reinterpret_cast<const uint4*>(codes + 16 * i);
      uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float y[4];
        from_e4m3(w[e], y);
        w[e] = to_e4m3(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
      }
      *reinterpret_cast<uint4*>(codes + 16 * i) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  // a power of two: the product with its reciprocal is the quotient
  const bool pow2 = (__float_as_uint(s) & 0x7fffffu) == 0u;
  const float inv = 1.f / s;
#pragma unroll
  for (int it = 0; it < ITEMS; ++it) {
    if (!there[it]) continue;
    const int i = it * kAppendThreads + threadIdx.x, t = i / CH, c = i % CH;
    uint8_t* to = codes + (held + t) * D + 8 * c;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float y[8];
#pragma unroll
      for (int f = 0; f < 8; ++f) y[f] = pow2 ? x[it][half][f] * inv : x[it][half][f] / s;
      *reinterpret_cast<uint2*>(to + half * HALF) =
          make_uint2(to_e4m3(y[0], y[1], y[2], y[3]), to_e4m3(y[4], y[5], y[6], y[7]));
    }
  }
}

template <int D>
__global__ __launch_bounds__(kAppendThreads) void append_16bit(const AppendParams p) {
  append_rows<D, true>(p, blockIdx.x);
}
// The pages first: they compute, and the queries' rows, which only move bytes, fill the memory's time beside them
// (10,677 tokens, 28/4 heads of 128: 45 us, one launch after the other 50; evenly mixed 43.7, but 64 tokens of 64
// sequences 6.1 instead of 5.4).
template <int D, int ITEMS>
__global__ __launch_bounds__(kAppendThreads) void append_8bit(const AppendParams p, int page_blocks) {
  const int block = blockIdx.x;
  if (block < page_blocks) append_pages<D, ITEMS>(p, block);
  else append_rows<D, false>(p, block - page_blocks);
}

template <int D>
pace_status_t launch_append(const AppendParams& p, int bits, long long row_blocks, long long page_blocks,
                            hipStream_t stream) {
  const dim3 th(kAppendThreads);
  if (bits == 16) {
    hipLaunchKernelGGL((append_16bit<D>), dim3(static_cast<unsigned>(row_blocks)), th, 0, stream, p);
  } else {
    const dim3 g(static_cast<unsigned>(page_blocks + (p.q ? row_blocks : 0)));
    const int items = (p.pool.page * (D / 16) + kAppendThreads - 1) / kAppendThreads, n = static_cast<int>(page_blocks);
    if (items <= 1) hipLaunchKernelGGL((append_8bit<D, 1>), g, th, 0, stream, p, n);
    else if (items <= 2) hipLaunchKernelGGL((append_8bit<D, 2>), g, th, 0, stream, p, n);
    else if (items <= 4) hipLaunchKernelGGL((append_8bit<D, 4>), g, th, 0, stream, p, n);
    else hipLaunchKernelGGL((append_8bit<D, 8>), g, th, 0, stream, p, n);
  }
  return check_launch("pace_cache_append");
}

// ---------------------------------------------------------------- attention
// Rows of one KV head: row x of sequence b is its query x / group, query head hk * group + x % group.
// Scores are kept in the log2 domain.  The keys that the rows of a workgroup may see are visited in
// tiles of 32, aligned to 32: first those of the sinks, then those of the window.
struct AttendParams {
  const uint16_t* q;
  const int32_t *cu, *len;
  uint16_t* o;
  float* lse;
  float* part;               // partial results [splits, n_q * Hq, D + 4]: D values, maximum, sum
  Pool pool;
  int n_q, Hq, group, B, max_q, max_len, window, sinks;
  int row_blocks, splits;    // row blocks of a KV head, most parts of its keys
  int want, size;            // parts that the longest should make; tiles of a part, 0: as many as that takes
  float scale_log2;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Keys per step of a wave: 16 KiB of K and V at d = 128 either way.
constexpr int tile_keys(int bits) { return bits == 16 ? 32 : 64; }

__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// Maximum of three in one instruction (fmaxf would first canonicalise values fresh from a matrix product).  A NaN wins: its
// row is NaN whatever its maximum is, and no comparison with it raises one.
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// Cached keys and values are read once: loads that do not ask the caches to keep them (attention over 131,071
// tokens 52 us against 58, 48 sequences in 8 bits 104 against 111; short ragged batches lose a little, 8 sequences of 20
// rows take 47 us instead of 45).
__device__ __forceinline__ u32x4 stream16(const void* p) { return __builtin_nontemporal_load(static_cast<const u32x4*>(p)); }
__device__ __forceinline__ u32x2 stream8(const void* p) { return __builtin_nontemporal_load(static_cast<const u32x2*>(p)); }

// Two e4m3 codes (the low or high pair of a dword) as two bf16 values: exact.
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_bf16(uint32_t u) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HI));
}
__device__ __forceinline__ uint4 e4m3_bf16x8(uint32_t a, uint32_t b) {
  return make_uint4(e4m3_bf16<false>(a), e4m3_bf16<true>(a), e4m3_bf16<false>(b), e4m3_bf16<true>(b));
}

// The sign bits of the values of a dword (two bf16, four e4m3) that are infinite or NaN.
template <int BITS>
__device__ __forceinline__ uint32_t not_finite(uint32_t u) {
  // all exponent bits set (e4m3: all bits but the sign): one more carries into the sign's place and no further
  return BITS == 16 ? ((u & 0x7f807f80u) + 0x00800080u) & 0x80008000u : ((u & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}

// What a sequence's queries are and the tiles that queries i_lo..i_hi of it see.
struct Span {
  int row0, nq, len;         // first row of q, queries, cached tokens
  int p_lo, p_hi;            // places of the first and last query
  int head_tiles, tail0, tiles;   // tiles [0, head_tiles) and [tail0, ...), tiles in all
  __device__ __forceinline__ int tile(int x) const { return x < head_tiles ? x : tail0 + x - head_tiles; }
};
__device__ __forceinline__ Span queries_of(const AttendParams& p, int b) {
  Span s;
  s.row0 = p.cu[b];
  s.nq = p.cu[b + 1] - s.row0;
  s.nq = s.nq > p.max_q ? p.max_q : s.nq;
  if (s.row0 < 0 || s.nq < 0) s.nq = 0;
  if (s.nq > p.n_q - s.row0) s.nq = p.n_q - s.row0;
  s.len = p.len[b];
  s.len = s.len > p.max_len ? p.max_len : s.len < 0 ? 0 : s.len;
  return s;
}
template <int T>
__device__ __forceinline__ void tiles_of(const AttendParams& p, int i_lo, int i_hi, Span* s) {
  s->p_lo = s->len - s->nq + i_lo;
  s->p_hi = s->len - s->nq + i_hi;
  const int end = s->p_hi < 0 ? 0 : s->p_hi / T + 1;
  s->tail0 = p.window == 0 || s->p_lo < p.window ? 0 : (s->p_lo - p.window + 1) / T;   // p_lo may be as low as -nq
  const int sinks = p.sinks < s->p_hi + 1 ? p.sinks : s->p_hi + 1;
  s->head_tiles = sinks <= 0 ? 0 : (sinks + T - 1) / T;
  if (s->tail0 <= s->head_tiles) { s->tail0 = 0; s->head_tiles = 0; }
  s->tiles = end - s->tail0 + s->head_tiles;
}
// Tiles of T keys that a row block may see at most in a sequence of up to `len` tokens: sinks and window each begin inside one.
__host__ __device__ __forceinline__ int most_tiles(int len, int T, int window, int sinks, int max_q) {
  const long long seen = static_cast<long long>(window) + sinks + max_q;
  const int keys = window > 0 && seen < len ? static_cast<int>(seen) : len;    // len <= 2^31 - 1,024
  return (keys + T - 1) / T + (window > 0 ? 2 : 0);
}
// Tiles of a part, where the longest sequence's should make `want`.  A part of fewer than four tiles costs more to join than
// it saves (64 tokens x 7 heads over 1,183: 18.5 us, parts of two tiles 23.9; one token over 5,000: 11.2 us, parts of one
// 12.1); more leave CUs idle (32 tokens over 1,183: 17.5 us, parts of eight 20.4).
constexpr int kLeastTiles = 4;
__device__ __forceinline__ int part_tiles(int tiles, int want) {
  const int part = (tiles + want - 1) / want;
  return part < kLeastTiles ? kLeastTiles : part;
}
// Tiles of a row block's parts: one size over all sequences, so that workgroups are alike where lengths are not.  The
// longest sequence sets it, not the caller's bound, in which a captured step leaves room: under a bound of 131,072, 48
// sequences of up to 16,384 tokens in 8 bits take 106 us (233 with parts cut from the bound; 105 under 16,384), 1,024
// tokens x 7 heads over 10,677 194 (362), 8 sequences of up to 1,183 16 (53).  Reading the lengths costs a few tenths of a
// microsecond in each of the two launches.  All the lanes of a wave call it.
template <int T>
__device__ __forceinline__ int part_of(const AttendParams& p) {
  if (p.size != 0) return p.size;
  int longest = p.len[0];
  if (p.B > 1) {
    int m = 0;
    for (int i = threadIdx.x & 63; i < p.B; i += 64) m = p.len[i] > m ? p.len[i] : m;
    const auto larger = [&](int y) { m = y > m ? y : m; };
    larger(dpp_u32<kDppQuadXor1>(m));
    larger(dpp_u32<kDppQuadXor2>(m));
    larger(dpp_u32<kDppRowHalfMirror>(m));
    larger(dpp_u32<kDppRowMirror>(m));
    for (int r = 0; r < 64; r += 16) longest = __builtin_amdgcn_readlane(m, r) > longest ? __builtin_amdgcn_readlane(m, r) : longest;
  }
  longest = longest < 0 ? 0 : longest < p.max_len ? longest : p.max_len;
  return part_tiles(most_tiles(longest, T, p.window, p.sinks, p.max_q), p.want);
}
__device__ __forceinline__ int splits_of(const AttendParams& p, int tiles, int part) {
  const int s = (tiles + part - 1) / part;
  return s < 1 ? 1 : s < p.splits ? s : p.splits;
}

// A sequence's table entry for a key (or its last one), and the page that it stands for: -1 where there is none.
__device__ __forceinline__ int entry_of(const AttendParams& p, const int32_t* table, int key) {
  const int j = key >> p.pool.shift;
  return table[j < p.pool.max_pages ? j : p.pool.max_pages - 1];
}
__device__ __forceinline__ int page_of(const AttendParams& p, int entry, int key) {
  return key >> p.pool.shift < p.pool.max_pages && entry >= 0 && entry < p.pool.num_pages ? entry : -1;
}

// Few rows over many keys: memory-bound.  A workgroup = W waves over one (sequence, KV head, block of 16 R
// rows, part of the keys); the waves take its tiles in turn, each with its own running maximum and sum, and
// join at the end.  Nothing passes through LDS before that:
//  S^T = K Q^T by 16x16x32 products.  Row m of the A operand may be any key; with key 8 (m / 4) + 4 t + m % 4 in
//    row m of product t, lane (r, g) ends with the scores of query row r and keys 8 g .. 8 g + 7, which is
//    where the B operand of the next product wants P^T.  The contracted d is permuted as the loads like it.
//  O^T = V^T P^T: a lane loads 8 values of each of its 8 keys (8 r .. 8 r + 7 of a row) and turns the 8 x 8
//    block in registers (one v_perm for two values), so that row m of product c is d = 8 m + c, and a lane
//    ends with 8 consecutive d of each of four blocks.
// A row's maximum is only raised when a score passes it by 2^8 (the lanes exchange scores when any row's does), so most
// tiles need no exchange; probabilities of up to 256 round like others.
// 131,071 bf16 tokens of 4 KV heads (268 MB): 45 us, the rate at which memory is read; 48 sequences of up to 16,384 tokens
// in 8 bits (484 MB) 96 us, 5.0 TB/s, the last parts of unequal lengths.  Short contexts wait for the chain of offsets,
// table entry, page and first tile: 1,183 tokens 7 us.
// Three waves per SIMD for 16 rows: 48 ragged sequences of up to 16,384 tokens in 8 bits take 104 us with three and
// 117 with two (the registers that two would have are not needed); 32 rows do not fit in three's.
template <int D, int BITS, int R, int W>
__global__ __launch_bounds__(64 * W, R == 1 ? 3 : 2) void attend_few(const AttendParams p) {
  constexpr int T = tile_keys(BITS), U = T / 32;      // keys per step, in blocks of 32
  constexpr int KS = (D + 31) / 32;                   // products along d
  constexpr int KW = BITS == 16 ? 4 : 2;              // dwords of 8 values
  constexpr int E = BITS / 8;
  __shared__ float join[W / 2][8 * 4 * R + 2 * R][64];
  __shared__ uint32_t poison[16 * R][D / 4];
  __shared__ int poisoned;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  int id = remap_block_id(blockIdx.x, gridDim.x);
  const int split = id % p.splits;
  id /= p.splits;
  const int rb = id % p.row_blocks;
  id /= p.row_blocks;
  const int hk = id % p.pool.heads, b = id / p.pool.heads;
  const int part = part_of<T>(p);
  Span sp = queries_of(p, b);
  const int rows = sp.nq * p.group, x0 = rb * 16 * R;
  if (x0 >= rows) return;
  const int x1 = x0 + 16 * R < rows ? x0 + 16 * R - 1 : rows - 1;
  tiles_of<T>(p, x0 / p.group, x1 / p.group, &sp);
  const int splits = splits_of(p, sp.tiles, part);
  if (split >= splits) return;
  const int t0 = static_cast<int>(static_cast<long long>(sp.tiles) * split / splits);
  const int t1 = static_cast<int>(static_cast<long long>(sp.tiles) * (split + 1) / splits);
  if (sp.p_lo != sp.p_hi) {
    for (int i = threadIdx.x; i < 16 * R * (D / 4); i += 64 * W) poison[i / (D / 4)][i % (D / 4)] = 0;
  }
  if (threadIdx.x == 0) poisoned = 0;
  __syncthreads();

  uint4 qf[R][KS];
  int place[R];
#pragma unroll
  for (int t = 0; t < R; ++t) {
    const int x = x0 + 16 * t + r, xi = x <= x1 ? x : x1;
    place[t] = sp.len - sp.nq + xi / p.group;
    const uint16_t* from = p.q + (static_cast<long long>(sp.row0 + xi / p.group) * p.Hq + hk * p.group + xi % p.group) * D;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = BITS == 8 && D == 128 ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
      qf[t][s] = d < D ? *reinterpret_cast<const uint4*>(from + d) : make_uint4(0, 0, 0, 0);
    }
  }

  const int32_t* table = p.pool.table + static_cast<long long>(b) * p.pool.max_pages;
  const long long head_bytes = static_cast<long long>(p.pool.page) * D * E;
  const int slot_mask = p.pool.page - 1;
  // lane constants: the K rows (product 0; product 1 is 4 rows on) and V rows of a block that a lane loads
  const int krow = 8 * (r >> 2) + (r & 3), khalf = r >> 3, vhalf = g >> 1;
  const int koff = ((krow & 15) * D + (BITS == 8 && D == 128 ? 16 * g : 8 * g)) * E;
  const int voff = ((8 * g & 15) * D + (8 * r < D ? 8 * r : 0)) * E;

  uint32_t kr[U][2][KS][KW], vr[U][8][KW];
  float ks[U], vs[U], ks_n[U], vs_n[U];
  // pages of the loaded tile's halves of 16; the table's entries for the next tile, untouched until they are needed (a
  // test right after the load would wait for it in every tile)
  int pg[2 * U], entry[2 * U];

  const auto look_up = [&](int base) {
#pragma unroll
    for (int h = 0; h < 2 * U; ++h) entry[h] = entry_of(p, table, base + 16 * h);
  };
  const auto take_pages = [&](int base) {
#pragma unroll
    for (int h = 0; h < 2 * U; ++h) pg[h] = page_of(p, entry[h], base + 16 * h);
  };
  const auto half_base = [&](const void* pool, int key, int page) {
    return static_cast<const char*>(pool) + (static_cast<long long>(page < 0 ? 0 : page) * p.pool.heads + hk) * head_bytes +
           static_cast<long long>(key & slot_mask) * D * E;
  };
  const auto load_k = [&](int base) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = base + 32 * u;
      const char* from = (khalf ? half_base(p.pool.k, at + 16, pg[2 * u + 1]) : half_base(p.pool.k, at, pg[2 * u])) + koff;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* f = from + 4 * t * D * E;
        if constexpr (BITS == 8 && D == 128) {
#pragma unroll
          for (int s = 0; s < KS; s += 2) {
            const u32x4 x = stream16(f + 32 * s);
            kr[u][t][s][0] = x.x; kr[u][t][s][1] = x.y; kr[u][t][s + 1][0] = x.z; kr[u][t][s + 1][1] = x.w;
          }
        } else {
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            // D = 80: the last product has 16 values, its upper lanes load the lower ones' again
            const int off = (32 * s - (32 * s + 32 > D && g >= 2 ? 16 : 0)) * E;
            if constexpr (BITS == 8) {
              const u32x2 x = stream8(f + off);
              kr[u][t][s][0] = x.x; kr[u][t][s][1] = x.y;
            } else {
              const u32x4 x = stream16(f + off);
              kr[u][t][s][0] = x.x; kr[u][t][s][1] = x.y; kr[u][t][s][2] = x.z; kr[u][t][s][3] = x.w;
            }
          }
        }
      }
      if constexpr (BITS == 8) {
        const int page = vhalf ? pg[2 * u + 1] : pg[2 * u];
        const long long ph = static_cast<long long>(page < 0 ? 0 : page) * p.pool.heads + hk;
        ks_n[u] = p.pool.k_scale[ph];
        vs_n[u] = p.pool.v_scale[ph];
      }
    }
  };
  const auto load_v = [&](int base) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = base + 32 * u;
      const char* from = (vhalf ? half_base(p.pool.v, at + 16, pg[2 * u + 1]) : half_base(p.pool.v, at, pg[2 * u])) + voff;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const char* f = from + j * D * E;
        if constexpr (BITS == 8) {
          const u32x2 x = stream8(f);
          vr[u][j][0] = x.x; vr[u][j][1] = x.y;
        } else {
          const u32x4 x = stream16(f);
          vr[u][j][0] = x.x; vr[u][j][1] = x.y; vr[u][j][2] = x.z; vr[u][j][3] = x.w;
        }
      }
    }
  };
  // the A operand of O^T's product c over block u
  const auto v_operand = [&](int u, int c) {
    uint32_t a[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (BITS == 8) {
        const uint32_t y =
            __builtin_amdgcn_perm(vr[u][2 * k + 1][c >> 2], vr[u][2 * k][c >> 2], (c & 2) ? 0x07030602u : 0x05010400u);
        a[k] = (c & 1) ? e4m3_bf16<true>(y) : e4m3_bf16<false>(y);
      } else {
        a[k] = __builtin_amdgcn_perm(vr[u][2 * k + 1][c >> 1], vr[u][2 * k][c >> 1], (c & 1) ? 0x07060302u : 0x05040100u);
      }
    }
    return make_uint4(a[0], a[1], a[2], a[3]);
  };

  f32x4 acc[R][8];
  float m[R], l[R];
#pragma unroll
  for (int t = 0; t < R; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  int x = t0 + w;
  if (x < t1) {
    look_up(T * sp.tile(x));
    take_pages(T * sp.tile(x));
    load_k(T * sp.tile(x));
    load_v(T * sp.tile(x));
    if (x + W < t1) look_up(T * sp.tile(x + W));
  }
  for (; x < t1; x += W) {
    const int base = T * sp.tile(x);
    const bool more = x + W < t1;
    const int next = more ? T * sp.tile(x + W) : 0;
    bool ok[2 * U], full = base + T - 1 <= sp.p_lo && (p.window == 0 || base > sp.p_hi - p.window || base + T <= p.sinks);
#pragma unroll
    for (int h = 0; h < 2 * U; ++h) {
      ok[h] = pg[h] >= 0;
      full = full && ok[h];                            // every row sees every key of the tile
    }
    f32x4 st[R][U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (BITS == 8) { ks[u] = ks_n[u]; vs[u] = vs_n[u]; }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int t = 0; t < R; ++t) st[t][u][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          uint4 a;
          if constexpr (BITS == 8) a = e4m3_bf16x8(kr[u][h][s][0], kr[u][h][s][1]);
          else a = make_uint4(kr[u][h][s][0], kr[u][h][s][1], kr[u][h][s][2], kr[u][h][s][3]);
          if (32 * s + 32 > D && g >= 2) a = make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int t = 0; t < R; ++t) st[t][u][h] = mfma16(a, qf[t][s], st[t][u][h]);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);                 // K's registers are free from here on, not earlier
    if (more) {
      take_pages(next);
      load_k(next);
      if (x + 2 * W < t1) look_up(T * sp.tile(x + 2 * W));
    }
    uint4 pf[R][U];
#pragma unroll
    for (int t = 0; t < R; ++t) {
      float s[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float f = BITS == 8 ? p.scale_log2 * ks[u] : p.scale_log2;
#pragma unroll
        for (int j = 0; j < 8; ++j) s[u][j] = st[t][u][j >> 2][j & 3] * f;
      }
      if (!full) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int key = base + 32 * u + 8 * g + j;
            const bool sees = (vhalf ? ok[2 * u + 1] : ok[2 * u]) && key <= place[t] &&
                              (p.window == 0 || key > place[t] - p.window || key < p.sinks);
            s[u][j] = sees ? s[u][j] : -INFINITY;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u)
        top = fmaxf(top, max3(max3(s[u][0], s[u][1], s[u][2]), max3(s[u][3], s[u][4], s[u][5]), fmaxf(s[u][6], s[u][7])));
      if (__any(top > m[t] + 8.f)) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mn = top > m[t] + 8.f ? top : m[t];   // a row's own scores alone decide about its sums
        const float k = mn == m[t] ? 1.f : exp2_fast(m[t] - mn);
        m[t] = mn;
        l[t] *= k;
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[t][c] *= k;
      }
      const float mz = m[t] == -INFINITY ? 0.f : m[t];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          e[j] = exp2_fast(s[u][j] - mz);
          l[t] += e[j];
          // a scale of hidden keys may be anything
          if constexpr (BITS == 8) e[j] = full || s[u][j] != -INFINITY ? e[j] * vs[u] : 0.f;
        }
        // probabilities are rounded to bf16 for the product (relative 2^-8); their sum is not
        pf[t][u] = pack8(e);
      }
    }
    bool odd = false;                                  // a V value that is not finite, seen by some rows only
    if (!full) {
      uint32_t wild = 0;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          // V rows that no row sees become 0 (0 * NaN is NaN)
          const int key = base + 32 * u + 8 * g + j;
          const bool sees = (vhalf ? ok[2 * u + 1] : ok[2 * u]) && key <= sp.p_hi &&
                            (p.window == 0 || key > sp.p_lo - p.window || key < p.sinks);
#pragma unroll
          for (int d = 0; d < KW; ++d) {
            vr[u][j][d] = sees ? vr[u][j][d] : 0u;
            wild |= not_finite<BITS>(vr[u][j][d]);
          }
        }
      odd = sp.p_lo != sp.p_hi && __any(wild != 0);
    }
    if (odd) {
      // Values that are not finite must reach the rows that see them and no others, but a hidden one's 0 times NaN is
      // NaN: the products take 0 for them, and `poison` notes which results get a +inf or -inf (1, 2; a NaN
      // counts as both).  Rare, so it reads V again, two values of a key per lane.
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int d = 0; d < KW; ++d) {
            asm volatile("" : "+v"(vr[u][j][d]));      // or the tests above stay in 32 registers until here
            const uint32_t m = not_finite<BITS>(vr[u][j][d]);
            vr[u][j][d] &= ~(BITS == 16 ? (m >> 15) * 0xffffu : (m >> 7) * 0xffu);
          }
      poisoned = 1;
#pragma unroll 1
      for (int key = base; key < base + T; ++key) {
        const int page = page_of(p, entry_of(p, table, key), key);
        if (page < 0 || 2 * lane >= D) continue;
        const char* from = half_base(p.pool.v, key, page) + 2 * lane * E;
        uint32_t kind = 0;                             // a byte for each of the lane's two values
        for (int e = 0; e < 2; ++e) {
          uint32_t mag, neg;
          if constexpr (BITS == 16) {
            const uint32_t h = *reinterpret_cast<const uint16_t*>(from + 2 * e);
            mag = h & 0x7fffu;
            neg = h >> 15;
          } else {
            mag = (*reinterpret_cast<const uint8_t*>(from + e) & 0x7fu) == 0x7fu ? 0x7fffu : 0u;
            neg = 0;
          }
          kind |= (mag > 0x7f80u ? 3u : mag == 0x7f80u ? 1u << neg : 0u) << 8 * e;
        }
        if (kind == 0) continue;
        for (int x = x0; x <= x1; ++x) {
          const int at = sp.len - sp.nq + x / p.group;
          if (key <= at && (p.window == 0 || key > at - p.window || key < p.sinks))
            atomicOr(&poison[x - x0][lane >> 1], kind << 16 * (lane & 1));
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint4 a = v_operand(u, c);
#pragma unroll
        for (int t = 0; t < R; ++t) acc[t][c] = mfma16(a, pf[t][u], acc[t][c]);
      }
    __builtin_amdgcn_sched_barrier(0);
    if (more) load_v(next);
  }

  // the waves join in halves: maximum, sum and O of the upper half go through LDS
#pragma unroll
  for (int h = W / 2; h >= 1; h >>= 1) {
    if (w >= h && w < 2 * h) {
#pragma unroll
      for (int t = 0; t < R; ++t) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) join[w - h][(t * 8 + c) * 4 + i][lane] = acc[t][c][i];
        join[w - h][32 * R + 2 * t][lane] = m[t];
        join[w - h][32 * R + 2 * t + 1][lane] = l[t];
      }
    }
    __syncthreads();
    if (w < h) {
#pragma unroll
      for (int t = 0; t < R; ++t) {
        const float m2 = join[w][32 * R + 2 * t][lane], l2 = join[w][32 * R + 2 * t + 1][lane];
        const float mn = fmaxf(m[t], m2);
        const float k1 = mn == m[t] ? 1.f : exp2_fast(m[t] - mn), k2 = mn == m2 ? 1.f : exp2_fast(m2 - mn);
        m[t] = mn;
        l[t] = l[t] * k1 + l2 * k2;
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[t][c][i] = acc[t][c][i] * k1 + join[w][(t * 8 + c) * 4 + i][lane] * k2;
      }
    }
    __syncthreads();
  }
  if (w == 0) {
    if (poisoned) {
#pragma unroll
      for (int t = 0; t < R; ++t)
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int d = 8 * (4 * g + i) + c;
            const uint32_t k = d < D ? poison[16 * t + r][d >> 2] >> 8 * (d & 3) : 0u;
            acc[t][c][i] += (k & 1u) ? INFINITY : 0.f;
            acc[t][c][i] -= (k & 2u) ? INFINITY : 0.f;
          }
    }
#pragma unroll
    for (int t = 0; t < R; ++t) {
      float sum = l[t] + __shfl_xor(l[t], 16, 64);
      sum += __shfl_xor(sum, 32, 64);
      const int x = x0 + 16 * t + r;
      if (x > x1) continue;
      const int n = sp.row0 + x / p.group, h = hk * p.group + x % p.group;
      const long long out = static_cast<long long>(n) * p.Hq + h;
      if (splits > 1) {
        const long long row = static_cast<long long>(split) * p.n_q * p.Hq + out;
        float* to = p.part + row * (D + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int d = 8 * (4 * g + i);
          if (d >= D) continue;
          *reinterpret_cast<float4*>(to + d) = make_float4(acc[t][0][i], acc[t][1][i], acc[t][2][i], acc[t][3][i]);
          *reinterpret_cast<float4*>(to + d + 4) = make_float4(acc[t][4][i], acc[t][5][i], acc[t][6][i], acc[t][7][i]);
        }
        if (g == 0) *reinterpret_cast<float2*>(to + D) = make_float2(m[t], sum);
        continue;
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = 8 * (4 * g + i);
        if (d >= D) continue;
        float y[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) y[c] = acc[t][c][i] * inv;
        *reinterpret_cast<uint4*>(p.o + out * D + d) = pack8(y);
      }
      if (g == 0 && p.lse) p.lse[static_cast<long long>(h) * p.n_q + n] = sum == 0.f ? -INFINITY : (m[t] + log2f(sum)) * kLn2;
    }
  }
}

// Many rows (drafts of many heads, the next chunk of a prompt): bound by the matrix products.  A workgroup = 8 waves
// of 32 rows of one KV head, as G groups: one over 256 rows, or two over the same 128 rows that take the tiles of 64 keys
// in turn and join at the end (so that two waves on every SIMD overlap one's products with the other's exponentials also
// where there are few rows).  A group stages its tile through registers (paged rows and 8-bit codes need their own
// addresses and a conversion) into LDS, the next one in flight while this one is worked on:
//  K row-major, rows 16 bytes apart in their banks; S^T = K Q^T by 32x32x16 products, so a lane owns one row (the
//    column) and 16 keys of each half of the tile.
//  V transposed on the way in (4 keys x 8 d in registers), [d][key] with the keys of each 16 in the order in which the
//    lanes hold P^T (groups of 4: 0, 2, 1, 3), so that O^T = V^T P^T takes P straight from registers; 16-byte pieces
//    swizzled by d.
// Operands are read from LDS four products ahead: one at a time, each product waited out its read (253 us against 211;
// eight ahead do not fit the registers, 239).
// With 256 rows the registers hold two tiles on their way, which hides most of their arrival (1,024 tokens x 7 heads
// over 10,677: 200 us against 212 with one); with 128 rows a thread stages twice as much, and they hold one.
// That case runs its 149 GFLOP at 760 TFLOP/s, its join included: its 112 row blocks in two parts are 224 workgroups, which
// leave 32 CUs without one; on the others two waves on a SIMD leave their waits (a third), the exponentials and the
// staging partly uncovered, and LDS and registers have no room for a third.
// NP: the pages of a tile, 1 (64 or more tokens a page) or 4 (one for each 16 keys).
constexpr int kManyTile = 64, kManyThreads = 512;
constexpr int many_rows(int groups) { return 256 / groups; }
typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(uint4 a, uint4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int D, int BITS, int NP, int G>
__global__ __launch_bounds__(kManyThreads, 2) void attend_many(const AttendParams p) {
  constexpr int T = kManyTile, E = BITS / 8, KS = D / 16, DT = (D + 31) / 32, KEYS = T / NP;
  constexpr int CPR = BITS == 16 ? D / 8 : D / 16;    // 16-byte pieces of a cached row
  constexpr int NT = kManyThreads / G, WAVES = 8 / G, ROWS = 32 * WAVES;
  constexpr int NK = (T * CPR + NT - 1) / NT;         // of them per thread
  constexpr int KROW = 17;                            // a K row's pieces in LDS
  constexpr int VD = 4 * G, VW = VD * E / 4, DG = 128 / VD;   // V: d per thread, their dwords, threads along d
  __shared__ uint4 kt[G][2][T * KROW];                // [group][buffer]: [key][pieces]
  __shared__ uint4 vt[G][2][32 * DT * 8];             // [d][8 pieces of 8 keys]
  __shared__ uint32_t poison[ROWS][D / 16];      // 2 bits for each value
  __shared__ int poisoned;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int gr = wave / WAVES, w = wave % WAVES, tid = threadIdx.x % NT, c32 = lane & 31, g = lane >> 5;
  int id = remap_block_id(blockIdx.x, gridDim.x);
  const int rb = id % p.row_blocks;
  id /= p.row_blocks;
  const int split = id % p.splits;
  id /= p.splits;
  const int hk = id % p.pool.heads, b = id / p.pool.heads;
  const int part = part_of<T>(p);
  Span sp = queries_of(p, b);
  const int rows = sp.nq * p.group, x0 = rb * ROWS;
  if (x0 >= rows) return;
  const int x1 = x0 + ROWS < rows ? x0 + ROWS - 1 : rows - 1;
  tiles_of<T>(p, x0 / p.group, x1 / p.group, &sp);
  const int splits = splits_of(p, sp.tiles, part);
  if (split >= splits) return;
  const int t0 = static_cast<int>(static_cast<long long>(sp.tiles) * split / splits);
  const int t1 = static_cast<int>(static_cast<long long>(sp.tiles) * (split + 1) / splits);
  for (int i = threadIdx.x; i < ROWS * (D / 16); i += kManyThreads) poison[i / (D / 16)][i % (D / 16)] = 0;
  if (threadIdx.x == 0) poisoned = 0;

  const int x = x0 + 32 * w + c32, xi = x <= x1 ? x : x1;
  const int place = sp.len - sp.nq + xi / p.group;
  u32x4 qf[KS];
  {
    const uint16_t* from = p.q + (static_cast<long long>(sp.row0 + xi / p.group) * p.Hq + hk * p.group + xi % p.group) * D + 8 * g;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const u32x4*>(from + 16 * s);
  }

  const int32_t* table = p.pool.table + static_cast<long long>(b) * p.pool.max_pages;
  const long long head_bytes = static_cast<long long>(p.pool.page) * D * E;
  const int slot_mask = p.pool.page - 1;
  const int dg = lane % DG, vkey = (64 / DG) * 4 * w + 4 * (lane / DG);   // V: this thread's VD d's and 4 keys
  const int vpart = NP == 1 ? 0 : w * 4 / WAVES;       // the part of the tile that they lie in
  constexpr int SETS = G == 1 ? 2 : 1;                 // tiles in flight; two groups have registers for one
  uint32_t kr[SETS][NK][4], vr[SETS][4][VW];
  int entry[NP], pg[SETS][NP], pg_v[SETS];             // the next tile's entries, the pages of those in flight
  float ks[NP], vs[NP], ks_n[SETS][NP], vs_n[SETS][NP];

  const auto look_up = [&](int base) {
#pragma unroll
    for (int h = 0; h < NP; ++h) entry[h] = entry_of(p, table, base + KEYS * h);
  };
  const auto row_of = [&](const void* pool, int key, int page) {
    return static_cast<const char*>(pool) + (static_cast<long long>(page < 0 ? 0 : page) * p.pool.heads + hk) * head_bytes +
           static_cast<long long>(key & slot_mask) * D * E;
  };
  // lane constants: the part of a tile that a thread's K pieces lie in, and where there; its V rows
  int koff[NK], kpart[NK];
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    const int at = i * NT + tid, row = at / CPR < T ? at / CPR : T - 1;
    kpart[i] = row / KEYS;
    koff[i] = (row % KEYS) * D * E + at % CPR * 16;
  }
  const int voff = (vkey % KEYS * D + (VD * dg < D ? VD * dg : 0)) * E;
  const auto load = [&](int base, auto set) {
    constexpr int S = decltype(set)::value;
    const char *kb[NP], *vb = nullptr;                 // the same for all lanes
#pragma unroll
    for (int h = 0; h < NP; ++h) {
      pg[S][h] = page_of(p, entry[h], base + KEYS * h);
      kb[h] = row_of(p.pool.k, base + KEYS * h, pg[S][h]);
      if (h == vpart) {
        vb = row_of(p.pool.v, base + KEYS * h, pg[S][h]);
        pg_v[S] = pg[S][h];
      }
      if constexpr (BITS == 8) {
        const long long ph = static_cast<long long>(pg[S][h] < 0 ? 0 : pg[S][h]) * p.pool.heads + hk;
        ks_n[S][h] = p.pool.k_scale[ph];
        vs_n[S][h] = p.pool.v_scale[ph];
      }
    }
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const char* from = kb[0];
      if constexpr (NP > 1) {
        // where the pieces of 16 rows fill whole waves, the part is the same for a wave
        const int part = 16 * CPR % 64 == 0 ? (i * NT + 64 * w) / (16 * CPR) : kpart[i];
        from = part < 2 ? (part == 0 ? kb[0] : kb[1]) : (part == 2 ? kb[2] : kb[3]);
      }
      const u32x4 y = *reinterpret_cast<const u32x4*>(from + koff[i]);
      kr[S][i][0] = y.x; kr[S][i][1] = y.y; kr[S][i][2] = y.z; kr[S][i][3] = y.w;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const char* from = vb + voff + j * D * E;
      if constexpr (VW == 4) {
        const u32x4 y = *reinterpret_cast<const u32x4*>(from);
        vr[S][j][0] = y.x; vr[S][j][1] = y.y; vr[S][j][2] = y.z; vr[S][j][3] = y.w;
      } else if constexpr (VW == 2) {
        const u32x2 y = *reinterpret_cast<const u32x2*>(from);
        vr[S][j][0] = y.x; vr[S][j][1] = y.y;
      } else {
        vr[S][j][0] = *reinterpret_cast<const uint32_t*>(from);
      }
    }
  };
  // every row of the workgroup sees every key of the tile (whose pages are in pg)
  const auto is_full = [&](int base, int s) {
    bool ok = base + T - 1 <= sp.p_lo && (p.window == 0 || base > sp.p_hi - p.window || base + T <= p.sinks);
#pragma unroll
    for (int h = 0; h < NP; ++h) ok = ok && pg[s][h] >= 0;
    return ok;
  };
  const auto store = [&](int base, int buf, auto set) {
    constexpr int S = decltype(set)::value;
    uint4* kl = kt[gr][buf];
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int at = i * NT + tid, row = at / CPR, piece = at % CPR;
      if (T * CPR % NT != 0 && row >= T) continue;
      if constexpr (BITS == 16) {
        kl[row * KROW + piece] = make_uint4(kr[S][i][0], kr[S][i][1], kr[S][i][2], kr[S][i][3]);
      } else {
        kl[row * KROW + 2 * piece] = e4m3_bf16x8(kr[S][i][0], kr[S][i][1]);
        kl[row * KROW + 2 * piece + 1] = e4m3_bf16x8(kr[S][i][2], kr[S][i][3]);
      }
    }
    if (!is_full(base, S)) {
      // V rows that no row sees become 0 (0 * NaN is NaN); where the rows differ, values that are not finite too, and
      // `poison` notes which results get a +inf or -inf instead (1, 2; a NaN counts as both)
      uint32_t wild = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = base + vkey + j;
        const bool sees = pg_v[S] >= 0 && key <= sp.p_hi && (p.window == 0 || key > sp.p_lo - p.window || key < p.sinks);
#pragma unroll
        for (int d = 0; d < VW; ++d) {
          vr[S][j][d] = sees ? vr[S][j][d] : 0u;
          const uint32_t m = not_finite<BITS>(vr[S][j][d]);
          wild |= m;
          if (sp.p_lo != sp.p_hi) vr[S][j][d] &= ~(BITS == 16 ? (m >> 15) * 0xffffu : (m >> 7) * 0xffu);
        }
      }
      if (sp.p_lo != sp.p_hi && __any(wild != 0)) {
        poisoned = 1;
#pragma unroll 1
        for (int key = base + (T / WAVES) * w; key < base + (T / WAVES) * (w + 1); ++key) {
          const int page = page_of(p, entry_of(p, table, key), key);
          if (page < 0 || 2 * lane >= D) continue;
          const char* from = row_of(p.pool.v, key, page) + 2 * lane * E;
          uint32_t kind = 0;
          for (int e = 0; e < 2; ++e) {
            uint32_t mag, neg;
            if constexpr (BITS == 16) {
              const uint32_t h = *reinterpret_cast<const uint16_t*>(from + 2 * e);
              mag = h & 0x7fffu;
              neg = h >> 15;
            } else {
              mag = (*reinterpret_cast<const uint8_t*>(from + e) & 0x7fu) == 0x7fu ? 0x7fffu : 0u;
              neg = 0;
            }
            kind |= (mag > 0x7f80u ? 3u : mag == 0x7f80u ? 1u << neg : 0u) << 2 * e;
          }
          if (kind == 0) continue;
          for (int y = x0; y <= x1; ++y) {
            const int at = sp.len - sp.nq + y / p.group;
            if (key <= at && (p.window == 0 || key > at - p.window || key < p.sinks))
              atomicOr(&poison[y - x0][lane >> 3], kind << 4 * (lane & 7));
          }
        }
      }
    }
    // 4 keys x VD d: for each d, the 4 keys are one 8-byte unit of its row
    uint2* vl = reinterpret_cast<uint2*>(vt[gr][buf]);
    if (VD * dg < D) {
      const int q = vkey >> 2, unit = (q & ~3) + 2 * (q & 1) + (q >> 1 & 1);       // keys 4 q of a chunk of 16: 0, 2, 1, 3
#pragma unroll
      for (int c = 0; c < VD; ++c) {
        uint2 y;
        if constexpr (BITS == 8) {
          const uint32_t lo = __builtin_amdgcn_perm(vr[S][1][c >> 2], vr[S][0][c >> 2], (c & 2) ? 0x07030602u : 0x05010400u);
          const uint32_t hi = __builtin_amdgcn_perm(vr[S][3][c >> 2], vr[S][2][c >> 2], (c & 2) ? 0x07030602u : 0x05010400u);
          y = (c & 1) ? make_uint2(e4m3_bf16<true>(lo), e4m3_bf16<true>(hi)) : make_uint2(e4m3_bf16<false>(lo), e4m3_bf16<false>(hi));
        } else {
          const uint32_t sel = (c & 1) ? 0x07060302u : 0x05040100u;
          y = make_uint2(__builtin_amdgcn_perm(vr[S][1][c >> 1], vr[S][0][c >> 1], sel), __builtin_amdgcn_perm(vr[S][3][c >> 1], vr[S][2][c >> 1], sel));
        }
        const int d = VD * dg + c;
        vl[d * 16 + (((unit >> 1) ^ ((d ^ (d >> 3)) & 7)) << 1 | (unit & 1))] = y;
      }
    }
  };

  f32x16 acc[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  const int mine = t1 - t0 - gr > 0 ? (t1 - t0 - gr + G - 1) / G : 0, most = (t1 - t0 + G - 1) / G;   // group 0 has the most
  bool full_cur = false, ok_cur[NP];
#pragma unroll
  for (int h = 0; h < NP; ++h) ok_cur[h] = false;
  const auto tile_base = [&](int i) { return T * sp.tile(t0 + gr + G * i); };
  const auto took = [&](int base, int s) {
    full_cur = is_full(base, s);
#pragma unroll
    for (int h = 0; h < NP; ++h) {
      ok_cur[h] = pg[s][h] >= 0;
      if constexpr (BITS == 8) { ks[h] = ks_n[s][h]; vs[h] = vs_n[s][h]; }
    }
  };
  constexpr std::integral_constant<int, 0> S0;
  constexpr std::integral_constant<int, SETS - 1> S1;
  __syncthreads();                                     // poison is clear
  if (mine > 0) {
    look_up(tile_base(0));
    load(tile_base(0), S0);
    store(tile_base(0), 0, S0);
    took(tile_base(0), 0);
    if (mine > 1) look_up(tile_base(1));
    if (SETS == 2 && mine > 1) {
      load(tile_base(1), S1);
      if (mine > 2) look_up(tile_base(2));
    }
  }
  // the queries have arrived: or the loop's first product waits, in every step, for whatever was loaded last
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[s]));
  __syncthreads();
  // One step: tile `it` lies in LDS, the next one in set `next` (SETS = 2: set `free` takes the one after) or on its way
  const auto step = [&](int it, auto free, auto next) {
    if (it + SETS < mine) load(tile_base(it + SETS), free);
    if (it + SETS + 1 < mine) look_up(tile_base(it + SETS + 1));
    if (it < mine) {
      const int base = tile_base(it), buf = it & 1;
      const uint4* kl = kt[gr][buf] + c32 * KROW + g;
      const uint4* vl[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) vl[c] = vt[gr][buf] + c32 * 8 + ((2 * c + g) ^ ((c32 ^ (c32 >> 3)) & 7));
      // d = 32 t + c32: an odd t flips bit 2 of the swizzle, which is bit 1 of c
      const auto v_at = [&](int k) { return vl[(k & 3) ^ ((k >> 2 & 1) << 1)][(k >> 2) * 256]; };
      const auto k_at = [&](int k) { return kl[(k & 1) * 32 * KROW + 2 * (k >> 1)]; };   // halves in turn
      f32x16 st[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) st[h][i] = 0.f;
      uint4 a[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] = k_at(k);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 2 * KS; ++k) {
        st[k & 1] = mfma32(a[k & 3], __builtin_bit_cast(uint4, qf[k >> 1]), st[k & 1]);
        if (k + 4 < 2 * KS) a[k & 3] = k_at(k + 4);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) a[k] = v_at(k);
      __builtin_amdgcn_sched_barrier(0);
      float f[NP];
#pragma unroll
      for (int h = 0; h < NP; ++h) f[h] = BITS == 8 ? p.scale_log2 * ks[h] : p.scale_log2;
      if (!full_cur) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = base + 32 * h + 8 * (i >> 2) + 4 * g + (i & 3);
            const bool sees = ok_cur[(2 * h + (i >> 3)) % NP] && key <= place &&
                              (p.window == 0 || key > place - p.window || key < p.sinks);
            st[h][i] = sees ? st[h][i] : -INFINITY;
          }
      }
      float top = -INFINITY;                           // scales are positive: the largest product times its scale
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int o = 8 * (c & 1);
        const float y = max3(max3(st[c >> 1][o], st[c >> 1][o + 1], st[c >> 1][o + 2]),
                             max3(st[c >> 1][o + 3], st[c >> 1][o + 4], st[c >> 1][o + 5]), fmaxf(st[c >> 1][o + 6], st[c >> 1][o + 7]));
        top = fmaxf(top, full_cur || y != -INFINITY ? y * f[c % NP] : -INFINITY);   // see below
      }
      if (__any(top > m + 8.f)) {
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mn = top > m + 8.f ? top : m, k = mn == m ? 1.f : exp2_fast(m - mn);
        m = mn;
        l *= k;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[t][i] *= k;
      }
      const float mz = m == -INFINITY ? 0.f : m;
      uint4 pf[4];
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float s = st[c >> 1][8 * (c & 1) + i];
          e[i] = exp2_fast(fmaf(s, f[c % NP], -mz));
          // the scales of pages that hold hidden keys alone may be anything, NaN and negative numbers among it
          if constexpr (BITS == 8) e[i] = full_cur || s != -INFINITY ? e[i] : 0.f;
          sum += e[i];
          if constexpr (BITS == 8) e[i] = full_cur || s != -INFINITY ? e[i] * vs[c % NP] : 0.f;
        }
        // probabilities are rounded to bf16 for the product (relative 2^-8); their sum is not
        pf[c] = pack8(e);
      }
      l += sum;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 4 * DT; ++k) {
        acc[k >> 2] = mfma32(a[k & 3], pf[k & 3], acc[k >> 2]);
        if (k + 4 < 4 * DT) a[k & 3] = v_at(k + 4);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (it + 1 < mine) {
      store(tile_base(it + 1), (it + 1) & 1, next);
      took(tile_base(it + 1), decltype(next)::value);
    }
    __syncthreads();
  };
  if constexpr (SETS == 1) {
    for (int it = 0; it < most; ++it) step(it, S0, S0);
  } else {
    for (int it = 0; it < most; it += 2) {
      step(it, S0, S1);
      if (it + 1 < most) step(it + 1, S1, S0);
    }
  }

  if constexpr (G == 2) {
    // group 1's maximum, sum and O go to group 0 through the K tiles' LDS
    float* join = reinterpret_cast<float*>(&kt[0][0][0]);
    constexpr int PART = DT == 4 ? 2 : DT;               // tiles of O at a time
    static_assert(sizeof(kt) >= (4 * PART * 16 + 8) * 64 * sizeof(float), "the waves' parts of O must fit the K tiles");
#pragma unroll
    for (int t = 0; t < DT; t += PART) {
      if (gr == 1) {
#pragma unroll
        for (int u = 0; u < PART; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) join[((w * PART + u) * 16 + i) * 64 + lane] = acc[t + u][i];
        if (t == 0) {
          join[(4 * PART * 16 + 2 * w) * 64 + lane] = m;
          join[(4 * PART * 16 + 2 * w + 1) * 64 + lane] = l;
        }
      }
      __syncthreads();
      if (gr == 0) {
        const float m2 = join[(4 * PART * 16 + 2 * w) * 64 + lane], l2 = join[(4 * PART * 16 + 2 * w + 1) * 64 + lane];
        const float mn = fmaxf(m, m2);
        const float k1 = mn == m ? 1.f : exp2_fast(m - mn), k2 = mn == m2 ? 1.f : exp2_fast(m2 - mn);
#pragma unroll
        for (int u = 0; u < PART; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            acc[t + u][i] = acc[t + u][i] * k1 + join[((w * PART + u) * 16 + i) * 64 + lane] * k2;
        if (t + PART >= DT) {
          l = l * k1 + l2 * k2;
          m = mn;
        }
      }
      __syncthreads();
    }
  }
  if (gr != 0) return;
  if (poisoned) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int d = 32 * t + 8 * (i >> 2) + 4 * g + (i & 3);
        const uint32_t k = d < D ? poison[32 * w + c32][d >> 4] >> 2 * (d & 15) : 0u;
        acc[t][i] += (k & 1u) ? INFINITY : 0.f;
        acc[t][i] -= (k & 2u) ? INFINITY : 0.f;
      }
  }
  const float sum = l + __shfl_xor(l, 32, 64);
  if (x > x1) return;
  const int n = sp.row0 + x / p.group, h = hk * p.group + x % p.group;
  const long long out = static_cast<long long>(n) * p.Hq + h;
  if (splits > 1) {
    float* to = p.part + (static_cast<long long>(split) * p.n_q * p.Hq + out) * (D + 4);
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = 32 * t + 8 * j + 4 * g;
        if (d < D) *reinterpret_cast<float4*>(to + d) = make_float4(acc[t][4 * j], acc[t][4 * j + 1], acc[t][4 * j + 2], acc[t][4 * j + 3]);
      }
    if (g == 0) *reinterpret_cast<float2*>(to + D) = make_float2(m, sum);
    return;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = 32 * t + 8 * j + 4 * g;
      if (d < D)
        *reinterpret_cast<uint2*>(p.o + out * D + d) = make_uint2(pack_bf16x2(acc[t][4 * j] * inv, acc[t][4 * j + 1] * inv),
                                                                  pack_bf16x2(acc[t][4 * j + 2] * inv, acc[t][4 * j + 3] * inv));
    }
  if (g == 0 && p.lse) p.lse[static_cast<long long>(h) * p.n_q + n] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * kLn2;
}

// Joins the parts of the rows whose keys were split.  W = 8: a workgroup per row, its waves take the parts in turn;
// W = 1: half a wave per row, for up to 8 parts (two parts of 28,672 rows: 75 us with their attention, 80 with a wave a
// row, 152 with a workgroup; 128 parts of 28 rows: 52 us with a workgroup, 70 with a wave).  Bound by its chain of launch,
// lengths and parts (3 to 5 us), which the waves of 28,672 rows go through four times over: 10.5 us for 37 MB.
constexpr int kJoinWaves = 8, kJoinLanes = 32;
template <int D, int T, int W>
__global__ __launch_bounds__(64 * kJoinWaves) void attend_join(const AttendParams p, int block_rows) {
  constexpr int L = W == 1 ? kJoinLanes : 64, V = 128 / L;     // lanes of a row, and values of each
  __shared__ float part[W][V + 1][64];
  const int lane = threadIdx.x & (L - 1), w = W == 1 ? 0 : threadIdx.x >> 6;
  int id = W == 1 ? blockIdx.x * (64 * kJoinWaves / L) + threadIdx.x / L : blockIdx.x;
  const int h = id % p.Hq;
  id /= p.Hq;
  const int i = id % p.max_q, b = id / p.max_q;
  const int tiles_part = part_of<T>(p);
  if (W == 1 && b >= p.B) return;
  Span sp = queries_of(p, b);
  if (i >= sp.nq) return;
  // the tiles of the row block that this row was in
  const int rows = sp.nq * p.group, x = i * p.group + h % p.group, x0 = x / block_rows * block_rows;
  const int x1 = x0 + block_rows < rows ? x0 + block_rows - 1 : rows - 1;
  tiles_of<T>(p, x0 / p.group, x1 / p.group, &sp);
  const int splits = splits_of(p, sp.tiles, tiles_part);
  if (splits == 1) return;
  const int n = sp.row0 + i;
  const long long row = static_cast<long long>(n) * p.Hq + h, all = static_cast<long long>(p.n_q) * p.Hq;
  float m = -INFINITY, sum = 0.f, y[V];
#pragma unroll
  for (int e = 0; e < V; ++e) y[e] = 0.f;
  for (int s0 = w; s0 < splits; s0 += 4 * W) {
    float ms[4], ls[4];
    float v[4][V];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = s0 + u * W;
      const float* from = p.part + ((s < splits ? s : s0) * all + row) * (D + 4);
      const float2 ml = *reinterpret_cast<const float2*>(from + D);
      ms[u] = s < splits ? ml.x : -INFINITY;
      ls[u] = s < splits ? ml.y : 0.f;
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        float2 z = make_float2(0.f, 0.f);
        if (s < splits && V * lane < D) z = *reinterpret_cast<const float2*>(from + V * lane + e);
        v[u][e] = z.x;
        v[u][e + 1] = z.y;
      }
    }
    const float mn = fmaxf(m, fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3])));
    const float k = m == mn ? 1.f : exp2_fast(m - mn);
    m = mn;
    sum *= k;
#pragma unroll
    for (int e = 0; e < V; ++e) y[e] *= k;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = ms[u] == mn ? 1.f : exp2_fast(ms[u] - mn);
      sum += ls[u] * f;
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] += v[u][e] * f;
    }
  }
  float top = m;
  if constexpr (W > 1) {
#pragma unroll
    for (int e = 0; e < V; ++e) part[w][e][lane] = y[e];
    part[w][V][lane] = lane == 0 ? m : sum;
    __syncthreads();
    if (w != 0) return;
    top = part[0][V][0];
#pragma unroll
    for (int u = 1; u < W; ++u) top = fmaxf(top, part[u][V][0]);
    sum = 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) y[e] = 0.f;
#pragma unroll
    for (int u = 0; u < W; ++u) {
      const float f = part[u][V][0] == top ? 1.f : exp2_fast(part[u][V][0] - top);
      sum += part[u][V][1] * f;
#pragma unroll
      for (int e = 0; e < V; ++e) y[e] += part[u][e][lane] * f;
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (V * lane < D) {
#pragma unroll
    for (int e = 0; e < V; e += 2)
      *reinterpret_cast<uint32_t*>(p.o + row * D + V * lane + e) = pack_bf16x2(y[e] * inv, y[e + 1] * inv);
  }
  if (lane == 0 && p.lse) p.lse[static_cast<long long>(h) * p.n_q + n] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// How a call is laid out: rows of a KV head per workgroup, and the parts that a row block's keys are split into.
struct AttendPlan {
  int rows, row_blocks, splits, want, size;
  long long blocks;
};
constexpr int kWaves = 4;
// Up to 32 rows go to attend_few: 8 sequences of 5 rows x 4 heads take 46 us there and 80 in attend_many, which keeps a
// tile for rows that are not there.  Beyond 128 rows attend_many takes 256 per workgroup (G = 1) where that leaves 32
// workgroups before any split: 1,024 tokens x 7 heads over 10,677 take 200 us against 211 with 128 rows, 4,096 tokens
// over 8,000 474 against 556, 40 tokens x 4 heads of 8 sequences 113 against 128.  Fewer blocks of 256 rows would need
// twice the parts of 128-row ones, and joining them costs more than reading the keys once less: 48 tokens (8 blocks)
// take 38 us with 256 rows and 32 with 128, 200 tokens (24 blocks) 74 and 62.
constexpr int kManyBlocks = 32;
AttendPlan plan_attention(int Hq, int heads, int bits, int B, int max_q, int max_len, int window, int sinks) {
  AttendPlan a;
  const long long rows = static_cast<long long>(max_q) * (Hq / heads);
  const long long wide = (rows + many_rows(1) - 1) / many_rows(1) * heads * B;
  a.rows = rows > many_rows(2) && wide >= kManyBlocks ? many_rows(1) : rows > 32 ? many_rows(2) : rows > 16 ? 32 : 16;
  a.row_blocks = static_cast<int>((rows + a.rows - 1) / a.rows);
  const long long base = static_cast<long long>(B) * heads * a.row_blocks;
  if (window >= max_len) window = 0;                  // such a window hides nothing
  const int tile = a.rows > 32 ? kManyTile : tile_keys(bits);
  // Workgroups to aim at.  Many rows: one on every CU, all that its registers hold (40 tokens x 4 heads of 8 sequences
  // 119 us; 512 in all 124, 1,024 155).  Few: two a CU where that is all that fits (32 rows: 8 sequences of 20 rows 47 us,
  // with four 54) or the sequences' parts are alike, whose number only costs in the join (one sequence of 131,071: 52 us,
  // with four 56; 24 that a window of 4,096 bounds: 30.7 and 33.2), else four: 48 sequences of up to 16,384 take 104 us,
  // with two 140.
  // Where sequences and heads alone give that many workgroups nothing is split, and a sequence far longer than the others
  // takes its own time: 256 sequences x 4 heads, one of 131,072 tokens and 255 of 1,000, 1,770 us (the long one in a call of
  // its own 54, the others 90).  Parts of at most 4,096 keys whatever the batch is make that 380 us, but their empty
  // workgroups cost a batch under a loose bound more than it has to lose (512 sequences x 8 heads of up to 2,048 tokens under
  // 131,072: 433 us, with such parts 645).
  const bool alike = B == 1 || (window > 0 && 2 * (static_cast<long long>(window) + sinks + max_q) <= max_len);
  const long long aim = a.rows > 32 ? 256 : a.rows == 32 || alike ? 512 : 1024;
  a.want = static_cast<int>(aim / base < 1 ? 1 : aim / base);
  const int least = (most_tiles(max_len, tile, window, sinks, max_q) + kLeastTiles - 1) / kLeastTiles;
  a.splits = least < a.want ? least : a.want;          // no length up to max_len makes more
  if (a.splits < 1) a.splits = 1;
  // nothing to split, or parts of the least size whatever the lengths are: nobody reads those of the other sequences
  a.size = a.splits == 1 || least <= a.want ? kLeastTiles : 0;
  a.blocks = base * a.splits;
  return a;
}
// Whether B sequences of max_q queries and Hq heads stay under 2^31 rows, as the plan and the kernels' numbers assume.
bool rows_fit(int B, int max_q, int Hq) {
  const long long lim = 1ll << 31, q = static_cast<long long>(B) * max_q;
  return q < lim && q * Hq < lim && static_cast<long long>(B) * Hq < lim;
}
size_t attend_bytes(const AttendPlan& a, int n_q, int Hq, int dim) {
  return a.splits == 1 ? 0 : static_cast<size_t>(a.splits) * n_q * Hq * (dim + 4) * sizeof(float);
}

template <int D, int BITS, int G>
void launch_many(const AttendParams& p, dim3 grid, hipStream_t stream) {
  if (p.pool.page >= kManyTile) hipLaunchKernelGGL((attend_many<D, BITS, 1, G>), grid, dim3(kManyThreads), 0, stream, p);
  else hipLaunchKernelGGL((attend_many<D, BITS, 4, G>), grid, dim3(kManyThreads), 0, stream, p);
}

template <int D, int T>
void launch_join(const AttendParams& p, const AttendPlan& a, hipStream_t stream) {
  const long long rows = static_cast<long long>(p.B) * p.max_q * p.Hq;
  constexpr int per = 64 * kJoinWaves / kJoinLanes;    // rows of a workgroup, for few parts
  const dim3 th(64 * kJoinWaves);
  if (a.splits <= 8)
    hipLaunchKernelGGL((attend_join<D, T, 1>), dim3(static_cast<unsigned>((rows + per - 1) / per)), th, 0, stream, p, a.rows);
  else
    hipLaunchKernelGGL((attend_join<D, T, kJoinWaves>), dim3(static_cast<unsigned>(rows)), th, 0, stream, p, a.rows);
}

template <int D, int BITS>
pace_status_t launch_attend(const AttendParams& p, const AttendPlan& a, hipStream_t stream) {
  const dim3 g(static_cast<unsigned>(a.blocks)), th(64 * kWaves);
  if (a.rows == 16) hipLaunchKernelGGL((attend_few<D, BITS, 1, kWaves>), g, th, 0, stream, p);
  else if (a.rows == 32) hipLaunchKernelGGL((attend_few<D, BITS, 2, kWaves>), g, th, 0, stream, p);
  else if (a.rows == many_rows(2)) launch_many<D, BITS, 2>(p, g, stream);
  else launch_many<D, BITS, 1>(p, g, stream);
  if (a.splits > 1) {
    if (a.rows > 32) launch_join<D, kManyTile>(p, a, stream);
    else launch_join<D, tile_keys(BITS)>(p, a, stream);
  }
  return check_launch("pace_cache_attention");
}

// ---------------------------------------------------------------- host checks
constexpr long long kMostThreads = (1ll << 32) - 64 * kJoinWaves;    // of a launch; a grid may round up to a workgroup more

pace_status_t check_cache(const pace_kv_cache* c, const int32_t* table, int max_pages, int B, const char* what,
                          Pool* out) {
  PACE_REQUIRE(c != nullptr && c->k && c->v && table, "%s: null cache or block_table", what);
  PACE_REQUIRE(c->bits == 16 || c->bits == 8, "%s: bits=%d not 16 or 8", what, c->bits);
  PACE_REQUIRE(c->bits == 16 || (c->k_scale && c->v_scale), "%s: 8-bit pages need k_scale and v_scale", what);
  PACE_REQUIRE(aligned16(c->k) && aligned16(c->v), "%s: the cache must be 16-byte aligned", what);
  PACE_REQUIRE(c->num_pages >= 1 && c->heads >= 1 && max_pages >= 1 && B >= 1,
               "%s: num_pages=%d heads=%d max_pages=%d B=%d", what, c->num_pages, c->heads, max_pages, B);
  PACE_REQUIRE(c->page >= 16 && c->page <= 256 && (c->page & (c->page - 1)) == 0,
               "%s: page=%d not 16, 32, 64, 128 or 256", what, c->page);
  if (c->dim != 80 && c->dim != 128)
    return set_error(PACE_ERR_UNSUPPORTED, "%s: head dim %d not in {80, 128}", what, c->dim);
  PACE_REQUIRE(static_cast<long long>(max_pages) * c->page <= (1ll << 31) - 1024, "%s: max_pages * page past 2^31 - 1024", what);
  out->k = c->k; out->v = c->v; out->k_scale = c->k_scale; out->v_scale = c->v_scale;
  out->table = table;
  out->num_pages = c->num_pages; out->max_pages = max_pages; out->heads = c->heads; out->page = c->page;
  out->shift = __builtin_ctz(static_cast<unsigned>(c->page));
  return PACE_OK;
}

// PACE_DEBUG: pages [first_b, last_b) of every sequence's table lie in the pool and, with `once`, no
// page occurs twice among them.
pace_status_t check_pages(const Pool& p, int B, const std::vector<int>& first, const std::vector<int>& last, bool once,
                          const char* what, hipStream_t stream) {
  std::vector<int32_t> t(static_cast<size_t>(p.max_pages));
  std::vector<char> seen(once ? static_cast<size_t>(p.num_pages) : 0, 0);
  for (int b = 0; b < B; ++b) {
    pace_status_t st = copy_to_host(t.data(), p.table + static_cast<long long>(b) * p.max_pages, p.max_pages, stream);
    if (st != PACE_OK) return st;
    for (int j = first[b]; j < last[b]; ++j) {
      PACE_REQUIRE(t[j] >= 0 && t[j] < p.num_pages, "%s: block_table[%d][%d] = %d outside [0, %d)", what, b, j, t[j],
                   p.num_pages);
      if (once) {
        PACE_REQUIRE(!seen[t[j]], "%s: page %d is written twice", what, t[j]);
        seen[t[j]] = 1;
      }
    }
  }
  return PACE_OK;
}

pace_status_t debug_append(const AppendParams& p, hipStream_t stream) {
  const char* what = "pace_cache_append";
  pace_status_t st = check_offsets(p.cu, p.B, p.n_new, p.max_new, "pace_cache_append: cu_new", stream);
  if (st != PACE_OK) return st;
  std::vector<int32_t> cu(p.B + 1), ctx(p.B);
  if ((st = copy_to_host(cu.data(), p.cu, p.B + 1, stream)) != PACE_OK ||
      (st = copy_to_host(ctx.data(), p.ctx, p.B, stream)) != PACE_OK)
    return st;
  std::vector<int> first(p.B), last(p.B);
  for (int b = 0; b < p.B; ++b) {
    const long long n = cu[b + 1] - cu[b], end = ctx[b] + n;
    PACE_REQUIRE(ctx[b] >= 0 && end <= static_cast<long long>(p.pool.max_pages) * p.pool.page,
                 "%s: sequence %d: %d cached and %lld new tokens in %d pages of %d", what, b, ctx[b], n,
                 p.pool.max_pages, p.pool.page);
    first[b] = ctx[b] >> p.pool.shift;
    last[b] = n ? static_cast<int>((end - 1) >> p.pool.shift) + 1 : first[b];
  }
  if ((st = check_pages(p.pool, p.B, first, last, true, what, stream)) != PACE_OK) return st;
  if (p.rows) return check_values(p.rows, cu[p.B], nullptr, 0, p.n_src - 1, "pace_cache_append: rows", stream);
  return PACE_OK;
}

pace_status_t debug_attention(const AttendParams& p, hipStream_t stream) {
  const char* what = "pace_cache_attention";
  pace_status_t st = check_offsets(p.cu, p.B, p.n_q, p.max_q, "pace_cache_attention: cu_q", stream);
  if (st != PACE_OK) return st;
  if ((st = check_values(p.len, p.B, nullptr, 0, p.max_len, "pace_cache_attention: seq_len", stream)) != PACE_OK) return st;
  std::vector<int32_t> len(p.B), cu(p.B + 1);
  if ((st = copy_to_host(len.data(), p.len, p.B, stream)) != PACE_OK ||
      (st = copy_to_host(cu.data(), p.cu, p.B + 1, stream)) != PACE_OK)
    return st;
  // the pages that some query sees: those of the sinks, and from the first query's window on
  std::vector<int> zero(p.B, 0), sinks(p.B), first(p.B), last(p.B);
  for (int b = 0; b < p.B; ++b) {
    const bool none = cu[b + 1] == cu[b];
    const long long from = p.window == 0 ? 0 : static_cast<long long>(len[b]) - (cu[b + 1] - cu[b]) - p.window + 1;
    first[b] = from <= 0 ? 0 : static_cast<int>(from >> p.pool.shift);
    last[b] = none ? 0 : (len[b] + p.pool.page - 1) >> p.pool.shift;
    sinks[b] = none ? 0 : ((p.sinks < len[b] ? p.sinks : len[b]) + p.pool.page - 1) >> p.pool.shift;
  }
  if ((st = check_pages(p.pool, p.B, zero, sinks, false, what, stream)) != PACE_OK) return st;
  return check_pages(p.pool, p.B, first, last, false, what, stream);
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" {

pace_status_t pace_cache_append(const uint16_t* q, long long q_stride, const uint16_t* k, long long k_stride,
                                const uint16_t* v, long long v_stride, int n_src, int Hq, const int32_t* rows,
                                const int32_t* cu_new, int B, int n_new, int max_new, const int32_t* ctx_len,
                                const int32_t* block_table, int max_pages, const int32_t* positions, int axes,
                                const int* sections, const float* inv_freq, const pace_kv_cache* cache,
                                uint16_t* q_out, hipStream_t stream) {
  AppendParams p{};
  pace_status_t st = check_cache(cache, block_table, max_pages, B, "pace_cache_append", &p.pool);
  if (st != PACE_OK) return st;
  const int d = cache->dim, hkv = cache->heads;
  PACE_REQUIRE(k && v && cu_new && ctx_len, "pace_cache_append: null device pointer");
  PACE_REQUIRE(q == nullptr || (q_out != nullptr && Hq >= 1), "pace_cache_append: q needs q_out and Hq >= 1");
  PACE_REQUIRE(aligned16(q) && aligned16(k) && aligned16(v) && aligned16(q_out),
               "pace_cache_append: q/k/v/q_out must be 16-byte aligned");
  PACE_REQUIRE(n_src >= 0 && n_new >= 0 && max_new >= 0 && max_new <= n_new && (rows != nullptr || n_new <= n_src),
               "pace_cache_append: n_src=%d n_new=%d max_new=%d", n_src, n_new, max_new);
  const long long kv = static_cast<long long>(hkv) * d, qr = q ? static_cast<long long>(Hq) * d : 0;
  PACE_REQUIRE(k_stride >= kv && v_stride >= kv && k_stride % 8 == 0 && v_stride % 8 == 0 &&
                   (q == nullptr || (q_stride >= qr && q_stride % 8 == 0)),
               "pace_cache_append: strides %lld, %lld, %lld must be multiples of 8 and hold a row", q_stride, k_stride,
               v_stride);
  PACE_REQUIRE((positions == nullptr) == (inv_freq == nullptr), "pace_cache_append: positions and inv_freq go together");
  p.end0 = p.end1 = d / 2;
  if (positions) {
    PACE_REQUIRE(axes == 1 || axes == 3, "pace_cache_append: axes=%d not 1 or 3", axes);
    if (axes == 3) {
      PACE_REQUIRE(sections && sections[0] >= 0 && sections[1] >= 0 && sections[2] >= 0 &&
                       static_cast<long long>(sections[0]) + sections[1] + sections[2] == d / 2,
                   "pace_cache_append: the three sections must sum to dim / 2 = %d", d / 2);
      p.end0 = sections[0];
      p.end1 = sections[0] + sections[1];
    }
  }
  const char* many = "pace_cache_append: too many sequences, tokens or heads";
  const long long lim = 1ll << 31;
  PACE_REQUIRE(n_new < lim - 1024 && static_cast<long long>(B) * max_new < lim, "%s", many);
  if (max_new == 0) return PACE_OK;
  p.q = q; p.k = k; p.v = v; p.qs = q_stride; p.ks = k_stride; p.vs = v_stride;
  p.rows = rows; p.cu = cu_new; p.ctx = ctx_len; p.pos = positions; p.freq = inv_freq; p.q_out = q_out;
  p.n_src = n_src; p.n_new = n_new; p.max_new = max_new; p.B = B; p.Hq = Hq;
  p.tokens = 1;
  while (p.tokens < kAppendTokens && static_cast<long long>(B) * max_new / (2 * p.tokens) >= 512) p.tokens *= 2;
  p.tiles = (max_new + p.tokens - 1) / p.tokens;
  p.pages = (max_new - 1 + cache->page - 1) / cache->page + 1;
  const long long row_blocks = static_cast<long long>(B) * p.tiles;
  const long long held = static_cast<long long>(B) * p.pages;
  PACE_REQUIRE(held < lim, "%s", many);
  const long long page_blocks = 2 * held * hkv;
  PACE_REQUIRE(row_blocks + page_blocks < kMostThreads / kAppendThreads && kAppendTokens * (static_cast<long long>(q ? Hq : 0) + 2ll * hkv) * d < lim, "%s", many);
  if (debug_checks()) {
    try {
      if ((st = debug_append(p, stream)) != PACE_OK) return st;
    } catch (const std::bad_alloc&) {
      return set_error(PACE_ERR_INVALID_ARG, "pace_cache_append: no host memory for the debug checks");
    }
  }
  return d == 80 ? launch_append<80>(p, cache->bits, row_blocks, page_blocks, stream)
                 : launch_append<128>(p, cache->bits, row_blocks, page_blocks, stream);
}

size_t pace_cache_attention_workspace_size(int n_q, int Hq, int heads, int dim, int bits, int B, int max_q, int max_len,
                                           int window, int sinks) {
  if (n_q < 1 || heads < 1 || Hq < heads || Hq % heads != 0 || dim < 1 || (bits != 16 && bits != 8) || B < 1 || max_q < 1 || max_len < 0 ||
      window < 0 || sinks < 0 || !rows_fit(B, max_q, Hq))
    return 0;
  const AttendPlan a = plan_attention(Hq, heads, bits, B, max_q, max_len, window, sinks);
  return attend_bytes(a, n_q, Hq, dim);
}

pace_status_t pace_cache_attention(const uint16_t* q, int n_q, int Hq, const pace_kv_cache* cache,
                                   const int32_t* cu_q, int B, int max_q, const int32_t* seq_len, int max_len,
                                   const int32_t* block_table, int max_pages, int window, int sinks, float scale,
                                   uint16_t* o, float* lse, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream) {
  AttendParams p{};
  pace_status_t st = check_cache(cache, block_table, max_pages, B, "pace_cache_attention", &p.pool);
  if (st != PACE_OK) return st;
  PACE_REQUIRE(q && o && cu_q && seq_len, "pace_cache_attention: null device pointer");
  PACE_REQUIRE(aligned16(q) && aligned16(o), "pace_cache_attention: q/o must be 16-byte aligned");
  PACE_REQUIRE(Hq >= 1 && Hq % cache->heads == 0, "pace_cache_attention: Hq=%d not a multiple of %d heads", Hq,
               cache->heads);
  PACE_REQUIRE(n_q >= 0 && max_q >= 0 && max_q <= n_q && max_len >= 0 &&
                   max_len <= static_cast<long long>(max_pages) * cache->page,
               "pace_cache_attention: n_q=%d max_q=%d max_len=%d (at most max_pages * page)", n_q, max_q, max_len);
  PACE_REQUIRE(window >= 0 && sinks >= 0, "pace_cache_attention: window=%d sinks=%d", window, sinks);
  PACE_REQUIRE(isfinite(scale) && scale > 0.f, "pace_cache_attention: scale must be positive");
  PACE_REQUIRE(rows_fit(B, max_q, Hq), "pace_cache_attention: too many queries and heads");
  if (max_q == 0) return PACE_OK;
  p.q = q; p.cu = cu_q; p.len = seq_len; p.o = o; p.lse = lse;
  p.n_q = n_q; p.Hq = Hq; p.group = Hq / cache->heads; p.B = B; p.max_q = max_q; p.max_len = max_len;
  p.window = window >= max_len ? 0 : window;
  p.sinks = sinks; p.scale_log2 = scale * kLog2e;
  const AttendPlan a = plan_attention(Hq, cache->heads, cache->bits, B, max_q, max_len, window, sinks);
  const long long joins = a.splits == 1 ? 0 : static_cast<long long>(B) * max_q * Hq * (a.splits <= 8 ? kJoinLanes : 64 * kJoinWaves);
  PACE_REQUIRE(a.blocks * (a.rows > 32 ? kManyThreads : 64 * kWaves) < kMostThreads && joins < kMostThreads,
               "pace_cache_attention: too many queries and heads");
  p.row_blocks = a.row_blocks;
  p.splits = a.splits;
  p.want = a.want;
  p.size = a.size;
  const size_t need = attend_bytes(a, n_q, Hq, cache->dim);
  if (need) {
    if (workspace == nullptr || workspace_bytes < need)
      return set_error(PACE_ERR_WORKSPACE, "pace_cache_attention: workspace %zu < %zu bytes", workspace_bytes, need);
    PACE_REQUIRE(aligned16(workspace), "pace_cache_attention: workspace must be 16-byte aligned");
    p.part = static_cast<float*>(workspace);
  }
  if (debug_checks()) {
    try {
      if ((st = debug_attention(p, stream)) != PACE_OK) return st;
    } catch (const std::bad_alloc&) {
      return set_error(PACE_ERR_INVALID_ARG, "pace_cache_attention: no host memory for the debug checks");
    }
  }
  if (cache->dim == 128)
    return cache->bits == 16 ? launch_attend<128, 16>(p, a, stream) : launch_attend<128, 8>(p, a, stream);
  return cache->bits == 16 ? launch_attend<80, 16>(p, a, stream) : launch_attend<80, 8>(p, a, stream);
}

}  // extern "C"
