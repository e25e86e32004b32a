// The paged cache of a pruned context: rotation of new queries and keys by their positions with the
// append of keys and values (bf16 pages, or e4m3 codes with a power-of-two scale for each page and
// head), and the attention of new tokens over the cached ones.
#include <math.h>

#include <new>
#include <vector>

#include "pace_internal.h"

namespace pace {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
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
  return r0 + n > p.n_new ? p.n_new - r0 : n;
}

constexpr int kAppendThreads = 256;
constexpr int kAppendTokens = 8;   // most tokens per workgroup

// Queries, and keys and values of bf16 pages.  A workgroup takes some tokens of one sequence: their
// angles' cos and sin go to LDS once (all heads share them), then every thread moves 16 values of one
// head (8 of each half, so that a pair meets in one thread) per step.
template <int D, bool KV>
__global__ __launch_bounds__(kAppendThreads) void append_rows(const AppendParams p) {
  constexpr int HALF = D / 2, CH = D / 16;
  __shared__ f32x2 cs[kAppendTokens * HALF];
  __shared__ int src_of[kAppendTokens];
  const int b = blockIdx.x / p.tiles, t0 = (blockIdx.x % p.tiles) * p.tokens;
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
// maximum and the store.
template <int D, int ITEMS>
__global__ __launch_bounds__(kAppendThreads) void append_pages(const AppendParams p) {
  constexpr int HALF = D / 2, CH = D / 16;
  __shared__ float red[kAppendThreads / 64];
  int id = blockIdx.x;
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
pace_status_t launch_append(const AppendParams& p, int bits, long long row_blocks, long long page_blocks,
                            hipStream_t stream) {
  const dim3 th(kAppendThreads);
  if (bits == 16) {
    hipLaunchKernelGGL((append_rows<D, true>), dim3(row_blocks), th, 0, stream, p);
  } else {
    if (p.q) hipLaunchKernelGGL((append_rows<D, false>), dim3(row_blocks), th, 0, stream, p);
    const dim3 g(page_blocks);
    const int items = (p.pool.page * (D / 16) + kAppendThreads - 1) / kAppendThreads;
    if (items <= 1) hipLaunchKernelGGL((append_pages<D, 1>), g, th, 0, stream, p);
    else if (items <= 2) hipLaunchKernelGGL((append_pages<D, 2>), g, th, 0, stream, p);
    else if (items <= 4) hipLaunchKernelGGL((append_pages<D, 4>), g, th, 0, stream, p);
    else hipLaunchKernelGGL((append_pages<D, 8>), g, th, 0, stream, p);
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
  float *part, *ml;          // partial results [splits, n_q * Hq, D] and their (maximum, sum)
  Pool pool;
  int n_q, Hq, group, B, max_q, max_len, window, sinks;
  int row_blocks, splits;
  float scale_log2;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;          // keys per step of a wave
constexpr int kSplitTiles = 8;     // least tiles per split of a sequence

__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Two e4m3 codes (the low or high pair of a dword) as two bf16 values: exact.
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_bf16(uint32_t u) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, HI));
}
__device__ __forceinline__ uint4 e4m3_bf16x8(uint32_t a, uint32_t b) {
  return make_uint4(e4m3_bf16<false>(a), e4m3_bf16<true>(a), e4m3_bf16<false>(b), e4m3_bf16<true>(b));
}

// What a sequence's queries are and the tiles that queries i_lo..i_hi of it see.
struct Span {
  int row0, nq, len;         // first row of q, queries, cached tokens
  int p_lo, p_hi;            // places of the first and last query
  int head_tiles, tail0, tiles;   // tiles [0, head_tiles) and [tail0, ...), tiles in all
  __device__ __forceinline__ int base(int x) const { return kTile * (x < head_tiles ? x : tail0 + x - head_tiles); }
};
__device__ __forceinline__ Span queries_of(const AttendParams& p, int b) {
  Span s;
  s.row0 = p.cu[b];
  s.nq = p.cu[b + 1] - s.row0;
  s.nq = s.nq > p.max_q ? p.max_q : s.nq;
  if (s.row0 < 0 || s.nq < 0) s.nq = 0;
  if (s.nq > p.n_q - s.row0) s.nq = p.n_q - s.row0;
  s.len = p.len[b];
  s.len = s.len > p.max_len ? p.max_len : s.len;
  return s;
}
__device__ __forceinline__ void tiles_of(const AttendParams& p, int i_lo, int i_hi, Span* s) {
  s->p_lo = s->len - s->nq + i_lo;
  s->p_hi = s->len - s->nq + i_hi;
  const int end = s->p_hi < 0 ? 0 : s->p_hi / kTile + 1;
  const int first = p.window == 0 ? 0 : s->p_lo - p.window + 1;      // p_lo < 2^31 and window >= 0: no overflow
  s->tail0 = first <= 0 ? 0 : first / kTile;
  const int sinks = p.sinks < s->p_hi + 1 ? p.sinks : s->p_hi + 1;
  s->head_tiles = sinks <= 0 ? 0 : (sinks + kTile - 1) / kTile;
  if (s->tail0 <= s->head_tiles) { s->tail0 = 0; s->head_tiles = 0; }
  s->tiles = end - s->tail0 + s->head_tiles;
}
// How many parts a sequence's tiles are split into.
__device__ __forceinline__ int splits_of(const AttendParams& p, int tiles) {
  const int most = (tiles + kSplitTiles - 1) / kSplitTiles;
  return most < 1 ? 1 : most < p.splits ? most : p.splits;
}

// A sequence's page of a 16-key half tile, or -1.
__device__ __forceinline__ int page_of(const AttendParams& p, const int32_t* table, int key) {
  const int j = key >> p.pool.shift;
  const int pg = j < p.pool.max_pages ? table[j] : -1;
  return pg >= 0 && pg < p.pool.num_pages ? pg : -1;
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
// A row's maximum is only raised when a score passes it by 2^8 (a wave-wide vote), so most tiles need no
// exchange between lanes; probabilities of up to 256 round like others.
template <int D, int BITS, int R, int W>
__global__ __launch_bounds__(64 * W) void attend_few(const AttendParams p) {
  constexpr int KS = (D + 31) / 32;                   // products along d
  constexpr int KW = BITS == 16 ? 4 : 2;              // dwords of 8 values
  __shared__ float join[W / 2][8 * 4 * R + 2 * R][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  int id = remap_block_id(blockIdx.x, gridDim.x);
  const int split = id % p.splits;
  id /= p.splits;
  const int rb = id % p.row_blocks;
  id /= p.row_blocks;
  const int hk = id % p.pool.heads, b = id / p.pool.heads;
  Span sp = queries_of(p, b);
  const int rows = sp.nq * p.group, x0 = rb * 16 * R;
  if (x0 >= rows) return;
  const int x1 = x0 + 16 * R < rows ? x0 + 16 * R - 1 : rows - 1;
  tiles_of(p, x0 / p.group, x1 / p.group, &sp);
  const int splits = splits_of(p, sp.tiles);
  if (split >= splits) return;
  const int t0 = static_cast<int>(static_cast<long long>(sp.tiles) * split / splits);
  const int t1 = static_cast<int>(static_cast<long long>(sp.tiles) * (split + 1) / splits);

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
  const long long head_bytes = static_cast<long long>(p.pool.page) * D * (BITS / 8);
  const int slot_mask = p.pool.page - 1;
  // lane constants: the K rows (product 0; product 1 is 4 rows on) and V rows of a tile that a lane loads
  const int krow = 8 * (r >> 2) + (r & 3), khalf = r >> 3, vhalf = g >> 1;
  const int kd = BITS == 8 && D == 128 ? 16 * g : 8 * g;
  const int koff = ((krow & 15) * D + kd) * (BITS / 8);
  const int voff = ((8 * g & 15) * D + (8 * r < D ? 8 * r : 0)) * (BITS / 8);

  uint32_t kr[2][KS][KW], vr[8][KW];
  float ks = 1.f, vs = 1.f, ks_n = 1.f, vs_n = 1.f;
  int pa, pb;                                          // pages of the loaded tile's halves

  const auto half_base = [&](const void* pool, int key, int pg) {
    return static_cast<const char*>(pool) + (static_cast<long long>(pg < 0 ? 0 : pg) * p.pool.heads + hk) * head_bytes +
           static_cast<long long>(key & slot_mask) * D * (BITS / 8);
  };
  const auto load_k = [&](int base, int a, int c) {
    const char* from = (khalf ? half_base(p.pool.k, base + 16, c) : half_base(p.pool.k, base, a)) + koff;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const char* f = from + 4 * t * D * (BITS / 8);
      if constexpr (BITS == 8 && D == 128) {
#pragma unroll
        for (int u = 0; u < KS / 2; ++u) {
          const uint4 x = *reinterpret_cast<const uint4*>(f + 64 * u);
          kr[t][2 * u][0] = x.x; kr[t][2 * u][1] = x.y; kr[t][2 * u + 1][0] = x.z; kr[t][2 * u + 1][1] = x.w;
        }
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          // D = 80: the last product has 16 values, its upper lanes load the lower ones' again
          const int at = (32 * s - (32 * s + 32 > D && g >= 2 ? 16 : 0)) * (BITS / 8);
          if constexpr (BITS == 8) {
            const uint2 x = *reinterpret_cast<const uint2*>(f + at);
            kr[t][s][0] = x.x; kr[t][s][1] = x.y;
          } else {
            const uint4 x = *reinterpret_cast<const uint4*>(f + at);
            kr[t][s][0] = x.x; kr[t][s][1] = x.y; kr[t][s][2] = x.z; kr[t][s][3] = x.w;
          }
        }
      }
    }
    if constexpr (BITS == 8) {
      const int pg = vhalf ? c : a;
      ks_n = p.pool.k_scale[static_cast<long long>(pg < 0 ? 0 : pg) * p.pool.heads + hk];
    }
  };
  const auto load_v = [&](int base, int a, int c) {
    const char* from = (vhalf ? half_base(p.pool.v, base + 16, c) : half_base(p.pool.v, base, a)) + voff;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const char* f = from + j * D * (BITS / 8);
      if constexpr (BITS == 8) {
        const uint2 x = *reinterpret_cast<const uint2*>(f);
        vr[j][0] = x.x; vr[j][1] = x.y;
      } else {
        const uint4 x = *reinterpret_cast<const uint4*>(f);
        vr[j][0] = x.x; vr[j][1] = x.y; vr[j][2] = x.z; vr[j][3] = x.w;
      }
    }
    if constexpr (BITS == 8) {
      const int pg = vhalf ? c : a;
      vs_n = p.pool.v_scale[static_cast<long long>(pg < 0 ? 0 : pg) * p.pool.heads + hk];
    }
  };
  // the A operand of O^T's product c from the loaded V rows (those of key `only`, or all: -1)
  const auto v_operand = [&](int c, int only) {
    uint32_t a[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (BITS == 8) {
        const uint32_t y = __builtin_amdgcn_perm(vr[2 * k + 1][c >> 2], vr[2 * k][c >> 2], (c & 2) ? 0x07030602u : 0x05010400u);
        a[k] = (c & 1) ? e4m3_bf16<true>(y) : e4m3_bf16<false>(y);
      } else {
        a[k] = __builtin_amdgcn_perm(vr[2 * k + 1][c >> 1], vr[2 * k][c >> 1], (c & 1) ? 0x07060302u : 0x05040100u);
      }
      if (only >= 0) a[k] = 8 * g + 2 * k == only ? a[k] & 0xffffu : 8 * g + 2 * k + 1 == only ? a[k] & 0xffff0000u : 0u;
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
  int pa_n = -1, pb_n = -1;
  if (x < t1) {
    const int base = sp.base(x);
    pa = page_of(p, table, base);
    pb = page_of(p, table, base + 16);
    load_k(base, pa, pb);
    load_v(base, pa, pb);
    if (x + W < t1) {
      const int nb = sp.base(x + W);
      pa_n = page_of(p, table, nb);
      pb_n = page_of(p, table, nb + 16);
    }
  }
  for (; x < t1; x += W) {
    const int base = sp.base(x);
    const bool more = x + W < t1;
    const int nbase = more ? sp.base(x + W) : 0;
    const bool ok_a = pa >= 0, ok_b = pb >= 0;
    if constexpr (BITS == 8) { ks = ks_n; vs = vs_n; }
    // every key of the tile is seen by every row
    const bool full = ok_a && ok_b && base + kTile - 1 <= sp.p_lo &&
                      (p.window == 0 || base > sp.p_hi - p.window || base + kTile <= p.sinks);
    f32x4 st[R][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int t = 0; t < R; ++t) st[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        uint4 a;
        if constexpr (BITS == 8) a = e4m3_bf16x8(kr[u][s][0], kr[u][s][1]);
        else a = make_uint4(kr[u][s][0], kr[u][s][1], kr[u][s][2], kr[u][s][3]);
        if (32 * s + 32 > D && g >= 2) a = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int t = 0; t < R; ++t) st[t][u] = mfma16(a, qf[t][s], st[t][u]);
      }
    }
    pa = pa_n;
    pb = pb_n;
    if (more) {
      load_k(nbase, pa, pb);
      if (x + 2 * W < t1) {
        const int nb = sp.base(x + 2 * W);
        pa_n = page_of(p, table, nb);
        pb_n = page_of(p, table, nb + 16);
      }
    }
    const float f = BITS == 8 ? p.scale_log2 * ks : p.scale_log2;
    uint4 pf[R];
    uint32_t seen[R];                                  // bit j: row sees key base + 8 g + j
    bool odd = false;                                  // some key is seen by some rows only and its V is not finite
#pragma unroll
    for (int t = 0; t < R; ++t) {
      float s[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = st[t][j >> 2][j & 3] * f;
      seen[t] = 0xffu;
      if (!full) {
        seen[t] = 0;
        const bool ok = vhalf ? ok_b : ok_a;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int key = base + 8 * g + j;
          const bool sees = ok && key <= place[t] && (p.window == 0 || key > place[t] - p.window || key < p.sinks);
          seen[t] |= sees ? 1u << j : 0u;
          s[j] = sees ? s[j] : -INFINITY;
        }
      }
      float top = s[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
      if (__any(top > m[t] + 8.f)) {
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mn = fmaxf(m[t], top);
        const float k = mn == m[t] ? 1.f : exp2_fast(m[t] - mn);
        m[t] = mn;
        l[t] *= k;
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[t][c] *= k;
      }
      const float mz = m[t] == -INFINITY ? 0.f : m[t];
      float e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        e[j] = exp2_fast(s[j] - mz);
        l[t] += e[j];
        if constexpr (BITS == 8) e[j] *= vs;
      }
      if (!full && BITS == 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = (seen[t] >> j & 1u) ? e[j] : 0.f;     // a scale nobody set may be NaN
      }
      // probabilities are rounded to bf16 for the product (relative 2^-8); their sum is not
      pf[t] = pack8(e);
    }
    if (!full) {
      // V rows that no row sees become 0 (0 * NaN is NaN)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int key = base + 8 * g + j;
        const bool sees = (vhalf ? ok_b : ok_a) && key <= sp.p_hi && (p.window == 0 || key > sp.p_lo - p.window || key < p.sinks);
#pragma unroll
        for (int d = 0; d < KW; ++d) vr[j][d] = sees ? vr[j][d] : 0u;
      }
      if (sp.p_lo != sp.p_hi) {
        // where the rows differ, V values that are not finite must reach only the rows that see them
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int d = 0; d < KW; ++d) {
            const uint32_t u = vr[j][d];
            if constexpr (BITS == 16) {
              bad |= (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u;
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) bad |= (u >> 8 * e & 0x7fu) == 0x7fu;
            }
          }
        odd = __any(bad);
      }
    }
    if (!odd) {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint4 a = v_operand(c, -1);
#pragma unroll
        for (int t = 0; t < R; ++t) acc[t][c] = mfma16(a, pf[t], acc[t][c]);
      }
    } else {
      // key by key, each added to the rows that see it alone
#pragma unroll 1
      for (int key = 0; key < kTile; ++key) {
        bool mine[R];
#pragma unroll
        for (int t = 0; t < R; ++t)
          mine[t] = __shfl(seen[t], (key >> 3) * 16 + r, 64) >> (key & 7) & 1u;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const uint4 a = v_operand(c, key);
#pragma unroll
          for (int t = 0; t < R; ++t) {
            const f32x4 y = mfma16(a, pf[t], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][c][i] += mine[t] ? y[i] : 0.f;
          }
        }
      }
    }
    if (more) load_v(nbase, pa, pb);
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
  if (w != 0) return;
#pragma unroll
  for (int t = 0; t < R; ++t) {
    float sum = l[t] + __shfl_xor(l[t], 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    const int x = x0 + 16 * t + r;
    if (x > x1) continue;
    const int n = sp.row0 + x / p.group, h = hk * p.group + x % p.group;
    const long long row = static_cast<long long>(n) * p.Hq + h;
    if (splits > 1) {
      const long long at = static_cast<long long>(split) * p.n_q * p.Hq + row;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = 8 * (4 * g + i);
        if (d >= D) continue;
        float4* to = reinterpret_cast<float4*>(p.part + at * D + d);
        to[0] = make_float4(acc[t][0][i], acc[t][1][i], acc[t][2][i], acc[t][3][i]);
        to[1] = make_float4(acc[t][4][i], acc[t][5][i], acc[t][6][i], acc[t][7][i]);
      }
      if (g == 0) *reinterpret_cast<float2*>(p.ml + 2 * at) = make_float2(m[t], sum);
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
      *reinterpret_cast<uint4*>(p.o + row * D + d) = pack8(y);
    }
    if (g == 0 && p.lse) p.lse[static_cast<long long>(h) * p.n_q + n] = sum == 0.f ? -INFINITY : (m[t] + log2f(sum)) * kLn2;
  }
}

// Joins the parts of the rows whose keys were split: one wave per row.
template <int D>
__global__ __launch_bounds__(256) void attend_join(const AttendParams p, int rows_per_block) {
  const int lane = threadIdx.x & 63;
  const long long id = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int h = static_cast<int>(id % p.Hq);
  const int i = static_cast<int>(id / p.Hq % p.max_q), b = static_cast<int>(id / p.Hq / p.max_q);
  if (b >= p.B) return;
  Span sp = queries_of(p, b);
  if (i >= sp.nq) return;
  // the tiles of the row block that this row was in
  const int rows = sp.nq * p.group, x = i * p.group + h % p.group, x0 = x / rows_per_block * rows_per_block;
  const int x1 = x0 + rows_per_block < rows ? x0 + rows_per_block - 1 : rows - 1;
  tiles_of(p, x0 / p.group, x1 / p.group, &sp);
  const int splits = splits_of(p, sp.tiles);
  if (splits == 1) return;
  const int n = sp.row0 + i;
  const long long row = static_cast<long long>(n) * p.Hq + h, all = static_cast<long long>(p.n_q) * p.Hq;
  float top = -INFINITY;
  for (int s = 0; s < splits; ++s) top = fmaxf(top, p.ml[2 * (s * all + row)]);
  float sum = 0.f, y0 = 0.f, y1 = 0.f;
  for (int s = 0; s < splits; ++s) {
    const long long at = s * all + row;
    const float m = p.ml[2 * at], k = m == top ? 1.f : exp2_fast(m - top);
    sum += p.ml[2 * at + 1] * k;
    if (2 * lane < D) {
      const float2 v = *reinterpret_cast<const float2*>(p.part + at * D + 2 * lane);
      y0 += v.x * k;
      y1 += v.y * k;
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (2 * lane < D) *reinterpret_cast<uint32_t*>(p.o + row * D + 2 * lane) = pack_bf16x2(y0 * inv, y1 * inv);
  if (lane == 0 && p.lse) p.lse[static_cast<long long>(h) * p.n_q + n] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// How a call is laid out: rows of a KV head per workgroup, and parts that a sequence's keys are split into.
struct AttendPlan {
  int rows, row_blocks, splits;
  long long blocks;
};
constexpr int kWaves = 8;
AttendPlan plan_attention(int Hq, int heads, int B, int max_q, int max_len, int window, int sinks) {
  AttendPlan a;
  const long long rows = static_cast<long long>(max_q) * (Hq / heads);
  a.rows = rows > 16 ? 32 : 16;
  a.row_blocks = static_cast<int>((rows + a.rows - 1) / a.rows);
  const long long base = static_cast<long long>(B) * heads * a.row_blocks;
  long long keys = max_len;
  if (window > 0 && static_cast<long long>(window) + sinks + max_q < keys) keys = static_cast<long long>(window) + sinks + max_q;
  const long long most = ((keys + kTile - 1) / kTile + kSplitTiles - 1) / kSplitTiles;
  // enough workgroups for two on every CU
  long long s = (512 + base - 1) / base;
  s = s > most ? most : s;
  a.splits = s < 1 ? 1 : static_cast<int>(s);
  a.blocks = base * a.splits;
  return a;
}

template <int D, int BITS>
pace_status_t launch_attend(const AttendParams& p, const AttendPlan& a, hipStream_t stream) {
  const dim3 g(static_cast<unsigned>(a.blocks)), th(64 * kWaves);
  if (a.rows == 16) hipLaunchKernelGGL((attend_few<D, BITS, 1, kWaves>), g, th, 0, stream, p);
  else hipLaunchKernelGGL((attend_few<D, BITS, 2, kWaves>), g, th, 0, stream, p);
  if (a.splits > 1) {
    const long long rows = static_cast<long long>(p.B) * p.max_q * p.Hq;
    hipLaunchKernelGGL(attend_join<D>, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(256), 0, stream, p, a.rows);
  }
  return check_launch("pace_cache_attention");
}

// ---------------------------------------------------------------- host checks
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
  PACE_REQUIRE(static_cast<long long>(max_pages) * c->page < (1ll << 31), "%s: max_pages * page past 2^31", what);
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
  std::vector<int32_t> len(p.B);
  if ((st = copy_to_host(len.data(), p.len, p.B, stream)) != PACE_OK) return st;
  std::vector<int> first(p.B, 0), last(p.B);
  for (int b = 0; b < p.B; ++b) last[b] = (len[b] + p.pool.page - 1) >> p.pool.shift;
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
  if (max_new == 0) return PACE_OK;
  p.q = q; p.k = k; p.v = v; p.qs = q_stride; p.ks = k_stride; p.vs = v_stride;
  p.rows = rows; p.cu = cu_new; p.ctx = ctx_len; p.pos = positions; p.freq = inv_freq; p.q_out = q_out;
  p.n_src = n_src; p.n_new = n_new; p.max_new = max_new; p.B = B; p.Hq = Hq;
  p.tokens = 1;
  while (p.tokens < kAppendTokens && static_cast<long long>(B) * max_new / (2 * p.tokens) >= 512) p.tokens *= 2;
  p.tiles = (max_new + p.tokens - 1) / p.tokens;
  p.pages = (max_new - 1 + cache->page - 1) / cache->page + 1;
  const long long row_blocks = static_cast<long long>(B) * p.tiles;
  const long long page_blocks = 2ll * B * p.pages * hkv;
  PACE_REQUIRE(row_blocks < (1ll << 31) && page_blocks < (1ll << 31) &&
                   static_cast<long long>(kAppendTokens) * (static_cast<long long>(Hq) + 2 * hkv) * d < (1ll << 31),
               "pace_cache_append: too many sequences, tokens or heads");
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

size_t pace_cache_attention_workspace_size(int n_q, int Hq, int heads, int dim, int B, int max_q, int max_len,
                                           int window, int sinks) {
  if (n_q < 1 || heads < 1 || Hq < heads || Hq % heads != 0 || dim < 1 || B < 1 || max_q < 1 || max_len < 0 ||
      window < 0 || sinks < 0)
    return 0;
  const AttendPlan a = plan_attention(Hq, heads, B, max_q, max_len, window, sinks);
  return a.splits == 1 ? 0 : static_cast<size_t>(a.splits) * n_q * Hq * (dim + 2) * sizeof(float);
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
  if (max_q == 0) return PACE_OK;
  p.q = q; p.cu = cu_q; p.len = seq_len; p.o = o; p.lse = lse;
  p.n_q = n_q; p.Hq = Hq; p.group = Hq / cache->heads; p.B = B; p.max_q = max_q; p.max_len = max_len;
  p.window = window >= max_len ? 0 : window;          // such a window hides nothing
  p.sinks = sinks; p.scale_log2 = scale * kLog2e;
  const AttendPlan a = plan_attention(Hq, cache->heads, B, max_q, max_len, window, sinks);
  PACE_REQUIRE(a.blocks < (1ll << 31) && static_cast<long long>(B) * max_q * Hq < (1ll << 31),
               "pace_cache_attention: too many queries and heads");
  p.row_blocks = a.row_blocks;
  p.splits = a.splits;
  const size_t need = pace_cache_attention_workspace_size(n_q, Hq, cache->heads, cache->dim, B, max_q, max_len, window, sinks);
  if (need) {
    if (workspace == nullptr || workspace_bytes < need)
      return set_error(PACE_ERR_WORKSPACE, "pace_cache_attention: workspace %zu < %zu bytes", workspace_bytes, need);
    PACE_REQUIRE(aligned16(workspace), "pace_cache_attention: workspace must be 16-byte aligned");
    p.part = static_cast<float*>(workspace);
    p.ml = p.part + static_cast<size_t>(a.splits) * n_q * Hq * cache->dim;
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
