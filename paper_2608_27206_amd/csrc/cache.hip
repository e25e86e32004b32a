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
struct AttendParams {
  const uint16_t* q;
  const int32_t *cu, *len;
  uint16_t* o;
  float* lse;
  Pool pool;
  int n_q, Hq, group, B, max_q, max_len, window, sinks;
  float scale_log2;
};

// One workgroup per (query, head), a key per thread and step.
template <int D, int BITS>
__global__ __launch_bounds__(256) void attend(const AttendParams p) {
  __shared__ float qs[D], ps[256], red[4], os[256];
  __shared__ long long at[256];
  int id = blockIdx.x;
  const int h = id % p.Hq;
  id /= p.Hq;
  const int b = id / p.max_q, i = id % p.max_q;
  const int row = p.cu[b] + i, nq = p.cu[b + 1] - p.cu[b];
  if (i >= nq || row < 0 || row >= p.n_q) return;
  int len = p.len[b];
  len = len > p.max_len ? p.max_len : len;
  const int place = len - nq + i, t = threadIdx.x;
  const int hk = h / p.group;
  if (t < D) {
    const uint32_t u = p.q[(static_cast<long long>(row) * p.Hq + h) * D + t];
    qs[t] = __uint_as_float(u << 16) * p.scale_log2;
  }
  constexpr int GR = 256 / D;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  const int dd = t % D, gg = t / D;
  for (int j0 = 0; j0 <= place; j0 += 256) {
    __syncthreads();
    const int j = j0 + t;
    float s = -INFINITY;
    long long off = -1;
    if (j <= place && (p.window == 0 || j > place - p.window || j < p.sinks)) {
      const int pi = j >> p.pool.shift;
      const int pg = pi < p.pool.max_pages ? p.pool.table[static_cast<long long>(b) * p.pool.max_pages + pi] : -1;
      if (pg >= 0 && pg < p.pool.num_pages) {
        const long long ph = static_cast<long long>(pg) * p.pool.heads + hk;
        off = (ph * p.pool.page + (j & (p.pool.page - 1))) * D;
        float a = 0.f;
        for (int d = 0; d < D; ++d) {
          float kv;
          if constexpr (BITS == 16) kv = __uint_as_float(static_cast<uint32_t>(static_cast<uint16_t*>(p.pool.k)[off + d]) << 16);
          else kv = __builtin_amdgcn_cvt_f32_fp8(static_cast<uint8_t*>(p.pool.k)[off + d], 0);
          a += kv * qs[d];
        }
        if constexpr (BITS == 8) a *= p.pool.k_scale[ph];
        s = a;
      }
    }
    at[t] = off;
    const float mt = fmaxf(m, block_reduce<1>(s, red));
    const float mz = mt == -INFINITY ? 0.f : mt;
    const float e = off >= 0 ? exp2f(s - mz) : 0.f;
    const float f = exp2f(m - mz);
    m = mt;
    l = l * f + block_reduce<0>(e, red);
    float w = e;
    if constexpr (BITS == 8) { if (off >= 0) w *= p.pool.v_scale[off / (static_cast<long long>(p.pool.page) * D)]; }
    ps[t] = w;
    __syncthreads();
    acc *= f;
    if (gg < GR)
      for (int k = gg; k < 256; k += GR)
        if (at[k] >= 0) {
          float vv;
          if constexpr (BITS == 16) vv = __uint_as_float(static_cast<uint32_t>(static_cast<uint16_t*>(p.pool.v)[at[k] + dd]) << 16);
          else vv = __builtin_amdgcn_cvt_f32_fp8(static_cast<uint8_t*>(p.pool.v)[at[k] + dd], 0);
          acc += ps[k] * vv;
        }
  }
  os[t] = acc;
  __syncthreads();
  if (t < D) {
    float r = 0.f;
    for (int g = 0; g < GR; ++g) r += os[g * D + t];
    p.o[(static_cast<long long>(row) * p.Hq + h) * D + t] = static_cast<uint16_t>(pack_bf16x2(l > 0.f || l != l ? r / l : 0.f, 0.f));
    if (t == 0 && p.lse) p.lse[static_cast<long long>(h) * p.n_q + row] = l > 0.f || l != l ? (m + log2f(l)) * kLn2 : -INFINITY;
  }
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
  return 0;
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
  p.window = window; p.sinks = sinks; p.scale_log2 = scale * kLog2e;
  const long long blocks = static_cast<long long>(B) * max_q * Hq;
  PACE_REQUIRE(blocks < (1ll << 31), "pace_cache_attention: too many queries and heads");
  if (debug_checks()) {
    try {
      if ((st = debug_attention(p, stream)) != PACE_OK) return st;
    } catch (const std::bad_alloc&) {
      return set_error(PACE_ERR_INVALID_ARG, "pace_cache_attention: no host memory for the debug checks");
    }
  }
  const dim3 g(static_cast<unsigned>(blocks)), th(256);
  if (cache->dim == 128 && cache->bits == 16) hipLaunchKernelGGL((attend<128, 16>), g, th, 0, stream, p);
  else if (cache->dim == 128) hipLaunchKernelGGL((attend<128, 8>), g, th, 0, stream, p);
  else if (cache->bits == 16) hipLaunchKernelGGL((attend<80, 16>), g, th, 0, stream, p);
  else hipLaunchKernelGGL((attend<80, 8>), g, th, 0, stream, p);
  return check_launch("pace_cache_attention");
}

}  // extern "C"
