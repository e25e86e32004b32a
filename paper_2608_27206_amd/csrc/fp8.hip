// A layer's 8-bit operators: rows and weights to OCP e4m3 codes with a scale for each block of 128, the RMS norm with the
// residual's addition in front of it, and the product of such codes with the epilogues of the bf16 product.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "fp8_plan.h"
#include "pace_internal.h"

namespace pace {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kE4m3Max = 448.f;
constexpr float kMinScale = 0x1p-120f;

__device__ __forceinline__ float lo_bf16(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ float bf16_f32(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
__device__ __forceinline__ uint16_t f32_bf16(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return static_cast<uint32_t>(f32_bf16(a)) | static_cast<uint32_t>(f32_bf16(b)) << 16;
}
__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8]) {
  const uint32_t v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = lo_bf16(v[i]);
    x[2 * i + 1] = hi_bf16(v[i]);
  }
}
// x / (1 + e^-x) = x 2^-8 / (2^-8 + 2^(t - 8) e^rest), t = -x log2(e) to a multiple of 2^-13 (from which 8 is taken exactly; t's rounding to
// fp32 alone would cost 2^-18 at x = -20) and rest = -x - t ln 2, under 2^-14.  The factor keeps the denominator in the range, to 2^126,
// whose reciprocals the unit gives.  The exponential and reciprocal units round once each, fp32's ln 2 adds 2^-29 of t: within 2^-20.5 of
// the value (2^-21 for x > -20) down to 2^-120 (x = -88, where the sigmoid becomes subnormal), 2^-16 down to 2^-127 (x = -92.9), where it
// comes as 0.  x / (1 + expf(-x)) would lose everything below x = -88.7.
__device__ __forceinline__ float silu(float x) {
  constexpr float kL = 1.44269504f, kLn2 = 0.693147181f;
  constexpr float kRound = 0x1.8p10f;                                            // fp32 ends at 2^-13 there
  const float c = __builtin_amdgcn_fmed3f(x, -200.f, 200.f);                     // past them e^-x is infinite, or 0 beside 1
  const float r = fmaf(c, -kL, kRound), t = r - kRound, rest = fmaf(t, -kLn2, -c);
  const float d = fmaf(__builtin_amdgcn_exp2f(r - (kRound + 8.f)), 1.f + rest, 0x1p-8f);
  return x * (__builtin_amdgcn_rcpf(d) * 0x1p-8f);
}

// What a value adds to its block's maximum: its magnitude, 0 where it is not finite.
__device__ __forceinline__ float magnitude(float x) { return fabsf(x) <= FLT_MAX ? fabsf(x) : 0.f; }
__device__ __forceinline__ float scale_of(float top) { return fmaxf(top / kE4m3Max, kMinScale); }
// What a block's codes are divided by.  Under 2^-92 both sides of the division grow by 2^64, so that its remainder stays normal.
struct Divisor {
  float scale, inv, up;
};
__device__ __forceinline__ Divisor divisor_of(float scale) {
  const float up = scale < 0x1p-92f ? 0x1p64f : 1.f;
  return {scale * up, 1.f / (scale * up), up};
}
// x / scale in fp32 (-0 stays -0): the product with the reciprocal, put right by its remainder, which one fused multiply-add gives.  For
// every mantissa of the scale this is the rounded quotient of every bf16 value, and of the fp32 values about each middle between two codes
// (2.3e9 quotients compared).  The product alone is another fp32 value for a quarter of the quotients, and another code where one of them is a
// middle.  What is not finite becomes NaN: an infinity's remainder is one (what the conversion makes of infinities depends on a mode bit).
__device__ __forceinline__ float quotient(float x, const Divisor& d) {
  const float a = x * d.up, q = a * d.inv;
  return fmaf(-fmaf(q, d.scale, -a), d.inv, q);
}
// The codes of x / scale: quotients are at most 448 (1 + 2^-23), which rounds to 448.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float e, const Divisor& d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(a, d), quotient(b, d), 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(c, d), quotient(e, d), r, true);
  return static_cast<uint32_t>(r);
}
__device__ __forceinline__ uint2 to_e4m3(const float (&x)[8], const Divisor& d) {
  return make_uint2(to_e4m3(x[0], x[1], x[2], x[3], d), to_e4m3(x[4], x[5], x[6], x[7], d));
}
__device__ __forceinline__ float magnitude8(const float (&x)[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, magnitude(x[i]));
  return m;
}
// The maximum over 16 neighbouring lanes, which hold a block of 128 values.
__device__ __forceinline__ float max16(float x) {
  x = fmaxf(x, dpp_f32<kDppQuadXor1>(x));
  x = fmaxf(x, dpp_f32<kDppQuadXor2>(x));
  x = fmaxf(x, dpp_f32<kDppRowHalfMirror>(x));
  return fmaxf(x, dpp_f32<kDppRowMirror>(x));
}

template <typename T>
bool whole(const T* p) { return reinterpret_cast<uintptr_t>(p) % sizeof(T) == 0; }   // lies at a multiple of its own size

// ---------------------------------------------------------------- quantisation
struct QuantParams {
  const uint16_t* x;
  uint8_t* q;
  float* scale;
  long long stride;
  int M, K, kb;
};

// Rows: scale = max(max |x| / 448, 2^-120), code = x / scale, in one read: 16 lanes hold a block of 128, blocks of a row after
// one another.  Bound by memory: 10,677 x 3,584 moves 115 MB in 23.2 us (4.9 TB/s; a copy reaches 5.1); one row takes 2.1.
__global__ __launch_bounds__(256) void quantize_rows(const QuantParams p) {
  const unsigned block = blockIdx.x * 16 + (threadIdx.x >> 4);   // under 2^28: a launch has fewer than 2^32 threads
  const int row = static_cast<int>(block / static_cast<unsigned>(p.kb)), kb = static_cast<int>(block - static_cast<unsigned>(row) * p.kb);
  if (row >= p.M) return;                              // whole groups of 16 lanes
  const int k = kb * kBlock + (threadIdx.x & 15) * 8;
  float x[8] = {};
  if (k < p.K) unpack8(*reinterpret_cast<const uint4*>(p.x + row * p.stride + k), x);
  const float scale = scale_of(max16(magnitude8(x)));
  if (k < p.K) *reinterpret_cast<uint2*>(p.q + static_cast<long long>(row) * p.K + k) = to_e4m3(x, divisor_of(scale));
  if ((threadIdx.x & 15) == 0) p.scale[static_cast<long long>(kb) * p.M + row] = scale;
}

// Weights: a workgroup per block of 128 x 128, its values in registers between the maximum and the store.  Bound by memory:
// 28,672 x 3,584 moves 308 MB in 66.3 us (4.6 TB/s).
__global__ __launch_bounds__(256) void quantize_blocks(const QuantParams p) {
  __shared__ float red[4];
  const int mb = blockIdx.x / p.kb, kb = blockIdx.x - mb * p.kb;
  const int k = kb * kBlock + (threadIdx.x & 15) * 8, r0 = mb * kBlock + (threadIdx.x >> 4);
  float x[8][8] = {};
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k < p.K && r0 + 16 * i < p.M) unpack8(*reinterpret_cast<const uint4*>(p.x + (r0 + 16 * i) * p.stride + k), x[i]);
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, magnitude8(x[i]));
  const float scale = scale_of(block_reduce<1>(top, red));
  const Divisor d = divisor_of(scale);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k < p.K && r0 + 16 * i < p.M)
      *reinterpret_cast<uint2*>(p.q + static_cast<long long>(r0 + 16 * i) * p.K + k) = to_e4m3(x[i], d);
  if (threadIdx.x == 0) p.scale[blockIdx.x] = scale;
}

// ---------------------------------------------------------------- RMS norm
struct NormParams {
  const uint16_t* x;
  const uint16_t* residual;    // or null
  const float* gamma;
  uint16_t* sum;               // or null
  uint16_t* y;                 // bf16 output, or
  uint8_t* q;                  // codes and
  float* scale;                // [kb, M]
  long long stride, rstride;
  float eps;
  int M, K;
};

// h = x + residual, y = h / sqrt(mean(h^2) + eps) * gamma: T threads a row, which stays in registers (NC pieces of 8
// values a thread), so it is read once; 16 neighbouring lanes hold a block of 128, whose scale needs no more than them.
// Bound by memory: 42,196 rows of 1,280 with the residual to 8 bits move 380 MB in 74 us (5.1 TB/s, the rate of a copy), 10,677
// of 3,584 268 MB in 50 (a wave a row, 64 values a lane: 58).  Few rows are bound by the chain loads -> sum -> norm -> maximum ->
// store (one of 3,584: 3.8 us, 6.6 in a single wave): they take 256 threads each, and gamma comes with the row (GAMMA).
template <int T, int NC, bool GAMMA>
__global__ __launch_bounds__(T < 256 ? 256 : T) void rmsnorm_rows(const NormParams p) {
  constexpr int ROWS = T < 256 ? 256 / T : 1;
  __shared__ float red[T / 64];
  const int t = threadIdx.x % T, row = blockIdx.x * ROWS + threadIdx.x / T;
  if (T == 64 && row >= p.M) return;                   // a wave of its own
  const int pieces = p.K / 8;
  const uint4* x = reinterpret_cast<const uint4*>(p.x + row * p.stride);
  const uint4* r = reinterpret_cast<const uint4*>(p.residual + row * p.rstride);
  uint4 xv[NC], rv[NC];
  float4 gv[GAMMA ? NC : 1][2];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = i * T + t;
    xv[i] = rv[i] = make_uint4(0, 0, 0, 0);
    if (c < pieces) {
      xv[i] = x[c];
      if (p.residual) rv[i] = r[c];
      if constexpr (GAMMA) {
        gv[i][0] = reinterpret_cast<const float4*>(p.gamma)[2 * c];
        gv[i][1] = reinterpret_cast<const float4*>(p.gamma)[2 * c + 1];
      }
    }
  }
  float h[NC][8];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    float add[8];
    unpack8(xv[i], h[i]);
    unpack8(rv[i], add);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] += add[e];
  }
  const auto squares = [&](float by) __attribute__((always_inline)) {     // the sum of the row's (h * by)^2
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) ss = fmaf(h[i][e] * by, h[i][e] * by, ss);
    if constexpr (T == 64) return wave_reduce_dpp(ss, [](float a, float b) { return a + b; });
    else return block_reduce<0>(ss, red);
  };
  // A sum past fp32 is taken again of values 2^-80 times as large: h is under 2^128, so K of their squares stay under 2^112.  One so small
  // that its squares lose bits, where eps is no larger, is taken again of values 2^64 times as large.
  float by = 1.f, ss = squares(1.f);
  if (ss > FLT_MAX || (ss < 0x1p-90f && p.eps < 0x1p-90f)) {             // the same for all of a row's threads
    by = ss > FLT_MAX ? 0x1p-80f : 0x1p64f;
    ss = squares(by);
  }
  const float inv = by / sqrtf(ss / static_cast<float>(p.K) + p.eps * by * by);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = i * T + t;
    if (i * T >= pieces) break;
    const bool in = c < pieces;
    if (in && p.sum)
      reinterpret_cast<uint4*>(p.sum + static_cast<long long>(row) * p.K)[c] =
          make_uint4(pack2(h[i][0], h[i][1]), pack2(h[i][2], h[i][3]), pack2(h[i][4], h[i][5]), pack2(h[i][6], h[i][7]));
    float y[8] = {};
    if (in) {
      const float4 g0 = GAMMA ? gv[GAMMA ? i : 0][0] : reinterpret_cast<const float4*>(p.gamma)[2 * c];
      const float4 g1 = GAMMA ? gv[GAMMA ? i : 0][1] : reinterpret_cast<const float4*>(p.gamma)[2 * c + 1];
      const float g[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = h[i][e] * inv * g[e];
    }
    if (p.y) {
      if (in)
        reinterpret_cast<uint4*>(p.y + static_cast<long long>(row) * p.K)[c] =
            make_uint4(pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7]));
      continue;
    }
    const float scale = scale_of(max16(magnitude8(y)));
    if (in) {
      reinterpret_cast<uint2*>(p.q + static_cast<long long>(row) * p.K)[c] = to_e4m3(y, divisor_of(scale));
      if ((t & 15) == 0) p.scale[static_cast<long long>(c / 16) * p.M + row] = scale;
    }
  }
}
// A wave a row, without a barrier, where it holds few values and there are rows enough to fill the card; a residual doubles the loads that it
// has to hold in flight.  A wave a row and 256 threads a row, captured, one card:
//   1,024 values: with the residual to 8 bits 1,183 rows 5.3 and 5.0 us, 4,096 9.6 and 10.3, 42,196 57.3 and 68.9 (to 16 bits 4.8 and 4.5,
//   8.6 and 8.6, 65.0 and 63.6); without 1,183 3.6 and 3.9, 42,196 33.3 and 56.6;
//   1,280 with the residual to 8 bits: 1,183 rows 6.6 and 5.4, 12,000 28.7 and 26.9, 20,000 40.8 and 42.0, 42,196 74.4 and 83.2; to 16
//   bits 83.1 and 76.8; 1,536 to 8 bits 20,000 rows 47.1 and 44.1;
//   1,280 without: 2,048 rows 5.4 and 5.2, 4,096 7.7 and 8.1, 42,196 43.6 and 63.4; 2,048 4,096 rows 10.5 and 10.2.
// 5,000 x 8,192: 52.8 us with 512 threads, 58.7 with 256, 60.5 with 1,024.
bool wave_a_row(int M, int K, bool residual, bool eight) {
  if (K <= 1024) return M >= 1024;
  return residual ? K <= 1280 && M >= 20000 && eight : K <= 1536 && M >= 4096;
}
template <int T, int NC, bool GAMMA>
void launch_norm(const NormParams& p, hipStream_t stream) {
  constexpr int rows = T < 256 ? 256 / T : 1;
  hipLaunchKernelGGL((rmsnorm_rows<T, NC, GAMMA>), dim3((p.M + rows - 1ll) / rows), dim3(T < 256 ? 256 : T), 0, stream, p);
}

// ---------------------------------------------------------------- product
struct Fp8Params {
  const uint8_t* x;
  const float* xs;             // [kb, M], rows xs_stride apart
  const uint8_t* w;
  const float* ws;             // [nb, kb]
  const float* bias;
  const uint16_t* R;
  void* C;
  float* cs;                   // scales of 8-bit outputs
  float* part;                 // [splits, M, N] sums for fp8_join, or null: the kernel finishes the output
  long long xs_stride, cs_stride;
  int M, N, K, kb, mode, splits, tiles_m, tiles_n;
  int width;                   // elements per access to C and R: 8, 4, 2 or 1 as their alignment allows
};

enum { kEpiBias = 0, kEpiResidual = 1, kEpiSwiglu = 2 };

__device__ __forceinline__ f32x4 mfma128(i32x8 a, i32x8 b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma32(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// A lane's 32 codes of a row and block: as they are, or as bf16 values, exactly.
struct Codes {
  i32x8 v;
};
struct Values {
  bf16x8 v[4];
};
__device__ __forceinline__ bf16x8 widen8(uint32_t a, uint32_t b) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
  return bf16x8{p.x, p.y, q.x, q.y, r.x, r.y, s.x, s.y};
}
__device__ __forceinline__ Codes lift(i32x8 u, Codes*) { return {u}; }
__device__ __forceinline__ Values lift(i32x8 u, Values*) {
  Values o;
#pragma unroll
  for (int q = 0; q < 4; ++q) o.v[q] = widen8(static_cast<uint32_t>(u[2 * q]), static_cast<uint32_t>(u[2 * q + 1]));
  return o;
}
// The sums of a block's 128 products: N rows of x (16 each) with N2 columns of w.
template <int N2, int N>
__device__ __forceinline__ void dot_block(const Codes* w, const Codes (&x)[N], f32x4 (&d)[N2 * N]) {
#pragma unroll
  for (int j = 0; j < N2; ++j)
#pragma unroll
    for (int i = 0; i < N; ++i) d[j * N + i] = mfma128(w[j].v, x[i].v);
}
template <int N2, int N>
__device__ __forceinline__ void dot_block(const Values* w, const Values (&x)[N], f32x4 (&d)[N2 * N]) {
#pragma unroll
  for (int t = 0; t < N2 * N; ++t) d[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int j = 0; j < N2; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) d[j * N + i] = mfma32(w[j].v[q], x[i].v[q], d[j * N + i]);
}
// keeps what has been computed where it stands, between the products of the same step
__device__ __forceinline__ void pin(Codes&) {}
__device__ __forceinline__ void pin(Values& o) {
#pragma unroll
  for (int q = 0; q < 4; ++q) asm volatile("" : "+v"(o.v[q]));
}

typedef __attribute__((address_space(3))) const char lds_char;
constexpr unsigned kOut = 0x7FFFFFF0u;   // an offset past every range: reads as zeros

__device__ __forceinline__ i32x4 rsrc_of(const void* base, unsigned bytes) {
  const unsigned long long a = reinterpret_cast<unsigned long long>(base);
  i32x4 r;
  r.x = __builtin_amdgcn_readfirstlane(static_cast<int>(a & 0xffffffffull));
  r.y = __builtin_amdgcn_readfirstlane(static_cast<int>((a >> 32) & 0xffffull));   // stride 0
  r.z = __builtin_amdgcn_readfirstlane(static_cast<int>(bytes));
  r.w = 0x00020000;
  return r;
}
// 64 lanes x 16 (4) bytes from the buffer to lds .. lds + 1023 (255); untracked by the compiler, awaited with wait_loads.  Nor does the
// compiler see here that a scalar which the vector unit wrote (a spilled descriptor's v_readlane) is read: that needs five wait states.
// build.py looks for them in what it has compiled and ends without them (wait_states.py; s_nop 4 here would cost up to 2%: 982 us for 967).
__device__ __forceinline__ void dma16(i32x4 r, unsigned lds, unsigned voff) {
  const unsigned m0 = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(r), "{m0}"(m0) : "memory");
}
__device__ __forceinline__ void dma4(i32x4 r, unsigned lds, unsigned voff) {
  const unsigned m0 = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff), "s"(r), "{m0}"(m0) : "memory");
}
// all but the last N of the wave's loads have arrived, and its LDS reads have returned
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

template <int W> struct Unit;
template <> struct Unit<8> { typedef uint4 type; };
template <> struct Unit<4> { typedef uint2 type; };
template <> struct Unit<2> { typedef uint32_t type; };
template <> struct Unit<1> { typedef uint16_t type; };
template <typename F>
__device__ __forceinline__ void with_width(int width, F f) {
  if (width == 8) f(std::integral_constant<int, 8>{});
  else if (width == 4) f(std::integral_constant<int, 4>{});
  else if (width == 2) f(std::integral_constant<int, 2>{});
  else f(std::integral_constant<int, 1>{});
}

// The bias of four neighbouring columns.
__device__ __forceinline__ f32x4 bias4(const Fp8Params& p, int n) {
  f32x4 b = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (p.bias && n + e < p.N) b[e] = p.bias[n + e];
  return b;
}

// A wave's part of a tile (rows from m, columns from n) without a residual, from its registers: lanes trade pieces so that each has 8
// neighbouring outputs of a row.  Every load that the wave has asked for has come before the first of them is stored.
__device__ __forceinline__ void trade16(uint32_t& a, uint32_t& b) {
  const auto y = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = y[0];
  b = y[1];
}
__device__ __forceinline__ void trade32(uint32_t& a, uint32_t& b) {
  const auto y = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = y[0];
  b = y[1];
}
// SwiGLU of a lane's part of a row, in elements 0 and 1 of each tile, and the maximum over the wave's part.
template <int NI>
__device__ __forceinline__ float swiglu_tops(f32x4 (&y)[NI]) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < NI; ++j) {
    y[j][0] = silu(y[j][0]) * y[j][1];
    y[j][1] = silu(y[j][2]) * y[j][3];
    top = fmaxf(top, fmaxf(magnitude(y[j][0]), magnitude(y[j][1])));
  }
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  return fmaxf(top, __shfl_xor(top, 32, 64));
}
// 8 bits: the WN waves that share a row hand their maxima on in top_of.
template <int MI, int NI, int WN, int BM>
__device__ __forceinline__ void finish_tile(const Fp8Params& p, f32x4 (&acc)[MI][NI], float (&top_of)[WN][BM], int wm, int m, int n, int r, int g, int wave) {
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const f32x4 b = bias4(p, n + 16 * j + 4 * g);
#pragma unroll
      for (int i = 0; i < MI; ++i) acc[i][j] += b;
    }
  }
  const int rows = p.M - m;                            // N is under 2^20: a tile's offsets hold 32 bits
  if (p.mode == kEpiSwiglu) {
    static_assert(NI == 4, "lane group g ends with the 8 outputs of tile g");
    const int cols = p.N / 2, c = n / 2 + 8 * g;
    if constexpr (WN * NI == 16) {
      if (p.cs) {
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const float top = swiglu_tops<NI>(acc[i]);
          if (g == 0) top_of[wave % WN][wm + 16 * i + r] = top;
          __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
        wait_loads<0>();
        uint8_t* const C = static_cast<uint8_t*>(p.C) + static_cast<long long>(m) * cols;
        float* const cs = p.cs + n / 256 * p.cs_stride + m;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const int row = 16 * i + r;
          float top = top_of[0][wm + row];
#pragma unroll
          for (int o = 1; o < WN; ++o) top = fmaxf(top, top_of[o][wm + row]);
          const float scale = scale_of(top);
          const Divisor d = divisor_of(scale);
          uint32_t a = to_e4m3(acc[i][0][0], acc[i][0][1], acc[i][1][0], acc[i][1][1], d);
          uint32_t b = to_e4m3(acc[i][2][0], acc[i][2][1], acc[i][3][0], acc[i][3][1], d);
          trade32(a, b);
          uint32_t even = (a & 0xffffu) | b << 16, odd = a >> 16 | (b & 0xffff0000u);
          trade16(even, odd);
          const uint2 v = make_uint2((even & 0xffffu) | odd << 16, even >> 16 | (odd & 0xffff0000u));
          if (row < rows && c < cols) *reinterpret_cast<uint2*>(C + static_cast<unsigned>(row * cols + c)) = v;
          if (row < rows && wave % WN == 0 && g == 0) cs[row] = scale;
          __builtin_amdgcn_sched_barrier(0);
        }
        return;
      }
    }
    uint16_t* const C = static_cast<uint16_t*>(p.C) + static_cast<long long>(m) * cols;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      uint32_t u[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) u[j] = pack2(silu(acc[i][j][0]) * acc[i][j][1], silu(acc[i][j][2]) * acc[i][j][3]);
      trade16(u[0], u[1]);
      trade16(u[2], u[3]);
      trade32(u[0], u[2]);
      trade32(u[1], u[3]);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][0][j] = __uint_as_float(u[j]);
      __builtin_amdgcn_sched_barrier(0);
    }
    wait_loads<0>();
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int row = 16 * i + r;
      if (row < rows && c < cols) *reinterpret_cast<f32x4*>(C + static_cast<unsigned>(row * cols + c)) = acc[i][0];
    }
    return;
  }
  const int c = n + 16 * (g & 1) + 8 * (g >> 1);
  uint16_t* const C = static_cast<uint16_t*>(p.C) + static_cast<long long>(m) * p.N;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
#pragma unroll
    for (int j = 0; j < NI; j += 2) {
      uint32_t u[4] = {pack2(acc[i][j][0], acc[i][j][1]), pack2(acc[i][j][2], acc[i][j][3]), pack2(acc[i][j + 1][0], acc[i][j + 1][1]),
                       pack2(acc[i][j + 1][2], acc[i][j + 1][3])};
      trade16(u[0], u[2]);
      trade16(u[1], u[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[i][j][e] = __uint_as_float(u[e]);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  wait_loads<0>();
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; j += 2) {
      const int row = 16 * i + r;
      if (row < rows && c + 16 * j < p.N) *reinterpret_cast<f32x4*>(C + static_cast<unsigned>(row * p.N + c + 16 * j)) = acc[i][j];
    }
}

// C = sum over blocks b of xs[b, m] ws[n / 128, b] (x_b . w_b): a workgroup has a tile of BM rows and BN columns, WM x WN waves with
// MI x NI tiles of 16 x 16 each (G groups of them take blocks in turn and join their sums in LDS).  w is the matrix instruction's
// first operand, so that a lane ends with four neighbouring columns of a row (SwiGLU's pairs in one lane).
//  - A stage is a block of 128 k's: its products need one scale per row (and one per wave for w), applied to the 16 x 16 sums in fp32
//    one unit later, under the next products.  T: Codes multiply as they are, Values after they became bf16 (exactly, under the
//    products, too: 1,373 TFLOP/s instead of 2,985 is what the library reaches, with 32-bit sums).
//  - Operands come straight into LDS, a ring of ST stages, in rows of 128 bytes whose 16-byte chunks are swapped so that fragments
//    are read without conflicts.  A barrier in a stage's middle frees w's part and half of x's, one before its last products the rest.
//  - Bounds: for 256 x 256, the matrix cores' 2,048 cycles a stage against LDS's 192 KB read at 128 bytes a cycle (1,536) and 64 KB
//    written at 64 (1,024); 8 KB more a stage cost 5 to 7%.  So LDS is the busiest part by this count, in smaller tiles more so (1.43 us a stage
//    of 256 x 256, 0.73 of 192 x 128, three eighths of its work): the largest tile that fills the card is best, and what bounds few rows is the
//    weights' bytes.  Four waves of 128 x 128 read a third less, but need 512 registers a lane, half of them beyond the
//    vector unit's reach: 616 us for 8192 cubed against 472.
//  - With few tiles, K goes to workgroups (`part`, fp8_join) or to G groups in one.  Measured, a call: 10,677 x 28,672 x 3,584 with
//    SwiGLU 967 us (2,270 TFLOP/s), its 8-bit output in wide sums 1,717 (1,278), 1,183 x 3,584 x 3,584 with a residual 27 (1,126),
//    48 x 3,584 x 14,336 14 with the join (3.6 TB/s), 8 x 28,672 x 3,584 24 (4.3).
//  - RUN: a workgroup takes one tile after another.  The last ST stages ask for the next tile's first ones, and the output
//    leaves from registers, since LDS already holds those.
template <typename T, int MI, int NI, int WM, int WN, int ST, int G, bool RUN>
__global__ __launch_bounds__(64 * WM * WN * G, 2) void gemm_fp8_tile(const Fp8Params p) {
  constexpr int BM = 16 * MI * WM, BN = 16 * NI * WN, NW = WM * WN, TH = 64 * NW * G;
  constexpr int kScales = (BM + 63) / 64 * 64;                   // floats of a stage, whole DMAs of them
  constexpr int kStage = (BM + BN) * kBlock;                     // bytes of a stage
  constexpr int kScaleSlots = ST + 1;
  constexpr bool kWide = sizeof(T) != sizeof(Codes), kAhead = kWide && NI % 2 == 0 && MI % 2 == 0;
  constexpr int MP = MI % 2 || kAhead ? 1 : 2, Q = MI / MP;      // tiles of x in a step, steps of a stage
  constexpr int JP = MP == 1 && NI % 2 == 0 ? 2 : 1, NU = NI / JP;   // tiles of w in a unit, units of a step
  // DMAs of a wave and stage, 8 rows each: the first part (w's rows, those of x that the first half of the steps reads, and the
  // scales) is asked for in mid-stage, the second at the end
  constexpr bool kTwo = Q % 4 == 0;
  constexpr bool kWhole = !kWide && G > 1 && 16 * (MI + NI) + 4 * MI * NI <= 128;
  constexpr int kWD = BN / 8 / NW, kXD = BM / 8 / NW, kLate = kTwo ? kXD / 2 : 0, kEarly = kWD + kXD - kLate + 1;
  static_assert(kWD * 8 * NW == BN && kXD * 8 * NW == BM && (!kTwo || kXD % 2 == 0) && NW % 2 == 0 && kBlock % (16 * NI) == 0 && kScales / 64 <= NW, "tile");
  constexpr int kRing = ST * G * kStage, kTile = BM * BN * 2, kJoin = (G - 1) * BM * BN * 4, kBoth = kTile > kJoin ? kTile : kJoin;
  __shared__ __align__(16) char lds[kRing > kBoth ? kRing : kBoth];
  __shared__ float scales[kScaleSlots * G][kScales];
  __shared__ float top_of[WN][BM];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), w = wave % NW, kg = wave / NW;
  const int r = lane & 15, g = lane >> 4;
  const int wm = (w / WN) * 16 * MI, wn = (w % WN) * 16 * NI;
  // XCD-contiguous order; groups of eight row tiles column by column, so that the workgroups that run together on an XCD
  // share a few rows of x and a few of w in its L2; few columns row by row (42,196 x 1,280 x 3,424, five across: 223 us; in eights,
  // of which an XCD holds one and a part, 228)
  const int per = p.tiles_m * p.tiles_n;
  const int lb = remap_block_id(blockIdx.x, gridDim.x);
  const int split = lb / per;
  int bm, bn, rows_m;                                  // the tile whose operands are asked for
  i32x4 ra, rb;
  const auto take = [&](int tl) __attribute__((always_inline)) {
    const int high = p.tiles_n < 8 ? 1 : 8, gsz = high * p.tiles_n, grp = tl / gsz, in = tl - grp * gsz;
    const int gm = min(high, p.tiles_m - high * grp);
    const int tn = in / gm, tm = high * grp + (in - tn * gm);
    bm = tm * BM;
    bn = tn * BN;
    rows_m = min(BM, p.M - bm);
    ra = rsrc_of(p.x + static_cast<long long>(bm) * p.K, static_cast<unsigned>(rows_m) * p.K);
    rb = rsrc_of(p.w + static_cast<long long>(bn) * p.K, static_cast<unsigned>(min(BN, p.N - bn)) * p.K);
  };
  take(lb - split * per);
  const int t0 = static_cast<int>(static_cast<long long>(p.kb) * split / p.splits);
  const int t1 = static_cast<int>(static_cast<long long>(p.kb) * (split + 1) / p.splits);
  const int nk = (t1 - t0 + G - 1) / G;                // stages; a group of waves takes block t0 + G * stage + its number
  const auto block_of = [&](int stage) { return t0 + G * stage + kg; };
  const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<unsigned long long>((lds_char*)(const void*)lds));

  // A DMA brings 8 rows; chunk c (16 bytes) of row r lies in slot c ^ ((r >> 1) & 7)
  const int r8 = lane >> 3, kc = ((lane & 7) ^ (4 * (w & 1) + (r8 >> 1))) * 16;
  unsigned off0 = static_cast<unsigned>(r8) * p.K + kc;
  const int k_end = min(p.K, t1 * kBlock);
  // A residual tile takes the place of the blocks after the last one: it is in LDS, laid out as the epilogue reads it, when
  // the last products are done (read there it cost a round of 256 x 256 tiles 15 us).
  const bool ring_r = G == 1 && !RUN && p.mode == kEpiResidual && !p.part && p.width == 8 && p.N < (1 << 20) && nk >= ST;
  constexpr int kCh = BN / 8;                                    // chunks of 8 values of a tile's row of 16 bits
  const i32x4 rr = ring_r ? rsrc_of(p.R + static_cast<long long>(bm) * p.N, static_cast<unsigned>(rows_m) * p.N * 2) : ra;
  const auto residual8 = [&](int lds_row, int buf) __attribute__((always_inline)) {
    const int at = buf * kStage + lds_row * kBlock, row = at / (BN * 2) + lane / kCh;      // 1,024 bytes: 512 / BN rows
    const int n = bn + ((lane % kCh) ^ (row & (kCh - 1))) * 8;
    dma16(rr, lds0 + at, at < kTile && row < rows_m && n < p.N ? (static_cast<unsigned>(row) * p.N + n) * 2u : kOut);
  };
  const auto rows8 = [&](const i32x4& rs, int row, int lds_row, int t, int buf, bool in_k, auto tail) __attribute__((always_inline)) {
    if constexpr (decltype(tail)::value) {
      if (ring_r && t >= t1) {
        residual8(lds_row, buf);
        return;
      }
    }
    // rows past the end lie past the buffer's range
    dma16(rs, lds0 + (buf * G + kg) * kStage + lds_row * kBlock, in_k ? off0 + static_cast<unsigned>(row) * p.K + t * kBlock : kOut);
  };
  // x's rows of 8 that wave w brings as its u-th: the first half of them is what the first half of the steps reads
  const auto x_row = [&](int u) __attribute__((always_inline)) {
    if constexpr (kTwo) {
      const int i = w + NW * (u % (kXD / 2));            // of BM / 16; a half of a wave's rows are MI of them
      return i / MI * (16 * MI) + u / (kXD / 2) * (8 * MI) + i % MI * 8;
    } else {
      return 8 * (w + NW * u);
    }
  };
  // DMA u of the stage's first part, and of its second
  const auto load_early = [&](int u, int t, int buf, int slot, auto tail) __attribute__((always_inline)) {
    const bool in_k = t * kBlock + kc < k_end;             // past the end of K, or of the part: zeros
    if (u < kWD) {
      rows8(rb, 8 * (w + NW * u), BM + 8 * (w + NW * u), t, buf, in_k, tail);
    } else if (u < kEarly - 1) {
      rows8(ra, x_row(u - kWD), x_row(u - kWD), t, buf, in_k, tail);
    } else {
      const int s = w % (kScales / 64) * 64;            // more waves than pieces: the same again
      dma4(rsrc_of(p.xs + t * p.xs_stride + bm, static_cast<unsigned>(rows_m) * 4),
           static_cast<unsigned>(reinterpret_cast<unsigned long long>((lds_char*)(const void*)&scales[0][0])) + ((slot * G + kg) * kScales + s) * 4,
           t < t1 ? static_cast<unsigned>(s + lane) * 4 : kOut);
    }
  };
  const auto load_late = [&](int u, int t, int buf, auto tail) __attribute__((always_inline)) {
    rows8(ra, x_row(kXD - kLate + u), x_row(kXD - kLate + u), t, buf, t * kBlock + kc < k_end, tail);
  };
  // fragments: a lane has chunks g and g + 4 of row r
  int at0 = r * kBlock + ((g ^ (r >> 1)) & 7) * 16;
  const auto frag = [&](int buf, int row) __attribute__((always_inline)) {
    const char* st = lds + (buf * G + kg) * kStage + row * kBlock;
    const i32x4 a = *reinterpret_cast<const i32x4*>(st + at0), b = *reinterpret_cast<const i32x4*>(st + (at0 ^ 64));
    return i32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  };
  const auto x_scale = [&](int slot, int i) __attribute__((always_inline)) { return scales[slot * G + kg][wm + 16 * i + r]; };
  // w's scales: one for the wave and block, 64 blocks in a register's lanes
  const auto scales_of = [&](int n0, int b) __attribute__((always_inline)) {
    const int nb = min(n0 + wn, p.N - 1) / kBlock;
    return b < p.kb ? p.ws[static_cast<long long>(nb) * p.kb + b] : 0.f;
  };
  int to_m = bm, to_n = bn;                            // the tile whose products are formed
  float wscales = 0.f;

  f32x4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const auto scales_from = [&](int stage) __attribute__((always_inline)) {
    wscales = scales_of(to_n, block_of(stage + lane));
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(wscales));   // now, and not at every use for all loads in flight
  };
  scales_from(0);
#pragma unroll
  for (int s = 0; s < ST; ++s) {
#pragma unroll
    for (int u = 0; u < kEarly; ++u) load_early(u, block_of(s), s, s, std::false_type{});
#pragma unroll
    for (int u = 0; u < kLate; ++u) load_late(u, block_of(s), s, std::false_type{});
  }
  wait_loads<RUN ? 0 : (ST - 1) * (kEarly + kLate)>();
  barrier();

  int cur = 0, cs = 0;                                 // the stage's buffer and scales
  if constexpr (kWhole) {
    // Both operands of a stage are in registers before it begins: the next stage's are read under its products, and the stage
    // opens with the one meeting at which its own buffer is free and the next one full.
    constexpr int JW = NI % 2 == 0 ? 2 : 1, U = MI * NI / 2, kReads = MI + NI, kReadIn = U > 2 ? U * 3 / 4 : U;
    T wf[2][NI];
    T xf[2][MI];
    float xsc[2][MI];
    T* const kind = nullptr;
    const auto read = [&](int l, auto to, int buf, int slot) __attribute__((always_inline)) {
      constexpr int P = decltype(to)::value;
      if (l < NI) {
        wf[P][l] = lift(frag(buf, BM + wn + 16 * l), kind);
      } else {
        xf[P][l - NI] = lift(frag(buf, wm + 16 * (l - NI)), kind);
        xsc[P][l - NI] = x_scale(slot, l - NI);
      }
    };
#pragma unroll
    for (int l = 0; l < kReads; ++l) read(l, std::integral_constant<int, 0>{}, 0, 0);
    // What a unit (two products) has formed goes into acc in the next one, under its products.
    f32x4 d[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
    float ds[2] = {0.f, 0.f};
    const auto add = [&](int u) __attribute__((always_inline)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f32x4& to = JW == 2 ? acc[u / (NI / JW)][u % (NI / JW) * 2 + t] : acc[2 * u + t][0];
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = fmaf(ds[t], d[t][e], to[e]);
        asm volatile("" : "+v"(to));                   // here, not behind the stage's branches
      }
    };
    const auto stage = [&](int k, auto from) __attribute__((always_inline)) {
      constexpr int P = decltype(from)::value;
      const int nxt = cur == ST - 1 ? 0 : cur + 1, ns = cs == kScaleSlots - 1 ? 0 : cs + 1, far = cs == 0 ? kScaleSlots - 1 : cs - 1;
      const float sw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wscales), k & 63));
      wait_loads<(ST - 2) * kEarly>();                 // the next stage has come, and this one's reads
      barrier();
#pragma unroll
      for (int u = 0; u < U; ++u) {
        f32x4 c[2];
        float s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int i = JW == 2 ? u / (NI / JW) : 2 * u + t, j = JW == 2 ? u % (NI / JW) * 2 + t : 0;
          c[t] = mfma128(wf[P][j].v, xf[P][i].v);
          s[t] = xsc[P][i] * sw;
        }
        add(u ? u - 1 : U - 1);
        // past the end of K the reads bring anything, and nothing uses it
#pragma unroll
        for (int l = 0; l < kReads; ++l)
          if (l * kReadIn / kReads == u) read(l, std::integral_constant<int, 1 - P>{}, nxt, ns);
#pragma unroll
        for (int l = 0; l < kEarly; ++l)
          if (l * U / kEarly == u) load_early(l, block_of(k + ST), cur, far, std::false_type{});
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          d[t] = c[t];
          ds[t] = s[t];
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);             // this unit's products first,
        __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);             // the sums of the one before under them
        __builtin_amdgcn_sched_barrier(0);
      }
      if ((k & 63) == 63 && k + 1 < nk) scales_from(k + 1);
      cur = nxt;
      cs = ns;
    };
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    int k = 0;
    for (; k + 1 < nk; k += 2) {
      stage(k, even);
      stage(k + 1, odd);
    }
    if (k < nk) stage(k, even);
    add(U - 1);
  } else {
    T* const kind = nullptr;
    T wf[NI], xa[MP];
    i32x8 xr[2][MP];
    float xsc[2][MP];
    const auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < NI; ++j) wf[j] = lift(frag(cur, BM + wn + 16 * j), kind);
#pragma unroll
      for (int i = 0; i < MP; ++i) {
        xr[0][i] = frag(cur, wm + 16 * i);
        xsc[0][i] = x_scale(cs, i);
        if (kAhead) xa[i] = lift(xr[0][i], kind);
      }
    };
    begin();
    // What a unit of products has formed goes into acc in the next one, under its products.
    f32x4 d[JP * MP];
    float ds[MP];
#pragma unroll
    for (int i = 0; i < MP; ++i) ds[i] = 0.f;
#pragma unroll
    for (int t = 0; t < JP * MP; ++t) d[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto add = [&](int q, int u) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < JP; ++j)
#pragma unroll
        for (int i = 0; i < MP; ++i) {
          f32x4& to = acc[q * MP + i][u * JP + j];
#pragma unroll
          for (int e = 0; e < 4; ++e) to[e] = fmaf(ds[i], d[j * MP + i][e], to[e]);
          asm volatile("" : "+v"(to));                   // here, not behind the stage's branches
        }
    };
    // Stage k: its first fragments are in registers.  Before its last step a wave, which then holds the last fragments, meets
    // the others; what is left of the stage's buffer takes stage k + ST, and the last products run under the first reads of
    // stage k + 1.  With four steps they meet in mid-stage too: then every wave holds w's rows and has read half of x's.
    // RUN: `ask` is the block that is asked for, perhaps of the next tile, whose first ST stages have come before this one's
    // output left (FRESH: of the first ST stages, 1 and 2, all but the last know the next stage to be there; the last stage, 3, leaves
    // the next one's fragments in LDS).
    int ask = 0;
    const auto stage = [&](int k, auto tail, auto fresh) __attribute__((always_inline)) {
      constexpr int FRESH = decltype(fresh)::value;
      const auto far_block = [&] { return RUN ? ask : block_of(k + ST); };
      const int nxt = cur == ST - 1 ? 0 : cur + 1, ns = cs == kScaleSlots - 1 ? 0 : cs + 1, far = cs == 0 ? kScaleSlots - 1 : cs - 1;
      const float sw = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(wscales), k & 63));
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const bool last = q == Q - 1;
        const int slot = q & 1, next_slot = last ? 0 : (q + 1) & 1;
        float s[MP];
        if (kTwo && q == Q / 2 - 1) {
          // this stage's second part has come; in flight are the stages after it
          if constexpr (FRESH == 1 || FRESH == 2) wait_reads();
          else wait_loads<(ST - 1) * (kEarly + kLate)>();
          barrier();
        }
        if (last) {
          // the next stage's first part has come
          if constexpr (FRESH == 1) wait_reads();
          else wait_loads<(ST - 2) * (kEarly + kLate) + (kTwo ? kLate + kEarly : 0)>();
          barrier();
        }
#pragma unroll
        for (int i = 0; i < MP; ++i) {
          if (!kAhead) xa[i] = lift(xr[slot][i], kind);
          s[i] = xsc[slot][i] * sw;
        }
        // past the end of K the reads bring anything, and nothing uses it
#pragma unroll
        for (int i = 0; i < MP; ++i) {
          if (last && FRESH == 3) break;
          xr[next_slot][i] = frag(last ? nxt : cur, wm + 16 * (last ? i : (q + 1) * MP + i));
          xsc[next_slot][i] = x_scale(last ? ns : cs, last ? i : (q + 1) * MP + i);
        }
        i32x8 wr[2 * JP];                                // the next stage's w before it is widened
        T xn[MP];
        const bool ahead = last && FRESH != 3;
        if (ahead && kWide) {
#pragma unroll
          for (int j = 0; j < JP; ++j) wr[j] = frag(nxt, BM + wn + 16 * j);
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          f32x4 c[JP * MP];
          dot_block<JP>(&wf[u * JP], xa, c);
          if (ahead && kWide && u + 1 < NU) {
#pragma unroll
            for (int j = 0; j < JP; ++j) wr[((u + 1) & 1) * JP + j] = frag(nxt, BM + wn + 16 * ((u + 1) * JP + j));
          }
          if (u) add(q, u - 1);
          else add(q ? q - 1 : Q - 1, NU - 1);
          // what the barriers have freed is asked for a piece at a time, behind the step's reads and under its products
          constexpr int kSlots = kTwo ? (Q / 2) * NU : NU, kFirst = kTwo ? Q / 2 - 1 : Q - 1;
          const int at = (q - kFirst) * NU + u;
          if (at >= 0 && at < kSlots) {
#pragma unroll
            for (int l = 0; l < kEarly; ++l)
              if (l * kSlots / kEarly == at) load_early(l, far_block(), cur, far, tail);
          }
          if (last) {
#pragma unroll
            for (int l = 0; l < kLate; ++l)
              if (l * NU / (kLate ? kLate : 1) == u) load_late(l, far_block(), cur, tail);
          }
          // the next step's x and the next stage's w are widened under the products, too
          if (kAhead && u == NU - 1 && (!last || ahead)) {
#pragma unroll
            for (int i = 0; i < MP; ++i) {
              xn[i] = lift(xr[next_slot][i], kind);
              pin(xn[i]);
            }
          }
          if (ahead) {
#pragma unroll
            for (int j = 0; j < JP; ++j) {
              T& to = wf[u * JP + j];
              if constexpr (kWide) to = lift(wr[(u & 1) * JP + j], kind);
              else to = lift(frag(nxt, BM + wn + 16 * (u * JP + j)), kind);
              pin(to);
            }
          }
#pragma unroll
          for (int t = 0; t < JP * MP; ++t) d[t] = c[t];
#pragma unroll
          for (int i = 0; i < MP; ++i) ds[i] = s[i];
          if constexpr (kWide) {
            const int each = 1 + (kAhead && u == NU - 1 ? 2 : 0) + (last ? 4 : 0) + (kAhead ? 0 : 2);   // VALU work for each product
#pragma unroll
            for (int t = 0; t < 4 * JP * MP; ++t) {
              __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
              if (each == 1) __builtin_amdgcn_sched_group_barrier(0x002, 1, 0);
              else if (each == 3) __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
              else if (each == 5) __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
              else __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
            }
          } else {
            __builtin_amdgcn_sched_group_barrier(0x008, JP * MP, 0);     // this unit's products first,
            __builtin_amdgcn_sched_group_barrier(0x002, 4 * JP * MP, 0); // the sums of the one before under them
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (kAhead && (!last || ahead)) {
#pragma unroll
          for (int i = 0; i < MP; ++i) xa[i] = xn[i];
        }
      }
      if ((k & 63) == 63 && k + 1 < nk) scales_from(k + 1);
      cur = nxt;
      cs = ns;
    };
    const std::integral_constant<int, 0> plain;
    if constexpr (RUN) {
      const std::integral_constant<int, 1> first;
      const std::integral_constant<int, 2> second;
      const std::integral_constant<int, 3> end;
      for (int done = gridDim.x;; done += gridDim.x) {
        to_m = bm;
        to_n = bn;
        int to_r = r, to_g = g;
        asm volatile("" : "+v"(off0), "+v"(at0), "+v"(to_r), "+v"(to_g));   // addresses formed anew, not kept while the output leaves
        for (int k = 0; k < ST - 1; ++k) {
          ask = k + ST;
          stage(k, std::false_type{}, first);
        }
        ask = 2 * ST - 1;
        stage(ST - 1, std::false_type{}, second);
        for (int k = ST; k < nk - ST; ++k) {
          ask = k + ST;
          stage(k, std::false_type{}, plain);
        }
        // the operands of the workgroup's next tile, or nothing
        const int left = min(per - done, static_cast<int>(gridDim.x));
        const bool more = static_cast<int>(blockIdx.x) < left;
        if (more) {
          take(done + remap_block_id(blockIdx.x, left));
        } else {
          rows_m = 0;
          ra.z = rb.z = 0;
        }
        float next = scales_of(bn, lane);
        for (int k = nk - ST; k < nk - 1; ++k) {
          ask = k + ST - nk;
          stage(k, std::false_type{}, plain);
        }
        ask = ST - 1;
        stage(nk - 1, std::false_type{}, end);
        add(Q - 1, NU - 1);
        finish_tile<MI, NI, WN, BM>(p, acc, top_of, wm, to_m + wm, to_n + wn, to_r, to_g, w);
        if (!more) return;
        asm volatile("" : "+v"(next));
        wscales = next;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < MP; ++i) ds[i] = 0.f;
#pragma unroll
        for (int t = 0; t < JP * MP; ++t) d[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        begin();
      }
    }
    int k = 0;
    if constexpr (G == 1) {
      for (; k < nk - ST; ++k) stage(k, std::false_type{}, plain);
      for (; k < nk; ++k) stage(k, std::true_type{}, plain);
    } else {
      for (; k < nk; ++k) stage(k, std::false_type{}, plain);
    }
    add(Q - 1, NU - 1);
  }
  wait_loads<0>();                                     // those past the end: the epilogue uses the same LDS
  if constexpr (G > 1) {
    __syncthreads();
    f32x4* from = reinterpret_cast<f32x4*>(lds) + w * (MI * NI * 64) + lane;   // each group's tile after the other's
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j)
        if (kg) from[(kg - 1) * (BM * BN / 4) + (i * NI + j) * 64] = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int o = 0; o < G - 1; ++o)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
          if (!kg) acc[i][j] += from[o * (BM * BN / 4) + (i * NI + j) * 64];
  }

  // epilogue: element e of tile (i, j) is row wm + 16 i + r, column wn + 16 j + 4 g + e
  if (p.part) {
    if (kg) return;
    float* part = p.part + static_cast<long long>(split) * p.M * p.N;
    const bool whole = p.N % 4 == 0;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int m = bm + wm + 16 * i + r;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int n = bn + wn + 16 * j + 4 * g;
        if (m >= p.M || n >= p.N) continue;
        float* to = part + static_cast<long long>(m) * p.N + n;
        if (whole) *reinterpret_cast<f32x4*>(to) = acc[i][j];
        else
          for (int e = 0; e < 4; ++e)
            if (n + e < p.N) to[e] = acc[i][j][e];
      }
    }
    return;
  }
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const f32x4 b = bias4(p, bn + wn + 16 * j + 4 * g);
#pragma unroll
      for (int i = 0; i < MI; ++i) acc[i][j] += b;
    }
  }
  __syncthreads();                                     // every wave has read its last stage
  const int mode = p.mode;
  if constexpr (BN == 256) {
    if (p.cs) {
      // SwiGLU to 8 bits: the tile's 128 outputs of a row are a block
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (kg) break;
        const float top = swiglu_tops<NI>(acc[i]);
        if (g == 0) top_of[w % WN][wm + 16 * i + r] = top;
      }
      __syncthreads();
      const auto row_scale = [&](int row) {
        float top = top_of[0][row];
#pragma unroll
        for (int c = 1; c < WN; ++c) top = fmaxf(top, top_of[c][row]);
        return scale_of(top);
      };
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (kg) break;
        const int row = wm + 16 * i + r;
        const Divisor d = divisor_of(row_scale(row));
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          const int c = (wn + 16 * j + 4 * g) / 2;
          *reinterpret_cast<uint16_t*>(lds + row * 128 + (((c >> 4) ^ (row & 7)) << 4) + (c & 15)) =
              static_cast<uint16_t>(to_e4m3(acc[i][j][0], acc[i][j][1], 0.f, 0.f, d));
        }
      }
      __syncthreads();
      const int cols = p.N / 2;
      uint8_t* C = static_cast<uint8_t*>(p.C);
      for (int c = tid; c < BM * 8; c += TH) {
        const int row = c >> 3, ch = c & 7, m = bm + row, n = bn / 2 + 16 * ch;
        if (m < p.M && n < cols)
          *reinterpret_cast<uint4*>(C + static_cast<long long>(m) * cols + n) = *reinterpret_cast<const uint4*>(lds + row * 128 + ((ch ^ (row & 7)) << 4));
      }
      for (int row = tid; row < rows_m; row += TH) p.cs[bn / 256 * p.cs_stride + bm + row] = row_scale(row);
      return;
    }
  }
  // 16 bits: the tile goes through LDS, 16-byte chunk ch of row i in slot ch ^ (i mod the chunks of a row), so that rows leave
  // in whole lines; a residual tile comes in the same way first
  uint16_t* tile = reinterpret_cast<uint16_t*>(lds);
  if (mode == kEpiResidual && !ring_r) {
    with_width(p.width, [&](auto WC) __attribute__((always_inline)) {
      constexpr int W = decltype(WC)::value, kUnits = BN / W;
      typedef typename Unit<W>::type U;
#pragma unroll 8
      for (int c = tid; c < BM * kUnits; c += TH) {
        const int row = c / kUnits, cl = c % kUnits * W;
        U v{};
        if (bm + row < p.M && bn + cl < p.N)
          v = *reinterpret_cast<const U*>(p.R + static_cast<long long>(bm + row) * p.N + bn + cl);
        *reinterpret_cast<U*>(&tile[row * BN + (((cl >> 3) ^ (row & (kCh - 1))) << 3) + (cl & 7)]) = v;
      }
    });
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    if (kg) break;
    const int row = wm + 16 * i + r;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int cl = wn + 16 * j + 4 * g;
      if (mode == kEpiSwiglu) {
        const int cg = cl >> 1;
        *reinterpret_cast<uint32_t*>(&tile[row * (BN / 2) + (((cg >> 3) ^ (row & (kCh / 2 - 1))) << 3) + (cg & 7)]) =
            pack2(silu(acc[i][j][0]) * acc[i][j][1], silu(acc[i][j][2]) * acc[i][j][3]);
      } else {
        uint2* at = reinterpret_cast<uint2*>(&tile[row * BN + (((cl >> 3) ^ (row & (kCh - 1))) << 3) + (cl & 7)]);
        f32x4 v = acc[i][j];
        if (mode == kEpiResidual) {
          const uint2 u = *at;
          v += f32x4{lo_bf16(u.x), hi_bf16(u.x), lo_bf16(u.y), hi_bf16(u.y)};
        }
        *at = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
      }
    }
  }
  __syncthreads();
  const bool glu = mode == kEpiSwiglu;
  const int cols = glu ? p.N / 2 : p.N, c0 = glu ? bn / 2 : bn;
  const int cpr = glu ? kCh / 2 : kCh, cbits = __builtin_ctz(cpr);
  uint16_t* C = static_cast<uint16_t*>(p.C);
  with_width(p.width, [&](auto WC) __attribute__((always_inline)) {
    constexpr int W = decltype(WC)::value, kLog = W == 8 ? 0 : W == 4 ? 1 : W == 2 ? 2 : 3;   // log2 of 8 / W
    typedef typename Unit<W>::type U;
    const int ubits = cbits + kLog;
    for (int c = tid; c < BM << ubits; c += TH) {
      const int row = c >> ubits, u = c & ((1 << ubits) - 1), ch = u >> kLog;
      const int m = bm + row, n = c0 + u * W;
      if (m >= p.M || n >= cols) continue;
      *reinterpret_cast<U*>(C + static_cast<long long>(m) * cols + n) =
          *reinterpret_cast<const U*>(&tile[(row * cpr + (ch ^ (row & (cpr - 1)))) * 8 + (u & (8 / W - 1)) * W]);
    }
  });
}

// Four neighbouring columns (fewer at the row's end) of a row from their finished sums: bias, residual or SwiGLU, 16 bits.
__device__ __forceinline__ void finish4(const Fp8Params& p, int m, int n, f32x4 y, f32x4 bias) {
  const bool whole = p.N % 4 == 0;
  y += bias;
  uint16_t* C = static_cast<uint16_t*>(p.C);
  if (p.mode == kEpiSwiglu) {
    uint16_t* to = C + static_cast<long long>(m) * (p.N / 2) + n / 2;
    to[0] = f32_bf16(silu(y[0]) * y[1]);
    if (n + 2 < p.N) to[1] = f32_bf16(silu(y[2]) * y[3]);
    return;
  }
  const long long at = static_cast<long long>(m) * p.N + n;
  if (whole && p.width >= 4) {
    if (p.mode == kEpiResidual) {
      const uint2 u = *reinterpret_cast<const uint2*>(p.R + at);
      y += f32x4{lo_bf16(u.x), hi_bf16(u.x), lo_bf16(u.y), hi_bf16(u.y)};
    }
    *reinterpret_cast<uint2*>(C + at) = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < p.N) C[at + e] = f32_bf16(p.mode == kEpiResidual ? y[e] + bf16_f32(p.R[at + e]) : y[e]);
}
__device__ __forceinline__ void store4(const Fp8Params& p, float* to, int n, f32x4 y) {
  if (p.N % 4 == 0) *reinterpret_cast<f32x4*>(to) = y;
  else
    for (int e = 0; e < 4; ++e)
      if (n + e < p.N) to[e] = y[e];
}

// Up to 16 rows: bound by the weights' bytes (one row of 4,608 x 3,584 7.0 us; 16.5 MB at the rate of a copy 3.2, the rest the chain of
// launch, four blocks a wave, and join; three or four blocks in flight and 16 waves gave nothing).  A workgroup's 8 waves share 16 columns and take the blocks of K in turn; a
// wave keeps two blocks in flight.  The codes become bf16 values, whose products the matrix cores sum in 32 bits.
__global__ __launch_bounds__(64 * kFewWaves, 2) void gemm_fp8_few(const Fp8Params p) {
  constexpr int W = kFewWaves, D = 2;
  __shared__ f32x4 join[W - 1][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int n0 = remap_block_id(blockIdx.x, gridDim.x) * 16;
  const int n = n0 + r < p.N ? n0 + r : p.N - 1;
  const uint8_t* wrow = p.w + static_cast<long long>(n) * p.K + 16 * g;
  const uint8_t* xrow = p.x + static_cast<long long>(r < p.M ? r : 0) * p.K + 16 * g;
  const float* ws = p.ws + static_cast<long long>(min(n0, p.N - 1) / kBlock) * p.kb;
  struct {
    u32x4 w[2], x[2];
    float xs, ws;
  } in[D];
  const auto load = [&](int i, int b) __attribute__((always_inline)) {
    const int k = b * kBlock;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      in[i].w[u] = in[i].x[u] = u32x4{0, 0, 0, 0};
      if (k + 64 * u + 16 * g >= p.K) continue;
      in[i].w[u] = *reinterpret_cast<const u32x4*>(wrow + k + 64 * u);
      if (r < p.M) in[i].x[u] = *reinterpret_cast<const u32x4*>(xrow + k + 64 * u);
    }
    in[i].xs = r < p.M ? p.xs[b * p.xs_stride + r] : 0.f;
    in[i].ws = ws[b];
  };
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < D; ++i)
    if (w + i * W < p.kb) load(i, w + i * W);
  f32x4 bias = {0.f, 0.f, 0.f, 0.f};                   // beside the weights: behind them it would be a wait of its own
  if (!p.part && w == 0) bias = bias4(p, n0 + 4 * g);
  for (int b0 = w; b0 < p.kb; b0 += D * W) {
#pragma unroll
    for (int i = 0; i < D; ++i) {
      const int b = b0 + i * W;
      if (b >= p.kb) break;
      f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          d = mfma32(widen8(in[i].w[u][2 * h], in[i].w[u][2 * h + 1]), widen8(in[i].x[u][2 * h], in[i].x[u][2 * h + 1]), d);
      const float s = in[i].xs * in[i].ws;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = fmaf(s, d[e], acc[e]);
      if (b + D * W < p.kb) load(i, b + D * W);
    }
  }
  if (w) join[w - 1][lane] = acc;
  __syncthreads();
  if (w) return;
#pragma unroll
  for (int i = 0; i < W - 1; ++i) acc += join[i][lane];
  const int at = n0 + 4 * g;
  if (r >= p.M || at >= p.N) return;
  if (p.part) store4(p, p.part + static_cast<long long>(r) * p.N + at, at, acc);
  else finish4(p, r, at, acc, bias);
}

// Adds the parts of a split K in their order and finishes the output, four columns a thread: 3.4 to 4.8 us with the launch for up to 3 MB
// of sums.  With 8 bits a wave has the 256
// columns of a block.
__global__ __launch_bounds__(256) void fp8_join(const Fp8Params p) {
  const int cols = (p.N + 1023) / 1024;
  const int m = blockIdx.x / cols, n = ((blockIdx.x - m * cols) * 256 + threadIdx.x) * 4;
  if (n >= p.N && !p.cs) return;
  const f32x4 bias = bias4(p, n);
  const float* from = p.part + static_cast<long long>(m) * p.N + n;
  const long long step = static_cast<long long>(p.M) * p.N;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  if (n < p.N) {
    if (p.N % 4 == 0) {
      for (int k = 0; k < p.splits; k += 4) {
        f32x4 v[4];                                    // loads in flight together, summed in order
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = k + u < p.splits ? *reinterpret_cast<const f32x4*>(from + (k + u) * step) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 4; ++u) y += v[u];
      }
    } else {
      for (int k = 0; k < p.splits; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < p.N) y[e] += from[k * step + e];
    }
  }
  if (!p.cs) {
    finish4(p, m, n, y, bias);
    return;
  }
  y += bias;
  const float a = silu(y[0]) * y[1], b = silu(y[2]) * y[3];
  const float scale = scale_of(wave_reduce_dpp(fmaxf(magnitude(a), magnitude(b)), [](float u, float v) { return fmaxf(u, v); }));
  if (n >= p.N) return;
  static_cast<uint16_t*>(p.C)[(static_cast<long long>(m) * (p.N / 2) + n / 2) / 2] = static_cast<uint16_t>(to_e4m3(a, b, 0.f, 0.f, divisor_of(scale)));
  if ((threadIdx.x & 63) == 0) p.cs[n / 256 * p.cs_stride + m] = scale;
}

// Elements that an access to C and R may move at once.
int width_of(const Fp8Params& p) {
  const uintptr_t bits = 2 * static_cast<uintptr_t>(p.mode == kEpiSwiglu ? p.N / 2 : p.N) | reinterpret_cast<uintptr_t>(p.C) |
                         (p.mode == kEpiResidual ? reinterpret_cast<uintptr_t>(p.R) : 0);
  return bits % 16 == 0 ? 8 : bits % 8 == 0 ? 4 : bits % 4 == 0 ? 2 : 1;
}
void launch_few(const Fp8Params& p, hipStream_t stream) {
  hipLaunchKernelGGL(gemm_fp8_few, dim3((p.N + 15) / 16), dim3(64 * kFewWaves), 0, stream, p);
}
void launch_join(const Fp8Params& p, hipStream_t stream) {
  hipLaunchKernelGGL(fp8_join, dim3((p.N + 1023) / 1024 * p.M), dim3(256), 0, stream, p);
}
template <typename T, int MI, int NI, int WM, int WN, int ST, int G = 1, bool RUN = false>
void launch_tile(Fp8Params p, int splits, hipStream_t stream) {
  p.tiles_m = (p.M + 16 * MI * WM - 1) / (16 * MI * WM);
  p.tiles_n = (p.N + 16 * NI * WN - 1) / (16 * NI * WN);
  p.splits = splits;
  if constexpr (RUN) {
    // A workgroup for each CU, one tile after another.  On one card, with a workgroup a tile beside it: 10,677 x 28,672 x 3,584 with
    // SwiGLU 1,010 us (1,065), its 8-bit output 1,820 (1,847), 8192 cubed 469 (480), 1,183 x 4,608 x 3,584, one tile a workgroup, 29.3
    // (29.9).  Not with a residual, which ends K's ring in the other form: 42,196 x 1,280 x 3,424 232 us (230), 10,677 x 3,584 x 3,584
    // 172 (162).
    const long long tiles = static_cast<long long>(p.tiles_m) * p.tiles_n;
    if (in_turn(ST, splits, p.part, p.N, p.K, p.cs || p.width == 8, p.mode == kEpiResidual)) {
      hipLaunchKernelGGL((gemm_fp8_tile<T, MI, NI, WM, WN, ST, G, true>), dim3(tiles < 256 ? static_cast<unsigned>(tiles) : 256), dim3(64 * WM * WN * G), 0, stream, p);
      return;
    }
  }
  hipLaunchKernelGGL((gemm_fp8_tile<T, MI, NI, WM, WN, ST, G, false>), dim3(static_cast<unsigned>(p.tiles_m) * p.tiles_n * splits), dim3(64 * WM * WN * G), 0, stream, p);
}

void (*const kLaunch[])(Fp8Params, int, hipStream_t) = {      // by the plan's tiles
#define PACE_FP8_LAUNCH(T, MI, NI, WM, WN, ST, G, RUN, ...) launch_tile<T, MI, NI, WM, WN, ST, G, RUN>,
    PACE_FP8_TILES(PACE_FP8_LAUNCH)
#undef PACE_FP8_LAUNCH
};

// A call asks for the workspace's size and then runs: the plan, which takes 0.4 us (one row) to 12 (42,196), is made once for both.
const Fp8Plan& plan_fp8(int M, int N, int K, bool eight, bool wide) {
  static thread_local struct {
    int M, N, K;
    bool eight, wide;
    Fp8Plan plan;
  } last = {};
  if (last.M != M || last.N != N || last.K != K || last.eight != eight || last.wide != wide) last = {M, N, K, eight, wide, make_plan(M, N, K, eight, wide)};
  return last.plan;
}

bool fp8_wide(int sums, bool eight) { return sums == PACE_SUMS_AUTO ? eight : sums == PACE_SUMS_WIDE; }

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" {

pace_status_t pace_quantize_fp8(const uint16_t* x, long long x_stride, int M, int K, int rows, uint8_t* q, float* scale,
                                hipStream_t stream) {
  PACE_REQUIRE(M >= 0 && K >= 16 && K % 16 == 0 && K <= (1 << 20), "pace_quantize_fp8: M=%d K=%d (K a positive multiple of 16, at most 2^20)", M, K);
  PACE_REQUIRE(rows == 1 || rows == kBlock, "pace_quantize_fp8: rows %d not in {1, 128}", rows);
  if (M == 0) return PACE_OK;
  PACE_REQUIRE(x && q && scale, "pace_quantize_fp8: null device pointer");
  PACE_REQUIRE(aligned16(x) && aligned16(q), "pace_quantize_fp8: x and q must be 16-byte aligned");
  PACE_REQUIRE(whole(scale), "pace_quantize_fp8: scale must be aligned to its type");
  PACE_REQUIRE(x_stride >= K && x_stride % 8 == 0 && x_stride < (1ll << 31), "pace_quantize_fp8: row stride %lld (a multiple of 8, at least K=%d)", x_stride, K);
  const int kb = (K + kBlock - 1) / kBlock;
  const long long blocks = static_cast<long long>(rows == 1 ? M : (M + 127ll) / kBlock) * kb, groups = rows == 1 ? (blocks + 15) / 16 : blocks;
  PACE_REQUIRE(fits(groups, 256), "pace_quantize_fp8: too many blocks (M=%d K=%d)", M, K);
  const QuantParams p{x, q, scale, x_stride, M, K, kb};
  const dim3 grid(static_cast<unsigned>(groups)), th(256);
  if (rows == 1) hipLaunchKernelGGL(quantize_rows, grid, th, 0, stream, p);
  else hipLaunchKernelGGL(quantize_blocks, grid, th, 0, stream, p);
  return check_launch("pace_quantize_fp8");
}

pace_status_t pace_rmsnorm(const uint16_t* x, long long x_stride, const uint16_t* residual, long long residual_stride,
                           const float* gamma, float eps, int M, int K, uint16_t* sum, uint16_t* y, uint8_t* q, float* scale,
                           hipStream_t stream) {
  PACE_REQUIRE(M >= 0 && K >= 16 && K % 16 == 0 && K <= 65536, "pace_rmsnorm: M=%d K=%d (K a positive multiple of 16, at most 65,536)", M, K);
  PACE_REQUIRE(eps > 0.f && eps <= FLT_MAX, "pace_rmsnorm: eps %g must be positive and finite", static_cast<double>(eps));
  if (M == 0) return PACE_OK;
  PACE_REQUIRE((y != nullptr) != (q != nullptr) && (q != nullptr) == (scale != nullptr), "pace_rmsnorm: either y, or q and scale");
  PACE_REQUIRE(x && gamma, "pace_rmsnorm: null device pointer");
  PACE_REQUIRE(aligned16(x) && aligned16(residual) && aligned16(gamma) && aligned16(sum) && aligned16(y) && aligned16(q),
               "pace_rmsnorm: tensors must be 16-byte aligned");
  PACE_REQUIRE(whole(scale), "pace_rmsnorm: scale must be aligned to its type");
  PACE_REQUIRE(x_stride >= K && x_stride % 8 == 0 && x_stride < (1ll << 31), "pace_rmsnorm: row stride %lld (a multiple of 8, at least K=%d)", x_stride, K);
  PACE_REQUIRE(!residual || (residual_stride >= K && residual_stride % 8 == 0 && residual_stride < (1ll << 31)),
               "pace_rmsnorm: residual's row stride %lld (a multiple of 8, at least K=%d)", residual_stride, K);
  const bool wave = wave_a_row(M, K, residual, q);
  PACE_REQUIRE(fits(M, wave ? 64 : K <= 4096 ? 256 : K <= 16384 ? 512 : 1024), "pace_rmsnorm: too many rows (M=%d)", M);
  const NormParams p{x, residual, gamma, sum, y, q, scale, x_stride, residual_stride, eps, M, K};
  if (wave && K <= 1024) launch_norm<64, 2, false>(p, stream);
  else if (wave) launch_norm<64, 3, false>(p, stream);
  else if (K <= 2048) launch_norm<256, 1, true>(p, stream);
  else if (K <= 4096) launch_norm<256, 2, true>(p, stream);
  else if (K <= 8192) launch_norm<512, 2, false>(p, stream);
  else if (K <= 16384) launch_norm<512, 4, false>(p, stream);
  else launch_norm<1024, 8, false>(p, stream);
  return check_launch("pace_rmsnorm");
}

size_t pace_gemm_fp8_workspace_size(int M, int N, int K, int bits, int sums) {
  if (M < 1 || N < 1 || K < 1 || M > kMostRows || N > (1 << 30) || K > (1 << 20)) return 0;
  return plan_fp8(M, N, K, bits == 8, fp8_wide(sums, bits == 8)).bytes;
}

pace_status_t pace_gemm_fp8(const uint8_t* x, const float* x_scale, long long x_scale_stride, const uint8_t* w, const float* w_scale,
                            const float* bias, const uint16_t* residual, void* C, float* c_scale, int M, int N, int K, int epilogue,
                            int sums, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  PACE_REQUIRE(epilogue >= 0 && epilogue <= 2, "pace_gemm_fp8: epilogue %d not in {0, 1, 2}", epilogue);
  PACE_REQUIRE(sums >= PACE_SUMS_AUTO && sums <= PACE_SUMS_WIDE, "pace_gemm_fp8: sums %d not in {0, 1, 2}", sums);
  PACE_REQUIRE(M >= 0 && N >= 1 && K >= 16 && K % 16 == 0 && K <= (1 << 20), "pace_gemm_fp8: M=%d N=%d K=%d (K a positive multiple of 16, at most 2^20)", M, N, K);
  PACE_REQUIRE(epilogue != 2 || N % 2 == 0, "pace_gemm_fp8: SwiGLU needs an even N");
  PACE_REQUIRE(!c_scale || (epilogue == 2 && N % 32 == 0), "pace_gemm_fp8: 8-bit output needs SwiGLU and N=%d a multiple of 32", N);
  if (M == 0) return PACE_OK;
  PACE_REQUIRE(x && x_scale && w && w_scale && C, "pace_gemm_fp8: null device pointer");
  PACE_REQUIRE(epilogue != 1 || residual != nullptr, "pace_gemm_fp8: residual epilogue without residual");
  PACE_REQUIRE(aligned16(x) && aligned16(w), "pace_gemm_fp8: x and w must be 16-byte aligned");
  PACE_REQUIRE(!c_scale || aligned16(C), "pace_gemm_fp8: codes of the output must be 16-byte aligned");
  PACE_REQUIRE(whole(x_scale) && whole(w_scale) && whole(bias) && whole(c_scale) && whole(residual) && whole(static_cast<uint16_t*>(C)),
               "pace_gemm_fp8: scales, bias, residual and C must be aligned to their types");
  PACE_REQUIRE(x_scale_stride >= M && x_scale_stride < (1ll << 40), "pace_gemm_fp8: x_scale_stride %lld < M=%d, or past 2^40", x_scale_stride, M);
  PACE_REQUIRE(M <= kMostRows && N <= (1 << 30), "pace_gemm_fp8: too many rows or columns (M=%d N=%d)", M, N);
  const Fp8Plan& a = plan_fp8(M, N, K, c_scale != nullptr, fp8_wide(sums, c_scale != nullptr));
  PACE_REQUIRE(a.runs > 0, "pace_gemm_fp8: too many rows or columns (M=%d N=%d)", M, N);
  if (a.bytes) {
    if (workspace == nullptr || workspace_bytes < a.bytes)
      return set_error(PACE_ERR_WORKSPACE, "pace_gemm_fp8: workspace %zu < %zu bytes", workspace_bytes, a.bytes);
    PACE_REQUIRE(aligned16(workspace), "pace_gemm_fp8: workspace must be 16-byte aligned");
  }
  const int cols = epilogue == 2 ? N / 2 : N;
  for (int i = 0; i < a.runs; ++i) {
    const Fp8Launch& l = a.run[i];
    Fp8Params p{};
    p.x = x + static_cast<long long>(l.m0) * K;
    p.xs = x_scale + l.m0;
    p.w = w;
    p.ws = w_scale;
    p.bias = bias;
    p.R = epilogue == 1 ? residual + static_cast<long long>(l.m0) * cols : nullptr;
    p.C = static_cast<char*>(C) + static_cast<long long>(l.m0) * cols * (c_scale ? 1 : 2);
    p.cs = c_scale ? c_scale + l.m0 : nullptr;
    p.part = l.part ? static_cast<float*>(workspace) : nullptr;
    p.xs_stride = x_scale_stride;
    p.cs_stride = M;
    p.M = l.rows;
    p.N = N;
    p.K = K;
    p.kb = (K + kBlock - 1) / kBlock;
    p.mode = epilogue;
    p.splits = l.splits;
    p.width = width_of(p);
    if (l.tile < 0) launch_few(p, stream);
    else kLaunch[l.tile](p, l.splits, stream);
    if (l.part) launch_join(p, stream);
  }
  return check_launch("pace_gemm_fp8");
}

}  // extern "C"
