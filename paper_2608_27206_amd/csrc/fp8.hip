// A layer's 8-bit operators: rows and weights to OCP e4m3 codes with a scale for each block of 128, the RMS norm with the
// residual's addition in front of it, and the product of such codes with the epilogues of the bf16 product.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "pace_internal.h"

namespace pace {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kBlock = 128;                    // values that share a scale
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
__device__ __forceinline__ float silu(float x) { return x / (1.f + expf(-x)); }

// What a value adds to its block's maximum: its magnitude, 0 where it is not finite.
__device__ __forceinline__ float magnitude(float x) { return fabsf(x) <= FLT_MAX ? fabsf(x) : 0.f; }
__device__ __forceinline__ float scale_of(float top) { return fmaxf(top / kE4m3Max, kMinScale); }
// x / scale by the reciprocal: within 2^-22 of the quotient, so a code differs from the quotient's only where that lies as
// near to the middle between two codes.  The largest scale is 2^128 / 448 and the least 2^-120: both reciprocals are normal.
// What is not finite becomes NaN (what the conversion makes of infinities depends on a mode bit); the others are at most
// 448 (1 + 2^-22), which rounds to 448.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d, float inv) {
  const float nan = __uint_as_float(0x7fc00000u);
  a = fabsf(a) <= FLT_MAX ? a * inv : nan;
  b = fabsf(b) <= FLT_MAX ? b * inv : nan;
  c = fabsf(c) <= FLT_MAX ? c * inv : nan;
  d = fabsf(d) <= FLT_MAX ? d * inv : nan;
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return static_cast<uint32_t>(r);
}
__device__ __forceinline__ uint2 to_e4m3(const float (&x)[8], float inv) {
  return make_uint2(to_e4m3(x[0], x[1], x[2], x[3], inv), to_e4m3(x[4], x[5], x[6], x[7], inv));
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

// ---------------------------------------------------------------- quantisation
struct QuantParams {
  const uint16_t* x;
  uint8_t* q;
  float* scale;
  long long stride;
  int M, K, kb;
};

// Rows: 16 lanes per block of 128, blocks of a row after one another.
__global__ __launch_bounds__(256) void quantize_rows(const QuantParams p) {
  const long long block = static_cast<long long>(blockIdx.x) * 16 + (threadIdx.x >> 4);
  const int row = static_cast<int>(block / p.kb), kb = static_cast<int>(block - static_cast<long long>(row) * p.kb);
  if (row >= p.M) return;                              // whole groups of 16 lanes
  const int k = kb * kBlock + (threadIdx.x & 15) * 8;
  float x[8] = {};
  if (k < p.K) unpack8(*reinterpret_cast<const uint4*>(p.x + row * p.stride + k), x);
  const float scale = scale_of(max16(magnitude8(x)));
  if (k < p.K) *reinterpret_cast<uint2*>(p.q + static_cast<long long>(row) * p.K + k) = to_e4m3(x, 1.f / scale);
  if ((threadIdx.x & 15) == 0) p.scale[static_cast<long long>(kb) * p.M + row] = scale;
}

// Weights: a workgroup per block of 128 x 128, its values in registers between the maximum and the store.
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
  const float scale = scale_of(block_reduce<1>(top, red)), inv = 1.f / scale;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (k < p.K && r0 + 16 * i < p.M)
      *reinterpret_cast<uint2*>(p.q + static_cast<long long>(r0 + 16 * i) * p.K + k) = to_e4m3(x[i], inv);
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
template <int T, int NC>
__global__ __launch_bounds__(T < 256 ? 256 : T) void rmsnorm_rows(const NormParams p) {
  constexpr int ROWS = T < 256 ? 256 / T : 1;
  __shared__ float red[T / 64];
  const int t = threadIdx.x % T, row = blockIdx.x * ROWS + threadIdx.x / T;
  if (T == 64 && row >= p.M) return;                   // a wave of its own
  const int pieces = p.K / 8;
  const uint4* x = reinterpret_cast<const uint4*>(p.x + row * p.stride);
  const uint4* r = reinterpret_cast<const uint4*>(p.residual + row * p.rstride);
  float h[NC][8];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = i * T + t;
    uint4 u = make_uint4(0, 0, 0, 0), v = u;
    if (c < pieces) {
      u = x[c];
      if (p.residual) v = r[c];
    }
    float add[8];
    unpack8(u, h[i]);
    unpack8(v, add);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[i][e] += add[e];
  }
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(h[i][e], h[i][e], ss);
  if constexpr (T == 64) ss = wave_reduce_dpp(ss, [](float a, float b) { return a + b; });
  else ss = block_reduce<0>(ss, red);
  const float inv = 1.f / sqrtf(ss / static_cast<float>(p.K) + p.eps);
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
      const float4 g0 = reinterpret_cast<const float4*>(p.gamma)[2 * c], g1 = reinterpret_cast<const float4*>(p.gamma)[2 * c + 1];
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
      reinterpret_cast<uint2*>(p.q + static_cast<long long>(row) * p.K)[c] = to_e4m3(y, 1.f / scale);
      if ((t & 15) == 0) p.scale[static_cast<long long>(c / 16) * p.M + row] = scale;
    }
  }
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
  float* part;                 // [splits, M, N]
  long long xs_stride;
  int M, N, K, kb, mode, splits;
};

__device__ __forceinline__ f32x4 mfma128(i32x8 a, i32x8 b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}

// One output value of 16 bits (or a SwiGLU pair's) from its finished sum.
__device__ __forceinline__ void fp8_store(const Fp8Params& p, int m, int n, float y, float y_pair) {
  const long long at = static_cast<long long>(m) * (p.mode == 2 ? p.N / 2 : p.N) + (p.mode == 2 ? n / 2 : n);
  if (p.mode == 1) y += bf16_f32(p.R[at]);
  if (p.mode == 2) y = silu(y) * y_pair;
  static_cast<uint16_t*>(p.C)[at] = f32_bf16(y);
}

// 64 x 64 of C by four waves, operands straight from memory.  W is the products' A operand: a lane then holds four
// neighbouring columns n of one row m, whose block of 128 has one scale for the lane.
__global__ __launch_bounds__(256) void gemm_fp8_direct(const Fp8Params p) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int tiles = (p.N + 63) / 64, tm = blockIdx.x / tiles;
  const int n0 = (blockIdx.x - tm * tiles) * 64 + (w & 1) * 32, m0 = tm * 64 + (w >> 1) * 32;
  f32x4 acc[2][2] = {};
  const auto load = [&](const uint8_t* base, int row, int rows, int k) {
    uint4 u[2] = {};
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (row < rows && k + 64 * h < p.K) u[h] = *reinterpret_cast<const uint4*>(base + static_cast<long long>(row) * p.K + k + 64 * h);
    return i32x8{static_cast<int>(u[0].x), static_cast<int>(u[0].y), static_cast<int>(u[0].z), static_cast<int>(u[0].w),
                 static_cast<int>(u[1].x), static_cast<int>(u[1].y), static_cast<int>(u[1].z), static_cast<int>(u[1].w)};
  };
  for (int b = 0; b < p.kb; ++b) {
    i32x8 wf[2], xf[2];
    float s[2];
    const float sw = n0 < p.N ? p.ws[static_cast<long long>(n0 / kBlock) * p.kb + b] : 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int m = m0 + 16 * i + r;
      wf[i] = load(p.w, n0 + 16 * i + r, p.N, b * kBlock + 16 * g);
      xf[i] = load(p.x, m, p.M, b * kBlock + 16 * g);
      s[i] = m < p.M ? p.xs[b * p.xs_stride + m] * sw : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f32x4 d = mfma128(wf[j], xf[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(s[i], d[e], acc[i][j][e]);
      }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int m = m0 + 16 * i + r;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = n0 + 16 * j + 4 * g + e;
        if (m >= p.M || n >= p.N) continue;
        if (p.part) p.part[static_cast<long long>(m) * p.N + n] = acc[i][j][e];
        else if (p.mode != 2) fp8_store(p, m, n, acc[i][j][e] + (p.bias ? p.bias[n] : 0.f), 0.f);
        else if (e % 2 == 0)
          fp8_store(p, m, n, acc[i][j][e] + (p.bias ? p.bias[n] : 0.f), acc[i][j][(e + 1) & 3] + (p.bias ? p.bias[n + 1] : 0.f));
      }
    }
}

// Adds the parts of a split K in their order and finishes the output.  With 8 bits a wave has the 256 columns of a block.
__global__ __launch_bounds__(256) void fp8_join(const Fp8Params p) {
  const int per = p.cs ? 4 : p.mode == 2 ? 2 : 1;
  const int cols = (p.N + 256 * per - 1) / (256 * per);
  const int m = blockIdx.x / cols, n = ((blockIdx.x - m * cols) * 256 + threadIdx.x) * per;
  float y[4] = {};
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (c >= per || n >= p.N) break;
    for (int k = 0; k < p.splits; ++k) y[c] += p.part[(static_cast<long long>(k) * p.M + m) * p.N + n + c];
    if (p.bias) y[c] += p.bias[n + c];
  }
  if (!p.cs) {
    if (n < p.N) fp8_store(p, m, n, y[0], y[1]);
    return;
  }
  const float a = silu(y[0]) * y[1], b = silu(y[2]) * y[3];
  const float scale = scale_of(wave_reduce_dpp(fmaxf(magnitude(a), magnitude(b)), [](float u, float v) { return fmaxf(u, v); }));
  if (n >= p.N) return;
  static_cast<uint16_t*>(p.C)[(static_cast<long long>(m) * (p.N / 2) + n / 2) / 2] = static_cast<uint16_t>(to_e4m3(a, b, 0.f, 0.f, 1.f / scale));
  if ((threadIdx.x & 63) == 0) p.cs[static_cast<long long>(n / 256) * p.M + m] = scale;
}

bool too_many_threads(long long groups, int threads) { return groups * threads >= (1ll << 32); }

size_t fp8_bytes(int M, int N, int bits) { return bits == 8 ? static_cast<size_t>(M) * N * sizeof(float) : 0; }

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
  PACE_REQUIRE(x_stride >= K && x_stride % 8 == 0 && x_stride < (1ll << 31), "pace_quantize_fp8: row stride %lld (a multiple of 8, at least K=%d)", x_stride, K);
  const int kb = (K + kBlock - 1) / kBlock;
  const long long blocks = static_cast<long long>(rows == 1 ? M : (M + 127ll) / kBlock) * kb, groups = rows == 1 ? (blocks + 15) / 16 : blocks;
  PACE_REQUIRE(!too_many_threads(groups, 256), "pace_quantize_fp8: too many blocks (M=%d K=%d)", M, K);
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
  PACE_REQUIRE(x_stride >= K && x_stride % 8 == 0 && x_stride < (1ll << 31), "pace_rmsnorm: row stride %lld (a multiple of 8, at least K=%d)", x_stride, K);
  PACE_REQUIRE(!residual || (residual_stride >= K && residual_stride % 8 == 0 && residual_stride < (1ll << 31)),
               "pace_rmsnorm: residual's row stride %lld (a multiple of 8, at least K=%d)", residual_stride, K);
  PACE_REQUIRE(!too_many_threads(M, K <= 4096 ? 64 : K <= 16384 ? 256 : 1024), "pace_rmsnorm: too many rows (M=%d)", M);
  const NormParams p{x, residual, gamma, sum, y, q, scale, x_stride, residual_stride, eps, M, K};
  if (K <= 1024) hipLaunchKernelGGL((rmsnorm_rows<64, 2>), dim3((M + 3ll) / 4), dim3(256), 0, stream, p);
  else if (K <= 4096) hipLaunchKernelGGL((rmsnorm_rows<64, 8>), dim3((M + 3ll) / 4), dim3(256), 0, stream, p);
  else if (K <= 16384) hipLaunchKernelGGL((rmsnorm_rows<256, 8>), dim3(M), dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((rmsnorm_rows<1024, 8>), dim3(M), dim3(1024), 0, stream, p);
  return check_launch("pace_rmsnorm");
}

size_t pace_gemm_fp8_workspace_size(int M, int N, int K, int bits) {
  if (M < 1 || N < 1 || K < 1) return 0;
  return fp8_bytes(M, N, bits);
}

pace_status_t pace_gemm_fp8(const uint8_t* x, const float* x_scale, long long x_scale_stride, const uint8_t* w, const float* w_scale,
                            const float* bias, const uint16_t* residual, void* C, float* c_scale, int M, int N, int K, int epilogue,
                            void* workspace, size_t workspace_bytes, hipStream_t stream) {
  PACE_REQUIRE(epilogue >= 0 && epilogue <= 2, "pace_gemm_fp8: epilogue %d not in {0, 1, 2}", epilogue);
  PACE_REQUIRE(M >= 0 && N >= 1 && K >= 16 && K % 16 == 0 && K <= (1 << 20), "pace_gemm_fp8: M=%d N=%d K=%d (K a positive multiple of 16, at most 2^20)", M, N, K);
  PACE_REQUIRE(epilogue != 2 || N % 2 == 0, "pace_gemm_fp8: SwiGLU needs an even N");
  PACE_REQUIRE(!c_scale || (epilogue == 2 && N % 32 == 0), "pace_gemm_fp8: 8-bit output needs SwiGLU and N=%d a multiple of 32", N);
  if (M == 0) return PACE_OK;
  PACE_REQUIRE(x && x_scale && w && w_scale && C, "pace_gemm_fp8: null device pointer");
  PACE_REQUIRE(epilogue != 1 || residual != nullptr, "pace_gemm_fp8: residual epilogue without residual");
  PACE_REQUIRE(aligned16(x) && aligned16(w), "pace_gemm_fp8: x and w must be 16-byte aligned");
  PACE_REQUIRE(!c_scale || aligned16(C), "pace_gemm_fp8: codes of the output must be 16-byte aligned");
  PACE_REQUIRE(x_scale_stride >= M, "pace_gemm_fp8: x_scale_stride %lld < M=%d", x_scale_stride, M);
  PACE_REQUIRE(N <= (1 << 30) && !too_many_threads((M + 63ll) / 64 * ((N + 63) / 64), 256), "pace_gemm_fp8: too many rows or columns (M=%d N=%d)", M, N);
  PACE_REQUIRE(!c_scale || !too_many_threads((N + 1023ll) / 1024 * M, 256), "pace_gemm_fp8: too many rows or columns (M=%d N=%d)", M, N);
  const size_t need = fp8_bytes(M, N, c_scale ? 8 : 16);
  if (need) {
    if (workspace == nullptr || workspace_bytes < need)
      return set_error(PACE_ERR_WORKSPACE, "pace_gemm_fp8: workspace %zu < %zu bytes", workspace_bytes, need);
    PACE_REQUIRE(aligned16(workspace), "pace_gemm_fp8: workspace must be 16-byte aligned");
  }
  const Fp8Params p{x, x_scale, w, w_scale, bias, residual, C, c_scale, need ? static_cast<float*>(workspace) : nullptr, x_scale_stride,
                    M, N, K, (K + kBlock - 1) / kBlock, epilogue, 1};
  hipLaunchKernelGGL(gemm_fp8_direct, dim3((N + 63) / 64 * ((M + 63) / 64)), dim3(256), 0, stream, p);
  if (need) hipLaunchKernelGGL(fp8_join, dim3((N + 1023) / 1024 * M), dim3(256), 0, stream, p);
  return check_launch("pace_gemm_fp8");
}

}  // extern "C"
