// Products of a few rows with weights of 4 bits: C = x W^T, W[n, k] = (q - zero) * scale with a scale (and
// zero) for each group of k, and the epilogues of the bf16 product.
#include "pace_internal.h"

namespace pace {
namespace {

struct W4Params {
  const uint16_t* x;
  const uint8_t* w;
  const uint16_t* scale;
  const uint8_t* zero;
  const float* bias;
  const uint16_t* R;
  uint16_t* C;
  int M, N, K, group, mode;
};

__device__ __forceinline__ float bf16_f32(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
__device__ __forceinline__ uint16_t f32_bf16(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }

// One wave per output column (or SwiGLU pair of them) and row of x.
__global__ __launch_bounds__(64) void gemm_w4(const W4Params p) {
  const int cols = p.mode == 2 ? p.N / 2 : p.N, per = p.mode == 2 ? 2 : 1;
  const int f = blockIdx.x, m = blockIdx.y, lane = threadIdx.x;
  const int ng = p.K / p.group;
  float y[2] = {0.f, 0.f};
  for (int c = 0; c < per; ++c) {
    const long long n = static_cast<long long>(f) * per + c;
    float acc = 0.f;
    for (int k = 2 * lane; k < p.K; k += 128) {
      const uint8_t b = p.w[n * (p.K / 2) + k / 2];
      const float s = bf16_f32(p.scale[n * ng + k / p.group]);
      const float z = p.zero ? p.zero[n * ng + k / p.group] : 8.f;
      acc += bf16_f32(p.x[static_cast<long long>(m) * p.K + k]) * ((b & 15) - z) * s;
      acc += bf16_f32(p.x[static_cast<long long>(m) * p.K + k + 1]) * ((b >> 4) - z) * s;
    }
    y[c] = wave_sum(acc) + (p.bias ? p.bias[n] : 0.f);
  }
  if (lane == 0) {
    const long long at = static_cast<long long>(m) * cols + f;
    float r = y[0];
    if (p.mode == 1) r += bf16_f32(p.R[at]);
    if (p.mode == 2) r = y[0] / (1.f + expf(-y[0])) * y[1];
    p.C[at] = f32_bf16(r);
  }
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" pace_status_t pace_gemm_w4(const uint16_t* x, const uint8_t* w, const uint16_t* scale, const uint8_t* zero,
                                      const float* bias, const uint16_t* residual, uint16_t* C, int M, int N, int K,
                                      int group, int epilogue, hipStream_t stream) {
  PACE_REQUIRE(x && w && scale && C, "pace_gemm_w4: null device pointer");
  PACE_REQUIRE(epilogue >= 0 && epilogue <= 2, "pace_gemm_w4: epilogue %d not in {0, 1, 2}", epilogue);
  PACE_REQUIRE(epilogue != 1 || residual != nullptr, "pace_gemm_w4: residual epilogue without residual");
  PACE_REQUIRE(epilogue != 2 || N % 2 == 0, "pace_gemm_w4: SwiGLU needs an even N");
  PACE_REQUIRE(group == 32 || group == 64 || group == 128, "pace_gemm_w4: group %d not in {32, 64, 128}", group);
  PACE_REQUIRE(M >= 1 && N >= 1 && K >= group && K % group == 0,
               "pace_gemm_w4: M=%d N=%d K=%d (K a positive multiple of group=%d)", M, N, K, group);
  PACE_REQUIRE(aligned16(x) && aligned16(w), "pace_gemm_w4: x and w must be 16-byte aligned");
  const long long lim = 1ll << 31;
  PACE_REQUIRE(2ll * M * K < lim && static_cast<long long>(N) * K / 2 < lim && 2ll * N * (K / group) < lim && 2ll * M * N < lim,
               "pace_gemm_w4: an operand reaches 2 GiB");
  W4Params p{x, w, scale, zero, bias, residual, C, M, N, K, group, epilogue};
  PACE_REQUIRE(M <= 65535, "pace_gemm_w4: M=%d past 65535", M);
  hipLaunchKernelGGL(gemm_w4, dim3(epilogue == 2 ? N / 2 : N, M), dim3(64), 0, stream, p);
  return check_launch("pace_gemm_w4");
}
