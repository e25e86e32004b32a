// Products of a few rows with weights of 4 bits: C = x W^T, W[n, k] = (q - zero) * scale with a scale (and
// zero) for each group of k, and the epilogues of the bf16 product.
#include <math.h>

#include "pace_internal.h"

namespace pace {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

struct W4Params {
  const uint16_t* x;
  const uint8_t* w;
  const uint16_t* scale;
  const uint8_t* zero;
  const float* bias;
  const uint16_t* R;
  uint16_t* C;
  float* part;               // [splits, M, N] sums where several workgroups share K
  int M, N, K, mode, splits, ntiles;
};

constexpr int kBlockK = 128;       // k per step of a wave: 16 bytes of weights per lane

__device__ __forceinline__ float bf16_f32(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
__device__ __forceinline__ uint16_t f32_bf16(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// One output value (or a SwiGLU pair's) from its finished sum.
__device__ __forceinline__ void w4_store(const W4Params& p, int m, int n, float y, float y_pair) {
  const int cols = p.mode == 2 ? p.N / 2 : p.N, c = p.mode == 2 ? n / 2 : n;
  const long long at = static_cast<long long>(m) * cols + c;
  if (p.mode == 1) y += bf16_f32(p.R[at]);
  if (p.mode == 2) y = y / (1.f + expf(-y)) * y_pair;
  p.C[at] = f32_bf16(y);
}

// C = x W^T by 16x16x32 products with x as the A operand (rows m) and W as B (columns n), so that a lane's
// column has one scale.  Bound by the weights' bytes: a wave streams 16 bytes per lane (32 k of one row) and step, the
// waves of a workgroup take the steps of K in turn and join through LDS.
//  A 4 x 4 transpose of dwords between the lane groups (v_permlane32_swap, v_permlane16_swap) turns the 32
//    consecutive k of a lane into 8 of each 32, so that every product lies in one scale group of 32 or more.
//  (w >> 4 i) & 0xf000f | 0x43004300 is the bf16 pair 128 + q of nibbles i and i + 4: exact, one instruction past the
//    shift.  The products thus sum x (128 + q); (128 + zero) sum x comes off for each group in fp32, sum x from one
//    more product with ones.  The A operand takes x in the same order of k.
template <int MT, int NT, int W, int GROUP>
__global__ __launch_bounds__(64 * W) void gemm_w4(const W4Params p) {
  constexpr int GB = kBlockK / GROUP, SPG = 4 / GB;             // groups per step, products per group
  __shared__ float join[W > 1 ? W / 2 : 1][MT * NT * 4][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int id = remap_block_id(blockIdx.x, gridDim.x);
  const int n0 = id % p.ntiles * 16 * NT, split = id / p.ntiles, m0 = blockIdx.y * 16 * MT;
  const int steps = (p.K + kBlockK - 1) / kBlockK;
  const int s0 = static_cast<int>(static_cast<long long>(steps) * split / p.splits);
  const int s1 = static_cast<int>(static_cast<long long>(steps) * (split + 1) / p.splits);
  const int groups = p.K / GROUP;

  const uint8_t* wrow[NT];
  const uint16_t* srow[NT];
  const uint8_t* zrow[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int n = n0 + 16 * t + r < p.N ? n0 + 16 * t + r : p.N - 1;
    wrow[t] = p.w + static_cast<long long>(n) * (p.K / 2);
    srow[t] = p.scale + static_cast<long long>(n) * groups;
    zrow[t] = p.zero ? p.zero + static_cast<long long>(n) * groups : nullptr;
  }
  const uint16_t* xrow[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = m0 + 16 * t + r < p.M ? m0 + 16 * t + r : p.M - 1;
    xrow[t] = p.x + static_cast<long long>(m) * p.K;
  }

  uint4 wq[NT];
  float sc[NT][GB], zc[NT][GB];
  uint4 xf[MT][4];
  const auto load_w = [&](int s) {
    const int k = s * kBlockK + 32 * g;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      wq[t] = *reinterpret_cast<const uint4*>(wrow[t] + (k < p.K ? k / 2 : 0));
#pragma unroll
      for (int q = 0; q < GB; ++q) {
        const int gi = s * GB + q < groups ? s * GB + q : groups - 1;
        sc[t][q] = bf16_f32(srow[t][gi]);
        zc[t][q] = 128.f + (p.zero ? static_cast<float>(zrow[t][gi]) : 8.f);
      }
    }
  };
  const auto load_x = [&](int s) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int k = s * kBlockK + 32 * q + 8 * g;
#pragma unroll
      for (int t = 0; t < MT; ++t)
        xf[t][q] = k < p.K ? *reinterpret_cast<const uint4*>(xrow[t] + k) : make_uint4(0, 0, 0, 0);
    }
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[a][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint4 ones = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);

  int s = s0 + w;
  if (s < s1) {
    load_w(s);
    load_x(s);
  }
  for (; s < s1; s += W) {
    // x in the nibbles' order (0 4, 1 5, 2 6, 3 7), and its sums by group
    uint4 xa[MT][4];
    f32x4 xs[MT][GB];
#pragma unroll
    for (int a = 0; a < MT; ++a) {
#pragma unroll
      for (int q = 0; q < GB; ++q) xs[a][q] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint4 u = xf[a][q];
        xa[a][q] = make_uint4(__builtin_amdgcn_perm(u.z, u.x, 0x05040100u), __builtin_amdgcn_perm(u.z, u.x, 0x07060302u),
                              __builtin_amdgcn_perm(u.w, u.y, 0x05040100u), __builtin_amdgcn_perm(u.w, u.y, 0x07060302u));
        xs[a][q / SPG] = mfma16(xa[a][q], ones, xs[a][q / SPG]);
      }
    }
    uint32_t d[NT][4];
    float sg[NT][GB], zg[NT][GB];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      d[t][0] = wq[t].x; d[t][1] = wq[t].y; d[t][2] = wq[t].z; d[t][3] = wq[t].w;
#pragma unroll
      for (int q = 0; q < GB; ++q) { sg[t][q] = sc[t][q]; zg[t][q] = zc[t][q]; }
    }
    if (s + W < s1) {
      load_w(s + W);
      load_x(s + W);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const u32x2 y = __builtin_amdgcn_permlane32_swap(d[t][q], d[t][q + 2], false, false);
        d[t][q] = y.x;
        d[t][q + 2] = y.y;
      }
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        const u32x2 y = __builtin_amdgcn_permlane16_swap(d[t][q], d[t][q + 1], false, false);
        d[t][q] = y.x;
        d[t][q + 1] = y.y;
      }
#pragma unroll
      for (int q = 0; q < GB; ++q) {
        f32x4 sum[MT];
#pragma unroll
        for (int a = 0; a < MT; ++a) sum[a] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = q * SPG; e < (q + 1) * SPG; ++e) {
          const uint32_t v = d[t][e];
          const uint4 b = make_uint4((v & 0xf000fu) | 0x43004300u, (v >> 4 & 0xf000fu) | 0x43004300u,
                                     (v >> 8 & 0xf000fu) | 0x43004300u, (v >> 12 & 0xf000fu) | 0x43004300u);
#pragma unroll
          for (int a = 0; a < MT; ++a) sum[a] = mfma16(xa[a][e], b, sum[a]);
        }
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc[a][t][i] = fmaf(sg[t][q], fmaf(-zg[t][q], xs[a][q][i], sum[a][i]), acc[a][t][i]);
      }
    }
  }

#pragma unroll
  for (int h = W / 2; h >= 1; h >>= 1) {
    if (w >= h && w < 2 * h) {
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) join[w - h][(a * NT + t) * 4 + i][lane] = acc[a][t][i];
    }
    __syncthreads();
    if (w < h) {
#pragma unroll
      for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[a][t][i] += join[w][(a * NT + t) * 4 + i][lane];
    }
    __syncthreads();
  }
  if (w != 0) return;
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int n = n0 + 16 * t + r;
      const float bias = p.bias && n < p.N && p.splits == 1 ? p.bias[n] : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int m = m0 + 16 * a + 4 * g + i;
        const float y = acc[a][t][i] + bias;
        const float pair = dpp_f32<kDppQuadXor1>(y);         // SwiGLU: the up value of an even lane's gate
        if (m >= p.M || n >= p.N) continue;
        if (p.splits > 1) p.part[(static_cast<long long>(split) * p.M + m) * p.N + n] = y;
        else if (p.mode != 2 || (n & 1) == 0) w4_store(p, m, n, y, pair);
      }
    }
}

// Sums the parts of a split K in their order and finishes the output.
__global__ __launch_bounds__(256) void w4_join(const W4Params p) {
  const int per = p.mode == 2 ? 2 : 1;
  const int n = (blockIdx.x * 256 + threadIdx.x) * per, m = blockIdx.y;
  if (n >= p.N) return;
  float y[2];
  for (int c = 0; c < per; ++c) {
    float s = 0.f;
    for (int k = 0; k < p.splits; ++k) s += p.part[(static_cast<long long>(k) * p.M + m) * p.N + n + c];
    y[c] = s + (p.bias ? p.bias[n + c] : 0.f);
  }
  w4_store(p, m, n, y[0], y[per - 1]);
}

struct W4Plan {
  int mt, nt, ntiles, splits;
};
constexpr int kW4Waves = 8;
W4Plan plan_w4(int M, int N, int K) {
  W4Plan a;
  a.mt = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  a.nt = a.mt;
  a.ntiles = (N + 16 * a.nt - 1) / (16 * a.nt);
  a.splits = 1;
  if (a.mt > 1) {
    const int most = ((K + kBlockK - 1) / kBlockK + 2 * kW4Waves - 1) / (2 * kW4Waves);
    const int s = 512 / a.ntiles;
    a.splits = s < 1 ? 1 : s < most ? s : most;
  }
  return a;
}

template <int MT, int NT>
void launch_w4(const W4Params& p, int group, hipStream_t stream) {
  const dim3 g(p.ntiles * p.splits, (p.M + 16 * MT - 1) / (16 * MT)), th(64 * kW4Waves);
  if (group == 32) hipLaunchKernelGGL((gemm_w4<MT, NT, kW4Waves, 32>), g, th, 0, stream, p);
  else if (group == 64) hipLaunchKernelGGL((gemm_w4<MT, NT, kW4Waves, 64>), g, th, 0, stream, p);
  else hipLaunchKernelGGL((gemm_w4<MT, NT, kW4Waves, 128>), g, th, 0, stream, p);
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" {

size_t pace_gemm_w4_workspace_size(int M, int N, int K) {
  if (M < 1 || N < 1 || K < 1) return 0;
  const W4Plan a = plan_w4(M, N, K);
  return a.splits == 1 ? 0 : static_cast<size_t>(a.splits) * M * N * sizeof(float);
}

pace_status_t pace_gemm_w4(const uint16_t* x, const uint8_t* w, const uint16_t* scale, const uint8_t* zero,
                           const float* bias, const uint16_t* residual, uint16_t* C, int M, int N, int K, int group,
                           int epilogue, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  PACE_REQUIRE(x && w && scale && C, "pace_gemm_w4: null device pointer");
  PACE_REQUIRE(epilogue >= 0 && epilogue <= 2, "pace_gemm_w4: epilogue %d not in {0, 1, 2}", epilogue);
  PACE_REQUIRE(epilogue != 1 || residual != nullptr, "pace_gemm_w4: residual epilogue without residual");
  PACE_REQUIRE(epilogue != 2 || N % 2 == 0, "pace_gemm_w4: SwiGLU needs an even N");
  PACE_REQUIRE(group == 32 || group == 64 || group == 128, "pace_gemm_w4: group %d not in {32, 64, 128}", group);
  PACE_REQUIRE(M >= 1 && N >= 1 && K >= group && K % group == 0,
               "pace_gemm_w4: M=%d N=%d K=%d (K a positive multiple of group=%d)", M, N, K, group);
  PACE_REQUIRE(aligned16(x) && aligned16(w), "pace_gemm_w4: x and w must be 16-byte aligned");
  const long long lim = 1ll << 31;
  PACE_REQUIRE(2ll * M * K < lim && static_cast<long long>(N) * K / 2 < lim && 2ll * N * (K / group) < lim &&
                   2ll * M * N < lim && M <= 65535,
               "pace_gemm_w4: an operand reaches 2 GiB, or M=%d is past 65,535", M);
  const W4Plan a = plan_w4(M, N, K);
  const size_t need = pace_gemm_w4_workspace_size(M, N, K);
  if (need) {
    if (workspace == nullptr || workspace_bytes < need)
      return set_error(PACE_ERR_WORKSPACE, "pace_gemm_w4: workspace %zu < %zu bytes", workspace_bytes, need);
    PACE_REQUIRE(aligned16(workspace), "pace_gemm_w4: workspace must be 16-byte aligned");
  }
  const W4Params p{x, w, scale, zero, bias, residual, C, static_cast<float*>(workspace), M, N, K, epilogue, a.splits, a.ntiles};
  if (a.mt == 1) launch_w4<1, 1>(p, group, stream);
  else if (a.mt == 2) launch_w4<2, 2>(p, group, stream);
  else launch_w4<4, 4>(p, group, stream);
  if (a.splits > 1)
    hipLaunchKernelGGL(w4_join, dim3(((epilogue == 2 ? N / 2 : N) + 255) / 256, M), dim3(256), 0, stream, p);
  return check_launch("pace_gemm_w4");
}

}  // extern "C"
