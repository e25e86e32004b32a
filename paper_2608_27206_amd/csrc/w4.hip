// Products of a few rows with weights of 4 bits: C = x W^T, W[n, k] = (q - zero) * scale with a scale (and
// zero) for each group of k, and the epilogues of the bf16 product.
#include <math.h>

#include <type_traits>

#include "pace_internal.h"

namespace pace {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

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

__device__ __forceinline__ float bf16_f32(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
__device__ __forceinline__ uint16_t f32_bf16(float f) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// What both kernels do: C = x W^T by 16x16x32 products with x as the A operand (rows m) and W as B (columns n), so that a
// lane's column has one scale.
//  A lane loads 16 bytes of its column's row: the 32 k's 32 g .. 32 g + 31 of a block of 128 (lane group g).  A 4 x 4
//    transpose of dwords between the lane groups (v_permlane32_swap, v_permlane16_swap) makes that 8 k's of each 32, so
//    that every product lies in one scale group of 32 or more.
//  (w >> 4 i) & 0xf000f | 0x43004300 is the bf16 pair 128 + q of nibbles i and i + 4: exact, one instruction past the
//    shift.  The products thus sum x (128 + q); (128 + zero) sum x comes off for each group in fp32.  The A operand
//    takes x in the same order of k (0 4, 1 5, 2 6, 3 7 of every 8).
__device__ __forceinline__ void transpose_groups(uint32_t (&d)[4]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const u32x2 y = __builtin_amdgcn_permlane32_swap(d[q], d[q + 2], false, false);
    d[q] = y.x;
    d[q + 2] = y.y;
  }
#pragma unroll
  for (int q = 0; q < 4; q += 2) {
    const u32x2 y = __builtin_amdgcn_permlane16_swap(d[q], d[q + 1], false, false);
    d[q] = y.x;
    d[q + 1] = y.y;
  }
}
// The constants lie in registers that the compiler knows nothing about: as literals they take two instructions, and eight
// rows through 28,672 columns of 3,584 23.7 us instead of 22.6.
struct Nibbles {
  uint32_t mask = 0xf000fu, base = 0x43004300u;
  __device__ __forceinline__ Nibbles() { asm volatile("" : "+s"(mask), "+v"(base)); }
  __device__ __forceinline__ uint4 operator()(uint32_t v) const {
    return make_uint4((v & mask) | base, (v >> 4 & mask) | base, (v >> 8 & mask) | base, (v >> 12 & mask) | base);
  }
};
__device__ __forceinline__ uint4 nibble_order(uint4 u) {
  return make_uint4(__builtin_amdgcn_perm(u.z, u.x, 0x05040100u), __builtin_amdgcn_perm(u.z, u.x, 0x07060302u),
                    __builtin_amdgcn_perm(u.w, u.y, 0x05040100u), __builtin_amdgcn_perm(u.w, u.y, 0x07060302u));
}
// Raw scales and zeros of groups first .. first + N - 1 of the row that begins at group `row` of the arrays.  TAIL: past
// the row's end, its last one's.  They are turned into numbers where they are used, so that the loads stay in flight.
template <int N>
struct Groups {
  uint16_t s[N];
  uint8_t z[N];
  template <bool TAIL>
  __device__ __forceinline__ void load(const W4Params& p, unsigned row, int first, int groups) {
    if constexpr (!TAIL) {
      __builtin_memcpy(s, p.scale + first + row, 2 * N);       // any alignment
      if (p.zero) __builtin_memcpy(z, p.zero + first + row, N);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const unsigned at = row + (first + i < groups ? first + i : groups - 1);
        s[i] = p.scale[at];
        if (p.zero) z[i] = p.zero[at];
      }
    }
  }
  __device__ __forceinline__ float scale(int i) const { return bf16_f32(s[i]); }
  __device__ __forceinline__ float zero(const W4Params& p, int i) const { return p.zero ? 128.f + static_cast<float>(z[i]) : 136.f; }
};

// One output value (or a SwiGLU pair's) from its finished sum.
__device__ __forceinline__ void w4_store(const W4Params& p, int m, int n, float y, float y_pair) {
  const int cols = p.mode == 2 ? p.N / 2 : p.N, c = p.mode == 2 ? n / 2 : n;
  const long long at = static_cast<long long>(m) * cols + c;
  if (p.mode == 1) y += bf16_f32(p.R[at]);
  if (p.mode == 2) y = y / (1.f + expf(-y)) * y_pair;
  p.C[at] = f32_bf16(y);
}

// Stages 8 k's of a row of x for the kernels below: in the nibbles' order to *to, and the sum over each group of G k's,
// which 16 consecutive lanes hold 128 of, by the lanes whose piece begins one.
template <int G>
__device__ __forceinline__ void stage_x(uint4 u, int piece, uint4* to, float* sums) {
  const uint32_t v[4] = {u.x, u.y, u.z, u.w};
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) s += __uint_as_float(v[e] << 16) + __uint_as_float(v[e] & 0xffff0000u);
  s += dpp_f32<kDppQuadXor1>(s);
  s += dpp_f32<kDppQuadXor2>(s);
  if (G >= 64) s += dpp_f32<kDppRowHalfMirror>(s);
  if (G >= 128) s += dpp_f32<kDppRowMirror>(s);
  *to = nibble_order(u);
  if (piece % (G / 8) == 0) *sums = s;
}

// Up to MR = 8 or 16 rows: bound by the weights' bytes.  Of a workgroup's 8 waves, W share NT tiles of 16 columns and take
// the steps of 256 k's (whole 128-byte lines of each row) of every chunk of K in turn; they join through LDS.  A wave keeps
// the next chunk's weights in flight while it works on one.  x passes through LDS, two chunks of it: straight from the
// caches, a lane's 16 bytes lie a row away from its neighbour's, 64 accesses a load, and these bound the kernel (eight
// rows through 28,672 columns of 3,584: 30 us against 24; 22 today).
// What is left there, with a floor of 10 us for 55 MB of weights, scales and zeros: 224 workgroups leave 32 CUs without
// one, the two waves of a column take eight and six of its 14 steps, and the four steps that each asks for before its
// first product (57% of the weights) arrive behind a barrier for x, so loads and products hardly overlap.  One row of 4608 x
// 3584 takes 7.8 us against 1.6 for its bytes: of eight waves two take one step and the others two, the second chunk's
// x is staged behind a barrier after the first one's products, and seven rows of zeros are staged beside the one.
constexpr int kW4Waves = 8;
template <int NT, int W, int GROUP, int MR>
__global__ __launch_bounds__(64 * kW4Waves, 2) void gemm_w4_few(const W4Params p) {
  const Nibbles nibbles;
  constexpr int STEP = 256, SC = MR == 8 ? 8 : 4, CHUNK = STEP * SC, PW = SC / W;   // steps of a chunk, and of a wave in it
  constexpr int GB = 128 / GROUP, SPG = 4 / GB, GS = 2 * GB, GC = CHUNK / GROUP;    // groups per 128 k's, step, chunk
  constexpr int PIECES = CHUNK / 8, LROW = PIECES + 1, NX = MR * PIECES / (64 * kW4Waves);
  static_assert(W <= SC, "a wave needs a step in every chunk");
  __shared__ uint4 xt[2][MR * LROW];
  __shared__ float xs[2][GC][MR];
  __shared__ float join[kW4Waves / W][W > 1 ? W / 2 : 1][NT * 4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int w = wave % W, set = wave / W;
  const int n0 = (remap_block_id(blockIdx.x, gridDim.x) * (kW4Waves / W) + set) * 16 * NT;
  const int steps = (p.K + STEP - 1) / STEP, chunks = (steps + SC - 1) / SC, groups = p.K / GROUP;

  // lane constants beside a base that only the step moves (every operand is under 2 GiB)
  unsigned woff[NT], row[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const unsigned n = n0 + 16 * t + r < p.N ? n0 + 16 * t + r : p.N - 1;
    woff[t] = n * (p.K / 2) + (32 * g < p.K ? 16 * g : 0);     // K under 128: a lane past the row's end stays inside it
    row[t] = n * groups;
  }
  const int xr = r < MR ? r : MR - 1;                  // rows past p.M hold anything: they are not stored

  u32x4 wq[PW][NT][2];
  Groups<GS> gq[PW][NT];
  uint4 xq[NX];
  const auto load_w = [&](int s, u32x4 (&to)[NT][2], Groups<GS> (&gt)[NT]) {
    const uint8_t* wb = p.w + static_cast<size_t>(s) * (STEP / 2);
    const bool whole = (s + 1) * STEP <= p.K;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        // past the end: the row's first block again, for x's zeros there
        const bool in = whole || s * STEP + 128 * u + 32 * g < p.K;
        to[t][u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>((in ? wb + 64 * u : p.w) + woff[t]));
      }
      if (whole) gt[t].template load<false>(p, row[t], s * GS, groups);
      else gt[t].template load<true>(p, row[t], s * GS, groups);
    }
  };
  const auto load_x = [&](int c) {
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const int at = i * 64 * kW4Waves + threadIdx.x, m = at / PIECES, k = c * CHUNK + at % PIECES * 8;
      xq[i] = make_uint4(0, 0, 0, 0);
      if (m < p.M && k < p.K) xq[i] = *reinterpret_cast<const uint4*>(p.x + static_cast<size_t>(m) * p.K + k);
    }
  };
  const auto store_x = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const int at = i * 64 * kW4Waves + threadIdx.x, m = at / PIECES, piece = at % PIECES;
      stage_x<GROUP>(xq[i], piece, &xt[buf][m * LROW + piece], &xs[buf][piece / (GROUP / 8)][m]);
    }
  };

  f32x4 acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  load_x(0);
#pragma unroll
  for (int j = 0; j < PW; ++j)
    if (w * PW + j < steps) load_w(w * PW + j, wq[j], gq[j]);
  store_x(0);
  __syncthreads();
  for (int c = 0; c < chunks; ++c) {
    const int buf = c & 1;
    if (c + 1 < chunks) load_x(c + 1);
#pragma unroll
    for (int j = 0; j < PW; ++j) {
      const int s = c * SC + w * PW + j;
      if (s >= steps) break;
      uint32_t d[NT][2][4];
      Groups<GS> gc[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int q = 0; q < 4; ++q) d[t][u][q] = wq[j][t][u][q];
        gc[t] = gq[j][t];
      }
      // one step in flight: on its way while this one is worked on; more of them: no need to move this one out of its way
      if (PW == 1 && s + SC < steps) load_w(s + SC, wq[j], gq[j]);
      const uint4* xl = &xt[buf][xr * LROW + (w * PW + j) * (STEP / 8) + g];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint4 xa[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) xa[q] = xl[16 * u + 4 * q];
#pragma unroll
        for (int q = 0; q < GB; ++q) {
          const float4 x = *reinterpret_cast<const float4*>(&xs[buf][(w * PW + j) * GS + GB * u + q][(4 * g) % MR]);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if (q == 0) transpose_groups(d[t][u]);
            f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = q * SPG; e < (q + 1) * SPG; ++e) sum = mfma16(xa[e], nibbles(d[t][u][e]), sum);
            const float sg = gc[t].scale(GB * u + q), zg = gc[t].zero(p, GB * u + q);
            acc[t][0] = fmaf(sg, fmaf(-zg, x.x, sum[0]), acc[t][0]);
            acc[t][1] = fmaf(sg, fmaf(-zg, x.y, sum[1]), acc[t][1]);
            acc[t][2] = fmaf(sg, fmaf(-zg, x.z, sum[2]), acc[t][2]);
            acc[t][3] = fmaf(sg, fmaf(-zg, x.w, sum[3]), acc[t][3]);
          }
        }
      }
      if (PW > 1 && s + SC < steps) load_w(s + SC, wq[j], gq[j]);
    }
    if (c + 1 < chunks) store_x(buf ^ 1);
    __syncthreads();
  }

#pragma unroll
  for (int h = W / 2; h >= 1; h >>= 1) {
    if (w >= h && w < 2 * h) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) join[set][w - h][t * 4 + i][lane] = acc[t][i];
    }
    __syncthreads();
    if (w < h) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[t][i] += join[set][w][t * 4 + i][lane];
    }
    __syncthreads();
  }
  if (w != 0) return;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int n = n0 + 16 * t + r;
    const float bias = p.bias && n < p.N ? p.bias[n] : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = 4 * g + i;
      const float y = acc[t][i] + bias;
      const float pair = dpp_f32<kDppQuadXor1>(y);             // SwiGLU: the up value of an even lane's gate
      if (m < p.M && n < p.N && (p.mode != 2 || (n & 1) == 0)) w4_store(p, m, n, y, pair);
    }
  }
}

// More rows (16 MT at a time), or long rows of few columns: here x would be read far more often than the weights, so the 4
// waves of a workgroup take 32 columns each and share x through LDS, 256 k's at a time; workgroups split K where the
// columns give too few, and w4_join adds their sums.  48 rows of 3584 x 14336 take 27 us, 4 of them the join, against 5.3
// for 29 MB: 18 parts write 12.4 MB of sums and the join reads them again, some parts have four of the 56 steps and some three,
// and a step's load, stage, barrier and products come one after the other, about 6 us; two workgroups on a CU cover a
// third of that.  Two steps in flight gave nothing (29.4 us).
// Many rows are served, not meant: each 64 of them turn the weights into pairs again, 1,183 through 28,672 columns of 3,584
// run at 460 TFLOP/s, 10,677 at 520, where the bf16 product of such weights reaches 970 and 1,165; it is faster from
// about 32 rows on there, from 100 for 4608 x 3584 and from 256 for 3584 x 14336.
template <int MT, int GROUP>
__global__ __launch_bounds__(256, 2) void gemm_w4_rows(const W4Params p) {
  const Nibbles nibbles;
  constexpr int NT = 2, STEP = 256, GB = 128 / GROUP, SPG = 4 / GB, GS = 2 * GB, ROWS = 16 * MT;
  constexpr int PIECES = STEP / 8, LROW = PIECES + 1, NX = ROWS * PIECES / 256;
  __shared__ uint4 xt[2][ROWS * LROW];                 // [row][pieces of 8 k's]
  __shared__ float xs[2][GS][ROWS];                    // [group][row]
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
  const int id = remap_block_id(blockIdx.x, gridDim.x);
  const int n0 = (id % p.ntiles * 4 + w) * 16 * NT, split = id / p.ntiles, m0 = blockIdx.y * ROWS;
  const int steps = (p.K + STEP - 1) / STEP, groups = p.K / GROUP;
  const int s0 = static_cast<int>(static_cast<long long>(steps) * split / p.splits);
  const int s1 = static_cast<int>(static_cast<long long>(steps) * (split + 1) / p.splits);

  unsigned woff[NT], row[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const unsigned n = n0 + 16 * t + r < p.N ? n0 + 16 * t + r : p.N - 1;
    woff[t] = n * (p.K / 2) + (32 * g < p.K ? 16 * g : 0);     // K under 128: a lane past the row's end stays inside it
    row[t] = n * groups;
  }
  // x: thread t stages piece t % 32 of rows t / 32 + 8 i
  const int piece = threadIdx.x % PIECES, xr = threadIdx.x / PIECES;

  u32x4 wq[NT][2];
  uint4 xq[NX];
  Groups<GS> gq[NT];
  const auto load = [&](int s) {
    const uint8_t* wb = p.w + static_cast<size_t>(s) * (STEP / 2);
    const bool whole = (s + 1) * STEP <= p.K;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        // past the end: the row's first block again, for x's zeros there
        const bool in = whole || s * STEP + 128 * u + 32 * g < p.K;
        wq[t][u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>((in ? wb + 64 * u : p.w) + woff[t]));
      }
      if (whole) gq[t].template load<false>(p, row[t], s * GS, groups);
      else gq[t].template load<true>(p, row[t], s * GS, groups);
    }
    const int k = s * STEP + 8 * piece;
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const int m = m0 + xr + 8 * i;
      xq[i] = make_uint4(0, 0, 0, 0);
      if (m < p.M && k < p.K) xq[i] = *reinterpret_cast<const uint4*>(p.x + static_cast<size_t>(m) * p.K + k);
    }
  };
  const auto stage = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NX; ++i)
      stage_x<GROUP>(xq[i], piece, &xt[buf][(xr + 8 * i) * LROW + piece], &xs[buf][piece / (GROUP / 8)][xr + 8 * i]);
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[a][t] = f32x4{0.f, 0.f, 0.f, 0.f};

  load(s0);                                            // splits never exceed the steps
  for (int s = s0; s < s1; ++s) {
    const int buf = (s - s0) & 1;
    stage(buf);
    uint32_t d[NT][2][4];
    Groups<GS> gc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q) d[t][u][q] = wq[t][u][q];
      gc[t] = gq[t];
    }
    if (s + 1 < s1) load(s + 1);
    __syncthreads();                                   // the buffer is written again two steps on, past the next barrier
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int t = 0; t < NT; ++t) transpose_groups(d[t][u]);
#pragma unroll
      for (int q = 0; q < GB; ++q) {
        f32x4 sum[MT][NT];
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
          for (int t = 0; t < NT; ++t) sum[a][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = q * SPG; e < (q + 1) * SPG; ++e) {
          uint4 b[NT];
#pragma unroll
          for (int t = 0; t < NT; ++t) b[t] = nibbles(d[t][u][e]);
#pragma unroll
          for (int a = 0; a < MT; ++a) {
            const uint4 x = xt[buf][(16 * a + r) * LROW + 16 * u + 4 * e + g];
#pragma unroll
            for (int t = 0; t < NT; ++t) sum[a][t] = mfma16(x, b[t], sum[a][t]);
          }
        }
#pragma unroll
        for (int a = 0; a < MT; ++a) {
          const float4 x = *reinterpret_cast<const float4*>(&xs[buf][GB * u + q][16 * a + 4 * g]);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const float sg = gc[t].scale(GB * u + q), zg = gc[t].zero(p, GB * u + q);
            acc[a][t][0] = fmaf(sg, fmaf(-zg, x.x, sum[a][t][0]), acc[a][t][0]);
            acc[a][t][1] = fmaf(sg, fmaf(-zg, x.y, sum[a][t][1]), acc[a][t][1]);
            acc[a][t][2] = fmaf(sg, fmaf(-zg, x.z, sum[a][t][2]), acc[a][t][2]);
            acc[a][t][3] = fmaf(sg, fmaf(-zg, x.w, sum[a][t][3]), acc[a][t][3]);
          }
        }
      }
    }
  }
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
        const float pair = dpp_f32<kDppQuadXor1>(y);           // SwiGLU: the up value of an even lane's gate
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
    const float* from = p.part + static_cast<long long>(m) * p.N + n + c;
    const long long step = static_cast<long long>(p.M) * p.N;
    float s = 0.f;
    for (int k = 0; k < p.splits; k += 8) {
      float v[8];                                      // loads in flight together, summed in order
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = k + u < p.splits ? from[(k + u) * step] : 0.f;
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
    y[c] = s + (p.bias ? p.bias[n + c] : 0.f);
  }
  w4_store(p, m, n, y[0], y[per - 1]);
}

struct W4Plan {
  int mt, nt, waves, ntiles, splits;   // mt = 0: gemm_w4_few; ntiles: workgroups along the columns
};
// Only tiles and waves depend on the group: the parts' workspace is sized without it.  Times are of calls whose weights come from
// memory, groups of 128 where nothing else is said.
W4Plan plan_w4(int M, int N, int K, int group) {
  W4Plan a;
  a.splits = 1;
  const int tiles = (N + 15) / 16, steps = (K + 255) / 256;
  if (M <= 16) {
    a.mt = 0;
    // All the waves that share a chunk where columns are few (eight rows, 4096 x 8192: 12.2 us with eight, 14.5 with four; 16
    // rows, 5120 x 5120: 14.2 with four, 17.4 with two), half of them where there are columns enough (eight rows,
    // 18,944 x 3584: 16.6 us with four, 19.8 with eight; 16 rows: 19.7 with two, 21.8 with four).  Groups of 32 keep them all: what
    // their scales take of a wave outweighs the join (eight rows, 18,944 x 3584: 21.6 us with eight, 27.5 with four; 16
    // rows: 24.2 with four, 31.7 with two).
    const int most = M <= 8 ? 8 : 4;
    a.waves = group == 32 || tiles <= (M <= 8 ? 384 : 1024) ? most : most / 2;
    // Two tiles a wave, and two waves, where that leaves a little less than a workgroup for every CU (eight rows, 32,768 x
    // 3584: 20.8 us against 22.1, 26,640 x 3584: 20.4 and 21.1, 24,592 x 3584: 20.3 and 19.7; one row, 27,648 x 8192 in
    // groups of 64: 40.6 and 37.3).
    const bool wide = M > 4 && M <= 8 && group > 32 && tiles > 1664 && tiles <= 2048;
    a.nt = wide ? 2 : 1;
    if (wide) a.waves = 2;
    a.ntiles = ((tiles + a.nt - 1) / a.nt * a.waves + kW4Waves - 1) / kW4Waves;
    // gemm_w4_rows splits K over workgroups instead where all the waves that a column can have take four steps or more one
    // after the other, and K is long beside the columns (eight rows, 4096 x 14336: 16.4 us against 19.2, 6144 x 14336: 22.3
    // and 22.2, 6144 x 8192: 15.3 and 14.2; 16 rows, 8192 x 8192: 18.4 and 21.8, x 5120: 16.3 and 14.5, 12,800 x 14336: 39.4
    // and 41.1, 16,384 x 14336: 46.2 and 43.8).  With fewer steps its join costs more than it saves (eight rows, 4096 x
    // 5120: 11.8 against 8.8).
    const bool split = (steps + most - 1) / most >= 4 && tiles <= (M <= 8 ? 7 : 24) * steps && tiles <= (M <= 8 ? 384 : 800);
    // 257 to 340 workgroups of 9 to 16 rows are a second round for a few CUs, while three parts of gemm_w4_rows fit one: worth
    // it from 20 steps on (16 rows, 18,944 x 8192: 36.1 us against 41.7, 20,480 x 5120: 27.5 and 28.4, x 3584: 20.2 and
    // 19.9; 24,576 x 8192, two parts: 47.0 and 42.6).
    const bool round = M > 8 && tiles > 1024 && tiles <= 1360 && steps >= 20;
    if (!split && !round) return a;
  }
  // rows at a time: no more than there are (17 rows, 3584 x 14336: 20.5 us with 32, 25.2 with 64)
  a.mt = M <= 16 ? 1 : M <= 32 ? 2 : M <= 48 ? 3 : 4;
  a.nt = 2;
  a.ntiles = (N + 127) / 128;
  const int rows = (M + 63) / 64;
  // two workgroups on every CU (48 rows, 3584 x 14336: 27.6 us; 256 workgroups 29.0, 768 31.8), of two steps each (of an
  // odd number of steps, one part has a single one)
  const int s = 512 / (a.ntiles * rows), parts = (steps + 1) / 2;
  a.splits = s < 1 ? 1 : s < parts ? s : parts;
  return a;
}

size_t w4_bytes(const W4Plan& a, int M, int N) {
  return a.splits == 1 ? 0 : static_cast<size_t>(a.splits) * M * N * sizeof(float);
}

template <int NT, int W, int MR>
void launch_few(const W4Params& p, int group, hipStream_t stream) {
  const dim3 g(p.ntiles), th(64 * kW4Waves);
  if constexpr (W == (MR == 8 ? 8 : 4)) {
    if (group == 32) {
      hipLaunchKernelGGL((gemm_w4_few<NT, W, 32, MR>), g, th, 0, stream, p);
      return;
    }
  }
  if (group == 64) hipLaunchKernelGGL((gemm_w4_few<NT, W, 64, MR>), g, th, 0, stream, p);
  else hipLaunchKernelGGL((gemm_w4_few<NT, W, 128, MR>), g, th, 0, stream, p);
}
void launch_few(const W4Params& p, const W4Plan& a, int group, hipStream_t stream) {
  if (p.M > 8) a.waves == 4 ? launch_few<1, 4, 16>(p, group, stream) : launch_few<1, 2, 16>(p, group, stream);
  else if (a.nt == 2) launch_few<2, 2, 8>(p, group, stream);
  else a.waves == 8 ? launch_few<1, 8, 8>(p, group, stream) : launch_few<1, 4, 8>(p, group, stream);
}
template <int MT>
void launch_rows(const W4Params& p, int group, hipStream_t stream) {
  const dim3 g(p.ntiles * p.splits, (p.M + 16 * MT - 1) / (16 * MT)), th(256);
  if (group == 32) hipLaunchKernelGGL((gemm_w4_rows<MT, 32>), g, th, 0, stream, p);
  else if (group == 64) hipLaunchKernelGGL((gemm_w4_rows<MT, 64>), g, th, 0, stream, p);
  else hipLaunchKernelGGL((gemm_w4_rows<MT, 128>), g, th, 0, stream, p);
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" {

size_t pace_gemm_w4_workspace_size(int M, int N, int K) {
  const long long lim = 1ll << 31;
  if (M < 1 || N < 1 || K < 1 || 2ll * M * K >= lim || 2ll * M * N >= lim || (N + 15ll) / 16 * 16 * K / 2 >= lim) return 0;
  return w4_bytes(plan_w4(M, N, K, 128), M, N);
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
  // whole tiles of columns: a launch of one workgroup each then stays under 2^32 threads
  PACE_REQUIRE(2ll * M * K < lim && (N + 15ll) / 16 * 16 * K / 2 < lim && 2ll * N * (K / group) < lim &&
                   2ll * M * N < lim && M <= 65535,
               "pace_gemm_w4: an operand reaches 2 GiB, or M=%d is past 65,535", M);
  const W4Plan a = plan_w4(M, N, K, group);
  const size_t need = w4_bytes(a, M, N);
  if (need) {
    if (workspace == nullptr || workspace_bytes < need)
      return set_error(PACE_ERR_WORKSPACE, "pace_gemm_w4: workspace %zu < %zu bytes", workspace_bytes, need);
    PACE_REQUIRE(aligned16(workspace), "pace_gemm_w4: workspace must be 16-byte aligned");
  }
  const W4Params p{x, w, scale, zero, bias, residual, C, static_cast<float*>(workspace), M, N, K, epilogue, a.splits, a.ntiles};
  if (a.mt == 0) launch_few(p, a, group, stream);
  else if (a.mt == 1) launch_rows<1>(p, group, stream);
  else if (a.mt == 2) launch_rows<2>(p, group, stream);
  else if (a.mt == 3) launch_rows<3>(p, group, stream);
  else launch_rows<4>(p, group, stream);
  if (a.splits > 1)
    hipLaunchKernelGGL(w4_join, dim3(((epilogue == 2 ? N / 2 : N) + 255) / 256, M), dim3(256), 0, stream, p);
  return check_launch("pace_gemm_w4");
}

}  // extern "C"
