// Block-scaled product of a few rows (NT layout, M up to 64: the tokens of a decoding step) with a large weight: bound by reading B once.
//
// A wave takes NB groups of 16 rows of B and a share of the contraction; the eight waves of a workgroup split the contraction between
// them and add their binary32 sums through LDS in a fixed order.  Operands go from memory straight into the registers of the matrix
// instruction (16 x 16 x 128: a lane's 32 bytes are one quarter of a row's scale block, so that its scale register holds the
// byte of its row and block); no LDS stage lies between, because nothing of B is used twice.  All loads of UNROLL blocks are issued
// before the first is used.  B is the instruction's first operand: a lane ends up with four consecutive columns of a row of C.
#include "gemm_common.h"

namespace {

constexpr int kWaves = 8;

template <int FA, int FB, int MB, int NB>
__global__ __launch_bounds__(64 * kWaves) void fp8_gemm_rows_kernel(GemmArgs g) {
  constexpr int UNROLL = MB + NB <= 5 ? 4 : 2;    // scale blocks in flight, within the registers
  __shared__ v4f part[kWaves][MB * NB][64];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int n0 = blockIdx.x * 16 * NB;
  const int i16 = l & 15, k32 = 32 * (l >> 4);
  // rows outside the operands repeat the last one: their results are not stored
  const uint8_t* b[NB];
  const uint8_t* sb[NB];
  const uint8_t* a[MB];
  const uint8_t* sa[MB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int n = min(n0 + 16 * j + i16, g.N - 1);
    b[j] = g.B + (int64_t)n * g.ldb + k32;
    sb[j] = g.sb.s + (int64_t)(n >> g.sb.shift) * g.sb.i_stride;
  }
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int m = min(16 * i + i16, g.M - 1);
    a[i] = g.A + (int64_t)m * g.lda + k32;
    sa[i] = g.sa.s + (int64_t)(m >> g.sa.shift) * g.sa.i_stride;
  }
  v4f acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

  const int share = (g.k_blocks + kWaves - 1) / kWaves;
  const int first = w * share, end = min(first + share, g.k_blocks);
  auto frag = [&](const uint8_t* p, int kb) {      // K % 16 == 0: a 16-byte piece lies inside the row or outside
    const int64_t k = (int64_t)PAIR_K * kb;
    v4i lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
    if (k + k32 < g.K) lo = *reinterpret_cast<const v4i*>(p + k);
    if (k + k32 + 16 < g.K) hi = *reinterpret_cast<const v4i*>(p + k + 16);
    return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  };
  for (int kb = first; kb < end; kb += UNROLL) {
    v8i fb[UNROLL][NB], fa[UNROLL][MB];
    int xb[UNROLL][NB], xa[UNROLL][MB];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (kb + u >= end) break;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        fb[u][j] = frag(b[j], kb + u);
        xb[u][j] = sb[j][(int64_t)(kb + u) * g.sb.k_stride];
      }
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        fa[u][i] = frag(a[i], kb + u);
        xa[u][i] = sa[i][(int64_t)(kb + u) * g.sa.k_stride];
      }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (kb + u >= end) break;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < MB; ++i)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u][j], fa[u][i], acc[i][j], FB, FA, 0, xb[u][j], 0, xa[u][i]);
    }
  }
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) part[w][i * NB + j][l] = acc[i][j];
  __syncthreads();
  // lane l holds row m = 16 i + l % 16 of C, columns n0 + 16 j + 4 (l / 16) + 0 .. 3
  for (int b2 = w; b2 < MB * NB; b2 += kWaves) {
    const int i = b2 / NB, j = b2 - i * NB;
    v4f s = part[0][b2][l];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) s += part[v][b2][l];
    const int m = 16 * i + i16, n = n0 + 16 * j + 4 * (l >> 4);
    if (m < g.M && n < g.N) {
      uint16_t* dst = g.C + (int64_t)m * g.ldc + n;
      const uint2 o = make_uint2(pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3]));
      if (g.vec_store) {                     // N % 4 == 0 there
        *reinterpret_cast<uint2*>(dst) = o;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < g.N) dst[e] = (uint16_t)((e < 2 ? o.x : o.y) >> (16 * (e & 1)));
      }
    }
  }
}

template <int FA, int FB, int MB>
fog_status launch_nb(const GemmArgs& g, hipStream_t s) {
  const int cus = fog_compute_units(), groups = (g.N + 15) / 16;
  // two groups a wave halve the reads of A; only where that leaves a workgroup for every compute unit
  if (groups >= 2 * cus) fp8_gemm_rows_kernel<FA, FB, MB, 2><<<(groups + 1) / 2, 64 * kWaves, 0, s>>>(g);
  else                   fp8_gemm_rows_kernel<FA, FB, MB, 1><<<groups, 64 * kWaves, 0, s>>>(g);
  return fog_launch_status();
}
template <int FA, int FB>
fog_status launch_mb(const GemmArgs& g, hipStream_t s) {
  switch ((g.M + 15) / 16) {
    case 1: return launch_nb<FA, FB, 1>(g, s);
    case 2: return launch_nb<FA, FB, 2>(g, s);
    case 3: return launch_nb<FA, FB, 3>(g, s);
    default: return launch_nb<FA, FB, 4>(g, s);
  }
}

}  // namespace

fog_status gemm_rows_launch(fog_fp8 fmt_a, fog_fp8 fmt_b, GemmArgs g, hipStream_t s) {
  g.vec_store = g.vec_store || ((reinterpret_cast<uintptr_t>(g.C) & 7) == 0 && g.ldc % 4 == 0);
  g.vec_store = g.vec_store && g.N % 4 == 0;
  if (fmt_a == FOG_E4M3) return fmt_b == FOG_E4M3 ? launch_mb<0, 0>(g, s) : launch_mb<0, 1>(g, s);
  return fmt_b == FOG_E4M3 ? launch_mb<1, 0>(g, s) : launch_mb<1, 1>(g, s);
}
