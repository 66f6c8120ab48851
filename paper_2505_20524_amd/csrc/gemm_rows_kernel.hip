// Block-scaled product of a few rows (NT layout, M up to 32: the tokens of a decoding step) with a large weight: bound by reading B once.
//
// A workgroup owns 16 rows of B, its four waves split the contraction between them and add their binary32 sums through LDS in a fixed
// order.  Every wave works by itself, without a barrier before that: it brings its operands by direct loads (buffer_load ... lds) into a
// ring of two stages of its own, 256 contraction bytes of 16 rows of B and of A's rows each.  A load instruction covers 4 rows of 256
// bytes, whole lines.  (With lanes that fetched their own fragments from memory, each asking for a line of its own, 4096 x 4096 took
// 6.4 us with one row and 7.7 with 16, 14336 x 4096 14.2 and 19.2, 256 x 14336 with four 12.3.)  The sixteen 16-byte chunks of a row
// are turned by the row's number on the way, so that the fragment reads touch every bank once.
// The matrix instruction (16 x 16 x 128) takes one scale block: a lane's 32 bytes are a quarter of its row's block, its scale register
// holds that row's byte.  B is the first operand: a lane ends up with four consecutive columns of a row of C.
// us, weights that no call has just read (at the rate of a large read, 6.99 TB/s): one row of 4096 x 4096 6.1 (2.4), of 14336 x 4096 13.4 (8.4), of
// 4096 x 14336 13.2 (8.4); 24 rows of 4096 x 4096 7.6 (2.4).  Eight waves a workgroup: 6.8, 18.2, 13.4; three stages: 6.3, 14.4, 13.5.
#include "gemm_common.h"

namespace {

constexpr int STAGE_K = 2 * PAIR_K;               // contraction bytes of a stage: two scale blocks
constexpr int OPERAND = 16 * STAGE_K;             // 4 KB of B; a quarter of that for each four rows of A
constexpr int SCALE = 256;                        // a dword for each of 2 blocks x 16 rows, twice
constexpr int RING = 2, WAVES = 4;
template <int AP> constexpr int STAGE = OPERAND + 1024 * AP + 2 * SCALE;   // B, A, scales of A, scales of B
// the fragments of a group of 16 rows are read whole: behind the last stage lies room for the rows that A does not have
template <int AP> constexpr int LDS_OF = WAVES * RING * STAGE<AP> + 1024 * ((AP + 3) / 4 * 4 - AP);

// AP: pieces of four rows that A has.  Rows behind them are read from whatever lies there: they are rows of C that are not stored.
template <int FA, int FB, int AP>
__global__ __launch_bounds__(64 * WAVES) void fp8_gemm_rows_kernel(GemmArgs g) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63;
  const int n0 = blockIdx.x * 16;
  const v4i rsrc_a = make_rsrc(g.A, g.a_bytes), rsrc_b = make_rsrc(g.B, g.b_bytes);
  const v4i rsrc_sa = make_rsrc(g.sa.s, g.sa.bytes), rsrc_sb = make_rsrc(g.sb.s, g.sb.bytes);
  constexpr int LOADS = 4 + AP + 2, MB = (AP + 3) / 4;      // MB: groups of 16 rows of A
  uint8_t* mine = smem + w * (RING * STAGE<AP>);
  const uint32_t lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)mine);

  // this wave's scale blocks, two to a stage
  const int stages_all = (g.k_blocks + 1) / 2, share = (stages_all + WAVES - 1) / WAVES;
  const int first = w * share, end = min(first + share, stages_all);

  // piece j of an operand's stage: rows 4 j + l / 16, place l % 16 of a row in LDS holds chunk (l % 16) ^ (row % 16) of the stage
  uint32_t off_a[AP], off_b[4];
  int chunk[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int row = 4 * j + (l >> 4);
    chunk[j] = 16 * ((l & 15) ^ row);
    off_b[j] = n0 + row < g.N ? (uint32_t)((int64_t)(n0 + row) * g.ldb + chunk[j]) : OOB;
  }
#pragma unroll
  for (int j = 0; j < AP; ++j) {
    const int row = 4 * j + (l >> 4);
    off_a[j] = row < g.M ? (uint32_t)((int64_t)row * g.lda + chunk[j & 3]) : OOB;
  }
  // scale bytes: a dword for each row of the stage's first block, then of its second
  const int ablk = l / (16 * MB) & 1, arow = l % (16 * MB), bblk = (l >> 4) & 1, brow = l & 15;
  const uint32_t soff_a = arow < g.M ? (uint32_t)(arow >> g.sa.shift) * g.sa.i_stride : OOB;
  const uint32_t soff_b = n0 + brow < g.N ? (uint32_t)((n0 + brow) >> g.sb.shift) * g.sb.i_stride : OOB;
  auto issue = [&](int s, int slot) {
    const uint32_t k = (uint32_t)s * STAGE_K, at = lds + slot * STAGE<AP>;
#pragma unroll
    for (int j = 0; j < 4; ++j) load_to_lds(rsrc_b, s < end && (int)k + chunk[j] < g.K ? off_b[j] + k : OOB, at + 1024u * j);
#pragma unroll
    for (int j = 0; j < AP; ++j) load_to_lds(rsrc_a, s < end && (int)k + chunk[j & 3] < g.K ? off_a[j] + k : OOB, at + OPERAND + 1024u * j);
    const int ab = 2 * s + ablk, bb = 2 * s + bblk;
    load_byte_to_lds(rsrc_sa, s < end && ab < g.k_blocks ? soff_a + (uint32_t)ab * g.sa.k_stride : OOB, at + OPERAND + 1024 * AP);
    load_byte_to_lds(rsrc_sb, s < end && bb < g.k_blocks ? soff_b + (uint32_t)bb * g.sb.k_stride : OOB, at + OPERAND + 1024 * AP + SCALE);
  };
  const int frow = l & 15, fchunk = 2 * (l >> 4);
  auto frag = [&](const uint8_t* operand, int b) {
    const v4i lo = *reinterpret_cast<const v4i*>(operand + frow * STAGE_K + 16 * ((8 * b + fchunk) ^ frow));
    const v4i hi = *reinterpret_cast<const v4i*>(operand + frow * STAGE_K + 16 * ((8 * b + fchunk + 1) ^ frow));
    return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  };

  v4f acc[MB];
#pragma unroll
  for (int i = 0; i < MB; ++i) acc[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int r = 0; r < RING; ++r) issue(first + r, r);
  int slot = 0;
  for (int s = first; s < end; ++s) {
    // the oldest stage in flight has landed
    constexpr int LEFT = (RING - 1) * LOADS;
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | (7 << 4) | (15 << 8) | ((LEFT >> 4) << 14));
    asm volatile("" ::: "memory");
    const uint8_t* st = mine + slot * STAGE<AP>;
    v8i fa[2][MB], fb[2];
    int xa[2][MB], xb[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      fb[b] = frag(st, b);
      xb[b] = *reinterpret_cast<const int*>(st + OPERAND + 1024 * AP + SCALE + 4 * (16 * b + frow));
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        fa[b][i] = frag(st + OPERAND + 4096 * i, b);
        xa[b][i] = *reinterpret_cast<const int*>(st + OPERAND + 1024 * AP + 4 * (16 * (MB * b + i) + frow));
      }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt = 0: the slot has been read and may be refilled
    asm volatile("" ::: "memory");
    issue(s + RING, slot);
    slot = slot + 1 == RING ? 0 : slot + 1;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < MB; ++i)
        acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[b], fa[b][i], acc[i], FB, FA, 0, xb[b], 0, xa[b][i]);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);        // vmcnt = 0: no direct load may still be writing LDS
  __syncthreads();
  v4f* part = reinterpret_cast<v4f*>(smem);
#pragma unroll
  for (int i = 0; i < MB; ++i) part[(i * WAVES + w) * 64 + l] = acc[i];
  __syncthreads();
  // lane l holds row m = 16 i + l % 16 of C, columns n0 + 4 (l / 16) + 0 .. 3; wave i adds up group i
  if (w >= MB) return;
  v4f sum = part[w * WAVES * 64 + l];
#pragma unroll
  for (int v = 1; v < WAVES; ++v) sum += part[(w * WAVES + v) * 64 + l];
  const int m = 16 * w + (l & 15), n = n0 + 4 * (l >> 4);
  if (m >= g.M || n >= g.N) return;
  uint16_t* dst = g.C + (int64_t)m * g.ldc + n;
  const uint2 o = make_uint2(pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3]));
  if (g.vec_store) {                         // N % 4 == 0 there
    *reinterpret_cast<uint2*>(dst) = o;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < g.N) dst[e] = (uint16_t)((e < 2 ? o.x : o.y) >> (16 * (e & 1)));
  }
}

template <int FA, int FB, int AP>
fog_status launch(const GemmArgs& g, hipStream_t s) {
  static bool configured = false;  // per instantiation; the attribute is sticky for the process
  if (!configured) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(fp8_gemm_rows_kernel<FA, FB, AP>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS_OF<AP>) != hipSuccess)
      return FOG_ERR_HIP;
    configured = true;
  }
  fp8_gemm_rows_kernel<FA, FB, AP><<<(g.N + 15) / 16, 64 * WAVES, LDS_OF<AP>, s>>>(g);
  return fog_launch_status();
}
template <int FA, int FB>
fog_status launch_rows(const GemmArgs& g, hipStream_t s) {
  switch ((g.M + 3) / 4) {
    case 1: return launch<FA, FB, 1>(g, s);
    case 2: return launch<FA, FB, 2>(g, s);
    case 3: return launch<FA, FB, 3>(g, s);
    case 4: return launch<FA, FB, 4>(g, s);
    case 5: return launch<FA, FB, 5>(g, s);
    case 6: return launch<FA, FB, 6>(g, s);
    case 7: return launch<FA, FB, 7>(g, s);
    default: return launch<FA, FB, 8>(g, s);
  }
}

}  // namespace

// Every workgroup reads all of A, so that with more rows, or more workgroups than the chip holds at a time (47 to 68 KiB of LDS each up to 16
// rows, three or two on a compute unit; 79 to 100 above, two up to 20 rows and one from there), the tiles of fog_fp8_gemm do as well.  us,
// this kernel and the tiles:
//   8 rows   8192 x 512 4.2, 4.4   14336 x 512 6.3, 4.8   14336 x 2048 9.5, 9.4   14336 x 4096 14.3, 16.5   8192 x 8192 14.2, 22.3
//   16 rows  8192 x 512 4.6, 4.3   14336 x 2048 11.9, 9.6   14336 x 4096 16.9, 16.6   14336 x 14336 46.5, 41.4   4096 x 4096 7.1, 11.8
//   32 rows  2048 x 512 3.8, 3.9   4096 x 1024 4.9, 5.2   4096 x 4096 8.2, 12.0   8192 x 1024 7.4, 5.3   8192 x 4096 13.9, 13.6
// Weights so narrow that N / 16 workgroups leave compute units idle: this kernel, the tiles with their contraction split (which takes a
// workspace) and whole:
//   4 rows   256 x 1024 3.0, 4.6, 4.6   256 x 4096 3.8, 8.4, 8.5   256 x 14336 6.9, 9.5, 20.7   1024 x 4096 4.2, 8.7, 8.7   2048 x 14336 11, 13.9, 31.0
//   16 rows  1024 x 4096 4.7, 8.7, 8.7   1024 x 14336 11.5, 11.6, 30.9   2048 x 1024 4.0, 5.2, 5.2   2048 x 14336 13, 13.7, 31.5
//   32 rows  256 x 1024 3.9, 4.7, 4.7   1024 x 4096 5.9, 8.8, 8.8   256 x 14336 10.3, 9.8, 21.1   1024 x 14336 14.7, 11.5, 31.8   2048 x 14336 16.0, 14.0, 32.3
// (a wave walks its quarter of the contraction through two stages: latency).  The split tiles gain 1 to 3 us from 24 rows of the longest
// contraction on, for callers that bring the room; without it the tiles lose twice.
bool gemm_rows_takes(int64_t M, int64_t N, int64_t K, int cus) {
  if (M <= 16) return N <= 32 * (int64_t)cus || (M <= 8 && K >= 4096);
  return M <= 32 && N <= 16 * (int64_t)cus && K >= 1024;
}

fog_status gemm_rows_launch(fog_fp8 fmt_a, fog_fp8 fmt_b, GemmArgs g, hipStream_t s) {
  g.vec_store = g.N % 4 == 0 && g.ldc % 4 == 0 && (reinterpret_cast<uintptr_t>(g.C) & 7) == 0;
  if (fmt_a == FOG_E4M3) return fmt_b == FOG_E4M3 ? launch_rows<0, 0>(g, s) : launch_rows<0, 1>(g, s);
  return fmt_b == FOG_E4M3 ? launch_rows<1, 0>(g, s) : launch_rows<1, 1>(g, s);
}
