// Casts to FP8 with a scale for each block of 128 elements: along a row, along a column, or for each 128 x 128 tile.
//
// The scale of a block is a power of two, 2^k with the largest k that keeps FP8MAX >= 2^margin 2^k max|x|, and is kept as the byte
// 127 - k of its reciprocal.  Multiplying by it is exact, so that the one rounding of an element is the cast's own, and the matrix
// instruction takes the byte as it is.  The price is up to one binary place of the format's range, not of its precision.
//
// One workgroup of 512 threads reads a tile of 128 x 128 elements once, 16 bytes a lane, 16 lanes a row, and keeps it in registers (16
// a thread): the maxima along rows are a reduction over 16 lanes, those along columns one over a thread's rows, the wave's four lanes
// of a column group and, through LDS, the waves.  Both forms of codes then come from the same registers: a tensor that a step
// multiplies along its rows and along its columns is read once for the two casts.  Bound by memory: 2 bytes read and 1 written (2 for
// both forms) per element.  us, launches from a graph (at the rates of a large read and a large fill, 6.99 and 6.86 TB/s): 8192 x 14336 rows 52
// (51), both 88 (68), tiles 53 (51); 1777 x 2064 rows 5.5 (1.6), both 6.8 (2.1).  Workgroups of 256 and of 1024 threads: 8192 x 14336 rows 55
// and 60, both 90 and 90, 1777 x 2064 both 7.8 and 6.7, 24 x 4096 rows 3.7 and 2.9 where these take 3.1.
// Rows that begin at any byte: 4096 x 4096 rows 16 us instead of 12, 8192 x 14336 rows 83 and both 184.
#include "common.h"
#include "launch.h"

namespace {

constexpr int BLK = 128;
constexpr int kThreads = 512;

struct BlockCastArgs {
  const uint16_t* x;
  uint8_t *q_row, *s_row, *q_col, *s_col;   // tile form: q_row, s_row
  int64_t ldx, ldq_row, lds_row, ldq_col, lds_col;
  int64_t rows, cols;
  int64_t tiles_c;
  int margin;
};

// k of the block's scale from the magnitude pattern of its abs-max (bf16 without sign; 0x7F80 and above: not finite)
template <int FMT>
FOG_DEVICE int block_exponent(uint32_t a, int margin) {
  if (a == 0u || a >= 0x7F80u) return 0;
  int e = (int)(a >> 7) - 127;
  uint32_t frac = a & 0x7Fu;
  if (a < 0x80u) {                  // subnormal: the leading one is the highest set bit
    const int top = 31 - __builtin_clz(a);
    e = top - 133;
    frac = (a << (7 - top)) & 0x7Fu;
  }
  // FP8MAX = 1.75 * 2^8 or 1.75 * 2^15; 1.75 has the fraction 0x60
  const int k = (FMT == FOG_E4M3 ? 8 : 15) - e - (frac > 0x60u ? 1 : 0) - margin;
  return k < -126 ? -126 : k > 126 ? 126 : k;
}
FOG_DEVICE float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// maximum of packed pairs of magnitudes over the lanes of a group of 16, to all of them
FOG_DEVICE uint32_t pkmax(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
}
FOG_DEVICE uint32_t max_over_16(uint32_t v) {
  v = pkmax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, true));   // row_ror:8, 4, 2, 1
  v = pkmax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x124, 0xF, 0xF, true));
  v = pkmax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x122, 0xF, 0xF, true));
  v = pkmax(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x121, 0xF, 0xF, true));
  return v;
}

// Eight elements under eight scales.  NAN_TEST: they may hold NaN (a block that is not finite).
template <int FMT, bool NAN_TEST>
FOG_DEVICE uint2 cast8(uint4 v, const float* f) {
  const float a = bf16lo(v.x) * f[0], b = bf16hi(v.x) * f[1], c = bf16lo(v.y) * f[2], d = bf16hi(v.y) * f[3];
  const float e = bf16lo(v.z) * f[4], g = bf16hi(v.z) * f[5], h = bf16lo(v.w) * f[6], i = bf16hi(v.w) * f[7];
  if (NAN_TEST) return make_uint2(cvt4_fp8_nan<FMT>(a, b, c, d), cvt4_fp8_nan<FMT>(e, g, h, i));
  return make_uint2(cvt4_fp8<FMT>(a, b, c, d), cvt4_fp8<FMT>(e, g, h, i));
}

// Codes are written through: the product that reads them next finds them in the memory-side cache, and nothing is left to write back
// while it runs (stored past the caches: a layer of 8192 x 2048 x 2048 forward and backward 152 us instead of 136, of 4096 x 4096 x 4096
// 217 and 205; the cast of 8192 x 12288 both ways by itself 72 and 75).
template <bool RAGGED>
FOG_DEVICE void store8(uint8_t* q, uint2 v, int n) {
  if (!RAGGED || n == 8) st_through8(q, v);
  else                   st_upto8(q, v, n);
}

// RAGGED: 8 does not divide the columns, and the last thread of a row takes its elements one by one.  STREAM: reads past the caches.
template <int FMT, bool ROW, bool COL, bool TILE, bool RAGGED, bool STREAM>
__global__ __launch_bounds__(kThreads) void block_cast_kernel(BlockCastArgs a) {
  constexpr int GROUP = kThreads / 16, PASSES = BLK / GROUP, WAVES = kThreads / 64;    // rows of a pass; pieces that a thread holds
  __shared__ uint32_t colmax[COL || TILE ? WAVES : 1][64];      // per wave: 128 columns' maxima in pairs
  __shared__ float colscale[COL ? BLK : 1];
  __shared__ uint8_t rowbyte[ROW ? BLK : 1];
  const int t = threadIdx.x, l = t & 63, w = t >> 6;
  const int64_t tr = (int64_t)blockIdx.x / a.tiles_c, tc = (int64_t)blockIdx.x - tr * a.tiles_c;
  const int64_t r0 = tr * BLK, c0 = tc * BLK;
  const int nrows = (int)(a.rows - r0 < BLK ? a.rows - r0 : BLK), ncols = (int)(a.cols - c0 < BLK ? a.cols - c0 : BLK);
  const int rr = t >> 4, cc = 8 * (t & 15);      // row of pass p: GROUP p + rr
  const int n = ncols - cc < 0 ? 0 : ncols - cc < 8 ? ncols - cc : 8;
  const uint16_t* x = a.x + (r0 + rr) * a.ldx + c0 + cc;

  uint4 v[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    v[p] = make_uint4(0, 0, 0, 0);
    if (GROUP * p + rr < nrows) {
      const uint16_t* from = x + GROUP * p * a.ldx;
      if (RAGGED && n < 8) v[p] = ld_upto8(from, n);
      else if (n > 0)      v[p] = STREAM ? ld_any_nt16(from) : ld_any16(from);
    }
  }
  // maxima of the columns: over a thread's rows, over the wave's four lanes of a column group, and through LDS over the waves
  if (COL || TILE) {
    uint32_t cm[4] = {0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      cm[0] = pkmax_abs_bf16(cm[0], v[p].x);
      cm[1] = pkmax_abs_bf16(cm[1], v[p].y);
      cm[2] = pkmax_abs_bf16(cm[2], v[p].z);
      cm[3] = pkmax_abs_bf16(cm[3], v[p].w);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      cm[i] = pkmax(cm[i], (uint32_t)__shfl_xor((int)cm[i], 16, 64));
      cm[i] = pkmax(cm[i], (uint32_t)__shfl_xor((int)cm[i], 32, 64));
    }
    if (l < 16) *reinterpret_cast<uint4*>(&colmax[w][4 * l]) = make_uint4(cm[0], cm[1], cm[2], cm[3]);
    __syncthreads();
  }
  int odd = 0;      // a column of the tile is not finite
  if (COL && t < 64) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) m = pkmax(m, colmax[i][t]);
    const int k0 = block_exponent<FMT>(m & 0xFFFFu, a.margin), k1 = block_exponent<FMT>(m >> 16, a.margin);
    // a scale with its sign bit set marks a column that is not finite
    colscale[2 * t] = (m & 0xFFFFu) >= 0x7F80u ? -1.0f : pow2(k0);
    colscale[2 * t + 1] = (m >> 16) >= 0x7F80u ? -1.0f : pow2(k1);
    uint8_t* s = a.s_col + tr * a.lds_col + c0 + 2 * t;
    if (2 * t < ncols) s[0] = (uint8_t)(127 - k0);
    if (2 * t + 1 < ncols) s[1] = (uint8_t)(127 - k1);
  }
  // rows: maxima over the 16 lanes that hold one
  if (ROW) {
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const uint32_t rowmax = max_of_pair(max_over_16(pkmax_abs_bf16(pkmax_abs_bf16(pkmax_abs_bf16(pkmax_abs_bf16(0u, v[p].x), v[p].y), v[p].z), v[p].w)));
      const int k = block_exponent<FMT>(rowmax, a.margin);
      const float f1 = pow2(k);
      const float f[8] = {f1, f1, f1, f1, f1, f1, f1, f1};
      const int r = GROUP * p + rr;
      if ((t & 15) == 0) rowbyte[r] = (uint8_t)(127 - k);
      if (r < nrows && n > 0) {
        const uint2 o = __builtin_expect(rowmax >= 0x7F80u, 0) ? cast8<FMT, true>(v[p], f) : cast8<FMT, false>(v[p], f);
        store8<RAGGED>(a.q_row + (r0 + r) * a.ldq_row + c0 + cc, o, n);
      }
    }
  }
  if (ROW || COL) __syncthreads();
  if (ROW && t < nrows) a.s_row[tc * a.lds_row + r0 + t] = rowbyte[t];
  if (COL) {
    const float4 lo = *reinterpret_cast<const float4*>(&colscale[cc]), hi = *reinterpret_cast<const float4*>(&colscale[cc + 4]);
    float f[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      odd |= f[i] < 0.0f;
      f[i] = fabsf(f[i]);
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = GROUP * p + rr;
      if (r < nrows && n > 0) {
        const uint2 o = __builtin_expect(odd, 0) ? cast8<FMT, true>(v[p], f) : cast8<FMT, false>(v[p], f);
        store8<RAGGED>(a.q_col + (r0 + r) * a.ldq_col + c0 + cc, o, n);
      }
    }
  }
  if (TILE) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) m = pkmax(m, colmax[i][l]);
    m = wave_max_u32(max_of_pair(m));
    const int k = block_exponent<FMT>(m, a.margin);
    const float f1 = pow2(k);
    const float f[8] = {f1, f1, f1, f1, f1, f1, f1, f1};
    if (t == 0) a.s_row[tr * a.lds_row + tc] = (uint8_t)(127 - k);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = GROUP * p + rr;
      if (r < nrows && n > 0) {
        const uint2 o = __builtin_expect(m >= 0x7F80u, 0) ? cast8<FMT, true>(v[p], f) : cast8<FMT, false>(v[p], f);
        store8<RAGGED>(a.q_row + (r0 + r) * a.ldq_row + c0 + cc, o, n);
      }
    }
  }
}

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <bool ROW, bool COL, bool TILE>
fog_status launch(BlockCastArgs a, fog_fp8 fmt, hipStream_t s) {
  a.tiles_c = (a.cols + BLK - 1) / BLK;
  const int64_t tiles = a.tiles_c * ((a.rows + BLK - 1) / BLK);
  // what the kernel before has left in the caches is worth finding up to about 16 M elements (past the caches and as ordinary loads: the layer of
  // 1777 x 3088 x 2064 86.0 and 81.5 us, 4096 x 8192 x 2048 forward 76.9 and 74.8, 4096 x 4096 x 4096 205 and 207, 8192 x 4096 x 14336 1180 and 1210)
  // (rows that begin inside a line share it with the row before: 4096 x 4097 both ways 24 us past the caches, 19.5 without)
  const bool ragged = a.cols % 8 != 0, stream = !ragged && a.rows * a.cols > ((int64_t)16 << 20);
  if (tiles >= (1 << 23)) return FOG_ERR_UNSUPPORTED;      // grids are counted in threads of 32 bits
#define FOG_BC(F, R, S) block_cast_kernel<F, ROW, COL, TILE, R, S><<<(int)tiles, kThreads, 0, s>>>(a)
#define FOG_BR(F)                                       \
  do {                                                  \
    if (ragged)      FOG_BC(F, true, false);            \
    else if (stream) FOG_BC(F, false, true);            \
    else             FOG_BC(F, false, false);           \
  } while (0)
  if (fmt == FOG_E4M3) FOG_BR(FOG_E4M3);
  else                 FOG_BR(FOG_E5M2);
#undef FOG_BR
#undef FOG_BC
  return fog_launch_status();
}

}  // namespace

extern "C" fog_status fog_quantize_block(const void* x_bf16, int64_t rows, int64_t cols, int64_t ldx, fog_fp8 fmt, int margin,
                                         uint8_t* q_row, int64_t ldq_row, uint8_t* s_row, int64_t lds_row,
                                         uint8_t* q_col, int64_t ldq_col, uint8_t* s_col, int64_t lds_col, void* stream) {
  if (rows < 0 || cols < 0 || margin < -64 || margin > 64) return FOG_ERR_SHAPE;
  if (fmt != FOG_E4M3 && fmt != FOG_E5M2) return FOG_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return FOG_OK;
  if (!x_bf16 || (!q_row && !q_col) || (!q_row) != (!s_row) || (!q_col) != (!s_col)) return FOG_ERR_NULL;
  if (ldx < cols || (q_row && (ldq_row < cols || lds_row < rows)) || (q_col && (ldq_col < cols || lds_col < cols))) return FOG_ERR_SHAPE;
  if (!aligned(x_bf16, 2)) return FOG_ERR_ALIGN;
  const BlockCastArgs a{reinterpret_cast<const uint16_t*>(x_bf16), q_row, s_row, q_col, s_col, ldx, ldq_row, lds_row, ldq_col, lds_col, rows, cols, 0, margin};
  hipStream_t s = (hipStream_t)stream;
  if (q_row && q_col) return launch<true, true, false>(a, fmt, s);
  return q_row ? launch<true, false, false>(a, fmt, s) : launch<false, true, false>(a, fmt, s);
}

extern "C" fog_status fog_quantize_tile(const void* x_bf16, int64_t rows, int64_t cols, int64_t ldx, fog_fp8 fmt, int margin,
                                        uint8_t* q, int64_t ldq, uint8_t* s, int64_t lds, void* stream) {
  if (rows < 0 || cols < 0 || margin < -64 || margin > 64) return FOG_ERR_SHAPE;
  if (fmt != FOG_E4M3 && fmt != FOG_E5M2) return FOG_ERR_UNSUPPORTED;
  if (rows == 0 || cols == 0) return FOG_OK;
  if (!x_bf16 || !q || !s) return FOG_ERR_NULL;
  if (ldx < cols || ldq < cols || lds < (cols + BLK - 1) / BLK) return FOG_ERR_SHAPE;
  if (!aligned(x_bf16, 2)) return FOG_ERR_ALIGN;
  const BlockCastArgs a{reinterpret_cast<const uint16_t*>(x_bf16), q, s, nullptr, nullptr, ldx, ldq, lds, 0, 0, rows, cols, 0, margin};
  return launch<false, false, true>(a, fmt, (hipStream_t)stream);
}
