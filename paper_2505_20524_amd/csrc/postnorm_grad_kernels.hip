// The way back through the post-norm and its residual connection: the two gradients that meet in the stream are added, the norm's output gradient is
// taken back to the sub-layer's result and cast for that sub-layer's products, and the gains' gradient is summed over the rows.
//
// Bound by memory: 6 bytes read and 3 (5 with dy) written an element.  A row belongs to W waves that keep it in registers between the sums over
// it and its results, so that every tensor is read once.  A lane keeps its columns over all rows of its wave, so that the gains' gradient is summed in registers;
// a workgroup's waves join in LDS, the workgroups' sums in a second launch, in a fixed order: the same bits on every run.
// 8192 x 4096: 55 us (5.4 TB/s) and 5 us for the second launch; 777 x 2064: 9 to 9.5 us and 4.5.
#include <cfloat>

#include "common.h"
#include "launch.h"
#include "layout.h"

namespace {

constexpr int kThreads = 512;
constexpr int WAVES = kThreads / 64;
constexpr int GROUPS = 512;              // most workgroups, two a CU: one row of sums and one abs-max each in the workspace
constexpr int COLS_MAX = 512 * 8 * WAVES;

struct Args {
  const uint16_t *dres, *dbranch, *y;
  const float *gamma, *scale;
  uint16_t *dstream, *dy;
  uint8_t* q;
  float* sums;             // [workgroups][cols], or NULL
  uint32_t* tops;          // [workgroups], or NULL
  int64_t ld_dres, ld_dbranch, ldy, ld_dstream, ld_dy, ldq, rows;
  int cols;
};

FOG_DEVICE void unpack8(uint4 v, float (&f)[8]) {
  f[0] = bf16lo(v.x); f[1] = bf16hi(v.x); f[2] = bf16lo(v.y); f[3] = bf16hi(v.y);
  f[4] = bf16lo(v.z); f[5] = bf16hi(v.z); f[6] = bf16lo(v.w); f[7] = bf16hi(v.w);
}
FOG_DEVICE uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
FOG_DEVICE uint4 fetch(const uint16_t* p, int n) { return n >= 8 ? ld_any_nt16(p) : ld_upto8(p, n); }
FOG_DEVICE void put(uint16_t* p, uint4 w, int n) {
  if (n >= 8) st_any_nt16(p, w);
  else st_upto8(p, w, n);
}
typedef u32x2 __attribute__((aligned(1))) u32x2_byte;
FOG_DEVICE void put_codes(uint8_t* p, uint2 w, int n) {
  if (n >= 8) {
    u32x2 v = {w.x, w.y};
    *reinterpret_cast<u32x2_byte*>(p) = v;
  } else {
    st_upto8(p, w, n);
  }
}
FOG_DEVICE void gains8(const float* p, int n, float (&g)[8]) {
  if (n >= 8) {
    const uint4 a = ld_any16(p), b = ld_any16(p + 4);
    g[0] = __uint_as_float(a.x); g[1] = __uint_as_float(a.y); g[2] = __uint_as_float(a.z); g[3] = __uint_as_float(a.w);
    g[4] = __uint_as_float(b.x); g[5] = __uint_as_float(b.y); g[6] = __uint_as_float(b.z); g[7] = __uint_as_float(b.w);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) g[k] = k < n ? p[k] : 0.0f;
  }
}

template <int FMT, int W, int C>
__global__ __launch_bounds__(kThreads) void postnorm_grad_kernel(Args a) {
  constexpr int ROWS = WAVES / W;           // rows of a workgroup at a time
  constexpr int WIDTH = 512 * C * W;        // most columns
  __shared__ __attribute__((aligned(16))) float joined[ROWS > 1 ? ROWS * WIDTH : 4];
  __shared__ float part[2][WAVES][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % W;
  const float rho = a.q ? *a.scale : 0.0f;
  const float cols = (float)a.cols;
  float sum[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[c][k] = 0.0f;
  // The gains of the lane's columns stay in registers where these suffice: the rows that stream through push them out of the first cache (8192 x 4096: 65 -> 60 us).
  constexpr bool KEPT = C <= 2;
  float kept[KEPT ? C : 1][8];
  if (KEPT) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (64 * (c * W + w) + lane);
      gains8(a.gamma + col, a.cols - col, kept[KEPT ? c : 0]);
    }
  }
  auto gains = [&](int c, int n, float (&g)[8]) {
    if (KEPT) {
#pragma unroll
      for (int k = 0; k < 8; ++k) g[k] = kept[KEPT ? c : 0][k];
    } else {
      gains8(a.gamma + 8 * (64 * (c * W + w) + lane), n, g);
    }
  };
  uint32_t top = 0u;
  int turn = 0;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t r = (int64_t)blockIdx.x * ROWS + wave / W;
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.rows; r0 += step, r += step, turn ^= 1) {
    const bool there = r < a.rows;
    uint4 y[C], G[C], b[C];
    float yy = 0.0f, ty = 0.0f;
    if (there) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = 8 * (64 * (c * W + w) + lane), n = a.cols - col;
        y[c] = G[c] = b[c] = make_uint4(0, 0, 0, 0);
        if (n > 0) {
          y[c] = fetch(a.y + r * a.ldy + col, n);
          G[c] = fetch(a.dres + r * a.ld_dres + col, n);
          if (a.dbranch) b[c] = fetch(a.dbranch + r * a.ld_dbranch + col, n);
        }
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = 8 * (64 * (c * W + w) + lane), n = a.cols - col;
        if (n <= 0) continue;
        float f[8], h[8], g[8];
        unpack8(G[c], f);
        if (a.dbranch) {
          unpack8(b[c], h);
#pragma unroll
          for (int k = 0; k < 8; ++k) f[k] += h[k];
          G[c] = pack8(f);
          unpack8(G[c], f);
        }
        if (a.dstream) put(a.dstream + r * a.ld_dstream + col, G[c], n);
        unpack8(y[c], h);
        gains(c, n, g);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          yy = __builtin_fmaf(h[k], h[k], yy);
          ty = __builtin_fmaf(f[k] * g[k], h[k], ty);
        }
      }
    }
    yy = wave_sum_f32(yy);
    ty = wave_sum_f32(ty);
    if (W > 1) {
      // two sets of words in turn: a wave that is a row ahead writes the other one
      if (lane == 0) { part[turn][wave][0] = yy; part[turn][wave][1] = ty; }
      __syncthreads();
      yy = ty = 0.0f;
#pragma unroll
      for (int i = 0; i < W; ++i) { yy += part[turn][wave - w + i][0]; ty += part[turn][wave - w + i][1]; }
    }
    if (!there) continue;
    // 1 / rms, correctly rounded square root and divisions; a row of zeros, or of numbers whose squares vanish, gets no gradient
    const float mean = yy / cols, inv = mean != 0.0f ? 1.0f / __builtin_sqrtf(mean) : 0.0f, along = inv != 0.0f ? ty / yy : 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = 8 * (64 * (c * W + w) + lane), n = a.cols - col;
      if (n <= 0) continue;
      float f[8], h[8], g[8];
      unpack8(G[c], f);
      unpack8(y[c], h);
      gains(c, n, g);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        sum[c][k] = __builtin_fmaf(f[k], h[k] * inv, sum[c][k]);
        f[k] = inv * __builtin_fmaf(-h[k], along, f[k] * g[k]);
      }
      const uint4 o = pack8(f);
      top = pkmax_abs_bf16(top, o.x); top = pkmax_abs_bf16(top, o.y); top = pkmax_abs_bf16(top, o.z); top = pkmax_abs_bf16(top, o.w);
      if (a.dy) put(a.dy + r * a.ld_dy + col, o, n);
      if (a.q) {
        unpack8(o, f);
        put_codes(a.q + r * a.ldq + col, make_uint2(cvt4_fp8_nan<FMT>(f[0] * rho, f[1] * rho, f[2] * rho, f[3] * rho),
                                                    cvt4_fp8_nan<FMT>(f[4] * rho, f[5] * rho, f[6] * rho, f[7] * rho)), n);
      }
    }
  }
  if (a.sums) {
    if (ROWS > 1) {
      // every set of waves leaves its sums in LDS; then each thread adds what the sets have for its columns, in order
#pragma unroll
      for (int c = 0; c < C; ++c) {
        float* to = joined + (wave / W) * WIDTH + 8 * (64 * (c * W + w) + lane);
        *reinterpret_cast<float4*>(to) = make_float4(sum[c][0], sum[c][1], sum[c][2], sum[c][3]);
        *reinterpret_cast<float4*>(to + 4) = make_float4(sum[c][4], sum[c][5], sum[c][6], sum[c][7]);
      }
      __syncthreads();
      float* out = a.sums + (int64_t)blockIdx.x * a.cols;
      for (int i = threadIdx.x; i < a.cols; i += kThreads) {
        float t = joined[i];
#pragma unroll
        for (int k = 1; k < ROWS; ++k) t += joined[k * WIDTH + i];
        out[i] = t;
      }
    } else {
      float* out = a.sums + (int64_t)blockIdx.x * a.cols;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int col = 8 * (64 * (c * W + w) + lane);
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (col + k < a.cols) out[col + k] = sum[c][k];
      }
    }
  }
  if (a.tops) {
    __shared__ uint32_t tops[WAVES];
    const uint32_t m = wave_max_u32(max_of_pair(top));
    if (lane == 0) tops[wave] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t t = tops[0];
#pragma unroll
      for (int i = 1; i < WAVES; ++i) t = t > tops[i] ? t : tops[i];
      a.tops[blockIdx.x] = t << 16;      // the float with that bf16 pattern
    }
  }
}

// The gains' gradient from the workgroups' sums: 32 columns a workgroup, four to a thread and a row in every 128, added in order.
constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void postnorm_grad_join_kernel(const float* __restrict__ sums, const uint32_t* __restrict__ tops, int groups, int cols,
                                                                          float* __restrict__ dgamma, int accumulate, uint32_t* __restrict__ amax) {
  constexpr int SLICES = kJoinThreads / 8, LOADS = GROUPS / SLICES;
  __shared__ float part[SLICES][33];
  if (dgamma) {
    const int x = threadIdx.x & 7, z = threadIdx.x >> 3, col = (int)blockIdx.x * 32 + 4 * x, n = cols - col;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    uint4 v[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int g = z + i * SLICES;
      v[i] = make_uint4(0, 0, 0, 0);
      if (g < groups && n > 0) {
        const float* p = sums + (int64_t)g * cols + col;
        if (n >= 4) v[i] = ld_any16(p);
        else v[i] = make_uint4(__float_as_uint(p[0]), n > 1 ? __float_as_uint(p[1]) : 0u, n > 2 ? __float_as_uint(p[2]) : 0u, 0u);
      }
    }
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      s[0] += __uint_as_float(v[i].x); s[1] += __uint_as_float(v[i].y); s[2] += __uint_as_float(v[i].z); s[3] += __uint_as_float(v[i].w);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) part[z][4 * x + k] = s[k];
    __syncthreads();
    // 32 threads a column: four slices each, then the wave's halves by lane exchanges
    const int c = threadIdx.x >> 5, l = threadIdx.x & 31;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < SLICES / 32; ++i) t += part[l + 32 * i][c];
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) t += __shfl_xor(t, o, 64);
    const int to = (int)blockIdx.x * 32 + c;
    if (l == 0 && to < cols) dgamma[to] = accumulate ? dgamma[to] + t : t;
  }
  if (amax && blockIdx.x == 0 && threadIdx.x < 64) {
    uint32_t m = 0u;
    for (int i = threadIdx.x; i < groups; i += 64) m = m > tops[i] ? m : tops[i];
    m = wave_max_u32(m);
    if (threadIdx.x == 0) *amax = m;
  }
}

template <int FMT, int W, int C>
void launch(const Args& a, int groups, hipStream_t s) {
  postnorm_grad_kernel<FMT, W, C><<<groups, kThreads, 0, s>>>(a);
}

// Waves of a row, two chunks of eight a lane (16 sums of the gains' gradient); rows of more columns than eight waves hold so take four and eight chunks.
// (One wave up to 4096 columns, with eight chunks a lane and one workgroup a CU: 8192 x 4096 105 us a call instead of 64, 777 x 2064 35 instead of 14.)
int waves_of(int64_t cols) { return cols <= 1024 ? 1 : cols <= 2048 ? 2 : cols <= 4096 ? 4 : 8; }
int groups_of(int64_t rows, int64_t cols) {
  const int64_t n = WAVES / waves_of(cols), g = (rows + n - 1) / n;
  return (int)(g < GROUPS ? g : GROUPS);
}

}  // namespace

extern "C" size_t fog_postnorm_residual_grad_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || cols > COLS_MAX) return 0;
  return (size_t)groups_of(rows, cols) * ((size_t)cols * sizeof(float) + sizeof(uint32_t));
}

extern "C" fog_status fog_postnorm_residual_grad(const void* dres_bf16, int64_t ld_dres, const void* dbranch_bf16, int64_t ld_dbranch, const void* y_bf16,
                                                 int64_t ldy, int64_t rows, int64_t cols, const float* gamma, fog_fp8 fmt, const float* scale,
                                                 void* dstream_bf16, int64_t ld_dstream, void* dy_bf16, int64_t ld_dy, uint8_t* q, int64_t ldq, float* amax_out,
                                                 float* dgamma, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  if (rows < 0 || cols < 0) return FOG_ERR_SHAPE;
  if (fmt != FOG_E4M3 && fmt != FOG_E5M2) return FOG_ERR_UNSUPPORTED;
  if (cols > COLS_MAX) return FOG_ERR_UNSUPPORTED;
  if (q && !scale) return FOG_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(gamma) | reinterpret_cast<uintptr_t>(scale) | reinterpret_cast<uintptr_t>(amax_out) | reinterpret_cast<uintptr_t>(dgamma)) & 3)
    return FOG_ERR_ALIGN;
  hipStream_t s = (hipStream_t)stream;
  Args a = {};
  int groups = 0;
  if (rows > 0 && cols > 0) {
    if (!dres_bf16 || !y_bf16 || !gamma) return FOG_ERR_NULL;
    FogMatrices m;
    fog_status st = m.add(dres_bf16, rows, cols, ld_dres, 2, false);
    if (st == FOG_OK) st = m.add(dbranch_bf16, rows, cols, ld_dbranch, 2, false);
    if (st == FOG_OK) st = m.add(y_bf16, rows, cols, ldy, 2, false);
    if (st == FOG_OK) st = m.add(gamma, 1, cols, cols, 4, false);
    if (st == FOG_OK) st = m.add(dstream_bf16, rows, cols, ld_dstream, 2, true);
    if (st == FOG_OK) st = m.add(dy_bf16, rows, cols, ld_dy, 2, true);
    if (st == FOG_OK) st = m.add(q, rows, cols, ldq, 1, true);
    if (st == FOG_OK) st = m.add(dgamma, 1, cols, cols, 4, true);
    if (st != FOG_OK) return st;
    if (!m.fine()) return FOG_ERR_UNSUPPORTED;
    groups = groups_of(rows, cols);
    if (dgamma || amax_out) {
      if (!workspace || workspace_bytes < fog_postnorm_residual_grad_workspace(rows, cols)) return FOG_ERR_WORKSPACE;
      if (reinterpret_cast<uintptr_t>(workspace) & 3) return FOG_ERR_ALIGN;
    }
    float* sums = reinterpret_cast<float*>(workspace);
    a.dres = reinterpret_cast<const uint16_t*>(dres_bf16); a.dbranch = reinterpret_cast<const uint16_t*>(dbranch_bf16); a.y = reinterpret_cast<const uint16_t*>(y_bf16);
    a.gamma = gamma; a.scale = scale; a.dstream = reinterpret_cast<uint16_t*>(dstream_bf16); a.dy = reinterpret_cast<uint16_t*>(dy_bf16); a.q = q;
    a.sums = dgamma ? sums : nullptr;
    a.tops = amax_out ? reinterpret_cast<uint32_t*>(sums + (int64_t)groups * cols) : nullptr;
    a.ld_dres = ld_dres; a.ld_dbranch = ld_dbranch; a.ldy = ldy; a.ld_dstream = ld_dstream; a.ld_dy = ld_dy; a.ldq = ldq; a.rows = rows; a.cols = (int)cols;
#define FOG_PNG(W, C) (fmt == FOG_E4M3 ? launch<FOG_E4M3, W, C>(a, groups, s) : launch<FOG_E5M2, W, C>(a, groups, s))
    if (cols <= 512) FOG_PNG(1, 1);
    else if (cols <= 1024) FOG_PNG(1, 2);
    else if (cols <= 2048) FOG_PNG(2, 2);
    else if (cols <= 4096) FOG_PNG(4, 2);
    else if (cols <= 8192) FOG_PNG(8, 2);
    else if (cols <= 16384) FOG_PNG(8, 4);
    else FOG_PNG(8, 8);
#undef FOG_PNG
  } else if ((!dgamma || accumulate || cols == 0) && !amax_out) {
    return FOG_OK;
  }
  if ((dgamma && cols > 0) || amax_out) {
    const int64_t blocks = dgamma && cols > 0 ? (cols + 31) / 32 : 1;
    postnorm_grad_join_kernel<<<(int)blocks, kJoinThreads, 0, s>>>(a.sums, a.tops, groups, (int)cols, cols > 0 ? dgamma : nullptr, accumulate, reinterpret_cast<uint32_t*>(amax_out));
  }
  return fog_launch_status();
}
