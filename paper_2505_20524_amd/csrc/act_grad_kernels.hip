// The gradients of the activations, on the way back between the two products of the feed-forward half (tanh: in front of attention): dx = dy f'(x), its cast for
// the products, and the sums that the activation's own parameters get.
//
// Bound by memory: 4 bytes read and 1 (3 with dx) written an element.
#include <cfloat>

#include "act_functions.h"
#include "common.h"
#include "launch.h"
#include "layout.h"

namespace {

constexpr int kThreads = 256;
constexpr int GROUPS = 2048;             // most workgroups: two sums and an abs-max each in the workspace

// f'(x), and what dy is multiplied by in the parameters' sums.
template <int ACT>
FOG_DEVICE float slope(float x, float p0, float p1, float& g0, float& g1) {
  g0 = g1 = 0.0f;
  if (ACT == ACT_XIELU) {
    float q = kExpm1Poly[4];
#pragma unroll
    for (int i = 3; i >= 0; --i) q = __builtin_fmaf(q, x, kExpm1Poly[i]);
    const float e = __builtin_amdgcn_exp2f(x * 1.44269504088896340736f) - 1.0f;
    const bool near = x > kExpm1Switch;
    const float curve = near ? x * x * q : e - x;                        // e^x - 1 - x
    if (x > 0.0f) {
      g0 = x * x;
      return __builtin_fmaf(2.0f * p0, x, 0.5f);
    }
    g1 = curve;
    return __builtin_fmaf(p1, near ? x + curve : e, 0.5f);
  }
  if (ACT == ACT_GELU) {
    // Phi(x) + x phi(x); for negative x both terms by the tail's exponential, which keeps their places
    const float t = fminf(fabsf(x), 14.0f);
    const float rinv = __builtin_amdgcn_rcpf(t + kTailK);
    const float u = (t - kTailK) * rinv;
    float p = kTailPoly[10];
#pragma unroll
    for (int i = 9; i >= 0; --i) p = __builtin_fmaf(p, u, kTailPoly[i]);
    const float e = __builtin_amdgcn_exp2f(t * t * -0.72134752044448170368f);
    const float tail = e * __builtin_fmaf(t, -0.39894228040143267794f, p * rinv);      // Phi(-t) - t phi(t)
    const float s = x < 0.0f ? tail : 1.0f - tail;
    return x != x ? x : s;
  }
  // alpha sech^2(alpha x) = alpha 4 e / (1 + e)^2 with e = e^(-2 |alpha x|)
  const float e = __builtin_amdgcn_exp2f(fabsf(p0 * x) * -2.88539008177792681472f);
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  const float s = 4.0f * e * r * r;
  g0 = x * s;
  return p0 * s;
}

struct Args {
  const uint16_t *x, *dy;
  const float* scale;
  uint16_t* dx;
  uint8_t* q;
  double* sums;            // [workgroups][2], or NULL
  uint32_t* tops;          // [workgroups], or NULL
  int64_t ldx, ld_dy, ld_dx, ldq, rows, cols, chunks;      // chunks: of eight elements in a row
  float p0, p1;
};

FOG_DEVICE void unpack8(uint4 v, float (&f)[8]) {
  f[0] = bf16lo(v.x); f[1] = bf16hi(v.x); f[2] = bf16lo(v.y); f[3] = bf16hi(v.y);
  f[4] = bf16lo(v.z); f[5] = bf16hi(v.z); f[6] = bf16lo(v.w); f[7] = bf16hi(v.w);
}
typedef u32x2 __attribute__((aligned(1))) u32x2_byte;

template <int ACT, int FMT>
__global__ __launch_bounds__(kThreads) void act_grad_kernel(Args a) {
  constexpr int U = 2;                   // chunks in flight
  const float rho = a.q ? *a.scale : 0.0f;
  const int64_t total = a.rows * a.chunks, stride = (int64_t)gridDim.x * kThreads;
  double s0 = 0.0, s1 = 0.0;
  uint32_t top = 0u;
  for (int64_t i0 = (int64_t)blockIdx.x * kThreads + threadIdx.x; i0 < total; i0 += U * stride) {
    uint4 vx[U], vd[U];
    int64_t r[U], c[U];
    int n[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * stride;
      r[u] = 0; c[u] = 8 * i; n[u] = 0;
      if (a.rows > 1 && i < total) {
        r[u] = total <= 0xFFFFFFFF ? (int64_t)((uint32_t)i / (uint32_t)a.chunks) : i / a.chunks;
        c[u] = 8 * (i - r[u] * a.chunks);
      }
      vx[u] = vd[u] = make_uint4(0, 0, 0, 0);
      if (i < total) {
        n[u] = a.cols - c[u] < 8 ? (int)(a.cols - c[u]) : 8;
        const uint16_t *x = a.x + r[u] * a.ldx + c[u], *dy = a.dy + r[u] * a.ld_dy + c[u];
        vx[u] = n[u] >= 8 ? ld_any_nt16(x) : ld_upto8(x, n[u]);
        vd[u] = n[u] >= 8 ? ld_any_nt16(dy) : ld_upto8(dy, n[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (n[u] == 0) break;
      float x[8], d[8], t0 = 0.0f, t1 = 0.0f;
      unpack8(vx[u], x);
      unpack8(vd[u], d);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float g0, g1;
        const float s = slope<ACT>(x[k], a.p0, a.p1, g0, g1);
        if (ACT != ACT_GELU) t0 = __builtin_fmaf(d[k], g0, t0);
        if (ACT == ACT_XIELU) t1 = __builtin_fmaf(d[k], g1, t1);
        d[k] *= s;
      }
      s0 += (double)t0;
      s1 += (double)t1;
      const uint4 o = make_uint4(pack_bf16x2(d[0], d[1]), pack_bf16x2(d[2], d[3]), pack_bf16x2(d[4], d[5]), pack_bf16x2(d[6], d[7]));
      top = pkmax_abs_bf16(top, o.x); top = pkmax_abs_bf16(top, o.y); top = pkmax_abs_bf16(top, o.z); top = pkmax_abs_bf16(top, o.w);
      if (a.dx) {
        uint16_t* to = a.dx + r[u] * a.ld_dx + c[u];
        if (n[u] >= 8) st_any_nt16(to, o);
        else st_upto8(to, o, n[u]);
      }
      if (a.q) {
        unpack8(o, d);
        const uint2 w = make_uint2(cvt4_fp8_nan<FMT>(d[0] * rho, d[1] * rho, d[2] * rho, d[3] * rho), cvt4_fp8_nan<FMT>(d[4] * rho, d[5] * rho, d[6] * rho, d[7] * rho));
        uint8_t* to = a.q + r[u] * a.ldq + c[u];
        if (n[u] >= 8) {
          u32x2 v = {w.x, w.y};
          *reinterpret_cast<u32x2_byte*>(to) = v;
        } else {
          st_upto8(to, w, n[u]);
        }
      }
    }
  }
  if (a.sums) {
    __shared__ double part[kThreads / 64][2];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) { s0 += __shfl_xor(s0, o, 64); s1 += __shfl_xor(s1, o, 64); }
    if ((threadIdx.x & 63) == 0) { part[threadIdx.x >> 6][0] = s0; part[threadIdx.x >> 6][1] = s1; }
    __syncthreads();
    if (threadIdx.x < 2) a.sums[2 * blockIdx.x + threadIdx.x] = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
  }
  if (a.tops) {
    __shared__ uint32_t tops[kThreads / 64];
    const uint32_t m = wave_max_u32(max_of_pair(top));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t t = tops[0];
#pragma unroll
      for (int w = 1; w < kThreads / 64; ++w) t = t > tops[w] ? t : tops[w];
      a.tops[blockIdx.x] = t << 16;      // the float with that bf16 pattern
    }
  }
}

// The workgroups' sums in order, and the largest of their maxima.
constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void act_grad_join_kernel(const double* __restrict__ sums, const uint32_t* __restrict__ tops, int groups, int count,
                                                                     float* __restrict__ dalpha, int accumulate, uint32_t* __restrict__ amax) {
  __shared__ double part[kJoinThreads / 64][2];
  __shared__ uint32_t most[kJoinThreads / 64];
  double s0 = 0.0, s1 = 0.0;
  uint32_t m = 0u;
  for (int i = threadIdx.x; i < groups; i += kJoinThreads) {
    if (dalpha) { s0 += sums[2 * i]; s1 += sums[2 * i + 1]; }
    if (amax) m = m > tops[i] ? m : tops[i];
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) { s0 += __shfl_xor(s0, o, 64); s1 += __shfl_xor(s1, o, 64); }
  m = wave_max_u32(m);
  if ((threadIdx.x & 63) == 0) { part[threadIdx.x >> 6][0] = s0; part[threadIdx.x >> 6][1] = s1; most[threadIdx.x >> 6] = m; }
  __syncthreads();
  if (threadIdx.x == 0) {
    s0 = s1 = 0.0;
    for (int w = 0; w < kJoinThreads / 64; ++w) { s0 += part[w][0]; s1 += part[w][1]; m = m > most[w] ? m : most[w]; }
    if (dalpha) {
      dalpha[0] = (float)((accumulate ? (double)dalpha[0] : 0.0) + s0);
      if (count > 1) dalpha[1] = (float)((accumulate ? (double)dalpha[1] : 0.0) + s1);
    }
    if (amax) *amax = m;
  }
}

template <int ACT>
fog_status act_grad(const void* x_bf16, int64_t ldx, const void* dy_bf16, int64_t ld_dy, int64_t rows, int64_t cols, float p0, float p1, fog_fp8 fmt,
                    const float* scale, void* dx_bf16, int64_t ld_dx, uint8_t* q, int64_t ldq, float* amax_out, float* dalpha, int accumulate, void* workspace,
                    size_t workspace_bytes, void* stream) {
  constexpr int COUNT = ACT == ACT_XIELU ? 2 : 1;
  if (rows < 0 || cols < 0) return FOG_ERR_SHAPE;
  if (fmt != FOG_E4M3 && fmt != FOG_E5M2) return FOG_ERR_UNSUPPORTED;
  if (q && !scale) return FOG_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(scale) | reinterpret_cast<uintptr_t>(amax_out) | reinterpret_cast<uintptr_t>(dalpha)) & 3) return FOG_ERR_ALIGN;
  hipStream_t s = (hipStream_t)stream;
  Args a = {};
  int groups = 0;
  if (rows > 0 && cols > 0) {
    if (!x_bf16 || !dy_bf16) return FOG_ERR_NULL;
    if ((double)rows * (double)cols > 140737488355328.0) return FOG_ERR_UNSUPPORTED;      // 2^47: more than an address space holds
    FogMatrices m;
    fog_status st = m.add(x_bf16, rows, cols, ldx, 2, false);
    if (st == FOG_OK) st = m.add(dy_bf16, rows, cols, ld_dy, 2, false);
    if (st == FOG_OK) st = m.add(dx_bf16, rows, cols, ld_dx, 2, true);
    if (st == FOG_OK) st = m.add(q, rows, cols, ldq, 1, true);
    if (st != FOG_OK) return st;
    if (!m.fine()) return FOG_ERR_UNSUPPORTED;
    if (dalpha || amax_out) {
      if (!workspace || workspace_bytes < fog_act_grad_workspace()) return FOG_ERR_WORKSPACE;
      if (reinterpret_cast<uintptr_t>(workspace) & 7) return FOG_ERR_ALIGN;
    }
    a.x = reinterpret_cast<const uint16_t*>(x_bf16); a.dy = reinterpret_cast<const uint16_t*>(dy_bf16); a.scale = scale;
    a.dx = reinterpret_cast<uint16_t*>(dx_bf16); a.q = q;
    a.sums = dalpha ? reinterpret_cast<double*>(workspace) : nullptr;
    a.tops = amax_out ? reinterpret_cast<uint32_t*>(reinterpret_cast<double*>(workspace) + 2 * GROUPS) : nullptr;
    a.ldx = ldx; a.ld_dy = ld_dy; a.ld_dx = ld_dx; a.ldq = ldq; a.rows = rows; a.cols = cols; a.p0 = p0; a.p1 = p1;
    if (rows == 1 || (ldx == cols && ld_dy == cols && (!dx_bf16 || ld_dx == cols) && (!q || ldq == cols))) {      // end to end: one long row
      a.cols = rows * cols;
      a.rows = 1;
    }
    a.chunks = (a.cols + 7) / 8;
    const int64_t want = (a.rows * a.chunks + 2 * kThreads - 1) / (2 * kThreads);
    groups = (int)(want < GROUPS ? want : GROUPS);
    if (fmt == FOG_E4M3) act_grad_kernel<ACT, FOG_E4M3><<<groups, kThreads, 0, s>>>(a);
    else                 act_grad_kernel<ACT, FOG_E5M2><<<groups, kThreads, 0, s>>>(a);
  } else if ((!dalpha || accumulate) && !amax_out) {
    return FOG_OK;
  }
  if (dalpha || amax_out)
    act_grad_join_kernel<<<1, kJoinThreads, 0, s>>>(a.sums, a.tops, groups, COUNT, dalpha, accumulate, reinterpret_cast<uint32_t*>(amax_out));
  return fog_launch_status();
}

}  // namespace

extern "C" size_t fog_act_grad_workspace(void) { return GROUPS * (2 * sizeof(double) + sizeof(uint32_t)); }

extern "C" fog_status fog_xielu_grad(const void* x_bf16, int64_t ldx, const void* dy_bf16, int64_t ld_dy, int64_t rows, int64_t cols, float alpha_p, float alpha_n,
                                     fog_fp8 fmt, const float* scale, void* dx_bf16, int64_t ld_dx, uint8_t* q, int64_t ldq, float* amax_out, float* dalpha,
                                     int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  if (!(alpha_p >= 0.0f) || !(alpha_n >= 0.0f) || !(alpha_p <= FLT_MAX) || !(alpha_n <= FLT_MAX)) return FOG_ERR_UNSUPPORTED;
  return act_grad<ACT_XIELU>(x_bf16, ldx, dy_bf16, ld_dy, rows, cols, alpha_p, alpha_n, fmt, scale, dx_bf16, ld_dx, q, ldq, amax_out, dalpha, accumulate, workspace,
                             workspace_bytes, stream);
}

extern "C" fog_status fog_gelu_grad(const void* x_bf16, int64_t ldx, const void* dy_bf16, int64_t ld_dy, int64_t rows, int64_t cols, fog_fp8 fmt, const float* scale,
                                    void* dx_bf16, int64_t ld_dx, uint8_t* q, int64_t ldq, float* amax_out, void* workspace, size_t workspace_bytes, void* stream) {
  return act_grad<ACT_GELU>(x_bf16, ldx, dy_bf16, ld_dy, rows, cols, 0.0f, 0.0f, fmt, scale, dx_bf16, ld_dx, q, ldq, amax_out, nullptr, 0, workspace, workspace_bytes,
                            stream);
}

extern "C" fog_status fog_tanh_grad(const void* x_bf16, int64_t ldx, const void* dy_bf16, int64_t ld_dy, int64_t rows, int64_t cols, float alpha, fog_fp8 fmt,
                                    const float* scale, void* dx_bf16, int64_t ld_dx, uint8_t* q, int64_t ldq, float* amax_out, float* dalpha, int accumulate,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!(alpha >= -FLT_MAX) || !(alpha <= FLT_MAX)) return FOG_ERR_UNSUPPORTED;
  return act_grad<ACT_TANH>(x_bf16, ldx, dy_bf16, ld_dy, rows, cols, alpha, 0.0f, fmt, scale, dx_bf16, ld_dx, q, ldq, amax_out, dalpha, accumulate, workspace,
                            workspace_bytes, stream);
}
