// The gradients of the activations, on the way back between the two products of the feed-forward half (tanh: in front of attention): dx = dy f'(x), its cast for
// the products, and the sums that the activation's own parameters get.
//
// Bound by memory: 4 bytes read and 1 (3 with dx) written an element.  xIELU of 8192 x 14336: a call takes 112 us (5.2 TB/s; 104 without the function itself),
// 5 of them the launch that joins the workgroups' sums in a fixed order; GeLU of 333 x 2736: 5 us and 2, less than a call takes on the host.
#include <cfloat>

#include "act_functions.h"
#include "common.h"
#include "launch.h"
#include "layout.h"

namespace {

constexpr int kThreads = 256;
constexpr int kTableThreads = 1024;
constexpr int GROUPS = 2048;             // most workgroups: two sums and an abs-max each in the workspace

// What f' and the parameters' sums need of an exponential, for a magnitude t = |x|:
//   xIELU  e^-t - 1, and e^-t - 1 + t        GeLU  Phi(-t) - t phi(t)        tanh  sech^2(alpha t)
struct Entry { float f, g; };
template <int ACT>
FOG_DEVICE Entry entry(float t, float p0) {
  if (ACT == ACT_XIELU) {
    const float x = -t;
    float q = kExpm1Poly[4];
#pragma unroll
    for (int i = 3; i >= 0; --i) q = __builtin_fmaf(q, x, kExpm1Poly[i]);
    const float e = __builtin_amdgcn_exp2f(x * 1.44269504088896340736f) - 1.0f;
    const bool near = x > kExpm1Switch;                                                 // there without cancellation: x^2 Q(x)
    const float curve = near ? x * x * q : e - x;
    return {near ? x + curve : e, curve};
  }
  if (ACT == ACT_GELU) {
    t = fminf(t, 14.0f);
    const float rinv = __builtin_amdgcn_rcpf(t + kTailK);
    const float u = (t - kTailK) * rinv;
    float p = kTailPoly[10];
#pragma unroll
    for (int i = 9; i >= 0; --i) p = __builtin_fmaf(p, u, kTailPoly[i]);
    const float e = __builtin_amdgcn_exp2f(t * t * -0.72134752044448170368f);
    return {e * __builtin_fmaf(t, -0.39894228040143267794f, p * rinv), 0.0f};           // one exponential for both terms
  }
  const float e = __builtin_amdgcn_exp2f(fabsf(p0) * t * -2.88539008177792681472f);      // 4 e / (1 + e)^2, e = e^(-2 |alpha| t)
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  return {4.0f * e * r * r, 0.0f};
}

// f'(x), and the parameters' sums of one element.  (The bounds that the xIELU's entries are held to, e^x - 1 >= x and e^x - 1 - x >= -1 - x, are true of the functions;
// they give what an entry of a table does not know, the function beyond the table's ends.  The maxima and minima let a NaN through.)
template <int ACT>
FOG_DEVICE float slope(float x, float d, Entry v, float p0, float p1, float& t0, float& t1) {
  if (ACT == ACT_XIELU) {
    const float e = __builtin_elementwise_maximum(v.f, x), curve = __builtin_elementwise_maximum(v.g, -1.0f - x);
    const bool up = x > 0.0f;
    // (The sums are chosen, not their terms: a zero in the place of a factor makes a NaN beside an infinity in the other.)
    const float u0 = __builtin_fmaf(d * x, x, t0), u1 = __builtin_fmaf(d, curve, t1);
    t0 = up ? u0 : t0;
    t1 = up ? t1 : u1;
    return up ? __builtin_fmaf(p0 + p0, x, 0.5f) : __builtin_fmaf(p1, e, 0.5f);
  }
  if (ACT == ACT_GELU) {
    const float s = x < 0.0f ? v.f : 1.0f - v.f;
    return __builtin_elementwise_minimum(s, __builtin_elementwise_maximum(x, 2.0f));    // s < 2: only a NaN in x goes through
  }
  t0 = __builtin_fmaf(d, x * v.f, t0);
  return p0 * __builtin_elementwise_minimum(v.f, __builtin_elementwise_maximum(x, 2.0f));
}

// ---------------------------------------------------------------- large tensors: the entries of a bf16 magnitude from a table in LDS
// (As the producers have it.)  Magnitudes (bf16 patterns) lo .. hi; smaller ones take the entry of lo, larger ones that of hi.
//   xIELU  2^-24 .. 32 (up to 2^-24 the second sum's term counts as 0)      GeLU  2^-24 .. 14: 1/2 and 0 outside      tanh  1 below |alpha| t = 2^-13, 0 from 64 on
struct Window { int lo, hi; };
template <int ACT>
__device__ constexpr Window window_of(uint32_t p0_bits) {
  if (ACT == ACT_GELU) return {(127 - 24) << 7, 0x4160};
  if (ACT == ACT_XIELU) return {(127 - 24) << 7, (127 + 5) << 7};
  const int e = (int)((p0_bits >> 23) & 0xFFu);                      // |alpha| < 2^(e - 126), and 2^(e - 127) <= |alpha| where e > 0
  const int lo = 254 - e - 14, hi = 254 - e + 6;                     // exponents: |alpha| lo < 2^-13, |alpha| hi >= 2^6 where hi is finite
  return {lo < 0 ? 0 : lo << 7, hi > 255 ? 255 << 7 : hi << 7};
}
constexpr int kTableMax = 30 * 128;

template <int ACT>
struct Table {
  static constexpr int BYTES = ACT == ACT_XIELU ? 8 : 4;
  const char* at;          // entry of magnitude b at byte BYTES (b - lo)
  us2 lo, hi;              // the window, twice
  // Where the entries of a pair of numbers lie, 16 bits each: four instructions on both (one by one eight; with the bounds of the slope 124 -> 119 us).
  __device__ __forceinline__ uint32_t places(uint32_t w) const {
    us2 b = __builtin_bit_cast(us2, w & 0x7FFF7FFFu);                // (clamped as integers: a NaN's pattern is above hi)
    b = __builtin_elementwise_min(__builtin_elementwise_max(b, lo), hi);
    return __builtin_bit_cast(uint32_t, (us2)((b - lo) << (unsigned short)(BYTES == 8 ? 3 : 2)));
  }
  __device__ __forceinline__ Entry entry_at(uint32_t place) const {
    const char* p = at + place;
    if (BYTES == 8) {
      const float2 v = *reinterpret_cast<const float2*>(p);
      return {v.x, v.y};
    }
    return {*reinterpret_cast<const float*>(p), 0.0f};
  }
  __device__ __forceinline__ Entry operator()(float x) const { return entry_at(places(__float_as_uint(x) >> 16) & 0xFFFFu); }
};

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

// A chunk: where it lies, how many of its eight elements are there, and these.
struct Chunk {
  int64_t r, c;
  int n;
  uint4 x, d;
};
FOG_DEVICE Chunk fetch(const Args& a, int64_t i, int64_t total) {
  Chunk k = {0, 8 * i, 0, make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  if (i >= total) return k;
  if (a.rows > 1) {
    k.r = total <= 0xFFFFFFFF ? (int64_t)((uint32_t)i / (uint32_t)a.chunks) : i / a.chunks;
    k.c = 8 * (i - k.r * a.chunks);
  }
  k.n = a.cols - k.c < 8 ? (int)(a.cols - k.c) : 8;
  const uint16_t *x = a.x + k.r * a.ldx + k.c, *dy = a.dy + k.r * a.ld_dy + k.c;
  k.x = k.n >= 8 ? ld_any_nt16(x) : ld_upto8(x, k.n);
  k.d = k.n >= 8 ? ld_any_nt16(dy) : ld_upto8(dy, k.n);
  return k;
}

FOG_DEVICE uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
// The larger magnitudes of pairs.
FOG_DEVICE uint32_t most8(uint32_t most, uint4 o) {
  return pkmax_abs_bf16(pkmax_abs_bf16(pkmax_abs_bf16(pkmax_abs_bf16(most, o.x), o.y), o.z), o.w);
}
FOG_DEVICE uint32_t larger(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b)));
}
// Whether numbers up to these stay within the format under the scale: they need neither a clamp nor a NaN test.
template <int FMT>
FOG_DEVICE bool fits(uint32_t most, float rho) {
  return __uint_as_float(max_of_pair(most) << 16) * fabsf(rho) <= (FMT == FOG_E4M3 ? 448.0f : 57344.0f);
}
template <int FMT>
FOG_DEVICE uint2 cast8(uint4 o, float rho, bool fine) {
  float d[8];
  unpack8(o, d);
  if (__builtin_expect(fine, 1))
    return make_uint2(cvt4_fp8_finite<FMT>(d[0] * rho, d[1] * rho, d[2] * rho, d[3] * rho), cvt4_fp8_finite<FMT>(d[4] * rho, d[5] * rho, d[6] * rho, d[7] * rho));
  return make_uint2(cvt4_fp8_nan<FMT>(d[0] * rho, d[1] * rho, d[2] * rho, d[3] * rho), cvt4_fp8_nan<FMT>(d[4] * rho, d[5] * rho, d[6] * rho, d[7] * rho));
}

template <int ACT, int FMT, typename F>
FOG_DEVICE void work(const Args& a, const Chunk& k, float rho, const F& look, double& s0, double& s1, uint32_t& top) {
  if (k.n == 0) return;
  float x[8], d[8], t0 = 0.0f, t1 = 0.0f;
  unpack8(k.x, x);
  unpack8(k.d, d);
#pragma unroll
  for (int i = 0; i < 8; ++i) d[i] *= slope<ACT>(x[i], d[i], look(x[i]), a.p0, a.p1, t0, t1);
  if (ACT != ACT_GELU) s0 += (double)t0;
  if (ACT == ACT_XIELU) s1 += (double)t1;
  const uint4 o = pack8(d);
  const uint32_t most = most8(0u, o);
  top = larger(top, most);
  if (a.dx) {
    uint16_t* to = a.dx + k.r * a.ld_dx + k.c;
    if (k.n >= 8) st_any_nt16(to, o);
    else st_upto8(to, o, k.n);
  }
  if (a.q) {
    const uint2 w = cast8<FMT>(o, rho, fits<FMT>(most, rho));
    uint8_t* to = a.q + k.r * a.ldq + k.c;
    if (k.n >= 8) {
      u32x2 v = {w.x, w.y};
      *reinterpret_cast<u32x2_byte*>(to) = v;
    } else {
      st_upto8(to, w, k.n);
    }
  }
}

// A workgroup's sums and maximum into its words.
template <int THREADS>
FOG_DEVICE void leave(const Args& a, double s0, double s1, uint32_t top) {
  if (a.sums) {
    __shared__ double part[THREADS / 64][2];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) { s0 += __shfl_xor(s0, o, 64); s1 += __shfl_xor(s1, o, 64); }
    if ((threadIdx.x & 63) == 0) { part[threadIdx.x >> 6][0] = s0; part[threadIdx.x >> 6][1] = s1; }
    __syncthreads();
    if (threadIdx.x < 2) {
      double t = part[0][threadIdx.x];
#pragma unroll
      for (int w = 1; w < THREADS / 64; ++w) t += part[w][threadIdx.x];
      a.sums[2 * blockIdx.x + threadIdx.x] = t;
    }
  }
  if (a.tops) {
    __shared__ uint32_t tops[THREADS / 64];
    const uint32_t m = wave_max_u32(max_of_pair(top));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t t = tops[0];
#pragma unroll
      for (int w = 1; w < THREADS / 64; ++w) t = t > tops[w] ? t : tops[w];
      a.tops[blockIdx.x] = t << 16;      // the float with that bf16 pattern
    }
  }
}

template <int ACT, int FMT>
__global__ __launch_bounds__(kThreads) void act_grad_kernel(Args a) {
  const float rho = a.q ? *a.scale : 0.0f;
  const int64_t total = a.rows * a.chunks, stride = (int64_t)gridDim.x * kThreads;
  double s0 = 0.0, s1 = 0.0;
  uint32_t top = 0u;
  auto look = [&](float x) { return entry<ACT>(fabsf(x), a.p0); };
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += 2 * stride) {
    const Chunk k0 = fetch(a, i, total), k1 = fetch(a, i + stride, total);
    work<ACT, FMT>(a, k0, rho, look, s0, s1, top);
    work<ACT, FMT>(a, k1, rho, look, s0, s1, top);
  }
  leave<kThreads>(a, s0, s1, top);
}

// Rows of whole sixteens, or one row of any length (FLAT): a wave takes 1024 elements at a time, in two halves so that each of its loads covers whole lines, and
// looks the entries up; two lanes store the codes of one's first and the other's second eight, sixteen bytes each.  Whole calls of xIELU, 8192 x 14336, from a graph:
// 123 us with sixteen elements in a row a lane and the next ones' loads under way, 114 like this (110 to 115 with three workgroups of 512 threads a compute unit and
// spilled registers, 115 with the loads under way), 112 with the sums chosen instead of their terms; 104 without the function: the rest is memory and two launches.
// One workgroup a compute unit fills its table once.
// Against the other kernel, 8192 x 14336 / 4096 x 4096 / 1024 x 4096: xIELU 138 -> 112 / 29.3 -> 20.8 / 11.9 -> 10.6 us, GeLU 140 -> 107 / 28.8 -> 19.1 / 11.1 -> 9.2, tanh
// 136 -> 107 / 25.6 -> 19.7 / 10.9 -> 10.0.
FOG_DEVICE uint32_t beside(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, false); }
template <int ACT, int FMT, bool FLAT>
__global__ __launch_bounds__(kTableThreads) void act_grad_table_kernel(Args a) {
  __shared__ __attribute__((aligned(16))) char table[kTableMax * Table<ACT>::BYTES];
  constexpr int WAVES = kTableThreads / 64;
  const Window win = window_of<ACT>(__float_as_uint(a.p0));
  for (int b = win.lo + (int)threadIdx.x; b <= win.hi; b += kTableThreads) {
    Entry v = entry<ACT>(__uint_as_float((uint32_t)b << 16), a.p0);
    if (ACT == ACT_XIELU && b == win.lo) v.g = 0.0f;                 // zeros, among others
    float* to = reinterpret_cast<float*>(table) + (b - win.lo) * (Table<ACT>::BYTES / 4);
    to[0] = v.f;
    if (Table<ACT>::BYTES == 8) to[1] = v.g;
  }
  const float rho = a.q ? *a.scale : 0.0f;
  const unsigned short lo = (unsigned short)win.lo, hi = (unsigned short)win.hi;
  const Table<ACT> look = {table, {lo, lo}, {hi, hi}};
  double s0 = 0.0, s1 = 0.0;
  uint32_t top = 0u;
  __syncthreads();
  // Chunks of eight elements: pairs of them are whole, so that a lane and its neighbour are there or not together.
  const int64_t chunks = 2 * (a.cols / 16), total = a.rows * chunks;
  const uint32_t lane = threadIdx.x & 63;
  const bool odd = (lane & 1) != 0;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  int64_t i = 128 * ((int64_t)blockIdx.x * WAVES + wave);            // the wave's first chunk: scalar, and with it the addresses of FLAT but for the lane's place
  auto at = [&](auto* base, uint32_t k, int64_t ld) {
    if (FLAT) return (base + 8 * i) + 8 * k;
    const int64_t j = i + k, r = total <= 0xFFFFFFFF ? (int64_t)((uint32_t)j / (uint32_t)chunks) : j / chunks;
    return base + r * ld + 8 * (j - r * chunks);
  };
  for (; i < total; i += 128 * (int64_t)gridDim.x * WAVES) {
    const uint32_t left = total - i < 128 ? (uint32_t)(total - i) : 128u;
    uint4 x[2], d[2], o[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      x[h] = d[h] = make_uint4(0, 0, 0, 0);
      if (lane + 64 * h < left) {
        x[h] = ld_any_nt16(at(a.x, lane + 64 * h, a.ldx));
        d[h] = ld_any_nt16(at(a.dy, lane + 64 * h, a.ld_dy));
      }
    }
    uint32_t most = 0u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float f[8], g[8], t0 = 0.0f, t1 = 0.0f;
      unpack8(x[h], f);
      unpack8(d[h], g);
      const uint32_t place[4] = {look.places(x[h].x), look.places(x[h].y), look.places(x[h].z), look.places(x[h].w)};
#pragma unroll
      for (int k = 0; k < 8; ++k)
        g[k] *= slope<ACT>(f[k], g[k], look.entry_at(k & 1 ? place[k >> 1] >> 16 : place[k >> 1] & 0xFFFFu), a.p0, a.p1, t0, t1);
      if (ACT != ACT_GELU) s0 += (double)t0;
      if (ACT == ACT_XIELU) s1 += (double)t1;
      o[h] = pack8(g);
      most = most8(most, o[h]);
    }
    top = larger(top, most);
    if (a.dx) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (lane + 64 * h < left) st_any_nt16(at(a.dx, lane + 64 * h, a.ld_dx), o[h]);
    }
    if (a.q) {
      const bool fine = fits<FMT>(most, rho);
      const uint2 u = cast8<FMT>(o[0], rho, fine), w = cast8<FMT>(o[1], rho, fine);
      const uint32_t p = beside(odd ? u.x : w.x), r = beside(odd ? u.y : w.y), k = odd ? lane + 63 : lane;
      if (k < left) st_any_nt16(at(a.q, k, a.ldq), make_uint4(odd ? p : u.x, odd ? r : u.y, odd ? w.x : p, odd ? w.y : r));
    }
  }
  if (FLAT && blockIdx.x == 0 && threadIdx.x < 2)          // what sixteen does not divide
    work<ACT, FMT>(a, fetch(a, total + threadIdx.x, a.chunks), rho, look, s0, s1, top);
  leave<kTableThreads>(a, s0, s1, top);
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
    const int64_t chunks = a.rows * a.chunks, want = (chunks + 2 * kThreads - 1) / (2 * kThreads);
    // A workgroup that fills a table has to have work for it: sixteen elements a thread.
    const int cus = fog_compute_units();
    const bool table = chunks >= 2 * (int64_t)cus * kTableThreads && cus <= GROUPS && (a.rows == 1 || a.cols % 16 == 0);
    groups = table ? cus : (int)(want < GROUPS ? want : GROUPS);
    if (table) {
#define FOG_TABLE(FLAT)                                                                                                        \
  (fmt == FOG_E4M3 ? act_grad_table_kernel<ACT, FOG_E4M3, FLAT><<<groups, kTableThreads, 0, s>>>(a)                            \
                   : act_grad_table_kernel<ACT, FOG_E5M2, FLAT><<<groups, kTableThreads, 0, s>>>(a))
      if (a.rows == 1) FOG_TABLE(true);
      else FOG_TABLE(false);
#undef FOG_TABLE
    } else {
      if (fmt == FOG_E4M3) act_grad_kernel<ACT, FOG_E4M3><<<groups, kThreads, 0, s>>>(a);
      else                 act_grad_kernel<ACT, FOG_E5M2><<<groups, kThreads, 0, s>>>(a);
    }
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
