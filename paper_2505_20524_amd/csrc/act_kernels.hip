// Element-wise producers of a GEMM or attention operand, fused with the FP8 cast (cast of Appendix E
// of the paper with a caller-provided scale, as under delayed scaling):
//   xIELU (Appendix B, equation xIELU: alpha_p x^2 + 0.5 x for x > 0,
//          alpha_n (e^x - 1) - alpha_n x + 0.5 x for x <= 0), the FOG-max activation;
//   GeLU  (Section 3, architecture table; read as x Phi(x), the exact form);
//   tanh_alpha(x) = tanh(alpha x) (Section 3), the query / key regulariser of the FOG-flash variant.
// The first two produce the second feed-forward GEMM's input, the third the attention's Q and K.
// The activated tensor is never stored as bf16: every element is read once (2 B) and one FP8 byte
// is written.  HBM-bound.
#include "act_functions.h"
#include "common.h"
#include "launch.h"

namespace {

constexpr int kThreads = 256;

__global__ void zero_u32a(uint32_t* p) { *p = 0u; }

template <int ACT, int FMT>
FOG_DEVICE uint2 act_cast8(uint4 v, float ap, float an, float rho, float& m, bool& nan) {
  float y[8] = {act<ACT>(bf16lo(v.x), ap, an), act<ACT>(bf16hi(v.x), ap, an), act<ACT>(bf16lo(v.y), ap, an), act<ACT>(bf16hi(v.y), ap, an),
                act<ACT>(bf16lo(v.z), ap, an), act<ACT>(bf16hi(v.z), ap, an), act<ACT>(bf16lo(v.w), ap, an), act<ACT>(bf16hi(v.w), ap, an)};
#pragma unroll
  for (int k = 0; k < 8; ++k) m = fmaxf(m, fabsf(y[k]));
  uint2 o;
  o.x = cvt4_fp8_nan<FMT>(y[0] * rho, y[1] * rho, y[2] * rho, y[3] * rho, &nan);
  o.y = cvt4_fp8_nan<FMT>(y[4] * rho, y[5] * rho, y[6] * rho, y[7] * rho, &nan);
  return o;
}

// Workgroup maximum raised into *amax_out; reduced on bit patterns (non-negative floats order like them,
// and the NaN pattern of a thread that saw a NaN orders above everything).
template <int THREADS = kThreads>
FOG_DEVICE void block_amax(float m, bool nan, uint32_t* amax_out) {
  const uint32_t h = wave_max_u32(amax_bits(m, nan));
  __shared__ uint32_t part[THREADS / 64];
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = h;
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t b = part[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) b = b > part[w] ? b : part[w];
    if (b > __hip_atomic_load(amax_out, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(amax_out, b);
  }
}

// Each thread turns 16 bf16 (two 16-byte loads) into 16 FP8 codes (one 16-byte store), two such chunks per trip.
template <int ACT, int FMT>
__global__ __launch_bounds__(kThreads) void act_rows_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t chunks_per_row,
                                                            int64_t ldx, float ap, float an, const float* __restrict__ scale,
                                                            uint8_t* __restrict__ q, int64_t ldq, uint32_t* __restrict__ amax_out) {
  const float rho = *scale;
  const int64_t total = rows * chunks_per_row;
  const int64_t stride = (int64_t)gridDim.x * kThreads;
  float m = 0.0f;
  bool nan = false;
  auto src_of = [&](int64_t i) {
    const int64_t r = i / chunks_per_row, c = i - r * chunks_per_row;
    return x + r * ldx + c * 16;
  };
  auto dst_of = [&](int64_t i) {
    const int64_t r = i / chunks_per_row, c = i - r * chunks_per_row;
    return q + r * ldq + c * 16;
  };
  auto emit = [&](uint4 a, uint4 b, uint8_t* dst) {
    const uint2 lo = act_cast8<ACT, FMT>(a, ap, an, rho, m, nan), hi = act_cast8<ACT, FMT>(b, ap, an, rho, m, nan);
    st_nt16(dst, make_uint4(lo.x, lo.y, hi.x, hi.y));
  };
  int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  for (; i + stride < total; i += 2 * stride) {
    const uint16_t* s0 = src_of(i);
    const uint16_t* s1 = src_of(i + stride);
    uint4 a0 = ld_nt16(s0), b0 = ld_nt16(s0 + 8), a1 = ld_nt16(s1), b1 = ld_nt16(s1 + 8);
    emit(a0, b0, dst_of(i));
    emit(a1, b1, dst_of(i + stride));
  }
  if (i < total) {
    const uint16_t* s0 = src_of(i);
    emit(ld_nt16(s0), ld_nt16(s0 + 8), dst_of(i));
  }
  if (amax_out) block_amax(m, nan, amax_out);
}

// ---------------------------------------------------------------- large tensors: the function of a bf16 magnitude from a table
// A bf16 input has 128 magnitudes per binade, and outside some 20 to 30 binades each function is a constant or linear.  A workgroup
// fills a table in LDS with what the evaluation above gives for the magnitudes of that window, and an element costs one LDS read,
// four to eight vector instructions and its cast instead of 20 to 30: GeLU of 4096 x 8192 32.0 -> 21.6 us and
// of 8192 x 14336 102.7 -> 69.9, xIELU of 8192 x 14336 80.7 -> 73.8, tanh of 4096 x 8192 36.7 -> 22.2 (whole calls with the abs-max).
// Results are the same bits.  One workgroup of 1024 threads per compute unit: each fills its table once (four entries per thread).
// Bound by HBM; before, by vector issue.
constexpr int kTableThreads = 1024;
constexpr int kTableMax = 30 * 128;
// Magnitudes (bf16 patterns) lo .. hi of the table; smaller ones take the entry of lo, larger ones that of hi.
//   GeLU   entry Phi(-t):  constant 1/2 in binary32 below 2^-23, 0 from 14 on.  x Phi(x) = max(x, -0) - t Phi(-t)
//   xIELU  entry e^-t - 1: -1 from 17 on.  e^x - 1 >= x, and x rounds to e^x - 1 below 2^-24: max(entry, x) is right on both sides
//   tanh   entry tanh(|alpha| t): 1 from |alpha| t = 9 on, and |alpha| t itself below 2^-12: min(entry, |alpha| t)
struct TableWindow { int lo, hi; };
template <int ACT>
__device__ constexpr TableWindow table_window(uint32_t p0_bits) {
  if (ACT == ACT_GELU) return {(127 - 24) << 7, 0x4160};             // 2^-24, 14
  if (ACT == ACT_XIELU) return {(127 - 24) << 7, (127 + 5) << 7};    // 2^-24, 32
  const int e = (int)((p0_bits >> 23) & 0xFFu);                      // |alpha| < 2^(e - 126), and 2^(e - 127) <= |alpha| where e > 0
  const int lo = 254 - e - 14, hi = 254 - e + 5;                     // exponents: |alpha| lo < 2^-13, |alpha| hi >= 2^5 where hi is finite
  return {lo < 0 ? 0 : lo << 7, hi > 255 ? 255 << 7 : hi << 7};
}
template <int ACT>
FOG_DEVICE float table_entry(int bits, float p0) {
  const float t = __uint_as_float((uint32_t)bits << 16);
  if (ACT == ACT_GELU) return gelu_tail(t);
  if (ACT == ACT_XIELU) return expm1_neg(-t);
  return tanh_fast(fabsf(p0) * t);
}
template <int ACT>
struct TableAct {
  const char* table;      // entry of magnitude b at byte 4 b - base
  uint32_t lo, hi, base;  // window as float patterns (tanh); 4 lo
  float p0, p1, p2;       // xIELU: alpha_p, alpha_n, 0.5 - alpha_n; tanh: |alpha|
  uint32_t sign;          // tanh: sign bit of alpha
  __device__ __forceinline__ float operator()(float x) const {
    // (clamped as integers: a NaN's pattern is above hi)
    uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    if (ACT == ACT_TANH) {
      b = b < lo ? lo : b;
      b = b > hi ? hi : b;
    } else {
      constexpr uint32_t LO = (uint32_t)table_window<ACT>(0u).lo << 16, HI = (uint32_t)table_window<ACT>(0u).hi << 16;
      b = b < LO ? LO : b > HI ? HI : b;
    }
    const float f = *reinterpret_cast<const float*>(table + ((b >> 14) - base));
    if (ACT == ACT_GELU) return __builtin_elementwise_maximum(x, -0.0f) - fminf(fabsf(x), 14.0f) * f;
    if (ACT == ACT_XIELU) {
      const float pos = __builtin_fmaf(p0 * x, x, 0.5f * x);
      const float neg = __builtin_fmaf(p1, fmaxf(f, x), p2 * x);   // for x > 0 an unused value
      return x > 0.0f ? pos : neg;
    }
    const float y = __builtin_elementwise_minimum(f, p0 * fabsf(x));
    return __uint_as_float(__float_as_uint(y) ^ ((__float_as_uint(x) & 0x80000000u) ^ sign));
  }
};

template <int ACT, int FMT>
__global__ __launch_bounds__(kTableThreads) void act_table_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t chunks_per_row,
                                                                  int64_t ldx, float p0, float p1, const float* __restrict__ scale,
                                                                  uint8_t* __restrict__ q, int64_t ldq, uint32_t* __restrict__ amax_out) {
  __shared__ float table[kTableMax];
  const int64_t total = rows * chunks_per_row, stride = (int64_t)gridDim.x * kTableThreads;
  auto offset = [&](int64_t i, int64_t ld) {
    if (rows == 1) return i * 16;
    const int64_t r = i / chunks_per_row;
    return r * ld + (i - r * chunks_per_row) * 16;
  };
  auto fetch = [&](int64_t i, uint4* v) {
    if (i < total) {
      const uint16_t* p = x + offset(i, ldx);
      // Ordinary loads at every size: on tensors that nothing has just read they are level with non-temporal ones or ahead (us, GeLU,
      // non-temporal -> ordinary: 8 M elements 12.7 -> 12.7, 16 M 17.4 -> 17.6, 32 M 24.9 -> 23.6, 64 M 43.1 -> 41.3, 112 M 70.9 -> 70.0;
      // xIELU 112 M 72.8 -> 73.4), on the same three in turn well ahead up to 32 M (8 M 12.4 -> 10.4, 32 M 25.2 -> 21.2).
      v[0] = *reinterpret_cast<const uint4*>(p);
      v[1] = *reinterpret_cast<const uint4*>(p + 8);
    }
  };
  int64_t i = (int64_t)blockIdx.x * kTableThreads + threadIdx.x;
  uint4 v[4], nx[4];
  fetch(i, v);
  fetch(i + stride, v + 2);
  const TableWindow win = table_window<ACT>(__float_as_uint(p0));
  for (int b = win.lo + (int)threadIdx.x; b <= win.hi; b += kTableThreads) table[b - win.lo] = table_entry<ACT>(b, p0);
  // (kept in vector registers: an instruction with a scalar operand takes half as long again)
  float rho = *scale;
  TableAct<ACT> f;
  f.table = reinterpret_cast<const char*>(table);
  f.lo = (uint32_t)win.lo << 16;
  f.hi = (uint32_t)win.hi << 16;
  f.base = 4u * (uint32_t)win.lo;
  f.p0 = ACT == ACT_TANH ? fabsf(p0) : p0;
  f.p1 = p1;
  f.p2 = 0.5f - p1;
  f.sign = __float_as_uint(p0) & 0x80000000u;
  asm volatile("" : "+v"(rho), "+v"(f.base), "+v"(f.p0), "+v"(f.p1), "+v"(f.p2), "+v"(f.sign));
  __syncthreads();
  float m = 0.0f;
  bool nan = false;
  auto cast8 = [&](uint4 w) {
    const float y[8] = {f(bf16lo(w.x)), f(bf16hi(w.x)), f(bf16lo(w.y)), f(bf16hi(w.y)), f(bf16lo(w.z)), f(bf16hi(w.z)), f(bf16lo(w.w)), f(bf16hi(w.w))};
#pragma unroll
    for (int k = 0; k < 8; ++k) m = fmaxf(m, fabsf(y[k]));
    return make_uint2(cvt4_fp8_nan<FMT>(y[0] * rho, y[1] * rho, y[2] * rho, y[3] * rho, &nan),
                      cvt4_fp8_nan<FMT>(y[4] * rho, y[5] * rho, y[6] * rho, y[7] * rho, &nan));
  };
  auto emit = [&](const uint4* w, int64_t at) {
    const uint2 lo = cast8(w[0]), hi = cast8(w[1]);
    // (Past the caches.  Written through as the casts' codes are, calls alone are slower from 32 M elements on, GeLU 21.2 -> 24.3 us, but a
    // product that reads the codes next gains more: feed-forward half of 4096 x 2048 x 8192 190.9 -> 186.1, 1024 x 1024 x 4096 48.9 -> 45.9.)
    st_nt16(q + offset(at, ldq), make_uint4(lo.x, lo.y, hi.x, hi.y));
  };
  while (i < total) {
    const int64_t n = i + 2 * stride;
    fetch(n, nx);
    fetch(n + stride, nx + 2);
    emit(v, i);
    if (i + stride < total) emit(v + 2, i + stride);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = nx[k];
    i = n;
  }
  if (amax_out) block_amax<kTableThreads>(m, nan, amax_out);
}

template <int ACT, int FMT>
__global__ __launch_bounds__(kThreads) void act_general_kernel(const uint16_t* __restrict__ x, int64_t rows, int64_t cols, int64_t ldx,
                                                               float ap, float an, const float* __restrict__ scale,
                                                               uint8_t* __restrict__ q, int64_t ldq, uint32_t* __restrict__ amax_out) {
  const float rho = *scale;
  const int64_t total = rows * cols;
  float m = 0.0f;
  bool nan = false;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
    const int64_t r = i / cols, c = i - r * cols;
    const float y = act<ACT>(bf16lo(x[r * ldx + c]), ap, an);
    m = fmaxf(m, fabsf(y));
    const float t = y * rho;
    q[r * ldq + c] = (uint8_t)(cvt4_fp8_nan<FMT>(t, t, t, t, &nan) & 0xFFu);
  }
  if (amax_out) block_amax(m, nan, amax_out);
}

template <int ACT, int FMT>
void launch_act(const uint16_t* x, int64_t rows, int64_t cols, int64_t ldx, float ap, float an, const float* scale, uint8_t* q,
                  int64_t ldq, uint32_t* amax_out, hipStream_t s) {
  const bool vec = cols % 16 == 0 && ldx % 16 == 0 && ldq % 16 == 0 && (reinterpret_cast<uintptr_t>(x) & 15u) == 0 &&
                   (reinterpret_cast<uintptr_t>(q) & 15u) == 0;
  if (vec) {
    int64_t r = rows, cpr = cols / 16, lx = ldx, lq = ldq;
    if (ldx == cols && ldq == cols) { cpr = rows * cpr; r = 1; lx = lq = cpr * 16; }  // contiguous: one long row
    // The table pays for itself from one chunk of 16 elements per thread on (us, GeLU / xIELU / tanh, without -> with): 4 M elements
    // 11.4 -> 9.8, 11.1 -> 10.5, 10.5 -> 9.7; 2 M elements 9.4 -> 9.1, 9.0 -> 9.5, 8.8 -> 9.1; 1 M 8.8 -> 8.9, 8.7 -> 9.1, 8.8 -> 8.9.
    // (Where the same three tensors of 4 M elements are cast over and over it is behind, 9.2 -> 10.0, 8.8 -> 10.3, 9.0 -> 9.8; behind the
    // product that writes its input it is ahead: feed-forward half of 1024 x 1024 x 4096 52.1 -> 50.3.)
    const int cus = fog_compute_units();
    if (r * cpr >= (int64_t)cus * kTableThreads) {
      act_table_kernel<ACT, FMT><<<cus, kTableThreads, 0, s>>>(x, r, cpr, lx, ap, an, scale, q, lq, amax_out);
      return;
    }
    int64_t blocks = (r * cpr + 2 * kThreads - 1) / (2 * kThreads);
    if (blocks > 2048) blocks = 2048;
    act_rows_kernel<ACT, FMT><<<(int)blocks, kThreads, 0, s>>>(x, r, cpr, lx, ap, an, scale, q, lq, amax_out);
    return;
  }
  int64_t blocks = (rows * cols + kThreads - 1) / kThreads;
  if (blocks > 8192) blocks = 8192;
  act_general_kernel<ACT, FMT><<<(int)blocks, kThreads, 0, s>>>(x, rows, cols, ldx, ap, an, scale, q, ldq, amax_out);
}

// Argument checks and dispatch shared by the three entry points (p0, p1: the activation's parameters).
template <int ACT>
fog_status act_quantize(const void* x_bf16, int64_t rows, int64_t cols, int64_t ldx, float p0, float p1, fog_fp8 fmt,
                        const float* scale, uint8_t* q, int64_t ldq, float* amax_out, void* stream) {
  if (!scale) return FOG_ERR_NULL;
  if (rows < 0 || cols < 0) return FOG_ERR_SHAPE;
  if (fmt != FOG_E4M3 && fmt != FOG_E5M2) return FOG_ERR_UNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  if (amax_out) zero_u32a<<<1, 1, 0, s>>>(reinterpret_cast<uint32_t*>(amax_out));
  if (rows == 0 || cols == 0) return fog_launch_status();
  if (!x_bf16 || !q) return FOG_ERR_NULL;
  if (ldx < cols || ldq < cols) return FOG_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(x_bf16) & 1u) return FOG_ERR_ALIGN;
  const uint16_t* x = reinterpret_cast<const uint16_t*>(x_bf16);
  uint32_t* am = reinterpret_cast<uint32_t*>(amax_out);
  if (fmt == FOG_E4M3) launch_act<ACT, FOG_E4M3>(x, rows, cols, ldx, p0, p1, scale, q, ldq, am, s);
  else                 launch_act<ACT, FOG_E5M2>(x, rows, cols, ldx, p0, p1, scale, q, ldq, am, s);
  return fog_launch_status();
}

}  // namespace

extern "C" fog_status fog_xielu_quantize(const void* x_bf16, int64_t rows, int64_t cols, int64_t ldx, float alpha_p, float alpha_n,
                                         fog_fp8 fmt, const float* scale, uint8_t* q, int64_t ldq, float* amax_out, void* stream) {
  if (!(alpha_p >= 0.0f) || !(alpha_n >= 0.0f) || !(alpha_p <= 3.402823466e38f) || !(alpha_n <= 3.402823466e38f)) return FOG_ERR_UNSUPPORTED;
  return act_quantize<ACT_XIELU>(x_bf16, rows, cols, ldx, alpha_p, alpha_n, fmt, scale, q, ldq, amax_out, stream);
}

extern "C" fog_status fog_gelu_quantize(const void* x_bf16, int64_t rows, int64_t cols, int64_t ldx, fog_fp8 fmt, const float* scale,
                                        uint8_t* q, int64_t ldq, float* amax_out, void* stream) {
  return act_quantize<ACT_GELU>(x_bf16, rows, cols, ldx, 0.0f, 0.0f, fmt, scale, q, ldq, amax_out, stream);
}

extern "C" fog_status fog_tanh_quantize(const void* x_bf16, int64_t rows, int64_t cols, int64_t ldx, float alpha, fog_fp8 fmt,
                                        const float* scale, uint8_t* q, int64_t ldq, float* amax_out, void* stream) {
  if (!(alpha >= -3.402823466e38f) || !(alpha <= 3.402823466e38f)) return FOG_ERR_UNSUPPORTED;
  return act_quantize<ACT_TANH>(x_bf16, rows, cols, ldx, alpha, 0.0f, fmt, scale, q, ldq, amax_out, stream);
}
