// The AdamW step over many tensors, states in binary32 or in FP8 with a scale for each 128 elements.
//
// Bound by memory: 28 bytes an element with bf16 weights, bf16 gradients, a binary32 master copy and binary32 states, 16 with FP8 states.
// Two blocks at 8B scale, 487 M elements: 2300 to 2360 us (5.9 TB/s) and 1320 to 1400 us (5.7 TB/s); 49 tensors of 4.8 M: 27 us.
// As the gradients' norm and clipping: up to BATCH tensors a launch, cut into pieces of PIECE elements, a workgroup for each piece.
//
// Every operation on the moments is rounded once to binary32, in the order that the header states (no fused multiply-adds), so that a
// state, and with it the scale of a block and the code of an element, is the same bits however the work is cut.
//
// FP8 states are rounded stochastically.  To the nearest code a second moment would hardly ever move: a step changes it by 1 - beta2 of itself (5 % at
// 0.95), half a code's step is 6 to 12 %.  A code is chosen with probabilities that keep the expected value, by a hash of seed, step, tensor and element: no
// state, the same on every run and whatever the launch looks like.  A second moment above zero keeps a code above zero, so that a
// first moment never stands over a root of 0.
#include <cfloat>
#include <cmath>

#include "common.h"
#include "launch.h"
#include "spans.h"

#pragma clang fp contract(off)

namespace {

constexpr int kThreads = 256;
constexpr int BATCH = 50;                // descriptions that fit a launch's arguments
// Elements of a piece, a multiple of a scale's 128.
constexpr int F32_PIECE = 2048, FP8_PIECE = 4096;
// Large launches of binary32 states (seven streams an element) are faster with fewer workgroups in flight: beyond MANY pieces (32 M elements) each asks for so much
// LDS that five fit a compute unit, and keeps four elements a thread in flight instead of eight.  us, without -> with: 4.8 M elements 26.5 -> 28.3, 33.6 M 163.7 ->
// 160.6, 101 M 494 -> 475, 403 M 1989 -> 1885.  (Pieces of 4096 and 8192 elements, without: 403 M 2019 and 2105.  FP8 states, whose arithmetic wants the waves: 1136 with
// pieces of 4096 and sixteen elements in flight, 1167 with 2048 and eight, 1438 with fewer workgroups.)
constexpr int MANY = 16384;
constexpr size_t ROOM = 32 << 10;
constexpr int GROUPS = 1 << 23;          // most workgroups of a launch: grids are counted in threads of 32 bits
constexpr int TENSORS_MAX = 1 << 24;

struct AdamBatch {
  void* p[BATCH];
  const void* g[BATCH];
  float* master[BATCH];
  void* m[BATCH];
  void* v[BATCH];
  uint8_t* ms[BATCH];
  uint8_t* vs[BATCH];
  int64_t n[BATCH];
  int first[BATCH];        // number of the tensor's first piece
  int number[BATCH];       // of the tensor in the call
  float decay[BATCH];
  uint8_t p32[BATCH], g32[BATCH];
  int count, pieces;
};

// What a step has in common: worked out on the host where the host knows all of it.
struct Common {
  float rate, root;
  uint32_t key;
};
struct AdamStep {
  double lr, log_beta1, log_beta2;
  const float* lr_dev;
  const int64_t* step_dev;
  const double* sumsq;
  int64_t step;
  uint64_t seed;
  Common common;
  float beta1, beta1c, beta2, beta2c, eps, max_norm;     // c: 1 - beta, from binary64
};
static_assert(sizeof(AdamBatch) + sizeof(AdamStep) <= 4096, "arguments of a launch");

FOG_DEVICE int tensor_of(const AdamBatch& b, int p) {
  int lo = 0, hi = b.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (b.first[mid] <= p) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Three rounds of shift and multiplication by odd numbers (the fractions of the golden ratio and of the roots of 2 and 3).
__host__ __device__ static inline uint32_t mix(uint32_t h) {
  h = (h ^ (h >> 16)) * 0x9E3779B1u;
  h = (h ^ (h >> 15)) * 0x6A09E667u;
  h = (h ^ (h >> 13)) * 0xBB67AE85u;
  return h ^ (h >> 16);
}
__host__ __device__ static inline uint32_t next_key(uint32_t key, uint32_t w) { return mix(key + 0x9E3779B9u + w); }

// The largest of the 32 lanes that hold a block of 128 elements.
template <int CTRL>
FOG_DEVICE uint32_t dpp_max(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, false);
  return v > o ? v : o;
}
FOG_DEVICE uint32_t block_max(uint32_t v) {
  v = dpp_max<0xB1>(v);           // lane ^ 1
  v = dpp_max<0x4E>(v);           // lane ^ 2
  v = dpp_max<0x141>(v);          // the other four of eight
  v = dpp_max<0x140>(v);          // the other eight of sixteen
  const uint32_t o = (uint32_t)__shfl_xor((int)v, 16, 64);
  return v > o ? v : o;
}

// k of a block's scale from the bits of its abs-max: floor(log2(FP8MAX / a)), limited to -126 .. 126; 0 where a is zero or not finite.
// FP8MAX is 1.75 * 2^8 or 1.75 * 2^15.
template <int FMT>
FOG_DEVICE int block_exponent(uint32_t a) {
  if (a == 0u || a >= 0x7F800000u) return 0;
  const int k = (FMT == FOG_E4M3 ? 8 : 15) - ((int)(a >> 23) - 127) - ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return k < -126 ? -126 : k > 126 ? 126 : k;
}

// One of the two codes beside y (which is no NaN), as a number: the places that the format drops, plus as many random bits, carry or do not.  Below the smallest
// normal number, where the format's steps stay equal, that number is added first: then the steps of the sum are those of the format.
template <int FMT>
FOG_DEVICE float round_by(float y, uint32_t r) {
  constexpr int DROP = FMT == FOG_E4M3 ? 20 : 21;
  constexpr float LOW = FMT == FOG_E4M3 ? 0.015625f : 6.103515625e-05f;
  r = FMT == FOG_E4M3 ? r & 0xFFFFFu : r >> 11;
  float a = fabsf(y);
  const float add = a < LOW ? LOW : 0.0f;
  a = __uint_as_float((__float_as_uint(a + add) + r) & ~((1u << DROP) - 1u)) - add;
  return FMT == FOG_E4M3 ? __builtin_copysignf(a, y) : a;      // (second moments have no sign)
}

// A lane takes four elements at a time, so that every load and store of a binary32 tensor covers whole lines: in eights, two instructions each touch half of every
// line (two blocks at 8B scale 2818 -> 2519 us, 49 small tensors 39 -> 32).
typedef u32x2 __attribute__((aligned(2))) u32x2_half;
typedef uint32_t __attribute__((aligned(1))) u32_byte;
// Four elements from p on, of which n are there; zeros behind them.
FOG_DEVICE void load4(const float* p, int n, float (&f)[4]) {
  if (n >= 4) {
    const uint4 a = ld_any_nt16(p);
    f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = i < n ? p[i] : 0.0f;
  }
}
FOG_DEVICE void load4(const uint16_t* p, int n, float (&f)[4]) {
  if (n >= 4) {
    const u32x2 a = __builtin_nontemporal_load(reinterpret_cast<const u32x2_half*>(p));
    f[0] = bf16lo(a[0]); f[1] = bf16hi(a[0]); f[2] = bf16lo(a[1]); f[3] = bf16hi(a[1]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = i < n ? bf16lo(p[i]) : 0.0f;
  }
}
FOG_DEVICE uint32_t load_codes(const uint8_t* p, int n) {
  if (n >= 4) return __builtin_nontemporal_load(reinterpret_cast<const u32_byte*>(p));
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n) w |= (uint32_t)p[i] << (8 * i);
  return w;
}
FOG_DEVICE void store4(float* p, int n, const float (&f)[4]) {
  if (n >= 4) {
    st_any_nt16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = f[i];
  }
}
FOG_DEVICE void store4(uint16_t* p, int n, uint2 w) {
  if (n >= 4) {
    u32x2 v = {w.x, w.y};
    __builtin_nontemporal_store(v, reinterpret_cast<u32x2_half*>(p));
  } else {
    st_upto8(p, make_uint4(w.x, w.y, 0u, 0u), n);
  }
}
FOG_DEVICE void store_codes(uint8_t* p, int n, uint32_t w) {
  if (n >= 4) __builtin_nontemporal_store(w, reinterpret_cast<u32_byte*>(p));
  else st_upto8(p, make_uint2(w, 0u), n);
}

template <int FMT>
FOG_DEVICE void decode4(uint32_t q, float by, float (&f)[4]) {
  f32x2 a, b;
  if (FMT == FOG_E4M3) {
    a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false); b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
  } else {
    a = __builtin_amdgcn_cvt_pk_f32_bf8((int)q, false); b = __builtin_amdgcn_cvt_pk_f32_bf8((int)q, true);
  }
  f[0] = a[0] * by; f[1] = a[1] * by; f[2] = b[0] * by; f[3] = b[1] * by;
}

// Codes of this lane's four elements of a block, and the block's scale byte.
template <int FMT>
FOG_DEVICE uint32_t encode4(const float (&x)[4], const uint32_t (&r)[4], uint32_t& byte) {
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    top = top > a ? top : a;
  }
  top = block_max(top);
  const int k = block_exponent<FMT>(top);
  byte = (uint32_t)(127 - k);
  const float by = __uint_as_float((uint32_t)(127 + k) << 23);
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = round_by<FMT>(x[i] * by, r[i]);
    if (FMT == FOG_E5M2) y[i] = x[i] > 0.0f ? fmaxf(y[i], 1.52587890625e-05f) : y[i];     // the smallest code above zero
  }
  // A NaN whose upper bits are set carries into the sign and would come out of round_by as a zero: NaNs take their own way, in blocks that hold one (a comparison
  // for each block; beside every rounding it would be one for each element).
  if (__builtin_expect(top > 0x7F800000u, 0)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = x[i] != x[i] ? x[i] : y[i];
  }
  return cvt4_fp8_finite<FMT>(y[0], y[1], y[2], y[3]);
}

__host__ __device__ static inline uint32_t step_key(uint64_t seed, uint64_t t) {
  return next_key(next_key(next_key(next_key(0u, (uint32_t)seed), (uint32_t)(seed >> 32)), (uint32_t)t), (uint32_t)(t >> 32));
}

struct Tensor {
  const void* g;
  void *p, *m, *v;
  float* master;
  uint8_t *ms, *vs;
  float keep, rate, root, c;
  uint32_t high, low;      // of the random numbers
  bool p32, g32;
};

// Four elements from element i of the tensor on, of which n are there (FULL: all).
struct Four {
  float g[4], m[4], v[4], p[4];
};
template <bool FP8, bool FULL>
FOG_DEVICE void load_four(const Tensor& t, int64_t i, int n, Four& f) {
  if (FULL) n = 4;
  if (t.g32) load4(reinterpret_cast<const float*>(t.g) + i, n, f.g);
  else load4(reinterpret_cast<const uint16_t*>(t.g) + i, n, f.g);
  if (t.master) load4(t.master + i, n, f.p);
  else if (t.p32) load4(reinterpret_cast<const float*>(t.p) + i, n, f.p);
  else load4(reinterpret_cast<const uint16_t*>(t.p) + i, n, f.p);
  if (FP8) {
    decode4<FOG_E4M3>(load_codes(reinterpret_cast<const uint8_t*>(t.m) + i, n), __uint_as_float((uint32_t)t.ms[i >> 7] << 23), f.m);
    decode4<FOG_E5M2>(load_codes(reinterpret_cast<const uint8_t*>(t.v) + i, n), __uint_as_float((uint32_t)t.vs[i >> 7] << 23), f.v);
  } else {
    load4(reinterpret_cast<const float*>(t.m) + i, n, f.m);
    load4(reinterpret_cast<const float*>(t.v) + i, n, f.v);
  }
}
template <bool FP8, bool FULL, bool NEAR>
FOG_DEVICE void step_four(const Tensor& t, const AdamStep& s, int64_t i, uint32_t at, int n, Four& f) {
  if (FULL) n = 4;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float gc = f.g[e] * t.c;
    f.m[e] = f.m[e] * s.beta1 + gc * s.beta1c;
    f.v[e] = f.v[e] * s.beta2 + gc * gc * s.beta2c;
    // Root and quotient are rounded correctly, at 25 instructions more than the hardware's own, which are off by up to a unit in the last place each.  With binary32
    // states these hide behind memory (two blocks at 8B scale 2310 us a step either way).  With FP8 states they do not (1450 us, not 1340), and a unit of 2^-23 is
    // nothing beside moments in steps of 2^-3 and 2^-2: NEAR takes the hardware's there.  A second moment below the smallest normal number then counts as 0: beside
    // an eps of 2^-38 and more its root, below 2^-63, does not show; FP8 states with a smaller eps have the kernel without NEAR.
    const float u = NEAR ? f.m[e] * t.rate * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(f.v[e]) * t.root + s.eps)
                         : f.m[e] * t.rate / (__builtin_sqrtf(f.v[e]) * t.root + s.eps);
    f.p[e] = f.p[e] * t.keep - u;
  }
  uint32_t r[4];
  if (FP8 || (!t.master && !t.p32)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = mix((at + (uint32_t)e) ^ t.high);
  }
  if (t.master) store4(t.master + i, n, f.p);
  if (t.p32) {
    store4(reinterpret_cast<float*>(t.p) + i, n, f.p);
  } else {
    uint2 w;
    if (t.master) {
      w = make_uint2(pack_bf16x2(f.p[0], f.p[1]), pack_bf16x2(f.p[2], f.p[3]));
    } else {
      // weights without a master copy: up where the sixteen places dropped, plus as many random bits, carry
      uint32_t h[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = f.p[e] != f.p[e] ? 0x7FC0u : (__float_as_uint(f.p[e]) + ((r[e] * 0x9E3779B1u) >> 16)) >> 16;
      w = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    }
    store4(reinterpret_cast<uint16_t*>(t.p) + i, n, w);
  }
  if (FP8) {
    uint32_t bm, bv;
    const uint32_t qm = encode4<FOG_E4M3>(f.m, r, bm), qv = encode4<FOG_E5M2>(f.v, r, bv);
    store_codes(reinterpret_cast<uint8_t*>(t.m) + i, n, qm);
    store_codes(reinterpret_cast<uint8_t*>(t.v) + i, n, qv);
    if ((threadIdx.x & 31) == 0) {
      t.ms[i >> 7] = (uint8_t)bm;
      t.vs[i >> 7] = (uint8_t)bv;
    }
  } else {
    store4(reinterpret_cast<float*>(t.m) + i, n, f.m);
    store4(reinterpret_cast<float*>(t.v) + i, n, f.v);
  }
}

// U: fours in flight.  NEAR: root and quotient by the hardware's instructions.
template <bool FP8, int PIECE, int U, bool NEAR>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamBatch b, AdamStep s) {
  Tensor t;
  t.c = 1.0f;
  if (s.sumsq) {
    const double norm = __builtin_sqrt(*s.sumsq);
    if (!(norm < __builtin_inf())) return;               // not finite: the step is left out
    if (norm > (double)s.max_norm) t.c = (float)((double)s.max_norm / norm);
  }
  double lr = s.lr;
  uint32_t key = s.common.key;
  t.rate = s.common.rate;
  t.root = s.common.root;
  if (s.lr_dev || s.step_dev) {
    int64_t n = s.step_dev ? *s.step_dev : s.step;
    if (n < 1) n = 1;
    if (s.lr_dev) lr = (double)*s.lr_dev;
    t.rate = (float)(lr / -expm1((double)n * s.log_beta1));        // 1 - beta^t without cancellation
    t.root = (float)(1.0 / __builtin_sqrt(-expm1((double)n * s.log_beta2)));
    key = step_key(s.seed, (uint64_t)n);
  }
  for (int piece = blockIdx.x; piece < b.pieces; piece += gridDim.x) {
    const int j = tensor_of(b, piece);
    const int64_t at = (int64_t)(piece - b.first[j]) * PIECE;
    const int64_t left = b.n[j] - at;
    const int n = (int)(left < PIECE ? left : PIECE);
    t.g = b.g[j]; t.p = b.p[j]; t.m = b.m[j]; t.v = b.v[j]; t.master = b.master[j]; t.ms = b.ms[j]; t.vs = b.vs[j];
    t.p32 = b.p32[j] != 0; t.g32 = b.g32[j] != 0;
    t.keep = (float)(1.0 - lr * (double)b.decay[j]);
    t.high = mix((uint32_t)((uint64_t)at >> 32) + next_key(key, (uint32_t)b.number[j]));
    t.low = (uint32_t)at;
    if (n == PIECE) {
#pragma unroll 1
      for (int i0 = 4 * (int)threadIdx.x; i0 < PIECE; i0 += 4 * kThreads * U) {
        Four f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) load_four<FP8, true>(t, at + i0 + 4 * kThreads * u, 4, f[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) step_four<FP8, true, NEAR>(t, s, at + i0 + 4 * kThreads * u, t.low + (uint32_t)(i0 + 4 * kThreads * u), 4, f[u]);
      }
    } else {
      const int whole = (n + 127) & ~127;                // whole blocks: their lanes stay together
#pragma unroll 1
      for (int i0 = 4 * (int)threadIdx.x; i0 < whole; i0 += 4 * kThreads) {
        Four f;
        load_four<FP8, false>(t, at + i0, n - i0, f);
        step_four<FP8, false, NEAR>(t, s, at + i0, t.low + (uint32_t)i0, n - i0, f);
      }
    }
  }
}

bool odd(const void* p, uintptr_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }

fog_status check_jobs(const fog_adamw_job* jobs, int count, bool fp8) {
  for (int i = 0; i < count; ++i) {
    const fog_adamw_job& j = jobs[i];
    if (j.n < 0) return FOG_ERR_SHAPE;
    if ((j.p_type != FOG_BF16 && j.p_type != FOG_F32) || (j.g_type != FOG_BF16 && j.g_type != FOG_F32)) return FOG_ERR_UNSUPPORTED;
    if (j.n > ((int64_t)1 << 36)) return FOG_ERR_UNSUPPORTED;      // a batch of such tensors has fewer than 2^31 pieces
    if (!(std::fabs(j.weight_decay) <= FLT_MAX) || (j.master && j.p_type == FOG_F32)) return FOG_ERR_UNSUPPORTED;
    if (j.n == 0) continue;
    if (!j.p || !j.g || !j.m || !j.v || (fp8 && (!j.m_scale || !j.v_scale))) return FOG_ERR_NULL;
    if (odd(j.p, j.p_type == FOG_F32 ? 4 : 2) || odd(j.g, j.g_type == FOG_F32 ? 4 : 2) || odd(j.master, 4) || (!fp8 && (odd(j.m, 4) || odd(j.v, 4))))
      return FOG_ERR_ALIGN;
  }
  FogSpans<7 * 64> spans(7 * (int64_t)count);
  if (!spans.ok()) return FOG_ERR_UNSUPPORTED;
  for (int i = 0; i < count; ++i) {
    const fog_adamw_job& j = jobs[i];
    const int64_t state = j.n * (fp8 ? 1 : 4), blocks = fp8 ? (j.n + 127) / 128 : 0;
    spans.add(j.p, j.n * (j.p_type == FOG_F32 ? 4 : 2), true);
    spans.add(j.g, j.n * (j.g_type == FOG_F32 ? 4 : 2), false);
    spans.add(j.master, j.n * 4, true);
    spans.add(j.m, state, true);
    spans.add(j.v, state, true);
    spans.add(j.m_scale, blocks, true);
    spans.add(j.v_scale, blocks, true);
  }
  return spans.apart() ? FOG_OK : FOG_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" fog_status fog_adamw(const fog_adamw_job* jobs, int count, fog_states states, double lr, const float* lr_dev, double beta1, double beta2,
                                double eps, int64_t step, const int64_t* step_dev, uint64_t seed, const double* sumsq, float max_norm, void* stream) {
  if (count < 0 || (!step_dev && step < 1)) return FOG_ERR_SHAPE;
  if (count > TENSORS_MAX || (states != FOG_STATES_F32 && states != FOG_STATES_FP8)) return FOG_ERR_UNSUPPORTED;
  const bool fp8 = states == FOG_STATES_FP8;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || (fp8 && (beta1 > 0.99 || beta2 > 0.99))) return FOG_ERR_UNSUPPORTED;
  if (!(eps >= FLT_MIN && eps <= FLT_MAX) || (!lr_dev && !(std::fabs(lr) <= FLT_MAX)) || (sumsq && !(max_norm >= 0.0f))) return FOG_ERR_UNSUPPORTED;
  if (odd(lr_dev, 4) || odd(step_dev, 8) || odd(sumsq, 8)) return FOG_ERR_ALIGN;
  if (count > 0 && !jobs) return FOG_ERR_NULL;
  const fog_status st = check_jobs(jobs, count, fp8);
  if (st != FOG_OK) return st;
  AdamStep s;
  s.lr = lr; s.log_beta1 = std::log(beta1); s.log_beta2 = std::log(beta2);
  s.lr_dev = lr_dev; s.step_dev = step_dev; s.sumsq = sumsq; s.step = step; s.seed = seed;
  s.beta1 = (float)beta1; s.beta1c = (float)(1.0 - beta1); s.beta2 = (float)beta2; s.beta2c = (float)(1.0 - beta2);
  s.eps = (float)eps; s.max_norm = max_norm;
  s.common = {0.0f, 0.0f, 0u};
  if (!lr_dev && !step_dev)
    s.common = {(float)(lr / -std::expm1((double)step * s.log_beta1)), (float)(1.0 / std::sqrt(-std::expm1((double)step * s.log_beta2))), step_key(seed, (uint64_t)step)};
  AdamBatch b;
  const int64_t piece = fp8 ? FP8_PIECE : F32_PIECE;
  bool launched = false;
  b.count = b.pieces = 0;
  auto flush = [&]() {
    if (b.count == 0) return;
    const int groups = b.pieces < GROUPS ? b.pieces : GROUPS;
    hipStream_t st = (hipStream_t)stream;
    if (fp8 && eps >= 0x1p-38) adamw_kernel<true, FP8_PIECE, 4, true><<<groups, kThreads, 0, st>>>(b, s);
    else if (fp8)              adamw_kernel<true, FP8_PIECE, 4, false><<<groups, kThreads, 0, st>>>(b, s);
    else if (b.pieces <= MANY) adamw_kernel<false, F32_PIECE, 2, false><<<groups, kThreads, 0, st>>>(b, s);
    else                       adamw_kernel<false, F32_PIECE, 1, false><<<groups, kThreads, ROOM, st>>>(b, s);
    launched = true;
    b.count = b.pieces = 0;
  };
  for (int i = 0; i < count; ++i) {
    const fog_adamw_job& j = jobs[i];
    if (j.n == 0) continue;
    if (b.count == BATCH) flush();
    const int a = b.count++;
    b.p[a] = j.p; b.g[a] = j.g; b.master[a] = j.master; b.m[a] = j.m; b.v[a] = j.v; b.ms[a] = j.m_scale; b.vs[a] = j.v_scale;
    b.n[a] = j.n; b.first[a] = b.pieces; b.number[a] = i; b.decay[a] = j.weight_decay;
    b.p32[a] = j.p_type == FOG_F32; b.g32[a] = j.g_type == FOG_F32;
    b.pieces += (int)((j.n + piece - 1) / piece);
  }
  flush();
  return launched ? fog_launch_status() : FOG_OK;
}
