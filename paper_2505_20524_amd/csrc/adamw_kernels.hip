// The AdamW step over many tensors, states in binary32 or in FP8 with a scale for each 128 elements.
//
// Bound by memory: 28 bytes an element with bf16 weights, bf16 gradients, a binary32 master copy and binary32 states, 16 with FP8 states.
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
constexpr int64_t PIECE = 8192;          // elements; a multiple of a scale's 128
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

struct AdamStep {
  double lr, log_beta1, log_beta2;
  const float* lr_dev;
  const int64_t* step_dev;
  const double* sumsq;
  int64_t step;
  uint64_t seed;
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
FOG_DEVICE uint32_t mix(uint32_t h) {
  h = (h ^ (h >> 16)) * 0x9E3779B1u;
  h = (h ^ (h >> 15)) * 0x6A09E667u;
  h = (h ^ (h >> 13)) * 0xBB67AE85u;
  return h ^ (h >> 16);
}
FOG_DEVICE uint32_t next_key(uint32_t key, uint32_t w) { return mix(key + 0x9E3779B9u + w); }

// The largest of the 16 lanes that hold a block of 128 elements.
template <int CTRL>
FOG_DEVICE uint32_t dpp_max(uint32_t v) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, false);
  return v > o ? v : o;
}
FOG_DEVICE uint32_t block_max(uint32_t v) {
  v = dpp_max<0xB1>(v);           // lane ^ 1
  v = dpp_max<0x4E>(v);           // lane ^ 2
  v = dpp_max<0x141>(v);          // the other four of eight
  return dpp_max<0x140>(v);       // the other eight of sixteen
}

// k of a block's scale from the bits of its abs-max: floor(log2(FP8MAX / a)), limited to -126 .. 126; 0 where a is zero or not finite.
// FP8MAX is 1.75 * 2^8 or 1.75 * 2^15.
template <int FMT>
FOG_DEVICE int block_exponent(uint32_t a) {
  if (a == 0u || a >= 0x7F800000u) return 0;
  const int k = (FMT == FOG_E4M3 ? 8 : 15) - ((int)(a >> 23) - 127) - ((a & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return k < -126 ? -126 : k > 126 ? 126 : k;
}

// One of the two codes beside y, as a number: the places that the format drops, plus as many random bits, carry or do not.  Below the smallest
// normal number, where the format's steps stay equal, that number is added first: then the steps of the sum are those of the format.
template <int FMT>
FOG_DEVICE float round_by(float y, uint32_t r) {
  constexpr int DROP = FMT == FOG_E4M3 ? 20 : 21;
  constexpr float LOW = FMT == FOG_E4M3 ? 0.015625f : 6.103515625e-05f;
  r = FMT == FOG_E4M3 ? r & 0xFFFFFu : r >> 11;
  float a = fabsf(y);
  const float add = a < LOW ? LOW : 0.0f;
  a = __uint_as_float((__float_as_uint(a + add) + r) & ~((1u << DROP) - 1u)) - add;
  return __builtin_copysignf(a, y);
}

typedef u32x2 __attribute__((aligned(1))) u32x2_byte;
// Eight elements from p on, of which n are there; zeros behind them.
FOG_DEVICE void load8(const float* p, int n, float (&f)[8]) {
  if (n >= 8) {
    const uint4 a = ld_any_nt16(p), b = ld_any_nt16(p + 4);
    f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
    f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y); f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? p[i] : 0.0f;
  }
}
FOG_DEVICE void load8(const uint16_t* p, int n, float (&f)[8]) {
  const uint4 a = n >= 8 ? ld_any_nt16(p) : ld_upto8(p, n);
  f[0] = bf16lo(a.x); f[1] = bf16hi(a.x); f[2] = bf16lo(a.y); f[3] = bf16hi(a.y);
  f[4] = bf16lo(a.z); f[5] = bf16hi(a.z); f[6] = bf16lo(a.w); f[7] = bf16hi(a.w);
}
FOG_DEVICE uint2 load_codes(const uint8_t* p, int n) {
  if (n >= 8) {
    const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2_byte*>(p));
    return make_uint2(v[0], v[1]);
  }
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  return make_uint2(w[0], w[1]);
}
FOG_DEVICE void store8(float* p, int n, const float (&f)[8]) {
  if (n >= 8) {
    st_any_nt16(p, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
    st_any_nt16(p + 4, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = f[i];
  }
}
FOG_DEVICE void store8(uint16_t* p, int n, uint4 w) {
  if (n >= 8) st_any_nt16(p, w);
  else st_upto8(p, w, n);
}
FOG_DEVICE void store_codes(uint8_t* p, int n, uint2 w) {
  if (n >= 8) {
    u32x2 v = {w.x, w.y};
    __builtin_nontemporal_store(v, reinterpret_cast<u32x2_byte*>(p));
  } else {
    st_upto8(p, w, n);
  }
}

template <int FMT>
FOG_DEVICE void decode8(uint2 q, float by, float (&f)[8]) {
  f32x2 a, b, c, d;
  if (FMT == FOG_E4M3) {
    a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, false); b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, true);
    c = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, false); d = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, true);
  } else {
    a = __builtin_amdgcn_cvt_pk_f32_bf8((int)q.x, false); b = __builtin_amdgcn_cvt_pk_f32_bf8((int)q.x, true);
    c = __builtin_amdgcn_cvt_pk_f32_bf8((int)q.y, false); d = __builtin_amdgcn_cvt_pk_f32_bf8((int)q.y, true);
  }
  f[0] = a[0] * by; f[1] = a[1] * by; f[2] = b[0] * by; f[3] = b[1] * by;
  f[4] = c[0] * by; f[5] = c[1] * by; f[6] = d[0] * by; f[7] = d[1] * by;
}

// Codes of a block's eight elements of this lane, and the block's scale byte.
template <int FMT>
FOG_DEVICE uint2 encode8(const float (&x)[8], const uint32_t (&r)[8], uint32_t& byte) {
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = __float_as_uint(x[i]) & 0x7FFFFFFFu;
    top = top > a ? top : a;
  }
  const int k = block_exponent<FMT>(block_max(top));
  byte = (uint32_t)(127 - k);
  const float by = __uint_as_float((uint32_t)(127 + k) << 23);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = round_by<FMT>(x[i] * by, r[i]);
    if (FMT == FOG_E5M2) y[i] = x[i] > 0.0f ? fmaxf(y[i], 1.52587890625e-05f) : y[i];     // the smallest code above zero
  }
  return make_uint2(cvt4_fp8_finite<FMT>(y[0], y[1], y[2], y[3]), cvt4_fp8_finite<FMT>(y[4], y[5], y[6], y[7]));
}

template <bool FP8>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamBatch b, AdamStep s) {
  float c = 1.0f;
  if (s.sumsq) {
    const double norm = __builtin_sqrt(*s.sumsq);
    if (!(norm < __builtin_inf())) return;               // not finite: the step is left out
    if (norm > (double)s.max_norm) c = (float)((double)s.max_norm / norm);
  }
  int64_t t = s.step_dev ? *s.step_dev : s.step;
  if (t < 1) t = 1;
  const double lr = s.lr_dev ? (double)*s.lr_dev : s.lr;
  // 1 - beta^t without cancellation
  const float rate = (float)(lr / -expm1((double)t * s.log_beta1)), root = (float)(1.0 / __builtin_sqrt(-expm1((double)t * s.log_beta2)));
  uint32_t key = 0u;
  key = next_key(key, (uint32_t)s.seed);
  key = next_key(key, (uint32_t)(s.seed >> 32));
  key = next_key(key, (uint32_t)t);
  key = next_key(key, (uint32_t)((uint64_t)t >> 32));
  for (int piece = blockIdx.x; piece < b.pieces; piece += gridDim.x) {
    const int j = tensor_of(b, piece);
    const int64_t at = (int64_t)(piece - b.first[j]) * PIECE;
    const int64_t left = b.n[j] - at;
    const int n = (int)(left < PIECE ? left : PIECE);
    const bool p32 = b.p32[j] != 0, g32 = b.g32[j] != 0;
    float* master = b.master[j];
    const float keep = (float)(1.0 - lr * (double)b.decay[j]);
    const uint32_t high = mix((uint32_t)((uint64_t)at >> 32) + next_key(key, (uint32_t)b.number[j]));
    const uint32_t low = (uint32_t)at;
    for (int i0 = 8 * (int)threadIdx.x; i0 < ((n + 127) & ~127); i0 += 8 * kThreads) {     // whole blocks: their lanes stay together
      const int64_t i = at + i0;
      const int k = n - i0 < 0 ? 0 : n - i0;
      float g[8], m[8], v[8], p[8];
      if (g32) load8(reinterpret_cast<const float*>(b.g[j]) + i, k, g);
      else load8(reinterpret_cast<const uint16_t*>(b.g[j]) + i, k, g);
      if (master) load8(master + i, k, p);
      else if (p32) load8(reinterpret_cast<const float*>(b.p[j]) + i, k, p);
      else load8(reinterpret_cast<const uint16_t*>(b.p[j]) + i, k, p);
      if (FP8) {
        decode8<FOG_E4M3>(load_codes(reinterpret_cast<const uint8_t*>(b.m[j]) + i, k), __uint_as_float((uint32_t)b.ms[j][i >> 7] << 23), m);
        decode8<FOG_E5M2>(load_codes(reinterpret_cast<const uint8_t*>(b.v[j]) + i, k), __uint_as_float((uint32_t)b.vs[j][i >> 7] << 23), v);
      } else {
        load8(reinterpret_cast<const float*>(b.m[j]) + i, k, m);
        load8(reinterpret_cast<const float*>(b.v[j]) + i, k, v);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float gc = g[e] * c;
        m[e] = m[e] * s.beta1 + gc * s.beta1c;
        v[e] = v[e] * s.beta2 + gc * gc * s.beta2c;
        p[e] = p[e] * keep - m[e] * rate / (__builtin_sqrtf(v[e]) * root + s.eps);
      }
      uint32_t r[8];
      if (FP8 || (!master && !p32)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = mix((low + (uint32_t)(i0 + e)) ^ high);
      }
      if (master) store8(master + i, k, p);
      if (p32) {
        store8(reinterpret_cast<float*>(b.p[j]) + i, k, p);
      } else {
        uint4 w;
        if (master) {
          w = make_uint4(pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7]));
        } else {
          // weights without a master copy: up where the sixteen places dropped, plus as many random bits, carry
          uint32_t h[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) h[e] = p[e] != p[e] ? 0x7FC0u : (__float_as_uint(p[e]) + ((r[e] * 0x9E3779B1u) >> 16)) >> 16;
          w = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
        }
        store8(reinterpret_cast<uint16_t*>(b.p[j]) + i, k, w);
      }
      if (FP8) {
        uint32_t bm, bv;
        const uint2 qm = encode8<FOG_E4M3>(m, r, bm), qv = encode8<FOG_E5M2>(v, r, bv);
        store_codes(reinterpret_cast<uint8_t*>(b.m[j]) + i, k, qm);
        store_codes(reinterpret_cast<uint8_t*>(b.v[j]) + i, k, qv);
        if ((threadIdx.x & 15) == 0) {
          b.ms[j][i >> 7] = (uint8_t)bm;
          b.vs[j][i >> 7] = (uint8_t)bv;
        }
      } else {
        store8(reinterpret_cast<float*>(b.m[j]) + i, k, m);
        store8(reinterpret_cast<float*>(b.v[j]) + i, k, v);
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
    if (j.n > ((int64_t)1 << 37)) return FOG_ERR_UNSUPPORTED;      // a batch of such tensors has fewer than 2^31 pieces
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
  AdamBatch b;
  bool launched = false;
  b.count = b.pieces = 0;
  auto flush = [&]() {
    if (b.count == 0) return;
    const int groups = b.pieces < GROUPS ? b.pieces : GROUPS;
    if (fp8) adamw_kernel<true><<<groups, kThreads, 0, (hipStream_t)stream>>>(b, s);
    else     adamw_kernel<false><<<groups, kThreads, 0, (hipStream_t)stream>>>(b, s);
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
    b.pieces += (int)((j.n + PIECE - 1) / PIECE);
  }
  flush();
  return launched ? fog_launch_status() : FOG_OK;
}
