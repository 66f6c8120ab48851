// Rotary positions between the projection and attention: the QK norm, the turn by the token's position, the FP8 cast and the change from the projection's
// layout to the heads that attention reads, in one pass; and the way back.
//
// Bound by memory: forward 2 bytes read and 1 written an element, backward 2 (4 with the norm) and 1 or 3.  Q and K of 2 x 4096 tokens, 32 and 8 heads of 128, and V:
// a whole call of the forward 31.5 us (50 M elements, 4.9 TB/s), of which some 4 are the launch behind it that takes the maxima together, backward with the
// norm 49.5 us (4.8 TB/s); 24 single tokens: 5 us and 2, less than a call takes on the host.  (That launch stands in for a zeroed word and an atomic from each of some thousand workgroups.  A call by one
// workgroup, without it, was slower even at the smallest sizes: 13 us.)
//
// A token's vector of one head (D elements) belongs to LPR lanes, a wave takes 64 / LPR tokens and walks some heads of them, so that the cosines
// and sines, 16 of them a lane, are loaded once for all of these.  A lane holds two runs of eight elements: in the half layout eight elements and their
// eight partners, side by side eight pairs that lie together, and sixteen elements behind the turned part: no element has its partner in another lane.
#include <cfloat>
#include <cmath>

#include "common.h"
#include "launch.h"
#include "layout.h"

namespace {

constexpr int kThreads = 256;
constexpr int WORDS = 16384;             // most workgroups of a launch: an abs-max of each in the workspace
constexpr int JOBS = FOG_ROPE_JOBS_MAX;
constexpr int HEADS_MAX = 1 << 24;

struct Job {
  fog_heads in, q;                       // in: x of the forward, dy of the backward
  const float* scale;
  int heads, first;                      // first: number of the job's first workgroup
  float gain;
  uint8_t rotate, e5m2;
};
struct Back {
  fog_heads x, dx;
};
// (A launch costs the host by its arguments: for Q, K and V of a decoding step, room for eight jobs of both directions in 1.4 KB took 8.1 us a call, eight of one in
// 0.9 KB 6.1.  So calls of up to FEW jobs have a form of their own.)
constexpr int FEW = 4;
template <bool GRAD, int N>
struct Jobs {
  Job job[N];
  int count;
};
template <int N>
struct Jobs<true, N> {
  Job job[N];
  int count;
  Back back[N];
};
struct Shape {
  const float* table;
  const void* pos;
  uint32_t* part;                        // a word for each workgroup, or NULL
  int64_t positions, offset;
  uint32_t tokens, S, groups;            // groups: of tokens that a job's workgroups walk side by side
  float inv_cols;                        // 1 / D
  bool overlap;                          // eight does not divide a stretch of the FULL form
  int D, rot, segment, pos_bytes;        // segment: heads of a workgroup
  int side;                              // log2 of the tokens that a workgroup takes side by side; its other vectors are more of their heads
};
static_assert(sizeof(Jobs<true, JOBS>) + sizeof(Shape) <= 4096, "arguments of a launch");

template <int CTRL>
FOG_DEVICE float dpp_add(float s) {
  return s + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(s), CTRL, 0xF, 0xF, false));
}
// Sum over the LPR lanes of a vector, in every lane.
template <int LPR>
FOG_DEVICE float row_sum(float s) {
  s = dpp_add<0xB1>(s);                  // lane ^ 1
  s = dpp_add<0x4E>(s);                  // lane ^ 2
  if (LPR >= 8) s = dpp_add<0x141>(s);   // the other four of eight
  if (LPR >= 16) s = dpp_add<0x140>(s);  // the other eight of sixteen
  if (LPR >= 32) s += __shfl_xor(s, 16, 64);
  if (LPR >= 64) s += __shfl_xor(s, 32, 64);
  return s;
}

// gain / rms, half a unit in the last place and a little more: one Newton step on the hardware's reciprocal square root with the residue of r^2 m - 1 to twice the
// places, which is both shorter and closer than a correctly rounded root and a division.  0 for a vector of zeros, NaN for one that holds a NaN.
FOG_DEVICE float inv_rms(float sumsq, float inv_cols, float gain) {
  const float m = sumsq * inv_cols;
  if (__builtin_expect(!(m >= 0x1p-100f && m <= 0x1p+100f), 0)) return m != 0.0f ? gain / __builtin_sqrtf(m) : 0.0f;
  const float r = __builtin_amdgcn_rsqf(m);
  const float h = r * r, l = __builtin_fmaf(r, r, -h);
  const float e = __builtin_fmaf(-m, l, __builtin_fmaf(-m, h, 1.0f));       // 1 - m r^2
  return gain * __builtin_fmaf(0.5f * r, e, r);
}

FOG_DEVICE void unpack8(uint4 v, float (&f)[8]) {
  f[0] = bf16lo(v.x); f[1] = bf16hi(v.x); f[2] = bf16lo(v.y); f[3] = bf16hi(v.y);
  f[4] = bf16lo(v.z); f[5] = bf16hi(v.z); f[6] = bf16lo(v.w); f[7] = bf16hi(v.w);
}
FOG_DEVICE uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

// Runs of eight elements; those of FULL are whole (or not there at all, n == 0).
template <bool FULL>
FOG_DEVICE uint4 fetch(const uint16_t* p, int n) {
  if (FULL) return n > 0 ? ld_any_nt16(p) : make_uint4(0, 0, 0, 0);
  return n >= 8 ? ld_any_nt16(p) : ld_upto8(p, n);
}
typedef u32x2 __attribute__((aligned(1))) u32x2_byte;
template <bool FULL>
FOG_DEVICE void store_codes(uint8_t* p, uint2 w, int n) {
  if (FULL ? n > 0 : n >= 8) {
    u32x2 v = {w.x, w.y};
    *reinterpret_cast<u32x2_byte*>(p) = v;
  } else if (!FULL) {
    st_upto8(p, w, n);
  }
}
// Codes of two runs whose next ones the neighbour lane has: the even lane stores both first runs, the odd one both second runs.  Written through: without, the next
// launch waits for what the caches still have to write back (31.7 -> 30.6 us forward, 51.7 -> 50.5 backward); past the caches 33.5 us, and 39 in pieces of eight.
FOG_DEVICE uint32_t beside(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, false); }
FOG_DEVICE void store_even(uint8_t* to, int offA, int offB, uint2 a, uint2 e, bool odd) {
  const uint32_t x = beside(odd ? a.x : e.x), y = beside(odd ? a.y : e.y);
  st_through16(to + (odd ? offB - 8 : offA), odd ? make_uint4(x, y, e.x, e.y) : make_uint4(a.x, a.y, x, y));
}
template <bool FULL>
FOG_DEVICE void store_half(uint16_t* p, uint4 w, int n) {
  if (FULL ? n > 0 : n >= 8) st_any16(p, w);
  else if (!FULL) st_upto8(p, w, n);
}
// Four floats at each of two addresses of a float.
FOG_DEVICE void floats8(const float* p, const float* r, float (&f)[8]) {
  const uint4 a = ld_any16(p), b = ld_any16(r);
  f[0] = __uint_as_float(a.x); f[1] = __uint_as_float(a.y); f[2] = __uint_as_float(a.z); f[3] = __uint_as_float(a.w);
  f[4] = __uint_as_float(b.x); f[5] = __uint_as_float(b.y); f[6] = __uint_as_float(b.z); f[7] = __uint_as_float(b.w);
}
// Zeros in the place of the first `skip` of sixteen elements.
FOG_DEVICE void skip16(float (&a)[8], float (&b)[8], int skip_a, int skip_b) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (k < skip_a) a[k] = 0.0f;
    if (k < skip_b) b[k] = 0.0f;
  }
}

// Eight numbers to codes.  With CLAMP they are limited to the format first; without it the wave's converts saturate.
template <bool CLAMP>
FOG_DEVICE uint2 convert8(const float (&y)[8], bool e5m2) {
  if (e5m2)
    return CLAMP ? make_uint2(cvt4_fp8<FOG_E5M2>(y[0], y[1], y[2], y[3]), cvt4_fp8<FOG_E5M2>(y[4], y[5], y[6], y[7]))
                 : make_uint2(cvt4_fp8_finite<FOG_E5M2>(y[0], y[1], y[2], y[3]), cvt4_fp8_finite<FOG_E5M2>(y[4], y[5], y[6], y[7]));
  return CLAMP ? make_uint2(cvt4_fp8<FOG_E4M3>(y[0], y[1], y[2], y[3]), cvt4_fp8<FOG_E4M3>(y[4], y[5], y[6], y[7]))
               : make_uint2(cvt4_fp8_finite<FOG_E4M3>(y[0], y[1], y[2], y[3]), cvt4_fp8_finite<FOG_E4M3>(y[4], y[5], y[6], y[7]));
}
// What convert8 does not do, for vectors that hold an infinity or a NaN: infinities become the largest finite number, a NaN a zero of its sign under a
// code's seven set bits.  (Beside the conversion and not in it: kernels of a few microseconds are as long as their code.)
FOG_DEVICE uint2 tame8(float (&y)[8]) {
  uint32_t n[2] = {0u, 0u};
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (y[k] != y[k]) n[k >> 2] |= 0x7Fu << (8 * (k & 3));
    y[k] = y[k] != y[k] ? __builtin_copysignf(0.0f, y[k]) : __builtin_amdgcn_fmed3f(y[k], -FLT_MAX, FLT_MAX);
  }
  return make_uint2(n[0], n[1]);
}
FOG_DEVICE uint2 with(uint2 q, uint2 n) { return make_uint2(q.x | n.x, q.y | n.y); }

// The turn by (c, s) of eight pairs, or with BACK its transpose.
template <bool INTER, bool BACK>
FOG_DEVICE void turn(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8]) {
  auto pair = [](float& u, float& w, float c, float s) {
    const float v = BACK ? __builtin_fmaf(u, c, w * s) : __builtin_fmaf(u, c, -(w * s));
    w = BACK ? __builtin_fmaf(w, c, -(u * s)) : __builtin_fmaf(w, c, u * s);
    u = v;
  };
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (!INTER) pair(a[k], b[k], c[k], s[k]);
    else if (k < 4) pair(a[2 * k], a[2 * k + 1], c[k], s[k]);
    else pair(b[2 * k - 8], b[2 * k - 7], c[k], s[k]);
  }
}

// What the runs of a call look like: of any length; whole (FULL); half a stretch apart in stretches of whole thirty-twos (EVEN).  Kernels of their own: with EVEN a
// choice in the FULL ones, 24 tokens took 6.5 us from a graph instead of 6.05, the gradient of 1 x 333 8.45 instead of 7.8, of 2 x 4096 50.6 instead of 49.3.
enum { ANY, FULL_RUNS, EVEN_RUNS };
template <int LPR, bool INTER, bool GRAD, int FORM, int N>
__global__ __launch_bounds__(kThreads) void rope_kernel(Jobs<GRAD, N> jobs, Shape sh) {
  constexpr int VECTORS = kThreads / LPR;       // of a workgroup at a time
  constexpr int U = GRAD ? 2 : 1;               // heads in flight
  constexpr bool FULL = FORM != ANY, EVEN = FORM == EVEN_RUNS;
  int j = 0;
  while (j + 1 < jobs.count && (int)blockIdx.x >= jobs.job[j + 1].first) ++j;
  const Job& job = jobs.job[j];
  const uint32_t at = blockIdx.x - job.first, segments = (uint32_t)((job.heads + sh.segment - 1) / sh.segment);
  // The segments of the same tokens on one XCD (workgroups eight apart), so that its L2 has their rows of the table for all but the first (2 x 4096: 34.4 -> 33.7 us).
  const uint32_t eights = sh.groups & ~7u;
  const bool apart = at < eights * segments;
  const uint32_t group0 = apart ? (at & 7u) + 8u * (at / (8u * segments)) : at / segments, segment = apart ? (at >> 3) % segments : at % segments;
  const int h0 = (int)segment * sh.segment, h1 = h0 + sh.segment < job.heads ? h0 + sh.segment : job.heads;
  const uint32_t vector = threadIdx.x / LPR, tokens = 1u << sh.side;
  const int slot = (int)(vector >> sh.side), slots = VECTORS >> sh.side;
  const int lane = threadIdx.x % LPR;
  const bool rotate = job.rotate != 0;
  const int half = rotate ? sh.rot >> 1 : 0, turners = (half + 7) >> 3;
  const bool on = lane < turners;
  // Where the lane's two runs begin and how long they are.  In the FULL form every run is of eight: the last one of a stretch that eight does not divide
  // reaches back over elements of the lane in front of it, which gives them the same values; only sums leave those out (skip).
  // EVEN: a lane's runs lie half a stretch apart in either layout, so that each load of a wave covers whole lines, and two lanes
  // store the codes of one's first and the other's second runs, sixteen bytes each (2 x 4096, 32/8 heads: 33.7 -> 31.6 us forward, 52.5 -> 51.6 backward).
  int offA, offB, nA, nB, skipA = 0, skipB = 0, first = 8 * lane;        // first, firstB: pairs whose cosines come first and from the fifth on
  const int rest = sh.D - 2 * half;
  if (EVEN) {
    const int width = on ? half : rest >> 1, l = on ? lane : lane - turners;
    offA = (on ? 0 : 2 * half) + 8 * l;
    offB = offA + width;
    nA = nB = 8 * l < width ? 8 : 0;
    if (INTER) first = 4 * lane;
  } else if (on) {
    const int pairs = half - 8 * lane < 8 ? half - 8 * lane : 8;
    if (FULL) first -= 8 - pairs;
    offA = (INTER ? 2 : 1) * first;
    offB = INTER ? offA + 8 : offA + half;
    nA = INTER ? (2 * pairs < 8 ? 2 * pairs : 8) : pairs;
    nB = INTER ? 2 * pairs - nA : pairs;
  } else {
    offA = 2 * half + 16 * (lane - turners);
    offB = offA + 8;
    const int n = sh.D - offA;
    nA = n < 0 ? 0 : n < 8 ? n : 8;
    nB = n - 8 < 0 ? 0 : n - 8 < 8 ? n - 8 : 8;
    if (FULL && n > 0 && n < 16) {
      offB = sh.D - 8;
      if (rest >= 16) offA = sh.D - 16;
    }
  }
  const int firstB = INTER && EVEN ? first + (half >> 1) : first + 4;
  if (FULL && !EVEN && nA + nB > 0) {
    if (on && !INTER) {
      skipA = skipB = 8 - nA;
    } else if (on || rest >= 16) {      // sixteen elements in a row, the last ones new
      const int skip = 16 - (nA + nB);
      skipA = skip < 8 ? skip : 8;
      skipB = skip - skipA;
    } else {
      skipB = 8 - nB;
    }
    nA = nB = 8;
  }
  const float rho = job.q.p ? *job.scale : 0.0f;
  const bool norm = job.gain > 0.0f, e5m2 = job.e5m2 != 0;
  if (!GRAD) saturating_converts();      // (the backward converts to bf16, which the mode would saturate too)
  float top = 0.0f;
  bool nan = false;
  uint32_t top_bits = 0u;
  for (uint32_t group = group0; group * (uint64_t)tokens < sh.tokens; group += sh.groups) {
    const uint32_t t = group * tokens + (vector & (tokens - 1));
    if (t >= sh.tokens) break;           // (whole vectors: their lanes leave together)
    const uint32_t b = t / sh.S, s = t - b * sh.S;
    const uint16_t* in = reinterpret_cast<const uint16_t*>(job.in.p) + b * job.in.batch + s * job.in.token;
    uint8_t* q = job.q.p ? reinterpret_cast<uint8_t*>(job.q.p) + b * job.q.batch + s * job.q.token : nullptr;
    const uint16_t* xin = nullptr;
    uint16_t* dx = nullptr;
    int64_t x_head = 0, dx_head = 0;
    if constexpr (GRAD) {
      const Back& back = jobs.back[j];
      if (norm) xin = reinterpret_cast<const uint16_t*>(back.x.p) + b * back.x.batch + s * back.x.token;
      if (back.dx.p) dx = reinterpret_cast<uint16_t*>(back.dx.p) + b * back.dx.batch + s * back.dx.token;
      x_head = back.x.head;
      dx_head = back.dx.head;
    }
    bool there = true;
    float c[8], sn[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) { c[k] = 1.0f; sn[k] = 0.0f; }
    if (rotate) {
      const int64_t p = !sh.pos ? sh.offset + (int64_t)s
                                : sh.pos_bytes == 8 ? reinterpret_cast<const int64_t*>(sh.pos)[t] : (int64_t)reinterpret_cast<const int32_t*>(sh.pos)[t];
      there = p >= 0 && p < sh.positions;
      if (on && there) {
        const float* row = sh.table + p * sh.rot + first;
        if (FULL) {
          const float* later = sh.table + p * sh.rot + firstB;
          floats8(row, later, c);
          floats8(row + half, later + half, sn);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (first + k < half) { c[k] = row[k]; sn[k] = row[half + k]; }
        }
      }
    }
    for (int h = h0 + slot; h < h1; h += U * slots) {
      uint4 va[U], vb[U], xa[U], xb[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        va[u] = vb[u] = xa[u] = xb[u] = make_uint4(0, 0, 0, 0);
        if (h + u * slots < h1) {
          const uint16_t* p = in + (h + u * slots) * job.in.head;
          va[u] = fetch<FULL>(p + offA, nA);
          vb[u] = fetch<FULL>(p + offB, nB);
          if (GRAD && norm) {
            const uint16_t* x = xin + (h + u * slots) * x_head;
            xa[u] = fetch<FULL>(x + offA, nA);
            xb[u] = fetch<FULL>(x + offB, nB);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h + u * slots >= h1) break;
        float a[8], e[8];
        unpack8(va[u], a);
        unpack8(vb[u], e);
        if (!GRAD) {
          float inv = 1.0f;
          if (norm) {
            float p[8], r[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) { p[k] = a[k]; r[k] = e[k]; }
            if (FORM == FULL_RUNS && sh.overlap) skip16(p, r, skipA, skipB);
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              sum[k & 3] = __builtin_fmaf(p[k], p[k], sum[k & 3]);
              sum[k & 3] = __builtin_fmaf(r[k], r[k], sum[k & 3]);
            }
            inv = inv_rms(row_sum<LPR>((sum[0] + sum[1]) + (sum[2] + sum[3])), sh.inv_cols, job.gain);
          }
          // the turn is linear: the norm's factor comes behind it, as one number with the scale
          if (on) turn<INTER, false>(a, e, c, sn);
          if (!there) {
#pragma unroll
            for (int k = 0; k < 8; ++k) a[k] = e[k] = 0.0f;
            inv = 0.0f;
          }
          float most = 0.0f;               // (a NaN stays: finite products need neither a clamp nor a NaN test)
#pragma unroll
          for (int k = 0; k < 8; ++k) most = __builtin_elementwise_maximum(most, __builtin_elementwise_maximum(fabsf(a[k]), fabsf(e[k])));
          float f = inv * rho;
          if (__builtin_expect(!(fabsf(f) <= FLT_MAX), 0)) {      // a short vector under a large scale: the factors one by one
#pragma unroll
            for (int k = 0; k < 8; ++k) { a[k] *= inv; e[k] *= inv; }
            most *= inv;
            inv = 1.0f;
            f = rho;
          }
          top = fmaxf(top, most * inv);
#pragma unroll
          for (int k = 0; k < 8; ++k) { a[k] *= f; e[k] *= f; }
          uint2 na = make_uint2(0, 0), ne = na;
          if (__builtin_expect(!(most * fabsf(f) <= FLT_MAX), 0)) {
            na = tame8(a);
            ne = tame8(e);
            nan |= (na.x | na.y | ne.x | ne.y) != 0u;
          }
          uint8_t* to = q + (h + u * slots) * job.q.head;
          const uint2 ca = with(convert8<false>(a, e5m2), na), ce = with(convert8<false>(e, e5m2), ne);
          if (EVEN) {
            if (nA > 0) store_even(to, offA, offB, ca, ce, (lane & 1) != 0);
          } else {
            store_codes<FULL>(to + offA, ca, nA);
            store_codes<FULL>(to + offB, ce, nB);
          }
        } else {
          if (on) turn<INTER, true>(a, e, c, sn);
          if (norm) {
            float x0[8], x1[8], p[8], r[8], xx = 0.0f, xd = 0.0f;
            unpack8(xa[u], x0);
            unpack8(xb[u], x1);
#pragma unroll
            for (int k = 0; k < 8; ++k) { p[k] = x0[k]; r[k] = x1[k]; }
            if (FORM == FULL_RUNS && sh.overlap) skip16(p, r, skipA, skipB);
#pragma unroll
            for (int k = 0; k < 8; ++k) { xx = __builtin_fmaf(p[k], p[k], xx); xd = __builtin_fmaf(p[k], a[k], xd); }
#pragma unroll
            for (int k = 0; k < 8; ++k) { xx = __builtin_fmaf(r[k], r[k], xx); xd = __builtin_fmaf(r[k], e[k], xd); }
            xx = row_sum<LPR>(xx);
            xd = row_sum<LPR>(xd);
            const float inv = inv_rms(xx, sh.inv_cols, job.gain), along = inv != 0.0f ? xd / xx : 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              a[k] = inv * __builtin_fmaf(-x0[k], along, a[k]);
              e[k] = inv * __builtin_fmaf(-x1[k], along, e[k]);
            }
          }
          uint4 wa = pack8(a), wb = pack8(e);
          if (!there) wa = wb = make_uint4(0, 0, 0, 0);
          uint32_t most = 0u;
          most = pkmax_abs_bf16(most, wa.x); most = pkmax_abs_bf16(most, wa.y); most = pkmax_abs_bf16(most, wa.z); most = pkmax_abs_bf16(most, wa.w);
          most = pkmax_abs_bf16(most, wb.x); most = pkmax_abs_bf16(most, wb.y); most = pkmax_abs_bf16(most, wb.z); most = pkmax_abs_bf16(most, wb.w);
          const uint32_t larger = max_of_pair(most);
          top_bits = top_bits > larger ? top_bits : larger;
          if (dx) {
            uint16_t* to = dx + (h + u * slots) * dx_head;
            store_half<FULL>(to + offA, wa, nA);
            store_half<FULL>(to + offB, wb, nB);
          }
          if (q) {
            unpack8(wa, a);
            unpack8(wb, e);
#pragma unroll
            for (int k = 0; k < 8; ++k) { a[k] *= rho; e[k] *= rho; }
            uint2 na = make_uint2(0, 0), ne = na;
            if (__builtin_expect(!(__uint_as_float(larger << 16) * fabsf(rho) <= FLT_MAX), 0)) {
              na = tame8(a);
              ne = tame8(e);
            }
            uint8_t* to = q + (h + u * slots) * job.q.head;
            const uint2 ca = with(convert8<true>(a, e5m2), na), ce = with(convert8<true>(e, e5m2), ne);
            if (EVEN) {
              if (nA > 0) store_even(to, offA, offB, ca, ce, (lane & 1) != 0);
            } else {
              store_codes<FULL>(to + offA, ca, nA);
              store_codes<FULL>(to + offB, ce, nB);
            }
          }
        }
      }
    }
  }
  if (sh.part) {
    const uint32_t m = wave_max_u32(GRAD ? top_bits << 16 : amax_bits(top, nan));
    __shared__ uint32_t wave[kThreads / 64];
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t r = wave[0];
#pragma unroll
      for (int w = 1; w < kThreads / 64; ++w) r = r > wave[w] ? r : wave[w];
      sh.part[blockIdx.x] = r;
    }
  }
}

// The largest of the words of all jobs that name a result.
struct Tops {
  uint32_t* amax[JOBS];
  int first[JOBS + 1];
  uint8_t same[JOBS];      // jobs that name the result of job j
};
// (512 threads against 256: half as many rounds of loads one behind the other, 51.4 -> 50.7 us for a whole gradient of 2 x 4096 tokens.)
constexpr int kTopThreads = 512;
__global__ __launch_bounds__(kTopThreads) void rope_top_kernel(Tops t, const uint32_t* __restrict__ part) {
  const int j = blockIdx.x;
  if (!t.amax[j] || (t.same[j] & ((1 << j) - 1))) return;      // the first of them writes it
  uint32_t m = 0u;
  for (int k = 0; k < JOBS; ++k)
    if (t.same[j] >> k & 1)
      for (int i = t.first[k] + (int)threadIdx.x; i < t.first[k + 1]; i += kTopThreads) m = m > part[i] ? m : part[i];
  m = wave_max_u32(m);
  __shared__ uint32_t wave[kTopThreads / 64];
  if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kTopThreads / 64; ++w) m = m > wave[w] ? m : wave[w];
    *t.amax[j] = m;
  }
}

// cos and sin of every position and pair from binary64 angles: far positions turn 10^5 times and more.  A thread keeps its pair's frequency for
// sixteen positions and more.  Bound by the binary64 functions: 4096 x 128 7 us, 131072 x 128 35 (10 for its stores alone), once for a program.
constexpr int TABLE_ROWS = 64;
__global__ __launch_bounds__(kThreads) void rope_table_kernel(fog_rope_scaling sc, int64_t first, int64_t positions, int half, float* __restrict__ table) {
  for (int i = threadIdx.x & 63; i < half; i += 64) {
    double f = exp2(-(double)i / (double)half * log2(sc.base));
    if (sc.factor != 1.0) {
      double keep = 0.0;
      if (sc.original > 0.0) {
        keep = (sc.original * f * 0.15915494309189533577 - sc.low) / (sc.high - sc.low);
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      }
      f = f * ((1.0 - keep) / sc.factor + keep);
    }
    for (int64_t p0 = (int64_t)blockIdx.x * TABLE_ROWS; p0 < positions; p0 += (int64_t)gridDim.x * TABLE_ROWS)
      for (int r = threadIdx.x >> 6; r < TABLE_ROWS; r += kThreads / 64) {
        if (p0 + r >= positions) break;
        double s, c;
        sincos((double)(first + p0 + r) * f, &s, &c);
        float* row = table + (p0 + r) * 2 * half;
        row[i] = (float)(c * sc.amplitude);
        row[half + i] = (float)(s * sc.amplitude);
      }
  }
}

// ---------------------------------------------------------------- host
// Where [B, S, heads] vectors of D elements lie.
fog_status make_box(const fog_heads& h, int B, int S, int heads, int D, int size, FogBox* box) {
  const int64_t n[3] = {B, S, heads}, stride[3] = {h.batch, h.token, h.head};
  return fog_make_box(h.p, 3, n, stride, D, size, box);
}

struct Call {
  FogBox in[2 * JOBS + 2], out[2 * JOBS];
  int ins = 0, outs = 0;
  fog_status add(const fog_heads& h, int B, int S, int heads, int D, int size, bool written) {
    const fog_status st = make_box(h, B, S, heads, D, size, written ? &out[outs] : &in[ins]);
    if (st != FOG_OK) return st;
    if (written && !fog_injective(out[outs])) return FOG_ERR_SHAPE;
    ++(written ? outs : ins);
    return FOG_OK;
  }
  // The table and the positions, which are read as well.
  fog_status add_common(const float* table, int64_t positions, int rot, const void* pos, int64_t tokens, int pos_bytes) {
    const int64_t n[2] = {positions, tokens}, stride[2] = {rot, 1};
    fog_status st = FOG_OK;
    if (table && rot > 0 && positions > 0) st = fog_make_box(table, 1, n, stride, rot, 4, &in[ins++]);
    if (st == FOG_OK && pos) st = fog_make_box(pos, 1, n + 1, stride + 1, 1, pos_bytes, &in[ins++]);
    return st;
  }
  bool fine() const {
    for (int i = 0; i < outs; ++i) {
      for (int k = 0; k < ins; ++k)
        if (!fog_apart_as_spans(out[i], in[k])) return false;
      for (int k = 0; k < i; ++k)
        if (!fog_apart(out[k], out[i])) return false;
    }
    return true;
  }
};

// What both directions look at before their jobs.
fog_status check_call(int count, const void* jobs, int B, int S, int D, int rot, fog_rope_layout layout, const float* table, int64_t positions, const void* pos,
                      int pos_bytes, int64_t offset) {
  if (count < 0 || count > JOBS || B < 0 || S < 0 || D < 0 || rot < 0 || rot > D || positions < 0) return FOG_ERR_SHAPE;
  if (count > 0 && !jobs) return FOG_ERR_NULL;
  if (layout != FOG_ROPE_HALF && layout != FOG_ROPE_INTERLEAVED) return FOG_ERR_UNSUPPORTED;
  if ((rot & 1) || D > FOG_ROPE_DIM_MAX || (int64_t)B * S > 0x7FFFFFFF) return FOG_ERR_UNSUPPORTED;
  if (pos && pos_bytes != 4 && pos_bytes != 8) return FOG_ERR_UNSUPPORTED;
  if (offset > ((int64_t)1 << 62) || offset < -((int64_t)1 << 62)) return FOG_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(table) & 3) || (pos && (reinterpret_cast<uintptr_t>(pos) & (uintptr_t)(pos_bytes - 1)))) return FOG_ERR_ALIGN;
  return FOG_OK;
}

template <bool GRAD>
fog_status launch(Jobs<GRAD, JOBS>& jobs, Shape& sh, float* const* amax, bool any_amax, int B, bool inter, void* workspace, hipStream_t s) {
  const int lanes = (sh.rot / 2 + 7) / 8 + (sh.D - sh.rot + 15) / 16, plain = (sh.D + 15) / 16, need = lanes > plain ? lanes : plain;
  const int lpr = need <= 4 ? 4 : need <= 8 ? 8 : need <= 16 ? 16 : need <= 32 ? 32 : 64;
  // Whole runs of eight everywhere: no stretch (turned pairs, the rest) is shorter than one.
  bool full = sh.D >= 8 && (sh.rot == 0 || sh.rot >= 16), plain_jobs = false;
  for (int j = 0; j < jobs.count; ++j) plain_jobs |= !jobs.job[j].rotate;
  if (sh.rot < sh.D) full = full && sh.D - sh.rot >= 8;
  const bool even = full && sh.rot % 32 == 0 && sh.D % 32 == 0;      // (then in jobs that are not turned, too)
  sh.overlap = sh.rot % 16 != 0 || (sh.D - sh.rot) % 16 != 0 || (plain_jobs && sh.D % 16 != 0);
  sh.tokens = (uint32_t)((int64_t)B * sh.S);
  sh.inv_cols = sh.D > 0 ? 1.0f / (float)sh.D : 0.0f;
  const int vectors = kThreads / lpr;
  while ((2 << sh.side) <= vectors && (1u << sh.side) < sh.tokens) ++sh.side;
  const int64_t groups = ((int64_t)sh.tokens + (1 << sh.side) - 1) >> sh.side;
  // Heads of a workgroup: as few as fill the chip, up to eight for each of its slots.
  const int64_t want = 8 * (int64_t)fog_compute_units(), slots = vectors >> sh.side;
  auto segments = [&](int64_t segment) {
    int64_t n = 0;
    for (int j = 0; j < jobs.count; ++j) n += (jobs.job[j].heads + segment - 1) / segment;
    return n;
  };
  int64_t segment = slots;
  while ((segment < 8 * slots && segments(segment) * groups > want) || segments(segment) > WORDS / 2) segment *= 2;
  sh.segment = (int)segment;
  const int64_t all = segments(segment), most = all > 0 ? WORDS / all : 1;
  sh.groups = (uint32_t)(groups < most ? groups : most);
  int next = 0;
  Tops tops = {};
  for (int j = 0; j < jobs.count; ++j) {
    jobs.job[j].first = tops.first[j] = next;
    next += (int)((jobs.job[j].heads + segment - 1) / segment) * (int)sh.groups;
    tops.amax[j] = reinterpret_cast<uint32_t*>(amax[j]);
    for (int k = 0; k < jobs.count; ++k)
      if (amax[j] && amax[k] == amax[j]) tops.same[j] |= (uint8_t)(1 << k);
  }
  for (int j = jobs.count; j <= JOBS; ++j) tops.first[j] = next;
  sh.part = any_amax ? reinterpret_cast<uint32_t*>(workspace) : nullptr;
  if (next > 0 && sh.tokens > 0 && sh.D > 0) {
    Jobs<GRAD, FEW> few;
    if (jobs.count <= FEW) {
      few.count = jobs.count;
      for (int j = 0; j < FEW; ++j) {
        few.job[j] = jobs.job[j];
        if constexpr (GRAD) few.back[j] = jobs.back[j];
      }
    }
#define FOG_ROPE(L)                                                                                                        \
  do {                                                                                                                     \
    if (!full)                  FOG_ROPE_FORM(L, ANY, JOBS, jobs);                                                          \
    else if (jobs.count <= FEW) { if (even) FOG_ROPE_FORM(L, EVEN_RUNS, FEW, few); else FOG_ROPE_FORM(L, FULL_RUNS, FEW, few); }       \
    else                        { if (even) FOG_ROPE_FORM(L, EVEN_RUNS, JOBS, jobs); else FOG_ROPE_FORM(L, FULL_RUNS, JOBS, jobs); }   \
  } while (0)
#define FOG_ROPE_FORM(L, FORM, N, args)                                                                                     \
  do {                                                                                                                      \
    if (inter) rope_kernel<L, true, GRAD, FORM, N><<<next, kThreads, 0, s>>>(args, sh);                                     \
    else rope_kernel<L, false, GRAD, FORM, N><<<next, kThreads, 0, s>>>(args, sh);                                          \
  } while (0)
    if (lpr == 4) FOG_ROPE(4);
    else if (lpr == 8) FOG_ROPE(8);
    else if (lpr == 16) FOG_ROPE(16);
    else if (lpr == 32) FOG_ROPE(32);
    else FOG_ROPE(64);
#undef FOG_ROPE
#undef FOG_ROPE_FORM
  } else {
    for (int j = 0; j <= JOBS; ++j) tops.first[j] = 0;
    if (!any_amax) return FOG_OK;
  }
  if (any_amax) rope_top_kernel<<<jobs.count, kTopThreads, 0, s>>>(tops, sh.part);
  return fog_launch_status();
}

}  // namespace

extern "C" fog_status fog_rope_table(const fog_rope_scaling* scaling, int64_t first, int64_t positions, int rot, float* table, void* stream) {
  fog_rope_scaling sc = {10000.0, 1.0, 0.0, 0.0, 0.0, 1.0};
  if (scaling) sc = *scaling;
  if (positions < 0 || rot < 0) return FOG_ERR_SHAPE;
  if ((rot & 1) || positions > ((int64_t)1 << 31) || first < -((int64_t)1 << 52) || first > ((int64_t)1 << 52)) return FOG_ERR_UNSUPPORTED;
  if (!(sc.base > 0.0) || !(sc.factor > 0.0) || !std::isfinite(sc.base) || !std::isfinite(sc.factor) || !std::isfinite(sc.amplitude)) return FOG_ERR_UNSUPPORTED;
  if (!(sc.original >= 0.0) || !std::isfinite(sc.original)) return FOG_ERR_UNSUPPORTED;
  if (sc.original > 0.0 && (!std::isfinite(sc.low) || !std::isfinite(sc.high) || !(sc.high > sc.low))) return FOG_ERR_UNSUPPORTED;
  if (positions == 0 || rot == 0) return FOG_OK;
  if (!table) return FOG_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(table) & 3) return FOG_ERR_ALIGN;
  const int64_t blocks = (positions + TABLE_ROWS - 1) / TABLE_ROWS;
  rope_table_kernel<<<(int)(blocks < (1 << 20) ? blocks : 1 << 20), kThreads, 0, (hipStream_t)stream>>>(sc, first, positions, rot / 2, table);
  return fog_launch_status();
}

extern "C" size_t fog_rope_workspace(void) { return WORDS * sizeof(uint32_t); }

extern "C" fog_status fog_rope_quantize(const fog_rope_job* jobs, int count, int B, int S, int D, int rot, fog_rope_layout layout, const float* table,
                                        int64_t positions, const void* pos, int pos_bytes, int64_t offset, void* workspace, size_t workspace_bytes,
                                        void* stream) {
  const fog_status st = check_call(count, jobs, B, S, D, rot, layout, table, positions, pos, pos_bytes, offset);
  if (st != FOG_OK) return st;
  Jobs<false, JOBS> all = {};
  Call call;
  float* amax[JOBS] = {};
  bool any_amax = false;
  const bool empty = B == 0 || S == 0 || D == 0;
  all.count = count;
  for (int j = 0; j < count; ++j) {
    const fog_rope_job& in = jobs[j];
    if (in.heads < 0) return FOG_ERR_SHAPE;
    if (in.heads > HEADS_MAX) return FOG_ERR_UNSUPPORTED;
    if ((in.fmt != FOG_E4M3 && in.fmt != FOG_E5M2) || !(in.gain >= 0.0f && in.gain <= FLT_MAX)) return FOG_ERR_UNSUPPORTED;
    if (!in.scale) return FOG_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(in.scale) | reinterpret_cast<uintptr_t>(in.amax)) & 3) return FOG_ERR_ALIGN;
    if (in.heads > 0 && !empty) {
      if (in.rotate && rot > 0 && !table) return FOG_ERR_NULL;
      fog_status s = call.add(in.x, B, S, in.heads, D, 2, false);
      if (s == FOG_OK) s = call.add(in.q, B, S, in.heads, D, 1, true);
      if (s != FOG_OK) return s;
    }
    Job& to = all.job[j];
    to.in = in.x; to.q = in.q; to.scale = in.scale; to.heads = empty ? 0 : in.heads; to.gain = in.gain; to.rotate = in.rotate && rot > 0; to.e5m2 = in.fmt == FOG_E5M2;
    amax[j] = in.amax;
    any_amax |= in.amax != nullptr;
  }
  const fog_status common = empty ? FOG_OK : call.add_common(table, positions, rot, pos, (int64_t)B * S, pos_bytes);
  if (common != FOG_OK) return common;
  if (!call.fine()) return FOG_ERR_UNSUPPORTED;
  if (any_amax && (!workspace || workspace_bytes < fog_rope_workspace())) return FOG_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 3) return FOG_ERR_ALIGN;
  Shape sh = {};
  sh.table = table; sh.pos = pos; sh.positions = positions; sh.offset = offset; sh.S = (uint32_t)S; sh.D = D; sh.rot = rot; sh.pos_bytes = pos_bytes;
  return launch<false>(all, sh, amax, any_amax, B, layout == FOG_ROPE_INTERLEAVED, workspace, (hipStream_t)stream);
}

extern "C" fog_status fog_rope_grad(const fog_rope_grad_job* jobs, int count, int B, int S, int D, int rot, fog_rope_layout layout, const float* table,
                                    int64_t positions, const void* pos, int pos_bytes, int64_t offset, void* workspace, size_t workspace_bytes, void* stream) {
  const fog_status st = check_call(count, jobs, B, S, D, rot, layout, table, positions, pos, pos_bytes, offset);
  if (st != FOG_OK) return st;
  Jobs<true, JOBS> all = {};
  Call call;
  float* amax[JOBS] = {};
  bool any_amax = false;
  const bool empty = B == 0 || S == 0 || D == 0;
  all.count = count;
  for (int j = 0; j < count; ++j) {
    const fog_rope_grad_job& in = jobs[j];
    if (in.heads < 0) return FOG_ERR_SHAPE;
    if (in.heads > HEADS_MAX) return FOG_ERR_UNSUPPORTED;
    if ((in.fmt != FOG_E4M3 && in.fmt != FOG_E5M2) || !(in.gain >= 0.0f && in.gain <= FLT_MAX)) return FOG_ERR_UNSUPPORTED;
    if (in.q.p && !in.scale) return FOG_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(in.scale) | reinterpret_cast<uintptr_t>(in.amax)) & 3) return FOG_ERR_ALIGN;
    if (in.heads > 0 && !empty) {
      if ((in.rotate && rot > 0 && !table) || (!in.q.p && !in.dx.p)) return FOG_ERR_NULL;
      fog_status s = call.add(in.dy, B, S, in.heads, D, 2, false);
      if (s == FOG_OK && in.gain > 0.0f) s = call.add(in.x, B, S, in.heads, D, 2, false);
      if (s == FOG_OK && in.dx.p) s = call.add(in.dx, B, S, in.heads, D, 2, true);
      if (s == FOG_OK && in.q.p) s = call.add(in.q, B, S, in.heads, D, 1, true);
      if (s != FOG_OK) return s;
    }
    Job& to = all.job[j];
    to.in = in.dy; all.back[j] = {in.x, in.dx}; to.q = in.q; to.scale = in.scale; to.heads = empty ? 0 : in.heads; to.gain = in.gain;
    to.rotate = in.rotate && rot > 0; to.e5m2 = in.fmt == FOG_E5M2;
    amax[j] = in.amax;
    any_amax |= in.amax != nullptr;
  }
  const fog_status common = empty ? FOG_OK : call.add_common(table, positions, rot, pos, (int64_t)B * S, pos_bytes);
  if (common != FOG_OK) return common;
  if (!call.fine()) return FOG_ERR_UNSUPPORTED;
  if (any_amax && (!workspace || workspace_bytes < fog_rope_workspace())) return FOG_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 3) return FOG_ERR_ALIGN;
  Shape sh = {};
  sh.table = table; sh.pos = pos; sh.positions = positions; sh.offset = offset; sh.S = (uint32_t)S; sh.D = D; sh.rot = rot; sh.pos_bytes = pos_bytes;
  return launch<true>(all, sh, amax, any_amax, B, layout == FOG_ROPE_INTERLEAVED, workspace, (hipStream_t)stream);
}
