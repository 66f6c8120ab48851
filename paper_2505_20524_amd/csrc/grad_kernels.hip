// The global norm of a step's gradients and their clipping to it.
//
// Both passes go over up to BATCH tensors a launch, cut into pieces of PIECE elements, so that one launch is as well filled by a single
// large tensor as by a hundred small ones.  Bound by memory: the norm reads every gradient once, clipping reads and writes it once.
// 33 gradients of 973 M elements in bf16 (1.95 GB): 922 us for both, 6.3 TB/s; 49 of 25 M: 29 us.  What that takes, us (33 / 49
// gradients): clipping by a workgroup for each piece instead of 2048 that walk, 1034 -> 960 / the same; its loads past the caches, 994
// -> 928 / 31 -> 29; 4096 workgroups for the sums instead of 2048 and 1024, 922, 928, 954 / the same.  Clipping from the last
// piece to the first, to find what the sums have left in the memory-side cache, loses: 938 -> 970 / 28 -> 31.
//
// Squares are added in binary64: the square of a binary32 number neither overflows nor vanishes there, so that the norm is finite
// whenever the gradients are, and a sum of 10^9 terms keeps all the places that a binary32 norm has.  The additions cost no time
// beside the reads.  Every workgroup leaves its sum in its own word and one workgroup adds the words in order: no atomics,
// the same result on every run.
#include <cfloat>

#include "common.h"
#include "launch.h"
#include "spans.h"

namespace {

constexpr int kThreads = 256;
constexpr int BATCH = 120;               // descriptions that fit a launch's arguments
constexpr int64_t PIECE = 8192;          // elements: 4 loads of 16 bytes a thread in bf16
constexpr int SUM_GROUPS = 4096;         // most workgroups of a launch that sums: one word of the workspace each
constexpr int TENSORS_MAX = 1 << 24;     // tensors of a call: their sums, SUM_GROUPS for each BATCH, are counted in 32 bits
constexpr int CLIP_GROUPS = 1 << 23;     // most workgroups of a launch that clips: grids are counted in threads of 32 bits

struct GradBatch {
  const void* g[BATCH];
  void* out[BATCH];
  int64_t n[BATCH];
  int first[BATCH];        // number of the tensor's first piece
  uint8_t f32[BATCH];
  int count, pieces;
};

// The tensor that piece p belongs to.
FOG_DEVICE int tensor_of(const GradBatch& b, int p) {
  int lo = 0, hi = b.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (b.first[mid] <= p) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

FOG_DEVICE void add_square(double& s, float v) {
  const double d = (double)v;
  s = __builtin_fma(d, d, s);
}

__global__ __launch_bounds__(kThreads) void sumsq_kernel(GradBatch b, double* __restrict__ part) {
  double s0 = 0.0, s1 = 0.0;
  for (int p = blockIdx.x; p < b.pieces; p += gridDim.x) {
    const int j = tensor_of(b, p);
    const int64_t at = (int64_t)(p - b.first[j]) * PIECE;
    const int n = (int)(b.n[j] - at < PIECE ? b.n[j] - at : PIECE);
    const bool f32 = b.f32[j] != 0;
    const uint8_t* base = reinterpret_cast<const uint8_t*>(b.g[j]) + at * (f32 ? 4 : 2);
    const int per = f32 ? 4 : 8, vecs = n / per, done = vecs * per;
    for (int i = threadIdx.x; i < vecs; i += 4 * kThreads) {
      uint4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        v[u] = make_uint4(0, 0, 0, 0);
        if (i + u * kThreads < vecs) v[u] = ld_any16(base + 16 * (int64_t)(i + u * kThreads));
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (f32) {
          add_square(s0, __uint_as_float(v[u].x)); add_square(s1, __uint_as_float(v[u].y));
          add_square(s0, __uint_as_float(v[u].z)); add_square(s1, __uint_as_float(v[u].w));
        } else {
          add_square(s0, bf16lo(v[u].x)); add_square(s1, bf16hi(v[u].x));
          add_square(s0, bf16lo(v[u].y)); add_square(s1, bf16hi(v[u].y));
          add_square(s0, bf16lo(v[u].z)); add_square(s1, bf16hi(v[u].z));
          add_square(s0, bf16lo(v[u].w)); add_square(s1, bf16hi(v[u].w));
        }
      }
    }
    for (int i = done + threadIdx.x; i < n; i += kThreads)
      add_square(s0, f32 ? reinterpret_cast<const float*>(base)[i] : bf16lo(reinterpret_cast<const uint16_t*>(base)[i]));
  }
  double s = s0 + s1;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
  __shared__ double wave[kThreads / 64];
  if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (wave[0] + wave[1]) + (wave[2] + wave[3]);
}

__global__ __launch_bounds__(1024) void sumsq_total_kernel(const double* __restrict__ part, int n, double* __restrict__ sumsq) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += part[i];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
  __shared__ double wave[16];
  if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < 16; ++w) t += wave[w];
    *sumsq = t;
  }
}

// max_norm / norm where the norm is finite and above max_norm, else 1.
FOG_DEVICE float clip_factor(double sumsq, float max_norm, double* norm) {
  const double r = __builtin_sqrt(sumsq);
  *norm = r;
  return r > (double)max_norm && r < __builtin_inf() ? (float)((double)max_norm / r) : 1.0f;
}

__global__ __launch_bounds__(kThreads) void clip_kernel(GradBatch b, const double* __restrict__ sumsq, float max_norm, float* __restrict__ norm_out) {
  double norm;
  const float c = clip_factor(*sumsq, max_norm, &norm);
  // a finite norm beyond binary32 is told as the largest finite number: what is not finite there says that the gradients are not
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm > (double)FLT_MAX && norm < __builtin_inf() ? FLT_MAX : (float)norm;
  for (int p = blockIdx.x; p < b.pieces; p += gridDim.x) {
    const int j = tensor_of(b, p);
    const int64_t at = (int64_t)(p - b.first[j]) * PIECE;
    const int n = (int)(b.n[j] - at < PIECE ? b.n[j] - at : PIECE);
    const bool f32 = b.f32[j] != 0;
    const uint8_t* src = reinterpret_cast<const uint8_t*>(b.g[j]) + at * (f32 ? 4 : 2);
    uint8_t* dst = reinterpret_cast<uint8_t*>(b.out[j]) + at * (f32 ? 4 : 2);
    if (src == dst && c == 1.0f) continue;       // nothing changes
    const int per = f32 ? 4 : 8, vecs = n / per, done = vecs * per;
    for (int i = threadIdx.x; i < vecs; i += 4 * kThreads) {
      uint4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i + u * kThreads < vecs) v[u] = ld_any_nt16(src + 16 * (int64_t)(i + u * kThreads));
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i + u * kThreads >= vecs) break;
        uint4 o = v[u];
        if (c != 1.0f) {
          if (f32)
            o = make_uint4(__float_as_uint(__uint_as_float(o.x) * c), __float_as_uint(__uint_as_float(o.y) * c),
                           __float_as_uint(__uint_as_float(o.z) * c), __float_as_uint(__uint_as_float(o.w) * c));
          else
            o = make_uint4(pack_bf16x2(bf16lo(o.x) * c, bf16hi(o.x) * c), pack_bf16x2(bf16lo(o.y) * c, bf16hi(o.y) * c),
                           pack_bf16x2(bf16lo(o.z) * c, bf16hi(o.z) * c), pack_bf16x2(bf16lo(o.w) * c, bf16hi(o.w) * c));
        }
        st_any_nt16(dst + 16 * (int64_t)(i + u * kThreads), o);
      }
    }
    for (int i = done + threadIdx.x; i < n; i += kThreads) {
      if (f32) {
        const uint32_t v = reinterpret_cast<const uint32_t*>(src)[i];
        reinterpret_cast<uint32_t*>(dst)[i] = c != 1.0f ? __float_as_uint(__uint_as_float(v) * c) : v;
      } else {
        const uint16_t v = reinterpret_cast<const uint16_t*>(src)[i];
        reinterpret_cast<uint16_t*>(dst)[i] = c != 1.0f ? (uint16_t)f32_to_bf16(bf16lo(v) * c) : v;
      }
    }
  }
}

fog_status check_jobs(const fog_grad_job* jobs, int count, bool with_out) {
  if (count < 0) return FOG_ERR_SHAPE;
  if (count > TENSORS_MAX) return FOG_ERR_UNSUPPORTED;
  if (count > 0 && !jobs) return FOG_ERR_NULL;
  for (int i = 0; i < count; ++i) {
    const fog_grad_job& j = jobs[i];
    if (j.n < 0) return FOG_ERR_SHAPE;
    if (j.type != FOG_BF16 && j.type != FOG_F32) return FOG_ERR_UNSUPPORTED;
    if (j.n > ((int64_t)1 << 37)) return FOG_ERR_UNSUPPORTED;      // a batch of such tensors has fewer than 2^31 pieces
    if (j.n == 0) continue;
    if (!j.g || (with_out && !j.out)) return FOG_ERR_NULL;
    const uintptr_t size = j.type == FOG_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(j.g) & (size - 1)) || (with_out && (reinterpret_cast<uintptr_t>(j.out) & (size - 1)))) return FOG_ERR_ALIGN;
  }
  return FOG_OK;
}

// Whether a result lies where another result, or a gradient that is not its own, lies: the pieces of a call are worked on in no order, and a
// gradient that is listed twice would be clipped once, twice or in parts.  (49 gradients with results elsewhere: 0.9 us of host time.)
fog_status check_overlaps(const fog_grad_job* jobs, int count) {
  FogSpans<256> spans(2 * (int64_t)count);
  if (!spans.ok()) return FOG_ERR_UNSUPPORTED;
  for (int i = 0; i < count; ++i) {
    const fog_grad_job& j = jobs[i];
    const int64_t bytes = j.n * (j.type == FOG_F32 ? 4 : 2);
    spans.add(j.out, bytes, true);
    if (j.g != j.out) spans.add(j.g, bytes, false);
  }
  return spans.apart() ? FOG_OK : FOG_ERR_UNSUPPORTED;
}

// The batches of a call, one after the other: take(batch) for each.
template <typename F>
void for_batches(const fog_grad_job* jobs, int count, F take) {
  GradBatch b;
  int pieces = 0;
  b.count = 0;
  auto flush = [&]() {
    if (b.count == 0) return;
    b.pieces = pieces;
    take(b);
    b.count = 0;
    pieces = 0;
  };
  for (int i = 0; i < count; ++i) {
    if (jobs[i].n == 0) continue;
    if (b.count == BATCH) flush();
    b.g[b.count] = jobs[i].g;
    b.out[b.count] = jobs[i].out;
    b.n[b.count] = jobs[i].n;
    b.f32[b.count] = jobs[i].type == FOG_F32;
    b.first[b.count] = pieces;
    pieces += (int)((jobs[i].n + PIECE - 1) / PIECE);
    ++b.count;
  }
  flush();
}

}  // namespace

extern "C" size_t fog_grad_sumsq_workspace(int count) {
  return count <= 0 || count > TENSORS_MAX ? 0 : (size_t)((count + BATCH - 1) / BATCH) * SUM_GROUPS * sizeof(double);
}

extern "C" fog_status fog_grad_sumsq(const fog_grad_job* jobs, int count, double* sumsq, void* workspace, size_t workspace_bytes, void* stream) {
  const fog_status st = check_jobs(jobs, count, false);
  if (st != FOG_OK) return st;
  if (!sumsq) return FOG_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(sumsq) & 7) return FOG_ERR_ALIGN;
  if (count > 0 && (!workspace || workspace_bytes < fog_grad_sumsq_workspace(count))) return FOG_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(workspace) & 7) return FOG_ERR_ALIGN;
  hipStream_t s = (hipStream_t)stream;
  double* part = reinterpret_cast<double*>(workspace);
  int words = 0;
  for_batches(jobs, count, [&](const GradBatch& b) {
    const int groups = b.pieces < SUM_GROUPS ? b.pieces : SUM_GROUPS;
    sumsq_kernel<<<groups, kThreads, 0, s>>>(b, part + words);
    words += groups;
  });
  sumsq_total_kernel<<<1, 1024, 0, s>>>(part, words, sumsq);
  return fog_launch_status();
}

extern "C" fog_status fog_grad_clip(const fog_grad_job* jobs, int count, const double* sumsq, float max_norm, float* norm, void* stream) {
  const fog_status st = check_jobs(jobs, count, true);
  if (st != FOG_OK) return st;
  if (!sumsq) return FOG_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(sumsq) & 7) return FOG_ERR_ALIGN;
  if (!(max_norm >= 0.0f)) return FOG_ERR_UNSUPPORTED;
  const fog_status apart = check_overlaps(jobs, count);
  if (apart != FOG_OK) return apart;
  hipStream_t s = (hipStream_t)stream;
  bool told = false;
  for_batches(jobs, count, [&](const GradBatch& b) {
    clip_kernel<<<b.pieces < CLIP_GROUPS ? b.pieces : CLIP_GROUPS, kThreads, 0, s>>>(b, sumsq, max_norm, told ? nullptr : norm);
    told = true;
  });
  if (!told && norm) {     // no elements: only the norm is asked for
    GradBatch b;
    b.count = 0;
    b.pieces = 0;
    clip_kernel<<<1, kThreads, 0, s>>>(b, sumsq, max_norm, norm);
  }
  return fog_launch_status();
}
