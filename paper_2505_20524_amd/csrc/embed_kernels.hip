// The embedding in front of the first block: scaled rows of the table as the residual stream and as FP8 codes, and the table's gradient.
//
// Forward: x = bf16(factor E[t]), its codes and abs-max in the same pass.  Bound by memory: 2 bytes read, 2 written and 1 for the codes
// per element.
//
// Gradient: dE[v] = factor sum over the tokens t with id v of dx[t], in binary32 and in the order of the tokens.  The tokens are
// sorted by id first, so that every sum is a run of the sorted order and no two writers meet: no atomics on sums, the same result on
// every run.
//   1. rank_tokens: up to RANK_MOST tokens.  A token's place is the number of tokens before it in the order, counted by comparing it with
//      all of them; every workgroup places a few tokens, so that the whole chip counts.
//      sort_tiles and merge_ranks: more tokens.  A workgroup sorts 1024 tokens by (id, position) in LDS; then a token's place is its
//      place in its tile plus, for every other tile, the number of that tile's tokens before it (a binary search); stable, because earlier
//      tiles count their equal ids and later ones do not.
//      Further workgroups of these launches write zeros to the whole table's gradient, which is most of the work where the table has many
//      more rows than there are tokens; looking up the rows that need none costs more than it saves (see fill_zeros).
//   2. sum_runs: a wave adds `chunk` consecutive tokens of the order on 512 columns and writes each run that begins and ends in
//      the chunk; what a run has in a chunk that it does not begin and end in goes to the workspace.
//   3. join_runs: adds the pieces of the runs that cross chunks, in order.
#include "common.h"
#include "launch.h"

namespace {

constexpr int kThreads = 256;

__global__ void zero_u32e(uint32_t* p) { *p = 0u; }

FOG_DEVICE int64_t token_at(const void* tokens, int wide, int64_t i) {
  return wide ? reinterpret_cast<const int64_t*>(tokens)[i] : (int64_t)reinterpret_cast<const int32_t*>(tokens)[i];
}

// ---------------------------------------------------------------- forward
struct EmbedArgs {
  const void* tokens;
  int wide;
  int64_t vocab, cols, ld_table, ldx, ldq;
  const uint16_t* table;
  float factor;
  const float* scale;
  uint16_t* x;
  uint8_t* q;
  uint32_t* amax_out;
  uint32_t pieces, per_row;    // pieces of eight elements of all rows, of a row
};

// A thread takes the pieces first, first + step, ... four at a time: all four ids, then all four pieces, are asked for before the first
// is used.  RAGGED: 8 does not divide the columns, the last piece of a row goes element by element.  Returns the thread's largest magnitude in
// packed pairs.
template <int FMT, bool RAGGED>
FOG_DEVICE uint32_t embed_pieces(const EmbedArgs& a, uint32_t first, uint32_t step) {
  constexpr int AHEAD = 4;
  const float rho = a.q ? *a.scale : 0.0f;
  uint32_t m = 0u;
  for (uint64_t base = first; base < a.pieces; base += (uint64_t)AHEAD * step) {
    uint32_t row[AHEAD], col[AHEAD];
    int64_t id[AHEAD];
    uint4 v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const uint64_t p = base + (uint64_t)u * step;
      row[u] = (uint32_t)p / a.per_row;
      col[u] = 8u * ((uint32_t)p - row[u] * a.per_row);
      id[u] = p < a.pieces ? token_at(a.tokens, a.wide, row[u]) : -1;
      if (id[u] >= a.vocab) id[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      v[u] = make_uint4(0, 0, 0, 0);
      if (id[u] < 0) continue;
      const uint16_t* e = a.table + id[u] * a.ld_table + col[u];
      if (!RAGGED || col[u] + 8 <= a.cols) v[u] = ld_any16(e);
      else                                 v[u] = ld_upto8(e, (int)(a.cols - col[u]));
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (base + (uint64_t)u * step >= a.pieces) break;
      const float f = a.factor;
      uint4 o = v[u];
      if (id[u] >= 0)
        o = make_uint4(pack_bf16x2(bf16lo(o.x) * f, bf16hi(o.x) * f), pack_bf16x2(bf16lo(o.y) * f, bf16hi(o.y) * f),
                       pack_bf16x2(bf16lo(o.z) * f, bf16hi(o.z) * f), pack_bf16x2(bf16lo(o.w) * f, bf16hi(o.w) * f));
      const int n = !RAGGED || col[u] + 8 <= a.cols ? 8 : (int)(a.cols - col[u]);
      m = pkmax_abs_bf16(m, o.x); m = pkmax_abs_bf16(m, o.y); m = pkmax_abs_bf16(m, o.z); m = pkmax_abs_bf16(m, o.w);
      if (n < 8) st_upto8(a.x + row[u] * a.ldx + col[u], o, n);
      else       st_through16(a.x + row[u] * a.ldx + col[u], o);
      if (a.q) {
        const uint2 c = make_uint2(cvt4_fp8_nan<FMT>(bf16lo(o.x) * rho, bf16hi(o.x) * rho, bf16lo(o.y) * rho, bf16hi(o.y) * rho),
                                   cvt4_fp8_nan<FMT>(bf16lo(o.z) * rho, bf16hi(o.z) * rho, bf16lo(o.w) * rho, bf16hi(o.w) * rho));
        if (n < 8) st_upto8(a.q + row[u] * a.ldq + col[u], c, n);
        else       st_through8(a.q + row[u] * a.ldq + col[u], c);
      }
    }
  }
  return m;
}

// The workgroup's largest magnitude as the bits of a float, in thread 0.
constexpr int EMBED_THREADS = 1024;
FOG_DEVICE uint32_t group_amax(uint32_t m) {
  __shared__ uint32_t part[EMBED_THREADS / 64];
  m = wave_max_u32(max_of_pair(m));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < EMBED_THREADS / 64; ++w) m = m > part[w] ? m : part[w];
  }
  return m << 16;      // the float with that bf16 pattern
}

// With an abs-max one workgroup a compute unit, which ends with one atomic at most: an atomic of each wave of 1112 rows of 3568, all at the
// same time, took 30 us where the rows take 8.  Rows and codes are written through, for the cast or the product that reads them next.  8192 x 4096
// of 131072 with codes, other ids and results each time (at the rates of a large read and a large fill, 6.99 and 6.86 TB/s: 24): 30 to 34 us by the
// profiler; from a graph, with the launch that clears the abs-max, 36 with ids as frequent as words and 39 with ids drawn evenly, 35 there
// with stores past the caches; but rows without codes and the block cast both ways behind them 48, and 52 with such stores.
template <int FMT, bool RAGGED>
__global__ __launch_bounds__(EMBED_THREADS) void embed_kernel(EmbedArgs a) {
  const uint32_t m = embed_pieces<FMT, RAGGED>(a, blockIdx.x * EMBED_THREADS + threadIdx.x, gridDim.x * EMBED_THREADS);
  if (!a.amax_out) return;
  const uint32_t top = group_amax(m);
  if (threadIdx.x == 0 && top > __hip_atomic_load(a.amax_out, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(a.amax_out, top);
}

// Up to SMALL pieces (a decoding step's tokens) with an abs-max: one workgroup, so that the abs-max needs no word that a launch before has
// cleared.  24 rows of 2048 take it 7.6 us and the caller 8.2; the first form, with a launch that cleared the word, took
// the caller 12.3.  Eight pieces ahead instead of four: no difference in turn (8.6 and 8.7 us).
constexpr uint32_t SMALL = 8 * EMBED_THREADS;
template <int FMT, bool RAGGED>
__global__ __launch_bounds__(EMBED_THREADS) void embed_small_kernel(EmbedArgs a) {
  const uint32_t top = group_amax(embed_pieces<FMT, RAGGED>(a, threadIdx.x, EMBED_THREADS));
  if (threadIdx.x == 0) *a.amax_out = top;
}

// ---------------------------------------------------------------- gradient: order of the tokens
constexpr int SORT_TILE = 1024;
constexpr int POS_BITS = 10;
// ids, the id behind the last (for tokens outside the table) and one more (the padding's) fit beside a position in the tile
constexpr int64_t VOCAB_MAX = ((int64_t)1 << (32 - POS_BITS)) - 2;

// Ids outside the table become `vocab`, which sorts last and is skipped.
FOG_DEVICE uint32_t sort_key(const void* tokens, int wide, int64_t count, int64_t vocab, int64_t i, int local) {
  if (i >= count) return 0xFFFFFFFFu;
  const int64_t id = token_at(tokens, wide, i);
  return (uint32_t)((id >= 0 && id < vocab ? id : vocab) << POS_BITS) | (uint32_t)local;
}

// Zeros for the rows of dE, 4 KB a workgroup; contiguous rows count as one.
struct Fill {
  uint8_t* p;
  int64_t row_bytes, ld_bytes;
  int64_t first, units;       // units of 4 KB that this launch writes
  uint32_t per_row;           // units of a row
  int one_row;
};
constexpr int FILL_UNIT = 16 * kThreads;
// Small workgroups that each write 16 bytes a thread and end: 2.1 GB take 313 us this way, 356 with four stores a thread, 343 and 377
// with workgroups of 1024 threads and one or two.  As one launch with the sums, which looked up what rows to leave out, the
// zeros took 358 to 420, the whole call 433 to 469 us.
FOG_DEVICE void fill_zeros(const Fill& f, int64_t group, int64_t groups) {
  const int t = threadIdx.x;
  for (int64_t u = f.first + group; u < f.first + f.units; u += groups) {
    int64_t row = 0, at = u * FILL_UNIT;
    if (!f.one_row) {
      row = (int64_t)((uint32_t)u / f.per_row);
      at = (int64_t)((uint32_t)u - (uint32_t)row * f.per_row) * FILL_UNIT;
    }
    uint8_t* p = f.p + row * f.ld_bytes;
    at += 16 * t;
    if (at + 16 <= f.row_bytes) {
      st_any16(p + at, make_uint4(0, 0, 0, 0));
    } else {
      for (; at < f.row_bytes; at += 2) *reinterpret_cast<uint16_t*>(p + at) = 0;
    }
  }
}

// Places RANK_TOKENS tokens a workgroup.  All tokens are in LDS; a quad of them is compared with a token by one of the 16 lanes that share
// that token, and the lanes' counts are added at the end.  One launch, where sorting takes two, but work that grows with the square of the
// tokens: whole calls on 512 columns by ranking and by sorting, us: 1024 tokens 16.1 and 19.0, 2048 18.1 and 19.1, 3000 20.6 and 19.6.
constexpr int RANK_TOKENS = 16, RANK_MOST = 2048;
__global__ __launch_bounds__(kThreads) void rank_tokens_kernel(const void* tokens, int wide, int count, int64_t vocab, uint32_t* ids, uint32_t* positions,
                                                              int work, Fill fill) {
  if ((int)blockIdx.x >= work) return fill_zeros(fill, (int)blockIdx.x - work, (int)gridDim.x - work);
  __shared__ uint4 other[RANK_MOST / 4];
  __shared__ int places[RANK_TOKENS];
  constexpr int GROUPS = kThreads / RANK_TOKENS, PER = RANK_MOST / kThreads;
  const int t = threadIdx.x, first = blockIdx.x * RANK_TOKENS, mine = first + t % RANK_TOKENS, quads = (count + 3) / 4;
  uint32_t staged[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const int i = t + u * kThreads;
    staged[u] = 0xFFFFFFFFu;
    if (i < count) {
      const int64_t id = token_at(tokens, wide, i);
      staged[u] = (uint32_t)(id >= 0 && id < vocab ? id : vocab);
    }
  }
#pragma unroll
  for (int u = 0; u < PER; ++u) reinterpret_cast<uint32_t*>(other)[t + u * kThreads] = staged[u];
  if (t < RANK_TOKENS) places[t] = 0;
  __syncthreads();
  const uint32_t id = mine < RANK_MOST ? reinterpret_cast<const uint32_t*>(other)[mine] : 0xFFFFFFFFu;
  int n = 0;
#pragma unroll 4
  for (int q = t / RANK_TOKENS; q < quads; q += GROUPS) {
    const uint4 o = other[q];
    const int at = 4 * q;
    if ((unsigned)(at - first) < (unsigned)RANK_TOKENS) {   // among this workgroup's own tokens: by id, then by position
      n += o.x < id || (o.x == id && at < mine);
      n += o.y < id || (o.y == id && at + 1 < mine);
      n += o.z < id || (o.z == id && at + 2 < mine);
      n += o.w < id || (o.w == id && at + 3 < mine);
    } else {
      const uint32_t limit = id + (at < first ? 1u : 0u);    // tokens before these with the same id come first
      n += o.x < limit;
      n += o.y < limit;
      n += o.z < limit;
      n += o.w < limit;
    }
  }
  atomicAdd(&places[t % RANK_TOKENS], n);
  __syncthreads();
  if (t < RANK_TOKENS && mine < count) {
    ids[places[t]] = id;
    positions[places[t]] = (uint32_t)mine;
  }
}

// The value of lane l ^ MASK.
template <int MASK>
FOG_DEVICE uint32_t of_lane_xor(uint32_t v) {
  if (MASK == 1) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);     // quads 1, 0, 3, 2
  if (MASK == 2) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);     // quads 2, 3, 0, 1
  if (MASK == 4) return (uint32_t)__builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true), 0x1B, 0xF, 0xF, true);   // xor 7, xor 3
  if (MASK == 8) return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, true);    // rows of 16 turned by 8
  return (uint32_t)__shfl_xor((int)v, MASK, 64);
}

// One step of the bitonic sort on key number 4 t + r of the tile: keys STRIDE apart, runs of SIZE in alternating order.
template <int SIZE, int STRIDE>
FOG_DEVICE void sort_step(uint32_t* v, uint4* lds) {
  const int t = threadIdx.x;
  if (STRIDE < 4) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (r & STRIDE) continue;
      const bool up = ((4 * t + r) & SIZE) == 0;
      const uint32_t lo = min(v[r], v[r + STRIDE]), hi = max(v[r], v[r + STRIDE]);
      v[r] = up ? lo : hi;
      v[r + STRIDE] = up ? hi : lo;
    }
    return;
  }
  const bool smaller = ((4 * t & SIZE) == 0) == ((4 * t & STRIDE) == 0);
  uint32_t o[4];
  if (STRIDE < 256) {
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = of_lane_xor<STRIDE / 4>(v[r]);
  } else {                                          // keys of another wave
    __syncthreads();
    lds[t] = make_uint4(v[0], v[1], v[2], v[3]);
    __syncthreads();
    const uint4 x = lds[t ^ (STRIDE / 4)];
    o[0] = x.x; o[1] = x.y; o[2] = x.z; o[3] = x.w;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = smaller ? min(v[r], o[r]) : max(v[r], o[r]);
}
template <int SIZE, int STRIDE>
FOG_DEVICE void sort_from(uint32_t* v, uint4* lds) {
  sort_step<SIZE, STRIDE>(v, lds);
  if constexpr (STRIDE > 1) sort_from<SIZE, STRIDE / 2>(v, lds);
  else if constexpr (SIZE < SORT_TILE) sort_from<2 * SIZE, SIZE>(v, lds);
}

// keys: tiles * SORT_TILE words.  A thread keeps four neighbouring keys; of the 55 steps 19 stay within a thread and 33 within a wave (a
// step on all keys in LDS took the tile 14.5 us, this one 3).
__global__ __launch_bounds__(kThreads) void sort_tiles_kernel(const void* tokens, int wide, int64_t count, int64_t vocab, uint32_t* keys, int work, Fill fill) {
  if ((int)blockIdx.x >= work) return fill_zeros(fill, (int)blockIdx.x - work, (int)gridDim.x - work);
  static_assert(SORT_TILE == 4 * kThreads, "four keys a thread");
  __shared__ uint4 lds[kThreads];
  const int64_t base = (int64_t)blockIdx.x * SORT_TILE;
  uint32_t v[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = sort_key(tokens, wide, count, vocab, base + 4 * threadIdx.x + r, 4 * threadIdx.x + r);
  sort_from<2, 1>(v, lds);
  reinterpret_cast<uint4*>(keys + base)[threadIdx.x] = make_uint4(v[0], v[1], v[2], v[3]);
}

// Numbers of four sorted tiles' keys below `limit` (four searches at a time: each step of one waits for LDS).
FOG_DEVICE int keys_below(const uint32_t (*tiles)[SORT_TILE], const uint32_t* limit) {
  int at[4] = {0, 0, 0, 0};
#pragma unroll
  for (int step = SORT_TILE / 2; step > 0; step /= 2)
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (tiles[u][at[u] + step - 1] < limit[u]) at[u] += step;
  int n = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) n += at[u] + (tiles[u][at[u]] < limit[u] ? 1 : 0);
  return n;
}

// A workgroup for each quarter of a tile.
constexpr int MERGE_TILES = 4;     // tiles in LDS at a time (16 KB: the workgroups that write zeros beside these are to fill the compute units)
constexpr int MERGE_PARTS = SORT_TILE / kThreads;
__global__ __launch_bounds__(kThreads) void merge_ranks_kernel(const uint32_t* __restrict__ keys, int64_t count, int tiles, uint32_t* __restrict__ ids,
                                                              uint32_t* __restrict__ positions, int work, Fill fill) {
  if ((int)blockIdx.x >= work) return fill_zeros(fill, (int)blockIdx.x - work, (int)gridDim.x - work);
  __shared__ __attribute__((aligned(16))) uint32_t k[MERGE_TILES][SORT_TILE];
  const int mine = blockIdx.x / MERGE_PARTS, in_tile = threadIdx.x + kThreads * (blockIdx.x % MERGE_PARTS);
  const uint32_t key = keys[(int64_t)mine * SORT_TILE + in_tile], id = key >> POS_BITS;
  int64_t rank = in_tile;
  const uint4* all = reinterpret_cast<const uint4*>(keys);
  constexpr int PER = MERGE_TILES * SORT_TILE / 4 / kThreads;     // 16-byte pieces a thread brings in
  uint4 next[PER];
  const int64_t pieces = (int64_t)tiles * (SORT_TILE / 4);
  auto fetch = [&](int base) {
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int64_t i = (int64_t)base * (SORT_TILE / 4) + threadIdx.x + u * kThreads;
      next[u] = i < pieces ? all[i] : make_uint4(0, 0, 0, 0);
    }
  };
  fetch(0);
  for (int base = 0; base < tiles; base += MERGE_TILES) {
    const int n = min(MERGE_TILES, tiles - base);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < PER; ++u) reinterpret_cast<uint4*>(&k[0][0])[threadIdx.x + u * kThreads] = next[u];
    __syncthreads();
    fetch(base + MERGE_TILES);
    for (int b = 0; b < n; b += 4) {
      uint32_t limit[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int tile = base + b + u;
        // a key of an earlier tile with the same id comes first; one of a later tile does not (id + 1 of a token fits its bits; the
        // padding behind the last tile's tokens sorts behind all of them and takes no place).  No key of its own tile, or behind the
        // last, lies below 0.
        limit[u] = tile == mine || tile >= tiles ? 0u : (tile < mine ? id + 1u : id) << POS_BITS;
      }
      rank += keys_below(k + b, limit);
    }
  }
  if (key != 0xFFFFFFFFu) {
    ids[rank] = id;
    positions[rank] = (uint32_t)((int64_t)mine * SORT_TILE + (key & (SORT_TILE - 1)));
  }
}

__global__ __launch_bounds__(kThreads) void fill_kernel(Fill fill) { fill_zeros(fill, blockIdx.x, gridDim.x); }

// ---------------------------------------------------------------- gradient: sums
constexpr int SLAB = 512;    // columns of a wave

struct GradArgs {
  const uint32_t *ids, *positions;
  const uint16_t* dx;
  void* dE;
  float *head, *tail;       // [chunks][cols]: what a chunk has of the run that began before it / that goes on behind it
  int64_t count, vocab, cols, ld_dx, ld_dE;
  float factor;
  int accumulate;
  int chunk;                // tokens of a wave, a power of two up to 64
  int slabs;                // ceil(cols / SLAB)
  int64_t chunks;
  int64_t units;            // waves: chunks * slabs
};

// RAGGED: 8 does not divide the columns, the last lane of a row takes its elements one by one.
template <bool F32, bool RAGGED>
struct Row {
  float v[8];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
  }
  // eight elements of dx of which n are inside the row
  static __device__ __forceinline__ uint4 load(const uint16_t* p, int n) {
    if (RAGGED && n < 8) return ld_upto8(p, n);
    return n > 0 ? ld_any_nt16(p) : make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void add(uint4 x) {
    v[0] += bf16lo(x.x); v[1] += bf16hi(x.x); v[2] += bf16lo(x.y); v[3] += bf16hi(x.y);
    v[4] += bf16lo(x.z); v[5] += bf16hi(x.z); v[6] += bf16lo(x.w); v[7] += bf16hi(x.w);
  }
  // n floats of a piece in the workspace, zeros behind them
  static __device__ __forceinline__ void load_floats(float* x, const float* p, int n) {
    if (RAGGED && n < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = i < n ? p[i] : 0.0f;
    } else {
      uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
      if (n > 0) {
        lo = ld_any16(p);
        hi = ld_any16(p + 4);
      }
      x[0] = __uint_as_float(lo.x); x[1] = __uint_as_float(lo.y); x[2] = __uint_as_float(lo.z); x[3] = __uint_as_float(lo.w);
      x[4] = __uint_as_float(hi.x); x[5] = __uint_as_float(hi.y); x[6] = __uint_as_float(hi.z); x[7] = __uint_as_float(hi.w);
    }
  }
  __device__ __forceinline__ void add_floats(const float* p, int n) {
    float x[8];
    load_floats(x, p, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += x[i];
  }
  static __device__ __forceinline__ uint4 bits(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  __device__ __forceinline__ void put_floats(float* p, int n) const {
    if (RAGGED && n < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = v[i];
    } else if (n > 0) {
      st_any16(p, bits(v));
      st_any16(p + 4, bits(v + 4));
    }
  }
  // the finished sum times the factor (added to what is there) to the table's gradient
  __device__ __forceinline__ void finish(const GradArgs& a, int64_t id, int64_t col, int n) const {
    if (n <= 0) return;
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = v[i] * a.factor;
    if (F32) {
      float* p = reinterpret_cast<float*>(a.dE) + id * a.ld_dE + col;
      if (a.accumulate) {
        float x[8];
        load_floats(x, p, n);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] += x[i];
      }
      if (RAGGED && n < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n) p[i] = r[i];
      } else {
        st_any_nt16(p, bits(r));
        st_any_nt16(p + 4, bits(r + 4));
      }
    } else {
      uint16_t* p = reinterpret_cast<uint16_t*>(a.dE) + id * a.ld_dE + col;
      if (a.accumulate) {
        const uint4 x = RAGGED && n < 8 ? ld_upto8(p, n) : ld_any16(p);
        r[0] += bf16lo(x.x); r[1] += bf16hi(x.x); r[2] += bf16lo(x.y); r[3] += bf16hi(x.y);
        r[4] += bf16lo(x.z); r[5] += bf16hi(x.z); r[6] += bf16lo(x.w); r[7] += bf16hi(x.w);
      }
      const uint4 o = make_uint4(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]), pack_bf16x2(r[4], r[5]), pack_bf16x2(r[6], r[7]));
      if (RAGGED && n < 8) st_upto8(p, o, n);
      else                 st_any_nt16(p, o);
    }
  }
};

template <bool F32, bool RAGGED>
__global__ __launch_bounds__(kThreads) void sum_runs_kernel(GradArgs a) {
  const int l = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= a.units) return;
  const int64_t c = unit / a.slabs, p0 = c * a.chunk;
  const int64_t col = (unit - c * a.slabs) * SLAB + 8 * l;
  const int n = a.cols - col >= 8 ? 8 : a.cols > col ? (int)(a.cols - col) : 0;
  const int len = (int)(a.count - p0 < a.chunk ? a.count - p0 : a.chunk);
  // a lane keeps one token of the chunk
  const int mine = l < len ? l : len - 1;
  const uint32_t id_l = a.ids[p0 + mine], pos_l = a.positions[p0 + mine];
  const uint32_t before = p0 > 0 ? a.ids[p0 - 1] : 0xFFFFFFFFu;
  const uint32_t after = p0 + len < a.count ? a.ids[p0 + len] : 0xFFFFFFFFu;
  constexpr int AHEAD = 8;
  Row<F32, RAGGED> sum;
  sum.clear();
  uint32_t cur = (uint32_t)__builtin_amdgcn_readlane((int)id_l, 0);
  bool began = cur != before;       // the current run begins in this chunk
  for (int i0 = 0; i0 < len; i0 += AHEAD) {
    uint4 v[AHEAD];
    uint32_t id[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int i = i0 + u < len ? i0 + u : len - 1;
      id[u] = (uint32_t)__builtin_amdgcn_readlane((int)id_l, i);
      const uint32_t pos = (uint32_t)__builtin_amdgcn_readlane((int)pos_l, i);
      v[u] = make_uint4(0, 0, 0, 0);
      if (i0 + u < len && id[u] < (uint32_t)a.vocab) v[u] = Row<F32, RAGGED>::load(a.dx + (int64_t)pos * a.ld_dx + col, n);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (i0 + u >= len) break;
      if (id[u] != cur) {
        if (began) sum.finish(a, cur, col, n);
        else       sum.put_floats(a.head + c * a.cols + col, n);
        sum.clear();
        cur = id[u];
        began = true;
      }
      sum.add(v[u]);
    }
  }
  if (cur >= (uint32_t)a.vocab) return;     // ids outside the table come last
  if (!began)            sum.put_floats(a.head + c * a.cols + col, n);
  else if (cur == after) sum.put_floats(a.tail + c * a.cols + col, n);
  else                   sum.finish(a, cur, col, n);
}

// A workgroup for each chunk and slab; those whose chunk ends inside a run that it began add up the run's pieces: the eight waves an eighth
// of the chunks each, then the eight sums in order.
constexpr int JOIN_WAVES = 8;
template <bool F32, bool RAGGED>
__global__ __launch_bounds__(64 * JOIN_WAVES) void join_runs_kernel(GradArgs a) {
  const int64_t c = (int64_t)blockIdx.x / a.slabs;
  const int64_t next = (c + 1) * a.chunk;              // first token of the next chunk
  if (next >= a.count) return;
  const uint32_t id = a.ids[next];
  if (id >= (uint32_t)a.vocab || a.ids[next - 1] != id) return;
  if (c * a.chunk > 0 && a.ids[c * a.chunk] == id && a.ids[c * a.chunk - 1] == id) return;      // begun before this chunk
  // chunks c + 1 .. c + m begin with a token of the run and have a piece of it: 64 of them are looked at together
  int64_t m = 0;
  for (;;) {
    const int64_t at = (c + 1 + m + (threadIdx.x & 63)) * a.chunk;
    const uint64_t out = __ballot(at >= a.count || a.ids[at < a.count ? at : 0] != id);
    m += out ? __builtin_ctzll(out) : 64;
    if (out) break;
  }
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const int64_t col = ((int64_t)blockIdx.x - c * a.slabs) * SLAB + 8 * l;
  const int n = a.cols - col >= 8 ? 8 : a.cols > col ? (int)(a.cols - col) : 0;
  const int64_t per = (m + JOIN_WAVES - 1) / JOIN_WAVES, b = c + 1 + w * per, e = b + per < c + m + 1 ? b + per : c + m + 1;
  Row<F32, RAGGED> sum;
  sum.clear();
  if (w == 0) sum.add_floats(a.tail + c * a.cols + col, n);
  constexpr int AHEAD = 8;
  for (int64_t i = b; i < e; i += AHEAD) {
    float v[AHEAD][8];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) Row<F32, RAGGED>::load_floats(v[u], a.head + (i + u) * a.cols + col, i + u < e ? n : 0);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int k = 0; k < 8; ++k) sum.v[k] += v[u][k];
  }
  __shared__ float part[JOIN_WAVES - 1][8][64];
  if (w > 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) part[w - 1][i][l] = sum.v[i];
  }
  __syncthreads();
  if (w > 0) return;
#pragma unroll
  for (int k = 0; k < JOIN_WAVES - 1; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum.v[i] += part[k][i][l];
  sum.finish(a, id, col, n);
}

// Tokens of a wave: as many as still give every compute unit eight waves, 64 at most, 8 at least (a load of eight rows is in flight).
int chunk_of(int64_t count, int64_t cols) {
  const int64_t slabs = (cols + SLAB - 1) / SLAB;
  int chunk = 64;
  while (chunk > 8 && (count + chunk - 1) / chunk * slabs < 8 * (int64_t)fog_compute_units()) chunk /= 2;
  return chunk;
}

struct GradRoom {   // the workspace in bytes
  size_t keys, order, pieces, total;
};
GradRoom room_of(int64_t count, int64_t cols) {
  GradRoom r;
  const int64_t tiles = (count + SORT_TILE - 1) / SORT_TILE;
  const int chunk = chunk_of(count, cols);
  r.keys = count > RANK_MOST ? (size_t)tiles * SORT_TILE * 4 : 0;
  r.order = ((size_t)count * 4 + 15) / 16 * 16;
  r.pieces = ((size_t)((count + chunk - 1) / chunk) * (size_t)cols * 4 + 15) / 16 * 16;
  r.total = r.keys + 2 * r.order + 2 * r.pieces;
  return r;
}

constexpr int64_t GROUPS_MAX = 1 << 22;    // workgroups of a launch (up to 512 threads each): grids are counted in threads of 32 bits

// The sizes that a call takes.  The sums have to fit one launch: where they come near its limit a wave takes 64 tokens (see chunk_of).
bool grad_takes(int64_t count, int64_t vocab, int64_t cols) {
  return count <= 0x7FFFFFFF && vocab <= VOCAB_MAX && cols <= 0x7FFFFFFF && (count + 63) / 64 * ((cols + SLAB - 1) / SLAB) <= GROUPS_MAX;
}

constexpr int64_t PIECES_MAX = 1 << 30;    // pieces of a launch of the forward
constexpr int64_t COLS_MAX = ((int64_t)1 << 32) - 8;     // and columns of a row, which embed_pieces counts in 32 bits, the eight behind the last piece among them

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace

extern "C" fog_status fog_embed_quantize(const void* tokens, int token_bytes, int64_t count, const void* table_bf16, int64_t vocab, int64_t cols,
                                         int64_t ld_table, float factor, fog_fp8 fmt, const float* scale, void* x_bf16, int64_t ldx,
                                         uint8_t* q, int64_t ldq, float* amax_out, void* stream) {
  if (count < 0 || vocab < 0 || cols < 0) return FOG_ERR_SHAPE;
  if (token_bytes != 4 && token_bytes != 8) return FOG_ERR_UNSUPPORTED;
  if (fmt != FOG_E4M3 && fmt != FOG_E5M2) return FOG_ERR_UNSUPPORTED;
  if (!(factor - factor == 0.0f)) return FOG_ERR_UNSUPPORTED;
  const bool any = count > 0 && cols > 0;
  if (any && cols > COLS_MAX) return FOG_ERR_UNSUPPORTED;
  if (any) {
    if (!tokens || !x_bf16 || (vocab > 0 && !table_bf16) || (q && !scale)) return FOG_ERR_NULL;
    if (ld_table < cols || ldx < cols || (q && ldq < cols)) return FOG_ERR_SHAPE;
    if (!aligned(tokens, token_bytes) || !aligned(table_bf16, 2) || !aligned(x_bf16, 2)) return FOG_ERR_ALIGN;
  }
  hipStream_t s = (hipStream_t)stream;
  EmbedArgs a{tokens, token_bytes == 8, vocab, cols, ld_table, ldx, ldq, reinterpret_cast<const uint16_t*>(table_bf16), factor, scale,
              reinterpret_cast<uint16_t*>(x_bf16), q, reinterpret_cast<uint32_t*>(amax_out), 0, 0};
  const int64_t per_row = (cols + 7) / 8;
  const bool ragged = cols % 8 != 0;
  if (any && amax_out && per_row <= SMALL && count * per_row <= SMALL) {
    a.per_row = (uint32_t)per_row;
    a.pieces = (uint32_t)(count * per_row);
#define FOG_EM(F, R) embed_small_kernel<F, R><<<1, EMBED_THREADS, 0, s>>>(a)
    if (fmt == FOG_E4M3) { if (ragged) FOG_EM(FOG_E4M3, true); else FOG_EM(FOG_E4M3, false); }
    else                 { if (ragged) FOG_EM(FOG_E5M2, true); else FOG_EM(FOG_E5M2, false); }
#undef FOG_EM
    return fog_launch_status();
  }
  if (amax_out) zero_u32e<<<1, 1, 0, s>>>(reinterpret_cast<uint32_t*>(amax_out));
  if (!any) return amax_out ? fog_launch_status() : FOG_OK;
  // pieces are counted in 32 bits: as many rows a launch as that allows
  const int64_t rows = PIECES_MAX / per_row;
  for (int64_t r = 0; r < count; r += rows) {
    const int64_t n = count - r < rows ? count - r : rows;
    EmbedArgs b = a;
    b.tokens = reinterpret_cast<const uint8_t*>(tokens) + r * token_bytes;
    b.x = a.x + r * ldx;
    b.q = a.q ? a.q + r * ldq : nullptr;
    b.per_row = (uint32_t)per_row;
    b.pieces = (uint32_t)(n * per_row);
    int64_t groups = (n * per_row + EMBED_THREADS - 1) / EMBED_THREADS;
    const int64_t most = (amax_out ? 1 : 4) * (int64_t)fog_compute_units();
    if (groups > most) groups = most;
#define FOG_EM(F, R) embed_kernel<F, R><<<(int)groups, EMBED_THREADS, 0, s>>>(b)
    if (fmt == FOG_E4M3) { if (ragged) FOG_EM(FOG_E4M3, true); else FOG_EM(FOG_E4M3, false); }
    else                 { if (ragged) FOG_EM(FOG_E5M2, true); else FOG_EM(FOG_E5M2, false); }
#undef FOG_EM
  }
  return fog_launch_status();
}

extern "C" size_t fog_embed_grad_workspace(int64_t count, int64_t vocab, int64_t cols) {
  if (count <= 0 || vocab <= 0 || cols <= 0 || !grad_takes(count, vocab, cols)) return 0;
  return room_of(count, cols).total;
}

extern "C" fog_status fog_embed_grad(const void* tokens, int token_bytes, int64_t count, const void* dx_bf16, int64_t ld_dx, int64_t vocab,
                                     int64_t cols, float factor, fog_real type, void* dE, int64_t ld_dE, int accumulate, void* workspace,
                                     size_t workspace_bytes, void* stream) {
  if (count < 0 || vocab < 0 || cols < 0) return FOG_ERR_SHAPE;
  if (token_bytes != 4 && token_bytes != 8) return FOG_ERR_UNSUPPORTED;
  if (type != FOG_BF16 && type != FOG_F32) return FOG_ERR_UNSUPPORTED;
  if (!(factor - factor == 0.0f)) return FOG_ERR_UNSUPPORTED;
  if (count > 0x7FFFFFFF || vocab > VOCAB_MAX || cols > 0x7FFFFFFF) return FOG_ERR_UNSUPPORTED;
  if (vocab == 0 || cols == 0 || (count == 0 && accumulate)) return FOG_OK;
  const int size = type == FOG_F32 ? 4 : 2;
  const int64_t row_units = (cols * size + FILL_UNIT - 1) / FILL_UNIT;
  if (!grad_takes(count, vocab, cols) || (!accumulate && ld_dE != cols && vocab * row_units > 0xFFFFFFFFll)) return FOG_ERR_UNSUPPORTED;
  if (!dE || (count > 0 && (!tokens || !dx_bf16))) return FOG_ERR_NULL;
  if (ld_dE < cols || (count > 0 && ld_dx < cols)) return FOG_ERR_SHAPE;
  if (!aligned(dE, size) || (count > 0 && (!aligned(tokens, token_bytes) || !aligned(dx_bf16, 2)))) return FOG_ERR_ALIGN;
  const GradRoom room = count > 0 ? room_of(count, cols) : GradRoom{};
  if (count > 0) {
    if (!workspace || workspace_bytes < room.total) return FOG_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return FOG_ERR_ALIGN;
  }
  uint8_t* ws = reinterpret_cast<uint8_t*>(workspace);
  uint32_t *keys = reinterpret_cast<uint32_t*>(ws), *ids = reinterpret_cast<uint32_t*>(ws + room.keys);
  uint32_t* positions = reinterpret_cast<uint32_t*>(ws + room.keys + room.order);
  GradArgs a{};
  a.ids = ids; a.positions = positions;
  a.dx = reinterpret_cast<const uint16_t*>(dx_bf16);
  a.dE = dE;
  a.head = reinterpret_cast<float*>(ws + room.keys + 2 * room.order);
  a.tail = reinterpret_cast<float*>(ws + room.keys + 2 * room.order + room.pieces);
  a.count = count; a.vocab = vocab; a.cols = cols; a.ld_dx = ld_dx; a.ld_dE = ld_dE;
  a.factor = factor;
  a.accumulate = accumulate != 0;
  a.chunk = count > 0 ? chunk_of(count, cols) : 64;
  a.slabs = (int)((cols + SLAB - 1) / SLAB);
  a.chunks = (count + a.chunk - 1) / a.chunk;
  a.units = a.chunks * a.slabs;
  Fill fill{reinterpret_cast<uint8_t*>(dE), cols * size, ld_dE * size, 0, 0, (uint32_t)row_units, ld_dE == cols};
  int64_t units = accumulate ? 0 : vocab * row_units;
  if (fill.one_row) {
    fill.row_bytes = vocab * cols * size;
    units = accumulate ? 0 : (fill.row_bytes + FILL_UNIT - 1) / FILL_UNIT;
  }
  hipStream_t s = (hipStream_t)stream;
  const int wide = token_bytes == 8;
  // the launches that put the tokens in order share the zeros
  auto share = [&](int64_t first, int64_t n) {
    fill.first = first;
    fill.units = n;
    return (int)(n < GROUPS_MAX ? n : GROUPS_MAX);
  };
  if (count == 0) {
    const int groups = share(0, units);
    fill_kernel<<<groups, kThreads, 0, s>>>(fill);
    return fog_launch_status();
  }
  if (count <= RANK_MOST) {
    const int work = (int)((count + RANK_TOKENS - 1) / RANK_TOKENS), groups = work + share(0, units);
    rank_tokens_kernel<<<groups, kThreads, 0, s>>>(tokens, wide, (int)count, vocab, ids, positions, work, fill);
  } else {
    const int tiles = (int)((count + SORT_TILE - 1) / SORT_TILE);
    int groups = tiles + share(0, units / 2);
    sort_tiles_kernel<<<groups, kThreads, 0, s>>>(tokens, wide, count, vocab, keys, tiles, fill);
    groups = tiles * MERGE_PARTS + share(units / 2, units - units / 2);
    merge_ranks_kernel<<<groups, kThreads, 0, s>>>(keys, count, tiles, ids, positions, tiles * MERGE_PARTS, fill);
  }
  const int groups = (int)((a.units + kThreads / 64 - 1) / (kThreads / 64));
#define FOG_EG(F, R)                                                                         \
  do {                                                                                       \
    sum_runs_kernel<F, R><<<groups, kThreads, 0, s>>>(a);                                    \
    if (a.chunks > 1) join_runs_kernel<F, R><<<(int)a.units, 64 * JOIN_WAVES, 0, s>>>(a);    \
  } while (0)
  const bool ragged = cols % 8 != 0;
  if (type == FOG_F32) { if (ragged) FOG_EG(true, true); else FOG_EG(true, false); }
  else                 { if (ragged) FOG_EG(false, true); else FOG_EG(false, false); }
#undef FOG_EG
  return fog_launch_status();
}
