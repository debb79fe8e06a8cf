// Low-rank adapters of many requests at once beside a shared projection (include/finetune/nvfp4_finetune.h), forwards and
// backwards.
//
//   h_t = A_l x_t,  out_t = base_t + s_l B_l h_t,  l = which[t]
//   dh_t = s_l B_l^T dy_t,  dx_t = dx_base_t + A_l^T dh_t,  dA_l = sum_t dh_t x_t^T,  dB_l = s_l sum_t dy_t h_t^T
//
// At r / 2 multiplications per byte all of this is bound by the bytes of x, base, out, dy: every kernel streams one of them and
// keeps what has the rank for a side in registers.  Tokens are taken in tiles of one adapter each, in the order of their adapters
// (k_plan), so that a tile's rows share the adapter's matrices in the matrix unit, wherever they stand.
//
//   k_plan     tokens in the order of their adapters (stable), tiles of 32; backwards also A and B transposed
//   k_shrink   [T][width] times [rank][width] -> [T][rank]            h from x and A, dh / s from dy and B^T
//   k_expand   base + s [T][rank] times [width][rank]                 out from h and B, dx from dh / s and A^T
//   k_outer    s [T][rank] times [T][width] over an adapter's tokens  dA from dh / s and x, dB from h and dy
//   k_join     sums what several workgroups of k_outer have of one adapter, in a fixed order
#include <hip/hip_runtime.h>

#include "finetune/nvfp4_finetune.h"
#include "launch.hpp"

namespace nvfp4_46 {
namespace {

constexpr int kMostRank = 128, kMostAdapters = 2048;
constexpr int kTile = 32;                       // tokens of a planned tile
constexpr int kFewTile = 16;                    // ... and of a tile that a workgroup finds for itself
constexpr int kFewTokens = 256;                 // up to here there is no plan (find_tile)
constexpr int kPlanThreads = 1024;
constexpr int kOuterWidth = 512;                // columns of a workgroup of k_outer, 128 a wave
constexpr int kBlock = 64;                      // columns of a step of k_shrink, of a block of k_expand

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Tile {
  int32_t start, count, adapter, unused;
};

// What k_plan writes.  Tokens without an adapter come last, as tiles of adapter -1.
struct Plan {
  int32_t *count;                               // tiles
  int32_t *tile_begin;                          // [L + 2]: the first tile of every adapter, of those without, the end
  int32_t *order;                               // [T]
  Tile *tiles;
};

// Where tiles come from: a plan, or (few tokens) `which` itself.
struct Tokens {
  const int32_t *which;
  Plan plan;
  int32_t T, L;
  bool few;
};

__device__ inline int32_t adapter_of(const int32_t *which, int32_t t, int32_t L) {
  const int32_t l = which[t];
  return l >= 0 && l < L ? l : -1;
}

// ---- tiles ----------------------------------------------------------------------------------------------------------

struct TileTokens {
  int32_t token[kTile];
  uint64_t same[kFewTokens / 64];               // tokens of this workgroup's adapter, a bit each
};

// The tile of `index` in `shared`, as (count, adapter); count 0: there is none.  All threads of the workgroup call it.  With a plan
// the index is that of a tile (rows == 16: of half a tile).  Without, it is a token's: the token leads a tile if a multiple of 16 of
// the tokens before it have its adapter, and the next of them go with it.
template <int NT>
__device__ inline Tile find_tile(const Tokens &k, TileTokens &shared, int32_t index, int rows) {
  Tile t{0, 0, -1, 0};
  if (!k.few) {
    const int halves = kTile / rows;
    if (index / halves >= *k.plan.count) return t;
    t = k.plan.tiles[index / halves];
    const int32_t skip = index % halves * rows;
    t.start += skip;
    t.count = t.count - skip < rows ? t.count - skip : rows;
    if (t.count <= 0) return {0, 0, -1, 0};
    if ((int)threadIdx.x < t.count) shared.token[threadIdx.x] = k.plan.order[t.start + threadIdx.x];
    __syncthreads();
    return t;
  }
  t.adapter = adapter_of(k.which, index, k.L);
  for (int32_t i = threadIdx.x; i < kFewTokens; i += NT) {          // (whole waves: NT and kFewTokens are multiples of 64)
    const bool same = i < k.T && adapter_of(k.which, i, k.L) == t.adapter;
    const uint64_t mask = __ballot(same);
    if ((threadIdx.x & 63) == 0) shared.same[i / 64] = mask;
  }
  __syncthreads();
  const auto before = [&](int32_t i) {
    int32_t n = __popcll(shared.same[i / 64] & (((uint64_t)1 << (i & 63)) - 1));
    for (int w = 0; w < i / 64; ++w) n += __popcll(shared.same[w]);
    return n;
  };
  const int32_t mine = before(index);
  if (mine % kFewTile) return {0, 0, -1, 0};
  int32_t all = 0;
  for (int w = 0; w < kFewTokens / 64; ++w) all += __popcll(shared.same[w]);
  t.count = all - mine < kFewTile ? all - mine : kFewTile;
  for (int32_t i = threadIdx.x; i < k.T; i += NT)
    if (shared.same[i / 64] >> (i & 63) & 1) {
      const int32_t at = before(i) - mine;
      if (at >= 0 && at < kFewTile) shared.token[at] = i;
    }
  __syncthreads();
  return t;
}

// ---- pieces ---------------------------------------------------------------------------------------------------------

__device__ inline bf16x8 load8(const __bf16 *p) { return *reinterpret_cast<const bf16x8 *>(p); }
__device__ inline f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// v as a sum of BF16 terms: two leave 2^-16 of it, three 2^-24.  Of an infinity or NaN the first term is all there is.
__device__ inline __bf16 term(float v, int which) {
  __bf16 hi = (__bf16)v;
  if (__builtin_isinf((float)hi) && __builtin_isfinite(v))          // rounded up past the largest BF16
    hi = __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(v) >> 16));
  if (which == 0) return hi;
  const float rest = __builtin_isfinite((float)hi) ? v - (float)hi : 0.0f;
  const __bf16 mid = (__bf16)rest;
  return which == 1 ? mid : (__bf16)(rest - (float)mid);
}

// ---- k_shrink ---------------------------------------------------------------------------------------------------------

struct ShrinkArgs {
  Tokens tokens;
  const __bf16 *x, *w;         // [T] rows of `width`, and [L][rank][width]
  float *h;                    // [splits][T][rank]
  int64_t ld, width;
  int32_t rank, steps;         // steps of 64 columns of a split
  bool zero;                   // rows without an adapter get zeros
};

// D[token][rank]: rows of x against rows of w, both adjacent in the summed index.  A lane takes 16 columns of a step, of row
// lane % 16 of each side: 128 bytes of a row lie in one step.  The waves of a workgroup take every W-th step of its split.
template <int MT, int RT, int W>
__global__ void __launch_bounds__(W * 64) k_shrink(ShrinkArgs a) {
  __shared__ TileTokens shared;
  __shared__ float part[W][MT * RT * 256];
  const Tile t = find_tile<W * 64>(a.tokens, shared, blockIdx.x, MT * 16);
  if (t.count == 0) return;
  float *const h = a.h + (int64_t)blockIdx.y * a.tokens.T * a.rank;
  if (t.adapter < 0) {
    if (a.zero)
      for (int i = threadIdx.x; i < t.count * a.rank; i += W * 64) h[(int64_t)shared.token[i / a.rank] * a.rank + i % a.rank] = 0.0f;
    return;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, row = lane & 15, group = lane / 16;
  const __bf16 *x[MT], *w[RT];
  for (int i = 0; i < MT; ++i) {
    const int n = i * 16 + row < t.count ? i * 16 + row : t.count - 1;            // (rows past the tile's are not kept)
    x[i] = a.x + shared.token[n] * a.ld + group * 16;
  }
  for (int i = 0; i < RT; ++i) {
    const int n = i * 16 + row < a.rank ? i * 16 + row : a.rank - 1;
    w[i] = a.w + ((int64_t)t.adapter * a.rank + n) * a.width + group * 16;
  }
  f32x4 acc[MT][RT] = {};
  const int64_t first = (int64_t)blockIdx.y * a.steps, all = (a.width + kBlock - 1) / kBlock;
  const int64_t last = first + a.steps < all ? first + a.steps : all;
  for (int64_t s = first + wave; s < last; s += W) {
    const int64_t k = s * kBlock;
    bf16x8 xs[MT][2], ws[RT][2];
    if (k + kBlock <= a.width) {
      for (int i = 0; i < MT; ++i)
        for (int c = 0; c < 2; ++c) xs[i][c] = load8(x[i] + k + c * 8);
      for (int i = 0; i < RT; ++i)
        for (int c = 0; c < 2; ++c) ws[i][c] = load8(w[i] + k + c * 8);
    } else {
      for (int c = 0; c < 2; ++c) {
        const bool in = k + group * 16 + c * 8 < a.width;
        for (int i = 0; i < MT; ++i) xs[i][c] = in ? load8(x[i] + k + c * 8) : bf16x8{};
        for (int i = 0; i < RT; ++i) ws[i][c] = in ? load8(w[i] + k + c * 8) : bf16x8{};
      }
    }
    for (int c = 0; c < 2; ++c)
      for (int i = 0; i < MT; ++i)
        for (int j = 0; j < RT; ++j) acc[i][j] = multiply(xs[i][c], ws[j][c], acc[i][j]);
  }
  for (int i = 0; i < MT; ++i)
    for (int j = 0; j < RT; ++j)
      for (int v = 0; v < 4; ++v) part[wave][(i * RT + j) * 256 + (group * 4 + v) * 16 + row] = acc[i][j][v];
  __syncthreads();
  for (int e = threadIdx.x; e < MT * RT * 256; e += W * 64) {
    const int n = e / (RT * 256) * 16 + e % 256 / 16, rank = e / 256 % RT * 16 + e % 16;
    float s = 0.0f;
    for (int i = 0; i < W; ++i) s += part[i][e];
    if (n < t.count && rank < a.rank) h[(int64_t)shared.token[n] * a.rank + rank] = s;
  }
}

// ---- k_expand ---------------------------------------------------------------------------------------------------------

struct ExpandArgs {
  Tokens tokens;
  const float *h;              // [parts][T][rank]
  float *h_out;                // their sum, where it is wanted and k_shrink has not written it; or nullptr
  const __bf16 *w;             // [L][width] rows of `rank`, `pitch` apart
  const float *scales;
  const void *base;
  void *out;
  int64_t ld_base, ld_out, width;
  int32_t rank, pitch, parts;
};

__device__ inline float h_of(const float *h, int32_t parts, int64_t stride) {
  float s = h[0];
  for (int p = 1; p < parts; ++p) s += h[p * stride];
  return s;
}

// Eight ranks of a row of w; where rows are not whole pieces of 16 bytes, one by one.
__device__ inline bf16x8 load_ranks(const __bf16 *row, int first, int rank, int pitch) {
  if (pitch % 8 == 0) return load8(row + first);
  bf16x8 v{};
  for (int i = 0; i < 8; ++i)
    if (first + i < rank) v[i] = row[first + i];
  return v;
}

// Eight columns of a row, as fp32.
template <typename T>
__device__ inline void load_columns(const T *p, float *v) {
  if constexpr (sizeof(T) == 4) {
    for (int i = 0; i < 2; ++i) {
      const f32x4 q = reinterpret_cast<const f32x4 *>(p)[i];
      for (int k = 0; k < 4; ++k) v[i * 4 + k] = q[k];
    }
  } else {
    const bf16x8 q = load8(p);
    for (int k = 0; k < 8; ++k) v[k] = (float)q[k];
  }
}
template <typename T>
__device__ inline void store_columns(T *p, const float *v) {
  if constexpr (sizeof(T) == 4) {
    for (int i = 0; i < 2; ++i) reinterpret_cast<f32x4 *>(p)[i] = f32x4{v[i * 4], v[i * 4 + 1], v[i * 4 + 2], v[i * 4 + 3]};
  } else {
    bf16x8 q;
    for (int k = 0; k < 8; ++k) q[k] = (__bf16)v[k];
    *reinterpret_cast<bf16x8 *>(p) = q;
  }
}

// D[column][token]: rows of w against h.  The summed index runs over pieces of eight ranks of every term of h (term), four pieces to a
// product: piece q is term q / pieces of ranks q % pieces, against the same ranks of w.  Row 4 a + b of product m of a block is column
// 16 a + 4 m + b, so that a lane ends up with 16 adjacent columns of its token.
template <typename T, int MT, int TERMS, int NM>
__global__ void __launch_bounds__(256) k_expand(ExpandArgs a) {
  __shared__ TileTokens shared;
  const Tile t = find_tile<256>(a.tokens, shared, blockIdx.x, MT * 16);
  if (t.count == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, row = lane & 15, group = lane / 16;
  const T *const base = static_cast<const T *>(a.base);
  T *const out = static_cast<T *>(a.out);
  const int64_t stride = (int64_t)a.tokens.T * a.rank, blocks = (a.width + kBlock - 1) / kBlock;
  if (a.h_out && blockIdx.y == 0)
    for (int i = threadIdx.x; i < t.count * a.rank; i += 256) {
      const int64_t at = (int64_t)shared.token[i / a.rank] * a.rank + i % a.rank;
      a.h_out[at] = t.adapter < 0 ? 0.0f : h_of(a.h + at, a.parts, stride);
    }
  if (t.adapter < 0) {
    if (base == out) return;
    for (int n = wave; n < t.count; n += 4)
      for (int64_t c = ((int64_t)blockIdx.y * 64 + lane) * 8; c < a.width; c += (int64_t)gridDim.y * 512) {
        float v[8] = {};
        if (base) load_columns(base + shared.token[n] * a.ld_base + c, v);
        store_columns(out + shared.token[n] * a.ld_out + c, v);
      }
    return;
  }
  const int pieces = (a.rank + 7) / 8;
  const float scale = a.scales[t.adapter];
  bf16x8 h[MT][NM];
  int ranks[NM];                                 // the first rank of a lane's piece, -1: none
#pragma unroll
  for (int m = 0; m < NM; ++m) {
    const int q = m * 4 + group, which = q / pieces, first = q % pieces * 8;
    ranks[m] = which < TERMS ? first : -1;
    for (int i = 0; i < MT; ++i) {
      const int n = i * 16 + row < t.count ? i * 16 + row : t.count - 1;
      const float *const from = a.h + (int64_t)shared.token[n] * a.rank + first;
      for (int k = 0; k < 8; ++k)
        h[i][m][k] = which < TERMS && first + k < a.rank ? term(scale * h_of(from + k, a.parts, stride), which) : (__bf16)0.0f;
    }
  }
  const __bf16 *const w = a.w + (int64_t)t.adapter * a.width * a.pitch;
  for (int64_t b = (int64_t)blockIdx.y * 4 + wave; b < blocks; b += (int64_t)gridDim.y * 4) {
    const int64_t c0 = b * kBlock;
    f32x4 acc[MT][4] = {};
#pragma unroll
    for (int m = 0; m < NM; ++m)
      for (int p = 0; p < 4; ++p) {
        const int64_t c = c0 + row / 4 * 16 + p * 4 + row % 4;
        const bf16x8 ws = ranks[m] >= 0 && c < a.width ? load_ranks(w + c * a.pitch, ranks[m], a.rank, a.pitch) : bf16x8{};
        for (int i = 0; i < MT; ++i) acc[i][p] = multiply(ws, h[i][m], acc[i][p]);
      }
    for (int i = 0; i < MT; ++i) {
      if (i * 16 + row >= t.count) continue;
      const int64_t n = shared.token[i * 16 + row];
      for (int half = 0; half < 2; ++half) {
        const int64_t c = c0 + group * 16 + half * 8;
        if (c >= a.width) continue;
        float v[8] = {};
        if (base) load_columns(base + n * a.ld_base + c, v);
        for (int k = 0; k < 8; ++k) v[k] += acc[i][half * 2 + k / 4][k % 4];
        store_columns(out + n * a.ld_out + c, v);
      }
    }
  }
}

// ---- k_plan -----------------------------------------------------------------------------------------------------------

struct PlanArgs {
  const int32_t *which;
  Plan plan;
  int32_t T, L;
  // backwards: A [L][rank][K] -> [L][K][pitch] and B [L][N][rank] -> [L][rank][N], a workgroup for 64 columns (rows) of one
  const __bf16 *a, *b;
  __bf16 *at, *bt;
  int64_t K, N, units;
  int32_t rank, pitch;
};

__device__ inline void plan_tokens(const PlanArgs &p) {
  extern __shared__ int32_t counts[];            // [16][L + 1]: of each wave's tokens; then where its next token of an adapter goes
  __shared__ int32_t waves[2][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int32_t groups = p.L + 1;
  for (int32_t i = threadIdx.x; i < 16 * groups; i += kPlanThreads) counts[i] = 0;
  __syncthreads();
  int32_t *const mine = counts + wave * groups;
  const int32_t slice = (p.T + 1023) / 1024 * 64, begin = wave * slice;
  const int32_t end = begin + slice < p.T ? begin + slice : p.T;
  // the lanes with this lane's group
  const auto alike = [&](int32_t l) {
    uint64_t m = ~(uint64_t)0;
    for (int32_t bit = 1; bit <= groups; bit <<= 1) {
      const uint64_t set = __ballot((l & bit) != 0);
      m &= l & bit ? set : ~set;
    }
    return m;
  };
  for (int pass = 0; pass < 2; ++pass) {
    for (int32_t t0 = begin; t0 < end; t0 += 64) {
      const int32_t t = t0 + lane;
      int32_t l = t < end ? adapter_of(p.which, t, p.L) : groups;       // (past the end: a group of its own, not counted)
      if (l < 0) l = p.L;
      const uint64_t m = alike(l);
      const int32_t before = __popcll(m & (((uint64_t)1 << lane) - 1)), at = t < end ? mine[l] : 0;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");          // (all lanes have read before one writes, and the other way)
      if (pass == 1 && t < end) p.plan.order[at + before] = t;
      if (before == 0 && t < end) mine[l] = at + __popcll(m);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    if (pass == 1) break;
    __syncthreads();
    // tokens and tiles of every group, summed up over the groups before it: each thread its adjacent groups
    const int32_t per = (groups + kPlanThreads - 1) / kPlanThreads, g0 = threadIdx.x * per;
    int32_t n[2] = {0, 0};
    for (int32_t g = g0; g < g0 + per && g < groups; ++g) {
      int32_t c = 0;
      for (int w = 0; w < 16; ++w) c += counts[w * groups + g];
      n[0] += c;
      n[1] += (c + kTile - 1) / kTile;
    }
    int32_t upto[2] = {n[0], n[1]};
    for (int d = 1; d < 64; d <<= 1)
      for (int k = 0; k < 2; ++k) {
        const int32_t other = __shfl_up(upto[k], d);
        if (lane >= d) upto[k] += other;
      }
    if (lane == 63)
      for (int k = 0; k < 2; ++k) waves[k][wave] = upto[k];
    __syncthreads();
    int32_t at[2];
    for (int k = 0; k < 2; ++k) {
      at[k] = upto[k] - n[k];
      for (int w = 0; w < wave; ++w) at[k] += waves[k][w];
    }
    for (int32_t g = g0; g < g0 + per && g < groups; ++g) {
      int32_t c = 0;
      for (int w = 0; w < 16; ++w) {
        const int32_t of = counts[w * groups + g];
        counts[w * groups + g] = at[0] + c;
        c += of;
      }
      p.plan.tile_begin[g] = at[1];
      for (int32_t i = 0; i * kTile < c; ++i)
        p.plan.tiles[at[1] + i] = {at[0] + i * kTile, c - i * kTile < kTile ? c - i * kTile : kTile, g < p.L ? g : -1, 0};
      at[0] += c;
      at[1] += (c + kTile - 1) / kTile;
      if (g == groups - 1) {
        p.plan.tile_begin[groups] = at[1];
        *p.plan.count = at[1];
      }
    }
    __syncthreads();
  }
}

__device__ inline void transpose(const PlanArgs &p, int64_t unit) {
  extern __shared__ int32_t space[];
  __bf16 *const tile = reinterpret_cast<__bf16 *>(space);              // [64][rank + 2]
  const int64_t of_a = (p.K + 63) / 64, of_b = (p.N + 63) / 64, l = unit / (of_a + of_b);
  int64_t c = unit % (of_a + of_b);
  const int lines = p.rank + 2;
  if (c < of_a) {
    c *= 64;
    const __bf16 *const from = p.a + l * p.rank * p.K;
    for (int i = threadIdx.x; i < p.rank * 64; i += kPlanThreads)
      if (c + i % 64 < p.K) tile[i % 64 * lines + i / 64] = from[i / 64 * p.K + c + i % 64];
    __syncthreads();
    __bf16 *const to = p.at + (l * p.K + c) * p.pitch;
    for (int i = threadIdx.x; i < 64 * p.pitch; i += kPlanThreads)
      if (c + i / p.pitch < p.K) to[i] = i % p.pitch < p.rank ? tile[i / p.pitch * lines + i % p.pitch] : (__bf16)0.0f;
  } else {
    c = (c - of_a) * 64;
    const __bf16 *const from = p.b + (l * p.N + c) * p.rank;
    for (int i = threadIdx.x; i < 64 * p.rank; i += kPlanThreads)
      if (c + i / p.rank < p.N) tile[i / p.rank * lines + i % p.rank] = from[i];
    __syncthreads();
    __bf16 *const to = p.bt + l * p.rank * p.N + c;
    for (int i = threadIdx.x; i < p.rank * 64; i += kPlanThreads)
      if (c + i % 64 < p.N) to[i / 64 * p.N + i % 64] = tile[i % 64 * lines + i / 64];
  }
}

__global__ void __launch_bounds__(kPlanThreads) k_plan(PlanArgs p) {
  if (blockIdx.x == 0)
    plan_tokens(p);
  else
    for (int64_t unit = (int64_t)blockIdx.x - 1; unit < p.units; unit += (int64_t)gridDim.x - 1) {
      transpose(p, unit);
      __syncthreads();
    }
}

// ---- k_outer ----------------------------------------------------------------------------------------------------------

struct OuterHalf {
  const __bf16 *x;             // [T] rows of `width`
  const float *h;              // [parts][T][rank]
  float *out;                  // [L][rank][width], or with `by_rank` [L][width][rank]
  float *parted;               // [2 ranges] of the same
  int64_t ld, width;
  int32_t parts, chunks;
  bool by_rank;
};
struct OuterArgs {
  Plan plan;
  const float *scales;
  int32_t T, L, rank, tiles;   // tiles of a range
  OuterHalf half[2];
};

// Which of an adapter's tiles a range has decides where its sum goes: all of them, to the output; else to a place that the range
// has for the adapter that began before it (0) or for the one that begins in it and goes on (1).
__device__ inline int64_t place(const Plan &p, int32_t adapter, int32_t range, int32_t tiles) {
  const bool before = p.tile_begin[adapter] < range * tiles, after = p.tile_begin[adapter + 1] > (range + 1) * tiles;
  return before ? 2 * range : after ? 2 * range + 1 : -1;
}

// D[column][rank], summed over the tokens of a tile.  Of 32 tokens and 128 columns lane (row, group) loads columns 8 row .. 8 row + 7 of
// tokens 8 group .. 8 group + 7, which transposes within the lane: product j has columns 8 row + j.
template <int RT>
__global__ void __launch_bounds__(256) k_outer(OuterArgs a) {
  const bool second = (int32_t)blockIdx.x >= a.half[0].chunks;
  const OuterHalf f = second ? a.half[1] : a.half[0];
  const int32_t chunk = (int32_t)blockIdx.x - (second ? a.half[0].chunks : 0), range = blockIdx.y, rank0 = blockIdx.z * RT * 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, row = lane & 15, group = lane / 16;
  const int64_t c0 = (int64_t)chunk * kOuterWidth + wave * 128, c = c0 + row * 8;
  if (c0 >= f.width) return;
  const bool in = c < f.width;
  const int64_t stride = (int64_t)a.T * a.rank, size = f.width * a.rank;
  const int32_t count = *a.plan.count, first = range * a.tiles, last = first + a.tiles < count ? first + a.tiles : count;
  f32x4 acc[RT][8] = {};
  int32_t adapter = -1;
  const auto flush = [&] {
    if (adapter < 0) return;
    const int64_t at = place(a.plan, adapter, range, a.tiles);
    float *const to = at < 0 ? f.out + adapter * size : f.parted + at * size;
    for (int r = 0; r < RT; ++r) {
      const int rank = rank0 + r * 16 + row;
      for (int v = 0; v < 4; ++v) {
        const int64_t col = c0 + (group * 4 + v) * 8;
        if (rank < a.rank && col < f.width) {
          if (f.by_rank) {
            for (int j = 0; j < 8; ++j) to[(col + j) * a.rank + rank] = acc[r][j][v];
          } else {
            for (int j = 0; j < 8; j += 4)
              *reinterpret_cast<f32x4 *>(to + rank * f.width + col + j) = f32x4{acc[r][j][v], acc[r][j + 1][v], acc[r][j + 2][v], acc[r][j + 3][v]};
          }
        }
      }
    }
    for (int r = 0; r < RT; ++r)
      for (int j = 0; j < 8; ++j) acc[r][j] = f32x4{};
  };
  for (int32_t i = first; i < last; ++i) {
    const Tile t = a.plan.tiles[i];
    if (t.adapter < 0) break;                    // (they come last)
    if (t.adapter != adapter) flush();
    adapter = t.adapter;
    const float scale = a.scales[adapter];
    int64_t token[8];
    u32x4 x[8];
    for (int q = 0; q < 8; ++q) {
      const int n = group * 8 + q;
      token[q] = a.plan.order[t.start + (n < t.count ? n : 0)];
      x[q] = in && n < t.count ? *reinterpret_cast<const u32x4 *>(f.x + token[q] * f.ld + c) : u32x4{};
    }
    bf16x8 xt[8];
    for (int j = 0; j < 8; ++j) {
      u32x4 p;
      for (int q = 0; q < 4; ++q) p[q] = __builtin_amdgcn_perm(x[2 * q + 1][j / 2], x[2 * q][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
      xt[j] = __builtin_bit_cast(bf16x8, p);
    }
    for (int r = 0; r < RT; ++r) {
      const int rank = rank0 + r * 16 + row;
      float v[8];
      for (int q = 0; q < 8; ++q)
        v[q] = rank < a.rank && group * 8 + q < t.count ? scale * h_of(f.h + token[q] * a.rank + rank, f.parts, stride) : 0.0f;
      for (int which = 0; which < 3; ++which) {
        bf16x8 hs;
        for (int q = 0; q < 8; ++q) hs[q] = term(v[q], which);
        for (int j = 0; j < 8; ++j) acc[r][j] = multiply(xt[j], hs, acc[r][j]);
      }
    }
  }
  flush();
}

// ---- k_join -----------------------------------------------------------------------------------------------------------

__global__ void __launch_bounds__(256) k_join(OuterArgs a) {
  const int32_t l = blockIdx.y, t0 = a.plan.tile_begin[l], t1 = a.plan.tile_begin[l + 1];
  const int32_t s0 = t0 / a.tiles, s1 = t1 > t0 ? (t1 - 1) / a.tiles : s0;
  if (t1 > t0 && s0 == s1) return;               // k_outer has written it
  for (int k = 0; k < 2; ++k) {
    const OuterHalf &f = a.half[k];
    const int64_t size = f.width * a.rank;       // (a multiple of 8)
    for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e < size; e += (int64_t)gridDim.x * 1024) {
      f32x4 s{};
      if (t1 > t0) {
        s = *reinterpret_cast<const f32x4 *>(f.parted + (2 * s0 + 1) * size + e);
        for (int64_t r = s0 + 1; r <= s1; ++r) s += *reinterpret_cast<const f32x4 *>(f.parted + 2 * r * size + e);
      }
      *reinterpret_cast<f32x4 *>(f.out + l * size + e) = s;
    }
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------

constexpr int64_t kMostTokens = (1 << 24) - 1, kMostWidth = 1 << 22;

bool sizes_fit(const nvfp4_adapters_params &p) {
  return p.tokens >= 0 && p.tokens <= kMostTokens && p.inp > 0 && p.inp <= kMostWidth && p.out > 0 && p.out <= kMostWidth &&
         p.inp % 8 == 0 && p.out % 8 == 0 && p.adapters > 0 && p.adapters <= kMostAdapters && p.rank > 0 && p.rank <= kMostRank;
}
bool stride_fits(int64_t ld, int64_t width, int64_t rows) {
  return ld >= width && ld <= (int64_t)1 << 40 && rows * ld <= (int64_t)1 << 40;
}
bool at(const void *ptr, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }
int64_t divide_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How a call's work is dealt out, and what it needs of the workspace: all of it follows from the sizes.
struct Layout {
  bool few;
  int64_t tiles;               // at most so many planned tiles
  int64_t splits_in, splits_out;     // of the sum over inp (h), over out (dh)
  int64_t ranges, range_tiles; // of k_outer
  int64_t count, tile_begin, order, table, h, at, bt, parted_a, parted_b, bytes;   // byte offsets

  // Splits of a sum so that there are workgroups for the compute units, each with two steps a wave at least
  static int64_t splits(int64_t tokens, bool few, int64_t width) {
    const int64_t steps = divide_up(width, kBlock), groups = few ? divide_up(tokens, 4) : divide_up(tokens, kTile);
    const int64_t want = divide_up(512, groups > 0 ? groups : 1), most = divide_up(steps, 16);
    const int64_t n = want < most ? want : most;
    return n < 1 ? 1 : n > 16 ? 16 : n;
  }
  Layout(const nvfp4_adapters_params &p, bool backward) {
    few = !backward && p.tokens <= kFewTokens;
    tiles = p.tokens / kTile + (p.adapters + 1 < p.tokens ? p.adapters + 1 : p.tokens);
    splits_in = splits(p.tokens, few, p.inp);
    splits_out = splits(p.tokens, few, p.out);
    const int64_t chunks = divide_up(p.inp, kOuterWidth) + divide_up(p.out, kOuterWidth);
    ranges = divide_up(512, chunks);
    range_tiles = divide_up(tiles, ranges);
    if (range_tiles < 1) range_tiles = 1;
    ranges = divide_up(tiles, range_tiles);
    int64_t end = 0;
    const auto take = [&](int64_t n) {
      const int64_t begin = end;
      end += divide_up(n, 256) * 256;
      return begin;
    };
    count = take(4);
    if (!few) {
      tile_begin = take((p.adapters + 2) * 4);
      order = take(p.tokens * 4);
      table = take(tiles * (int64_t)sizeof(Tile));
    }
    h = take((backward ? splits_out : splits_in) * p.tokens * p.rank * 4);
    if (backward) {
      at = take(p.adapters * p.inp * pitch(p) * 2);
      bt = take(p.adapters * p.out * p.rank * 2);
      parted_a = take(2 * ranges * p.rank * p.inp * 4);
      parted_b = take(2 * ranges * p.rank * p.out * 4);
    }
    bytes = end;
  }
  static int64_t pitch(const nvfp4_adapters_params &p) { return divide_up(p.rank, 8) * 8; }
  Plan plan(char *w) const {
    return {reinterpret_cast<int32_t *>(w + count), reinterpret_cast<int32_t *>(w + tile_begin), reinterpret_cast<int32_t *>(w + order),
            reinterpret_cast<Tile *>(w + table)};
  }
};

int run_plan(const nvfp4_adapters_params &p, const Layout &d, char *w, const int32_t *which, const void *a, const void *b,
             hipStream_t s) {
  PlanArgs g{which, d.plan(w), (int32_t)p.tokens, (int32_t)p.adapters, static_cast<const __bf16 *>(a), static_cast<const __bf16 *>(b),
             reinterpret_cast<__bf16 *>(w + d.at), reinterpret_cast<__bf16 *>(w + d.bt), p.inp, p.out,
             a ? p.adapters * (divide_up(p.inp, 64) + divide_up(p.out, 64)) : 0, (int32_t)p.rank, (int32_t)Layout::pitch(p)};
  const size_t counts = 16 * (size_t)(p.adapters + 1) * 4, tile = a ? 64 * (size_t)(p.rank + 2) * 2 : 0;
  constexpr size_t kMostLds = 16 * (kMostAdapters + 1) * 4;
  if (counts > 48 * 1024 &&
      hipFuncSetAttribute(reinterpret_cast<const void *>(k_plan), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMostLds) != hipSuccess)
    return NVFP4_ERR_HIP;
  return launch(k_plan, dim3((uint32_t)(1 + (g.units < 65536 ? g.units : 65536))), dim3(kPlanThreads), counts > tile ? counts : tile, s, g);
}

template <int MT, int RT, int W>
int run_shrink_of(const ShrinkArgs &g, int64_t tiles, int64_t splits, hipStream_t s) {
  return launch(k_shrink<MT, RT, W>, dim3((uint32_t)tiles, (uint32_t)splits), dim3(W * 64), 0, s, g);
}
int run_shrink(ShrinkArgs g, const Layout &d, int64_t splits, hipStream_t s) {
  g.steps = (int32_t)divide_up(divide_up(g.width, kBlock), splits);
  const int64_t tiles = d.few ? g.tokens.T : d.tiles;
  if (d.few) {
    if (g.rank <= 16) return run_shrink_of<1, 1, 8>(g, tiles, splits, s);
    if (g.rank <= 32) return run_shrink_of<1, 2, 8>(g, tiles, splits, s);
    if (g.rank <= 64) return run_shrink_of<1, 4, 8>(g, tiles, splits, s);
    return run_shrink_of<1, 8, 4>(g, tiles, splits, s);
  }
  if (g.rank <= 16) return run_shrink_of<2, 1, 8>(g, tiles, splits, s);
  if (g.rank <= 32) return run_shrink_of<2, 2, 8>(g, tiles, splits, s);
  if (g.rank <= 64) return run_shrink_of<2, 4, 4>(g, tiles, splits, s);
  return run_shrink_of<2, 8, 4>(g, tiles, splits, s);
}

template <typename T, int TERMS, int NM>
int run_expand_of(const ExpandArgs &g, const Layout &d, hipStream_t s) {
  const int64_t blocks = divide_up(g.width, kBlock * 4), tiles = d.few ? g.tokens.T : d.tiles;
  const int64_t want = divide_up(2048, tiles);
  const dim3 grid((uint32_t)tiles, (uint32_t)(want < blocks ? want : blocks));
  return d.few ? launch(k_expand<T, 1, TERMS, NM>, grid, dim3(256), 0, s, g) : launch(k_expand<T, 2, TERMS, NM>, grid, dim3(256), 0, s, g);
}
int run_expand(const ExpandArgs &g, const Layout &d, bool f32, hipStream_t s) {
  const int64_t products = divide_up((f32 ? 3 : 2) * divide_up(g.rank, 8), 4);
  if (f32) {
    if (products <= 2) return run_expand_of<float, 3, 2>(g, d, s);
    if (products <= 3) return run_expand_of<float, 3, 3>(g, d, s);
    if (products <= 6) return run_expand_of<float, 3, 6>(g, d, s);
    return run_expand_of<float, 3, 12>(g, d, s);
  }
  if (products <= 1) return run_expand_of<__bf16, 2, 1>(g, d, s);
  if (products <= 2) return run_expand_of<__bf16, 2, 2>(g, d, s);
  if (products <= 4) return run_expand_of<__bf16, 2, 4>(g, d, s);
  return run_expand_of<__bf16, 2, 8>(g, d, s);
}

}  // namespace
}  // namespace nvfp4_46

using namespace nvfp4_46;

extern "C" size_t nvfp4_adapters_workspace_bytes(const nvfp4_adapters_params *p, int backward) {
  return p && sizes_fit(*p) ? (size_t)Layout(*p, backward != 0).bytes : 0;
}

extern "C" int nvfp4_adapters_forward(const void *x, const nvfp4_adapters_params *p, const void *base, const void *a, const void *b,
                                      const int32_t *which, const float *scales, float *h, void *out, void *workspace,
                                      size_t workspace_bytes, void *stream) {
  if (!p || !a || !b || !scales || !workspace) return NVFP4_ERR_NULL;
  if (p->tokens != 0 && (!x || !which || !out)) return NVFP4_ERR_NULL;
  if (!sizes_fit(*p) || !stride_fits(p->ld_x, p->inp, p->tokens) || (base && !stride_fits(p->ld_base, p->out, p->tokens)) ||
      !stride_fits(p->ld_out, p->out, p->tokens))
    return NVFP4_ERR_SHAPE;
  if (!at(x, 16) || !at(base, 16) || !at(a, 16) || !at(b, 16) || !at(out, 16) || !at(workspace, 16) || !at(which, 4) ||
      !at(scales, 4) || !at(h, 4) || p->ld_x % 8 || (base && p->ld_base % 8) || p->ld_out % 8)
    return NVFP4_ERR_ALIGN;
  const Layout d(*p, false);
  if (p->out_dtype > NVFP4_OUT_F32 || workspace_bytes < (size_t)d.bytes) return NVFP4_ERR_PARAM;
  if (p->tokens == 0) return NVFP4_OK;
  char *const w = static_cast<char *>(workspace);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (!d.few)
    if (const int rc = run_plan(*p, d, w, which, nullptr, nullptr, s)) return rc;
  const Tokens tokens{which, d.plan(w), (int32_t)p->tokens, (int32_t)p->adapters, d.few};
  const bool direct = h && d.splits_in == 1;                 // k_shrink's one part is h itself
  float *const parts = direct ? h : reinterpret_cast<float *>(w + d.h);
  if (const int rc = run_shrink({tokens, static_cast<const __bf16 *>(x), static_cast<const __bf16 *>(a), parts, p->ld_x, p->inp,
                                 (int32_t)p->rank, 0, direct}, d, d.splits_in, s))
    return rc;
  return run_expand({tokens, parts, direct ? nullptr : h, static_cast<const __bf16 *>(b), scales, base, out, p->ld_base, p->ld_out,
                     p->out, (int32_t)p->rank, (int32_t)p->rank, (int32_t)d.splits_in}, d, p->out_dtype == NVFP4_OUT_F32, s);
}

extern "C" int nvfp4_adapters_backward(const void *dy, const nvfp4_adapters_params *p, const void *x, const float *h, const void *a,
                                       const void *b, const int32_t *which, const float *scales, const void *dx_base, void *dx,
                                       float *da, float *db, void *workspace, size_t workspace_bytes, void *stream) {
  if (!p || !a || !b || !scales || !da || !db || !workspace) return NVFP4_ERR_NULL;
  if (p->tokens != 0 && (!dy || !x || !h || !which)) return NVFP4_ERR_NULL;
  if (!sizes_fit(*p) || !stride_fits(p->ld_x, p->inp, p->tokens) || !stride_fits(p->ld_dy, p->out, p->tokens) ||
      (dx && dx_base && !stride_fits(p->ld_base, p->inp, p->tokens)) || (dx && !stride_fits(p->ld_out, p->inp, p->tokens)))
    return NVFP4_ERR_SHAPE;
  if (!at(dy, 16) || !at(x, 16) || !at(a, 16) || !at(b, 16) || !at(dx_base, 16) || !at(dx, 16) || !at(da, 16) || !at(db, 16) ||
      !at(workspace, 16) || !at(h, 4) || !at(which, 4) || !at(scales, 4) || p->ld_x % 8 || p->ld_dy % 8 ||
      (dx && dx_base && p->ld_base % 8) || (dx && p->ld_out % 8))
    return NVFP4_ERR_ALIGN;
  const Layout d(*p, true);
  if (workspace_bytes < (size_t)d.bytes) return NVFP4_ERR_PARAM;
  char *const w = static_cast<char *>(workspace);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool any = p->tokens != 0;
  if (const int rc = run_plan(*p, d, w, which, any ? a : nullptr, b, s)) return rc;
  const Tokens tokens{which, d.plan(w), (int32_t)p->tokens, (int32_t)p->adapters, false};
  float *const parts = reinterpret_cast<float *>(w + d.h);
  const int32_t rank = (int32_t)p->rank;
  OuterArgs g{d.plan(w), scales, (int32_t)p->tokens, (int32_t)p->adapters, rank, (int32_t)d.range_tiles,
              {{static_cast<const __bf16 *>(x), parts, da, reinterpret_cast<float *>(w + d.parted_a), p->ld_x, p->inp,
                (int32_t)d.splits_out, (int32_t)divide_up(p->inp, kOuterWidth), false},
               {static_cast<const __bf16 *>(dy), h, db, reinterpret_cast<float *>(w + d.parted_b), p->ld_dy, p->out, 1,
                (int32_t)divide_up(p->out, kOuterWidth), true}}};
  if (any) {
    if (const int rc = run_shrink({tokens, static_cast<const __bf16 *>(dy), reinterpret_cast<const __bf16 *>(w + d.bt), parts, p->ld_dy,
                                   p->out, rank, 0, false}, d, d.splits_out, s))
      return rc;
    if (dx)
      if (const int rc = run_expand({tokens, parts, nullptr, reinterpret_cast<const __bf16 *>(w + d.at), scales, dx_base, dx,
                                     p->ld_base, p->ld_out, p->inp, rank, (int32_t)Layout::pitch(*p), (int32_t)d.splits_out}, d, false, s))
        return rc;
    const dim3 grid((uint32_t)(g.half[0].chunks + g.half[1].chunks), (uint32_t)d.ranges, rank <= 64 ? 1 : 2);
    if (const int rc = launch(rank <= 16 ? k_outer<1> : rank <= 32 ? k_outer<2> : k_outer<4>, grid, dim3(256), 0, s, g))
      return rc;
  }
  const int64_t most = divide_up(p->rank * (p->inp > p->out ? p->inp : p->out), 1024);
  return launch(k_join, dim3((uint32_t)(most < 256 ? most : 256), (uint32_t)p->adapters), dim3(256), 0, s, g);
}
