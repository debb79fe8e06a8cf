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
//   k_plan     tokens in the order of their adapters (stable), tiles of 32
//   k_shrink   [T][width] times [rank][width] -> [T][rank]            h from x and A, dh / s from dy and B
//   k_expand   base + s [T][rank] times [width][rank]                 out from h and B, dx from dh / s and A
//   k_outer    s [T][rank] times [T][width] over an adapter's tokens  dA from dh / s and x, dB from h and dy
//   k_join     sums what several workgroups of k_outer have of one adapter, in a fixed order
//
// Forwards that is two launches up to kFewTokens tokens and three beyond, backwards four and five.  Whole calls, among others:
// 16384 tokens, 4096 x 4096, rank 16, four adapters 117 us (405 MB: 3.5 TB/s, a copy 5.1), of which plan 9, shrink 39, expand 71; backwards 8192
// tokens, 8192 x 8192, rank 32, eight adapters 205 us (563 MB): plan 9, shrink 40, expand 80, outer 75, join 6.  One token 8.5 us: two launches.
#include <hip/hip_runtime.h>

#include "finetune/nvfp4_finetune.h"
#include "launch.hpp"

namespace nvfp4_46 {
namespace {

constexpr int kMostRank = 128, kMostAdapters = 2048;          // (by the instances of the kernels, by the LDS of k_plan)
constexpr int kTile = 32;                       // tokens of a planned tile
constexpr int kFewTile = 16;                    // ... and of a tile that a workgroup finds for itself
// Forwards, up to here there is no plan (find_tile).  Without / with one, several batches and their adapters in turn, 4096 x 4096, rank 16, 16
// adapters: 96 tokens 9.7 / 15.7 us, 192 12.1 / 16.5, 256 17.9 / 16.6; where every token reads much of an adapter, earlier: 8192 x 8192, rank 64, 32
// adapters: 128 tokens 41 / 32, 256 47 / 31 (28 and 29 at 128 tokens of one batch again and again, whose adapters stay in the caches).
constexpr int kFewTokens = 192;
// Backwards, up to here an adapter's gradients are one workgroup's sums and k_join is not needed.  4096 x 4096, rank 16: 256 tokens of
// one adapter 21.7 us so, 23.2 with k_join, 512 tokens of 16 adapters 30.4 / 34.1, 512 of one 24.6 / 24.7.
constexpr int kWholeTokens = 512;
constexpr int kPlanThreads = 1024;
constexpr int kOuterWidth = 128;                // columns of a workgroup of k_outer
constexpr int kBlock = 64;                      // columns of a block of k_expand

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Tile {
  int32_t adapter, count;      // (tokens without an adapter come last, as tiles of adapter -1)
};

// What k_plan writes.
struct Plan {
  int32_t *count;                               // tiles
  int32_t *tile_begin;                          // [L + 2]: the first tile of every adapter, of those without, the end
  Tile *tiles;
  int32_t *order;                               // [tiles][32]: their tokens, -1 past a tile's last
};

// A workgroup's stretch of `units` (tiles, or halves of them).  Where there is a workgroup for each that there can be, it is known before
// the plan's count has been read.
__device__ inline void stretch(const Plan &plan, int32_t per_tile, bool single, int32_t &first, int32_t &last) {
  const int32_t all = per_tile * *plan.count, per = single ? 1 : (all + (int32_t)gridDim.x - 1) / (int32_t)gridDim.x;
  first = (int32_t)blockIdx.x * per;
  last = first + per < all ? first + per : all;
}

// Where tiles come from: a plan, or (few tokens) `which` itself.
struct Tokens {
  const int32_t *which;
  Plan plan;
  int32_t T, L;
};

__device__ inline int32_t adapter_of(const int32_t *which, int32_t t, int32_t L) {
  const int32_t l = which[t];
  return l >= 0 && l < L ? l : -1;
}

// ---- tiles ----------------------------------------------------------------------------------------------------------

struct TileTokens {
  int32_t token[kFewTile];
  uint64_t same[kFewTokens / 64];               // tokens of this workgroup's adapter, a bit each
};

// Without a plan: the tile that the token `index` leads, its tokens in `shared`; count 0: it leads none.  All threads of the workgroup
// call it.  A token leads a tile if a multiple of 16 of the tokens before it have its adapter, and the next of them go with it.
template <int NT>
__device__ inline Tile find_tile(const Tokens &k, TileTokens &shared, int32_t index) {
  Tile t{adapter_of(k.which, index, k.L), 0};
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
  if (mine % kFewTile) return t;
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
// A wave's number as the one value that it is: conditions on it become branches.  Lanes that are masked off do not keep the matrix
// unit from writing, so a product under a condition has to be jumped over, not masked.
__device__ inline int wave_of(uint32_t thread) { return __builtin_amdgcn_readfirstlane(thread / 64); }
__device__ inline f32x4 multiply(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// The BF16 next to v on the side of 0 (never v itself); 0 of 0.
__device__ inline float below(float v) {
  const uint32_t bits = __float_as_uint(v);
  return bits << 1 ? __uint_as_float((bits - 1) & 0xffff0000u) : v;
}
// v as a sum of three BF16 terms, eight of its 24 bits each, exactly; where the result is BF16 too, whose rounding hides what a third term adds
// only where neither the ranks' products nor the base cancel.  (Two terms, 2^-16 of v left, / three: 16384 x 4096, rank 16 115 / 116 us, rank 64
// 146 / 149; 4096 tokens, rank 128 89 / 93.)
// All terms have v's sign and none is 0 unless v is, so that an infinity that meets them in a product comes out as if it met v: with terms rounded to
// nearest inf times the second, 0 or of the other sign, made a NaN of it.  (Below 2^-110 BF16 has no numbers for all three.)  Of an infinity, or NaN,
// the first term is all there is, and the others must not be 0.
__device__ inline __bf16 term(float v, int which) {
  const bool finite = __builtin_isfinite(v);
  if (which == 0) return (__bf16)(finite ? below(v) : v);
  const float rest = finite ? v - below(v) : __builtin_copysignf(1.0f, v), mid = below(rest);
  return (__bf16)(which == 1 ? mid : rest - mid);
}

// ---- k_shrink ---------------------------------------------------------------------------------------------------------

struct ShrinkArgs {
  Tokens tokens;
  const __bf16 *x, *w;         // [T] rows of `width`, and [L][rank][width], or ACROSS [L][width][rank]
  float *parts;                // [splits][T][pitch]
  float *h;                    // [T][rank], where one split is all and it is wanted; 0 for tokens without an adapter
  // backwards: the forward pass' h [T][rank], whose terms go to k_outer from here
  const float *terms_of, *scales;
  __bf16 *terms;
  int64_t ld, width;
  int32_t rank, pitch;
  int32_t steps;               // 32 columns each, of a wave: at most NF
  int32_t term_ranks, splits;
  bool single;                 // a workgroup for every 16 tokens
};

constexpr int kShrinkWaves = 8;

// D[token][rank]: rows of x against rows of w (ACROSS: its columns, turned in LDS once an adapter).  A wave has its own columns and keeps
// their part of w in registers while it goes through 16 tokens at a time of the workgroup's stretch of the plan; the waves' sums meet in
// LDS.  A load has 64 adjacent bytes of 16 rows; the columns of the next tokens are on their way while these are multiplied.
// Bound by the loads of x.  16384 x 4096 (134 MB) by itself: 29 us at rank 16, 33 at 32, 39 at 64, 53 at 128; the loads alone 22.5 to 25.  With
// w read again for every tile, through the L2, it was 35 to 44 at rank 16 and 52 at 64.
template <bool FEW, bool ACROSS, int RT, int NF>
__global__ void __launch_bounds__(kShrinkWaves * 64, RT * NF <= 8 && !(ACROSS && RT == 4) ? 4 : 2) k_shrink(ShrinkArgs a) {
  constexpr int kThreads = kShrinkWaves * 64, kBuffers = RT <= 4 ? 2 : 1;
  __shared__ TileTokens shared;
  __shared__ float part[kBuffers][kShrinkWaves][RT * 256];
  __shared__ __align__(16) __bf16 turned[ACROSS ? kShrinkWaves : 1][ACROSS ? 32 * RT * 16 + 64 : 8];
  const int lane = threadIdx.x & 63, wave = wave_of(threadIdx.x), row = lane & 15, group = lane / 16;
  int32_t first = 0, last = 1, token = 0;        // 16 tokens each
  int32_t adapter_here = -1, count_here = 0;     // of the only tile
  if constexpr (FEW) {
    const Tile t = find_tile<kThreads>(a.tokens, shared, blockIdx.x);
    if (t.count == 0) return;
    adapter_here = t.adapter;
    count_here = t.count;
  } else {
    if (a.single) {                              // asked for together with the count
      adapter_here = a.tokens.plan.tiles[blockIdx.x / 2].adapter;
      count_here = a.tokens.plan.tiles[blockIdx.x / 2].count;
      token = a.tokens.plan.order[(int64_t)blockIdx.x * 16 + row];
    }
    stretch(a.tokens.plan, 2, a.single, first, last);
  }
  const auto tile_of = [&](int32_t i) {          // the 16 tokens i
    if constexpr (FEW) return Tile{adapter_here, count_here};
    const int32_t adapter = a.single ? adapter_here : a.tokens.plan.tiles[i / 2].adapter;
    const int32_t left = (a.single ? count_here : a.tokens.plan.tiles[i / 2].count) - i % 2 * 16;
    return Tile{adapter, left < 16 ? left : 16};
  };
  const auto token_of = [&](int32_t i, int n) -> int32_t {      // -1: there is none
    if constexpr (FEW) return n < count_here ? shared.token[n] : -1;
    return a.tokens.plan.order[(int64_t)i * 16 + n];
  };
  const int32_t all_steps = (int32_t)((a.width + 31) / 32), step0 = ((int32_t)blockIdx.y * kShrinkWaves + wave) * a.steps;
  const int32_t mine = all_steps - step0 < a.steps ? all_steps - step0 : a.steps;
  const int32_t width = (int32_t)a.width, c0 = step0 * 32 + group * 8;
  const bool whole = mine == NF && (step0 + NF) * 32 <= width;
  const auto fetch = [&](bf16x8 *to, const __bf16 *from) {      // (where there is no such column, another)
#pragma unroll
    for (int f = 0; f < NF; ++f) to[f] = load8(from + (c0 + f * 32 < width ? c0 + f * 32 : width - 8));
  };
  const auto clear = [&](bf16x8 *to) {           // what is no column of this wave's counts as 0, whatever was loaded
    if (whole) return;
#pragma unroll
    for (int f = 0; f < NF; ++f)
      if (f >= mine || c0 + f * 32 >= width) to[f] = bf16x8{};
  };
  if constexpr (!FEW) {
    if ((int32_t)blockIdx.y == a.splits) {       // backwards there is one more row of workgroups, for the terms of h
      for (int32_t tile = (first + 1) / 2; tile < (last + 1) / 2; ++tile) {       // those that begin in this stretch
        const int32_t l = a.tokens.plan.tiles[tile].adapter;
        if (l < 0) break;
        for (int e = threadIdx.x; e < kTile * a.term_ranks; e += kThreads) {
          const int n = e % kTile, rank = e / kTile;
          const int32_t of = a.tokens.plan.order[(int64_t)tile * kTile + n];
          const bool is = of >= 0 && rank < a.rank;
          const float h = a.terms_of[(int64_t)(is ? of : 0) * a.rank + (is ? rank : 0)], v = is ? a.scales[l] * h : 0.0f;
          for (int which = 0; which < 3; ++which) a.terms[(((int64_t)tile * 3 + which) * a.term_ranks + rank) * kTile + n] = term(v, which);
        }
      }
      return;
    }
  }
  const auto row_of = [&](int32_t token) { return a.x + (int64_t)(token < 0 ? 0 : token) * a.ld; };
  bf16x8 w[RT][NF], x[NF];
  int32_t buffer = 0;
  if (first < last) {
    fetch(x, row_of(!FEW && a.single ? token : token_of(first, row)));
    if (first + 1 < last) token = token_of(first + 1, row);
  }
  for (int32_t i = first; i < last;) {           // one adapter after the other
    const int32_t adapter = tile_of(i).adapter;
    if (adapter < 0) break;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int n = r * 16 + row < a.rank ? r * 16 + row : a.rank - 1;            // (ranks past the last are not kept)
      if constexpr (!ACROSS) {
        fetch(w[r], a.w + ((int64_t)adapter * a.rank + n) * a.width);
        clear(w[r]);
      } else {
        // 32 columns of a step are 4 rank adjacent pieces of 16 bytes, 64 of them to a load
        const __bf16 *const from = a.w + (int64_t)adapter * a.width * a.rank;
        const int64_t most = (int64_t)width * a.rank / 8 - 1;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const int64_t piece = (int64_t)(step0 + f) * 4 * a.rank + r * 64 + lane;
          w[r][f] = load8(from + (piece < most ? piece : most) * 8);
        }
      }
    }
    if constexpr (ACROSS) {                      // the other way round, a step at a time through the wave's own LDS
      __bf16 *const turn = turned[ACROSS ? wave : 0];
      const int pieces = 4 * a.rank;
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        for (int r = 0; r < RT; ++r)             // (8 columns are `rank` pieces; 32 bytes between them keep their banks apart)
          if (const int piece = r * 64 + lane; piece < pieces) *reinterpret_cast<bf16x8 *>(turn + piece * 8 + piece / a.rank * 16) = w[r][f];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        int32_t line = group * (8 * a.rank + 16);
        asm("" : "+v"(line));                    // (the places are found again for each step: kept, they would not leave registers)
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const int n = r * 16 + row < a.rank ? r * 16 + row : a.rank - 1;
          for (int k = 0; k < 8; ++k) w[r][f][k] = turn[line + k * a.rank + n];
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_sched_barrier(0);
      }
      for (int r = 0; r < RT; ++r) clear(w[r]);
    }
    for (; i < last; ++i) {
      const Tile t = tile_of(i);
      if (t.adapter != adapter) break;
      const int32_t to = token_of(i, threadIdx.x % 256 / 16);         // (where this thread's sums go, the same for all of them)
      clear(x);
      f32x4 acc[RT] = {};
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[r] = multiply(x[f], w[r][f], acc[r]);
      __builtin_amdgcn_sched_barrier(0);         // (the next columns go where these were: a second place for them costs a workgroup a CU)
      if (i + 1 < last) {
        fetch(x, row_of(token));
        if (i + 2 < last) token = token_of(i + 2, row);
      }
      if (t.count <= 0) continue;                // (the second half of a tile of 16)
      // (a buffer is written again only after the barrier of the tile in between, which all waves reach done with reading it)
      float(*const p)[RT * 256] = part[buffer];
      if (kBuffers == 1) __syncthreads();
      else buffer ^= 1;
#pragma unroll
      for (int r = 0; r < RT; ++r)
        for (int v = 0; v < 4; ++v) p[wave][r * 256 + (group * 4 + v) * 16 + row] = acc[r][v];
      __syncthreads();
      for (int e = threadIdx.x; e < RT * 256; e += kThreads) {
        const int rank = e / 256 * 16 + e % 16;
        float s = 0.0f;
        for (int k = 0; k < kShrinkWaves; ++k) s += p[k][e];
        if (to >= 0 && rank < a.pitch) {
          a.parts[((int64_t)blockIdx.y * a.tokens.T + to) * a.pitch + rank] = rank < a.rank ? s : 0.0f;
          if (a.h && rank < a.rank) a.h[(int64_t)to * a.rank + rank] = s;
        }
      }
    }
  }
  if (a.h)                                       // tokens without an adapter come last
    for (int32_t i = last; i-- > first && tile_of(i).adapter < 0;)
      for (int e = threadIdx.x; e < tile_of(i).count * a.rank; e += kThreads)
        a.h[(int64_t)token_of(i, e / a.rank) * a.rank + e % a.rank] = 0.0f;
}

// ---- k_expand ---------------------------------------------------------------------------------------------------------

struct ExpandArgs {
  Tokens tokens;
  const float *parts;          // [splits][T][h_pitch]
  float *h;                    // their sum [T][rank], where it is wanted and k_shrink has not written it; or nullptr
  __bf16 *terms;               // backwards: the three terms of s h for k_outer, [tile][term][rank][token]; or nullptr
  const __bf16 *w;             // [L][width][rank], or kAcross [L][rank][width]
  const float *scales;
  const void *base;
  void *out;                   // nullptr: only the terms
  int64_t ld_base, ld_out, width;
  int32_t rank, h_pitch, splits, term_ranks;
  bool single;                 // a workgroup for every tile
};

// How the matrix of k_expand lies: rows of ranks that are whole pieces of 16 bytes, or not, or the other way round [rank][width].
enum { kWhole, kRagged, kAcross };

// Eight columns of a row as they are in memory, and as fp32.
template <typename T>
struct Columns {
  u32x4 raw[sizeof(T) / 2];
  __device__ void load(const T *p) {
    for (size_t i = 0; i < sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const u32x4 *>(p)[i];
  }
  __device__ float at(int k) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[k / 4][k % 4]);
    const uint32_t w = raw[0][k / 2];
    return __uint_as_float(k % 2 ? w & 0xffff0000u : w << 16);
  }
  __device__ void add(int k0, f32x4 v) {         // to columns k0 .. k0 + 3
    if constexpr (sizeof(T) == 4) {
      for (int k = 0; k < 4; ++k) raw[k0 / 4][k] = __float_as_uint(at(k0 + k) + v[k]);
    } else {
      for (int k = 0; k < 4; k += 2) {
        const bf16x2 q{(__bf16)(at(k0 + k) + v[k]), (__bf16)(at(k0 + k + 1) + v[k + 1])};
        raw[0][(k0 + k) / 2] = __builtin_bit_cast(uint32_t, q);
      }
    }
  }
  __device__ void store(T *p) const {
    for (size_t i = 0; i < sizeof(T) / 2; ++i) reinterpret_cast<u32x4 *>(p)[i] = raw[i];
  }
};

// D[column][token]: rows of w against s h, which enters as terms (term).  Row 4 a + b of product p of a block is column
// 32 (p / 2) + 8 a + 4 (p % 2) + b, so that a lane ends up with twice 8 adjacent columns of its token, 64 bytes in four lanes.  The
// summed index of a product is four pieces of eight ranks: F > 0: 32 ranks of one term, F times.  F == 0, rank <= 16: the one or two pieces
// of every term side by side, the third by halves, which fill the four that there are (0 must not meet w, as an infinity would be NaN).
// A wave has a block of columns of its own and keeps their part of w in registers while it goes through the workgroup's stretch of the
// plan; per tile the workgroup sums the parts of s h and splits them once, into LDS, while the tile's columns of base are on their way.
// Bound by base and out.  16384 x 4096 BF16 (268 MB), within the call: 70 us at rank 16, 73 at 32, 94 at 64, 138 at 128; a copy of as much 57.
// Planned, BF16: eight waves a workgroup, two workgroups a compute unit, where 128 registers are enough (up to 32 ranks), or one, where 168 are
// not (beyond 64); four waves, and three workgroups, in between: 33 to 64 ranks in 128 registers left up to 148 bytes a thread to scratch memory.
// fp32 four waves, and three or two.  Whole calls with spills / without, 4096 x 4096, rank 64: 4096 tokens 72.4 / 68.5 us, backwards 128 / 120; 16384
// tokens 146.7 / 147.7, backwards 276 / 270.
// Ranks that are no multiple of 8 (kRagged) go through LDS too; element by element from memory they took registers, and spilled.  So / through
// LDS: 16384 tokens, rank 12 138 / 116 us, rank 100 250 / 205, 128 tokens of 8 adapters, rank 100 64 / 29.
template <bool FEW, typename T, int F>
constexpr int expand_waves = !FEW && sizeof(T) == 2 && F != 2 ? 8 : 4;

template <bool FEW, int LIES, typename T, int F>
__global__ void __launch_bounds__((expand_waves<FEW, T, F>)*64, F == 4 ? 2 : (expand_waves<FEW, T, F>) == 8 ? 4 : 3) k_expand(ExpandArgs a) {
  constexpr int kTerms = 3, kSpans = F ? F : 1, kProducts = F ? kTerms : 2;
  constexpr int MT = FEW ? 1 : 2, kWaves = expand_waves<FEW, T, F>, kThreads = kWaves * 64, kRows = MT * 16;
  __shared__ TileTokens shared;
  // An odd number of pieces, a row a bank further; of many pieces, which would leave LDS for one workgroup, an even one, the places in a row
  // exchanged instead.
  __shared__ bf16x8 split[FEW ? 1 : 2][kRows][kTerms * kSpans * 4 + (F == 4 ? 0 : 1)];
  const auto place = [](int n, int piece) { return F == 4 ? piece ^ (n & 15) : piece; };
  __shared__ __align__(16) __bf16 turned[LIES == kWhole ? 1 : kWaves][LIES == kAcross ? 32 * 68 : LIES == kRagged ? 32 * (F ? F * 32 : 16) : 8];
  const int lane = threadIdx.x & 63, wave = wave_of(threadIdx.x), row = lane & 15, group = lane / 16;
  int32_t first = 0, last = 1, in[MT];           // in: this lane's token of each 16, -1: there is none
  int32_t adapter_here = -1, count_here = 0;     // of the only tile
  if constexpr (FEW) {
    const Tile t = find_tile<kThreads>(a.tokens, shared, blockIdx.x);
    if (t.count == 0) return;
    adapter_here = t.adapter;
    count_here = t.count;
  } else {
    if (a.single) {                              // asked for together with the count
      adapter_here = a.tokens.plan.tiles[blockIdx.x].adapter;
      count_here = a.tokens.plan.tiles[blockIdx.x].count;
      for (int m = 0; m < MT; ++m) in[m] = a.tokens.plan.order[(int64_t)blockIdx.x * kRows + m * 16 + row];
    }
    stretch(a.tokens.plan, 1, a.single, first, last);
  }
  const auto tile_of = [&](int32_t i) {
    if constexpr (FEW) return Tile{adapter_here, count_here};
    return a.single ? Tile{adapter_here, count_here} : Tile{a.tokens.plan.tiles[i].adapter, a.tokens.plan.tiles[i].count};
  };
  const auto token_of = [&](int32_t i, int n) -> int32_t {       // -1: there is none
    if constexpr (FEW) return n < count_here ? shared.token[n] : -1;
    return a.tokens.plan.order[(int64_t)i * kRows + n];
  };
  const T *const base = static_cast<const T *>(a.base);
  T *const out = static_cast<T *>(a.out);
  const int pieces = (a.rank + 7) / 8, two = pieces - 1;            // (F == 0: one piece or two, so that `two` divides by shifts)
  const int32_t width = (int32_t)a.width, c0 = ((int32_t)blockIdx.y * kWaves + wave) * kBlock;
  const bool idle = c0 >= width || !out;         // a wave past the last column only helps with h
  const auto column = [&](int half) { return c0 + half * 32 + group * 8; };

  const auto prepare = [&](int32_t i, int buffer) {
    const Tile t = tile_of(i);
    if (t.adapter < 0) return;
    const float scale = a.scales[t.adapter];
    const bool mine = FEW ? blockIdx.y == 0 : i % (int32_t)gridDim.y == (int32_t)blockIdx.y;      // whose h or terms it is to write
    for (int e = threadIdx.x; e < kRows * kSpans * 8; e += kThreads) {          // four ranks of a token each
      const int n = e / (kSpans * 8), from = e % (kSpans * 8) * 4;
      const int32_t token = token_of(i, n);
      f32x4 v{};
      if (token >= 0 && from < a.h_pitch) {
        const float *const part = a.parts + (int64_t)token * a.h_pitch + from;
        for (int p0 = 0; p0 < a.splits; p0 += 4) {                  // (four on their way; past the last once more the last)
          f32x4 q[4];
          for (int p = 0; p < 4; ++p)
            q[p] = *reinterpret_cast<const f32x4 *>(part + (int64_t)(p0 + p < a.splits ? p0 + p : a.splits - 1) * a.tokens.T * a.h_pitch);
          for (int p = 0; p < 4; ++p)
            if (p0 + p < a.splits) v += q[p];
        }
        if (a.h && mine)
          for (int k = 0; k < 4; ++k)
            if (from + k < a.rank) a.h[(int64_t)token * a.rank + from + k] = v[k];
        v *= scale;
      }
      for (int which = 0; which < kTerms; ++which) {
        bf16x4 q;
        for (int k = 0; k < 4; ++k) q[k] = term(v[k], which);
        if (!F && which == 2) q *= (__bf16)0.5f;                      // (the products have it twice)
        reinterpret_cast<bf16x4 *>(&split[buffer][n][place(n, which * kSpans * 4 + from / 8)])[from / 4 % 2] = q;
      }
      if (a.terms && mine && from < a.term_ranks) {
        __bf16 *const to = a.terms + ((int64_t)i * 3 * a.term_ranks + from) * kTile + n;
        for (int which = 0; which < 3; ++which)
          for (int k = 0; k < 4; ++k) to[(which * a.term_ranks + k) * kTile] = term(v[k], which);
      }
    }
  };

  Columns<T> v[MT][2] = {};                      // (without a base 0)
  const auto fetch = [&](int32_t i) {            // (rows and columns that there are not: others, which are not kept)
    if (FEW || !a.single)
      for (int m = 0; m < MT; ++m) in[m] = token_of(i, m * 16 + row);
    if (base)
      for (int m = 0; m < MT; ++m)
        for (int half = 0; half < 2; ++half)
          v[m][half].load(base + (int64_t)(in[m] < 0 ? 0 : in[m]) * a.ld_base + (column(half) < width ? column(half) : width - 8));
    else
      for (int m = 0; m < MT; ++m)
        for (int half = 0; half < 2; ++half) v[m][half] = {};
  };
  bf16x8 w[4][kSpans];
  const auto fetch_w = [&](int32_t adapter) {
    const __bf16 *const of = a.w + (int64_t)adapter * a.width * a.rank;
    const auto column_of = [&](int p) { return c0 + p / 2 * 32 + row / 4 * 8 + p % 2 * 4 + row % 4; };
    if constexpr (LIES == kWhole) {
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int f = 0; f < kSpans; ++f) {
          const int piece = F ? f * 4 + group : group & two;
          w[p][f] = load8(of + (int64_t)(column_of(p) < width ? column_of(p) : width - 1) * a.rank + (piece < pieces ? piece * 8 : 0));
          if (F && piece >= pieces) w[p][f] = bf16x8{};
        }
    } else if constexpr (LIES == kRagged) {
      // 32 columns are 4 rank adjacent pieces of 16 bytes, 64 of them to a load; the wave's own LDS gives them back by columns and ranks.
      constexpr int kLoads = F ? 2 * F : 1;
      __bf16 *const turn = turned[LIES == kRagged ? wave : 0];
      const __bf16 *const from = of + (int64_t)c0 * a.rank;
      const int32_t most = (width - c0) * a.rank / 8 - 1;              // (of 64 columns, or of fewer where the matrix ends)
      int32_t lane0 = lane;
      asm("" : "+v"(lane0));                     // (the places are found again for each adapter and piece: kept, they would not leave registers)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int32_t piece = half * 4 * a.rank + i * 64 + lane0;
          w[half * 2 + i / kSpans][i % kSpans] = load8(from + (piece < most ? piece : most) * 8);
        }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
          if (i * 64 + lane0 < 4 * a.rank) *reinterpret_cast<bf16x8 *>(turn + (i * 64 + lane0) * 8) = w[half * 2 + i / kSpans][i % kSpans];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int p = half * 2; p < half * 2 + 2; ++p)
#pragma unroll
          for (int f = 0; f < kSpans; ++f) {
            int32_t rank = (F ? f * 4 + group : group & two) * 8, line = (column_of(p) - c0 - half * 32) * a.rank;
            asm("" : "+v"(rank), "+v"(line));
            for (int k = 0; k < 8; ++k) w[p][f][k] = rank + k < a.rank ? turn[line + rank + k] : (__bf16)0.0f;
            __builtin_amdgcn_sched_barrier(0);
          }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      // A load has eight ranks' 64 columns; 32 ranks at a time are turned in the wave's own LDS.
      __bf16 *const turn = turned[LIES == kAcross ? wave : 0];
      constexpr int kLine = 68;                  // (eight lines are 16 banks further)
#pragma unroll
      for (int f = 0; f < kSpans; ++f)
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const int rank = f * 32 + p * 8 + lane / 8;
          const int32_t c = c0 + lane % 8 * 8;
          w[p][f] = load8(of + (int64_t)(rank < a.rank ? rank : a.rank - 1) * a.width + (c < width ? c : width - 8));
          if (rank >= a.rank) w[p][f] = bf16x8{};
        }
#pragma unroll
      for (int f = 0; f < kSpans; ++f) {
        for (int p = 0; p < 4; ++p)
          for (int k = 0; k < 2; ++k)
            reinterpret_cast<bf16x4 *>(turn + (p * 8 + lane / 8) * kLine + lane % 8 * 8)[k] = k ? bf16x4{w[p][f][4], w[p][f][5], w[p][f][6], w[p][f][7]}
                                                                                              : bf16x4{w[p][f][0], w[p][f][1], w[p][f][2], w[p][f][3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const int piece = F ? group : group & two;
          for (int k = 0; k < 8; ++k) w[p][f][k] = turn[(piece * 8 + k) * kLine + column_of(p) - c0];
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
  };
  int buffer = 0, i = first;
  int32_t adapter = -1;
  if (first < last) {
    adapter = tile_of(first).adapter;
    if (!idle) {
      fetch(first);
      if (adapter >= 0) fetch_w(adapter);
    }
    prepare(first, 0);
  }
  __syncthreads();
  while (i < last && adapter >= 0) {             // one adapter after the other
    for (; i < last && tile_of(i).adapter == adapter; ++i) {
      if (!idle) {
        f32x4 acc[MT][4] = {};
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int f = 0; f < kSpans; ++f)
#pragma unroll
            for (int n = 0; n < kProducts; ++n) {
              if (!F && n == 1 && pieces == 1) break;        // (all terms of eight ranks are one product)
              bf16x8 h;
              if (F) {
                h = split[buffer][m * 16 + row][place(row, n * kSpans * 4 + f * 4 + group)];
              } else {
                const int q = n * 4 + group, which = q >> two < 2 ? q >> two : 2;
                h = split[buffer][m * 16 + row][which * 4 + (q & two)];
              }
#pragma unroll
              for (int p = 0; p < 4; ++p) acc[m][p] = multiply(w[p][f], h, acc[m][p]);
            }
#pragma unroll
        for (int m = 0; m < MT; ++m)
          for (int half = 0; half < 2; ++half) {
            for (int k = 0; k < 2; ++k) v[m][half].add(4 * k, acc[m][half * 2 + k]);
            if (in[m] >= 0 && column(half) < width) v[m][half].store(out + (int64_t)in[m] * a.ld_out + column(half));
          }
        __builtin_amdgcn_sched_barrier(0);
        if (i + 1 < last) fetch(i + 1);
      }
      if (i + 1 < last) prepare(i + 1, FEW ? 0 : buffer ^ 1);
      if (!FEW) __syncthreads();                 // (each buffer is written again a barrier after it was read)
      buffer ^= 1;
    }
    if (i < last) {
      adapter = tile_of(i).adapter;
      if (adapter >= 0 && !idle) fetch_w(adapter);
    }
  }
  // Tokens without an adapter come last.
  for (; i < last; ++i) {
    const Tile t = tile_of(i);
    if (a.h && blockIdx.y == 0)
      for (int e = threadIdx.x; e < t.count * a.rank; e += kThreads) a.h[(int64_t)token_of(i, e / a.rank) * a.rank + e % a.rank] = 0.0f;
    if (idle || base == out) continue;
    fetch(i);
    for (int m = 0; m < MT; ++m)
      for (int half = 0; half < 2; ++half)
        if (in[m] >= 0 && column(half) < width) v[m][half].store(out + (int64_t)in[m] * a.ld_out + column(half));
  }
}

// ---- k_plan -----------------------------------------------------------------------------------------------------------

struct PlanArgs {
  const int32_t *which;
  Plan plan;
  int32_t T, L;
};

// Stable counting sort by one workgroup, each wave its own stretch of the tokens, 64 at a time, or 256 where they have one adapter.
// Bound by the instructions of its sixteen waves: 5 us for 2048 tokens, 9 for 16384 in segments (17 at 64 at a time).
__global__ void __launch_bounds__(kPlanThreads) k_plan(PlanArgs p) {
  extern __shared__ int32_t counts[];            // [16][groups + 1]: each wave's tokens of a group, then how many come before them
  const int32_t groups = p.L + 1, line = groups + 1;
  int32_t *const tile_begin = counts + 16 * line, *const members = tile_begin + groups + 1;
  __shared__ int32_t waves[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  for (int32_t i = threadIdx.x; i < 16 * line; i += kPlanThreads) counts[i] = 0;
  __syncthreads();
  int32_t *const mine = counts + wave * line;
  const int32_t slice = (p.T + 1023) / 1024 * 64, begin = wave * slice;
  const int32_t end = begin + slice < p.T ? begin + slice : p.T;
  // the lanes with this lane's group
  const auto alike = [&](int32_t l) {
    uint64_t m = ~(uint64_t)0;
    if (__ballot(l == __builtin_amdgcn_readfirstlane(l)) == m) return m;       // (requests one after the other: nearly always)
    for (int32_t bit = 1; bit <= groups; bit <<= 1) {
      const uint64_t set = __ballot((l & bit) != 0);
      m &= l & bit ? set : ~set;
    }
    return m;
  };
  constexpr int kAhead = 16;                     // loads on their way
  int32_t group[kAhead];
  for (int pass = 0; pass < 2; ++pass) {
    for (int32_t t0 = begin; t0 < end; t0 += 64 * kAhead) {
      if (pass == 0 || slice > 64 * kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int32_t t = t0 + i * 64 + lane;
          group[i] = t < end ? p.which[t] : 0;
          // (past the end: a group of its own, which nobody reads)
          group[i] = t >= end ? groups : group[i] >= 0 && group[i] < p.L ? group[i] : p.L;
        }
      }
#pragma unroll
      for (int i0 = 0; i0 < kAhead; i0 += 4) {
        if (t0 + i0 * 64 >= end) break;
        // A wave's LDS instructions run in their order, so the lanes have all read before the first of each group adds; the fences keep
        // the compiler to it.
        const int32_t one = __builtin_amdgcn_readfirstlane(group[i0]);
        if (__ballot(group[i0] == one && group[i0 + 1] == one && group[i0 + 2] == one && group[i0 + 3] == one) == ~(uint64_t)0) {
          if (pass == 1) {                       // requests one after the other: nearly always
            int32_t *const to = p.plan.order + (int64_t)tile_begin[one] * kTile + mine[one] + lane;
            for (int i = 0; i < 4; ++i) to[i * 64] = t0 + (i0 + i) * 64 + lane;
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          if (lane == 0) __hip_atomic_fetch_add(mine + one, 256, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          continue;
        }
#pragma unroll
        for (int i = i0; i < i0 + 4; ++i) {
          const int32_t t = t0 + i * 64 + lane, l = group[i];
          if (t0 + i * 64 >= end) break;
          const uint64_t m = alike(l);
          const int32_t before = __popcll(m & (((uint64_t)1 << lane) - 1));
          if (pass == 1) {
            const int32_t at = mine[l];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (t < end) p.plan.order[(int64_t)tile_begin[l] * kTile + at + before] = t;
          }
          if (before == 0) __hip_atomic_fetch_add(mine + l, __popcll(m), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
      }
    }
    __syncthreads();
    if (pass == 1) break;
    // the waves' tokens of a group one after the other, the groups' tiles one after the other: each thread its adjacent groups
    const int32_t per = (groups + kPlanThreads - 1) / kPlanThreads, g0 = threadIdx.x * per;
    int32_t tiles = 0;
    for (int32_t g = g0; g < g0 + per && g < groups; ++g) {
      int32_t n = 0;
      for (int w = 0; w < 16; ++w) {
        const int32_t of = counts[w * line + g];
        counts[w * line + g] = n;
        n += of;
      }
      members[g] = n;
      tiles += (n + kTile - 1) / kTile;
    }
    int32_t upto = tiles;
    for (int d = 1; d < 64; d <<= 1) {
      const int32_t other = __shfl_up(upto, d);
      if (lane >= d) upto += other;
    }
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    int32_t at = upto - tiles;
    for (int w = 0; w < wave; ++w) at += waves[w];
    for (int32_t g = g0; g < g0 + per && g < groups; ++g) {
      tile_begin[g] = at;
      at += (members[g] + kTile - 1) / kTile;
      if (g == groups - 1) tile_begin[groups] = at;
    }
    __syncthreads();
    for (int32_t g = threadIdx.x; g <= groups; g += kPlanThreads) p.plan.tile_begin[g] = tile_begin[g];
    if (threadIdx.x == 0) *p.plan.count = tile_begin[groups];
    for (int32_t i = threadIdx.x; i < tile_begin[groups]; i += kPlanThreads) {
      int32_t lo = 0, hi = groups - 1;           // the last group that begins at tile i or before (those without tiles begin there too)
      while (lo < hi) {
        const int32_t mid = (lo + hi + 1) / 2;
        if (tile_begin[mid] <= i) lo = mid;
        else hi = mid - 1;
      }
      const int32_t left = members[lo] - (i - tile_begin[lo]) * kTile;
      p.plan.tiles[i] = {lo < p.L ? lo : -1, left < kTile ? left : kTile};
      for (int32_t n = left; n < kTile; ++n) p.plan.order[(int64_t)i * kTile + n] = -1;
    }
  }
}

// ---- k_outer ----------------------------------------------------------------------------------------------------------

struct OuterHalf {
  const __bf16 *x;             // [T] rows of `width`
  const __bf16 *terms;         // [tiles][3][term_ranks][32]: of s h
  float *out;                  // [L][rank][width], or with `by_rank` [L][width][rank]
  float *parted;               // [2 ranges] of the same
  int64_t ld, width;
  int32_t chunks;
  bool by_rank;
};
struct OuterArgs {
  Plan plan;
  int32_t L, rank, term_ranks, tiles;        // tiles of a range
  bool whole;                  // ranges have whole adapters, those that begin among their tiles
  OuterHalf half[2];
};

// Which of an adapter's tiles a range has decides where its sum goes: all of them, to the output; else to a place that the range
// has for the adapter that began before it (0) or for the one that begins in it and goes on (1).
__device__ inline int64_t place(const Plan &p, int32_t adapter, int32_t range, int32_t tiles) {
  const bool before = p.tile_begin[adapter] < range * tiles, after = p.tile_begin[adapter + 1] > (range + 1) * tiles;
  return before ? 2 * range : after ? 2 * range + 1 : -1;
}

// D[column][rank], summed over the tokens of a tile.  Of 32 tokens and 128 columns lane (row, group) loads columns 8 row .. 8 row + 7 of
// tokens 8 group .. 8 group + 7, which transposes within the lane: product j has columns 8 row + j.  The waves of a workgroup have the
// same columns and every fourth tile of an adapter each; their sums meet in LDS, so that a workgroup leaves one sum an adapter.
template <int RT>
__global__ void __launch_bounds__(256, RT <= 2 ? 2 : 1) k_outer(OuterArgs a) {
  __shared__ float sums[4][2048];
  const bool second = (int32_t)blockIdx.x >= a.half[0].chunks;
  const OuterHalf f = second ? a.half[1] : a.half[0];
  const int32_t chunk = (int32_t)blockIdx.x - (second ? a.half[0].chunks : 0), range = blockIdx.y, rank0 = blockIdx.z * RT * 16;
  const int lane = threadIdx.x & 63, wave = wave_of(threadIdx.x), row = lane & 15, group = lane / 16;
  const int64_t c0 = (int64_t)chunk * kOuterWidth, c = c0 + row * 8, size = f.width * a.rank;
  const __bf16 *const from = f.x + (c < f.width ? c : f.width - 8);          // (columns past the last are not kept)
  const int32_t count = *a.plan.count;
  const auto boundary = [&](int32_t i) {
    if (i >= count) return count;
    const int32_t l = a.plan.tiles[i].adapter;
    return !a.whole || l < 0 || a.plan.tile_begin[l] == i ? i : a.plan.tile_begin[l + 1];
  };
  const int32_t first = boundary(range * a.tiles), last = boundary((range + 1) * a.tiles);
  // eight columns of rank rank0 + r 16 + row, from c0 + (group 4 + wave) 8
  const auto put = [&](float *to, int r, const float *v) {
    const int rank = rank0 + r * 16 + row;
    const int64_t col = c0 + (group * 4 + wave) * 8;
    if (rank >= a.rank || col >= f.width) return;
    if (f.by_rank) {
      for (int j = 0; j < 8; ++j) to[(col + j) * a.rank + rank] = v[j];
    } else {
      for (int j = 0; j < 8; j += 4) *reinterpret_cast<f32x4 *>(to + rank * f.width + col + j) = f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]};
    }
  };
  if (range == 0)                                // adapters without tokens
    for (int32_t l = 0; l < a.L; ++l)
      if (a.plan.tile_begin[l] == a.plan.tile_begin[l + 1])
        for (int r = 0; r < RT; ++r) {
          const float zero[8] = {};
          put(f.out + l * size, r, zero);
        }
  const auto segment_end = [&](int32_t i, int32_t adapter) {
    const int32_t end = a.plan.tile_begin[adapter + 1];
    return end < last ? end : last;
  };
  // this wave's first tile of the segments from i on, `last`: there is none
  const auto first_from = [&](int32_t i) {
    while (i < last) {
      const int32_t l = a.plan.tiles[i].adapter;
      if (l < 0) return last;                    // (they come last)
      const int32_t end = segment_end(i, l);
      if (i + wave < end) return i + wave;
      i = end;
    }
    return last;
  };
  f32x4 acc[RT][8];
  u32x4 x[8];
  bf16x8 hs[RT][3];
  u32x4 token[2];
  const auto fetch_tokens = [&](int32_t i) {
    for (int k = 0; k < 2; ++k) token[k] = reinterpret_cast<const u32x4 *>(a.plan.order + (int64_t)i * kTile + group * 8)[k];
  };
  const auto fetch_x = [&] {
    for (int q = 0; q < 8; ++q) {
      const int32_t t = (int32_t)token[q / 4][q % 4];
      x[q] = *reinterpret_cast<const u32x4 *>(from + (int64_t)(t < 0 ? 0 : t) * f.ld);
    }
  };
  const auto fetch_terms = [&](int32_t i) {
    for (int r = 0; r < RT; ++r)
      for (int which = 0; which < 3; ++which)
        hs[r][which] = load8(f.terms + ((i * (int64_t)3 + which) * a.term_ranks + rank0 + r * 16 + row) * kTile + group * 8);
  };
  // this wave's tile after `i`
  const auto after = [&](int32_t i) {
    const int32_t end = segment_end(i, a.plan.tiles[i].adapter);
    return i + 4 < end ? i + 4 : first_from(end);
  };
  // a tile's tokens are asked for a tile before its columns and terms, those while the tile before is multiplied
  int32_t mine = first_from(first), next = last;
  if (mine < last) {
    fetch_tokens(mine);
    fetch_x();
    fetch_terms(mine);
    next = after(mine);
    if (next < last) fetch_tokens(next);
  }
  for (int32_t i = first; i < last;) {
    const int32_t adapter = a.plan.tiles[i].adapter;
    if (adapter < 0) break;
    const int32_t end = segment_end(i, adapter);
    for (int r = 0; r < RT; ++r)
      for (int j = 0; j < 8; ++j) acc[r][j] = f32x4{};
    while (mine < end) {
      const Tile t = a.plan.tiles[mine];
      if (t.count < kTile)                       // (the terms there are 0, but what was loaded need not be finite)
        for (int q = 0; q < 8; ++q)
          if (group * 8 + q >= t.count) x[q] = u32x4{};
      bf16x8 xt[8];
      for (int j = 0; j < 8; ++j) {
        u32x4 p;
        for (int q = 0; q < 4; ++q) p[q] = __builtin_amdgcn_perm(x[2 * q + 1][j / 2], x[2 * q][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
        xt[j] = __builtin_bit_cast(bf16x8, p);
      }
      __builtin_amdgcn_sched_barrier(0);         // (the next tile's columns go where these were, its terms where these are)
      if (next < last) fetch_x();
      for (int r = 0; r < RT; ++r)
        for (int which = 0; which < 3; ++which)
          for (int j = 0; j < 8; ++j) acc[r][j] = multiply(xt[j], hs[r][which], acc[r][j]);
      __builtin_amdgcn_sched_barrier(0);
      mine = next;
      if (mine < last) {
        fetch_terms(mine);
        next = after(mine);
        if (next < last) fetch_tokens(next);
      }
    }
    const int64_t at = a.whole ? -1 : place(a.plan, adapter, range, a.tiles);
    float *const to = at < 0 ? f.out + adapter * size : f.parted + at * size;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      for (int j = 0; j < 8; ++j)
        for (int v = 0; v < 4; ++v) sums[wave][(j * 4 + v) * 64 + lane] = acc[r][j][v];
      __syncthreads();
      float v[8];
      for (int j = 0; j < 8; ++j) {
        const int e = (j * 4 + wave) * 64 + lane;
        v[j] = (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
      }
      put(to, r, v);
      __syncthreads();
    }
    i = end;
  }
}

// ---- k_join -----------------------------------------------------------------------------------------------------------

// Adapters whose tokens lie in several ranges.
__global__ void __launch_bounds__(256) k_join(OuterArgs a) {
  const int32_t l = blockIdx.y, t0 = a.plan.tile_begin[l], t1 = a.plan.tile_begin[l + 1];
  const int32_t s0 = t0 / a.tiles, s1 = (t1 - 1) / a.tiles;
  if (t1 <= t0 || s0 == s1) return;              // k_outer has written it
  const OuterHalf &f = a.half[blockIdx.z];
  const int64_t size = f.width * a.rank;         // (a multiple of 8)
  for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e < size; e += (int64_t)gridDim.x * 1024) {
    f32x4 s = *reinterpret_cast<const f32x4 *>(f.parted + (2 * (int64_t)s0 + 1) * size + e);
    for (int32_t r = s0 + 1; r <= s1; r += 4) {                     // (four on their way; past the last once more the last)
      f32x4 v[4];
      for (int k = 0; k < 4; ++k) v[k] = *reinterpret_cast<const f32x4 *>(f.parted + 2 * (int64_t)(r + k < s1 ? r + k : s1) * size + e);
      for (int k = 0; k < 4; ++k)
        if (r + k <= s1) s += v[k];
    }
    *reinterpret_cast<f32x4 *>(f.out + l * size + e) = s;
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------

constexpr int64_t kMostTokens = (1 << 24) - 1, kMostWidth = 1 << 22;

bool sizes_fit(const nvfp4_adapters_params &p) {
  return p.tokens >= 0 && p.tokens <= kMostTokens && p.inp > 0 && p.inp <= kMostWidth && p.out > 0 && p.out <= kMostWidth &&
         p.inp % 8 == 0 && p.out % 8 == 0 && p.adapters > 0 && p.adapters <= kMostAdapters && p.rank > 0 && p.rank <= kMostRank;
}
bool stride_fits(int64_t ld, int64_t width, int64_t rows) {
  return ld >= width && ld <= ((int64_t)1 << 40) / (rows > 0 ? rows : 1);
}
bool at(const void *ptr, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }
int64_t divide_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How a call's work is dealt out, and what it needs of the workspace: all of it follows from the sizes.
struct Layout {
  bool few, whole;
  int64_t tiles;               // at most so many planned tiles
  int64_t steps_in, steps_out, splits_in, splits_out;        // of k_shrink's sums over inp (h), over out (dh)
  int64_t ranges, range_tiles; // of k_outer
  int64_t count, tile_begin, order, table, parts, terms_a, terms_b, parted_a, parted_b, bytes;   // byte offsets

  // Steps of 32 columns that a wave of k_shrink keeps w of in registers: as many as fit (ranks; ACROSS needs more of them to turn w),
  // fewer where there would not be workgroups for half of the compute units, but not below two.  The splits of the sum follow: each
  // is one more part for k_expand to add up.
  static int64_t shrink_steps(int64_t tokens, bool few, int64_t width, int64_t rank, bool across) {
    const int64_t all = divide_up(width, 32), groups = few ? divide_up(tokens, 4) : divide_up(tokens, 16);
    int64_t steps = (rank <= 64 ? 8 : 4) / (across ? 2 : 1);
    while (steps > 2 && groups * divide_up(all, steps * kShrinkWaves) < 128) steps /= 2;
    const int64_t splits = divide_up(all, steps * kShrinkWaves);
    return divide_up(all, splits * kShrinkWaves);            // evenly
  }
  static int64_t splits(int64_t steps, int64_t width) { return divide_up(divide_up(width, 32), steps * kShrinkWaves); }
  Layout(const nvfp4_adapters_params &p, bool backward) {
    few = !backward && p.tokens <= kFewTokens;
    whole = p.tokens <= kWholeTokens;
    tiles = p.tokens / kTile + (p.adapters + 1 < p.tokens ? p.adapters + 1 : p.tokens);
    steps_in = shrink_steps(p.tokens, few, p.inp, p.rank, false);
    steps_out = shrink_steps(p.tokens, few, p.out, p.rank, true);
    splits_in = splits(steps_in, p.inp);
    splits_out = splits(steps_out, p.out);
    const int64_t chunks = divide_up(p.inp, kOuterWidth) + divide_up(p.out, kOuterWidth);
    ranges = divide_up(512, chunks);
    range_tiles = divide_up(tiles, ranges);
    if (range_tiles < 4) range_tiles = 4;        // (a tile for each wave)
    ranges = tiles ? divide_up(tiles, range_tiles) : 1;
    int64_t end = 0;
    const auto take = [&](int64_t n) {
      const int64_t begin = end;
      end += divide_up(n, 256) * 256;
      return begin;
    };
    count = take(4);
    if (!few) {
      tile_begin = take((p.adapters + 2) * 4);
      order = take(tiles * kTile * 4);
      table = take(tiles * (int64_t)sizeof(Tile));
    }
    parts = take((backward ? splits_out : splits_in) * p.tokens * pitch(p) * 4);
    if (backward) {
      terms_a = take(tiles * 3 * term_ranks(p) * kTile * 2);
      terms_b = take(tiles * 3 * term_ranks(p) * kTile * 2);
      parted_a = take(whole ? 0 : 2 * ranges * p.rank * p.inp * 4);
      parted_b = take(whole ? 0 : 2 * ranges * p.rank * p.out * 4);
    }
    bytes = end;
  }
  static int64_t pitch(const nvfp4_adapters_params &p) { return divide_up(p.rank, 8) * 8; }
  static int64_t term_ranks(const nvfp4_adapters_params &p) { return p.rank <= 16 ? 16 : p.rank <= 32 ? 32 : p.rank <= 64 ? 64 : 128; }
  Plan plan(char *w) const {
    return {reinterpret_cast<int32_t *>(w + count), reinterpret_cast<int32_t *>(w + tile_begin), reinterpret_cast<Tile *>(w + table),
            reinterpret_cast<int32_t *>(w + order)};
  }
};

// LDS words of k_plan
constexpr size_t plan_words(int64_t adapters) { return 16 * (size_t)(adapters + 2) + (size_t)(adapters + 2) + (size_t)(adapters + 1); }

int run_plan(const nvfp4_adapters_params &p, const Layout &d, char *w, const int32_t *which, hipStream_t s) {
  const size_t bytes = plan_words(p.adapters) * 4, most = plan_words(kMostAdapters) * 4;
  if (bytes > 48 * 1024 &&
      hipFuncSetAttribute(reinterpret_cast<const void *>(k_plan), hipFuncAttributeMaxDynamicSharedMemorySize, (int)most) != hipSuccess)
    return NVFP4_ERR_HIP;
  return launch(k_plan, dim3(1), dim3(kPlanThreads), bytes, s, PlanArgs{which, d.plan(w), (int32_t)p.tokens, (int32_t)p.adapters});
}

template <bool ACROSS, int RT, int NF>
int run_shrink_of(ShrinkArgs g, const Layout &d, int64_t splits, hipStream_t s) {
  g.splits = (int32_t)splits;
  if (d.few)                                     // (a backward pass has a plan)
    return launch(k_shrink<!ACROSS, ACROSS, RT, NF>, dim3((uint32_t)g.tokens.T, (uint32_t)splits), dim3(kShrinkWaves * 64), 0, s, g);
  // two workgroups a compute unit where registers allow it
  const int64_t most = divide_up(RT * NF <= 8 ? 512 : 256, splits);
  g.single = 2 * d.tiles <= most;
  const dim3 grid((uint32_t)(g.single ? 2 * d.tiles : most), (uint32_t)(splits + (g.terms_of ? 1 : 0)));
  return launch(k_shrink<false, ACROSS, RT, NF>, grid, dim3(kShrinkWaves * 64), 0, s, g);
}
template <bool ACROSS, int RT>
int run_shrink_of(const ShrinkArgs &g, const Layout &d, int64_t splits, hipStream_t s) {
  if (g.steps <= 2) return run_shrink_of<ACROSS, RT, 2>(g, d, splits, s);
  if constexpr (!ACROSS || RT <= 4)
    if (g.steps <= 4) return run_shrink_of<ACROSS, RT, 4>(g, d, splits, s);
  if constexpr (!ACROSS && RT <= 4) return run_shrink_of<ACROSS, RT, 8>(g, d, splits, s);
  return NVFP4_ERR_UNSUPPORTED;                  // (shrink_steps gives no more)
}
template <bool ACROSS>
int run_shrink(const ShrinkArgs &g, const Layout &d, int64_t splits, hipStream_t s) {
  if (g.rank <= 16) return run_shrink_of<ACROSS, 1>(g, d, splits, s);
  if (g.rank <= 32) return run_shrink_of<ACROSS, 2>(g, d, splits, s);
  if (g.rank <= 64) return run_shrink_of<ACROSS, 4>(g, d, splits, s);
  return run_shrink_of<ACROSS, 8>(g, d, splits, s);
}

template <int LIES, typename T, int F>
int run_expand_of(ExpandArgs g, const Layout &d, hipStream_t s) {
  if (d.few) {
    const dim3 grid((uint32_t)g.tokens.T, (uint32_t)divide_up(g.width, kBlock * 4));
    return launch(k_expand<LIES != kAcross, LIES, T, F>, grid, dim3(256), 0, s, g);             // (a backward pass has a plan)
  }
  constexpr int kWaves = expand_waves<false, T, F>;
  const int64_t across = g.out ? divide_up(g.width, kBlock * kWaves) : 1;
  // (two to four turns of the workgroups that a card holds at once; BF16, 33 to 64 ranks, 16384 tokens: two 147.7 us, two and two thirds 162.6)
  const int64_t most = divide_up(F <= 1 ? 2048 : (F == 2 ? (sizeof(T) == 2 ? 768 : 1024) : 512) * (kWaves == 4 ? 2 : 1), across);
  g.single = d.tiles <= most;
  const dim3 grid((uint32_t)(g.single ? d.tiles : most), (uint32_t)across);
  return launch(k_expand<false, LIES, T, F>, grid, dim3(kWaves * 64), 0, s, g);
}
template <int LIES, typename T>
int run_expand(const ExpandArgs &g, const Layout &d, hipStream_t s) {
  if (g.rank <= 16) return run_expand_of<LIES, T, 0>(g, d, s);
  if (g.rank <= 32) return run_expand_of<LIES, T, 1>(g, d, s);
  if (g.rank <= 64) return run_expand_of<LIES, T, 2>(g, d, s);
  return run_expand_of<LIES, T, 4>(g, d, s);
}
template <typename T>
int run_expand(const ExpandArgs &g, const Layout &d, hipStream_t s) {
  return g.rank % 8 ? run_expand<kRagged, T>(g, d, s) : run_expand<kWhole, T>(g, d, s);
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
  if (!p) return NVFP4_ERR_NULL;
  if (!sizes_fit(*p)) return NVFP4_ERR_SHAPE;    // (first: what has no element, a workspace among it, may well have no address)
  if (!a || !b || !scales || !workspace) return NVFP4_ERR_NULL;
  if (p->tokens != 0 && (!x || !which || !out)) return NVFP4_ERR_NULL;
  if (!stride_fits(p->ld_x, p->inp, p->tokens) || (base && !stride_fits(p->ld_base, p->out, p->tokens)) ||
      !stride_fits(p->ld_out, p->out, p->tokens) || (base == out && p->ld_base != p->ld_out))
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
    if (const int rc = run_plan(*p, d, w, which, s)) return rc;
  const Tokens tokens{which, d.plan(w), (int32_t)p->tokens, (int32_t)p->adapters};
  float *const parts = reinterpret_cast<float *>(w + d.parts);
  const int32_t rank = (int32_t)p->rank, pitch = (int32_t)Layout::pitch(*p);
  ShrinkArgs g{};
  g.tokens = tokens;
  g.x = static_cast<const __bf16 *>(x);
  g.w = static_cast<const __bf16 *>(a);
  g.parts = parts;
  g.h = d.splits_in == 1 ? h : nullptr;
  g.ld = p->ld_x;
  g.width = p->inp;
  g.rank = rank;
  g.pitch = pitch;
  g.steps = (int32_t)d.steps_in;
  if (const int rc = run_shrink<false>(g, d, d.splits_in, s)) return rc;
  const ExpandArgs e{tokens, parts, d.splits_in == 1 ? nullptr : h, nullptr, static_cast<const __bf16 *>(b), scales, base, out,
                     p->ld_base, p->ld_out, p->out, rank, pitch, (int32_t)d.splits_in, 0, false};
  return p->out_dtype == NVFP4_OUT_F32 ? run_expand<float>(e, d, s) : run_expand<__bf16>(e, d, s);
}

extern "C" int nvfp4_adapters_backward(const void *dy, const nvfp4_adapters_params *p, const void *x, const float *h, const void *a,
                                       const void *b, const int32_t *which, const float *scales, const void *dx_base, void *dx,
                                       float *da, float *db, void *workspace, size_t workspace_bytes, void *stream) {
  if (!p) return NVFP4_ERR_NULL;
  if (!sizes_fit(*p)) return NVFP4_ERR_SHAPE;
  if (!a || !b || !scales || !da || !db || !workspace) return NVFP4_ERR_NULL;
  if (p->tokens != 0 && (!dy || !x || !h || !which)) return NVFP4_ERR_NULL;
  if (!stride_fits(p->ld_x, p->inp, p->tokens) || !stride_fits(p->ld_dy, p->out, p->tokens) ||
      (dx && dx_base && !stride_fits(p->ld_base, p->inp, p->tokens)) || (dx && !stride_fits(p->ld_out, p->inp, p->tokens)) ||
      (dx && dx_base == dx && p->ld_base != p->ld_out))
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
  if (const int rc = run_plan(*p, d, w, which, s)) return rc;
  const Tokens tokens{which, d.plan(w), (int32_t)p->tokens, (int32_t)p->adapters};
  float *const parts = reinterpret_cast<float *>(w + d.parts);
  __bf16 *const terms_a = reinterpret_cast<__bf16 *>(w + d.terms_a), *const terms_b = reinterpret_cast<__bf16 *>(w + d.terms_b);
  const int32_t rank = (int32_t)p->rank, pitch = (int32_t)Layout::pitch(*p), term_ranks = (int32_t)Layout::term_ranks(*p);
  const OuterArgs g{d.plan(w), (int32_t)p->adapters, rank, term_ranks, (int32_t)d.range_tiles, d.whole,
                    {{static_cast<const __bf16 *>(x), terms_a, da, reinterpret_cast<float *>(w + d.parted_a), p->ld_x, p->inp,
                      (int32_t)divide_up(p->inp, kOuterWidth), false},
                     {static_cast<const __bf16 *>(dy), terms_b, db, reinterpret_cast<float *>(w + d.parted_b), p->ld_dy, p->out,
                      (int32_t)divide_up(p->out, kOuterWidth), true}}};
  if (any) {
    const ShrinkArgs dh{tokens, static_cast<const __bf16 *>(dy), static_cast<const __bf16 *>(b), parts, nullptr, h, scales,
                        terms_b, p->ld_dy, p->out, rank, pitch, (int32_t)d.steps_out, term_ranks, 0, false};
    if (const int rc = run_shrink<true>(dh, d, d.splits_out, s)) return rc;
    const ExpandArgs e{tokens, parts, nullptr, terms_a, static_cast<const __bf16 *>(a), scales, dx_base, dx,
                       p->ld_base, p->ld_out, p->inp, rank, pitch, (int32_t)d.splits_out, term_ranks, false};
    if (const int rc = run_expand<kAcross, __bf16>(e, d, s)) return rc;
  }
  // A workgroup has up to 64 ranks, which read x and dy once; where its sums go to the output at once, up to 32, since the gradients are
  // much of the bytes then and more workgroups write them.  32 / 64, 4096 x 4096, rank 64: one token 26.1 / 29.1 us, 512 of one adapter
  // 31.6 / 35.0, of 64 adapters 119 / 146; beyond, 8192 tokens of 8 adapters 180 / 173, at 8192 x 8192 328 / 300.
  const int ranks = rank <= 16 ? 16 : rank <= 32 || d.whole ? 32 : 64;
  const dim3 grid((uint32_t)(g.half[0].chunks + g.half[1].chunks), (uint32_t)d.ranges, (uint32_t)divide_up(rank, ranks));
  if (const int rc = launch(ranks == 16 ? k_outer<1> : ranks == 32 ? k_outer<2> : k_outer<4>, grid, dim3(256), 0, s, g)) return rc;
  if (d.whole || d.ranges == 1) return NVFP4_OK;
  const int64_t most = divide_up(p->rank * (p->inp > p->out ? p->inp : p->out), 1024);
  return launch(k_join, dim3((uint32_t)(most < 256 ? most : 256), (uint32_t)p->adapters, 2), dim3(256), 0, s, g);
}
