// Tokens to their experts, and back (include/finetune/nvfp4_finetune.h).
//
//   xs[place[t][j]] = x_t,  y_t = base_t + sum_j w[t][j] ys[place[t][j]],
//   dys[place[t][j]] = w[t][j] dy_t,  dw[t][j] = <dy_t, ys[place[t][j]]>
//
// All of it is bound by the bytes of the rows.  Every kernel goes by tokens: a token's row is read once and written to all its places
// (or is summed from them, in the order of j), so nothing is added atomically and a row of 16 bytes or more per lane is whole lines of memory
// wherever it stands.
//
//   k_sort_count, k_sort    pairs in the order of their experts (stable)
//   k_spread                x to its places
//   k_combine               weighted sums of places
//   k_combine_backward      both gradients, ys read once
//
// Among others, 16384 tokens of 4096 columns, four experts each, BF16: sort 11 us (two launches), spread 128 (671 MB: 5.2 TB/s, a copy 5.1), combine 131 to 140
// (779 MB: 5.6 to 5.9); gradients of 5001 x 2880, eight each, 93 (479 MB); back from 5001 x 2880 fp32, six each, 82 (386 MB).  64 tokens: sort 4 us, spread 3.5,
// the two calls 7.8 to 9.7 (the host's part of them as long); 64 tokens of 4096 columns, eight each: combine 4.1, its gradients 9.9 (one place after the other);
// gradients of 8192 tokens of 64 columns, eight each, 13.9.
#include <hip/hip_runtime.h>

#include "finetune/nvfp4_finetune.h"
#include "launch.hpp"

namespace nvfp4_46 {
namespace {

constexpr int64_t kMostTokens = (1 << 24) - 1, kMostWidth = 1 << 22, kMostTop = 64, kMostExperts = 1024, kMostPairs = (int64_t)1 << 30;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kHeld = 4;                        // steps of 64 pairs that a wave keeps in registers
constexpr int64_t kSortOne = 4096;              // pairs that one workgroup sorts by itself
constexpr int64_t kSortBlocks = 128;            // ... and of more pairs at most so many workgroups

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// ---- eight adjacent columns ---------------------------------------------------------------------------------------------

template <typename T>
struct Piece;
template <>
struct Piece<__bf16> {
  bf16x8 v;
  template <bool PAST = false>
  __device__ void load(const __bf16 *p) {
    const auto *const q = reinterpret_cast<const bf16x8 *>(p);
    if constexpr (PAST) v = __builtin_nontemporal_load(q);
    else v = *q;
  }
  template <bool PAST = false>
  __device__ void store(__bf16 *p) const {
    auto *const q = reinterpret_cast<bf16x8 *>(p);
    if constexpr (PAST) __builtin_nontemporal_store(v, q);
    else *q = v;
  }
  __device__ f32x8 wide() const { return __builtin_convertvector(v, f32x8); }
  __device__ void round(f32x8 f) { v = __builtin_convertvector(f, bf16x8); }
};
template <>
struct Piece<float> {
  f32x4 lo, hi;
  template <bool PAST = false>
  __device__ void load(const float *p) {
    const auto *const q = reinterpret_cast<const f32x4 *>(p);
    if constexpr (PAST) lo = __builtin_nontemporal_load(q), hi = __builtin_nontemporal_load(q + 1);
    else lo = q[0], hi = q[1];
  }
  template <bool PAST = false>
  __device__ void store(float *p) const {
    auto *const q = reinterpret_cast<f32x4 *>(p);
    if constexpr (PAST) __builtin_nontemporal_store(lo, q), __builtin_nontemporal_store(hi, q + 1);
    else q[0] = lo, q[1] = hi;
  }
  __device__ f32x8 wide() const { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
  __device__ void round(f32x8 f) {
    lo = __builtin_shufflevector(f, f, 0, 1, 2, 3);
    hi = __builtin_shufflevector(f, f, 4, 5, 6, 7);
  }
};
// (the same type: as it is, every bit of a NaN too)
template <typename T>
__device__ inline void convert(Piece<T> &to, const Piece<T> &from) { to = from; }
__device__ inline void convert(Piece<float> &to, const Piece<__bf16> &from) { to.round(from.wide()); }
__device__ inline void convert(Piece<__bf16> &to, const Piece<float> &from) { to.round(from.wide()); }

// ---- sort ---------------------------------------------------------------------------------------------------------------

struct SortArgs {
  const void *ids;
  int32_t *counts;             // [workgroups][experts + 1], where there is more than one
  int32_t *place, *token, *begin;
  int32_t pairs, top, experts;
  int32_t per;                 // pairs of a workgroup
  bool wide;                   // ids are 64 bits
};

// The group of a pair: its expert, `experts` for none.
__device__ inline int32_t group_of(const SortArgs &a, int32_t pair) {
  if (a.wide) {
    const int64_t id = static_cast<const int64_t *>(a.ids)[pair];
    return id >= 0 && id < a.experts ? (int32_t)id : a.experts;
  }
  const int32_t id = static_cast<const int32_t *>(a.ids)[pair];
  return id >= 0 && id < a.experts ? id : a.experts;
}

// How many pairs of its stretch every group has, of each workgroup.
__global__ void __launch_bounds__(kSortThreads) k_sort_count(SortArgs a) {
  __shared__ int32_t count[kMostExperts + 1];
  const int32_t groups = a.experts + 1, first = (int32_t)blockIdx.x * a.per;
  const int32_t last = a.pairs - first < a.per ? a.pairs : first + a.per;
  for (int32_t g = threadIdx.x; g < groups; g += kSortThreads) count[g] = 0;
  __syncthreads();
  for (int32_t i = first + (int32_t)threadIdx.x; i < last; i += kSortThreads) atomicAdd(&count[group_of(a, i)], 1);
  __syncthreads();
  for (int32_t g = threadIdx.x; g < groups; g += kSortThreads) a.counts[(int64_t)blockIdx.x * groups + g] = count[g];
}

// Stable counting sort, bound by turns to memory one after the other: 256 pairs 3.9 us, 65536 4.7 for the counts and 6.5.  A wave has an adjacent part of
// its workgroup's stretch, 64 pairs at a time: how many of each group (pass 0), then, from where the group's first pair of the wave goes, every
// pair's place (pass 1).
__global__ void __launch_bounds__(kSortThreads) k_sort(SortArgs a) {
  extern __shared__ int32_t counts[];            // [16][line]: each wave's pairs of a group, then where the next of them goes
  const int32_t groups = a.experts + 1, line = groups + 1;
  int32_t *const prior = counts + kSortWaves * line, *const total = prior + groups;      // pairs of earlier workgroups, of all
  __shared__ int32_t sums[kSortWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  int32_t *const mine = counts + wave * line;
  for (int32_t i = threadIdx.x; i < kSortWaves * line + 2 * groups; i += kSortThreads) counts[i] = 0;
  __syncthreads();
  const int32_t first = (int32_t)blockIdx.x * a.per, stop = a.pairs - first < a.per ? a.pairs : first + a.per;
  const int32_t slice = a.per / kSortWaves, begin = first + wave * slice;
  const int32_t end = stop - begin < slice ? stop : begin + slice;        // (of a wave past the stretch: before its begin)
  // the lanes with this lane's group
  const auto alike = [&](int32_t l) {
    uint64_t m = ~(uint64_t)0;
    for (int32_t bit = 1; bit <= groups; bit <<= 1) {
      const uint64_t set = __ballot((l & bit) != 0);
      m &= l & bit ? set : ~set;
    }
    return m;
  };
  const auto load = [&](int32_t i) { return i < end ? group_of(a, i) : groups; };         // (past the end: a group of its own, which nobody reads)
  int32_t held[kHeld];                           // the first ones, for both passes
#pragma unroll
  for (int n = 0; n < kHeld; ++n) held[n] = load(begin + n * 64 + lane);
  for (int pass = 0; pass < 2; ++pass) {
    const auto take = [&](int32_t i0, int32_t l) __attribute__((always_inline)) {
      const int32_t i = i0 + lane;
      const uint64_t m = alike(l);
      const int32_t before = __popcll(m & (((uint64_t)1 << lane) - 1));
      // A wave's LDS instructions run in their order, so the lanes have all read before the first of each group adds; the fences keep
      // the compiler to it.
      if (pass == 1) {
        const int32_t at = mine[l] + before;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (i < end) {
          const bool is = l < a.experts;
          a.place[i] = is ? at : ~at;
          a.token[at] = is ? (int32_t)((uint32_t)i / (uint32_t)a.top) : -1;
        }
      }
      if (before == 0) __hip_atomic_fetch_add(mine + l, __popcll(m), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
#pragma unroll
    for (int n = 0; n < kHeld; ++n)
      if (begin + n * 64 < end) take(begin + n * 64, held[n]);
    for (int32_t i0 = begin + kHeld * 64; i0 < end; i0 += 64) take(i0, load(i0 + lane));
    if (pass == 1) break;
    if (gridDim.x > 1) {
      // (as many threads to a group as there are; whole numbers, whose sums do not depend on their order)
      const int32_t parts = groups < kSortThreads ? kSortThreads / groups : 1;
      for (int32_t i = threadIdx.x; i < parts * groups; i += kSortThreads) {
        const int32_t g = i % groups;
        int32_t before = 0, all = 0;
        for (int32_t b = i / groups; b < (int32_t)gridDim.x; b += parts) {
          const int32_t n = a.counts[(int64_t)b * groups + g];
          all += n;
          before += b < (int32_t)blockIdx.x ? n : 0;
        }
        atomicAdd(prior + g, before);
        atomicAdd(total + g, all);
      }
    }
    __syncthreads();
    // the groups one after the other, in each the workgroups', in each the waves' pairs: a thread has adjacent groups
    const int32_t per = (groups + kSortThreads - 1) / kSortThreads, g0 = (int32_t)threadIdx.x * per;
    int32_t here = 0;
    for (int32_t g = g0; g < g0 + per && g < groups; ++g) {
      int32_t n = 0;
      for (int w = 0; w < kSortWaves; ++w) {
        const int32_t of = counts[w * line + g];
        counts[w * line + g] = n;
        n += of;
      }
      if (gridDim.x == 1) total[g] = n;
      here += total[g];
    }
    int32_t upto = here;
    for (int d = 1; d < 64; d <<= 1) {
      const int32_t other = __shfl_up(upto, d);
      if (lane >= d) upto += other;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int32_t at = upto - here;
    for (int w = 0; w < wave; ++w) at += sums[w];
    for (int32_t g = g0; g < g0 + per && g < groups; ++g) {
      for (int w = 0; w < kSortWaves; ++w) counts[w * line + g] += at + prior[g];
      if (blockIdx.x == 0) a.begin[g] = at;      // (of the group without an expert: the end of the last expert's)
      at += total[g];
    }
    __syncthreads();
  }
}

// ---- spread -------------------------------------------------------------------------------------------------------------

struct RowArgs {
  const void *token_rows;      // x, base, dy
  void *token_out;             // y
  const void *slot_rows;       // ys
  void *slot_out;              // xs, dys
  const int32_t *place;
  const float *weights;
  float *dweights;
  int64_t ld_token, ld_base, ld_slot, ld_dslot;
  int32_t tokens, top, pieces; // pieces of eight columns to a row
  int32_t slots;
  int32_t lanes;               // to a token: 64 / lanes tokens share a wave where rows are short
};

constexpr int kRowThreads = 256;

// Where a lane works: its token and its first piece; the next ones are `lanes` further on.
struct Spot {
  int32_t token, piece;
};
template <int U>
__device__ inline Spot spot_of(const RowArgs &a) {
  const int32_t in = (int32_t)threadIdx.x & (a.lanes - 1), of = (int32_t)threadIdx.x / a.lanes;
  return {(int32_t)blockIdx.x * (kRowThreads / a.lanes) + of, (int32_t)blockIdx.y * (a.lanes * U) + in};
}

// Bound by its stores.  A wave holds up to 64 U pieces of a token's row and writes them to one place after the other; a pair without an expert has a slot
// of its own too, which its wave clears, so that no slot is left out and none written twice.
template <typename TI, typename TO, int U, bool PAST>
__global__ void __launch_bounds__(kRowThreads) k_spread(RowArgs a) {
  const Spot at = spot_of<U>(a);
  if (at.token >= a.tokens) return;
  const TI *const x = static_cast<const TI *>(a.token_rows) + (int64_t)at.token * a.ld_token;
  Piece<TO> v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int32_t piece = at.piece + u * a.lanes;
    Piece<TI> in;
    if (piece < a.pieces) {
      in.load(x + (int64_t)piece * 8);
      convert(v[u], in);
    }
  }
  const int32_t *const place = a.place + (int64_t)at.token * a.top;
  for (int32_t j = 0; j < a.top; ++j) {
    const int32_t p = place[j], slot = p < 0 ? ~p : p;
    if (slot >= a.slots) continue;
    TO *const to = static_cast<TO *>(a.slot_out) + (int64_t)slot * a.ld_slot;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t piece = at.piece + u * a.lanes;
      if (piece >= a.pieces) continue;
      Piece<TO> out = v[u];
      if (p < 0) out.round(f32x8{});
      out.template store<PAST>(to + (int64_t)piece * 8);
    }
  }
}

// ---- combine ------------------------------------------------------------------------------------------------------------

constexpr int kAhead = 4;                        // places whose rows are on their way at once

// Bound by its loads: the pieces of four places are on their way together (place by place, and through the caches, 16384 x 4096 took 178 us instead of
// 132).  Slots of pairs without an expert are not read.
template <typename TS, typename TT, int U, bool PAST>
__global__ void __launch_bounds__(kRowThreads) k_combine(RowArgs a) {
  const Spot at = spot_of<U>(a);
  if (at.token >= a.tokens) return;
  f32x8 sum[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int32_t piece = at.piece + u * a.lanes;
    sum[u] = f32x8{};
    if (a.token_rows && piece < a.pieces) {
      Piece<TT> base;
      base.load(static_cast<const TT *>(a.token_rows) + (int64_t)at.token * a.ld_base + (int64_t)piece * 8);
      sum[u] = base.wide();
    }
  }
  const int32_t *const place = a.place + (int64_t)at.token * a.top;
  const float *const weights = a.weights ? a.weights + (int64_t)at.token * a.top : nullptr;
  for (int32_t j0 = 0; j0 < a.top; j0 += kAhead) {
    int32_t p[kAhead];
    float w[kAhead];
    Piece<TS> in[kAhead][U];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      p[i] = j0 + i < a.top ? place[j0 + i] : -1;
      w[i] = weights && j0 + i < a.top ? weights[j0 + i] : 1.0f;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (p[i] < 0 || p[i] >= a.slots) continue;
      const TS *const from = static_cast<const TS *>(a.slot_rows) + (int64_t)p[i] * a.ld_slot;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at.piece + u * a.lanes < a.pieces) in[i][u].template load<PAST>(from + (int64_t)(at.piece + u * a.lanes) * 8);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (p[i] < 0 || p[i] >= a.slots) continue;
#pragma unroll
      for (int u = 0; u < U; ++u) sum[u] += w[i] * in[i][u].wide();
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int32_t piece = at.piece + u * a.lanes;
    if (piece >= a.pieces) continue;
    Piece<TT> out;
    out.round(sum[u]);
    out.store(static_cast<TT *>(a.token_out) + (int64_t)at.token * a.ld_token + (int64_t)piece * 8);
  }
}

// WAVES waves have a token, each P pieces a lane at a time, and keep those of dy while they go through the places; a row of more pieces than that is
// gone through again and again.  (ys may be dys: an element is read before the same lane writes it.)
template <typename TS, typename TT, int WAVES, int P, bool PAST>
__global__ void __launch_bounds__(kRowThreads) k_combine_backward(RowArgs a) {
  constexpr int kTokens = kRowThreads / 64 / WAVES, kLanes = 64 * WAVES;
  __shared__ float part[2][kTokens][WAVES];
  const int32_t in = (int32_t)threadIdx.x % kLanes, of = (int32_t)threadIdx.x / kLanes, wave = __builtin_amdgcn_readfirstlane(in / 64);
  const int32_t token = __builtin_amdgcn_readfirstlane((int32_t)blockIdx.x * kTokens + of);
  const bool is_token = token < a.tokens;
  if (WAVES == 1 && !is_token) return;           // (no barriers)
  const TT *const dy = static_cast<const TT *>(a.token_rows) + (int64_t)token * a.ld_token;
  Piece<TT> held[P];
  const auto fetch = [&](int32_t first) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (is_token && first + i * kLanes < a.pieces) held[i].load(dy + (int64_t)(first + i * kLanes) * 8);
  };
  fetch(in);
  const bool whole = a.pieces <= P * kLanes;
  for (int32_t j = 0; j < a.top; ++j) {
    const int32_t p = is_token ? a.place[(int64_t)token * a.top + j] : 0, slot = p < 0 ? ~p : p;
    const bool there = is_token && slot < a.slots, is = there && p >= 0;
    const float w = is ? a.weights[(int64_t)token * a.top + j] : 0.0f;
    const TS *const ys = static_cast<const TS *>(a.slot_rows) + (int64_t)slot * a.ld_slot;
    TS *const dys = static_cast<TS *>(a.slot_out) + (int64_t)slot * a.ld_dslot;
    float dot = 0.0f;
    for (int32_t first = in; there && first < a.pieces; first += P * kLanes) {
      if (!whole) fetch(first);
      Piece<TS> y[P];
      if (is) {
#pragma unroll
        for (int i = 0; i < P; ++i)
          if (first + i * kLanes < a.pieces) y[i].template load<PAST>(ys + (int64_t)(first + i * kLanes) * 8);
      }
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (first + i * kLanes >= a.pieces) continue;
        Piece<TS> out;
        if (is) {
          const f32x8 dv = held[i].wide(), yv = y[i].wide();
          for (int k = 0; k < 8; ++k) dot += dv[k] * yv[k];
          out.round(w * dv);
        } else {
          out.round(f32x8{});
        }
        out.template store<PAST>(dys + (int64_t)(first + i * kLanes) * 8);
      }
    }
    for (int d = 32; d > 0; d >>= 1) dot += __shfl_xor(dot, d);
    if constexpr (WAVES > 1) {
      float(*const mine)[WAVES] = part[j & 1];   // (read again only behind the next place's barrier)
      if (in % 64 == 0) mine[of][wave] = dot;
      __syncthreads();
      dot = 0.0f;
      for (int i = 0; i < WAVES; ++i) dot += mine[of][i];
    }
    if (is_token && in == 0) a.dweights[(int64_t)token * a.top + j] = is ? dot : 0.0f;
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------

int64_t divide_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool at(const void *ptr, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }
bool pairs_fit(const nvfp4_experts_params &p) {
  return p.tokens >= 0 && p.tokens <= kMostTokens && p.top > 0 && p.top <= kMostTop && p.tokens * p.top <= kMostPairs;
}
bool sort_fits(const nvfp4_experts_params &p) { return pairs_fit(p) && p.experts > 0 && p.experts <= kMostExperts; }
bool width_fits(const nvfp4_experts_params &p) { return pairs_fit(p) && p.width > 0 && p.width <= kMostWidth && p.width % 8 == 0; }
bool stride_fits(int64_t ld, int64_t width, int64_t rows) {
  return ld >= width && ld <= ((int64_t)1 << 40) / (rows > 0 ? rows : 1);
}
bool types_fit(const nvfp4_experts_params &p) { return p.token_dtype <= NVFP4_X_F32 && p.slot_dtype <= NVFP4_X_F32; }

int64_t sort_blocks(const nvfp4_experts_params &p) {
  const int64_t pairs = p.tokens * p.top;
  if (pairs <= kSortOne) return 1;
  const int64_t blocks = divide_up(pairs, kSortThreads);
  return blocks < kSortBlocks ? blocks : kSortBlocks;
}
int64_t sort_bytes(const nvfp4_experts_params &p) {
  const int64_t blocks = sort_blocks(p);
  return blocks == 1 ? 16 : divide_up(blocks * (p.experts + 1) * 4, 16) * 16;
}
constexpr size_t sort_lds(int64_t experts) { return (kSortWaves * (experts + 2) + 2 * (experts + 1)) * 4; }

// Tokens across, columns down: lanes to a token, and the grid for U pieces a lane.
template <int U>
dim3 row_grid(RowArgs &a) {
  int32_t lanes = 1;
  while (lanes < 64 && lanes < a.pieces) lanes *= 2;
  a.lanes = lanes;
  return dim3((uint32_t)divide_up(a.tokens, kRowThreads / lanes), (uint32_t)divide_up(a.pieces, lanes * U));
}

// More rows of slots than the caches keep are written, and read for the last time, past them.  BF16, us, through / past: spread 33.5 / 35.7 for 134 MB,
// 66 / 61 for 262, 139 / 118 for 537; combine 38.6 / 34.1 for 134 MB, 49 / 43 for 131 of two places a token, 149 / 131 for 537 (fp32 80 / 82
// for 346); gradients 50 / 55 for 134 MB, 94.4 / 93.7 for 230, 114 / 105 for 268.
bool past_caches(const nvfp4_experts_params &p, int64_t mbytes) {
  return p.tokens * p.top * p.width * (p.slot_dtype == NVFP4_X_F32 ? 4 : 2) > mbytes << 20;
}
// Four pieces a lane where that leaves eight waves for each compute unit (us, one / two / four: spread of 16384 x 4096, past the caches, 139 / 141 / 118,
// combine 150 / 157 / 131), else one (1000 tokens, 2048 columns, combine 5.8 / 6.1 / 7.0).
bool many(const nvfp4_experts_params &p) { return p.tokens * divide_up(p.width, 8 * 64 * 4) >= 2048; }

// kernel<types of slots and tokens> for the types of a call
template <typename F>
int by_types(const nvfp4_experts_params &p, F f) {
  const bool s = p.slot_dtype == NVFP4_X_F32, t = p.token_dtype == NVFP4_X_F32;
  return s ? t ? f(float{}, float{}) : f(float{}, __bf16{}) : t ? f(__bf16{}, float{}) : f(__bf16{}, __bf16{});
}

RowArgs row_args(const nvfp4_experts_params &p, const int32_t *place) {
  RowArgs a{};
  a.place = place;
  a.ld_token = p.ld_token;
  a.ld_base = p.ld_base;
  a.ld_slot = p.ld_slot;
  a.ld_dslot = p.ld_dslot;
  a.tokens = (int32_t)p.tokens;
  a.top = (int32_t)p.top;
  a.pieces = (int32_t)(p.width / 8);
  a.slots = (int32_t)(p.tokens * p.top);
  return a;
}

}  // namespace
}  // namespace nvfp4_46

using namespace nvfp4_46;

extern "C" size_t nvfp4_experts_workspace_bytes(const nvfp4_experts_params *p) {
  return p && sort_fits(*p) ? (size_t)sort_bytes(*p) : 0;
}

extern "C" int nvfp4_experts_sort(const void *ids, const nvfp4_experts_params *p, int32_t *place, int32_t *token, int32_t *begin,
                                  void *workspace, size_t workspace_bytes, void *stream) {
  if (!p) return NVFP4_ERR_NULL;
  if (!sort_fits(*p)) return NVFP4_ERR_SHAPE;
  if (!begin || !workspace || (p->tokens != 0 && (!ids || !place || !token))) return NVFP4_ERR_NULL;
  if (p->index_dtype > NVFP4_INDEX_I64) return NVFP4_ERR_PARAM;
  if (!at(ids, p->index_dtype == NVFP4_INDEX_I64 ? 8 : 4) || !at(place, 4) || !at(token, 4) || !at(begin, 4) || !at(workspace, 16))
    return NVFP4_ERR_ALIGN;
  if (workspace_bytes < (size_t)sort_bytes(*p)) return NVFP4_ERR_PARAM;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t pairs = p->tokens * p->top, blocks = sort_blocks(*p);
  // (whole steps of 64 pairs for each wave)
  const int64_t per = pairs ? divide_up(divide_up(pairs, blocks), kSortThreads) * kSortThreads : kSortThreads;
  const int64_t used = pairs ? divide_up(pairs, per) : 1;
  const SortArgs a{ids, static_cast<int32_t *>(workspace), place, token, begin, (int32_t)pairs, (int32_t)p->top,
                   (int32_t)p->experts, (int32_t)per, p->index_dtype == NVFP4_INDEX_I64};
  if (used > 1)
    if (const int rc = launch(k_sort_count, dim3((uint32_t)used), dim3(kSortThreads), 0, s, a)) return rc;
  const size_t bytes = sort_lds(p->experts);
  // (the limit belongs to the kernel and not to the call, so it is always the same)
  if (bytes > 48 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(k_sort), hipFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)sort_lds(kMostExperts)) != hipSuccess)
    return NVFP4_ERR_HIP;
  return launch(k_sort, dim3((uint32_t)used), dim3(kSortThreads), bytes, s, a);
}

extern "C" int nvfp4_experts_spread(const void *x, const nvfp4_experts_params *p, const int32_t *place, void *xs, void *stream) {
  if (!p) return NVFP4_ERR_NULL;
  if (!width_fits(*p)) return NVFP4_ERR_SHAPE;
  if (p->tokens != 0 && (!x || !place || !xs)) return NVFP4_ERR_NULL;
  if (!stride_fits(p->ld_token, p->width, p->tokens) || !stride_fits(p->ld_slot, p->width, p->tokens * p->top)) return NVFP4_ERR_SHAPE;
  if (!at(x, 16) || !at(xs, 16) || !at(place, 4) || p->ld_token % 8 || p->ld_slot % 8) return NVFP4_ERR_ALIGN;
  if (!types_fit(*p)) return NVFP4_ERR_PARAM;
  if (p->tokens == 0) return NVFP4_OK;
  RowArgs a = row_args(*p, place);
  a.token_rows = x;
  a.slot_out = xs;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return by_types(*p, [&](auto slot, auto token) {
    typedef decltype(slot) TO;
    typedef decltype(token) TI;
    const bool four = many(*p), past = four && past_caches(*p, 192);
    const dim3 grid = four ? row_grid<4>(a) : row_grid<1>(a);
    return launch(past ? k_spread<TI, TO, 4, true> : four ? k_spread<TI, TO, 4, false> : k_spread<TI, TO, 1, false>, grid, dim3(kRowThreads), 0, s, a);
  });
}

extern "C" int nvfp4_experts_combine(const void *ys, const nvfp4_experts_params *p, const int32_t *place, const float *weights,
                                     const void *base, void *y, void *stream) {
  if (!p) return NVFP4_ERR_NULL;
  if (!width_fits(*p)) return NVFP4_ERR_SHAPE;
  if (p->tokens != 0 && (!ys || !place || !y)) return NVFP4_ERR_NULL;
  if (!stride_fits(p->ld_token, p->width, p->tokens) || !stride_fits(p->ld_slot, p->width, p->tokens * p->top) ||
      (base && !stride_fits(p->ld_base, p->width, p->tokens)) || (base && base == y && p->ld_base != p->ld_token))
    return NVFP4_ERR_SHAPE;
  if (!at(ys, 16) || !at(y, 16) || !at(base, 16) || !at(place, 4) || !at(weights, 4) || p->ld_token % 8 || p->ld_slot % 8 ||
      (base && p->ld_base % 8))
    return NVFP4_ERR_ALIGN;
  if (!types_fit(*p)) return NVFP4_ERR_PARAM;
  if (p->tokens == 0) return NVFP4_OK;
  RowArgs a = row_args(*p, place);
  a.token_rows = base;
  a.token_out = y;
  a.slot_rows = ys;
  a.weights = weights;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return by_types(*p, [&](auto slot, auto token) {
    typedef decltype(slot) TS;
    typedef decltype(token) TT;
    const bool four = many(*p), past = four && past_caches(*p, 96);
    const dim3 grid = four ? row_grid<4>(a) : row_grid<1>(a);
    return launch(past ? k_combine<TS, TT, 4, true> : four ? k_combine<TS, TT, 4, false> : k_combine<TS, TT, 1, false>, grid, dim3(kRowThreads), 0, s,
                  a);
  });
}

extern "C" int nvfp4_experts_combine_backward(const void *dy, const nvfp4_experts_params *p, const void *ys, const int32_t *place,
                                              const float *weights, void *dys, float *dweights, void *stream) {
  if (!p) return NVFP4_ERR_NULL;
  if (!width_fits(*p)) return NVFP4_ERR_SHAPE;
  if (p->tokens != 0 && (!dy || !ys || !place || !weights || !dys || !dweights)) return NVFP4_ERR_NULL;
  if (!stride_fits(p->ld_token, p->width, p->tokens) || !stride_fits(p->ld_slot, p->width, p->tokens * p->top) ||
      !stride_fits(p->ld_dslot, p->width, p->tokens * p->top) || (ys && ys == dys && p->ld_slot != p->ld_dslot))
    return NVFP4_ERR_SHAPE;
  if (!at(dy, 16) || !at(ys, 16) || !at(dys, 16) || !at(place, 4) || !at(weights, 4) || !at(dweights, 4) || p->ld_token % 8 ||
      p->ld_slot % 8 || p->ld_dslot % 8)
    return NVFP4_ERR_ALIGN;
  if (!types_fit(*p)) return NVFP4_ERR_PARAM;
  if (p->tokens == 0) return NVFP4_OK;
  RowArgs a = row_args(*p, place);
  a.token_rows = dy;
  a.slot_rows = ys;
  a.slot_out = dys;
  a.weights = weights;
  a.dweights = dweights;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return by_types(*p, [&](auto slot, auto token) {
    typedef decltype(slot) TS;
    typedef decltype(token) TT;
    const auto run = [&](auto kernel, int tokens) { return launch(kernel, dim3((uint32_t)divide_up(a.tokens, tokens)), dim3(kRowThreads), 0, s, a); };
    // (two waves a token for short rows, us, two / four waves: 4000 x 1024 12.4 / 15.4, 1000 x 2048 8.8 / 8.6, 4096 x 4096 50 / 50, 5001 x 2880 99.8 / 94.4)
    if (a.pieces <= 64) return run(k_combine_backward<TS, TT, 1, 1, false>, 4);
    if (a.pieces <= 256) return run(k_combine_backward<TS, TT, 2, 2, false>, 2);
    return past_caches(*p, 192) ? run(k_combine_backward<TS, TT, 4, 2, true>, 1) : run(k_combine_backward<TS, TT, 4, 2, false>, 1);
  });
}
