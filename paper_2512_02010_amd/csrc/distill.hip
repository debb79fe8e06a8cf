// Distillation from a teacher's top logits (include/finetune/nvfp4_finetune.h): loss, gradient, and both in one pass.
//
// Per row y = z / temperature, lse = log sum exp y, p = softmax(teacher / temperature) over the list:
//   loss = sum_j p_j (log p_j - (y_{i_j} - lse)),   dz_v = w / temperature (exp(y_v - lse) - sum_{j: i_j = v} p_j).
// All of it is bound by the bytes of the logits: a row is read once for its maximum and sum together (the sum is rescaled when
// the maximum grows), and the list, which is short, is dealt with by the first wave while the others stream.  Sums, maxima, the list's
// probabilities and the loss are fp32; only the gradient is rounded to the logits' type, once.
//
// Whole calls, among others (a copy of as many bytes: 5.1 TB/s): loss of 4096 x 50021 BF16 76 us (5.4 TB/s, read only); gradient of 2047 x 50021
// BF16 93 us (4.4), of 1024 x 32768 fp32 44 to 58 (4.6 to 6, by what the caches hold); step of 4096 x 131072 BF16 460 us (4.7), of 255 x 50021
// fp32 22 us (4.7).  A row or a few: 5 to 7 us a call, the launch's own; a step of one row of 131072, which one workgroup takes, 19.
#include <hip/hip_runtime.h>

#include <cmath>

#include "finetune/nvfp4_finetune.h"
#include "launch.hpp"

namespace nvfp4_46 {
namespace {

constexpr int kMostTop = 1024;
constexpr int64_t kMostRows = 1 << 21;        // (a workgroup of 1024 each: a grid has fewer than 2^32 threads)
constexpr float kInf = __builtin_inff();
constexpr float kLeastTemperature = 0x1p-126f;      // (a little below half of it, log2(e) / temperature is infinite)

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct DistillArgs {
  const void *logits;
  void *dlogits;
  const void *teacher, *index;
  const float *lse_in, *weight;
  float *loss, *lse;
  int64_t ld;
  int32_t vocab, top;
  float c, inv_t;              // log2(e) / temperature and 1 / temperature
  uint32_t teacher_f32, index_wide;
};

// ---- rows in pieces of 16 bytes --------------------------------------------------------------------------------
// A row begins anywhere (its length may be odd): pieces are cut at multiples of 16 bytes of the address.  What lies before the first and
// after the last whole piece, fewer than a piece's elements each, are the row's edges: a thread takes one of them by itself.

__device__ inline float up(uint32_t w, int i) { return __uint_as_float(i ? w & 0xffff0000u : w << 16); }

template <typename T>
__device__ inline void unpack(u32x4 w, float *x) {
  if constexpr (sizeof(T) == 4) {
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  } else {
    for (int i = 0; i < 8; ++i) x[i] = up(w[i / 2], i % 2);
  }
}
template <typename T>
__device__ inline u32x4 pack(const float *x) {
  u32x4 w;
  if constexpr (sizeof(T) == 4) {
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[i]);
  } else {
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
  }
  return w;
}
template <typename T>
__device__ inline float element(const void *p, int64_t i) {
  if constexpr (sizeof(T) == 4) return static_cast<const float *>(p)[i];
  return __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
}
template <typename T>
__device__ inline void set_element(void *p, int64_t i, float x) {
  if constexpr (sizeof(T) == 4)
    static_cast<float *>(p)[i] = x;
  else
    static_cast<__bf16 *>(p)[i] = (__bf16)x;
}

// What goes past the caches (past_caches).
enum { kThrough, kLoads, kBoth };

template <typename T>
struct Row {
  static constexpr int kPer = 16 / sizeof(T);
  char *at;                    // the first whole piece
  int32_t pieces;              // whole ones
  int32_t before, after;       // elements on either edge
  __device__ Row(const void *base, int64_t row, int64_t ld, int32_t vocab) {
    const char *p = static_cast<const char *>(base) + row * ld * (int64_t)sizeof(T);
    before = (int32_t)((-reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    if (before > vocab) before = vocab;
    pieces = (vocab - before) / kPer;
    after = vocab - before - pieces * kPer;
    at = const_cast<char *>(p) + before * (int64_t)sizeof(T);
  }
  // (a row's bytes fit 32 bits, which leaves an address one register a thread)
  template <int PAST = kThrough>
  __device__ u32x4 load(int32_t v) const {
    const u32x4 *const p = reinterpret_cast<const u32x4 *>(at + (uint32_t)v * 16u);
    if constexpr (PAST >= kLoads) return __builtin_nontemporal_load(p);
    return *p;
  }
  template <int PAST>
  __device__ void store(int32_t v, const float *x) const {
    if constexpr (PAST >= kBoth)
      __builtin_nontemporal_store(pack<T>(x), reinterpret_cast<u32x4 *>(at + (uint32_t)v * 16u));
    else
      *reinterpret_cast<u32x4 *>(at + (uint32_t)v * 16u) = pack<T>(x);
  }
  // The edge element of a thread, counted from the first whole piece; kNoEdge: it has none.
  static constexpr int64_t kNoEdge = INT64_MIN;
  __device__ int64_t edge(int32_t thread) const {
    if (thread < before) return thread - before;
    return thread >= kPer && thread - kPer < after ? (int64_t)pieces * kPer + thread - kPer : kNoEdge;
  }
};

// ---- maximum and sum together ---------------------------------------------------------------------------------------

// sum exp2((z - m) c) over what was seen so far, m its maximum (-inf: nothing but -inf was seen)
struct Running {
  float m = -kInf, s = 0.0f;
};
__device__ inline float exp2_diff(float z, float m, float c) { return __builtin_amdgcn_exp2f((z - m) * c); }
__device__ inline Running join(Running a, Running b, float c) {
  const float m = fmaxf(a.m, b.m), at = m == -kInf ? 0.0f : m;
  return {m, a.s * exp2_diff(a.m, at, c) + b.s * exp2_diff(b.m, at, c)};
}
template <int N>
__device__ inline void add(Running &r, const float *x, float c) {
  float m = r.m;
  for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
  const float at = m == -kInf ? 0.0f : m;        // (-inf - -inf is no number; exp2(-inf) is 0)
  float s = r.s * exp2_diff(r.m, at, c);
  for (int i = 0; i < N; ++i) s += exp2_diff(x[i], at, c);
  r = {m, s};
}

__device__ inline float wave_max(float v) {
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ inline float wave_sum(float v) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ inline Running wave_join(Running r, float c) {
  for (int d = 32; d; d >>= 1) r = join(r, {__shfl_xor(r.m, d), __shfl_xor(r.s, d)}, c);
  return r;
}

// ---- the list ---------------------------------------------------------------------------------------------------------

// In dynamic LDS, as long as the list is (list_bytes).
struct List {
  float *p, *log_p, *z;        // the teacher's probability, its logarithm, the logit itself
  int32_t *index;              // -1: no entry
  int32_t *table;              // 2^bits, at least twice the entries: to find words that stand twice in
  int32_t *any, *twice;        // there is an entry; there are two of one word
  int bits;
  // (`which`: the first or the second)
  __device__ explicit List(int32_t top, int which = 0) {
    extern __shared__ float space[];
    bits = 32 - __clz(2 * top - 1);
    if (bits < 6) bits = 6;
    p = space + which * (4 * top + 2 + (1 << bits));
    log_p = p + top;
    z = log_p + top;
    index = reinterpret_cast<int32_t *>(z + top);
    any = index + top;
    twice = any + 1;
    table = twice + 1;
  }
};
size_t list_bytes(int64_t top) {
  int64_t table = 64;
  while (table < 2 * top) table *= 2;
  return (size_t)(4 * top + 2 + table) * 4;
}

// By the first wave, each lane its own entries (nothing to wait for in between).  Logits and words that stand twice are asked for among
// the words [first, last).
template <typename T>
__device__ inline void read_list(const List &l, const DistillArgs &a, int64_t row, int64_t first, int64_t last) {
  const int lane = threadIdx.x & 63;
  const void *logits = static_cast<const char *>(a.logits) + row * a.ld * (int64_t)sizeof(T);
  for (int j = lane; j < 1 << l.bits; j += 64) l.table[j] = -1;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float m = -kInf;
  bool any = false, twice = false;
  for (int j = lane; j < a.top; j += 64) {
    const int64_t e = row * a.top + j;
    const int64_t i = a.index_wide ? static_cast<const int64_t *>(a.index)[e] : static_cast<const int32_t *>(a.index)[e];
    const float t = a.teacher_f32 ? element<float>(a.teacher, e) : element<__bf16>(a.teacher, e);
    const bool entry = i >= 0 && i < a.vocab && t != -kInf;
    l.index[j] = entry ? (int32_t)i : -1;
    l.log_p[j] = t;
    if (entry) m = fmaxf(m, t);
    any |= entry;
    if (entry && i >= first && i < last) {
      l.z[j] = element<T>(logits, i);
      uint32_t h = (uint32_t)i * 0x9E3779B1u >> (32 - l.bits);
      for (;; h = (h + 1) & ((1u << l.bits) - 1)) {      // (at least half of the table stays free)
        const int32_t there = atomicCAS(&l.table[h], -1, (int32_t)i);
        twice |= there == (int32_t)i;
        if (there == -1 || there == (int32_t)i) break;
      }
    }
  }
  m = wave_max(m);
  float s = 0.0f;
  for (int j = lane; j < a.top; j += 64) {
    const float e = l.index[j] < 0 ? 0.0f : exp2_diff(l.log_p[j], m, a.c);
    l.p[j] = e;
    s += e;
  }
  s = wave_sum(s);
  const float log_s = logf(s), inv_s = 1.0f / s;
  for (int j = lane; j < a.top; j += 64) {
    l.p[j] = l.index[j] < 0 ? 0.0f : l.p[j] * inv_s;
    l.log_p[j] = (l.log_p[j] - m) * a.inv_t - log_s;
  }
  const bool some = __ballot(any) != 0, two = __ballot(twice) != 0;
  if (lane == 0) {
    *l.any = some;
    *l.twice = two;
  }
}
// By the first wave.  y - lse is (z - m) / temperature - log s, from the row's maximum m and sum s: m / temperature need not be a number
// of fp32 (a row of nothing but the type's lowest value, at a temperature below 1), nor z - m, but half of it is.
__device__ inline float list_loss(const List &l, const DistillArgs &a, Running row) {
  const float log_s = logf(row.s), half_m = 0.5f * row.m, twice_inv_t = 2.0f * a.inv_t;
  float s = 0.0f;
  for (int j = threadIdx.x & 63; j < a.top; j += 64)
    if (l.index[j] >= 0 && l.p[j] != 0.0f) s += l.p[j] * (l.log_p[j] - ((0.5f * l.z[j] - half_m) * twice_inv_t - log_s));
  return wave_sum(s);
}

// exp(z / temperature - lse)
__device__ inline float probability(float z, float inv_t, float lse) {
  constexpr float kLog2e = 1.44269504088896340736f;
  return __builtin_amdgcn_exp2f(fmaf(z, inv_t, -lse) * kLog2e);
}
// The places of the list among the words [first, last) of a row are written again, after what stands there now: the caller has the
// workgroup's stores and the list behind a barrier.  `probability_of` is that of the other words.
template <typename T, int NT, typename P>
__device__ inline void rewrite_list(const List &l, const DistillArgs &a, int64_t row, int64_t first, int64_t last, float g, P &&probability_of) {
  if (!*l.any) return;
  char *const d = static_cast<char *>(a.dlogits) + row * a.ld * (int64_t)sizeof(T);
  for (int j = threadIdx.x; j < a.top; j += NT) {
    const int32_t at = l.index[j];
    if (at < first || at >= last) continue;
    float p = l.p[j];
    if (*l.twice) {
      p = 0.0f;
      for (int k = 0; k < a.top; ++k) p += l.index[k] == at ? l.p[k] : 0.0f;
    }
    set_element<T>(d, at, g * (probability_of(l.z[j]) - p));
  }
}

// ---- whole workgroups -----------------------------------------------------------------------------------------------

template <int NT>
struct Scratch {
  float m[NT / 64], s[NT / 64];
};

// The waves' sums together; one barrier.
template <int NT>
__device__ inline Running join_waves(float *m, float *s, Running run, float c) {
  run = wave_join(run, c);
  if ((threadIdx.x & 63) == 0) {
    m[threadIdx.x / 64] = run.m;
    s[threadIdx.x / 64] = run.s;
  }
  __syncthreads();
  run = {};
  for (int i = 0; i < NT / 64; ++i) run = join(run, {m[i], s[i]}, c);
  return run;
}
template <typename T, int NT>
__device__ inline Running row_sum(Scratch<NT> &sh, const Row<T> &r, float c) {
  constexpr int kAhead = 4, kPer = Row<T>::kPer;
  Running run;
  for (int32_t v0 = threadIdx.x; v0 < r.pieces; v0 += NT * kAhead) {
    u32x4 w[kAhead];
    for (int i = 0; i < kAhead; ++i) w[i] = r.load(v0 + i * NT < r.pieces ? v0 + i * NT : r.pieces - 1);
    float x[kAhead * kPer];
    for (int i = 0; i < kAhead; ++i) {
      unpack<T>(w[i], x + i * kPer);
      if (v0 + i * NT >= r.pieces)
        for (int k = 0; k < kPer; ++k) x[i * kPer + k] = -kInf;
    }
    add<kAhead * kPer>(run, x, c);
  }
  if (const int64_t e = r.edge(threadIdx.x); e != Row<T>::kNoEdge) {
    const float x = element<T>(r.at, e);
    add<1>(run, &x, c);
  }
  return join_waves<NT>(sh.m, sh.s, run, c);
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT) k_distill_forward(DistillArgs a) {
  __shared__ Scratch<NT> sh;
  const List list(a.top);
  const int64_t row = blockIdx.x;
  if (threadIdx.x < 64) read_list<T>(list, a, row, 0, a.vocab);
  const Running run = row_sum<T, NT>(sh, Row<T>(a.logits, row, a.ld, a.vocab), a.c);
  if (threadIdx.x < 64) {
    const float loss = *list.any ? list_loss(list, a, run) : 0.0f;
    if (threadIdx.x == 0) {
      a.loss[row] = loss;
      if (a.lse) a.lse[row] = run.m * a.inv_t + logf(run.s);
    }
  }
}

// `per` pieces of a row for a workgroup.  The next pieces are asked for before these are written; the first before the list is read, which
// takes two turns to memory (2047 x 50021 BF16, all of it through the caches: 97 us, one piece at a time and after the list 113).
template <typename T, int NT, int PAST>
__global__ void __launch_bounds__(NT) k_distill_backward(DistillArgs a, int32_t per) {
  constexpr int kAhead = 4, kPer = Row<T>::kPer;
  const List list(a.top);
  const int64_t row = blockIdx.x;
  const Row<T> r(a.logits, row, a.ld, a.vocab), d(a.dlogits, row, a.ld, a.vocab);
  const int32_t first = (int32_t)blockIdx.y * per, last = r.pieces - first < per ? r.pieces : first + per;
  // this workgroup's words: its pieces, and the edge that they touch
  const bool begins = blockIdx.y == 0, ends = blockIdx.y == gridDim.y - 1;
  const auto word_of = [&](int32_t piece) { return (int64_t)(piece < r.pieces ? piece : r.pieces) * kPer + r.before; };
  const int64_t word0 = begins ? 0 : word_of(first), word1 = ends ? a.vocab : word_of(first + per);
  const float lse = a.lse_in[row], g = a.weight ? a.weight[row] * a.inv_t : a.inv_t;
  u32x4 w[kAhead];
  const auto fetch = [&](int32_t v0) {
    for (int i = 0; i < kAhead; ++i) w[i] = r.template load<PAST>(v0 + i * NT < last ? v0 + i * NT : last - 1);
  };
  if (first < last) fetch(first + threadIdx.x);
  if (threadIdx.x < 64) read_list<T>(list, a, row, word0, word1);
  __syncthreads();             // (dlogits may be the logits: the list's are read before any is written)
  const bool any = *list.any;
  const auto of = [&](float z) { return any ? g * probability(z, a.inv_t, lse) : 0.0f; };
  for (int32_t v0 = first + threadIdx.x; v0 < last; v0 += NT * kAhead) {
    float x[kAhead][kPer];
    for (int i = 0; i < kAhead; ++i) {
      unpack<T>(w[i], x[i]);
      for (int k = 0; k < kPer; ++k) x[i][k] = of(x[i][k]);
    }
    if (v0 + NT * kAhead < last) fetch(v0 + NT * kAhead);
    for (int i = 0; i < kAhead; ++i)
      if (v0 + i * NT < last) d.template store<PAST>(v0 + i * NT, x[i]);
  }
  if (const int64_t e = r.edge(threadIdx.x); e != Row<T>::kNoEdge && (e < 0 ? begins : ends)) set_element<T>(d.at, e, of(element<T>(r.at, e)));
  __syncthreads();
  rewrite_list<T, NT>(list, a, row, word0, word1, g, [&](float z) { return probability(z, a.inv_t, lse); });
}

// Sum and gradient of a row too long for registers (k_distill_rows), which is read twice: 2048 x 151936 BF16 277 us (4.5 TB/s of the bytes
// that it would take once).
template <typename T, int NT, int PAST>
__global__ void __launch_bounds__(NT) k_distill_step(DistillArgs a) {
  constexpr int kPer = Row<T>::kPer;
  __shared__ Scratch<NT> sh;
  const List list(a.top);
  const int64_t row = blockIdx.x;
  const Row<T> r(a.logits, row, a.ld, a.vocab), d(a.dlogits, row, a.ld, a.vocab);
  if (threadIdx.x < 64) read_list<T>(list, a, row, 0, a.vocab);
  const Running run = row_sum<T, NT>(sh, r, a.c);
  const float g = a.weight ? a.weight[row] * a.inv_t : a.inv_t, inv_s = 1.0f / run.s, gs = g * inv_s, most = run.m;
  if (threadIdx.x < 64) {
    const float loss = *list.any ? list_loss(list, a, run) : 0.0f;
    if (threadIdx.x == 0) a.loss[row] = loss;
  }
  const bool any = *list.any;
  const auto of = [&](float z) { return any ? gs * exp2_diff(z, most, a.c) : 0.0f; };
  for (int32_t v = threadIdx.x; v < r.pieces; v += NT) {
    float x[kPer];
    unpack<T>(r.template load<PAST>(v), x);
    for (int k = 0; k < kPer; ++k) x[k] = of(x[k]);
    d.template store<PAST>(v, x);
  }
  if (const int64_t e = r.edge(threadIdx.x); e != Row<T>::kNoEdge) set_element<T>(d.at, e, of(element<T>(r.at, e)));
  __syncthreads();
  rewrite_list<T, NT>(list, a, row, 0, a.vocab, g, [&](float z) { return exp2_diff(z, most, a.c) * inv_s; });
}

// The same with the row in registers, NV pieces a thread.  A workgroup takes row after row: where a piece of the gradient has been
// written, that piece of the next row is asked for, and kLag pieces later it enters the next row's sum.  So loads and stores are on
// their way together, and the exponentials of both passes lie over them.  4096 x 131072 BF16: read twice 656 us, in registers 533, with
// the next row's sum between the stores 477 (and past the caches 460).
template <typename T, int NT, int NV, int PAST>
__global__ void __launch_bounds__(NT) k_distill_rows(DistillArgs a, int32_t rows) {
  constexpr int kPer = Row<T>::kPer, kLag = NV / 4;
  __shared__ Scratch<NT> sh[2];                  // (and two lists: each is written again two barriers after it was read)
  u32x4 w[NV];
  float edge = 0.0f;
  int32_t thread = threadIdx.x;
  const auto fetch = [&](const Row<T> &of, int i) {              // (pieces past the last: the last once more)
    const int32_t v = thread + i * NT;
    if (of.pieces > 0) w[i] = of.template load<PAST>(v < of.pieces ? v : of.pieces - 1);
  };
  const auto fetch_edge = [&](const Row<T> &of) {
    if (const int64_t e = of.edge(threadIdx.x); e != Row<T>::kNoEdge) edge = element<T>(of.at, e);
  };
  const auto sum = [&](const Row<T> &of, int i, Running &run) {
    float x[kPer];
    asm("" : "+v"(w[i]));                        // (what is unpacked here is not kept for the gradient: there would be no registers)
    unpack<T>(w[i], x);
    if (thread + i * NT < of.pieces) add<kPer>(run, x, a.c);
  };
  Running run;
  {
    const Row<T> of(a.logits, blockIdx.x, a.ld, a.vocab);
#pragma unroll
    for (int i = 0; i < NV; ++i) fetch(of, i);
    fetch_edge(of);
    if (threadIdx.x < 64) read_list<T>(List(a.top, 0), a, blockIdx.x, 0, a.vocab);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      sum(of, i, run);
      __builtin_amdgcn_sched_barrier(0);         // (one piece after the other: side by side they would not fit the registers)
    }
  }
  int turn = 0;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
    asm("" : "+v"(thread));                      // (the pieces' places are found again for each row, not kept)
    const List list(a.top, turn);
    const Row<T> r(a.logits, row, a.ld, a.vocab), d(a.dlogits, row, a.ld, a.vocab);
    const int64_t e = r.edge(threadIdx.x);
    if (e != Row<T>::kNoEdge) add<1>(run, &edge, a.c);
    run = join_waves<NT>(sh[turn].m, sh[turn].s, run, a.c);
    const float g = a.weight ? a.weight[row] * a.inv_t : a.inv_t, inv_s = 1.0f / run.s, gs = g * inv_s, most = run.m;
    const bool any = *list.any;
    if (threadIdx.x < 64) {
      const float loss = any ? list_loss(list, a, run) : 0.0f;
      if (threadIdx.x == 0) a.loss[row] = loss;
    }
    const int64_t next = row + gridDim.x;
    const bool more = next < rows;
    const Row<T> then(a.logits, more ? next : row, a.ld, a.vocab);
    if (e != Row<T>::kNoEdge) set_element<T>(d.at, e, any ? gs * exp2_diff(edge, most, a.c) : 0.0f);
    if (more) fetch_edge(then);
    run = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int32_t v = thread + i * NT;
      float x[kPer];
      asm("" : "+v"(w[i]));
      unpack<T>(w[i], x);
      for (int k = 0; k < kPer; ++k) x[k] = any ? gs * exp2_diff(x[k], most, a.c) : 0.0f;
      if (v < r.pieces) d.template store<PAST>(v, x);
      if (more) fetch(then, i);
      __builtin_amdgcn_sched_barrier(0);
      if (more && i >= kLag) sum(then, i - kLag, run);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (more) {
#pragma unroll
      for (int i = NV - kLag; i < NV; ++i) {
        sum(then, i, run);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();
    rewrite_list<T, NT>(list, a, row, 0, a.vocab, g, [&](float z) { return exp2_diff(z, most, a.c) * inv_s; });
    if (threadIdx.x < 64 && more) read_list<T>(List(a.top, turn ^ 1), a, next, 0, a.vocab);
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------

// (`more`: the call's other pointers are given.  Sizes come first: what has no element may well have no address.)
int check(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index, bool more) {
  if (!p) return NVFP4_ERR_NULL;
  if (p->rows < 0 || p->rows > kMostRows || p->vocab <= 0 || p->vocab > (int64_t)1 << 29 || p->ld < p->vocab ||
      p->ld > (int64_t)1 << 40 || p->rows * p->ld > (int64_t)1 << 40 || p->top <= 0 || p->top > kMostTop)
    return NVFP4_ERR_SHAPE;
  if (p->rows != 0 && (!logits || !teacher || !index || !more)) return NVFP4_ERR_NULL;
  if (!(p->temperature >= kLeastTemperature) || !(p->temperature < kInf) || p->x_dtype > NVFP4_X_F32 || p->teacher_dtype > NVFP4_X_F32 ||
      p->index_dtype > NVFP4_INDEX_I64)
    return NVFP4_ERR_PARAM;
  return NVFP4_OK;
}
bool at(const void *ptr, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }
bool aligned(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index) {
  return at(logits, p->x_dtype ? 4 : 2) && at(teacher, p->teacher_dtype ? 4 : 2) && at(index, p->index_dtype ? 8 : 4);
}
DistillArgs args(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index) {
  DistillArgs a{};
  a.logits = logits;
  a.teacher = teacher;
  a.index = index;
  a.ld = p->ld;
  a.vocab = (int32_t)p->vocab;
  a.top = (int32_t)p->top;
  a.c = (float)(1.44269504088896340736 / (double)p->temperature);
  a.inv_t = (float)(1.0 / (double)p->temperature);
  a.teacher_f32 = p->teacher_dtype == NVFP4_X_F32;
  a.index_wide = p->index_dtype == NVFP4_INDEX_I64;
  return a;
}

constexpr int kComputeUnits = 256;            // of an MI355X: where there are others, only how rows are dealt out is less even

template <typename T, int NT, int NV, int PAST>
int run_rows(const DistillArgs &a, int64_t rows, int per_cu, hipStream_t s) {
  const int64_t most = (int64_t)kComputeUnits * per_cu;
  return launch(k_distill_rows<T, NT, NV, PAST>, dim3((uint32_t)(rows < most ? rows : most)), dim3(NT), 2 * list_bytes(a.top), s, a,
                (int32_t)rows);
}
template <typename T, int PAST>
int run_step(const DistillArgs &a, int64_t rows, hipStream_t s) {
  // As many workgroups a compute unit as its registers hold: 16 to 32 waves.  (Of 4097 to 8192 pieces 1024 threads with eight each would leave
  // room for one only.)
  const int64_t pieces = a.vocab / (int64_t)(16 / sizeof(T));        // (whole ones, at most)
  if (pieces <= 256 * 4) return run_rows<T, 256, 4, PAST>(a, rows, 8, s);
  if (pieces <= 256 * 8) return run_rows<T, 256, 8, PAST>(a, rows, 7, s);
  if (pieces <= 256 * 16) return run_rows<T, 256, 16, PAST>(a, rows, 4, s);
  if (pieces <= 512 * 16) return run_rows<T, 512, 16, PAST>(a, rows, 2, s);
  if (pieces <= 1024 * 16) return run_rows<T, 1024, 16, PAST>(a, rows, 1, s);
  return launch(k_distill_step<T, 1024, PAST>, dim3((uint32_t)rows), dim3(1024), list_bytes(a.top), s, a);
}
template <typename T, int PAST>
int run_backward(const DistillArgs &a, int64_t rows, hipStream_t s) {
  const int64_t per = 16 / sizeof(T), pieces = a.vocab / per > 0 ? a.vocab / per : 1;      // (whole ones, at most)
  // few rows: several workgroups a row, of 1024 pieces at least
  int64_t splits = 1;
  while (splits < 256 && rows * splits < 512 && pieces / (2 * splits) >= 1024) splits *= 2;
  return launch(k_distill_backward<T, 256, PAST>, dim3((uint32_t)rows, (uint32_t)splits), dim3(256), list_bytes(a.top), s, a,
                (int32_t)((pieces + splits - 1) / splits));
}

// Logits are read here for the last time: where they and the gradient do not fit the device's last cache (256 MB) together, they are loaded past
// the caches, which leaves them to the gradient's reader; where it can hardly hold the gradient alone, that is stored past them too.  In us, all
// through / loads past / both, gradients of BF16 (50021 words) with several batches in turn: 80 MB 43 / 36 / 42, 128 MB 66 / 64 / 64, 192 MB
// 93 / 95 / 91, 260 MB 123 / 127 / 121, 540 MB 247 / 261 / 248; of fp32 (32768 words): 39 / 33 / 36, 59 / 58 / 54, 87 / 86 / 79, 119 / 120 / 109,
// 234 / 241 / 217; steps the same way.  With one batch again and again, of which the cache still has a part: BF16 30 / 35 / 40, 48 / 51 / 62, 88 / 70 / 89,
// 121 / 94 / 120, 247 / 263 / 246.  So storing past begins to pay between 120 MB, where nothing is in the cache, and 300 MB, where as much is as there can be.
int past_caches(const nvfp4_distill_params *p) {
  const int64_t megabytes = p->rows * p->vocab * (p->x_dtype ? 4 : 2) >> 20;
  return megabytes > 192 ? kBoth : megabytes > 96 ? kLoads : kThrough;
}

template <typename T>
int run_step(int past, const DistillArgs &a, int64_t rows, hipStream_t s) {
  return past == kBoth ? run_step<T, kBoth>(a, rows, s) : past == kLoads ? run_step<T, kLoads>(a, rows, s) : run_step<T, kThrough>(a, rows, s);
}
template <typename T>
int run_backward(int past, const DistillArgs &a, int64_t rows, hipStream_t s) {
  return past == kBoth ? run_backward<T, kBoth>(a, rows, s) : past == kLoads ? run_backward<T, kLoads>(a, rows, s)
                                                                            : run_backward<T, kThrough>(a, rows, s);
}

}  // namespace
}  // namespace nvfp4_46

using namespace nvfp4_46;

extern "C" int nvfp4_distill_forward(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index,
                                     float *loss, float *lse, void *stream) {
  if (const int rc = check(logits, p, teacher, index, loss)) return rc;
  if (!aligned(logits, p, teacher, index) || !at(loss, 4) || !at(lse, 4)) return NVFP4_ERR_ALIGN;
  if (p->rows == 0) return NVFP4_OK;
  DistillArgs a = args(logits, p, teacher, index);
  a.loss = loss;
  a.lse = lse;
  return launch(p->x_dtype ? k_distill_forward<float, 256> : k_distill_forward<__bf16, 256>, dim3((uint32_t)p->rows), dim3(256),
                list_bytes(p->top), static_cast<hipStream_t>(stream), a);
}

extern "C" int nvfp4_distill_backward(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index,
                                      const float *lse, const float *weight, void *dlogits, void *stream) {
  if (const int rc = check(logits, p, teacher, index, lse && dlogits)) return rc;
  if (!aligned(logits, p, teacher, index) || !at(lse, 4) || !at(weight, 4) || !at(dlogits, p->x_dtype ? 4 : 2) ||
      (reinterpret_cast<uintptr_t>(dlogits) ^ reinterpret_cast<uintptr_t>(logits)) % 16)
    return NVFP4_ERR_ALIGN;
  if (p->rows == 0) return NVFP4_OK;
  DistillArgs a = args(logits, p, teacher, index);
  a.lse_in = lse;
  a.weight = weight;
  a.dlogits = dlogits;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p->x_dtype ? run_backward<float>(past_caches(p), a, p->rows, s) : run_backward<__bf16>(past_caches(p), a, p->rows, s);
}

extern "C" int nvfp4_distill_step(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index,
                                  const float *weight, float *loss, void *dlogits, void *stream) {
  if (const int rc = check(logits, p, teacher, index, loss && dlogits)) return rc;
  if (!aligned(logits, p, teacher, index) || !at(loss, 4) || !at(weight, 4) || !at(dlogits, p->x_dtype ? 4 : 2) ||
      (reinterpret_cast<uintptr_t>(dlogits) ^ reinterpret_cast<uintptr_t>(logits)) % 16)
    return NVFP4_ERR_ALIGN;
  if (p->rows == 0) return NVFP4_OK;
  DistillArgs a = args(logits, p, teacher, index);
  a.loss = loss;
  a.weight = weight;
  a.dlogits = dlogits;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return p->x_dtype ? run_step<float>(past_caches(p), a, p->rows, s) : run_step<__bf16>(past_caches(p), a, p->rows, s);
}
