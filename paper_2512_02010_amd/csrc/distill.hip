// Distillation from a teacher's top logits (include/finetune/nvfp4_finetune.h): loss, gradient, and both in one pass.
//
// Per row y = z / temperature, lse = log sum exp y, p = softmax(teacher / temperature) over the list:
//   loss = sum_j p_j (log p_j - (y_{i_j} - lse)),   dz_v = w / temperature (exp(y_v - lse) - sum_{j: i_j = v} p_j).
// All of it is bound by the bytes of the logits: a row is read once for its maximum and sum together (the sum is rescaled when
// the maximum grows), and the list, which is short, is dealt with by the first wave while the others stream.
#include <hip/hip_runtime.h>

#include <cmath>

#include "finetune/nvfp4_finetune.h"
#include "launch.hpp"

namespace nvfp4_46 {
namespace {

constexpr int kMostTop = 1024;
constexpr int64_t kMostRows = 1 << 21;        // (a workgroup of 1024 each: a grid has fewer than 2^32 threads)
constexpr float kInf = __builtin_inff();

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
// A row begins anywhere (its length may be odd): pieces are cut at multiples of 16 bytes of the address, and the first and last
// piece hold elements of this row only, one by one.

template <typename T>
struct Row {
  static constexpr int kPer = 16 / sizeof(T);
  char *at;                    // the first piece
  int32_t off, end;            // this row's elements are [off, end) counted from there
  __device__ Row(const void *base, int64_t row, int64_t ld, int32_t vocab) {
    const char *p = static_cast<const char *>(base) + row * ld * (int64_t)sizeof(T);
    off = (int32_t)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
    at = const_cast<char *>(p) - off * sizeof(T);
    end = off + vocab;         // (vocab < 2^31 - 8 by the host's check)
  }
  __device__ int32_t pieces() const { return (end + kPer - 1) / kPer; }
  __device__ bool whole(int32_t v) const { return v * kPer >= off && (v + 1) * kPer <= end; }
};

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
// Piece v; elements of other rows come as -inf, whose exponential is 0.
template <typename T>
__device__ inline u32x4 load_piece(const Row<T> &r, int32_t v) {
  if (r.whole(v)) return *reinterpret_cast<const u32x4 *>(r.at + (int64_t)v * 16);
  float x[Row<T>::kPer];
  for (int i = 0; i < Row<T>::kPer; ++i) {
    const int32_t e = v * Row<T>::kPer + i;
    x[i] = e >= r.off && e < r.end ? element<T>(r.at, e) : -kInf;
  }
  return pack<T>(x);
}
template <typename T>
__device__ inline void store_piece(const Row<T> &r, int32_t v, const float *x) {
  if (r.whole(v)) {
    *reinterpret_cast<u32x4 *>(r.at + (int64_t)v * 16) = pack<T>(x);
    return;
  }
  for (int i = 0; i < Row<T>::kPer; ++i) {
    const int32_t e = v * Row<T>::kPer + i;
    if (e >= r.off && e < r.end) set_element<T>(r.at, e, x[i]);
  }
}

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

struct List {
  float p[kMostTop], log_p[kMostTop], z[kMostTop];     // the teacher's probability, its logarithm, the logit itself
  int32_t index[kMostTop];                             // -1: no entry
  int32_t any;
};

// By the first wave, each lane its own entries (nothing to wait for in between); z only where it is asked for.
template <typename T>
__device__ inline void read_list(List &l, const DistillArgs &a, int64_t row, bool want_z) {
  const int lane = threadIdx.x & 63;
  const void *logits = static_cast<const char *>(a.logits) + row * a.ld * (int64_t)sizeof(T);
  float m = -kInf;
  bool any = false;
  for (int j = lane; j < a.top; j += 64) {
    const int64_t e = row * a.top + j;
    const int64_t i = a.index_wide ? static_cast<const int64_t *>(a.index)[e] : static_cast<const int32_t *>(a.index)[e];
    const float t = a.teacher_f32 ? element<float>(a.teacher, e) : element<__bf16>(a.teacher, e);
    const bool entry = i >= 0 && i < a.vocab && t != -kInf;
    l.index[j] = entry ? (int32_t)i : -1;
    l.log_p[j] = t;
    if (entry) m = fmaxf(m, t);
    any |= entry;
    if (want_z) l.z[j] = entry ? element<T>(logits, i) : 0.0f;
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
  if (__ballot(any) != 0) {
    if (lane == 0) l.any = 1;
  } else if (lane == 0) {
    l.any = 0;
  }
}
// By the first wave.
__device__ inline float list_loss(const List &l, const DistillArgs &a, float lse) {
  float s = 0.0f;
  for (int j = threadIdx.x & 63; j < a.top; j += 64)
    if (l.index[j] >= 0 && l.p[j] != 0.0f) s += l.p[j] * (l.log_p[j] - (l.z[j] * a.inv_t - lse));
  return wave_sum(s);
}

// ---- whole workgroups -----------------------------------------------------------------------------------------------

template <int NT>
struct Scratch {
  List list;
  float m[NT / 64], s[NT / 64];
};

template <typename T, int NT>
__device__ inline Running row_sum(Scratch<NT> &sh, const Row<T> &r, float c) {
  constexpr int kAhead = 4, kPer = Row<T>::kPer;
  Running run;
  for (int32_t v0 = threadIdx.x; v0 < r.pieces(); v0 += NT * kAhead) {
    u32x4 w[kAhead];
    for (int i = 0; i < kAhead; ++i)
      if (v0 + i * NT < r.pieces()) w[i] = load_piece(r, v0 + i * NT);
    float x[kAhead * kPer];
    for (int i = 0; i < kAhead; ++i) {
      unpack<T>(w[i], x + i * kPer);
      if (v0 + i * NT >= r.pieces())
        for (int k = 0; k < kPer; ++k) x[i * kPer + k] = -kInf;
    }
    add<kAhead * kPer>(run, x, c);
  }
  run = wave_join(run, c);
  if ((threadIdx.x & 63) == 0) {
    sh.m[threadIdx.x / 64] = run.m;
    sh.s[threadIdx.x / 64] = run.s;
  }
  __syncthreads();
  run = {};
  for (int i = 0; i < NT / 64; ++i) run = join(run, {sh.m[i], sh.s[i]}, c);
  return run;
}
__device__ inline float lse_of(Running r, float inv_t) { return r.m * inv_t + logf(r.s); }

// The gradient of pieces [first, last), then of the list's places among them.
template <typename T, int NT>
__device__ inline void gradient(const List &l, const DistillArgs &a, int64_t row, int32_t first, int32_t last, float lse) {
  constexpr int kPer = Row<T>::kPer;
  const Row<T> r(a.logits, row, a.ld, a.vocab), d(a.dlogits, row, a.ld, a.vocab);
  const float g = a.weight ? a.weight[row] * a.inv_t : a.inv_t;
  constexpr float kLog2e = 1.44269504088896340736f;
  for (int32_t v = first + threadIdx.x; v < last; v += NT) {
    float x[kPer];
    unpack<T>(load_piece(r, v), x);
    for (int i = 0; i < kPer; ++i) x[i] = l.any ? g * __builtin_amdgcn_exp2f((x[i] * a.inv_t - lse) * kLog2e) : 0.0f;
    store_piece(d, v, x);
  }
  __syncthreads();             // the places of the list are written again, after what stands there now
  if (!l.any) return;
  for (int j = threadIdx.x; j < a.top; j += NT) {
    const int32_t at = l.index[j], v = (at + r.off) / kPer;
    if (at < 0 || v < first || v >= last) continue;
    float p = 0.0f;
    for (int k = 0; k < a.top; ++k) p += l.index[k] == at ? l.p[k] : 0.0f;
    set_element<T>(d.at, at + r.off, g * (__builtin_amdgcn_exp2f((l.z[j] * a.inv_t - lse) * kLog2e) - p));
  }
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT) k_distill_forward(DistillArgs a) {
  __shared__ Scratch<NT> sh;
  const int64_t row = blockIdx.x;
  if (threadIdx.x < 64) read_list<T>(sh.list, a, row, true);
  const float lse = lse_of(row_sum<T, NT>(sh, Row<T>(a.logits, row, a.ld, a.vocab), a.c), a.inv_t);
  if (threadIdx.x < 64) {
    const float loss = sh.list.any ? list_loss(sh.list, a, lse) : 0.0f;
    if (threadIdx.x == 0) {
      a.loss[row] = loss;
      if (a.lse) a.lse[row] = lse;
    }
  }
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT) k_distill_backward(DistillArgs a, int32_t pieces) {
  __shared__ List list;
  const int64_t row = blockIdx.x;
  if (threadIdx.x < 64) read_list<T>(list, a, row, true);
  __syncthreads();
  const int32_t first = (int32_t)blockIdx.y * pieces, all = Row<T>(a.logits, row, a.ld, a.vocab).pieces();
  gradient<T, NT>(list, a, row, first, all - first < pieces ? all : first + pieces, a.lse_in[row]);
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT) k_distill_step(DistillArgs a) {
  __shared__ Scratch<NT> sh;
  const int64_t row = blockIdx.x;
  const Row<T> r(a.logits, row, a.ld, a.vocab);
  if (threadIdx.x < 64) read_list<T>(sh.list, a, row, true);
  const float lse = lse_of(row_sum<T, NT>(sh, r, a.c), a.inv_t);
  if (threadIdx.x < 64) {
    const float loss = sh.list.any ? list_loss(sh.list, a, lse) : 0.0f;
    if (threadIdx.x == 0) a.loss[row] = loss;
  }
  gradient<T, NT>(sh.list, a, row, 0, r.pieces(), lse);
}

// ---- host -----------------------------------------------------------------------------------------------------------

// (`more`: the call's other pointers are given)
int check(const void *logits, const nvfp4_distill_params *p, const void *teacher, const void *index, bool more) {
  if (!p || (p->rows != 0 && (!logits || !teacher || !index || !more))) return NVFP4_ERR_NULL;
  if (p->rows < 0 || p->rows > kMostRows || p->vocab <= 0 || p->vocab > ((int64_t)1 << 31) - 16 || p->ld < p->vocab ||
      p->ld > (int64_t)1 << 40 || p->rows * p->ld > (int64_t)1 << 40 || p->top <= 0 || p->top > kMostTop)
    return NVFP4_ERR_SHAPE;
  if (!(p->temperature > 0.0f) || !(p->temperature < kInf) || p->x_dtype > NVFP4_X_F32 || p->teacher_dtype > NVFP4_X_F32 ||
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
                0, static_cast<hipStream_t>(stream), a);
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
  const int32_t per = p->x_dtype ? 4 : 8, pieces = (int32_t)((p->vocab + per - 1) / per) + 1;    // (one more where rows begin inside)
  return launch(p->x_dtype ? k_distill_backward<float, 256> : k_distill_backward<__bf16, 256>, dim3((uint32_t)p->rows, 1),
                dim3(256), 0, static_cast<hipStream_t>(stream), a, pieces);
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
  return launch(p->x_dtype ? k_distill_step<float, 256> : k_distill_step<__bf16, 256>, dim3((uint32_t)p->rows), dim3(256), 0,
                static_cast<hipStream_t>(stream), a);
}
