// Low-rank adapters of many requests at once beside a shared projection (include/finetune/nvfp4_finetune.h), forwards and
// backwards.
//
//   h_t = A_l x_t,  out_t = base_t + s_l B_l h_t,  l = which[t]
//   dh_t = s_l B_l^T dy_t,  dx_t = dx_base_t + A_l^T dh_t,  dA_l = sum_t dh_t x_t^T,  dB_l = s_l sum_t dy_t h_t^T
//
// The plainest kernels that are right for every size: one workgroup for each token, or for each line of a gradient.
#include <hip/hip_runtime.h>

#include "finetune/nvfp4_finetune.h"
#include "launch.hpp"

namespace nvfp4_46 {
namespace {

constexpr int kMostRank = 128, kMostAdapters = 2048;

struct AdapterArgs {
  const __bf16 *x, *dy, *a, *b;
  const void *base;
  const int32_t *which;
  const float *scales, *h_in;
  float *h, *dh, *da, *db;
  void *out;
  int64_t T, K, N, L, r, ld_x, ld_base, ld_out, ld_dy;
};

__device__ inline int32_t adapter_of(const AdapterArgs &a, int64_t t) {
  const int32_t l = a.which[t];
  return l >= 0 && l < a.L ? l : -1;
}
__device__ inline float wave_sum(float v) {
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// h (kBack: dh) of one token: a wave for every fourth row of A (column of B)
template <bool kBack>
__global__ void __launch_bounds__(256) k_low_rank(AdapterArgs a) {
  const int64_t t = blockIdx.x;
  const int lane = threadIdx.x & 63;
  const int32_t l = adapter_of(a, t);
  for (int64_t j = threadIdx.x / 64; j < a.r; j += 4) {
    float s = 0.0f;
    if (l >= 0 && !kBack)
      for (int64_t k = lane; k < a.K; k += 64) s = fmaf((float)a.x[t * a.ld_x + k], (float)a.a[(l * a.r + j) * a.K + k], s);
    if (l >= 0 && kBack)
      for (int64_t n = lane; n < a.N; n += 64) s = fmaf((float)a.dy[t * a.ld_dy + n], (float)a.b[(l * a.N + n) * a.r + j], s);
    s = wave_sum(s);
    if (lane == 0) (kBack ? a.dh : a.h)[t * a.r + j] = kBack && l >= 0 ? s * a.scales[l] : s;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) k_expand(AdapterArgs a) {
  const int64_t t = blockIdx.x, n = (int64_t)blockIdx.y * 256 + threadIdx.x;
  if (n >= a.N) return;
  const int32_t l = adapter_of(a, t);
  float s = 0.0f;
  if (l >= 0)
    for (int64_t j = 0; j < a.r; ++j) s = fmaf(a.h[t * a.r + j], (float)a.b[(l * a.N + n) * a.r + j], s);
  const float base = a.base ? (float)static_cast<const T *>(a.base)[t * a.ld_base + n] : 0.0f;
  static_cast<T *>(a.out)[t * a.ld_out + n] = (T)(l >= 0 ? base + a.scales[l] * s : base);
}

__global__ void __launch_bounds__(256) k_dx(AdapterArgs a) {
  const int64_t t = blockIdx.x, k = (int64_t)blockIdx.y * 256 + threadIdx.x;
  if (k >= a.K) return;
  const int32_t l = adapter_of(a, t);
  float s = a.base ? (float)static_cast<const __bf16 *>(a.base)[t * a.ld_base + k] : 0.0f;
  if (l >= 0)
    for (int64_t j = 0; j < a.r; ++j) s = fmaf(a.dh[t * a.r + j], (float)a.a[(l * a.r + j) * a.K + k], s);
  static_cast<__bf16 *>(a.out)[t * a.ld_out + k] = (__bf16)s;
}

__global__ void __launch_bounds__(256) k_da(AdapterArgs a) {
  const int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x, j = blockIdx.y, l = blockIdx.z;
  if (k >= a.K) return;
  float s = 0.0f;
  for (int64_t t = 0; t < a.T; ++t)
    if (a.which[t] == l) s = fmaf(a.dh[t * a.r + j], (float)a.x[t * a.ld_x + k], s);
  a.da[(l * a.r + j) * a.K + k] = s;
}
__global__ void __launch_bounds__(256) k_db(AdapterArgs a) {
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x, j = blockIdx.y, l = blockIdx.z;
  if (n >= a.N) return;
  float s = 0.0f;
  for (int64_t t = 0; t < a.T; ++t)
    if (a.which[t] == l) s = fmaf(a.h_in[t * a.r + j], (float)a.dy[t * a.ld_dy + n], s);
  a.db[(l * a.N + n) * a.r + j] = s * a.scales[l];
}

// ---- host -----------------------------------------------------------------------------------------------------------

constexpr int64_t kMostTokens = (1 << 24) - 1, kMostWidth = 1 << 22;

bool sizes_fit(const nvfp4_adapters_params &p) {
  return p.tokens >= 0 && p.tokens <= kMostTokens && p.inp > 0 && p.inp <= kMostWidth && p.out > 0 && p.out <= kMostWidth && p.inp % 8 == 0 &&
         p.out % 8 == 0 && p.adapters > 0 && p.adapters <= kMostAdapters && p.rank > 0 && p.rank <= kMostRank;
}
bool stride_fits(int64_t ld, int64_t width, int64_t rows) {
  return ld >= width && ld <= (int64_t)1 << 40 && rows * ld <= (int64_t)1 << 40;
}
bool at(const void *ptr, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }

size_t workspace_bytes_of(const nvfp4_adapters_params &p) { return (size_t)(p.tokens * p.rank * 4 + 15) / 16 * 16 + 16; }

AdapterArgs args(const nvfp4_adapters_params &p) {
  AdapterArgs a{};
  a.T = p.tokens;
  a.K = p.inp;
  a.N = p.out;
  a.L = p.adapters;
  a.r = p.rank;
  a.ld_x = p.ld_x;
  a.ld_base = p.ld_base;
  a.ld_out = p.ld_out;
  a.ld_dy = p.ld_dy;
  return a;
}

}  // namespace
}  // namespace nvfp4_46

using namespace nvfp4_46;

extern "C" size_t nvfp4_adapters_workspace_bytes(const nvfp4_adapters_params *p, int) {
  return p && sizes_fit(*p) ? workspace_bytes_of(*p) : 0;
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
  if (p->out_dtype > NVFP4_OUT_F32 || workspace_bytes < workspace_bytes_of(*p)) return NVFP4_ERR_PARAM;
  if (p->tokens == 0) return NVFP4_OK;
  AdapterArgs g = args(*p);
  g.x = static_cast<const __bf16 *>(x);
  g.a = static_cast<const __bf16 *>(a);
  g.b = static_cast<const __bf16 *>(b);
  g.base = base;
  g.which = which;
  g.scales = scales;
  g.h = h ? h : static_cast<float *>(workspace);
  g.out = out;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (const int rc = launch(k_low_rank<false>, dim3((uint32_t)g.T), dim3(256), 0, s, g)) return rc;
  return launch(p->out_dtype ? k_expand<float> : k_expand<__bf16>, dim3((uint32_t)g.T, (uint32_t)((g.N + 255) / 256)), dim3(256),
                0, s, g);
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
  if (workspace_bytes < workspace_bytes_of(*p)) return NVFP4_ERR_PARAM;
  AdapterArgs g = args(*p);
  g.x = static_cast<const __bf16 *>(x);
  g.dy = static_cast<const __bf16 *>(dy);
  g.a = static_cast<const __bf16 *>(a);
  g.b = static_cast<const __bf16 *>(b);
  g.base = dx_base;
  g.which = which;
  g.scales = scales;
  g.h_in = h;
  g.dh = static_cast<float *>(workspace);
  g.da = da;
  g.db = db;
  g.out = dx;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const auto blocks = [](int64_t n) { return (uint32_t)((n + 255) / 256); };
  if (g.T) {
    if (const int rc = launch(k_low_rank<true>, dim3((uint32_t)g.T), dim3(256), 0, s, g)) return rc;
    if (dx)
      if (const int rc = launch(k_dx, dim3((uint32_t)g.T, blocks(g.K)), dim3(256), 0, s, g)) return rc;
  }
  if (const int rc = launch(k_da, dim3(blocks(g.K), (uint32_t)g.r, (uint32_t)g.L), dim3(256), 0, s, g)) return rc;
  return launch(k_db, dim3(blocks(g.N), (uint32_t)g.r, (uint32_t)g.L), dim3(256), 0, s, g);
}
