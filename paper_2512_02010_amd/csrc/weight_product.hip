// Activations as they are times a quantized weight, or those of many experts (include/finetune/nvfp4_finetune.h):
//
//   out[s][n] = alpha_e sum_k x[row(s)][k] value(code_e[n][k]) value(scale_e[n][k / 16])
//
// value(code) has two significant bits and value(scale) four: their product is exact in BF16, so that the BF16 matrix instruction multiplies
// exact operands and accumulates in fp32.  fp32 activations are sums of three BF16 terms, a matrix instruction for each.
#include <hip/hip_runtime.h>

#include "finetune/nvfp4_finetune.h"
#include "launch.hpp"

namespace nvfp4_46 {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int64_t kMostRows = (1 << 24) - 1, kMostWidth = 1 << 22, kMostExperts = 1024, kMostSlots = (int64_t)1 << 30;

struct ProductArgs {
  const void *x;
  const int32_t *token, *begin;        // NULL: rows as they stand, one expert
  const uint8_t *codes, *scales;
  const float *alpha;
  void *out;
  int64_t ld_x, ld_out;
  int32_t rows, slots, inp, out_width, experts;
  int32_t scale_shift;                 // 4: scales of 16 x 16 tiles
};

// ---- pieces -------------------------------------------------------------------------------------------------------------

// v as a sum of three BF16 terms, eight of its 24 bits each, exactly.  (Below 2^-110 BF16 has no numbers for all three.)  Of an infinity the first
// term is all there is: a weight is finite, so that what the others, 0, add is 0.  Of a NaN the second is one too.
__device__ inline void terms_of(float v, float (&t)[3]) {
  const auto cut = [](float f) { return __uint_as_float(__float_as_uint(f) & 0xffff0000u); };
  t[0] = cut(v);
  const float rest = t[0] == v ? 0.0f : v - t[0];
  t[1] = cut(rest);
  t[2] = rest == t[1] ? 0.0f : rest - t[1];
}

// Two fp32 numbers that are BF16 numbers, in one word.
__device__ inline uint32_t pack_exact(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
// Eight codes times one scale, exactly.
__device__ inline bf16x8 expand8(uint32_t word, float scale) {
  const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 1);
  const f32x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, 3);
  const u32x4 w = {pack_exact(p0.x * scale, p0.y * scale), pack_exact(p1.x * scale, p1.y * scale),
                   pack_exact(p2.x * scale, p2.y * scale), pack_exact(p3.x * scale, p3.y * scale)};
  return __builtin_bit_cast(bf16x8, w);
}

// The expert's rows of out, whatever begin holds.
struct Rows {
  int32_t first, last;
};
__device__ inline Rows rows_of(const ProductArgs &a, int32_t e) {
  if (!a.begin) return {0, a.slots};
  int32_t first = a.begin[e], last = a.begin[e + 1];
  first = first < 0 ? 0 : first < a.slots ? first : a.slots;
  last = last < first ? first : last < a.slots ? last : a.slots;
  return {first, last};
}

// ---- k_few --------------------------------------------------------------------------------------------------------------

constexpr int kFewWaves = 8;

// A workgroup has 16 columns of out and an expert's rows, 16 MT of them at a time; its waves share K, 128 at a time, and their sums meet in LDS.
// Lane l loads 16 bytes, 32 codes, of column l % 16 and x of row l % 16, in pieces of 64 adjacent bytes to four lanes.
template <typename T, typename TO, int MT>
__global__ void __launch_bounds__(kFewWaves * 64) k_few(ProductArgs a) {
  constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;
  __shared__ float part[kFewWaves][MT][4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), line = lane & 15, group = lane / 16;
  const int32_t e = (int32_t)blockIdx.y, n0 = (int32_t)blockIdx.x * 16, N = a.out_width, K = a.inp;
  TO *const out = static_cast<TO *>(a.out);
  if (e == a.experts) {                          // behind the last expert's rows
    for (int32_t s = rows_of(a, e - 1).last + (int32_t)threadIdx.x / 16; s < a.slots; s += kFewWaves * 4)
      if (n0 + (int32_t)threadIdx.x % 16 < N) out[(int64_t)s * a.ld_out + n0 + threadIdx.x % 16] = (TO)0.0f;
    return;
  }
  const Rows r = rows_of(a, e);
  if (r.first >= r.last) return;
  const int32_t n = n0 + line < N ? n0 + line : N - 1;
  const uint8_t *const codes = a.codes + ((int64_t)e * N + n) * (K / 2);
  const uint8_t *const scales = a.scales + ((int64_t)e * (N >> a.scale_shift) + (n >> a.scale_shift)) * (K / 16);
  const float alpha = a.alpha[e];
  for (int32_t m0 = r.first; m0 < r.last; m0 += 16 * MT) {
    const T *row[MT];
    bool is[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int32_t s = m0 + m * 16 + line;
      int32_t from = s < r.last ? s : r.last - 1;
      if (a.token) from = a.token[from];
      is[m] = from >= 0 && from < a.rows;
      row[m] = static_cast<const T *>(a.x) + (int64_t)(is[m] ? from : 0) * a.ld_x;
    }
    f32x4 acc[MT] = {};
    for (int32_t k0 = wave * 128; k0 < K; k0 += kFewWaves * 128) {
      // of 32 codes, and of each of 4 x 8 numbers of x, there are all or none (K is a multiple of 32)
      u32x4 w{};
      if (k0 + group * 32 < K) w = *reinterpret_cast<const u32x4 *>(codes + (k0 + group * 32) / 2);
      float sc[4];
      bf16x8 x[MT][4][kTerms];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const bool there = k0 + s * 32 < K;
        sc[s] = there ? __builtin_amdgcn_cvt_f32_fp8((int)scales[(k0 + s * 32) / 16 + group / 2], 0) : 0.0f;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const T *const from = row[m] + k0 + s * 32 + group * 8;
          if constexpr (kTerms == 1) {
            x[m][s][0] = there && is[m] ? *reinterpret_cast<const bf16x8 *>(from) : bf16x8{};
          } else {
            const f32x8 v = there && is[m] ? *reinterpret_cast<const f32x8 *>(from) : f32x8{};
            for (int i = 0; i < 8; ++i) {
              float t[3];
              terms_of(v[i], t);
              for (int c = 0; c < 3; ++c) x[m][s][c][i] = (__bf16)t[c];
            }
          }
        }
      }
      // what lane group g holds of step s, and the other way round: then step s is the codes k0 + 32 s + 8 g
      const u32x2 a02 = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false));
      const u32x2 a13 = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false));
      const u32x2 b01 = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a02[0], a13[0], false, false));
      const u32x2 b23 = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a02[1], a13[1], false, false));
      const uint32_t words[4] = {b01[0], b01[1], b23[0], b23[1]};
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const bf16x8 b = expand8(words[s], sc[s]);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int c = kTerms - 1; c >= 0; --c) acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[m][s][c], b, acc[m], 0, 0, 0);
      }
    }
    __syncthreads();                             // (the sums of the rows before have been read)
#pragma unroll
    for (int m = 0; m < MT; ++m)
      for (int v = 0; v < 4; ++v) part[wave][m][v][lane] = acc[m][v];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 256; i += kFewWaves * 64) {
      const int m = i / 256, in = i % 256, l = in / 64 * 16 + in % 16, v = in / 16 % 4;       // row 4 (in / 64) + v of the tile, column in % 16
      float sum = 0.0f;
      for (int w = 0; w < kFewWaves; ++w) sum += part[w][m][v][l];
      const int32_t s = m0 + m * 16 + in / 16;
      if (s < r.last && n0 + in % 16 < N) out[(int64_t)s * a.ld_out + n0 + in % 16] = (TO)(sum * alpha);
    }
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------

int64_t divide_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool at(const void *ptr, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }
bool stride_fits(int64_t ld, int64_t width, int64_t rows) {
  return ld >= width && ld <= ((int64_t)1 << 40) / (rows > 0 ? rows : 1);
}
bool sizes_fit(const nvfp4_product_params &p) {
  return p.rows >= 0 && p.rows <= kMostRows && p.inp > 0 && p.inp <= kMostWidth && p.inp % 32 == 0 && p.out > 0 && p.out <= kMostWidth &&
         p.experts > 0 && p.experts <= kMostExperts && p.slots >= 0 && p.slots <= kMostSlots &&
         (!(p.flags & NVFP4_GEMM_B_TILE_SCALES) || p.out % 16 == 0);
}

template <typename T, typename TO>
int run_product(const ProductArgs &a, hipStream_t s) {
  const dim3 grid((uint32_t)divide_up(a.out_width, 16), (uint32_t)(a.experts + (a.begin ? 1 : 0)));
  return launch(k_few<T, TO, 1>, grid, dim3(kFewWaves * 64), 0, s, a);
}

int product(const void *x, const nvfp4_product_params *p, const int32_t *token, const int32_t *begin, const void *codes,
            const void *scales, const float *alpha, void *out, void *stream) {
  if (!stride_fits(p->ld_x, p->inp, p->rows) || !stride_fits(p->ld_out, p->out, p->slots)) return NVFP4_ERR_SHAPE;
  if (!at(x, 16) || !at(token, 4) || !at(begin, 4) || !at(codes, 16) || !at(scales, 16) || !at(alpha, 4) || !at(out, 16) || p->ld_x % 8)
    return NVFP4_ERR_ALIGN;
  if (p->x_dtype > NVFP4_X_F32 || p->out_dtype > NVFP4_OUT_F32 || (p->flags & ~(uint32_t)NVFP4_GEMM_B_TILE_SCALES)) return NVFP4_ERR_PARAM;
  if (p->slots == 0) return NVFP4_OK;
  const ProductArgs a{x, token, begin, static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(scales), alpha, out,
                      p->ld_x, p->ld_out, (int32_t)p->rows, (int32_t)p->slots, (int32_t)p->inp, (int32_t)p->out, (int32_t)p->experts,
                      p->flags & NVFP4_GEMM_B_TILE_SCALES ? 4 : 0};
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool of32 = p->x_dtype == NVFP4_X_F32, to32 = p->out_dtype == NVFP4_OUT_F32;
  return of32 ? to32 ? run_product<float, float>(a, s) : run_product<float, __bf16>(a, s)
              : to32 ? run_product<__bf16, float>(a, s) : run_product<__bf16, __bf16>(a, s);
}

}  // namespace
}  // namespace nvfp4_46

using namespace nvfp4_46;

extern "C" int nvfp4_weight_product(const void *x, const nvfp4_product_params *p, const void *codes, const void *scales,
                                    const float *alpha, void *out, void *stream) {
  if (!p) return NVFP4_ERR_NULL;
  if (!sizes_fit(*p) || p->experts != 1 || p->slots != p->rows) return NVFP4_ERR_SHAPE;
  if (!codes || !scales || !alpha || (p->rows != 0 && (!x || !out))) return NVFP4_ERR_NULL;
  return product(x, p, nullptr, nullptr, codes, scales, alpha, out, stream);
}

extern "C" int nvfp4_experts_product(const void *x, const nvfp4_product_params *p, const int32_t *token, const int32_t *begin,
                                     const void *codes, const void *scales, const float *alpha, void *out, void *stream) {
  if (!p) return NVFP4_ERR_NULL;
  if (!sizes_fit(*p)) return NVFP4_ERR_SHAPE;
  if (!begin || !codes || !scales || !alpha || (p->rows != 0 && !x) || (p->slots != 0 && !out)) return NVFP4_ERR_NULL;
  if (!token && p->slots != p->rows) return NVFP4_ERR_SHAPE;
  return product(x, p, token, begin, codes, scales, alpha, out, stream);
}
