// Activations as they are times a quantized weight, or those of many experts (include/finetune/nvfp4_finetune.h):
//
//   out[s][n] = alpha_e sum_k x[row(s)][k] value(code_e[n][k]) value(scale_e[n][k / 16])
//
// value(code) has two significant bits and value(scale) four: their product is exact in BF16, so that the BF16 matrix instruction multiplies
// exact operands and accumulates in fp32.  fp32 activations are sums of three BF16 terms, a matrix instruction for each.
//
//   k_few      few rows: bound by the codes (0.5625 bytes a weight) and by x, which every workgroup reads from its die's L2
//   k_tiles    tiles of out: bound by the matrix unit, and for large ones by the chip's power
//
// One launch a call.  Among others, on different cards, rows x K x N: 1 x 4096 x 4096 5.2 to 5.6 us (9.4 MB), 24 x 8192 x 8192 11.9 to 12.9 (scales of tiles,
// 33.8 MB of weights; of rows, 37.7 MB, 12.6), 4096 x 8192 x 8192 410 to 447 (1.23 to 1.34 PFLOP/s; a BF16 product of the vendor's library, without a
// weight to expand, 410 to 424), 500 x 4096 x 10001 fp32 155 (three products: 0.8 PFLOP/s); 32 tokens, four each of 64 experts, 2048 to 1024, 15.3 to
// 17.2 (65 MB of weights: 3.8 to 4.2 TB/s), 4096 of 32, 2048 to 4096, 306 to 325 (0.83 to 0.88 PFLOP/s).  fp32 activations and results: 1 x 4096 x 4096 9.1,
// 4 x 8192 x 8192 17.7, 12 x 8192 x 8192 33, 32 tokens of 64 experts as above 35, 4096 of 32 914 (three products: 0.88 PFLOP/s).
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

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

// f(0), f(1), ..., f(N - 1) with the number as a constant
template <int N, typename F>
__device__ __forceinline__ void each_number(F f) {
  if constexpr (N > 0) {
    each_number<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

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
// term is all there is: a weight is finite, so that what the others, 0, add is 0.  Of a NaN the rest is one.
__device__ inline void terms_of(float v, float (&t)[3]) {
  const auto cut = [](float f) { return __uint_as_float(__float_as_uint(f) & 0xffff0000u); };
  t[0] = cut(v);
  const float rest = t[0] == v ? 0.0f : v - t[0];
  t[1] = cut(rest);
  t[2] = rest - t[1];
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

// Byte `i` of four scales.
__device__ inline float scale_of(uint32_t bytes, int i) {
  return i == 0 ? __builtin_amdgcn_cvt_f32_fp8((int)bytes, 0) : i == 1 ? __builtin_amdgcn_cvt_f32_fp8((int)bytes, 1)
       : i == 2 ? __builtin_amdgcn_cvt_f32_fp8((int)bytes, 2) : __builtin_amdgcn_cvt_f32_fp8((int)bytes, 3);
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
// Rows of out that no expert has, numbered through: those in front of the first one's, then those behind the last one's.
struct Others {
  int32_t front, skipped, count;
  __device__ int32_t row(int32_t i) const { return i < front ? i : i + skipped; }
};
__device__ inline Others others_of(const ProductArgs &a) {
  const int32_t front = rows_of(a, 0).first, last = rows_of(a, a.experts - 1).last, behind = last > front ? last : front;
  return {front, behind - front, front + a.slots - behind};
}

// What a lane copies in place of x past the end of K (a weight's scale there is any finite number, so x has to be 0).
__device__ const u32x4 kZeros = {0, 0, 0, 0};

// M0 = LDS byte address of lane 0's piece.  It needs a wait state before a copy reads it.
#define NV_COPY16(lds, address) \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(address) : "memory", "m0")
#define NV_COPY16_AT(lds, offset, base) \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0")
#define NV_COPY2_AT(lds, offset, base) \
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ushort %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0")

__device__ inline const uint8_t *uniform(const uint8_t *p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const uint8_t *>(((uint64_t)hi << 32) | lo);
}

// ---- k_few --------------------------------------------------------------------------------------------------------------

// Few rows: bound by the codes, which pass through a compute unit once.  A workgroup has 32 columns of out and an expert's rows, XR of them at a time; its W
// waves share K, every W-th chunk of 256 each, and their sums meet in LDS.  A wave copies its chunks into a ring of NST stages of its own, eight
// neighbouring lanes a column's 128 bytes of codes, 16 bytes of scales a lane (WHOLE: K is a multiple of 256; else two bytes at a time), two rows (one
// of fp32) of x at a time, as many as there are.  Loads straight to registers, as the matrix instruction wants its operands, are 64 requests of 16
// bytes each and took as long without any arithmetic: 8192 x 8192, one row 13.6 us (loads alone) to 14.4, 16 rows 18.3; through these copies 10.1 and 13.7
// (the shapes that run_product names are the best of nine, by rows).
template <typename T_, int XR_, int W_, int NST_, bool WHOLE_>
struct FewShape {
  typedef T_ T;
  static constexpr int XR = XR_, W = W_, NST = NST_;
  static constexpr bool WHOLE = WHOLE_;
  static constexpr int UX = 256 * (int)sizeof(T) / 16, RX = 64 / UX, NX = XR / RX;         // units of a row of x; rows of a copy; copies
  static constexpr int NS = WHOLE ? 1 : 4, kOthers = 4 + NS;
  static constexpr uint32_t kScales = 32 * 128, kX = kScales + (WHOLE ? 512 : 1024), kStage = kX + XR * UX * 16;
  static constexpr uint32_t kLds = W * NST * kStage;
  static_assert(XR <= 16 && XR % RX == 0 && kLds >= W * 2048 && kLds <= 160 * 1024 && (NST - 1) * (kOthers + NX) < 63, "");
};

template <typename S, typename TO>
__global__ void __launch_bounds__(S::W * 64) k_few(ProductArgs a) {
  typedef typename S::T T;
  constexpr int kTerms = sizeof(T) == 4 ? 3 : 1, XR = S::XR, W = S::W, NST = S::NST, UX = S::UX, RX = S::RX, NX = S::NX;
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ uint8_t is_row[16];                 // 0: the token is none of x's rows
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), line = lane & 15, group = lane / 16;
  const int32_t e = (int32_t)blockIdx.y, n0 = (int32_t)blockIdx.x * 32, N = a.out_width, K = a.inp;
  TO *const out = static_cast<TO *>(a.out) + n0;
  const int32_t rows_n = N - n0 < 32 ? N - n0 : 32;
  const bool none = e == a.experts;              // the rows that no expert has
  const Rows r = none ? Rows{0, 0} : rows_of(a, e);
  if (none || a.rows == 0) {
    const Others o = none ? others_of(a) : Others{0, r.first, r.last - r.first};
    for (int32_t i = (int32_t)(blockIdx.z * (W * 2) + threadIdx.x / 32); i < o.count; i += (int32_t)gridDim.z * (W * 2))
      if ((int32_t)threadIdx.x % 32 < rows_n) out[(int64_t)o.row(i) * a.ld_out + threadIdx.x % 32] = (TO)0.0f;
    return;
  }
  if (r.first >= r.last) return;
  const int32_t row_codes = K / 2, row_scales = K / 16, chunks = (K + 255) / 256;
  const uint8_t *const codes = uniform(a.codes + ((int64_t)e * N + n0) * row_codes);
  const uint8_t *const scales = uniform(a.scales + ((int64_t)e * (N >> a.scale_shift) + (n0 >> a.scale_shift)) * row_scales);
  const float alpha = a.alpha[e];
  const uint8_t *const own = lds + wave * (NST * S::kStage);
  const uint32_t own_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds + wave * (NST * S::kStage);
  for (int32_t m0 = r.first + (int32_t)blockIdx.z * XR; m0 < r.last; m0 += (int32_t)gridDim.z * XR) {
    const int32_t rows_m = r.last - m0 < XR ? r.last - m0 : XR, nx = (rows_m + RX - 1) / RX;
    // ---- where a lane's copies come from.  Unit u of a column stands at the place u ^ (column / 2 % 8), unit u of a row of x at u ^ (row % 16), so that
    // sixteen lanes that read a unit of sixteen lines meet all banks.
    uint32_t at_c[4], at_s[S::NS];
    const uint8_t *from_x[NX];
    const auto offsets = [&](uint32_t last) __attribute__((always_inline)) {     // units past `last` give that one instead
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t n = i * 8 + lane / 8, have = (int32_t)n < rows_n ? n : (uint32_t)rows_n - 1, u = lane % 8 ^ (n >> 1 & 7);
        at_c[i] = have * (uint32_t)row_codes + (u < last ? u : last) * 16;
        if constexpr (!S::WHOLE) at_s[i] = (have >> a.scale_shift) * (uint32_t)row_scales + ((uint32_t)lane % 8 < last ? lane % 8 : last) * 2;
      }
      if constexpr (S::WHOLE) at_s[0] = (uint32_t)((lane & 31) < rows_n ? lane & 31 : rows_n - 1) >> a.scale_shift, at_s[0] *= (uint32_t)row_scales;
    };
    offsets(7);
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const int32_t m = i * RX + lane / UX, s = m0 + (m < rows_m ? m : rows_m - 1), from = a.token ? a.token[s] : s;
      const bool is = from >= 0 && from < a.rows;
      from_x[i] = reinterpret_cast<const uint8_t *>(static_cast<const T *>(a.x) + (is ? from : 0) * a.ld_x) + (lane % UX ^ (m & 15)) * 16;
      if (wave == 0 && lane % UX == 0) is_row[m] = is;
    }
    const auto copy_chunk = [&](int32_t c, uint32_t stage) __attribute__((always_inline)) {
      const uint32_t to = own_at + stage * S::kStage;
      if (!S::WHOLE && c == chunks - 1) {
        const uint32_t left = (uint32_t)(K - c * 256) / 32;
        offsets(left - 1);
#pragma unroll
        for (int i = 0; i < NX; ++i) {
          const uint32_t u = lane % UX ^ ((i * RX + lane / UX) & 15);
          if (u >= left * (32 * sizeof(T) / 16)) from_x[i] = reinterpret_cast<const uint8_t *>(&kZeros) - (int64_t)c * (256 * sizeof(T));
        }
      }
      const uint8_t *const c_at = codes + c * 128, *const s_at = scales + c * 16;
#pragma unroll
      for (int i = 0; i < 4; ++i) NV_COPY16_AT(to + i * 1024, at_c[i], c_at);
      if constexpr (S::WHOLE) {
        if (lane < 32) NV_COPY16_AT(to + S::kScales, at_s[0], s_at);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) NV_COPY2_AT(to + S::kScales + i * 256, at_s[i], s_at);
      }
#pragma unroll
      for (int i = 0; i < NX; ++i)
        if (i < nx) {
          const uint8_t *const from = from_x[i] + (int64_t)c * (256 * sizeof(T));
          NV_COPY16(to + S::kX + i * 1024, from);
        }
    };
    // until but the copies of `young` stages have landed
    const auto wait = [&](auto young) __attribute__((always_inline)) {
      constexpr int n = decltype(young)::value;
      if constexpr (n == 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      else
        each_number<NX>([&](auto i) __attribute__((always_inline)) {
          if (nx == decltype(i)::value + 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n * (S::kOthers + decltype(i)::value + 1)) : "memory");
        });
    };
    f32x4 acc[2] = {};
    // lane group g has the codes 64 g .. 64 g + 63 of a column's chunk, step s of eight of them
    const auto multiply = [&](uint32_t stage, auto after) __attribute__((always_inline)) {
      const uint8_t *const st = own + stage * S::kStage;
      u32x4 raw[2][2];
      uint32_t sc[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t n = j * 16 + line;
#pragma unroll
        for (int q = 0; q < 2; ++q) raw[j][q] = *reinterpret_cast<const u32x4 *>(st + n * 128 + ((2 * group + q) ^ (n >> 1 & 7)) * 16);
        if constexpr (S::WHOLE) {
          sc[j] = *reinterpret_cast<const uint32_t *>(st + S::kScales + n * 16 + 4 * group);
        } else {
          const u32x2 s = *reinterpret_cast<const u32x2 *>(st + S::kScales + n * 32 + 8 * group);
          sc[j] = __builtin_amdgcn_perm(s[1], s[0], 0x05040100u);
        }
      }
      T x[8][8];
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        const uint8_t *const row = st + S::kX + (line % XR) * (UX * 16);
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
          const uint32_t u = (group * 8 + s) * (sizeof(T) / 2) + h;
          *reinterpret_cast<u32x4 *>(&x[s][h * (16 / sizeof(T))]) = *reinterpret_cast<const u32x4 *>(row + (u ^ (line % XR)) * 16);
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      after();
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        bf16x8 xs[kTerms];
        if constexpr (kTerms == 1) {
          xs[0] = *reinterpret_cast<bf16x8 *>(&x[s][0]);
        } else {
          u32x4 w[3];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float lo[3], hi[3];
            terms_of(x[s][2 * k], lo);
            terms_of(x[s][2 * k + 1], hi);
            for (int c = 0; c < 3; ++c) w[c][k] = pack_exact(lo[c], hi[c]);
          }
          for (int c = 0; c < 3; ++c) xs[c] = __builtin_bit_cast(bf16x8, w[c]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const bf16x8 b = expand8(raw[j][s / 4][s % 4], scale_of(sc[j], s / 2));
#pragma unroll
          for (int c = kTerms - 1; c >= 0; --c) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xs[c], b, acc[j], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    int32_t c = wave;
    uint32_t stage = 0;
#pragma unroll
    for (int p = 0; p < NST; ++p)
      if (c + W * p < chunks) copy_chunk(c + W * p, p);
    const auto step = [&](auto after) __attribute__((always_inline)) {
      multiply(stage, after);
      c += W;
      stage = stage + 1 == (uint32_t)NST ? 0u : stage + 1;
    };
    while (c + W * NST < chunks) {
      wait(std::integral_constant<int, NST - 1>{});
      step([&] { copy_chunk(c + W * NST, stage); });
    }
    // the last NST, with nothing left to copy
    each_number<NST>([&](auto p) __attribute__((always_inline)) {
      constexpr int young = NST - 1 - decltype(p)::value;
      if (c + W * young < chunks && c < chunks) {
        wait(std::integral_constant<int, young>{});
        step([] {});
      }
    });
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                             // (no wave's stages are read any more)
    float(*const part)[2][4][64] = reinterpret_cast<float(*)[2][4][64]>(lds);
#pragma unroll
    for (int j = 0; j < 2; ++j)
      for (int v = 0; v < 4; ++v) part[wave][j][v][lane] = acc[j][v];
    __syncthreads();
    for (int i = threadIdx.x; i < rows_m * 32; i += W * 64) {
      const int n = i % 32, m = i / 32, l = m / 4 * 16 + n % 16;
      float sum = 0.0f;
      for (int w = 0; w < W; ++w) sum += part[w][n / 16][m % 4][l];
      if (n < rows_n) out[(int64_t)(m0 + m) * a.ld_out + n] = (TO)(is_row[m] ? sum * alpha : 0.0f);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (the counts above are of copies alone)
    __syncthreads();                             // before the next rows are copied there
  }
}

// ---- k_tiles ------------------------------------------------------------------------------------------------------------

// A workgroup's tile of out is BM x BN; SM x SN waves hold WM x WN tiles of the matrix instruction (32 x 32) each, in KS copies that share K: copy kg
// takes 64 of every chunk of 64 KS.  NST chunks of x, codes and scales are in LDS or on their way there.
//
// What bounds it.  A step of 16 of K is WM WN matrix instructions of 32 cycles and 17 vector instructions for each of WN fragments of the weight (four
// conversions, eight multiplications, four packings, a scale; of fp32 also 60 for each of WM fragments of x); they overlap where the program
// interleaves them: without, a turn of 256 x 256 at K = 8192 took 182 us, so 160, with two waves to a SIMD 144.  (Timing only, of the 160: with the weight not
// expanded 155, without copies 144, neither 135; the matrix instructions alone would take 109 at 2.4 GHz.)  Of a full chip power is the bound:
// 410 to 447 us for 4096 x 8192 x 8192, on different cards.  For short K what comes before and after the loop counts: finding the tile, the first chunks,
// the sums' way out, 7 to 15 us a turn of large tiles.
template <typename T_, int WM_, int WN_, int SM_, int SN_, int KS_, int NST_>
struct Shape {
  typedef T_ T;
  static constexpr int WM = WM_, WN = WN_, SM = SM_, SN = SN_, KS = KS_, NST = NST_;
  static constexpr int kWaves = SM * SN * KS, kThreads = 64 * kWaves, BM = 32 * WM * SM, BN = 32 * WN * SN, CK = 64 * KS;
  static constexpr int UA = CK * (int)sizeof(T) / 16, UB = CK / 32;       // 16-byte units of a row of x, of codes (= pairs of scales)
  static constexpr uint32_t kCodes = BM * UA * 16, kScales = kCodes + BN * UB * 16, kStage = kScales + BN * UB * 4;
  static constexpr int NA = BM * UA / 64 / kWaves, NB = BN * UB / 64 / kWaves, kCopies = NA + 2 * NB;     // copy instructions of a wave
  // the sums on their way out, 32 rows of every wave at a time: floats from row to row, of a wave by itself where it has all of K, else of all of them
  static constexpr int kPitch = KS == 1 ? 32 * WN + 4 : BN + 4;
  static constexpr uint32_t kSums = (KS == 1 ? SM * SN : KS * SM) * 32 * kPitch * 4;
  static constexpr uint32_t kLds = NST * kStage > kSums ? NST * kStage : kSums;
  static_assert(BM * UA % (64 * kWaves) == 0 && BN * UB % (64 * kWaves) == 0 && 64 % UA == 0 && 64 % UB == 0, "whole copies");
  static_assert(kLds <= 160 * 1024 && (NST - 2) * kCopies < 63, "LDS; vmcnt counts to 63");
};

// A tile's rows: of expert e, or (e = experts) numbers of those that no expert has.
struct Unit {
  int32_t e, first, last;
};

// Which tile this workgroup has; last <= first: none.  Workgroups go to the eight dies in turn and each die has its own L2: every die takes an
// adjacent eighth of the tiles that there are, a row of tiles one after the other.
template <int BM, int THREADS>
__device__ inline Unit unit_of(const ProductArgs &a, int32_t tiles_n, int32_t &n) {
  __shared__ int32_t sums[THREADS / 64];
  __shared__ Unit found;
  int32_t units;
  const auto tile_of = [&](int32_t &unit) {
    const int64_t all = (int64_t)units * tiles_n;
    const int32_t share = (int32_t)((all + 7) / 8), seq = (int32_t)(blockIdx.x >> 3);
    const int64_t tile = (int64_t)(blockIdx.x & 7) * share + seq;
    if (seq >= share || tile >= all) return false;
    unit = (int32_t)(tile / tiles_n);
    n = (int32_t)(tile % tiles_n);
    return true;
  };
  if (!a.begin) {
    units = (a.slots + BM - 1) / BM;
    int32_t unit;
    if (!tile_of(unit)) return {0, 0, 0};
    return {0, unit * BM, a.slots - unit * BM < BM ? a.slots : (unit + 1) * BM};
  }
  // experts one after the other, each thread adjacent ones, the rows that none has as one more
  const int32_t groups = a.experts + 1, per = (groups + THREADS - 1) / THREADS, g0 = (int32_t)threadIdx.x * per;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const auto rows = [&](int32_t g) -> Rows {
    if (g < a.experts) return rows_of(a, g);
    return {0, others_of(a).count};
  };
  int32_t mine = 0;
  for (int32_t g = g0; g < g0 + per && g < groups; ++g) {
    const Rows r = rows(g);
    mine += (r.last - r.first + BM - 1) / BM;
  }
  int32_t upto = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const int32_t other = __shfl_up(upto, d);
    if (lane >= d) upto += other;
  }
  if (lane == 63) sums[wave] = upto;
  if (threadIdx.x == 0) found = {0, 0, 0};
  __syncthreads();
  int32_t before = upto - mine, unit;
  units = 0;
  for (int w = 0; w < THREADS / 64; ++w) {
    if (w < wave) before += sums[w];
    units += sums[w];
  }
  const bool any = tile_of(unit);
  for (int32_t g = g0; any && g < g0 + per && g < groups; ++g) {
    const Rows r = rows(g);
    const int32_t tiles = (r.last - r.first + BM - 1) / BM, t = unit - before;
    if (t >= 0 && t < tiles) found = {g, r.first + t * BM, r.last - r.first - t * BM < BM ? r.last : r.first + (t + 1) * BM};
    before += tiles;
  }
  __syncthreads();
  return found;
}

template <typename S, typename TO>
__global__ void __launch_bounds__(S::kThreads, 1) k_tiles(ProductArgs a, int32_t tiles_n) {
  typedef typename S::T T;
  typedef float f32x16 __attribute__((ext_vector_type(16)));
  constexpr int WM = S::WM, WN = S::WN, UA = S::UA, UB = S::UB, NA = S::NA, NB = S::NB, kTerms = sizeof(T) == 4 ? 3 : 1;
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ uint8_t is_row[S::BM];              // 0: the token is none of x's rows
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), line = lane & 31, half = lane / 32;
  const int kg = wave / (S::SM * S::SN), wm = wave / S::SN % S::SM, wn = wave % S::SN;
  int32_t tile_n;
  const Unit unit = unit_of<S::BM, S::kThreads>(a, tiles_n, tile_n);
  if (unit.last <= unit.first) return;
  const int32_t N = a.out_width, K = a.inp, n0 = tile_n * S::BN, rows_m = unit.last - unit.first;
  const int32_t rows_n = N - n0 < S::BN ? N - n0 : S::BN;
  if (unit.e == a.experts) {
    // (a begin that falls can make the count of tiles pass 32 bits and several threads find this one: only rows that there are)
    const Others o = others_of(a);
    TO *const rest = static_cast<TO *>(a.out) + n0;
    for (int32_t i = threadIdx.x; i < S::BM * S::BN; i += S::kThreads) {
      const int32_t m = i / S::BN, n = i % S::BN;
      if (m < rows_m && m < o.count - unit.first && n < rows_n) rest[(int64_t)o.row(unit.first + m) * a.ld_out + n] = (TO)0.0f;
    }
    return;
  }
  TO *const out = static_cast<TO *>(a.out) + (int64_t)unit.first * a.ld_out + n0;
  const auto row_of = [&](int32_t m) {           // of x; -1: none
    const int32_t s = unit.first + (m < rows_m ? m : rows_m - 1), from = a.token ? a.token[s] : s;
    return from >= 0 && from < a.rows ? from : -1;
  };
  for (int32_t m = threadIdx.x; m < S::BM; m += S::kThreads) is_row[m] = row_of(m) >= 0;
  const float alpha = a.alpha[unit.e];

  // ---- where a lane's copies come from.  Unit u of a row stands at the place u ^ swz(row), so that sixteen lanes that read a unit of sixteen
  // rows meet all banks.
  const auto swz_a = [](uint32_t row) { return UA == 8 ? row >> 1 & 7 : row & 15; };
  const auto swz_b = [](uint32_t row) { return row / (16 / UB) & (UB - 1); };
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
  const int32_t row_codes = K / 2, row_scales = K / 16;
  const uint8_t *from_a[NA];
  uint32_t unit_a[NA], at_b[NB], at_s[NB];
#pragma unroll
  for (int i = 0; i < NA; ++i) {
    const uint32_t row = ((wave + S::kWaves * i) * 64 + lane) / UA, u = lane % UA ^ swz_a(row);
    const int32_t r = row_of((int32_t)row);
    from_a[i] = reinterpret_cast<const uint8_t *>(static_cast<const T *>(a.x) + (int64_t)(r < 0 ? 0 : r) * a.ld_x) + u * 16;
    unit_a[i] = u;
  }
  const auto offsets = [&](uint32_t last) __attribute__((always_inline)) {       // units past `last` give that one instead
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const uint32_t row = ((wave + S::kWaves * i) * 64 + lane) / UB, have = (int32_t)row < rows_n ? row : (uint32_t)rows_n - 1;
      uint32_t u = lane % UB ^ swz_b(row);
      u = u < last ? u : last;
      at_b[i] = have * (uint32_t)row_codes + u * 16;
      at_s[i] = (have >> a.scale_shift) * (uint32_t)row_scales + u * 2;
    }
  };
  const uint8_t *const codes = uniform(a.codes + ((int64_t)unit.e * N + n0) * row_codes);
  const uint8_t *const scales = uniform(a.scales + ((int64_t)unit.e * (N >> a.scale_shift) + (n0 >> a.scale_shift)) * row_scales);
  const int32_t chunks = (K + S::CK - 1) / S::CK;
  const bool ragged = K % S::CK != 0;
  const auto last_chunk = [&](int32_t c) __attribute__((always_inline)) {        // before the copies of chunk c
    if (!ragged || c != chunks - 1) return;
    const uint32_t left = (uint32_t)(K - c * S::CK) / 32;
    offsets(left - 1);
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (unit_a[i] >= left * (32 * sizeof(T) / 16)) from_a[i] = reinterpret_cast<const uint8_t *>(&kZeros) - (int64_t)c * (S::CK * sizeof(T));
  };
  const auto copy = [&](int32_t c, uint32_t stage, auto number) __attribute__((always_inline)) {
    constexpr int i = decltype(number)::value;
    const uint32_t to = lds0 + stage * S::kStage;
    if constexpr (i < NA) {
      const uint8_t *const from = from_a[i] + (int64_t)c * (S::CK * sizeof(T));
      NV_COPY16(to + (wave + S::kWaves * i) * 1024, from);
    } else if constexpr (i < NA + NB) {
      const uint32_t offset = at_b[i - NA];
      const uint8_t *const base = codes + c * (S::CK / 2);
      NV_COPY16_AT(to + S::kCodes + (wave + S::kWaves * (i - NA)) * 1024, offset, base);
    } else {
      const uint32_t offset = at_s[i - NA - NB];
      const uint8_t *const base = scales + c * (S::CK / 16);
      NV_COPY2_AT(to + S::kScales + (wave + S::kWaves * (i - NA - NB)) * 256, offset, base);
    }
  };
  const auto clamp = [&](int32_t c) { return __builtin_amdgcn_readfirstlane(c < chunks ? c : chunks - 1); };

  // ---- what a lane reads of a chunk: 32 codes of a column, k = 32 half + 0 .. 31 of the wave's 64, their two scales, and in step s x of k = 32 half + 8 s
  u32x4 raw[WN];
  uint32_t raw_scales[WN];
  bf16x8 fb[2][WN], fa[2][WM][kTerms];
  const auto read_b = [&](uint32_t stage, int j) __attribute__((always_inline)) {
    const uint32_t row = (wn * WN + j) * 32 + line, u = (kg * 2 + half) ^ swz_b(row);
    const uint8_t *const at = lds + stage * S::kStage;
    raw[j] = *reinterpret_cast<const u32x4 *>(at + S::kCodes + (row * UB + u) * 16);
    raw_scales[j] = *reinterpret_cast<const uint32_t *>(at + S::kScales + (row * UB + u) * 4);
  };
  const auto expand_b = [&](int s, int j) __attribute__((always_inline)) {
    fb[s & 1][j] = expand8(raw[j][s], scale_of(raw_scales[j], s / 2));
  };
  const auto read_a = [&](uint32_t stage, int s, int i) __attribute__((always_inline)) {
    const uint32_t row = (wm * WM + i) * 32 + line;
    const uint8_t *const at = lds + stage * S::kStage + row * (UA * 16);
    if constexpr (kTerms == 1) {
      fa[s & 1][i][0] = *reinterpret_cast<const bf16x8 *>(at + ((kg * 8 + half * 4 + s) ^ swz_a(row)) * 16);
    } else {
      const uint32_t u = kg * 16 + half * 8 + s * 2;
      const f32x4 v[2] = {*reinterpret_cast<const f32x4 *>(at + (u ^ swz_a(row)) * 16),
                          *reinterpret_cast<const f32x4 *>(at + ((u + 1) ^ swz_a(row)) * 16)};
      u32x4 w[3];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float lo[3], hi[3];
        terms_of(v[k / 2][k % 2 * 2], lo);
        terms_of(v[k / 2][k % 2 * 2 + 1], hi);
        for (int c = 0; c < 3; ++c) w[c][k] = pack_exact(lo[c], hi[c]);
      }
      for (int c = 0; c < 3; ++c) fa[s & 1][i][c] = __builtin_bit_cast(bf16x8, w[c]);
    }
  };

  f32x16 acc[WM][WN] = {};
  offsets(UB - 1);
#pragma unroll 1
  for (int32_t c = 0; c < S::NST - 1; ++c) {
    last_chunk(clamp(c));
    each_number<S::kCopies>([&](auto i) __attribute__((always_inline)) { copy(clamp(c), c, i); });
  }
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((S::NST - 2) * S::kCopies) : "memory");
#pragma unroll
  for (int j = 0; j < WN; ++j) read_b(0, j);
#pragma unroll
  for (int i = 0; i < WM; ++i) read_a(0, 0, i);
#pragma unroll
  for (int j = 0; j < WN; ++j) expand_b(0, j);
  // Chunk c stands in stage c % NST.  In its first three steps of four the copies of chunk c + NST - 1 start, into the stage of chunk c - 1, which every
  // wave had read when it came to the barrier of chunk c - 1.  In the last step all waves meet, with chunk c + 1 there, and begin to read it.
  uint32_t stage = 0, freed = S::NST - 1;
#pragma unroll 1
  for (int32_t c = 0; c < chunks; ++c) {
    const uint32_t next = stage + 1 == (uint32_t)S::NST ? 0u : stage + 1;
    const int32_t ahead = clamp(c + S::NST - 1);
    if (c + S::NST - 1 == chunks - 1) last_chunk(ahead);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s == 3) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S::NST - 2) * S::kCopies) : "memory");
      const auto multiply = [&](int i, int j) __attribute__((always_inline)) {
#pragma unroll
        for (int t = kTerms - 1; t >= 0; --t)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[s & 1][j], fa[s & 1][i][t], acc[i][j], 0, 0, 0);
      };
      if constexpr (kTerms == 1 && WM * WN >= 8) {
        // A part of the step for every column tile, its instructions told apart: the expansion of the next step's fragment between the matrix
        // instructions of this one.
#pragma unroll
        for (int j = 0; j < WN; ++j) {
          if (s < 3)
            each_number<S::kCopies>([&](auto i) __attribute__((always_inline)) {
              if (decltype(i)::value * (3 * WN) / S::kCopies == s * WN + j) copy(ahead, freed, i);
            });
          __builtin_amdgcn_sched_barrier(0);
          int reads = 0;
          if (s == 3 && j == 0) {
#pragma unroll
            for (int b = 0; b < WN; ++b) read_b(next, b);
            ++reads;
          }
          // (all of the rows' pieces with the first column: the next step begins with them)
#pragma unroll
          for (int i = j * 2; i < WM && i < j * 2 + 2; ++i) {
            read_a(s == 3 ? next : stage, (s + 1) & 3, i);
            ++reads;
          }
          // in the last step a column later, when its codes have come
          if (s < 3) expand_b((s + 1) & 3, j);
          else if (j > 0) expand_b(0, j - 1);
          if (s == 3 && j == WN - 1) expand_b(0, j);
#pragma unroll
          for (int i = 0; i < WM; ++i) multiply(i, j);
          if (reads) __builtin_amdgcn_sched_group_barrier(0x100, 16, 0);
          constexpr int kEach = (20 + WM - 1) / WM;
          const int each = s == 3 && j == WN - 1 ? 2 * kEach : kEach;
#pragma unroll
          for (int i = 0; i < WM; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (each == kEach) __builtin_amdgcn_sched_group_barrier(0x002, kEach, 0);
            else __builtin_amdgcn_sched_group_barrier(0x002, 2 * kEach, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
        if (s == 3) {
#pragma unroll
          for (int j = 0; j < WN; ++j) read_b(next, j);
        } else {
          each_number<S::kCopies>([&](auto i) __attribute__((always_inline)) {
            if (decltype(i)::value * 3 / S::kCopies == s) copy(ahead, freed, i);
          });
        }
#pragma unroll
        for (int i = 0; i < WM; ++i) read_a(s == 3 ? next : stage, (s + 1) & 3, i);
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
          for (int j = 0; j < WN; ++j) multiply(i, j);
#pragma unroll
        for (int j = 0; j < WN; ++j) expand_b((s + 1) & 3, j);
        if constexpr (kTerms == 3) {             // (the next step's terms and fragments among this one's matrix instructions)
          constexpr int kAll = 3 * WM * WN, kEach = (64 * WM + 20 * WN + kAll - 1) / kAll;
          __builtin_amdgcn_sched_group_barrier(0x100, 2 * WM + 2 * WN, 0);
#pragma unroll
          for (int q = 0; q < kAll; ++q) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, kEach, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    freed = stage;
    stage = next;
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

  // ---- sums -> LDS -> out, 32 rows of every wave at a time: the operands were exchanged in the matrix instruction, so that four
  // accumulators are adjacent columns
  constexpr int G = sizeof(TO) == 4 ? 4 : 8;
  float *const sums = reinterpret_cast<float *>(lds);
  const auto put = [&](float *to, int pitch, int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < WN; ++j)
#pragma unroll
      for (int v = 0; v < 16; v += 4)
        *reinterpret_cast<f32x4 *>(to + line * pitch + j * 32 + 2 * v + 4 * half) =
            f32x4{acc[i][j][v], acc[i][j][v + 1], acc[i][j][v + 2], acc[i][j][v + 3]};
  };
  // G columns of row m, times alpha (lines of out begin wherever its stride puts them)
  const auto store = [&](int32_t m, int32_t col, const f32x4 (&v)[G / 4]) __attribute__((always_inline)) {
    if (m >= rows_m || col >= rows_n) return;
    typedef TO piece_of __attribute__((ext_vector_type(G)));
    typedef piece_of piece_anywhere __attribute__((aligned(sizeof(TO))));
    TO *const to = out + (int64_t)m * a.ld_out + col;
    const bool is = is_row[m];
    piece_of p;
    for (int g = 0; g < G; ++g) p[g] = (TO)(is ? v[g / 4][g % 4] * alpha : 0.0f);
    if (col + G <= rows_n) *reinterpret_cast<piece_anywhere *>(to) = p;
    else
      for (int g = 0; g < G; ++g)
        if (col + g < rows_n) to[g] = p[g];
  };
  if constexpr (S::KS == 1) {                    // a wave by itself, without barriers: its LDS instructions run in their order
    constexpr int kPitch = S::kPitch, kAcross = 32 * WN / G;
    float *const own = sums + wave * (32 * kPitch);
#pragma unroll
    for (int i = 0; i < WM; ++i) {
      put(own, kPitch, i);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 4
      for (int piece = lane; piece < 32 * kAcross; piece += 64) {
        const int in = piece / kAcross, col = piece % kAcross * G;
        f32x4 v[G / 4];
        for (int g = 0; g < G / 4; ++g) v[g] = *reinterpret_cast<const f32x4 *>(own + in * kPitch + col + 4 * g);
        store((wm * WM + i) * 32 + in, wn * (32 * WN) + col, v);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  } else {
    constexpr int kRows = 32 * S::SM, kPieces = kRows * S::BN / G;
#pragma unroll
    for (int i = 0; i < WM; ++i) {
      if (i) __syncthreads();
      put(sums + (kg * kRows + wm * 32) * S::kPitch + wn * (32 * WN), S::kPitch, i);
      __syncthreads();
#pragma unroll 2
      for (int piece = (int)threadIdx.x; piece < kPieces; piece += S::kThreads) {
        const int in = piece / (S::BN / G), col = piece % (S::BN / G) * G;
        f32x4 v[G / 4] = {};
        for (int k = 0; k < S::KS; ++k)
          for (int g = 0; g < G / 4; ++g) v[g] += *reinterpret_cast<const f32x4 *>(sums + (k * kRows + in) * S::kPitch + col + 4 * g);
        store(in / 32 * (32 * WM) + i * 32 + in % 32, col, v);
      }
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

// ---- which kernel -----------------------------------------------------------------------------------------------------------
//
// Sizes here are rows x N x K, of several experts rows, then N x K.
// Few rows for each expert: k_few, whose passes over an expert's weight stand one after the other, so that the rows of a pass decide.  (us, BF16, rows of
// a pass 4 / 8 / 16: 1 x 4096 x 4096 5.4 / 6.1 / 5.9, 4 x 15376 x 3584 9.3 / 10.3 / 11.8, 8 x 28672 x 4096 28 / 18.3 / 24, 16 x 8192 x 8192 30 / 19.6 / 13.7; 32
// tokens of 4 among 64 experts, 1024 x 2048, 17.9 / 16.7 / 25.7.  Against the best tiles: 16 x 8192 x 8192 13.7 / 14, 28 x 480 x 512 5.4 / 4.8, 96 rows of 8
// experts, 1024 x 2560, 7.3 / 11.2; but 200 of 32, 3216 x 256, 20 / 17.7 and 1024 of 64, 1024 x 2048, 54 / 34.5.)
// Else k_tiles in the shape that takes least by the estimate below: turns of tiles over the 256 compute units, each a + f microseconds for 1024 of K and
// besides.  The constants are fitted to 230 products, up to 8192 tokens, K 256 to 8192, up to 16384 columns, 1 to 128 experts (uneven), each
// in all shapes: the choice is 2.2 % (fp32: 0.4 %) slower than the best of each on average.  (us at K = 8192 for up to one turn / 4096 x 8192 x 8192, BF16: 32 x 32
// 14 / 1374, 64 x 32 23 / 1112, 64 x 64 30 / 835, 64 x 128 47.5 / 740, 128 x 128 55 to 70 / 510, 128 x 256 100 / 448, in two parts of K
// 84 / 450, 256 x 256 144 / 411 to 428.  A wave of 128 x 64 expands least and leaves room for a second one on its SIMD: waves of 128 x 128 one by one took 160 /
// 418 to 435, of 64 x 128 in tiles of 128 x 256 122 / 505.)
// (K: in two parts of K)
enum Kernel { kFew4, kFew8, kFew16, kTile32, kTile64x32, kTile64, kTile64x128, kTile64x256, kTile64x256K, kTile128, kTile128x256, kTile128x256K,
              kTile256 };

struct Cost {
  Kernel kernel;
  int32_t rows, columns;
  bool pair;                   // two workgroups fit a compute unit's LDS: then the last turn costs half of what is missing in it, else all
  double a, f;                 // us a turn: for 1024 of K, and besides
};
constexpr Cost kCostBf16[] = {{kTile32, 32, 32, false, 0.96, 3.8},       {kTile64x32, 64, 32, false, 1.86, 3.7},
                              {kTile64, 64, 64, false, 3.02, 4.3},       {kTile64x128, 64, 128, false, 5.7, 4.5},
                              {kTile128, 128, 128, false, 7.3, 6.5},     {kTile128x256K, 128, 256, false, 12.0, 8.7},
                              {kTile128x256, 128, 256, true, 12.6, 6.8}, {kTile256, 256, 256, false, 21.4, 15.0}};
constexpr Cost kCostF32[] = {{kTile32, 32, 32, true, 3.5, 2.7},          {kTile64, 64, 64, false, 8.6, 5.3},
                             {kTile64x128, 64, 128, false, 14.1, 5.9},   {kTile64x256K, 64, 256, false, 19.9, 8.3},
                             {kTile64x256, 64, 256, true, 24.1, 7.8},    {kTile128x256, 128, 256, false, 39.2, 10.5}};

// (of several experts' tiles, whose number follows from what the router did, a tenth more may well begin another turn)
double turns_of(double tiles, bool pair, bool several) {
  const double t = tiles / 256, whole = std::ceil(several ? 1.1 * t : t);
  return whole <= 1 ? 1 : pair ? (t + whole) / 2 : whole;
}
// Tiles down the rows: half a tile of every expert's is empty on average, and each that has rows has one.
double tiles_down(const ProductArgs &a, int32_t rows) {
  if (a.experts == 1) return (double)divide_up(a.slots, rows);
  const double used = a.experts < a.slots ? a.experts : a.slots, more = (double)a.slots / rows - used / 2;
  return used + (more > 0 ? more : 0);
}
template <int N>
Kernel least(const ProductArgs &a, const Cost (&costs)[N]) {
  Kernel best = costs[0].kernel;
  double least = 1e300;
  for (const Cost &c : costs) {
    const double us = turns_of(tiles_down(a, c.rows) * (double)divide_up(a.out_width, c.columns), c.pair, a.experts > 1) * (c.a * a.inp / 1024 + c.f);
    if (us < least) least = us, best = c.kernel;
  }
  return best;
}
// (of fp32 rows half as many stand in a stage)
Kernel choose(const ProductArgs &a, bool f32) {
  if (a.rows == 0) return kFew4;                 // (out is 0)
  const int64_t used = a.experts < a.slots ? a.experts : a.slots, wide = a.experts * divide_up(a.out_width, 32);
  if (a.experts == 1) {
    if (a.slots <= (f32 ? 2 : 4)) return kFew4;
    if (!f32 && a.slots <= 8) return kFew8;
    if (a.slots <= (f32 ? 12 : 16)) return kFew16;
  } else if (a.inp > 512 || used * divide_up(a.out_width, 32) < 2048) {
    // (else thousands of workgroups with a chunk or two for each wave: 512 rows of 128 experts, 2048 x 512, 45 us, in tiles of 128 x 256 35; 1024 x 2048 44 / 59)
    if (a.slots <= (f32 ? used * 5 / 2 : used * 4)) return kFew8;
    if (a.slots <= (f32 ? used * 8 : used * 16) && wide <= 512) return kFew16;
  }
  return f32 ? least(a, kCostF32) : least(a, kCostBf16);
}

template <typename S, typename TO>
int run_few_of(const ProductArgs &a, hipStream_t s) {
  // More workgroups where one expert may have hundreds of rows, though the others then have few: 1024 rows of one among 256 would be 128 passes of a
  // workgroup's.  Those without a row end at once, but 8192 of them take 4 us and more, of every call, so that shares end where their workgroups pass 24576
  // (us evenly / all of one expert, shares: 256 rows of 64 experts, N x K 1024 x 2048, one 20.6 / 80.6, two 20.8 / 50.9, five 24.7 / 26.4, it gets two, as many
  // as 256 rows ask for; 1024 rows of 256, 1024 x 2048, one 80 / 322, two 84 / 219, five 97 / 103, it gets two).  So a batch of very many experts that is
  // nearly all one's keeps most of its passes: 4096 rows of 1024 experts, 512 x 1024, gets one share, 99 / 915, where five would be 138 / 241.
  const int64_t across = divide_up(a.out_width, 32), groups = a.experts + (a.begin ? 1 : 0);
  const int64_t rows_shares = a.begin && a.experts > 1 ? 1 + a.slots / 256 : 1, room = 24576 / (across * groups);
  const int64_t shares = rows_shares < room ? rows_shares : room > 0 ? room : 1;
  const dim3 grid((uint32_t)across, (uint32_t)groups, (uint32_t)(shares < 16 ? shares : 16));
  // (the limit belongs to the kernel and not to the call, so it is always the same)
  if (S::kLds > 48 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(k_few<S, TO>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)S::kLds) != hipSuccess)
    return NVFP4_ERR_HIP;
  return launch(k_few<S, TO>, grid, dim3(S::W * 64), S::kLds, s, a);
}
template <typename T, typename TO, int XR, int W, int NST>
int run_few(const ProductArgs &a, hipStream_t s) {
  return a.inp % 256 ? run_few_of<FewShape<T, XR, W, NST, false>, TO>(a, s) : run_few_of<FewShape<T, XR, W, NST, true>, TO>(a, s);
}
template <typename S, typename TO>
int run_tiles(const ProductArgs &a, hipStream_t s) {
  const int64_t tiles_n = divide_up(a.out_width, S::BN);
  const int64_t groups = a.begin ? (a.experts + 1 < a.slots ? a.experts + 1 : a.slots) : 0;
  const int64_t units = a.begin ? a.slots / S::BM + groups : divide_up(a.slots, S::BM);       // at most
  if (S::kLds > 48 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(k_tiles<S, TO>), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)S::kLds) != hipSuccess)
    return NVFP4_ERR_HIP;
  const int64_t grid = divide_up(units * tiles_n, 8) * 8;
  // More threads than a launch has: a thousand experts of two million columns and more, whose rows may be few, or an output of a terabyte.  The grid of
  // k_few has an axis for columns and one for experts.
  if (grid * S::kThreads > 0xffffffff) return run_few<typename S::T, TO, (int)(32 / sizeof(typename S::T)), 8, 1>(a, s);
  return launch(k_tiles<S, TO>, dim3((uint32_t)grid), dim3(S::kThreads), S::kLds, s, a, (int32_t)tiles_n);
}

template <typename TO>
int run_product(const ProductArgs &a, __bf16, hipStream_t s) {
  typedef __bf16 T;
  switch (choose(a, false)) {
    case kFew4: return run_few<T, TO, 4, 8, 1>(a, s);
    case kFew8: return run_few<T, TO, 8, 4, 2>(a, s);
    case kFew16: return run_few<T, TO, 16, 8, 1>(a, s);
    case kTile32: return run_tiles<Shape<T, 1, 1, 1, 1, 8, 3>, TO>(a, s);
    case kTile64x32: return run_tiles<Shape<T, 2, 1, 1, 1, 4, 3>, TO>(a, s);
    case kTile64: return run_tiles<Shape<T, 2, 2, 1, 1, 4, 3>, TO>(a, s);
    case kTile64x128: return run_tiles<Shape<T, 2, 2, 1, 2, 2, 4>, TO>(a, s);
    case kTile128: return run_tiles<Shape<T, 4, 2, 1, 2, 2, 3>, TO>(a, s);
    case kTile128x256: return run_tiles<Shape<T, 4, 2, 1, 4, 1, 3>, TO>(a, s);
    case kTile128x256K: return run_tiles<Shape<T, 4, 2, 1, 4, 2, 3>, TO>(a, s);
    case kTile256: return run_tiles<Shape<T, 4, 2, 2, 4, 1, 3>, TO>(a, s);
    default: return NVFP4_ERR_UNSUPPORTED;       // (not among the costs)
  }
}
template <typename TO>
int run_product(const ProductArgs &a, float, hipStream_t s) {
  typedef float T;
  switch (choose(a, true)) {
    case kFew4: return run_few<T, TO, 2, 8, 1>(a, s);
    case kFew8: return run_few<T, TO, 4, 4, 2>(a, s);
    case kFew16: return run_few<T, TO, 8, 8, 1>(a, s);
    case kTile32: return run_tiles<Shape<T, 1, 1, 1, 1, 4, 2>, TO>(a, s);
    case kTile64: return run_tiles<Shape<T, 2, 2, 1, 1, 4, 2>, TO>(a, s);
    case kTile64x128: return run_tiles<Shape<T, 2, 2, 1, 2, 2, 3>, TO>(a, s);
    case kTile64x256: return run_tiles<Shape<T, 2, 4, 1, 2, 1, 3>, TO>(a, s);
    case kTile64x256K: return run_tiles<Shape<T, 2, 4, 1, 2, 2, 2>, TO>(a, s);
    case kTile128x256: return run_tiles<Shape<T, 2, 4, 2, 2, 1, 3>, TO>(a, s);
    default: return NVFP4_ERR_UNSUPPORTED;
  }
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
  return of32 ? to32 ? run_product<float>(a, float{}, s) : run_product<__bf16>(a, float{}, s)
              : to32 ? run_product<float>(a, __bf16{}, s) : run_product<__bf16>(a, __bf16{}, s);
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
