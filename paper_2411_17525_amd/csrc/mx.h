// The microscaled (MX) formats: blocks of 32 consecutive values of a row, each
// value a 4-bit (E2M1) or 6-bit (E2M3) float, with one power of two per block
// (E8M0: the byte is the exponent + 127). Shared by mx_quant.hip and
// mx_product.hip.
#pragma once

#include "internal.h"

namespace higgs {

constexpr int kMxBlock = 32;
// Both element formats have a largest binary exponent of 2 (6 and 7.5), so a
// block's exponent is that of its largest magnitude less 2.
constexpr int kMxTop = 2;

inline int mx_block_bytes(int fmt) { return fmt == HIGGS_MX_FP4 ? 16 : 24; }
inline int64_t mx_blocks(int64_t in) { return (in + kMxBlock - 1) / kMxBlock; }

// RHT signs, a bit set where sigma_j = -1, as the lanes hold a group of 2048 or 4096, or
// 1024 values of smaller ones: bits q % 16 and 16 + q % 16 of word 64 (q / 16) + l those of
// values 128 q + 2 l and 128 q + 2 l + 1. A kernel argument.
struct MxSigns {
  uint32_t w[128];
};
// (mx_quant.hip; each thread keeps those of the last four pairs of seed and group size. To
// make them takes a call's host time: one row of 4096 -> 4096 takes 6.6 us with up to four
// seeds in turn and 10.8 with 64 for g = 1024, 11.1 and 28.9 for g = 4096)
void mx_signs(uint64_t seed, int g, MxSigns* s);

// Activations in the product's order, so that what a wave loads of a stage (128
// values of K) is consecutive: per 32 rows and stage, two halves (64 values) of
// 64 units, unit l = block l / 32 of row l % 32; 16 bytes per unit, and for
// E2M3 the blocks' last 8 bytes behind the half's 64 first parts. The scale
// bytes of a stage's four blocks as a word per row: [stage][rows32].
struct MxTiles {
  uint8_t* codes;
  uint8_t* scales;
  int64_t stages;  // of a row: an even number, 2 ceil(in / 256), zeros behind `in`
  int64_t rows32;  // rows, rounded up to whole tiles of 32
};
// Weight scales for the product: rows x blocks bytes to [stage][rows] words.
struct MxScaleWords {
  const uint8_t* from;
  uint32_t* to;
  int64_t rows;
  int blocks, stages;
};
constexpr int mx_half_bytes(int fmt) { return fmt == HIGGS_MX_FP4 ? 1024 : 1536; }

// Kernel launchers. g = 0: no rotation. The arguments have been checked.
hipError_t launch_mx_quantize(const void* w, higgs_dtype dtype, int64_t rows, int64_t in, int fmt,
                              int g, uint64_t seed, uint8_t* codes, uint8_t* scales,
                              hipStream_t stream);
// Activations into the product's order (batch * in <= 2^34) and, in the same launch,
// weight scale words (none where words.to is NULL).
hipError_t launch_mx_tiles(const void* x, higgs_dtype dtype, int64_t batch, int64_t in, int fmt,
                           int g, uint64_t seed, const MxTiles& tiles, const MxScaleWords& words,
                           hipStream_t stream);
hipError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows,
                                int64_t in, int fmt, int g, uint64_t seed, void* w,
                                higgs_dtype dtype, hipStream_t stream);
hipError_t launch_mx_layer_error(const void* w, higgs_dtype dtype, int64_t out, int64_t in,
                                 const uint8_t* codes, const uint8_t* scales, int g, uint64_t seed,
                                 double* row_err, double* t2, hipStream_t stream);
// Few rows (mx_decode.hip): activations from `tiles`, or, where mx_decode_fuses,
// raw ones converted on the way (`tiles` is not read). batch <= 32.
bool mx_decode_fuses(int64_t batch, int64_t in, int g);
hipError_t launch_mx_decode(const void* x, higgs_dtype x_dtype, int64_t batch, int fmt,
                            const MxTiles& tiles, const uint8_t* codes, const uint8_t* scales,
                            int g, uint64_t seed, int64_t out, int64_t in, void* y,
                            higgs_dtype y_dtype, hipStream_t stream);
int64_t mx_qmatmul_workspace_bytes(int64_t batch, int64_t out, int64_t in, int fmt, int g);
hipError_t launch_mx_qmatmul(const void* x, higgs_dtype x_dtype, int64_t batch, int fmt,
                             const uint8_t* codes, const uint8_t* scales, int g, uint64_t seed,
                             int64_t out, int64_t in, void* y, higgs_dtype y_dtype,
                             void* workspace, hipStream_t stream);

// ---- device: one value ----

// A double rounded to 21 significant bits towards zero with the last bit set
// where anything was dropped (round to odd), as fp32: rounding that again to
// nearest, ties to even, to any format of up to 19 bits gives what one rounding
// of the double gives. Exact in fp32 where |v| is 0 or in its normal range.
__device__ inline float mx_odd_f32(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = uint32_t(u), hi = uint32_t(u >> 32);
  // (as an instruction: the compiler makes a comparison and a selection of it)
  uint32_t any;
  asm("v_min_u32 %0, 1, %1" : "=v"(any) : "v"(lo));
  return float(__builtin_bit_cast(double, uint64_t(hi | any) << 32));
}

// 16 scaled values (|v| < 8) to codes, rounded to nearest with ties to even and
// saturated: 2 words of E2M1 codes, or 3 of E2M3, the least significant bits
// first.
template <int FMT>
__device__ inline void mx_encode16(const float (&v)[16], uint32_t* out) {
  if constexpr (FMT == HIGGS_MX_FP4) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t r = 0;
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[8 * h], v[8 * h + 1], 1.0f, 0);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[8 * h + 2], v[8 * h + 3], 1.0f, 1);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[8 * h + 4], v[8 * h + 5], 1.0f, 2);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[8 * h + 6], v[8 * h + 7], 1.0f, 3);
      out[h] = r;
    }
  } else {
    // The instruction takes the even and the odd values of 32. It writes its first result
    // before it has read all of them: as a builtin it got v[2:7] from v[0:15] and lost a
    // value, so the result's registers are kept apart here.
    typedef float f32x16 __attribute__((ext_vector_type(16)));
    typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
    f32x16 even = {}, odd = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      even[i] = v[2 * i];
      odd[i] = v[2 * i + 1];
    }
    u32x6 r;
    asm("v_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, 1.0\n\ts_nop 1"
        : "=&v"(r)
        : "v"(even), "v"(odd));
#pragma unroll
    for (int i = 0; i < 3; ++i) out[i] = r[i];
  }
}

// The values of 16 codes (2 or 3 words, least significant bits first) of a block with
// scale byte `byte`, exact (below 2^-126 too; byte 255: NaN).
template <int FMT>
__device__ inline void mx_decode16(const uint32_t* in, uint32_t byte, float (&v)[16]) {
  // (the instructions take the exponent field of the scale: 0 is 2^-127, 255 NaN)
  const float scale = __builtin_bit_cast(float, byte << 23);
  if constexpr (FMT == HIGGS_MX_FP4) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[h], scale, 0);
      const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[h], scale, 1);
      const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[h], scale, 2);
      const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(in[h], scale, 3);
      float* const o = v + 8 * h;
      o[0] = a[0], o[1] = a[1], o[2] = b[0], o[3] = b[1];
      o[4] = c[0], o[5] = c[1], o[6] = d[0], o[7] = d[1];
    }
  } else {
    typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
    typedef float f32x32 __attribute__((ext_vector_type(32)));
    f32x32 r;  // (registers of its own, as above)
    asm("v_cvt_scalef32_pk32_f32_fp6 %0, %1, %2\n\ts_nop 1"
        : "=&v"(r)
        : "v"(u32x6{in[0], in[1], in[2], 0, 0, 0}), "v"(scale));
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = r[i];
  }
}

__device__ inline float bf16_to_f32(uint32_t b) { return __builtin_bit_cast(float, b << 16); }
// Two values to bf16 in one word, to nearest with ties to even (one instruction).
__device__ inline uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{__bf16(lo), __bf16(hi)});
}

}  // namespace higgs
