// Device parts that the microscaled quantizers and the product share: loads and
// stores of 16 values, block scales, the rotation of a segment of 1024.
#pragma once

#include "mx.h"
#include "wave_fwht.h"

namespace higgs {

// LDS dwords per wave: fwht_rows's scratch, or 1024 fp32 values
constexpr int kMxWaveLds = kFwhtRows > 1024 ? kFwhtRows : 1024;

// 16 consecutive values from p (aligned to the type only).
template <typename InT>
__device__ inline void load16(const InT* p, float (&v)[16]) {
  if constexpr (sizeof(InT) == 2) {
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8), aligned(2)));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u16x8 u = *reinterpret_cast<const u16x8*>(p + 8 * h);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[8 * h + i] = bf16_to_f32(u[i]);
    }
  } else {
    typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const f32x4 u = *reinterpret_cast<const f32x4*>(p + 4 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * h + i] = u[i];
    }
  }
}

template <typename InT>
__device__ inline float load1(const InT* p) {
  if constexpr (sizeof(InT) == 2) {
    return bf16_to_f32(*p);
  } else {
    return *p;
  }
}

// n values (0 .. 16) from p, zeros behind them.
template <typename InT>
__device__ inline void load16_upto(const InT* p, int n, float (&v)[16]) {
  if (n >= 16) {
    load16(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = i < n ? load1(p + i) : 0.f;
}

template <typename OutT>
__device__ inline void store16(OutT* p, const float (&v)[16]) {
  if constexpr (sizeof(OutT) == 2) {
    typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4_a2 u;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        u[i] = pack_bf16(v[8 * h + 2 * i], v[8 * h + 2 * i + 1]);
      *reinterpret_cast<u32x4_a2*>(p + 8 * h) = u;
    }
  } else {
    typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int h = 0; h < 4; ++h)
      *reinterpret_cast<f32x4*>(p + 4 * h) =
          f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
  }
}

template <typename OutT>
__device__ inline void store16_upto(OutT* p, int n, const float (&v)[16]) {
  if (n >= 16) {
    store16(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < n) {
      if constexpr (sizeof(OutT) == 2) {
        p[i] = OutT(pack_bf16(v[i], 0.f));
      } else {
        p[i] = v[i];
      }
    }
}

// Codes of 16 values: 2 (E2M1) or 3 (E2M3) words.
template <int FMT>
constexpr int kWords16 = FMT == HIGGS_MX_FP4 ? 2 : 3;

template <int FMT>
__device__ inline void store_codes16(uint8_t* p, const uint32_t* c) {
#pragma unroll
  for (int i = 0; i < kWords16<FMT>; ++i) reinterpret_cast<uint32_t*>(p)[i] = c[i];
}
template <int FMT>
__device__ inline void load_codes16(const uint8_t* p, uint32_t* c) {
#pragma unroll
  for (int i = 0; i < kWords16<FMT>; ++i) c[i] = reinterpret_cast<const uint32_t*>(p)[i];
}

// The scale byte of a block from the largest fp32 or fp64 exponent field of its
// values (255: NaN or infinity).
__device__ inline uint32_t scale_byte_f32(uint32_t field) {
  if (field == 255) return 255;
  return field < uint32_t(kMxTop) ? 0 : field - kMxTop;
}
__device__ inline uint32_t scale_byte_f64(uint32_t field) {
  if (field >= 1023 + 128) return 255;
  const int b = int(field) - 1023 + 127 - kMxTop;
  return uint32_t(b < 0 ? 0 : b);
}
__device__ inline uint32_t field_f64(double v) {
  return uint32_t(__builtin_bit_cast(uint64_t, v) >> 52) & 0x7ff;
}
// 2^-E of a scale byte, as a double; 0 for the NaN byte (every code is 0 then).
__device__ inline double inverse_scale(uint32_t byte) {
  return byte == 255 ? 0.0
                     : __builtin_bit_cast(double, uint64_t(1023 + 127 - byte) << 52);
}
__device__ inline float odd_scaled(double v, uint32_t byte) {
  return byte == 255 ? 0.f : mx_odd_f32(v * inverse_scale(byte));
}

// The butterflies' sum times 1 / sqrt(g); a zero gets the sign + (which one the
// sum leaves depends on its order).
__device__ inline double normalised(double v, double root) {
  return __builtin_fma(v, root, 0.0);
}

// Place of element n of a segment of 1024 in LDS: runs of 16 permuted so that
// the four rows of lanes hit distinct banks.
__device__ inline int lds_place(int n) { return n ^ ((((n >> 6) ^ (n >> 8)) & 3) << 4); }

// Moves 16 fp32 values per lane from fwht_rows's places to 16 consecutive ones
// per lane through the wave's LDS.
template <int G>
__device__ inline void rows_to_lanes(float (&v)[16], float* lds, int lane) {
  wave_lds_sync();
#pragma unroll
  for (int r = 0; r < 16; ++r) lds[lds_place(fwht_rows_lane<G>(lane) + fwht_rows_reg<G>(r))] = v[r];
  wave_lds_sync();
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  const f32x4* p = reinterpret_cast<const f32x4*>(lds + lds_place(16 * lane));
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    const f32x4 u = p[h];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[4 * h + i] = u[i];
  }
  wave_lds_sync();
}
// And back.
template <int G>
__device__ inline void lanes_to_rows(float (&v)[16], float* lds, int lane) {
  wave_lds_sync();
  typedef float f32x4 __attribute__((ext_vector_type(4)));
  f32x4* p = reinterpret_cast<f32x4*>(lds + lds_place(16 * lane));
#pragma unroll
  for (int h = 0; h < 4; ++h) p[h] = f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
  wave_lds_sync();
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = lds[lds_place(fwht_rows_lane<G>(lane) + fwht_rows_reg<G>(r))];
  wave_lds_sync();
}

// This lane's 16 sign bits for elements 16 lane .. of a segment of 1024.
template <int G>
__device__ inline uint32_t lane_signs(const MxSigns& s, int lane) {
  const int j = (16 * lane) & (G - 1);
  return s.w[j >> 5] >> (j & 16);
}

template <int G>
__device__ inline void signed_f64(const float (&x)[16], uint32_t neg, double (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = double((neg >> i) & 1 ? -x[i] : x[i]);
}

// Rotates a segment of 1024 values (groups of G), 16 consecutive ones per lane in
// x, and quantizes it: codes of the lane's 16 values of the result (consecutive
// ones again), and in lanes with lane % 16 < 8 the scale byte of block *block of
// the segment. neg: the lane's sign bits; lds: the wave's kMxWaveLds dwords.
template <int G, int FMT>
__device__ inline void mx_rotate_segment(float (&x)[16], uint32_t neg, double root, uint32_t* lds,
                                         int lane, uint32_t (&c)[kWords16<FMT>], uint32_t* byte,
                                         int* block) {
  double v[16];
  signed_f64<G>(x, neg, v);
  fwht_rows<G>(v, lds, lane);
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = normalised(v[r], root);
  // block b = r / 2: registers 2b and 2b + 1 of the row's 16 lanes
  uint32_t of[8];
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    uint32_t f = max(field_f64(v[2 * b]), field_f64(v[2 * b + 1]));
    f = max(f, lane_xor_small<1>(f));
    f = max(f, lane_xor_small<2>(f));
    f = max(f, lane_xor_small<4>(f));
    f = max(f, lane_xor_small<8>(f));
    of[b] = scale_byte_f64(f);
  }
  uint32_t mine = of[0];
  int e = fwht_rows_reg<G>(0);
#pragma unroll
  for (int b = 1; b < 8; ++b)
    if ((lane & 7) == b) {
      mine = of[b];
      e = fwht_rows_reg<G>(2 * b);
    }
  *byte = mine;
  *block = (fwht_rows_lane<G>(lane & ~15) | e) / 32;
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = odd_scaled(v[r], of[r / 2]);
  rows_to_lanes<G>(x, reinterpret_cast<float*>(lds), lane);
  mx_encode16<FMT>(x, c);
}

// Quantizes the two halves of a block in two neighbouring lanes: 16 values each in
// x, the block's scale byte in both.
template <int FMT>
__device__ inline uint32_t mx_plain_halves(float (&x)[16], uint32_t (&c)[kWords16<FMT>]) {
  uint32_t f = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) f = max(f, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
  f = max(f, lane_xor_small<1>(f));
  const uint32_t byte = scale_byte_f32(f >> 23);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = byte == 255 ? 0.f : __builtin_ldexpf(x[i], 127 - int(byte));
  mx_encode16<FMT>(x, c);
  return byte;
}

}  // namespace higgs
