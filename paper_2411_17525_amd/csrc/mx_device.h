// Device parts that the microscaled quantizers and the product share: loads and
// stores of 16 values, block scales, the rotation of a segment of 1024.
#pragma once

#include "mx.h"
#include "wave_fwht.h"

namespace higgs {

// LDS dwords per wave for a rotation: 1024 fp64 values.
constexpr int kMxWaveLds = 2048;

// fwht_rows with whole values in LDS: the same sums in the same places from half the
// LDS instructions and without moves that put the halves of a value together, for
// twice the scratch (1024 values, 128-byte aligned).
template <int G>
__device__ inline void mx_fwht_rows(double (&v)[16], uint32_t* scratch, int lane) {
  static_assert(G == 64 || G == 128 || G == 256 || G == 512 || G == 1024, "block size");
  typedef double f64x2 __attribute__((ext_vector_type(2)));
  wave_lds_sync();  // this wave's earlier accesses come first
  fwht_in_lane<16>(v);
  // value i of lane c of a row at 16 c + i, the pairs of a lane permuted by its low
  // bits: eight lanes hit distinct banks
  double* const row = reinterpret_cast<double*>(scratch) + 256 * (lane >> 4);
  const int c = lane & 15;
#pragma unroll
  for (int p = 0; p < 8; ++p)
    *reinterpret_cast<f64x2*>(row + 16 * c + 2 * (p ^ (c & 7))) = f64x2{v[2 * p], v[2 * p + 1]};
  wave_lds_sync();
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = row[16 * i + 2 * ((c >> 1) ^ (i & 7)) + (c & 1)];
  wave_lds_sync();
#pragma unroll
  for (int h = 1; h < 16 && 16 * h < G; h <<= 1)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if ((i & h) == 0) {
        const double x = v[i], y = v[i + h];
        v[i] = x + y;
        v[i + h] = x - y;
      }
  if constexpr (G >= 512) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lane_swap<16>(v[i], v[i + 8]);
      const double x = v[i], y = v[i + 8];
      v[i] = x + y;
      v[i + 8] = x - y;
    }
  }
  if constexpr (G == 1024) {
#pragma unroll
    for (int h = 0; h < 16; h += 8)
#pragma unroll
      for (int i = h; i < h + 4; ++i) {
        lane_swap<32>(v[i], v[i + 4]);
        const double x = v[i], y = v[i + 4];
        v[i] = x + y;
        v[i + 4] = x - y;
      }
  }
}

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

// The scale byte of a block from the largest fp32 exponent field of its values (255:
// NaN or infinity).
__device__ inline uint32_t scale_byte_f32(uint32_t field) {
  if (field == 255) return 255;
  return field < uint32_t(kMxTop) ? 0 : field - kMxTop;
}
// Exponent field of a double times 2^shift (11 bits plus shift), and the block's scale
// byte from the largest: 2^128 or more, infinities and NaN are kMxBad or above.
constexpr int kMxBad = 1023 + 128;
__device__ inline int field_f64(double v) {
  return int(uint32_t(__builtin_bit_cast(uint64_t, v) >> 52) & 0x7ff);
}
__device__ inline int scale_exponent_f64(int field) { return max(field - (1023 - 127 + kMxTop), 0); }
// 2^-E / 2^shift for the scale exponent E + 127.
__device__ inline double inverse_scale(int byte, int shift) {
  return __builtin_bit_cast(double, uint64_t(uint32_t(1023 + 127 - shift - byte) << 20) << 32);
}
// v times a power of two, for the conversion to codes; a zero gets the sign + (which
// one the butterflies leave depends on their order).
__device__ inline float odd_scaled(double v, double inverse) {
  return mx_odd_f32(__builtin_fma(v, inverse, 0.0));
}

// log2(sqrt(G)) where that is whole: the factor 1 / sqrt(G) is then exact and joins
// the block's power of two; 0 otherwise (the values are multiplied first).
template <int G>
constexpr int kRootShift = G == 64 ? 3 : G == 256 ? 4 : G == 1024 ? 5 : G == 4096 ? 6 : 0;

// Largest of v over the 16 lanes of a DPP row, in all of them.
__device__ inline uint32_t row_max(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x128, 0xF, 0xF, true)));  // row_ror:8
  v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x124, 0xF, 0xF, true)));
  v = max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x122, 0xF, 0xF, true)));
  return max(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x121, 0xF, 0xF, true)));
}

// Place of element n of a segment of 1024 in LDS: runs of 16 permuted so that
// the four rows of lanes hit distinct banks.
__device__ inline int lds_place(int n) { return n ^ ((((n >> 6) ^ (n >> 8)) & 3) << 4); }

// Moves 16 fp32 values per lane from mx_fwht_rows's places to 16 consecutive ones
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

// x with the signs of the lane's 16 values (bit i of neg), in fp64.
__device__ inline void signed_f64(const float (&x)[16], uint32_t neg, double (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    v[i] = double(__builtin_bit_cast(
        float, __builtin_bit_cast(uint32_t, x[i]) ^ ((neg << (31 - i)) & 0x80000000u)));
}

// Rotates a segment of 1024 values (groups of G), 16 consecutive ones per lane in
// x, and quantizes it: codes of the lane's 16 values of the result (consecutive
// ones again), and in lanes with lane % 16 < 8 the scale byte of block *block of
// the segment. neg: the lane's sign bits; lds: the wave's kMxWaveLds dwords.
template <int G, int FMT>
__device__ inline void mx_rotate_segment(float (&x)[16], uint32_t neg, double root, uint32_t* lds,
                                         int lane, uint32_t (&c)[kWords16<FMT>], uint32_t* byte,
                                         int* block) {
  constexpr int kShift = kRootShift<G>;
  double v[16];
  signed_f64(x, neg, v);
  mx_fwht_rows<G>(v, lds, lane);
  if constexpr (kShift == 0) {
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] *= root;
  }
  // block b = r / 2: registers 2b and 2b + 1 of the row's 16 lanes. A NaN or an
  // infinity of the input is in all values of its group: the larger of two is one too.
  int of[8], top = 0;
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const double m = __builtin_fmax(__builtin_fabs(v[2 * b]), __builtin_fabs(v[2 * b + 1]));
    const int f =
        int(row_max(uint32_t(__builtin_bit_cast(uint64_t, m) >> 32) & 0x7fffffffu) >> 20) - kShift;
    top = max(top, f);
    of[b] = scale_exponent_f64(f);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) x[r] = odd_scaled(v[r], inverse_scale(of[r / 2], kShift));
  if (__any(top >= kMxBad)) {  // (kShift: an infinity's field is 2047)
#pragma unroll
    for (int b = 0; b < 8; ++b)
      if (of[b] > 255 - kMxTop - 1) {
        of[b] = 255;
        x[2 * b] = x[2 * b + 1] = 0.f;
      }
  }
  uint32_t mine = uint32_t(of[0]);
  int e = fwht_rows_reg<G>(0);
#pragma unroll
  for (int b = 1; b < 8; ++b)
    if ((lane & 7) == b) {
      mine = uint32_t(of[b]);
      e = fwht_rows_reg<G>(2 * b);
    }
  *byte = mine;
  *block = (fwht_rows_lane<G>(lane & ~15) | e) / 32;
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
