// Device parts that the microscaled quantizers and the product share: loads and
// stores of 16 values, block scales, the rotation of a segment of 1024.
#pragma once

#include "mx.h"
#include "wave_fwht.h"

namespace higgs {

// Rotation of a segment of 1024 values by a wave, 16 per lane, groups of G (64 ..
// 1024). With n = 512 .. 1 for the bits 9 .. 0 of a value's place, lane bits from low
// to high, the values lie
//   in pairs:  register bits 0, 7, 8, 9   lane bits 1 .. 6    v[2 r + b] is 128 r + 2 lane + b
//   between:   register bits 0, 4, 5, 6   lane bits 1, 2, 3, 7, 8, 9
//   in runs:   register bits 0 .. 3       lane bits 4 .. 9    v[i] is 16 lane + i
// and go from one order to the next through LDS as pairs (16 bytes of fp64). Butterflies
// are done over register bits only: in pairs those of 0, 7, 8, 9, between of 4, 5, 6, in
// runs of 1, 2, 3. In pairs a load or store of the wave is one run of memory; in runs a
// lane holds half a block: its largest, codes and scale take one step across lanes.
// (With the values in runs first, 4 + 4 bits in registers, the last two by permlane
// swaps and the way back to runs through LDS, a segment's quantization took 650
// instructions, not 343.)
template <typename T>
constexpr int kMxWaveLds = 576 * 2 * int(sizeof(T)) / 4;  // dwords per wave

template <int H, typename T>
__device__ inline void mx_butterflies(T (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if ((i & H) == 0) {
      const T x = v[i], y = v[i + H];
      v[i] = x + y;
      v[i + H] = x - y;
    }
}

// H per group, from pairs to runs, or (BACK) from runs to pairs, there without the
// butterflies of bit 0, which are the caller's. Pair p is at p + 8 (p / 64) of the scratch
// between pairs and the middle order, at p + p / 8 between that and runs: both sides of
// both reach distinct banks.
template <int G, bool BACK, typename T>
__device__ inline void mx_fwht(T (&v)[16], uint32_t* scratch, int lane) {
  static_assert(G == 64 || G == 128 || G == 256 || G == 512 || G == 1024, "group size");
  typedef T pair_t __attribute__((ext_vector_type(2)));
  pair_t* const pairs = reinterpret_cast<pair_t*>(scratch) + lane;
  pair_t* const middle = reinterpret_cast<pair_t*>(scratch) + (lane & 7) + 72 * (lane >> 3);
  pair_t* const runs = reinterpret_cast<pair_t*>(scratch) + 9 * lane;
  auto write = [&](pair_t* p, int step) __attribute__((always_inline)) {
    wave_lds_sync();  // this wave's earlier accesses come first
#pragma unroll
    for (int i = 0; i < 8; ++i) p[step * i] = pair_t{v[2 * i], v[2 * i + 1]};
    wave_lds_sync();
  };
  auto read = [&](const pair_t* p, int step) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const pair_t u = p[step * i];
      v[2 * i] = u[0];
      v[2 * i + 1] = u[1];
    }
  };
  auto high = [&]() __attribute__((always_inline)) {
    if constexpr (G >= 256) mx_butterflies<2>(v);
    if constexpr (G >= 512) mx_butterflies<4>(v);
    if constexpr (G >= 1024) mx_butterflies<8>(v);
  };
  auto low = [&]() __attribute__((always_inline)) {
    mx_butterflies<2>(v);
    mx_butterflies<4>(v);
    mx_butterflies<8>(v);
  };
  if constexpr (!BACK) {
    mx_butterflies<1>(v);
    high();
    write(pairs, 72);
    read(middle, 8);
  } else {
    low();
    write(runs, 1);
    read(middle, 9);
  }
  mx_butterflies<2>(v);
  mx_butterflies<4>(v);
  if constexpr (G >= 128) mx_butterflies<8>(v);
  if constexpr (!BACK) {
    write(middle, 9);
    read(runs, 1);
    low();
  } else {
    write(middle, 8);
    read(pairs, 72);
    high();
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
__device__ inline int scale_exponent_f64(int field) {
  return max(field - (1023 - 127 + kMxTop), 0);
}
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

// Groups of 2048 and 4096 are 2 and 4 segments, held by one wave: butterflies between
// them, and of each as in a group of 1024.
template <int G>
constexpr int kSegments = G > 1024 ? G / 1024 : 1;
template <int S, typename T>
__device__ inline void mx_across(T (&v)[S][16]) {
#pragma unroll
  for (int h = 1; h < S; h <<= 1)
#pragma unroll
    for (int s = 0; s < S; ++s)
      if ((s & h) == 0)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const T x = v[s][i], y = v[s + h][i];
          v[s][i] = x + y;
          v[s + h][i] = x - y;
        }
}

// Signs of the lane's pairs of segment `seg` of a group: bit 15 of word r that of the
// first value, bit 31 that of the second.
struct MxPairSigns {
  uint32_t m[8];
};
template <int G>
struct MxLaneSigns {
  uint32_t w[(kSegments<G> + 1) / 2];
  __device__ MxLaneSigns(const MxSigns& s, int lane) {
#pragma unroll
    for (int i = 0; i < (kSegments<G> + 1) / 2; ++i) w[i] = s.w[64 * i + lane];
  }
  __device__ MxPairSigns of(int seg) {
    // (of several segments they are made anew each time, not kept over a loop: 16 and
    // 32 registers)
    if constexpr (kSegments<G> > 1) asm volatile("" : "+v"(w[seg >> 1]));
    MxPairSigns p;
#pragma unroll
    for (int r = 0; r < 8; ++r) p.m[r] = (w[seg >> 1] << (15 - r - 8 * (seg & 1))) & 0x80008000u;
    return p;
  }
};
// Waves per SIMD that a rotation's kernel is compiled for: its LDS and registers (32 per
// segment for fp64 values) allow as many.
template <int G>
constexpr int kRotationWaves = kSegments<G> == 4 ? 2 : 4;

// A lane's pairs as loaded.
template <typename InT>
struct MxPairs {
  static constexpr int kWords = sizeof(InT) == 2 ? 1 : 2;  // per pair
  uint32_t u[8 * kWords];
};
// Of the n values (a multiple of 64) from p on; zeros behind them.
template <typename InT>
__device__ inline MxPairs<InT> load_pairs(const InT* p, int64_t n, int lane) {
  constexpr int kWords = MxPairs<InT>::kWords;
  MxPairs<InT> w;
  auto load = [&](int r) __attribute__((always_inline)) {
    const uint32_t* const q = reinterpret_cast<const uint32_t*>(p + 128 * r + 2 * lane);
#pragma unroll
    for (int i = 0; i < kWords; ++i) w.u[kWords * r + i] = q[i];
  };
  if (n >= 1024) {
#pragma unroll
    for (int r = 0; r < 8; ++r) load(r);
  } else {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w.u[kWords * r + i] = 0;
      if (128 * r + 2 * lane < n) load(r);
    }
  }
  return w;
}
// With their signs, in fp64.
template <typename InT>
__device__ inline void signed_pairs(const MxPairs<InT>& w, const MxPairSigns& s, double (&v)[16]) {
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    uint32_t a, b;
    if constexpr (sizeof(InT) == 2) {
      b = (w.u[r] ^ s.m[r]) & 0xffff0000u;
      a = (w.u[r] ^ s.m[r]) << 16;
    } else {
      a = w.u[2 * r] ^ (s.m[r] << 16);
      b = w.u[2 * r + 1] ^ (s.m[r] & 0x80000000u);
    }
    v[2 * r] = double(__builtin_bit_cast(float, a));
    v[2 * r + 1] = double(__builtin_bit_cast(float, b));
  }
}

// The way back: n values from pairs, with their signs.
template <typename OutT>
__device__ inline void store_pairs(OutT* p, int64_t n, const MxPairSigns& s, int lane,
                                   const float (&v)[16]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  auto store = [&](int r) __attribute__((always_inline)) {
    if constexpr (sizeof(OutT) == 2) {
      *reinterpret_cast<uint32_t*>(p + 128 * r + 2 * lane) =
          pack_bf16(v[2 * r], v[2 * r + 1]) ^ s.m[r];
    } else {
      const uint32_t a = __builtin_bit_cast(uint32_t, v[2 * r]) ^ (s.m[r] << 16);
      const uint32_t b = __builtin_bit_cast(uint32_t, v[2 * r + 1]) ^ (s.m[r] & 0x80000000u);
      *reinterpret_cast<f32x2*>(p + 128 * r + 2 * lane) =
          f32x2{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
    }
  };
  if (n >= 1024) {
#pragma unroll
    for (int r = 0; r < 8; ++r) store(r);
  } else {
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (128 * r + 2 * lane < n) store(r);
  }
}

// Rotates a segment of 1024 values (groups of G; of larger ones after mx_across), in
// pairs in v, and quantizes it: codes
// of values 16 lane .. 16 lane + 15 of the result, and the scale byte of their block, lane
// / 2, in both its lanes. lds: the wave's kMxWaveLds<double> dwords.
template <int G, int FMT>
__device__ inline void mx_rotate_segment(double (&v)[16], double root, uint32_t* lds, int lane,
                                         uint32_t (&c)[kWords16<FMT>], uint32_t* byte) {
  constexpr int kShift = kRootShift<G>;
  mx_fwht<G < 1024 ? G : 1024, false>(v, lds, lane);
  if constexpr (kShift == 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= root;
  }
  // A NaN or an infinity of the input is in all values of its group: the larger of two
  // is one too.
  double m[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    m[i] = __builtin_fmax(__builtin_fabs(v[2 * i]), __builtin_fabs(v[2 * i + 1]));
#pragma unroll
  for (int n = 4; n > 0; n >>= 1)
#pragma unroll
    for (int i = 0; i < n; ++i) m[i] = __builtin_fmax(m[i], m[i + n]);
  uint32_t hi = uint32_t(__builtin_bit_cast(uint64_t, m[0]) >> 32) & 0x7fffffffu;
  hi = max(hi, uint32_t(lane_xor_small<1>(hi)));
  const int field = int(hi >> 20) - kShift, e = scale_exponent_f64(field);
  const double inverse = inverse_scale(e, kShift);
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = odd_scaled(v[i], inverse);
  *byte = uint32_t(e);
  if (field >= kMxBad) {  // (kShift: an infinity's field is 2047)
    *byte = 255;
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
  }
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
