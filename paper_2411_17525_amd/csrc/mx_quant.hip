// Quantization to the microscaled formats, the way back and the layer error.
//
// A block of 32 consecutive values v of a row (rotated first where g > 0, as a
// HIGGS layer's: H (sigma v) / sqrt(g)) is stored as E = max(floor(log2 max|v|)
// - 2, -127) and the codes of v 2^-E, rounded to nearest with ties to even and
// saturated at the format's largest magnitude. Blocks that hold a NaN, an
// infinity or, rotated, a magnitude of 2^128 or more get scale byte 255 (NaN)
// and codes 0. The rotation is computed in fp64, for codes are decided at
// borders: bf16 and fp32 inputs of ordinary range are summed exactly, so the
// codes are those of the exact rotation.
//
// With a rotation, a wavefront takes segments of 1024 values (of g for g =
// 2048 and 4096). Rows are whole groups there, so the matrix is one run of groups.
// What bounds these kernels is the issue of vector instructions: a segment's quantization
// takes 343 (160 of them the butterflies, in fp64 at the rate of fp32) and 74% of the
// cycles issue one; LDS is busy in 41%. 14336 x 4096 bf16 to E2M1 with g = 1024, kernels
// in a row on changing inputs: 45 to 49 us (3.0 to 3.3 TB/s), with g = 2048 50 and g = 4096
// 62 (12% more instructions per value, and no loads ahead; two waves per SIMD for 4096);
// its layer error 46 (3.2 TB/s), the way back 35 (4.2 TB/s, near a copy's rate). One
// kernel by itself behind a fill of the caches takes 5 to 10 us more.

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "mx_device.h"

namespace higgs {

void mx_signs(uint64_t seed, int g, MxSigns* s) {
  struct Entry {
    uint64_t seed = 0;
    int g = 0;
    MxSigns s;
  };
  static thread_local Entry kept[4];
  static thread_local int next = 0;
  for (const Entry& e : kept)
    if (e.g == g && e.seed == seed) {
      *s = e.s;
      return;
    }
  Entry& e = kept[next];
  next = (next + 1) % 4;
  e.g = g;
  e.seed = seed;
  for (uint32_t& w : e.s.w) w = 0;
  for (int j = 0; j < g; ++j) {
    if (!rht_sign_negative(seed, uint32_t(j))) continue;
    for (int n = j; n < std::max(g, 1024); n += g)
      e.s.w[64 * (n / 2048) + n / 2 % 64] |= 1u << (16 * (n % 2) + n / 128 % 16);
  }
  *s = e.s;
}

namespace {

constexpr int kWaves = 4;

// ---- quantization ----

template <int G, int FMT, typename InT>
__global__ __launch_bounds__(64 * kWaves, kRotationWaves<G>) void mx_quantize_rht(
    const InT* __restrict__ w, int64_t total, const MxSigns signs, double root,
    uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  constexpr int S = kSegments<G>;
  __shared__ __attribute__((aligned(16))) uint32_t s_lds[kWaves][kMxWaveLds<double>];
  const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
  MxLaneSigns<G> neg(signs, lane);
  const int64_t step = int64_t(gridDim.x) * kWaves * 1024 * S;
  int64_t k = (int64_t(blockIdx.x) * kWaves + wave) * 1024 * S;
  MxPairs<InT> next;  // one segment's values are loaded ahead (45 us for 14336 x 4096, not 50)
  if constexpr (S == 1) next = load_pairs(w + k, total - k, lane);
  for (; k < total; k += step) {
    double v[S][16];
    if constexpr (S == 1) {
      signed_pairs(next, neg.of(0), v[0]);
      if (k + step < total) next = load_pairs(w + k + step, total - k - step, lane);
    } else {
#pragma unroll
      for (int s = 0; s < S; ++s)
        signed_pairs(load_pairs(w + k + 1024 * s, 1024, lane), neg.of(s), v[s]);
    }
    mx_across(v);
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if (s > 0) __builtin_amdgcn_sched_barrier(0);  // (one segment's registers at a time)
      uint32_t c[kWords16<FMT>], byte;
      mx_rotate_segment<G, FMT>(v[s], root, s_lds[wave], lane, c, &byte);
      const int64_t at = k + 1024 * s + 16 * lane;
      if (S > 1 || at < total) {  // total is a multiple of 64 (and of groups)
        store_codes16<FMT>(codes + (at / 16) * (4 * kWords16<FMT>), c);
        if ((lane & 1) == 0) scales[at / 32] = uint8_t(byte);
      }
    }
  }
}

// Weight scales, row after row, to words of a stage's four blocks, stage after
// stage; zeros behind a row's end. A wave reads 16 bytes each of 64 rows and writes
// four runs of 64 words. part of parts: its share of the stages.
__device__ inline void scale_words(const MxScaleWords& s, int64_t rows64, int part, int parts) {
  const int64_t row = rows64 * 64 + (threadIdx.x & 63);
  if (row >= s.rows) return;
  const uint8_t* const p = s.from + row * s.blocks;
  for (int t0 = (part * (int(blockDim.x) >> 6) + int(threadIdx.x >> 6)) * 4; t0 < s.stages;
       t0 += parts * (int(blockDim.x) >> 6) * 4) {
    if (t0 * 4 + 16 <= s.blocks) {
      typedef uint32_t u32x4_a1 __attribute__((ext_vector_type(4), aligned(1)));
      const u32x4_a1 u = *reinterpret_cast<const u32x4_a1*>(p + t0 * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) s.to[(t0 + i) * s.rows + row] = u[i];
    } else {
      for (int t = t0; t < min(t0 + 4, s.stages); ++t) {
        uint32_t w = 0;
        for (int j = 0; j < 4; ++j)
          if (t * 4 + j < s.blocks) w |= uint32_t(p[t * 4 + j]) << (8 * j);
        s.to[t * s.rows + row] = w;
      }
    }
  }
}

// Activations into the product's order: a block takes 4 rows x 1024 values, a wave
// one row's; the codes meet in LDS, so that what goes to memory are runs of 4 rows'
// units (64 and 32 bytes; written by row they are 16 and 8 bytes apart: 16 us
// instead of 7 for 2048 x 4096 without a rotation). The launch's last blocks put the
// weights' scales into words. 8 rows per block take 3 to 8% longer, blocks that loop
// over rows with the next ones loaded ahead 15%.
constexpr int kTileRows = 4;

template <int G, int FMT, typename InT>
__global__ __launch_bounds__(64 * kTileRows) void mx_to_tiles(const InT* __restrict__ x, int batch,
                                                              int in, int parts, int blocks,
                                                              const MxSigns signs, double root,
                                                              const MxTiles t,
                                                              const MxScaleWords words,
                                                              int word_parts) {
  // 32 blocks of a segment (8 stages x 2 halves x 2) x kTileRows rows
  constexpr int kUnits = 32 * kTileRows;
  __shared__ __attribute__((aligned(16))) uint8_t s_head[kUnits * 16];
  __shared__ __attribute__((aligned(16))) uint8_t s_tail[FMT == HIGGS_MX_FP6 ? kUnits * 8 : 16];
  __shared__ uint32_t s_scale[8 * kTileRows];
  __shared__ __attribute__((aligned(16))) uint32_t
      s_lds[G > 0 ? kTileRows : 1][G > 0 ? kMxWaveLds<double> : 4];
  if (int(blockIdx.x) >= blocks) {
    const int i = int(blockIdx.x) - blocks;
    scale_words(words, i / word_parts, i % word_parts, word_parts);
    return;
  }
  const int tid = int(threadIdx.x), lane = tid & 63, wave = tid >> 6;
  const int group = int(blockIdx.x) / parts, part = int(blockIdx.x) - group * parts;
  const int row = group * kTileRows + wave, r0 = group * kTileRows;
  const InT* const p = x + int64_t(row) * in;
  constexpr int S = kSegments<G>;
  double v[S][16];
  if (G > 0 && row < batch) {
    MxLaneSigns<G> neg(signs, lane);
#pragma unroll
    for (int s = 0; s < S; ++s)
      signed_pairs(load_pairs(p + 1024 * (S * part + s), S > 1 ? 1024 : in - 1024 * part, lane),
                   neg.of(s), v[s]);
    mx_across(v);
  }
#pragma unroll
  for (int s = 0; s < S; ++s) {
    const int seg = S * part + s;
    if (s > 0) __syncthreads();
    if (row < batch) {
      uint32_t c[kWords16<FMT>], byte;  // (the scale byte of block lane / 2 of the segment)
      if constexpr (G > 0) {
        mx_rotate_segment<G, FMT>(v[s], root, s_lds[wave], lane, c, &byte);
      } else {
        const int k = 1024 * seg + 16 * lane, left = in - k;
        float u[16];
        load16_upto(p + (left > 0 ? k : 0), left < 0 ? 0 : left > 16 ? 16 : left, u);
        byte = mx_plain_halves<FMT>(u, c);
      }
      // half-block `lane` of the segment: block lane / 2, which is unit (lane / 2) * kTileRows +
      // wave
      const int unit = (lane >> 1) * kTileRows + wave;
      uint32_t* const h = reinterpret_cast<uint32_t*>(s_head + unit * 16);
      if constexpr (FMT == HIGGS_MX_FP4) {
        *reinterpret_cast<uint2*>(h + (lane & 1) * 2) = make_uint2(c[0], c[1]);
      } else {
        uint32_t* const tl = reinterpret_cast<uint32_t*>(s_tail + unit * 8);
        if ((lane & 1) == 0) {
          h[0] = c[0];
          h[1] = c[1];
          h[2] = c[2];
        } else {
          h[3] = c[0];
          tl[0] = c[1];
          tl[1] = c[2];
        }
      }
      if ((lane & 1) == 0)
        reinterpret_cast<uint8_t*>(
            s_scale)[((lane >> 3) * kTileRows + wave) * 4 + (lane >> 1 & 3)] = uint8_t(byte);
    }
    __syncthreads();
    // unit u = (stage, half, block of the half, row); rows behind the batch are written
    // too (of their own tile: never read as results)
    const int stage0 = 8 * seg, stages = min(8, int(t.stages) - stage0);
    uint8_t* const tile = t.codes + (int64_t(r0 / 32) * t.stages + stage0) * 2 * mx_half_bytes(FMT);
    if (tid < kUnits) {
      const int r = tid % kTileRows, blk = tid / kTileRows;  // blk = 4 stage + 2 half + j
      if (blk < 4 * stages)
        *reinterpret_cast<uint4*>(tile + (blk >> 1) * mx_half_bytes(FMT) +
                                  ((blk & 1) * 32 + r0 % 32 + r) * 16) =
            *reinterpret_cast<const uint4*>(s_head + tid * 16);
    } else if (FMT == HIGGS_MX_FP6) {
      const int u = tid - kUnits, r = u % kTileRows, blk = u / kTileRows;
      if (blk < 4 * stages)
        *reinterpret_cast<uint2*>(tile + (blk >> 1) * mx_half_bytes(FMT) + 1024 +
                                  ((blk & 1) * 32 + r0 % 32 + r) * 8) =
            *reinterpret_cast<const uint2*>(s_tail + u * 8);
    }
    if (tid < 8 * kTileRows && tid / kTileRows < stages)
      *reinterpret_cast<uint32_t*>(t.scales + ((stage0 + tid / kTileRows) * t.rows32 + r0 +
                                               tid % kTileRows) * 4) = s_scale[tid];
  }
}

// No rotation: a lane takes 16 consecutive values, half a block. units: halves
// of blocks per row; the last block of a row may end early.
template <int FMT, typename InT>
__global__ __launch_bounds__(256) void mx_quantize_plain(const InT* __restrict__ w, int64_t rows,
                                                         int64_t in, int64_t units,
                                                         uint8_t* __restrict__ codes,
                                                         uint8_t* __restrict__ scales) {
  const int64_t total = rows * units, step = int64_t(gridDim.x) * 256;
  // (total is even, so both halves of a block are in range or neither is)
  for (int64_t u = int64_t(blockIdx.x) * 256 + threadIdx.x; u < total; u += step) {
    const int64_t row = u / units, k = (u - row * units) * 16;
    const int64_t left = in - k;
    float x[16];
    load16_upto(w + row * in + (left > 0 ? k : 0), int(left < 0 ? 0 : left > 16 ? 16 : left), x);
    uint32_t c[kWords16<FMT>];
    const uint32_t byte = mx_plain_halves<FMT>(x, c);
    store_codes16<FMT>(codes + u * (4 * kWords16<FMT>), c);
    if ((u & 1) == 0) scales[u / 2] = uint8_t(byte);
  }
}

// ---- the way back ----

// Values are rotated back times 2^-16: sums of 4096 of the largest, 7.5 * 2^127, stay in
// fp32's range, so that only results beyond it are infinite, and multiples of 2^-146
// (steps of 2^-3 in blocks of the smallest exponent, -127) are still exact in it. The
// shift is part of the power of two that the decoding multiplies by; what scale bytes
// below 16 cannot hold of it, the first butterflies multiply by (both values of each are
// of one block; exact).
constexpr uint32_t kBackShift = 16;
template <int FMT>
__device__ inline void mx_decode16_back(const uint32_t* c, uint32_t byte, float (&v)[16]) {
  const uint32_t part = min(byte, kBackShift);
  mx_decode16<FMT>(c, byte == 255 ? 255 : byte - part, v);
  const float rest = __builtin_bit_cast(float, (127 - kBackShift + part) << 23);
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const float x = v[i] * rest, y = v[i + 1];
    v[i] = __builtin_fmaf(y, rest, x);
    v[i + 1] = __builtin_fmaf(-y, rest, x);
  }
}

// 2^16 / sqrt(G) as a float and, where it is no power of two, the rest of it: the product
// with both is rounded once (by the rounded factor alone fp32 results of G = 128, 512 and
// 2048 are off by up to a whole step).
struct MxBackRoot {
  float high, low;
};

// Rotated back in fp32 (stored values are not decided at borders): codes of 16
// consecutive values per lane, values stored as pairs.
template <int G, int FMT, typename OutT>
__global__ __launch_bounds__(64 * kWaves, kRotationWaves<G>) void mx_dequantize_rht(
    const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t total,
    const MxSigns signs, const MxBackRoot root, OutT* __restrict__ w) {
  constexpr int S = kSegments<G>;
  __shared__ __attribute__((aligned(16))) uint32_t s_lds[kWaves][kMxWaveLds<float>];
  const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
  MxLaneSigns<G> neg(signs, lane);
  const int64_t step = int64_t(gridDim.x) * kWaves * 1024 * S;
  for (int64_t k = (int64_t(blockIdx.x) * kWaves + wave) * 1024 * S; k < total; k += step) {
    float x[S][16];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int64_t at = k + 1024 * s + 16 * lane;
      uint32_t c[kWords16<FMT>] = {}, byte = 0;
      if (S > 1 || at < total) {
        load_codes16<FMT>(codes + (at / 16) * (4 * kWords16<FMT>), c);
        byte = scales[at / 32];
      }
      mx_decode16_back<FMT>(c, byte, x[s]);
    }
#pragma unroll
    for (int s = 0; s < S; ++s) mx_fwht<G < 1024 ? G : 1024, true>(x[s], s_lds[wave], lane);
    mx_across(x);
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        x[s][i] = kRootShift<G> != 0 ? x[s][i] * root.high
                                     : __builtin_fmaf(x[s][i], root.high, x[s][i] * root.low);
      store_pairs(w + k + 1024 * s, S > 1 ? 1024 : total - k, neg.of(s), lane, x[s]);
    }
  }
}

template <int FMT, typename OutT>
__global__ __launch_bounds__(256) void mx_dequantize_plain(const uint8_t* __restrict__ codes,
                                                           const uint8_t* __restrict__ scales,
                                                           int64_t rows, int64_t in, int64_t units,
                                                           OutT* __restrict__ w) {
  const int64_t total = rows * units, step = int64_t(gridDim.x) * 256;
  for (int64_t u = int64_t(blockIdx.x) * 256 + threadIdx.x; u < total; u += step) {
    const int64_t row = u / units, k = (u - row * units) * 16;
    const int64_t left = in - k;
    if (left <= 0) continue;  // the second half of a row's last block
    uint32_t c[kWords16<FMT>];
    load_codes16<FMT>(codes + u * (4 * kWords16<FMT>), c);
    float x[16];
    mx_decode16<FMT>(c, scales[u / 2], x);
    store16_upto(w + row * in + k, int(left > 16 ? 16 : left), x);
  }
}

// ---- layer error ----

// err = sum (v - q 2^E)^2 over a (rotated) row and norm = sum w^2, fp64, summed in a
// fixed order. A block takes kWaves / split rows, a row `split` waves (1, 2 or 4).
struct MxErrorRow {
  int64_t row;
  int part;  // this wave's of the row's
  __device__ MxErrorRow(int split, int wave)
      : row(int64_t(blockIdx.x) * (kWaves / split) + wave / split), part(wave % split) {}
};
__device__ inline void row_sums(double err, double norm, int lane, int wave, int split,
                                int64_t rows, double* row_err) {
  __shared__ double s_sum[kWaves][2];
  err = wave_sum(err, lane);
  norm = wave_sum(norm, lane);
  if (lane == 0) {
    s_sum[wave][0] = err;
    s_sum[wave][1] = norm;
  }
  __syncthreads();
  const int here = kWaves / split, tid = int(threadIdx.x), r = tid >> 1;
  const int64_t row = int64_t(blockIdx.x) * here + r;
  if (r < here && row < rows) {
    double t = 0.0;
    for (int q = 0; q < split; ++q) t += s_sum[r * split + q][tid & 1];
    row_err[2 * row + (tid & 1)] = t;
  }
}

template <int G, typename InT>
__global__ __launch_bounds__(64 * kWaves, kSegments<G> == 2 ? 3 : kRotationWaves<G>)
void mx_error_rht(
    const InT* __restrict__ w, int64_t rows, int64_t in, int split, const MxSigns signs,
    double root, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
    double* __restrict__ row_err) {
  constexpr int S = kSegments<G>;
  __shared__ __attribute__((aligned(16))) uint32_t s_lds[kWaves][kMxWaveLds<double>];
  const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
  const MxErrorRow mine(split, wave);
  MxLaneSigns<G> neg(signs, lane);
  double err = 0.0, norm = 0.0;
  int64_t k = 1024 * S * mine.part;
  const int64_t step = 1024 * S * split, end = mine.row < rows ? in : 0, row0 = mine.row * in;
  // one bf16 segment's loads go ahead (45 us for 4096 x 14336, not 48; fp32 ones spill)
  constexpr bool kAhead = S == 1 && sizeof(InT) == 2;
  struct {
    MxPairs<InT> x;
    uint32_t c[2], byte;
  } next;
  auto load = [&](int64_t at) __attribute__((always_inline)) {
    next.x = load_pairs(w + row0 + at, S > 1 ? 1024 : end - at, lane);
    next.c[0] = next.c[1] = next.byte = 0;
    const int64_t here = row0 + at + 16 * lane;
    if (S > 1 || at + 16 * lane < end) {
      load_codes16<HIGGS_MX_FP4>(codes + here / 2, next.c);
      next.byte = scales[here / 32];
    }
  };
  if constexpr (kAhead) load(k);
  for (; k < end; k += step) {
    double v[S][16];
    uint32_t c[S][2], byte[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      __builtin_amdgcn_sched_barrier(0);  // (one segment's registers at a time)
      if constexpr (!kAhead) load(k + 1024 * s);
      signed_pairs(next.x, neg.of(s), v[s]);
      c[s][0] = next.c[0];
      c[s][1] = next.c[1];
      byte[s] = next.byte;
      if constexpr (kAhead)
        if (k + step < end) load(k + step);
#pragma unroll
      for (int i = 0; i < 16; ++i) norm = __builtin_fma(v[s][i], v[s][i], norm);
    }
    mx_across(v);
#pragma unroll
    for (int s = 0; s < S; ++s) {
      __builtin_amdgcn_sched_barrier(0);
      mx_fwht<G < 1024 ? G : 1024, false>(v[s], s_lds[wave], lane);
      float q[16];
      mx_decode16<HIGGS_MX_FP4>(c[s], byte[s], q);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const double d = __builtin_fma(v[s][i], root, -double(q[i]));
        err = __builtin_fma(d, d, err);
      }
    }
  }
  row_sums(err, norm, lane, wave, split, rows, row_err);
}

template <typename InT>
__global__ __launch_bounds__(64 * kWaves) void mx_error_plain(
    const InT* __restrict__ w, int64_t rows, int64_t in, int64_t units, int split,
    const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
    double* __restrict__ row_err) {
  const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
  const MxErrorRow mine(split, wave);
  double err = 0.0, norm = 0.0;
  for (int64_t u = 64 * mine.part + lane; mine.row < rows && u < units; u += 64 * split) {
    const int64_t left = in - 16 * u;
    if (left <= 0) continue;
    const int n = int(left > 16 ? 16 : left);
    float x[16], q[16];
    load16_upto(w + mine.row * in + 16 * u, n, x);
    uint32_t c[2];
    load_codes16<HIGGS_MX_FP4>(codes + (mine.row * units + u) * 8, c);
    mx_decode16<HIGGS_MX_FP4>(c, scales[(mine.row * units + u) / 2], q);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < n) {
        const double v = double(x[i]), d = v - double(q[i]);
        norm = __builtin_fma(v, v, norm);
        err = __builtin_fma(d, d, err);
      }
  }
  row_sums(err, norm, lane, wave, split, rows, row_err);
}

__global__ __launch_bounds__(1024) void mx_t2(const double* __restrict__ row_err, int64_t rows,
                                              double* __restrict__ t2) {
  __shared__ double s_sum[2][16];
  const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
  double err = 0.0, norm = 0.0;
  for (int64_t r = threadIdx.x; r < rows; r += 1024) {
    err += row_err[2 * r];
    norm += row_err[2 * r + 1];
  }
  err = wave_sum(err, lane);
  norm = wave_sum(norm, lane);
  if (lane == 0) {
    s_sum[0][wave] = err;
    s_sum[1][wave] = norm;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double e = 0.0, n = 0.0;
    for (int q = 0; q < 16; ++q) {
      e += s_sum[0][q];
      n += s_sum[1][q];
    }
    t2[0] = n == 0.0 ? 0.0 : e / n;
  }
}

// Blocks for segments (of G values) of `total`, a wave each, four to a block: at most
// eight blocks per compute unit, the kernels loop over the rest.
template <int G>
unsigned segment_blocks(int64_t total) {
  constexpr int64_t kBlock = 1024 * kSegments<G> * kWaves;
  return unsigned(std::min<int64_t>((total + kBlock - 1) / kBlock, 2048));
}
unsigned unit_blocks(int64_t units) {
  return unsigned(std::min<int64_t>((units + 255) / 256, 1 << 20));
}

// Calls f(std::integral_constant<int, G>) for the group size.
template <typename F>
void for_group(int g, F f) {
  switch (g) {
    case 64: f(std::integral_constant<int, 64>{}); break;
    case 128: f(std::integral_constant<int, 128>{}); break;
    case 256: f(std::integral_constant<int, 256>{}); break;
    case 512: f(std::integral_constant<int, 512>{}); break;
    case 1024: f(std::integral_constant<int, 1024>{}); break;
    case 2048: f(std::integral_constant<int, 2048>{}); break;
    default: f(std::integral_constant<int, 4096>{}); break;
  }
}

template <int FMT, typename InT>
hipError_t quantize_typed(const InT* w, int64_t rows, int64_t in, int g, uint64_t seed,
                          uint8_t* codes, uint8_t* scales, hipStream_t stream) {
  if (g == 0) {
    const int64_t units = 2 * mx_blocks(in);
    hipLaunchKernelGGL((mx_quantize_plain<FMT, InT>), dim3(unit_blocks(rows * units)), dim3(256),
                       0, stream, w, rows, in, units, codes, scales);
    return hipGetLastError();
  }
  MxSigns signs;
  mx_signs(seed, g, &signs);
  const double root = 1.0 / std::sqrt(double(g));
  const int64_t total = rows * in;
  for_group(g, [&](auto G) {
    constexpr int kG = decltype(G)::value;
    hipLaunchKernelGGL((mx_quantize_rht<kG, FMT, InT>), dim3(segment_blocks<kG>(total)),
                       dim3(64 * kWaves), 0, stream, w, total, signs, root, codes, scales);
  });
  return hipGetLastError();
}

template <int FMT, typename InT>
hipError_t tiles_typed(const InT* x, int64_t batch, int64_t in, int g, uint64_t seed,
                       const MxTiles& t, const MxScaleWords& words, hipStream_t stream) {
  MxSigns signs;
  double root = 0.0;
  if (g > 0) {
    mx_signs(seed, g, &signs);
    root = 1.0 / std::sqrt(double(g));
  }
  const int part = std::max(g, 1024), parts = int((in + part - 1) / part);
  const int64_t blocks = (batch + kTileRows - 1) / kTileRows * parts;
  const int word_parts = int(std::min<int64_t>((words.stages + 31) / 32, 64));
  const int64_t word_blocks = words.to == nullptr ? 0 : (words.rows + 63) / 64 * word_parts;
  const auto launch = [&](auto G) {
    hipLaunchKernelGGL((mx_to_tiles<decltype(G)::value, FMT, InT>),
                       dim3(unsigned(blocks + word_blocks)), dim3(64 * kTileRows), 0, stream, x,
                       int(batch), int(in), parts, int(blocks), signs, root, t, words, word_parts);
  };
  if (g == 0)
    launch(std::integral_constant<int, 0>{});
  else
    for_group(g, launch);
  return hipGetLastError();
}

template <int FMT, typename OutT>
hipError_t dequantize_typed(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t in,
                            int g, uint64_t seed, OutT* w, hipStream_t stream) {
  if (g == 0) {
    const int64_t units = 2 * mx_blocks(in);
    hipLaunchKernelGGL((mx_dequantize_plain<FMT, OutT>), dim3(unit_blocks(rows * units)),
                       dim3(256), 0, stream, codes, scales, rows, in, units, w);
    return hipGetLastError();
  }
  MxSigns signs;
  mx_signs(seed, g, &signs);
  const double factor = std::ldexp(1.0 / std::sqrt(double(g)), kBackShift);
  const MxBackRoot root{float(factor), float(factor - double(float(factor)))};
  const int64_t total = rows * in;
  for_group(g, [&](auto G) {
    constexpr int kG = decltype(G)::value;
    hipLaunchKernelGGL((mx_dequantize_rht<kG, FMT, OutT>), dim3(segment_blocks<kG>(total)),
                       dim3(64 * kWaves), 0, stream, codes, scales, total, signs, root, w);
  });
  return hipGetLastError();
}

template <typename InT>
hipError_t error_typed(const InT* w, int64_t out, int64_t in, const uint8_t* codes,
                       const uint8_t* scales, int g, uint64_t seed, double* row_err,
                       hipStream_t stream) {
  // waves of a row: one where the rows' waves fill the card, more of fewer rows (14336 x
  // 4096, g = 1024: 46 us with one, 58 with four; 1000 x 4096: 8.2 and 7.4)
  const int64_t segments = (in + std::max(g, 1024) - 1) / std::max(g, 1024);
  int split = 1;
  while (split < kWaves && out * split < 4096 && split < segments) split *= 2;
  const dim3 grid{unsigned((out * split + kWaves - 1) / kWaves)}, block{64 * kWaves};
  if (g == 0) {
    hipLaunchKernelGGL((mx_error_plain<InT>), grid, block, 0, stream, w, out, in,
                       2 * mx_blocks(in), split, codes, scales, row_err);
    return hipGetLastError();
  }
  MxSigns signs;
  mx_signs(seed, g, &signs);
  const double root = 1.0 / std::sqrt(double(g));
  for_group(g, [&](auto G) {
    hipLaunchKernelGGL((mx_error_rht<decltype(G)::value, InT>), grid, block, 0, stream, w, out, in,
                       split, signs, root, codes, scales, row_err);
  });
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const void* w, higgs_dtype dtype, int64_t rows, int64_t in, int fmt,
                              int g, uint64_t seed, uint8_t* codes, uint8_t* scales,
                              hipStream_t stream) {
  const auto run = [&](const auto* p) {
    return fmt == HIGGS_MX_FP4
               ? quantize_typed<HIGGS_MX_FP4>(p, rows, in, g, seed, codes, scales, stream)
               : quantize_typed<HIGGS_MX_FP6>(p, rows, in, g, seed, codes, scales, stream);
  };
  return dtype == HIGGS_F32 ? run(static_cast<const float*>(w))
                            : run(static_cast<const uint16_t*>(w));
}

hipError_t launch_mx_tiles(const void* x, higgs_dtype dtype, int64_t batch, int64_t in, int fmt,
                           int g, uint64_t seed, const MxTiles& tiles, const MxScaleWords& words,
                           hipStream_t stream) {
  const float* xf = static_cast<const float*>(x);
  const uint16_t* xb = static_cast<const uint16_t*>(x);
  if (fmt == HIGGS_MX_FP4)
    return dtype == HIGGS_F32
               ? tiles_typed<HIGGS_MX_FP4>(xf, batch, in, g, seed, tiles, words, stream)
               : tiles_typed<HIGGS_MX_FP4>(xb, batch, in, g, seed, tiles, words, stream);
  return dtype == HIGGS_F32
             ? tiles_typed<HIGGS_MX_FP6>(xf, batch, in, g, seed, tiles, words, stream)
             : tiles_typed<HIGGS_MX_FP6>(xb, batch, in, g, seed, tiles, words, stream);
}

hipError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows,
                                int64_t in, int fmt, int g, uint64_t seed, void* w,
                                higgs_dtype dtype, hipStream_t stream) {
  float* wf = static_cast<float*>(w);
  uint16_t* wb = static_cast<uint16_t*>(w);
  if (fmt == HIGGS_MX_FP4)
    return dtype == HIGGS_F32
               ? dequantize_typed<HIGGS_MX_FP4>(codes, scales, rows, in, g, seed, wf, stream)
               : dequantize_typed<HIGGS_MX_FP4>(codes, scales, rows, in, g, seed, wb, stream);
  return dtype == HIGGS_F32
             ? dequantize_typed<HIGGS_MX_FP6>(codes, scales, rows, in, g, seed, wf, stream)
             : dequantize_typed<HIGGS_MX_FP6>(codes, scales, rows, in, g, seed, wb, stream);
}

hipError_t launch_mx_layer_error(const void* w, higgs_dtype dtype, int64_t out, int64_t in,
                                 const uint8_t* codes, const uint8_t* scales, int g, uint64_t seed,
                                 double* row_err, double* t2, hipStream_t stream) {
  const hipError_t st =
      dtype == HIGGS_F32
          ? error_typed(static_cast<const float*>(w), out, in, codes, scales, g, seed, row_err,
                        stream)
          : error_typed(static_cast<const uint16_t*>(w), out, in, codes, scales, g, seed, row_err,
                        stream);
  if (st != hipSuccess || t2 == nullptr) return st;
  hipLaunchKernelGGL(mx_t2, dim3(1), dim3(1024), 0, stream, row_err, out, t2);
  return hipGetLastError();
}

}  // namespace higgs
