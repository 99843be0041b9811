// The microscaled product for few activation rows: a stream of the weights.
//
// A block takes tiles of 16 outputs, one after another; its waves share K in
// chunks of 512 (256 bytes of a weight row). A wave's chunk of a tile, 4 KiB, goes
// from memory into the wave's own LDS slots, requested one chunk ahead and with whole
// lines of each row, and from there into the 16x16x128 scaled matrix instruction, whose
// other operand is up to 16 activation rows; 32 with two of them. The waves' sums
// of a tile meet in LDS and are added in the waves' order.
//
// The activations come from the product's workspace (MxTiles), or, for calls that
// convert little (FUSED), each block rotates and quantizes them itself while its
// first weights are on their way, into LDS: one launch instead of two.
//
// What bounds it is the way from memory to LDS where a wave has many chunks (4 x 4096 ->
// 28672: 14.1 us among others, 62 MB, 4.4 TB/s), and where it has few its own waiting, 2.4
// us per chunk: a request is conditional (none behind the last tile, scale bytes one by
// one in a row's last chunk), so that the compiler cannot count the loads in flight and
// every second step of the loop waits for all of them, the chunk just requested included
// (16 x 14336 -> 4096: 16 us behind the conversion, 31 MB, 2 TB/s). One row of 4096 -> 4096
// takes 7.3 us, of which a launch and the conversion are half. 3 slots and 14 waves gained
// nothing, two blocks per compute unit with two tiles of rows lost.

#include <algorithm>

#include "mx_device.h"

namespace higgs {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kMaxWaves = 8;
// Values that a block converts itself; with a rotation at most 14 segments of 1024, two
// per wave. Above that the conversion takes longer than the launch that it saves (3 x 4096
// -> 4096 8.4 us fused and 8.8 not, 4 x 4096 9.5 and 8.9; with two waves, 4 x 1024 -> 1024
// 5.7 and 6.3, 16 x 1024 13.5 and 6.7).
constexpr int kFusedValues = 16384;
constexpr int kFusedSegments = 14;

// As few waves as take equal shares of a row's chunks in as many turns as the most would.
int waves_of(int64_t in) {
  const int64_t chunks = (in + 511) / 512, turns = (chunks + kMaxWaves - 1) / kMaxWaves;
  return int((chunks + turns - 1) / turns);
}

struct Args {
  const void* x;  // FUSED: raw activations
  MxTiles t;      // otherwise
  const uint8_t* wc;
  const uint8_t* ws;
  void* y;
  int64_t out;
  int batch, in, blocks, stages, chunks, tiles;
  int x_bf16, y_bf16;
  double root;
  MxSigns signs;
};

__device__ inline __amdgpu_buffer_rsrc_t rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, int(bytes), 0x00020000);
}

// The wave's LDS reads and writes are done, then all waves meet (loads to LDS for
// later chunks stay in flight).
__device__ inline void wait_lds_and_meet() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// G: FUSED with groups of G (0: no rotation); -1: activations from t. NT: tiles of
// 16 activation rows.
template <int FMT, int G, int NT>
__global__ __launch_bounds__(64 * kMaxWaves) void mx_decode(const Args a) {
  constexpr bool kFused = G >= 0;
  constexpr int kRingSlots = 2;
  constexpr int kSlot = 4096, kUnit2 = FMT == HIGGS_MX_FP6 ? 8 : 0;
  // LDS: the waves' slots, the last of them the rotation's scratch first; two tiles'
  // partial sums; FUSED: the activations (16- and 8-byte parts, scale words)
  constexpr int kWaveRing =
      (kRingSlots - 1) * kSlot + (G > 0 ? std::max(kSlot, kMxWaveLds<double> * 4) : kSlot);
  constexpr int kRing = kMaxWaves * kWaveRing, kPart = kMaxWaves * NT * 16 * 16 * 4;
  constexpr int kXBlocks = kFused ? kFusedValues / 32 + 16 * 16 : 0;  // (whole stages per row)
  constexpr int kX = kRing + 2 * kPart, kXTail = kX + kXBlocks * 16;
  constexpr int kXScale = kXTail + kXBlocks * kUnit2, kLds = kXScale + kXBlocks;
  static_assert(kLds <= 160 * 1024, "LDS");
  __shared__ __attribute__((aligned(1024))) uint8_t s_mem[kLds];

  const int tid = int(threadIdx.x), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int waves = int(blockDim.x) >> 6;
  const int r16 = lane & 15, q = lane >> 4;

  // ---- weights: chunk c of tile t into the wave's slot ----
  const __amdgpu_buffer_rsrc_t wrs = rsrc(a.wc, uint32_t(a.out * a.blocks * 16));
  uint8_t* const ring = s_mem + wave * kWaveRing;
  const int mine = (a.chunks - wave + waves - 1) / waves;  // chunks wave, wave + waves, ..
  // 4 rows of 256 bytes per load; a row's 16 blocks are permuted so that 16 rows of one
  // block lie in distinct banks
  auto issue = [&](int tile, int chunk, int slot) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = 4 * j + q, unit = r16 ^ row;
      const int64_t o = min(int64_t(tile) * 16 + row, a.out - 1);
      const uint32_t at = uint32_t(o) * uint32_t(a.blocks * 16) + uint32_t(chunk * 256 + unit * 16);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(wrs, (lds_void*)(ring + slot * kSlot + j * 1024), 16,
                                               int(at), 0, 0, 0);
    }
  };
  // ---- the scale bytes of the lane's row: a word per stage of the chunk ----
  auto load_scales = [&](int tile, int chunk, uint32_t (&s)[4]) {
    const uint8_t* const p =
        a.ws + min(int64_t(tile) * 16 + r16, a.out - 1) * a.blocks + chunk * 16;
    const int left = a.blocks - chunk * 16;
    if (left >= 16) {
      typedef uint32_t u32x4_a1 __attribute__((ext_vector_type(4), aligned(1)));
      const u32x4_a1 u = *reinterpret_cast<const u32x4_a1*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = u[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[i] = 0;
        for (int j = 0; j < 4; ++j)
          if (4 * i + j < left) s[i] |= uint32_t(p[4 * i + j]) << (8 * j);
      }
    }
  };

  // Items of the wave: its chunks of the block's tiles. An item's weights are requested
  // before its scales: loads arrive in order, so that where these have arrived the
  // weights have.
  struct Next {
    int tile, k;
  };
  auto advance = [&](Next& n) {
    if (++n.k == mine) {
      n.k = 0;
      n.tile += int(gridDim.x);
    }
  };
  struct Item {
    uint32_t ws[4], xs[4][NT];
    i32x8 x[4][NT];
  };
  Next next{int(blockIdx.x), 0};  // the next item to request
  auto request = [&](Item& f, int slot) {
    if (next.tile < a.tiles) {
      issue(next.tile, wave + next.k * waves, slot);
      // (the order that the waits rest on: no scale load is moved before these)
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      load_scales(next.tile, wave + next.k * waves, f.ws);
    }
  };
  Item f0 = {}, f1 = {};
  request(f0, 0);

  // ---- FUSED: the activations into LDS; block kb of row b is unit kb * batch + b ----
  const int batch = a.batch;
  if constexpr (kFused) {
    auto put = [&](int b, int half, const uint32_t* c) {
      uint8_t* const head = s_mem + kX + ((half >> 1) * batch + b) * 16;
      if constexpr (FMT == HIGGS_MX_FP4) {
        *reinterpret_cast<u32x2*>(head + (half & 1) * 8) = u32x2{c[0], c[1]};
      } else {
        uint32_t* const h = reinterpret_cast<uint32_t*>(head);
        uint32_t* const t =
            reinterpret_cast<uint32_t*>(s_mem + kXTail + ((half >> 1) * batch + b) * 8);
        if ((half & 1) == 0) {
          h[0] = c[0];
          h[1] = c[1];
          h[2] = c[2];
        } else {
          h[3] = c[0];
          t[0] = c[1];
          t[1] = c[2];
        }
      }
    };
    auto put_scale = [&](int b, int kb, uint32_t byte) {
      s_mem[kXScale + ((kb >> 2) * batch + b) * 4 + (kb & 3)] = uint8_t(byte);
    };
    if constexpr (G > 0) {
      uint32_t* const lds = reinterpret_cast<uint32_t*>(ring + (kRingSlots - 1) * kSlot);
      MxLaneSigns<G> neg(a.signs, lane);
      const int segs = (a.in + 1023) / 1024;  // of a row; the last may end early
      for (int i = wave; i < batch * segs; i += waves) {
        const int b = i / segs, seg = i - b * segs;
        const int64_t at = int64_t(b) * a.in + 1024 * seg;
        const int left = a.in - 1024 * seg;
        double v[16];
        if (a.x_bf16)
          signed_pairs(load_pairs(static_cast<const uint16_t*>(a.x) + at, left, lane), neg.of(0),
                       v);
        else
          signed_pairs(load_pairs(static_cast<const float*>(a.x) + at, left, lane), neg.of(0), v);
        uint32_t c[kWords16<FMT>], byte;
        mx_rotate_segment<G, FMT>(v, a.root, lds, lane, c, &byte);
        // (up to the end of the row's last stage: zeros behind its values)
        const int half = 64 * seg + lane;
        if (half < 8 * a.stages) {
          put(b, half, c);
          if ((lane & 1) == 0) put_scale(b, half >> 1, byte);
        }
      }
    } else {
      const int units = 8 * a.stages;
      for (int u = tid; u < batch * units; u += 64 * waves) {
        const int b = u / units, half = u - b * units;
        const int left = a.in - 16 * half, n = left < 0 ? 0 : left > 16 ? 16 : left;
        const int64_t at = int64_t(b) * a.in + (left > 0 ? 16 * half : 0);
        float x[16];
        if (a.x_bf16)
          load16_upto(static_cast<const uint16_t*>(a.x) + at, n, x);
        else
          load16_upto(static_cast<const float*>(a.x) + at, n, x);
        uint32_t c[kWords16<FMT>];
        const uint32_t byte = mx_plain_halves<FMT>(x, c);
        put(b, half, c);
        if ((half & 1) == 0) put_scale(b, half >> 1, byte);
      }
    }
    wait_lds_and_meet();
  }

  // ---- activations of stage t: block q of row r16 (+ 16) ----
  auto load_x = [&](int t, int n, i32x8& x, uint32_t& s) {
    u32x4 u;
    u32x2 v = {0, 0};
    if constexpr (kFused) {
      const int at = (4 * t + q) * batch + min(r16, batch - 1);
      u = *reinterpret_cast<const u32x4*>(s_mem + kX + at * 16);
      if constexpr (FMT == HIGGS_MX_FP6)
        v = *reinterpret_cast<const u32x2*>(s_mem + kXTail + at * 8);
      s = *reinterpret_cast<const uint32_t*>(s_mem + kXScale + (t * batch + min(r16, batch - 1)) * 4);
    } else {
      const uint8_t* const p = a.t.codes + (t * 2 + (q >> 1)) * mx_half_bytes(FMT);
      const int unit = (q & 1) * 32 + n * 16 + r16;
      u = *reinterpret_cast<const u32x4*>(p + unit * 16);
      if constexpr (FMT == HIGGS_MX_FP6) v = *reinterpret_cast<const u32x2*>(p + 1024 + unit * 8);
      s = *reinterpret_cast<const uint32_t*>(a.t.scales + (t * 32 + n * 16 + r16) * 4);
    }
    x = i32x8{int(u[0]), int(u[1]), int(u[2]), int(u[3]), int(v[0]), int(v[1]), 0, 0};
  };

  auto load_xs = [&](Item& f, int chunk) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int n = 0; n < NT; ++n)
        load_x(min(4 * chunk + s, a.stages - 1), n, f.x[s][n], f.xs[s][n]);
  };
  load_xs(f0, wave);
  if (mine == 1) load_xs(f1, wave);  // (one chunk per wave: the same for every tile)

  // ---- the stream: item f in slot `slot`, the next one requested into g ----
  int tile = int(blockIdx.x), k = 0, turn = 0;
  f32x4 acc[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto step = [&](Item& f, Item& g, int slot) {
    advance(next);
    __builtin_amdgcn_sched_barrier(0);
    request(g, slot ^ 1);
    if (mine > 1) load_xs(g, wave + next.k * waves);
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::"v"(f.ws[0]), "v"(f.ws[1]), "v"(f.ws[2]), "v"(f.ws[3]) : "memory");
    const int chunk = wave + k * waves;
    const uint8_t* const w0 = ring + slot * kSlot + r16 * 256;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4 u = *reinterpret_cast<const u32x4*>(w0 + ((4 * s + q) ^ r16) * 16);
      const i32x8 w = {int(u[0]), int(u[1]), int(u[2]), int(u[3]), 0, 0, 0, 0};
      if (4 * chunk + s < a.stages) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
          acc[n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              f.x[s][n], w, acc[n], FMT == HIGGS_MX_FP4 ? 4 : 2, 4, 0, int(f.xs[s][n] >> (8 * q)),
              0, int(f.ws[s] >> (8 * q)));
      }
    }
    // (the slot's reads are done before it is requested again, in the next step: their
    // data has been used above)
    if (++k < mine) return;
    // the tile's partial sums: rows 4 q + i of column r16
    k = 0;
    float* const part = reinterpret_cast<float*>(s_mem + kRing + turn * kPart);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int b = n * 16 + 4 * q + i;
        if (b < batch) part[(wave * NT * 16 + b) * 16 + r16] = acc[n][i];
      }
    wait_lds_and_meet();
    for (int i = tid; i < batch * 16; i += 64 * waves) {
      float t = 0.f;
      for (int w = 0; w < waves; ++w) t += part[w * NT * 256 + i];
      const int64_t o = int64_t(tile) * 16 + (i & 15);
      if (o < a.out) {
        const int64_t at = (i >> 4) * a.out + o;
        if (a.y_bf16)
          static_cast<uint16_t*>(a.y)[at] = uint16_t(pack_bf16(t, 0.f));
        else
          static_cast<float*>(a.y)[at] = t;
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
    tile += int(gridDim.x);
    turn ^= 1;
  };
  while (true) {
    step(f0, f1, 0);
    if (tile >= a.tiles) break;
    step(f1, f0, 1);
    if (tile >= a.tiles) break;
  }
}

template <int FMT, int G, int NT>
hipError_t launch(const Args& a, hipStream_t stream) {
  // as many blocks as the compute units hold, or fewer: two each, one where the
  // activations are in LDS too or with two tiles of them (16 x 4096 -> 28672 with 256
  // blocks instead of 512: 21.3 us, not 18.7)
  constexpr int kBlocks = G < 0 && NT == 1 ? 512 : 256;
  hipLaunchKernelGGL((mx_decode<FMT, G, NT>), dim3(unsigned(std::min(a.tiles, kBlocks))),
                     dim3(unsigned(64 * waves_of(a.in))), 0, stream, a);
  return hipGetLastError();
}

template <int FMT>
hipError_t launch_fmt(const Args& a, bool fused, int g, hipStream_t stream) {
  if (!fused)
    return a.batch <= 16 ? launch<FMT, -1, 1>(a, stream)
                         : launch<FMT, -1, 2>(a, stream);
  switch (g) {
    case 0: return launch<FMT, 0, 1>(a, stream);
    case 64: return launch<FMT, 64, 1>(a, stream);
    case 128: return launch<FMT, 128, 1>(a, stream);
    case 256: return launch<FMT, 256, 1>(a, stream);
    case 512: return launch<FMT, 512, 1>(a, stream);
    default: return launch<FMT, 1024, 1>(a, stream);
  }
}

}  // namespace

bool mx_decode_fuses(int64_t batch, int64_t in, int g) {
  if (batch > 16 || g > 1024 || batch * in > kFusedValues) return false;
  const int64_t segments = batch * ((in + 1023) / 1024);
  return g == 0 || (segments <= kFusedSegments && segments <= 2 * waves_of(in));
}

hipError_t launch_mx_decode(const void* x, higgs_dtype x_dtype, int64_t batch, int fmt,
                            const MxTiles& tiles, const uint8_t* codes, const uint8_t* scales,
                            int g, uint64_t seed, int64_t out, int64_t in, void* y,
                            higgs_dtype y_dtype, hipStream_t stream) {
  const bool fused = mx_decode_fuses(batch, in, g);
  Args a;
  a.x = x;
  a.t = tiles;
  a.wc = codes;
  a.ws = scales;
  a.y = y;
  a.out = out;
  a.batch = int(batch);
  a.in = int(in);
  a.blocks = int(mx_blocks(in));
  a.stages = int((in + 127) / 128);
  a.chunks = (a.stages + 3) / 4;
  a.tiles = int((out + 15) / 16);
  a.x_bf16 = x_dtype == HIGGS_BF16;
  a.y_bf16 = y_dtype == HIGGS_BF16;
  a.root = 0.0;
  if (fused && g > 0) {
    a.root = 1.0 / std::sqrt(double(g));
    mx_signs(seed, g, &a.signs);
  }
  return fmt == HIGGS_MX_FP4 ? launch_fmt<HIGGS_MX_FP4>(a, fused, g, stream)
                             : launch_fmt<HIGGS_MX_FP6>(a, fused, g, stream);
}

}  // namespace higgs
