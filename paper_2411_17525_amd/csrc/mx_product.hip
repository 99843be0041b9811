// y = x_hat W_hat^T for a 4-bit (E2M1) layer: the activations are rotated
// (where g > 0) and converted to E2M1 or E2M3 blocks by the quantizer's kernel,
// then multiplied by the scaled matrix instruction, which takes both operands'
// codes and one power of two per 32 values of K and lane. Products of these
// formats are exact in it (with E4M3 activations it drops low bits and runs at half
// the rate, so those of more than 4 bits are E2M3); sums are fp32.
//
// Operands of v_mfma_scale_f32_32x32x64_f8f6f4 (either format): lane l holds
// the block l / 32 of two (32 consecutive values of K) of row l % 32 and its
// scale byte; of the result it holds column l % 32, rows i % 4 + 8 (i / 4) +
// 4 (l / 32). The activations are the rows, the weights the columns.
//
// What bounds it: matrix instructions at the clock that they leave (47% of the cycles at
// 1.75 GHz for 2048 x 4096 -> 28672 with E2M3, 150 us in two launches behind a fill of the
// caches, 3.2 PFLOP/s; the instruction alone, fed from LDS, reaches 5.7), the starts and
// outputs of tiles, which all compute units reach together, and for few tiles the latency
// of a stage's loads.

#include <algorithm>

#include "mx.h"
#include "wave_fwht.h"

namespace higgs {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void lds_void;

#define MX_INLINE __attribute__((always_inline))

struct Args {
  MxTiles x;
  const uint8_t* wc;
  const uint32_t* ws;  // weight scales, a word per stage and row: [stage][pitch]
  void* y;             // or fp32 partial sums [split][batch][out]
  int64_t batch, out;
  int64_t pitch;  // of a row of y and of ws, in values: out, or more for a part of the outputs
  int blocks;  // of a weight row
  int splits;  // of K
  int mtiles, ntiles, band;
};

template <int N>
__device__ inline void wait_vm() {
  // vmcnt <= N, the other counters free
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

__device__ inline __amdgpu_buffer_rsrc_t rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, int(bytes), 0x00020000);
}

// All of the wave's LDS reads have arrived, then all waves of the block meet.
__device__ inline void wait_lds_and_meet() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// f(0), f(1), ... f(N - 1) with constants.
template <int N, int I = 0, typename F>
__device__ MX_INLINE inline void for_each(const F& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    for_each<N, I + 1>(f);
  }
}

// A block computes tiles of BM activation rows x BN outputs over a range of K with
// WM x WN waves, one after another, stage by stage of 128 values: the stage's
// activations, weights and scale words go from memory to LDS, from there into the
// operands. The loads run NB - 1/2 stages ahead. Weights are loaded for two stages at
// a time, 128 bytes of a row: the address unit takes about as long for half a line as
// for a whole one (62, 88 and 106 GB/s per compute unit in pieces of 64, 128 and 256
// bytes), and that time is what the products have to hide. So that every stage loads as much,
// the block's first half of columns has its pairs of stages at (0, 1), (2, 3) ..,
// the second at (-1, 0), (1, 2) .. (NB is odd; a range of K has an even number of
// stages). The loads run on into the next tile, so that its first stages arrive while
// this one's outputs are stored. A stage is computed in halves; the
// operands of a half are read while the other half is multiplied, and the one
// barrier of a stage stands between its halves: there the next stage has landed
// and this one has been read by all waves.
template <int BM, int BN, int WM, int WN, int NB, int PERCU, int FMT, typename OutT>
__global__ __launch_bounds__(64 * WM * WN, WM * WN * PERCU / 4) void mx_product_tiles(
    const Args a) {
  constexpr int kWaves = WM * WN;
  constexpr int kHalf = mx_half_bytes(FMT), kTile = 2 * kHalf;
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  // LDS: NB stages of activations and scale words; of each half of the columns
  // (NB + 1) / 2 pairs of weights
  constexpr int kXRows = BM < 64 ? 64 : BM;  // scale words come by 64
  constexpr int kXBytes = BM / 32 * kTile, kXScale = kXBytes, kWScale = kXScale + kXRows * 4;
  constexpr int kStage = kWScale + BN * 4, kPair = BN / 2 * 128, kWeights = NB * kStage;
  constexpr int kPairs = (NB + 1) / 2, kLds = kWeights + 2 * kPairs * kPair;
  // loads of 1 KiB (codes) and 256 bytes (scales) per stage, and per wave; a wave
  // without one repeats the last
  constexpr int kXLoads = kXBytes / 1024, kWLoads = kPair / 1024, kSLoads = (kXRows + BN) / 64;
  constexpr int kXPer = (kXLoads + kWaves - 1) / kWaves, kWPer = kWLoads / kWaves;
  constexpr int kSPer = (kSLoads + kWaves - 1) / kWaves, kLoads = kXPer + kSPer + kWPer;
  static_assert(BM % 32 == 0 && BN % 64 == 0 && NB % 2 == 1 && NB >= 3, "tile");
  static_assert(PERCU * kLds <= 160 * 1024 && (NB - 1) * kLoads + kWPer < 64, "tile");
  __shared__ __attribute__((aligned(1024))) uint8_t s_mem[kLds];

  const int tid = int(threadIdx.x), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int r32 = lane & 31, hi = lane >> 5;

  // ---- the block's tiles: consecutive ones per XCD, dealt to its blocks in turn; a band
  //      of row tiles of one column after another (their weights stay in the XCD's L2) ----
  const int total = a.mtiles * a.ntiles * a.splits;
  const int xcd = int(blockIdx.x) % 8, step = (int(gridDim.x) + 7) / 8;  // (its blocks)
  const int end = (xcd + 1) * (total / 8) + min(xcd + 1, total % 8);
  struct Tile {
    int item, mt, nt, split, first, count;
  };
  const int stages = int(a.x.stages);
  auto locate = [&](int item) MX_INLINE {
    auto uniform = [](int v) MX_INLINE { return __builtin_amdgcn_readfirstlane(v); };
    Tile r;
    r.item = item;
    r.split = uniform(item / (a.mtiles * a.ntiles));
    const int tile = item - r.split * (a.mtiles * a.ntiles);
    const int band = uniform(tile / (a.band * a.ntiles)), rest = tile - band * (a.band * a.ntiles);
    const int high = min(a.band, a.mtiles - band * a.band);
    r.nt = uniform(rest / high);
    r.mt = band * a.band + rest - r.nt * high;
    r.first = uniform(stages / 2 * r.split / a.splits) * 2;
    r.count = uniform(stages / 2 * (r.split + 1) / a.splits) * 2 - r.first;
    return r;
  };
  Tile now = locate(xcd * (total / 8) + min(xcd, total % 8) + int(blockIdx.x) / 8);

  // ---- loads: stage `lstage` of tile `ltile`, ahead of the products. Past the last tile
  //      they read nothing (no records, or offsets out of range), but are issued: the
  //      waits count them ----
  Tile ltile = now;
  int lstage = 0;
  constexpr uint32_t kNowhere = 0xC0000000u;  // (codes are below 2 GiB)
  const __amdgpu_buffer_rsrc_t wrs = rsrc(a.wc, uint32_t(a.out * a.blocks * 16));
  const uint8_t *xp, *xsp;
  const uint32_t* wsp;
  uint32_t xbytes, xsbytes, wsbytes;
  uint32_t xoff[kXPer], woff[2][kWPer], soff[kSPer];  // (woff[0]: of the next stage's half)
  // 8 rows of 128 bytes per load; a row's eight blocks are permuted so that 16 rows of
  // one block lie in distinct banks (of 64, two rows)
  static_assert(kWLoads % kWaves == 0 && kWaves % 2 == 0, "row = 8 wave + lane / 8 mod 16");
  const int wunit = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
  // LDS row 32 (TN w + n) + c holds column TN (32 w + c) + n of the tile: a lane's TN
  // accumulators of a row are consecutive outputs
  auto row_offset = [&](const Tile& t, int i, int side) MX_INLINE {
    const int place = (wave + i * kWaves) * 8 + lane / 8 + side * (BN / 2);
    const int row = place / (32 * TN) * (32 * TN) + place % 32 * TN + place / 32 % TN;
    const int64_t o = min(int64_t(t.nt) * BN + row, a.out - 1);
    // (the second half's first pair begins a stage early: what that reads is not used)
    return uint32_t(o) * uint32_t(a.blocks * 16) + uint32_t(t.first * 64 + wunit * 16 - side * 64);
  };
  auto begin_tile = [&] MX_INLINE {  // activations and scales of ltile from its first stage
    const bool live = ltile.item < end;
    const int64_t m0 = int64_t(ltile.mt) * BM, n0 = int64_t(ltile.nt) * BN;
    const int mrows = int(min(int64_t(BM), a.x.rows32 - m0));  // a multiple of 32
    const int nrows = int(min(int64_t(BN), a.out - n0));
    xp = a.x.codes + (m0 / 32 * stages + ltile.first) * kTile;
    xsp = a.x.scales + (ltile.first * a.x.rows32 + m0) * 4;
    wsp = a.ws + ltile.first * a.pitch + n0;
    xbytes = live ? uint32_t(((mrows / 32 - 1) * stages + ltile.count) * kTile) : 0;
    xsbytes = live ? uint32_t(((ltile.count - 1) * a.x.rows32 + mrows) * 4) : 0;
    wsbytes = live ? uint32_t(((ltile.count - 1) * a.pitch + nrows) * 4) : 0;
#pragma unroll
    for (int i = 0; i < kXPer; ++i) {
      const int j = min(wave + i * kWaves, kXLoads - 1);
      const int at = j * 1024 + lane * 16, t = min(at / kTile, mrows / 32 - 1);
      xoff[i] = uint32_t(t * stages * kTile + at % kTile);
    }
#pragma unroll
    for (int i = 0; i < kSPer; ++i) {
      const int j = min(wave + i * kWaves, kSLoads - 1);
      soff[i] = j < kXRows / 64 ? uint32_t(min(j * 64 + lane, mrows - 1) * 4)
                                : uint32_t(min((j - kXRows / 64) * 64 + lane, nrows - 1) * 4);
    }
  };
  begin_tile();
#pragma unroll
  for (int i = 0; i < kWPer; ++i) {
    woff[0][i] = row_offset(now, i, 1);
    woff[1][i] = row_offset(now, i, 0);
  }
  // Before the loads of a tile's last stage: the second columns' pair that it begins
  // ends with the next tile's first stage (the upper four blocks of each row).
  uint32_t cross[kWPer];
  auto begin_stage = [&] MX_INLINE {
    if (lstage != ltile.count - 1) return;
    const int item = ltile.item + step;
    if (item < end) {
      ltile = locate(item);
#pragma unroll
      for (int i = 0; i < kWPer; ++i) cross[i] = row_offset(ltile, i, 1);
    } else {
      ltile.item = item;
#pragma unroll
      for (int i = 0; i < kWPer; ++i) cross[i] = kNowhere;
    }
    lstage = -1;
#pragma unroll
    for (int i = 0; i < kWPer; ++i) woff[0][i] = wunit >= 4 ? cross[i] : woff[0][i];
  };
  auto end_stage = [&] MX_INLINE {
    if (++lstage != 0) return;
    begin_tile();
#pragma unroll
    for (int i = 0; i < kWPer; ++i) {
      woff[0][i] = ltile.item < end ? row_offset(ltile, i, 0) : kNowhere;
      woff[1][i] = cross[i] + 128;
    }
  };
  // Load k of this wave (constant) into stage buffer buf and, the weights of column half
  // `side`, into its pair buffer lpair; the offsets one stage or pair on, the weights'
  // exchanged with the other half's.
  auto issue = [&](auto K, int side, int buf, int lpair) MX_INLINE {
    constexpr int k = decltype(K)::value;
    uint8_t* const s = s_mem + buf * kStage;
    if constexpr (k < kXPer) {
      const int j = min(wave + k * kWaves, kXLoads - 1);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(xp, xbytes), (lds_void*)(s + j * 1024), 16,
                                               int(xoff[k]), 0, 0, 0);
      xoff[k] += kTile;
    } else if constexpr (k < kXPer + kSPer) {
      constexpr int i = k - kXPer;
      const int j = min(wave + i * kWaves, kSLoads - 1);
      const bool is_x = j < kXRows / 64;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rsrc(is_x ? static_cast<const void*>(xsp) : wsp, is_x ? xsbytes : wsbytes),
          (lds_void*)(s + kXScale + j * 256), 4, int(soff[i]), 0, 0, 0);
      soff[i] += uint32_t(is_x ? a.x.rows32 : a.pitch) * 4;
    } else {
      constexpr int i = k - kXPer - kSPer;
      const int j = wave + i * kWaves;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          wrs, (lds_void*)(s_mem + kWeights + (side * kPairs + lpair) * kPair + j * 1024), 16,
          int(woff[0][i]), 0, 0, 0);
      const uint32_t other = woff[1][i];
      woff[1][i] = woff[0][i] + 128;
      woff[0][i] = other;
    }
  };

  // ---- operands of half h of the stage in buffer buf ----
  struct Half {
    uint32_t x[TM][6], w[TN][4];
  };
  uint32_t words[TM + TN], scales[TM + TN];  // the next stage's scale words; this one's
  // (the tails' addresses apart: two of them read by one instruction would have to
  // be moved into place)
  uint32_t tail[TM];
#pragma unroll
  for (int m = 0; m < TM; ++m) {
    tail[m] = uint32_t((wm * TM + m) * kTile + 1024 + lane * 8);
    asm volatile("" : "+v"(tail[m]));
  }
  // read k of a half's operands, in the order in which the products need them: the
  // first row tile, all column tiles, the other row tiles; then the scale words
  constexpr int kXReads = FMT == HIGGS_MX_FP6 ? 2 : 1;
  constexpr int kReads = TM * kXReads + TN, kScaleReads = TM + 1;
  auto read = [&](auto K, Half& f, int t, int buf, int pair0, int pair1, int h) MX_INLINE {
    constexpr int k = decltype(K)::value;
    const uint8_t* const s = s_mem + buf * kStage;
    if constexpr (k >= kReads) {
      constexpr int q = k - kReads;
      if constexpr (q < TM) {
        words[q] =
            *reinterpret_cast<const uint32_t*>(s + kXScale + ((wm * TM + q) * 32 + r32) * 4);
      } else {
        typedef uint32_t run_t __attribute__((ext_vector_type(TN)));
        const run_t u = *reinterpret_cast<const run_t*>(s + kWScale + (wn * 32 + r32) * TN * 4);
#pragma unroll
        for (int n = 0; n < TN; ++n) words[TM + n] = u[n];
      }
    } else if constexpr (k >= kXReads && k < kXReads + TN) {
      constexpr int n = k - kXReads;
      const int row = (wn * TN + n) * 32 + r32;
      const int side = row / (BN / 2);  // (the same in all lanes)
      const int pair = __builtin_amdgcn_readfirstlane(side ? kPairs + pair1 : pair0);
      const int odd = __builtin_amdgcn_readfirstlane((t + side) & 1);
      const int unit = (4 * odd + 2 * h + hi) ^ ((row >> 1) & 7);
      const u32x4 u = *reinterpret_cast<const u32x4*>(
          s_mem + kWeights + pair * kPair + (row - side * (BN / 2)) * 128 + unit * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) f.w[n][i] = u[i];
    } else {
      constexpr int q = k < kXReads ? k : k - TN, m = q / kXReads, part = q % kXReads;
      if constexpr (part == 0) {
        const u32x4 u =
            *reinterpret_cast<const u32x4*>(s + (wm * TM + m) * kTile + h * kHalf + lane * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) f.x[m][i] = u[i];
      } else {
        const u32x2 u = *reinterpret_cast<const u32x2*>(s + tail[m] + h * kHalf);
        f.x[m][4] = u[0];
        f.x[m][5] = u[1];
      }
    }
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int m = 0; m < TM; ++m)
#pragma unroll
    for (int n = 0; n < TN; ++n) acc[m][n] = f32x16{};
  // product k of a half; the scale bytes of half h are byte 2 h + lane / 32 of the words,
  // moved down by lane / 32 bytes in `scales`
  auto multiply = [&](auto K, const Half& f, auto H) MX_INLINE {
    constexpr int m = decltype(K)::value / TN, n = decltype(K)::value % TN;
    constexpr int h = decltype(H)::value, kFormat = FMT == HIGGS_MX_FP4 ? 4 : 2;
    const i32x8 x = {int(f.x[m][0]), int(f.x[m][1]), int(f.x[m][2]), int(f.x[m][3]),
                     FMT == HIGGS_MX_FP6 ? int(f.x[m][4]) : 0,
                     FMT == HIGGS_MX_FP6 ? int(f.x[m][5]) : 0, 0, 0};
    const i32x8 w = {int(f.w[n][0]), int(f.w[n][1]), int(f.w[n][2]), int(f.w[n][3]), 0, 0, 0, 0};
    acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
        x, w, acc[m][n], kFormat, 4, 2 * h, int(scales[m]), 2 * h, int(scales[TM + n]));
  };
  using H0 = std::integral_constant<int, 0>;
  using H1 = std::integral_constant<int, 1>;

  // One half of a stage: its products, behind each a share of the reads of the
  // half that comes next (done by three quarters of the products) and of the loads
  // [L0, L1) (spread over all: a wave that issues several at a time waits for the
  // address unit, and its products wait behind them). The order is kept as written.
  constexpr int kProducts = TM * TN;
  struct Place {
    int stage, buf, pair0, pair1;  // pair0, pair1: the pair buffers of both column halves
  };
  auto half = [&](const Half& now, auto H, Half& next, const Place& np, int nh, auto L0, auto L1,
                  int lside, int lbuf, int lpair) MX_INLINE {
    constexpr int kOver = kProducts >= 4 ? kProducts * 3 / 4 : kProducts;
    constexpr int l0 = decltype(L0)::value, nl = decltype(L1)::value - l0;
    constexpr int kAll = kReads + (decltype(H)::value == 1 ? kScaleReads : 0);
    for_each<kProducts>([&](auto I) MX_INLINE {
      constexpr int i = decltype(I)::value;
      multiply(I, now, H);
      constexpr int ra = kAll * (i < kOver ? i : kOver) / kOver;
      constexpr int rb = kAll * (i + 1 < kOver ? i + 1 : kOver) / kOver;
      for_each<rb - ra>([&](auto J) MX_INLINE {
        read(std::integral_constant<int, ra + decltype(J)::value>{}, next, np.stage, np.buf,
             np.pair0, np.pair1, nh);
      });
      constexpr int la = l0 + nl * i / kProducts, lb = l0 + nl * (i + 1) / kProducts;
      for_each<lb - la>([&](auto J) MX_INLINE {
        issue(std::integral_constant<int, la + decltype(J)::value>{}, lside, lbuf, lpair);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // The loads for stage t + NB go out from the meeting of stage t on, where their
  // buffers are free: the first of them in its half 1, the others in half 0 of stage
  // t + 1. So at the meeting of stage t the loads for the stages from t + 2 may be
  // outstanding, those for t + 1 not.
  using L0 = std::integral_constant<int, 0>;
  using LH = std::integral_constant<int, (kLoads + 1) / 2>;
  using LN = std::integral_constant<int, kLoads>;
  for_each<kWPer>([&](auto K) MX_INLINE {  // (the second columns' pair that ends with stage 0)
    issue(std::integral_constant<int, kXPer + kSPer + decltype(K)::value>{}, 1, 0, 0);
  });
  for_each<NB - 1>([&](auto T) MX_INLINE {
    constexpr int t = decltype(T)::value;
    begin_stage();
    for_each<kLoads>([&](auto K) MX_INLINE { issue(K, t & 1, t, (t + 1) / 2); });
    end_stage();
  });
  begin_stage();
  for_each<LH::value>([&](auto K) MX_INLINE { issue(K, 0, NB - 1, NB / 2); });
  wait_vm<(NB - 2) * kLoads + LH::value>();
  wait_lds_and_meet();
  Half f0, f1;
  for_each<kReads + kScaleReads>([&](auto K) MX_INLINE { read(K, f0, 0, 0, 0, 0, 0); });
  // lpair: the pair buffer of the loads for stage t + NB - 1; pair0, pair1: those of
  // stage t. A pair's buffer is taken up two stages later by the pair kPairs on.
  Place at{0, 0, 0, 0};
  int before = NB - 1, lpair = NB / 2;
  auto wrap = [](int v, int n) MX_INLINE { return v == n ? 0 : v; };
  // Stores of whole tiles stay in flight over the first meeting of the next tile: at
  // least that many operations are younger than the loads it waits for.
  constexpr int kStores = TM * 16;
  constexpr int kRelaxed = (NB - 2) * kLoads + kStores < 63 ? (NB - 2) * kLoads + kStores : 63;
  bool relaxed = false;
  while (true) {
    for (int t = 0; t < now.count; ++t) {
      const int odd = t & 1;
      const Place next{t + 1, wrap(at.buf + 1, NB), wrap(at.pair0 + odd, kPairs),
                       wrap(at.pair1 + 1 - odd, kPairs)};
#pragma unroll
      for (int q = 0; q < TM + TN; ++q) scales[q] = words[q] >> (8 * hi);
      __builtin_amdgcn_sched_barrier(0);
      half(f0, H0{}, f1, at, 1, LH{}, LN{}, odd, before, lpair);
      if (relaxed) {
        wait_vm<kRelaxed>();
        relaxed = false;
      } else {
        wait_vm<(NB - 2) * kLoads>();
      }
      end_stage();
      begin_stage();
      wait_lds_and_meet();
      __builtin_amdgcn_sched_barrier(0);
      // (stage t + NB's columns' half is that of stage t + 1: its last pair has ended)
      const int freed = odd ? at.pair0 : at.pair1;
      half(f1, H1{}, f0, next, 0, L0{}, LH{}, 1 - odd, at.buf, freed);
      before = at.buf;
      lpair = freed;
      at = next;
    }
    at.stage = 0;

    // ---- outputs: register i of accumulator n holds row i % 4 + 8 (i / 4) + 4 hi, column
    //      TN r32 + n ----
    const bool partial = a.splits > 1;
    const int64_t bw = int64_t(now.mt) * BM + wm * TM * 32;
    const int64_t ow = int64_t(now.nt) * BN + wn * TN * 32;
    const int brows = int(min(a.batch - bw, int64_t(BM))) - 4 * hi;
    const int ocols = int(min(a.out - ow, int64_t(BN))) - TN * r32;
    const bool full = a.batch - bw >= TM * 32 && a.out - ow >= TN * 32;
    auto each_row = [&](auto f) MX_INLINE {
#pragma unroll
      for (int m = 0; m < TM; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) f(m, i, m * 32 + i % 4 + 8 * (i / 4));
    };
    if (sizeof(OutT) == 4 || partial) {
      typedef float run_t __attribute__((ext_vector_type(TN), aligned(4)));
      float* const y = static_cast<float*>(a.y) + (partial ? now.split * a.batch * a.pitch : 0) +
                       bw * a.pitch + ow;
      const uint32_t lane_at = uint32_t(4 * hi) * uint32_t(a.pitch) + uint32_t(TN * r32);
      each_row([&](int m, int i, int b) MX_INLINE {
        if (full) {
          run_t v;
#pragma unroll
          for (int n = 0; n < TN; ++n) v[n] = acc[m][n][i];
          *reinterpret_cast<run_t*>(y + b * a.pitch + lane_at) = v;
        } else if (b < brows) {
#pragma unroll
          for (int n = 0; n < TN; ++n)
            if (n < ocols) y[b * a.pitch + lane_at + n] = acc[m][n][i];
        }
      });
    } else {
      uint16_t* const y = static_cast<uint16_t*>(a.y) + bw * a.pitch + ow;
      const uint32_t lane_at = uint32_t(4 * hi) * uint32_t(a.pitch) + uint32_t(TN * r32);
      each_row([&](int m, int i, int b) MX_INLINE {
        uint32_t v[(TN + 1) / 2];
#pragma unroll
        for (int n = 0; n < TN; n += 2)
          v[n / 2] = pack_bf16(acc[m][n][i], n + 1 < TN ? acc[m][n + 1 < TN ? n + 1 : n][i] : 0.f);
        if (full && TN > 1) {
          typedef uint32_t run_t __attribute__((ext_vector_type((TN + 1) / 2), aligned(2)));
          run_t u;
#pragma unroll
          for (int n = 0; n < TN / 2; ++n) u[n] = v[n];
          *reinterpret_cast<run_t*>(y + b * a.pitch + lane_at) = u;
        } else if (b < brows) {
#pragma unroll
          for (int n = 0; n < TN; ++n)
            if (n < ocols) y[b * a.pitch + lane_at + n] = uint16_t(v[n / 2] >> (16 * (n & 1)));
        }
      });
    }
    if (now.item + step >= end) break;
    now = locate(now.item + step);
    relaxed = full;
#pragma unroll
    for (int m = 0; m < TM; ++m)
#pragma unroll
      for (int n = 0; n < TN; ++n) acc[m][n] = f32x16{};
  }
  wait_vm<0>();
}

// Sums of the splits in their order, four outputs at a time.
template <typename OutT>
__global__ __launch_bounds__(256) void mx_sum_splits(const float* __restrict__ part, int splits,
                                                     int64_t total, OutT* __restrict__ y) {
  typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (i >= total) return;
  const int n = int(min(total - i, int64_t(4)));
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (n == 4) {
    for (int s = 0; s < splits; ++s) {
      const f32x4_a4 u = *reinterpret_cast<const f32x4_a4*>(part + s * total + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += u[j];
    }
  } else {
    for (int s = 0; s < splits; ++s)
      for (int j = 0; j < n; ++j) v[j] += part[s * total + i + j];
  }
  if constexpr (sizeof(OutT) == 4) {
    if (n == 4)
      *reinterpret_cast<float4*>(y + i) = make_float4(v[0], v[1], v[2], v[3]);
    else
      for (int j = 0; j < n; ++j) y[i + j] = v[j];
  } else {
    if (n == 4)
      *reinterpret_cast<uint2*>(y + i) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    else
      for (int j = 0; j < n; ++j) y[i + j] = OutT(pack_bf16(v[j], 0.f));
  }
}

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

// The block shapes, and what a block takes (us): a stage where its loads bound it, a
// stage's share of its compute unit where that is what bounds it, the start and the
// outputs of a tile. Fitted to 2500 calls of 20 .. 2048 rows and nine layers (outputs
// x K from 512 x 512 to 28672 x 4096), each under every shape and 1 .. 8 splits: the
// plan that is fastest by these numbers takes 0.7% longer than the fastest measured
// one on average, 11% at most.
struct Shape {
  int bm, bn, percu;
  double latency, share, tile;
};
constexpr Shape kShapes[] = {{256, 256, 1, 0.54, 0.82, 5.7},
                             {128, 128, 2, 0.43, 0.38, 2.9},
                             {64, 128, 2, 0.37, 0.28, 2.6},
                             {32, 128, 2, 0.26, 0.25, 1.9},
                             {128, 256, 1, 0.13, 0.57, 4.2}};
constexpr int64_t kCus = 256;

double plan_us(const Shape& s, int splits, int64_t batch, int64_t out, int64_t in,
               int64_t stages) {
  const int64_t items = (batch + s.bm - 1) / s.bm * ((out + s.bn - 1) / s.bn) * splits;
  const int64_t rounds = items / (kCus * s.percu), rest = items % (kCus * s.percu);
  const double n = double((stages / 2 + splits - 1) / splits * 2);
  double t = double(rounds) * (s.tile + n * std::max(s.latency, s.percu * s.share));
  if (rest > 0)
    t += s.tile + n * std::max(s.latency, double((rest + kCus - 1) / kCus) * s.share);
  t = std::max(t, double(out) * double(in) * 0.54 / 4.5e6);  // the weights from memory
  // partial sums written and read at 9.7 TB/s (mostly in cache), a launch of 2.9 us
  if (splits > 1) t += 2.9 + double(batch) * double(out) * 4 * (2 * splits + 1) / 9.7e6;
  return t;
}

// Up to 16 rows the weights are streamed (mx_decode); up to 32 where that is faster: a
// block's share of the tiles of 16 outputs times a wave's share of the chunks, 2.4 us
// each, against the tile product with its scale words (20 x 4096 -> 4096: 8.9 us
// against 12.7; 20 x 13824 -> 5120: 25.1 against 20.3).
constexpr int64_t kStreamRows = 32;
double stream_us(int64_t out, int64_t in) {
  const int64_t tiles = (out + 15) / 16, chunks = (in + 511) / 512;
  return 1.6 + 2.4 * double((tiles + kCus - 1) / kCus) * double((chunks + 7) / 8);
}

struct Choice {
  int shape, splits;
  double us;
};
// The fastest shape and number of splits (up to max_splits) of a product.
Choice best_of(int64_t batch, int64_t out, int64_t in, int64_t stages, int max_splits) {
  Choice best{-1, 1, 0.0};
  for (const Shape& s : kShapes)
    for (int k = 1; k <= max_splits && k <= stages / 2; ++k) {
      const double t = plan_us(s, k, batch, out, in, stages);
      if (best.shape < 0 || t < best.us) best = Choice{int(&s - kShapes), k, t};
    }
  return best;
}

// A call's product, or two over parts of the outputs, and workspace: activation codes
// and scales, weight scale words, partial sums.
struct Plan {
  Choice main;      // shape -1: mx_decode
  Choice rest;      // of the outputs from `cut`, where that is below `out`
  int64_t cut;
  int64_t stages, rows32, x_bytes, xs_bytes, ws_bytes, part_bytes;
  int64_t bytes() const { return x_bytes + xs_bytes + ws_bytes + part_bytes; }
};
Plan plan_of(int64_t batch, int64_t out, int64_t in, int fmt, int g) {
  Plan p{};
  p.main = Choice{-1, 1, 0.0};
  p.cut = out;
  p.stages = (in + 255) / 256 * 2;
  p.rows32 = (batch + 31) / 32 * 32;
  p.x_bytes = up256(p.rows32 / 32 * p.stages * 2 * mx_half_bytes(fmt));
  p.xs_bytes = up256(p.rows32 * p.stages * 4);
  if (batch > 16) {
    const Choice c = best_of(batch, out, in, p.stages, 8);
    if (batch > kStreamRows ||
        c.us + double(out) * double(in) * 0.052e-6 < stream_us(out, in))
      p.main = c;
  }
  if (p.main.shape < 0) {
    if (mx_decode_fuses(batch, in, g)) p.x_bytes = p.xs_bytes = 0;
    return p;
  }
  // Tiles that fill whole rounds of a shape as one product, the columns left over as
  // another of smaller blocks instead of a round that leaves units idle (in two and in one,
  // fp32 outputs: 2048 x 4096 -> 18432 122.9 us and 127.7, 1024 x 4096 -> 35840 120.8 and
  // 126.8, but 2048 x 1024 -> 9001 38.4 and 31.2; 2048 x 4096 -> 28672 to bf16 159.4 and
  // 159.7).
  for (const Shape& s : kShapes) {
    const int64_t mt = (batch + s.bm - 1) / s.bm, nt = (out + s.bn - 1) / s.bn;
    const int64_t rounds = mt * nt / (kCus * s.percu);
    const int64_t cut = rounds * kCus * s.percu / mt * s.bn;
    if (rounds < 1 || cut < 1 || cut >= out) continue;
    const Choice first{int(&s - kShapes), 1, plan_us(s, 1, batch, cut, in, p.stages)};
    const Choice rest = best_of(batch, out - cut, in, p.stages, 1);
    // (and a launch's gap)
    if (first.us + rest.us + 3.0 < p.main.us + (p.cut < out ? p.rest.us + 3.0 : 0.0)) {
      p.main = first;
      p.rest = rest;
      p.cut = cut;
    }
  }
  p.ws_bytes = up256(out * p.stages * 4);
  p.part_bytes = p.main.splits > 1 ? up256(p.main.splits * batch * out * 4) : 0;
  return p;
}

template <int BM, int BN, int WM, int WN, int NB, int PERCU, int FMT, typename OutT>
hipError_t launch_tiles(const Args& a, hipStream_t stream) {
  hipLaunchKernelGGL((mx_product_tiles<BM, BN, WM, WN, NB, PERCU, FMT, OutT>),
                     dim3(unsigned(std::min(a.mtiles * a.ntiles * a.splits, 256 * PERCU))),
                     dim3(64 * WM * WN), 0, stream, a);
  return hipGetLastError();
}

template <int FMT, typename OutT>
hipError_t launch_shape(int shape, Args a, hipStream_t stream) {
  a.mtiles = int((a.batch + kShapes[shape].bm - 1) / kShapes[shape].bm);
  a.ntiles = int((a.out + kShapes[shape].bn - 1) / kShapes[shape].bn);
  // bands of equal height near four (2048 x 4096 -> 28672, conversion included, takes 159.4
  // us with four row tiles, 162.0 with two, 161.3 with eight), up to six in one
  const int bands = std::max(1, (a.mtiles + 1) / 4);
  a.band = (a.mtiles + bands - 1) / bands;
  // (4-bit activations leave room for five stages of two blocks of 64 x 128: 19.0 us for 200
  // x 4096 -> 8192, 21.9 with three; 128 x 256 gains nothing from five)
  switch (shape) {
    case 0: return launch_tiles<256, 256, 4, 2, 3, 1, FMT, OutT>(a, stream);
    case 1: return launch_tiles<128, 128, 2, 2, 3, 2, FMT, OutT>(a, stream);
    case 2:
      return launch_tiles<64, 128, 2, 2, FMT == HIGGS_MX_FP4 ? 5 : 3, 2, FMT, OutT>(a, stream);
    case 3: return launch_tiles<32, 128, 1, 4, 5, 2, FMT, OutT>(a, stream);
    default: return launch_tiles<128, 256, 2, 4, 3, 1, FMT, OutT>(a, stream);
  }
}

template <int FMT, typename OutT>
hipError_t launch_product(const Plan& p, const Args& args, float* part, hipStream_t stream) {
  Args a = args;
  a.splits = p.main.splits;
  a.out = p.cut;
  if (a.splits > 1) a.y = part;
  hipError_t st = launch_shape<FMT, OutT>(p.main.shape, a, stream);
  if (st != hipSuccess) return st;
  if (p.cut < args.out) {
    a.out = args.out - p.cut;
    a.wc += p.cut * a.blocks * 16;
    a.ws += p.cut;
    a.y = static_cast<OutT*>(args.y) + p.cut;
    return launch_shape<FMT, OutT>(p.rest.shape, a, stream);
  }
  if (a.splits == 1) return hipSuccess;
  const int64_t total = a.batch * a.out;
  hipLaunchKernelGGL((mx_sum_splits<OutT>), dim3(unsigned((total + 1023) / 1024)), dim3(256), 0,
                     stream, part, a.splits, total, static_cast<OutT*>(args.y));
  return hipGetLastError();
}

}  // namespace

int64_t mx_qmatmul_workspace_bytes(int64_t batch, int64_t out, int64_t in, int fmt, int g) {
  return plan_of(batch, out, in, fmt, g).bytes();
}

hipError_t launch_mx_qmatmul(const void* x, higgs_dtype x_dtype, int64_t batch, int fmt,
                             const uint8_t* codes, const uint8_t* scales, int g, uint64_t seed,
                             int64_t out, int64_t in, void* y, higgs_dtype y_dtype,
                             void* workspace, hipStream_t stream) {
  const Plan p = plan_of(batch, out, in, fmt, g);
  uint8_t* const w = static_cast<uint8_t*>(workspace);
  uint32_t* const words = reinterpret_cast<uint32_t*>(w + p.x_bytes + p.xs_bytes);
  float* const part = reinterpret_cast<float*>(w + p.x_bytes + p.xs_bytes + p.ws_bytes);
  Args a{};
  a.x = MxTiles{w, w + p.x_bytes, p.stages, p.rows32};
  hipError_t st = hipSuccess;
  const MxScaleWords w_scales{scales, p.ws_bytes > 0 ? words : nullptr, out, int(mx_blocks(in)),
                              int(p.stages)};
  if (p.x_bytes > 0)
    st = launch_mx_tiles(x, x_dtype, batch, in, fmt, g, seed, a.x, w_scales, stream);
  if (st != hipSuccess) return st;
  if (p.main.shape < 0)
    return launch_mx_decode(x, x_dtype, batch, fmt, a.x, codes, scales, g, seed, out, in, y,
                            y_dtype, stream);
  a.wc = codes;
  a.ws = words;
  a.y = y;
  a.batch = batch;
  a.out = out;
  a.pitch = out;
  a.blocks = int(mx_blocks(in));
  if (fmt == HIGGS_MX_FP4)
    return y_dtype == HIGGS_F32 ? launch_product<HIGGS_MX_FP4, float>(p, a, part, stream)
                                : launch_product<HIGGS_MX_FP4, uint16_t>(p, a, part, stream);
  return y_dtype == HIGGS_F32 ? launch_product<HIGGS_MX_FP6, float>(p, a, part, stream)
                              : launch_product<HIGGS_MX_FP6, uint16_t>(p, a, part, stream);
}

}  // namespace higgs
