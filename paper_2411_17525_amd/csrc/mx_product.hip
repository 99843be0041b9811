// y = x_hat W_hat^T for a 4-bit (E2M1) layer: the activations are rotated
// (where g > 0) and converted to E2M1 or E2M3 blocks by the quantizer's kernel,
// then multiplied by the scaled matrix instruction, which takes both operands'
// codes and one power of two per 32 values of K and lane. Products of these
// formats and their sums of 64 are exact in it; sums are fp32.
//
// Operands of v_mfma_scale_f32_32x32x64_f8f6f4 (either format): lane l holds
// the block l / 32 of two (32 consecutive values of K) of row l % 32 and its
// scale byte; of the result it holds column l % 32, rows i % 4 + 8 (i / 4) +
// 4 (l / 32). The activations are the rows, the weights the columns: a store of
// one register then writes 32 consecutive outputs.

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
  const uint8_t* ws;
  void* y;         // or fp32 partial sums [split][batch][out]
  int64_t batch, out;
  int blocks;      // of a weight row
  int ws_pitch;    // bytes of a row of weight scales, a multiple of 4
  int splits;      // of K
  int mtiles, ntiles;
};

constexpr int kBufs = 3;  // stages in LDS

template <int N>
__device__ inline void wait_vm() {
  // vmcnt <= N, the other counters free
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

__device__ inline __amdgpu_buffer_rsrc_t rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, int(bytes), 0x00020000);
}

// A block computes BM activation rows x BN outputs over a range of K with WM x WN
// waves, stage by stage of 128 values: the stage's activations, weights and scale
// words go from memory to LDS (kBufs stages; the loads run two and a half stages
// ahead), from there into the operands. A stage is computed in halves; the
// operands of a half are read while the other half is multiplied, and the one
// barrier of a stage stands between its halves: there the next stage has landed
// and this one has been read by all waves.
template <int BM, int BN, int WM, int WN, int FMT, typename OutT>
__global__ __launch_bounds__(64 * WM * WN, 1) void mx_product_tiles(const Args a) {
  constexpr int kWaves = WM * WN;
  constexpr int kHalf = mx_half_bytes(FMT), kTile = 2 * kHalf;
  constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr int kXBytes = BM / 32 * kTile, kWBytes = BN * 64;
  constexpr int kXScale = kXBytes + kWBytes, kWScale = kXScale + BM * 4;
  constexpr int kStage = kWScale + BN * 4;
  // loads of 1 KiB (codes) and 256 bytes (scales) per stage, and per wave; a wave
  // without one repeats the last
  constexpr int kXLoads = kXBytes / 1024, kWLoads = kWBytes / 1024;
  constexpr int kSLoads = (BM + BN) / 64;
  constexpr int kXPer = (kXLoads + kWaves - 1) / kWaves, kWPer = (kWLoads + kWaves - 1) / kWaves;
  constexpr int kSPer = (kSLoads + kWaves - 1) / kWaves;
  constexpr int kLoads = kXPer + kWPer + kSPer;
  static_assert(BM % 64 == 0 && BN % 64 == 0 && kBufs * kStage <= 160 * 1024, "tile");
  __shared__ __attribute__((aligned(1024))) uint8_t s_mem[kBufs * kStage];

  const int tid = int(threadIdx.x), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const int r32 = lane & 31, hi = lane >> 5;

  // ---- the block's tile: consecutive tiles per XCD, eight row tiles of one column
  //      after another (their weights stay in the XCD's L2) ----
  const int total = a.mtiles * a.ntiles * a.splits;
  const int xcd = int(blockIdx.x) % 8, turn = int(blockIdx.x) / 8;
  const int item = xcd * (total / 8) + min(xcd, total % 8) + turn;
  const int split = item / (a.mtiles * a.ntiles);
  const int tile = item - split * (a.mtiles * a.ntiles);
  constexpr int kBand = 8;
  const int band = tile / (kBand * a.ntiles), rest = tile - band * (kBand * a.ntiles);
  const int high = min(kBand, a.mtiles - band * kBand);
  const int nt = rest / high, mt = band * kBand + rest - nt * high;
  const int64_t m0 = int64_t(mt) * BM, n0 = int64_t(nt) * BN;
  const int stages = int(a.x.stages);
  const int first = int(int64_t(stages) * split / a.splits);
  const int count = int(int64_t(stages) * (split + 1) / a.splits) - first;

  // ---- loads of a stage ----
  const int mrows = int(min(int64_t(BM), a.x.rows32 - m0));   // a multiple of 32
  const int nrows = int(min(int64_t(BN), a.out - n0));
  const __amdgpu_buffer_rsrc_t xrs =
      rsrc(a.x.codes + m0 / 32 * stages * kTile, uint32_t(mrows / 32 * stages * kTile));
  const __amdgpu_buffer_rsrc_t wrs = rsrc(a.wc + n0 * a.blocks * 16, uint32_t(nrows * a.blocks * 16));
  const __amdgpu_buffer_rsrc_t xss = rsrc(a.x.scales + m0 * 4, uint32_t(((stages - 1) * a.x.rows32 + mrows) * 4));
  const __amdgpu_buffer_rsrc_t wss = rsrc(a.ws + n0 * a.ws_pitch, uint32_t(nrows * a.ws_pitch));
  uint32_t xoff[kXPer], woff[kWPer], soff[kSPer];
#pragma unroll
  for (int i = 0; i < kXPer; ++i) {
    const int j = min(wave + i * kWaves, kXLoads - 1);
    const int at = j * 1024 + lane * 16, t = min(at / kTile, mrows / 32 - 1);
    xoff[i] = uint32_t((t * stages + first) * kTile + at % kTile);
  }
#pragma unroll
  for (int i = 0; i < kWPer; ++i) {
    // 16 rows of 64 bytes; a row's four blocks are permuted so that eight rows of
    // one block lie in distinct banks
    const int row = min(wave + i * kWaves, kWLoads - 1) * 16 + lane / 4;
    const int unit = (lane & 3) ^ ((row >> 1) & 3);
    woff[i] = uint32_t(min(row, nrows - 1) * a.blocks * 16 + first * 64 + unit * 16);
  }
#pragma unroll
  for (int i = 0; i < kSPer; ++i) {
    const int j = min(wave + i * kWaves, kSLoads - 1);
    if (j < BM / 64)
      soff[i] = uint32_t((int64_t(first) * a.x.rows32 + min(j * 64 + lane, mrows - 1)) * 4);
    else
      soff[i] = uint32_t(min((j - BM / 64) * 64 + lane, nrows - 1) * a.ws_pitch + first * 4);
  }
  auto issue = [&](int buf) MX_INLINE {
    uint8_t* const s = s_mem + buf * kStage;
#pragma unroll
    for (int i = 0; i < kXPer; ++i) {
      const int j = min(wave + i * kWaves, kXLoads - 1);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(xrs, (lds_void*)(s + j * 1024), 16, int(xoff[i]), 0,
                                               0, 0);
      xoff[i] += kTile;
    }
#pragma unroll
    for (int i = 0; i < kWPer; ++i) {
      const int j = min(wave + i * kWaves, kWLoads - 1);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(wrs, (lds_void*)(s + kXBytes + j * 1024), 16,
                                               int(woff[i]), 0, 0, 0);
      woff[i] += 64;
    }
#pragma unroll
    for (int i = 0; i < kSPer; ++i) {
      const int j = min(wave + i * kWaves, kSLoads - 1);
      const bool is_x = j < BM / 64;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(is_x ? xss : wss, (lds_void*)(s + kXScale + j * 256),
                                               4, int(soff[i]), 0, 0, 0);
      soff[i] += is_x ? uint32_t(a.x.rows32 * 4) : 4u;
    }
  };

  // ---- operands of half h of the stage in buffer buf ----
  struct Half {
    i32x8 x[TM], w[TN];
    int xs[TM], ws[TN];
  };
  auto read = [&](Half& f, int buf, int h) MX_INLINE {
    const uint8_t* const s = s_mem + buf * kStage;
#pragma unroll
    for (int m = 0; m < TM; ++m) {
      const uint8_t* const p = s + (wm * TM + m) * kTile + h * kHalf;
      const u32x4 u = *reinterpret_cast<const u32x4*>(p + lane * 16);
      f.x[m] = i32x8{int(u[0]), int(u[1]), int(u[2]), int(u[3]), 0, 0, 0, 0};
      if constexpr (FMT == HIGGS_MX_FP6) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(p + 1024 + lane * 8);
        f.x[m][4] = int(v[0]);
        f.x[m][5] = int(v[1]);
      }
      f.xs[m] = *reinterpret_cast<const int*>(s + kXScale + ((wm * TM + m) * 32 + r32) * 4);
    }
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      const int row = (wn * TN + n) * 32 + r32;
      const int unit = (2 * h + hi) ^ ((row >> 1) & 3);
      const u32x4 u = *reinterpret_cast<const u32x4*>(s + kXBytes + row * 64 + unit * 16);
      f.w[n] = i32x8{int(u[0]), int(u[1]), int(u[2]), int(u[3]), 0, 0, 0, 0};
      f.ws[n] = *reinterpret_cast<const int*>(s + kWScale + row * 4);
    }
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int m = 0; m < TM; ++m)
#pragma unroll
    for (int n = 0; n < TN; ++n) acc[m][n] = f32x16{};
  auto multiply = [&](const Half& f, auto H) MX_INLINE {
    constexpr int h = decltype(H)::value;  // its scale is byte 2 h + lane / 32 of the word
    constexpr int kFormat = FMT == HIGGS_MX_FP4 ? 4 : 2;
    int xs[TM], ws[TN];
#pragma unroll
    for (int m = 0; m < TM; ++m) xs[m] = int(uint32_t(f.xs[m]) >> (8 * hi));
#pragma unroll
    for (int n = 0; n < TN; ++n) ws[n] = int(uint32_t(f.ws[n]) >> (8 * hi));
#pragma unroll
    for (int m = 0; m < TM; ++m)
#pragma unroll
      for (int n = 0; n < TN; ++n)
        acc[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
            f.x[m], f.w[n], acc[m][n], kFormat, 4, 2 * h, xs[m], 2 * h, ws[n]);
  };
  using H0 = std::integral_constant<int, 0>;
  using H1 = std::integral_constant<int, 1>;

  for (int t = 0; t < min(kBufs, count); ++t) issue(t);
  Half f0, f1;
  if (count >= kBufs)
    wait_vm<2 * kLoads>();
  else
    wait_vm<0>();
  __syncthreads();
  read(f0, 0, 0);
  int buf = 0;
  for (int t = 0; t < count; ++t) {
    const int next = buf == kBufs - 1 ? 0 : buf + 1;
    read(f1, buf, 1);
    multiply(f0, H0{});
    // the next stage's loads are the oldest but kLoads (stage t + 2); the last
    // stages just wait for all
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (t + 2 < count)
      wait_vm<kLoads>();
    else
      wait_vm<0>();
    asm volatile("s_barrier" ::: "memory");
    if (t + kBufs < count) issue(buf);
    read(f0, next, 0);
    multiply(f1, H1{});
    buf = next;
  }

  // ---- outputs ----
  const bool partial = a.splits > 1;
  const int64_t bw = m0 + wm * TM * 32 + 4 * hi, ow = n0 + wn * TN * 32 + r32;
  const int64_t at = (partial ? split * a.batch * a.out : 0) + bw * a.out + ow;
  const int brows = int(min(a.batch - bw, int64_t(BM))), ocols = int(min(a.out - ow, int64_t(BN)));
  float* const yf = static_cast<float*>(a.y) + at;
  uint16_t* const yb = static_cast<uint16_t*>(a.y) + at;
#pragma unroll
  for (int m = 0; m < TM; ++m)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int b = m * 32 + i % 4 + 8 * (i / 4);
      const int64_t row = b * a.out;
#pragma unroll
      for (int n = 0; n < TN; ++n)
        if (b < brows && n * 32 < ocols) {
          if (sizeof(OutT) == 4 || partial)
            yf[row + n * 32] = acc[m][n][i];
          else
            yb[row + n * 32] = uint16_t(f32_to_bf16(acc[m][n][i]));
        }
    }
}

// Rows of scale bytes to a pitch of whole words, zeros behind the row.
__global__ __launch_bounds__(256) void mx_pad_scales(const uint8_t* __restrict__ s, int64_t rows,
                                                     int blocks, int pitch,
                                                     uint32_t* __restrict__ d) {
  const int words = pitch / 4;
  const int64_t total = rows * words, step = int64_t(gridDim.x) * 256;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += step) {
    const int64_t row = i / words;
    const int k = int(i - row * words) * 4;
    uint32_t w = 0;
    for (int j = 0; j < 4; ++j)
      if (k + j < blocks) w |= uint32_t(s[row * blocks + k + j]) << (8 * j);
    d[i] = w;
  }
}

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

// The workspace: activation codes and scales, padded weight scales (only where
// the caller's have another pitch or alignment).
struct Plan {
  int64_t stages, rows32, x_bytes, xs_bytes, ws_bytes;
  int64_t bytes() const { return x_bytes + xs_bytes + ws_bytes; }
};
Plan plan_of(int64_t batch, int64_t out, int64_t in, int fmt) {
  Plan p;
  p.stages = (in + 127) / 128;
  p.rows32 = (batch + 31) / 32 * 32;
  p.x_bytes = up256(p.rows32 / 32 * p.stages * 2 * mx_half_bytes(fmt));
  p.xs_bytes = up256(p.rows32 * p.stages * 4);
  p.ws_bytes = up256(out * p.stages * 4);
  return p;
}

template <int BM, int BN, int WM, int WN, int FMT, typename OutT>
hipError_t launch_tiles(Args a, hipStream_t stream) {
  a.mtiles = int((a.batch + BM - 1) / BM);
  a.ntiles = int((a.out + BN - 1) / BN);
  a.splits = 1;
  const auto kernel = mx_product_tiles<BM, BN, WM, WN, FMT, OutT>;
  hipLaunchKernelGGL(kernel, dim3(unsigned(a.mtiles * a.ntiles * a.splits)), dim3(64 * WM * WN),
                     0, stream, a);
  return hipGetLastError();
}

}  // namespace

int64_t mx_qmatmul_workspace_bytes(int64_t batch, int64_t out, int64_t in, int fmt, int g) {
  (void)g;
  return plan_of(batch, out, in, fmt).bytes();
}

hipError_t launch_mx_qmatmul(const void* x, higgs_dtype x_dtype, int64_t batch, int fmt,
                             const uint8_t* codes, const uint8_t* scales, int g, uint64_t seed,
                             int64_t out, int64_t in, void* y, higgs_dtype y_dtype,
                             void* workspace, hipStream_t stream) {
  const Plan p = plan_of(batch, out, in, fmt);
  uint8_t* const w = static_cast<uint8_t*>(workspace);
  Args a{};
  a.x = MxTiles{w, w + p.x_bytes, p.stages, p.rows32};
  hipError_t st = launch_mx_tiles(x, x_dtype, batch, in, fmt, g, seed, a.x, stream);
  if (st != hipSuccess) return st;
  a.wc = codes;
  a.ws = scales;
  a.y = y;
  a.batch = batch;
  a.out = out;
  a.blocks = int(mx_blocks(in));
  a.ws_pitch = a.blocks;
  if (a.blocks % 4 != 0 || reinterpret_cast<uintptr_t>(scales) % 4 != 0) {
    a.ws_pitch = int(p.stages * 4);
    uint32_t* const d = reinterpret_cast<uint32_t*>(w + p.x_bytes + p.xs_bytes);
    const int64_t words = out * p.stages;
    hipLaunchKernelGGL(mx_pad_scales, dim3(unsigned(std::min<int64_t>((words + 255) / 256, 4096))),
                       dim3(256), 0, stream, scales, out, a.blocks, a.ws_pitch, d);
    st = hipGetLastError();
    if (st != hipSuccess) return st;
    a.ws = reinterpret_cast<const uint8_t*>(d);
  }
  if (fmt == HIGGS_MX_FP4)
    return y_dtype == HIGGS_F32
               ? launch_tiles<256, 256, 2, 2, HIGGS_MX_FP4, float>(a, stream)
               : launch_tiles<256, 256, 2, 2, HIGGS_MX_FP4, uint16_t>(a, stream);
  return y_dtype == HIGGS_F32
             ? launch_tiles<256, 256, 2, 2, HIGGS_MX_FP6, float>(a, stream)
             : launch_tiles<256, 256, 2, 2, HIGGS_MX_FP6, uint16_t>(a, stream);
}

}  // namespace higgs
