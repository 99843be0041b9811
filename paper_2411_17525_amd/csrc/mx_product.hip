// y = x_hat W_hat^T for a 4-bit (E2M1) layer: the activations are rotated
// (where g > 0) and converted to E2M1 or E2M3 blocks by the quantizer's kernel,
// then multiplied by the scaled matrix instruction, which takes both operands'
// codes and one power of two per 32 values of K and lane. Products of these
// formats and their sums of 128 are exact in it; sums are fp32.
//
// Operands of v_mfma_scale_f32_16x16x128_f8f6f4 (either format): lane l holds
// the block l / 16 of four (32 consecutive values of K) of row l % 16 and its
// scale byte; of the result it holds column l % 16, rows 4 (l / 16) ..

#include "mx.h"

namespace higgs {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Args {
  const uint8_t* xc;  // activation codes and scales, as mx_quantize writes them
  const uint8_t* xs;
  const uint8_t* wc;
  const uint8_t* ws;
  void* y;
  int64_t batch, out, blocks;  // blocks of 32 in a row
};

template <int FMT>
__device__ inline i32x8 load_operand(const uint8_t* p) {
  i32x8 a = {0, 0, 0, 0, 0, 0, 0, 0};
  if constexpr (FMT == HIGGS_MX_FP4) {
    const u32x4 u = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = int(u[i]);
  } else {
    const u32x2* q = reinterpret_cast<const u32x2*>(p);
#pragma unroll
    for (int h = 0; h < 3; ++h) {
      const u32x2 u = q[h];
      a[2 * h] = int(u[0]);
      a[2 * h + 1] = int(u[1]);
    }
  }
  return a;
}

// The instruction's code for a format.
template <int FMT>
constexpr int kMfmaFormat = FMT == HIGGS_MX_FP4 ? 4 : 2;

// One wave: 16 output features x 16 activation rows, all of K.
template <int FMT, typename OutT>
__global__ __launch_bounds__(64) void mx_product_16(const Args a) {
  const int lane = int(threadIdx.x), r = lane & 15, q = lane >> 4;
  const int64_t o0 = int64_t(blockIdx.x) * 16, b0 = int64_t(blockIdx.y) * 16;
  const int64_t orow = min(o0 + r, a.out - 1), brow = min(b0 + r, a.batch - 1);
  constexpr int kBytes = FMT == HIGGS_MX_FP4 ? 16 : 24;
  const uint8_t* wc = a.wc + orow * a.blocks * 16;
  const uint8_t* ws = a.ws + orow * a.blocks;
  const uint8_t* xc = a.xc + brow * a.blocks * kBytes;
  const uint8_t* xs = a.xs + brow * a.blocks;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int64_t k = q; k - q < a.blocks; k += 4) {
    i32x8 w = {0, 0, 0, 0, 0, 0, 0, 0}, x = w;
    int sw = 0, sx = 0;
    if (k < a.blocks) {
      w = load_operand<HIGGS_MX_FP4>(wc + k * 16);
      x = load_operand<FMT>(xc + k * kBytes);
      sw = ws[k];
      sx = xs[k];
    }
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, 4, kMfmaFormat<FMT>, 0, sw,
                                                           0, sx);
  }
  if (b0 + r >= a.batch) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t o = o0 + 4 * q + i;
    if (o >= a.out) continue;
    if constexpr (sizeof(OutT) == 4) {
      static_cast<float*>(a.y)[(b0 + r) * a.out + o] = acc[i];
    } else {
      static_cast<uint16_t*>(a.y)[(b0 + r) * a.out + o] = uint16_t(f32_to_bf16(acc[i]));
    }
  }
}

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

}  // namespace

int64_t mx_qmatmul_workspace_bytes(int64_t batch, int64_t out, int64_t in, int fmt, int g) {
  (void)out;
  (void)g;
  return up256(batch * mx_blocks(in) * mx_block_bytes(fmt)) + up256(batch * mx_blocks(in));
}

hipError_t launch_mx_qmatmul(const void* x, higgs_dtype x_dtype, int64_t batch, int fmt,
                             const uint8_t* codes, const uint8_t* scales, int g, uint64_t seed,
                             int64_t out, int64_t in, void* y, higgs_dtype y_dtype,
                             void* workspace, hipStream_t stream) {
  uint8_t* const xc = static_cast<uint8_t*>(workspace);
  uint8_t* const xs = xc + up256(batch * mx_blocks(in) * mx_block_bytes(fmt));
  const hipError_t st =
      launch_mx_quantize(x, x_dtype, batch, in, fmt, g, seed, xc, xs, stream);
  if (st != hipSuccess) return st;
  const Args a{xc, xs, codes, scales, y, batch, out, mx_blocks(in)};
  const dim3 grid(unsigned((out + 15) / 16), unsigned((batch + 15) / 16)), block(64);
  if (fmt == HIGGS_MX_FP4) {
    if (y_dtype == HIGGS_F32)
      hipLaunchKernelGGL((mx_product_16<HIGGS_MX_FP4, float>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((mx_product_16<HIGGS_MX_FP4, uint16_t>), grid, block, 0, stream, a);
  } else {
    if (y_dtype == HIGGS_F32)
      hipLaunchKernelGGL((mx_product_16<HIGGS_MX_FP6, float>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((mx_product_16<HIGGS_MX_FP6, uint16_t>), grid, block, 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace higgs
