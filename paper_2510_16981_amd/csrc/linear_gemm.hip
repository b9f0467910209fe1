// Matrix products of 8-bit linear layers: C = A B^T of two 8-bit matrices, and
// the weight gradient dW = X^T dY of an 8-bit and a 16-bit one.
#include "linear_device.h"

namespace muonbp {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t scale_at(const BlocksRef& m, int64_t row, int64_t col) {
  return gload<uint32_t, 4>(m.scales + col / kGroupCols * m.scale_ld + row) >> (8 * (col / kBlockCols % 4)) & 255u;
}

template <typename T>
__device__ __forceinline__ void finish(const DenseRef& c, int64_t row, int64_t col, float v, bool accumulate) {
  T* p = static_cast<T*>(c.ptr) + row * c.ld + col;
  if (accumulate) v += to_f(*p);
  *p = T(v);
}

// One 64 x 64 tile a workgroup, a 32 x 32 quarter a wave, operands straight from
// memory: lane l has row l % 32 of A and of B and 32 of every 64 bytes.
template <typename T, Fp8 F>
__global__ __launch_bounds__(kThreads) void k_product(BlocksRef a, BlocksRef b, DenseRef c, bool accumulate) {
  const int64_t wide = (c.cols + 63) / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t m0 = blockIdx.x / wide * 64 + 32 * (wave >> 1), n0 = blockIdx.x % wide * 64 + 32 * (wave & 1);
  const int64_t m = m0 + (lane & 31), n = n0 + (lane & 31);
  f32x16_t acc = {};
  for (int64_t k = 0; k < a.cols; k += 64) {
    const int64_t at = k + 32 * (lane >> 5);
    uint32_t x[8] = {}, y[8] = {};
    uint32_t sx = 127, sy = 127;
    if (m < a.rows) {
      sx = scale_at(a, m, k);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = gload<uint32_t, 4>(a.data + m * a.ld + at + 4 * i);
    }
    if (n < b.rows) {
      sy = scale_at(b, n, k);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = gload<uint32_t, 4>(b.data + n * b.ld + at + 4 * i);
    }
    if constexpr (sizeof(T) == 2) {
      i32x8_t xv, yv;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xv[i] = int(x[i]);
        yv[i] = int(y[i]);
      }
      acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xv, yv, acc, F == Fp8::E4M3 ? 0 : 1, 0, 0, int(sx), 0,
                                                            int(sy));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x2_t x0 = widen4<F>(x[2 * i], scale_of(sx)), x1 = widen4<F>(x[2 * i + 1], scale_of(sx));
        const u32x2_t y0 = widen4<Fp8::E4M3>(y[2 * i], scale_of(sy)), y1 = widen4<Fp8::E4M3>(y[2 * i + 1], scale_of(sy));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8_t, u32x4_t{x0[0], x0[1], x1[0], x1[1]}),
            __builtin_bit_cast(bf16x8_t, u32x4_t{y0[0], y0[1], y1[0], y1[1]}), acc, 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int64_t row = m0 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
    if (row < c.rows && n < c.cols) finish<T>(c, row, n, acc[v], accumulate);
  }
}

// One 64 x 64 tile of dW a workgroup; 16 tokens at a time go through LDS as
// bf16, transposed.
template <typename T, Fp8 F>
__global__ __launch_bounds__(kThreads) void k_weight_grad(BlocksRef x, DenseRef dy, DenseRef dw, bool accumulate) {
  __shared__ __attribute__((aligned(16))) uint16_t xs[64][16], ys[64][16];
  const int64_t wide = (dw.cols + 63) / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t i0 = blockIdx.x / wide * 64, o0 = blockIdx.x % wide * 64;
  const int wi = 32 * (wave >> 1), wo = 32 * (wave & 1);
  f32x16_t acc = {};
  for (int64_t t0 = 0; t0 < x.rows; t0 += 16) {
    const int64_t t = t0 + (tid >> 4);
    const int c = 4 * (tid & 15);
    u32x2_t q = {0, 0};
    if (t < x.rows && i0 + c < x.cols)
      q = widen4<F>(gload<uint32_t, 4>(x.data + t * x.ld + i0 + c), scale_of(scale_at(x, t, i0 + c)));
    xs[c][tid >> 4] = uint16_t(q[0]);
    xs[c + 1][tid >> 4] = uint16_t(q[0] >> 16);
    xs[c + 2][tid >> 4] = uint16_t(q[1]);
    xs[c + 3][tid >> 4] = uint16_t(q[1] >> 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t o = o0 + c + e;
      ys[c + e][tid >> 4] = t < x.rows && o < dy.cols
                                ? gload<uint16_t, 2>(static_cast<const uint16_t*>(dy.ptr) + t * dy.ld + o)
                                : uint16_t(0);
    }
    __syncthreads();
    const bf16x8_t p = *reinterpret_cast<const bf16x8_t*>(&xs[wi + (lane & 31)][8 * (lane >> 5)]);
    const bf16x8_t r = *reinterpret_cast<const bf16x8_t*>(&ys[wo + (lane & 31)][8 * (lane >> 5)]);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p, r, acc, 0, 0, 0);
    __syncthreads();
  }
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const int64_t row = i0 + wi + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3), col = o0 + wo + (lane & 31);
    if (row < dw.rows && col < dw.cols) finish<T>(dw, row, col, acc[v], accumulate);
  }
}

}  // namespace

hipError_t launch_product(DType out_t, Fp8 a_fmt, const BlocksRef& a, const BlocksRef& b, const DenseRef& c,
                          bool accumulate, const SplitSpace&, int, hipStream_t s) {
  const unsigned tiles = unsigned((c.rows + 63) / 64 * ((c.cols + 63) / 64));
  auto go = [&](auto k) { k<<<tiles, kThreads, 0, s>>>(a, b, c, accumulate); };
  if (out_t == DType::BF16)
    a_fmt == Fp8::E4M3 ? go(k_product<bf16, Fp8::E4M3>) : go(k_product<bf16, Fp8::E5M2>);
  else
    a_fmt == Fp8::E4M3 ? go(k_product<float, Fp8::E4M3>) : go(k_product<float, Fp8::E5M2>);
  return hipGetLastError();
}

hipError_t launch_weight_grad(DType out_t, Fp8 x_fmt, const BlocksRef& x, const DenseRef& dy, const DenseRef& dw,
                              bool accumulate, const SplitSpace&, int, hipStream_t s) {
  const unsigned tiles = unsigned((dw.rows + 63) / 64 * ((dw.cols + 63) / 64));
  auto go = [&](auto k) { k<<<tiles, kThreads, 0, s>>>(x, dy, dw, accumulate); };
  if (out_t == DType::BF16)
    x_fmt == Fp8::E4M3 ? go(k_weight_grad<bf16, Fp8::E4M3>) : go(k_weight_grad<bf16, Fp8::E5M2>);
  else
    x_fmt == Fp8::E4M3 ? go(k_weight_grad<float, Fp8::E4M3>) : go(k_weight_grad<float, Fp8::E5M2>);
  return hipGetLastError();
}

}  // namespace muonbp
