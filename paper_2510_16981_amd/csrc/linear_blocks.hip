// Kernels between 16- or 32-bit matrices and 8-bit blocks, and the gated
// activation with 8-bit checkpoints.  All stream their operands once and are
// bound by memory (traced, inputs not cached): 16384 x 4096 quantized in 39 us
// (5.2 TB/s) and restored in 30 (6.6), gated 8192 x 14336 forward in 165 us (5.7) and
// backward in 169 (5.6); a large copy reaches 4.97.
//
// One wave holds one row of one group of 512 columns: lane l has columns 8 l ..
// 8 l + 7 (16 bytes of bf16 in, 8 bytes out), 16 lanes one block of 128, and the
// wave one word of scales.  (Two or four rows a wave were no faster: in a loop over
// the same buffers, partly cached, 16384 x 4096 quantized in 35.4 against 34.7 us,
// 64 x 4096 in 3.6 against 2.5.)
#include "linear_device.h"

namespace muonbp {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// The row and the group of columns of this wave; neighbouring waves hold
// neighbouring groups of a row.
struct Strip {
  int64_t row, group, col;
  int lane;
  __device__ __forceinline__ explicit Strip(int64_t cols) {
    lane = threadIdx.x & 63;
    const uint32_t groups = uint32_t((cols + kGroupCols - 1) / kGroupCols);
    const uint32_t w = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    row = w / groups;
    group = w % groups;
    col = group * kGroupCols + 8 * lane;
  }
};

unsigned strip_blocks(int64_t rows, int64_t cols) {
  return unsigned((rows * ((cols + kGroupCols - 1) / kGroupCols) + kWaves - 1) / kWaves);
}

// Eight values of a row (n of them inside the matrix) to 8 bits: the values
// and the biased exponent of the lane's block.
template <Fp8 F>
__device__ __forceinline__ u32x2_t round_block(const float f[8], uint32_t& byte) {
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, finite_abs(f[i]));
  byte = scale_byte<F>(max16(a));
  return pack8<F>(f, inverse_of(byte));
}

// The word of scales of this wave's row: a byte for each of its 16-lane rows,
// 0 for a block past the matrix.
__device__ __forceinline__ uint32_t scale_word(uint32_t byte, bool in) {
  const int b = in ? int(byte) : 0;
  return uint32_t(__builtin_amdgcn_readlane(b, 0)) | uint32_t(__builtin_amdgcn_readlane(b, 16)) << 8 |
         uint32_t(__builtin_amdgcn_readlane(b, 32)) << 16 | uint32_t(__builtin_amdgcn_readlane(b, 48)) << 24;
}

__device__ __forceinline__ int left(int64_t cols, int64_t col) {
  const int64_t n = cols - col;
  return int(n < 0 ? 0 : n > 8 ? 8 : n);
}

// Columns up to the end of the last block are written (zeros past the
// matrix).
__device__ __forceinline__ bool block_in(int64_t cols, int64_t col) { return (col & ~int64_t(kBlockCols - 1)) < cols; }

template <Fp8 F>
__device__ __forceinline__ void store_blocks(const BlocksRef& o, const Strip& s, const float f[8]) {
  uint32_t byte;
  const u32x2_t q = round_block<F>(f, byte);
  const bool in = block_in(o.cols, s.col);
  if (in) gstore<u32x2_t, 8>(o.data + s.row * o.ld + s.col, q);
  const uint32_t w = scale_word(byte, in);
  if (s.lane == 0) gstore<uint32_t, 4>(o.scales + s.group * o.scale_ld + s.row, w);
}

template <Fp8 F>
__device__ __forceinline__ void load_blocks(const BlocksRef& x, const Strip& s, float f[8]) {
  if (block_in(x.cols, s.col)) {
    const uint32_t w = gload<uint32_t, 4>(x.scales + s.group * x.scale_ld + s.row);
    unpack8<F>(gload<u32x2_t, 8>(x.data + s.row * x.ld + s.col), scale_of(w >> (8 * (s.lane >> 4)) & 255u), f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
  }
}

template <typename T, Fp8 F>
__global__ __launch_bounds__(kThreads) void k_quantize(DenseRef x, BlocksRef out) {
  const Strip s(x.cols);
  if (s.row >= x.rows) return;
  float f[8];
  load8(static_cast<const T*>(x.ptr) + s.row * x.ld + s.col, left(x.cols, s.col), f);
  store_blocks<F>(out, s, f);
}

template <typename T, Fp8 F>
__global__ __launch_bounds__(kThreads) void k_restore(BlocksRef x, DenseRef out) {
  const Strip s(x.cols);
  if (s.row >= x.rows) return;
  float f[8];
  load_blocks<F>(x, s, f);
  store8(static_cast<T*>(out.ptr) + s.row * out.ld + s.col, left(x.cols, s.col), f);
}

// One workgroup a 128 x 128 tile: thread t has columns 8 (t % 16) .. + 7 of rows
// t / 16, 16 + t / 16, ...; the tile's max through LDS, then the values in rows
// and, through LDS, in columns.  4096 x 14336 in bf16 to both layouts: 52 us
// (4.5 TB/s).
constexpr int kTilePitch = kBlockCols + 4;

template <typename T, Fp8 F>
__global__ __launch_bounds__(kThreads) void k_quantize_weight(DenseRef w, BlocksRef out, BlocksRef out_t) {
  __shared__ uint32_t top[kWaves];
  __shared__ __attribute__((aligned(16))) uint8_t tile[kBlockCols * kTilePitch];
  const int64_t wide = (w.cols + kBlockCols - 1) / kBlockCols;
  const int64_t bi = blockIdx.x / wide, bj = blockIdx.x % wide;
  const int64_t r0 = bi * kBlockCols, c0 = bj * kBlockCols;
  const int tid = threadIdx.x, tr = tid >> 4, tc = 8 * (tid & 15);
  const int n = left(w.cols, c0 + tc);
  float f[8][8];
  uint32_t a = 0;
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int64_t r = r0 + 16 * p + tr;
    load8(static_cast<const T*>(w.ptr) + r * w.ld + c0 + tc, r < w.rows ? n : 0, f[p]);
  }
#pragma unroll
  for (int p = 0; p < 8; ++p)
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, finite_abs(f[p][i]));
  a = max16(a);
  a = max(a, uint32_t(__shfl_xor(int(a), 16)));
  a = max(a, uint32_t(__shfl_xor(int(a), 32)));
  if ((tid & 63) == 0) top[tid >> 6] = a;
  __syncthreads();
  a = max(max(top[0], top[1]), max(top[2], top[3]));
  const uint32_t byte = scale_byte<F>(a);
  const float inv = inverse_of(byte);
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int64_t r = r0 + 16 * p + tr;
    const u32x2_t q = pack8<F>(f[p], inv);
    if (out.data && r < w.rows) gstore<u32x2_t, 8>(out.data + r * out.ld + c0 + tc, q);
    if (out_t.data) {
      uint32_t* t = reinterpret_cast<uint32_t*>(tile + (16 * p + tr) * kTilePitch + tc);
      t[0] = q[0];
      t[1] = q[1];
    }
  }
  // Scales a byte at a time (the other bytes of a word are other tiles'); the
  // last tile of a row of tiles clears the bytes past it.
  auto scales = [&](const BlocksRef& o, int64_t row, int64_t block) {
    uint8_t* at = reinterpret_cast<uint8_t*>(o.scales + block / 4 * o.scale_ld + row);
    gstore<uint8_t, 1>(at + block % 4, uint8_t(byte));
    if ((block + 1) * kBlockCols >= o.cols)
      for (int64_t k = block % 4 + 1; k < 4; ++k) gstore<uint8_t, 1>(at + k, uint8_t(0));
  };
  if (tid < kBlockCols) {
    if (out.data && r0 + tid < w.rows) scales(out, r0 + tid, bj);
    if (out_t.data && c0 + tid < w.cols) scales(out_t, c0 + tid, bi);
  }
  if (!out_t.data) return;
  __syncthreads();
  // Row c of the transpose: 16 bytes of 16 rows at a time.
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int c = 32 * p + (tid >> 3), k = 16 * (tid & 7);
    union {
      uint8_t b[16];
      u32x4_t v;
    } u;
#pragma unroll
    for (int i = 0; i < 16; ++i) u.b[i] = tile[(k + i) * kTilePitch + c];
    if (c0 + c < w.cols) gstore<u32x4_t, 16>(out_t.data + (c0 + c) * out_t.ld + r0 + k, u.v);
  }
}

// s = 1 / (1 + exp(-g)) and 1 - s, from e = exp(-|g|) <= 1: 1 / (1 + e) and
// e / (1 + e).  Neither overflows, cancels or loses a tiny s (a reciprocal of
// 1 + exp(-g) past 2^126 would be flushed to zero); exp to 1 ulp, the
// reciprocal of 1 + e in [1, 2] by the hardware's (1 ulp).
__device__ __forceinline__ void logistic(float g, float& s, float& rest) {
  const float e = expf(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.f + e), q = e * r;
  s = g >= 0.f ? r : q;
  rest = g >= 0.f ? q : r;
}

template <typename T, Fp8 FK, Fp8 FH>
__global__ __launch_bounds__(kThreads) void k_gated_forward(DenseRef gate, DenseRef up, DenseRef h, BlocksRef h8,
                                                            BlocksRef gate8, BlocksRef up8) {
  const Strip s(gate.cols);
  if (s.row >= gate.rows) return;
  const int n = left(gate.cols, s.col);
  float g[8], u[8], y[8];
  load8(static_cast<const T*>(gate.ptr) + s.row * gate.ld + s.col, n, g);
  load8(static_cast<const T*>(up.ptr) + s.row * up.ld + s.col, n, u);
  if (gate8.data) {
    store_blocks<FK>(gate8, s, g);
    store_blocks<FK>(up8, s, u);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float l, rest;
    logistic(g[i], l, rest);
    y[i] = g[i] * l * u[i];
  }
  if (h.ptr) store8(static_cast<T*>(h.ptr) + s.row * h.ld + s.col, n, y);
  if (h8.data) store_blocks<FH>(h8, s, y);
}

template <typename T, Fp8 FK, Fp8 FD>
__global__ __launch_bounds__(kThreads) void k_gated_backward(DenseRef dh, BlocksRef gate, BlocksRef up,
                                                             DenseRef dgate, DenseRef dup, BlocksRef dgate8,
                                                             BlocksRef dup8) {
  const Strip s(dh.cols);
  if (s.row >= dh.rows) return;
  const int n = left(dh.cols, s.col);
  float d[8], g[8], u[8], dg[8], du[8];
  load8(static_cast<const T*>(dh.ptr) + s.row * dh.ld + s.col, n, d);
  load_blocks<FK>(gate, s, g);
  load_blocks<FK>(up, s, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float l, rest;
    logistic(g[i], l, rest);
    du[i] = d[i] * (g[i] * l);
    dg[i] = d[i] * u[i] * (l * (1.f + g[i] * rest));
  }
  if (dgate.ptr) {
    store8(static_cast<T*>(dgate.ptr) + s.row * dgate.ld + s.col, n, dg);
    store8(static_cast<T*>(dup.ptr) + s.row * dup.ld + s.col, n, du);
  }
  if (dgate8.data) {
    store_blocks<FD>(dgate8, s, dg);
    store_blocks<FD>(dup8, s, du);
  }
}

// f(T{}, integral_constant<Fp8>) for the element type and format at hand.
template <typename F>
hipError_t with_type(DType t, F&& f) {
  return t == DType::F32 ? f(float{}) : f(bf16{});
}
template <typename F>
hipError_t with_format(Fp8 v, F&& f) {
  return v == Fp8::E4M3 ? f(std::integral_constant<Fp8, Fp8::E4M3>{}) : f(std::integral_constant<Fp8, Fp8::E5M2>{});
}

}  // namespace

hipError_t launch_quantize(DType in_t, Fp8 fmt, const DenseRef& x, const BlocksRef& out, hipStream_t s) {
  return with_type(in_t, [&](auto t) {
    return with_format(fmt, [&](auto f) {
      return launch(k_quantize<decltype(t), decltype(f)::value>, strip_blocks(x.rows, x.cols), kThreads, s, x, out);
    });
  });
}

hipError_t launch_quantize_weight(DType in_t, Fp8 fmt, const DenseRef& w, const BlocksRef& out,
                                  const BlocksRef& out_t, hipStream_t s) {
  const int64_t tiles =
      ((w.rows + kBlockCols - 1) / kBlockCols) * ((w.cols + kBlockCols - 1) / kBlockCols);
  return with_type(in_t, [&](auto t) {
    return with_format(fmt, [&](auto f) {
      return launch(k_quantize_weight<decltype(t), decltype(f)::value>, unsigned(tiles), kThreads, s, w, out, out_t);
    });
  });
}

hipError_t launch_restore(DType out_t, Fp8 fmt, const BlocksRef& x, const DenseRef& out, hipStream_t s) {
  return with_type(out_t, [&](auto t) {
    return with_format(fmt, [&](auto f) {
      return launch(k_restore<decltype(t), decltype(f)::value>, strip_blocks(x.rows, x.cols), kThreads, s, x, out);
    });
  });
}

hipError_t launch_gated_forward(DType t, const DenseRef& gate, const DenseRef& up, const DenseRef& h,
                                const BlocksRef& h8, Fp8 h_fmt, const BlocksRef& gate8, const BlocksRef& up8,
                                Fp8 kept_fmt, hipStream_t s) {
  return with_type(t, [&](auto e) {
    return with_format(kept_fmt, [&](auto fk) {
      return with_format(h_fmt, [&](auto fh) {
        return launch(k_gated_forward<decltype(e), decltype(fk)::value, decltype(fh)::value>,
                      strip_blocks(gate.rows, gate.cols), kThreads, s, gate, up, h, h8, gate8, up8);
      });
    });
  });
}

hipError_t launch_gated_backward(DType t, const DenseRef& dh, const BlocksRef& gate, const BlocksRef& up,
                                 Fp8 kept_fmt, const DenseRef& dgate, const DenseRef& dup,
                                 const BlocksRef& dgate8, const BlocksRef& dup8, Fp8 d_fmt, hipStream_t s) {
  return with_type(t, [&](auto e) {
    return with_format(kept_fmt, [&](auto fk) {
      return with_format(d_fmt, [&](auto fd) {
        return launch(k_gated_backward<decltype(e), decltype(fk)::value, decltype(fd)::value>,
                      strip_blocks(dh.rows, dh.cols), kThreads, s, dh, gate, up, dgate, dup, dgate8, dup8);
      });
    });
  });
}

}  // namespace muonbp
