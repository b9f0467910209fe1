// Launchers of the 8-bit linear-layer kernels (gfx950).  Each returns the
// launch status; every operand has been checked by the C entry points.
#pragma once
#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "kernels.h"
#include "linear_plan.h"

namespace muonbp {

enum class Fp8 { E4M3 = 0, E5M2 = 1 };

// Device views (see muonbp_dense and muonbp_blocks).
struct DenseRef {
  void* ptr;
  int64_t rows, cols, ld;
};
struct BlocksRef {
  uint8_t* data;
  uint32_t* scales;
  int64_t rows, cols, ld, scale_ld;
};

// out <- x, one scale a block of 128 columns.
hipError_t launch_quantize(DType in_t, Fp8 fmt, const DenseRef& x, const BlocksRef& out, hipStream_t s);
// out and out_t (data NULL: not wanted) <- w and its transpose, one scale a
// 128 x 128 tile.
hipError_t launch_quantize_weight(DType in_t, Fp8 fmt, const DenseRef& w, const BlocksRef& out,
                                  const BlocksRef& out_t, hipStream_t s);
// out <- the values of x.
hipError_t launch_restore(DType out_t, Fp8 fmt, const BlocksRef& x, const DenseRef& out, hipStream_t s);
// h / h8 <- silu(gate) up; gate8, up8 <- gate, up (ptr / data NULL: not wanted).
hipError_t launch_gated_forward(DType t, const DenseRef& gate, const DenseRef& up, const DenseRef& h,
                                const BlocksRef& h8, Fp8 h_fmt, const BlocksRef& gate8, const BlocksRef& up8,
                                Fp8 kept_fmt, hipStream_t s);
hipError_t launch_gated_backward(DType t, const DenseRef& dh, const BlocksRef& gate, const BlocksRef& up,
                                 Fp8 kept_fmt, const DenseRef& dgate, const DenseRef& dup,
                                 const BlocksRef& dgate8, const BlocksRef& dup8, Fp8 d_fmt, hipStream_t s);

// Sums of tiles whose long axis is split over workgroups: sums holds
// sum_floats fp32 values, counts kSplitCounts zeroed counters (left zeroed).
struct SplitSpace {
  float* sums;
  int64_t sum_floats;
  int* counts;
};

// c <- [c +] a b^T, a in fmt, b in e4m3; fp32_sums: of bf16 results too.
hipError_t launch_product(DType out_t, Fp8 a_fmt, const BlocksRef& a, const BlocksRef& b, const DenseRef& c,
                          bool accumulate, bool fp32_sums, const SplitSpace& split, int cus, hipStream_t s);
// dw <- [dw +] x^T dy, x in fmt, dy bf16.
hipError_t launch_weight_grad(DType out_t, Fp8 x_fmt, const BlocksRef& x, const DenseRef& dy, const DenseRef& dw,
                              bool accumulate, const SplitSpace& split, int cus, hipStream_t s);

}  // namespace muonbp
