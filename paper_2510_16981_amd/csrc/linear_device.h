// Device helpers shared by the 8-bit linear-layer kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <tuple>

#include "linear.h"

namespace muonbp {

// Launches a kernel and returns the status of that launch, which
// hipGetLastError() after a <<<>>> is not: it also reports what an earlier call
// of the thread left behind.  A refused launch leaves nothing behind.
template <typename... P, typename... A>
hipError_t launch(void (*kernel)(P...), unsigned groups, unsigned threads, hipStream_t s, const A&... args) {
  std::tuple<P...> values(args...);
  const hipError_t e = std::apply(
      [&](auto&... v) {
        void* at[] = {&v...};
        return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(groups), dim3(threads), at, 0, s);
      },
      values);
  if (e != hipSuccess) (void)hipGetLastError();
  return e;
}

typedef __bf16 bf16;
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

// Accesses through the global address space (a flat access would count
// against the LDS wait counter too), at any element alignment: the hardware
// splits what is not aligned.
template <typename V, int ALIGN>
struct Loose {
  typedef V type __attribute__((aligned(ALIGN)));
};
template <typename V, int ALIGN>
__device__ __forceinline__ V gload(const void* p) {
  typedef typename Loose<V, ALIGN>::type T;
  return *(const __attribute__((address_space(1))) T*)(reinterpret_cast<uintptr_t>(p));
}
template <typename V, int ALIGN>
__device__ __forceinline__ void gstore(void* p, V v) {
  typedef typename Loose<V, ALIGN>::type T;
  *(__attribute__((address_space(1))) T*)(reinterpret_cast<uintptr_t>(p)) = v;
}

__device__ __forceinline__ float bits_f(uint32_t b) { return __builtin_bit_cast(float, b); }
__device__ __forceinline__ uint32_t f_bits(float f) { return __builtin_bit_cast(uint32_t, f); }

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(bf16 x) { return float(x); }

// f <- n <= 8 consecutive elements at p, zeros past them.  (One by one, all are
// loaded before the first is used: past n, the first element again.)
__device__ __forceinline__ void load8(const bf16* p, int n, float f[8]) {
  if (n >= 8) {
    const u32x4_t v = gload<u32x4_t, 2>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bits_f(v[i] << 16);
      f[2 * i + 1] = bits_f(v[i] & 0xffff0000u);
    }
  } else if (n > 0) {
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = gload<uint16_t, 2>(p + (i < n ? i : 0));
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? bits_f(h[i] << 16) : 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
  }
}
__device__ __forceinline__ void load8(const float* p, int n, float f[8]) {
  if (n >= 8) {
    const f32x4_t a = gload<f32x4_t, 4>(p), b = gload<f32x4_t, 4>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = a[i];
      f[i + 4] = b[i];
    }
  } else if (n > 0) {
    float h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = gload<float, 4>(p + (i < n ? i : 0));
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < n ? h[i] : 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
  }
}

// n <= 8 values rounded to the element type, at p.
__device__ __forceinline__ void store8(bf16* p, int n, const float f[8]) {
  union {
    bf16 h[8];
    uint16_t b[8];
    u32x4_t v;
  } u;
#pragma unroll
  for (int i = 0; i < 8; ++i) u.h[i] = bf16(f[i]);
  if (n >= 8) {
    gstore<u32x4_t, 2>(p, u.v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) gstore<uint16_t, 2>(p + i, u.b[i]);
  }
}
__device__ __forceinline__ void store8(float* p, int n, const float f[8]) {
  if (n >= 8) {
    gstore<f32x4_t, 4>(p, f32x4_t{f[0], f[1], f[2], f[3]});
    gstore<f32x4_t, 4>(p + 4, f32x4_t{f[4], f[5], f[6], f[7]});
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) gstore<float, 4>(p + i, f[i]);
  }
}

// |x| as bits, or 0 for NaN and infinities (they do not count in a block's max).
__device__ __forceinline__ uint32_t finite_abs(float x) {
  const uint32_t a = f_bits(x) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}

// The largest of v over each 16 lanes, in all of them (rotations inside a
// 16-lane row: no LDS).
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x128, 0xf, 0xf, false)));
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x124, 0xf, 0xf, false)));
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x122, 0xf, 0xf, false)));
  return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x121, 0xf, 0xf, false)));
}

// The biased exponent 127 + e of the scale of a block whose largest finite
// value has the bits a: with a = m 2^k, 1 <= m < 2, the type's largest value
// is 1.75 2^top, so e = k - top, and one more where m > 1.75; at least -110,
// which keeps every value of the types (down to 2^-16) a normal fp32 and bf16
// number.
template <Fp8 F>
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
  constexpr int top = F == Fp8::E4M3 ? 8 : 15;
  const int e = int(a >> 23) - top + ((a & 0x7fffffu) > 0x600000u);
  return uint32_t(max(e, 127 - 110));
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return bits_f(byte << 23); }
// 1 / 2^(byte - 127), for bytes from 17 to 248.
__device__ __forceinline__ float inverse_of(uint32_t byte) { return bits_f((254u - byte) << 23); }

// Eight values times inv (a power of two: exact), rounded to 8 bits.
template <Fp8 F>
__device__ __forceinline__ u32x2_t pack8(const float f[8], float inv) {
  u32x2_t r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = 0;
    const float* g = f + 4 * i;
    if constexpr (F == Fp8::E4M3) {
      w = __builtin_amdgcn_cvt_pk_fp8_f32(g[0] * inv, g[1] * inv, w, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(g[2] * inv, g[3] * inv, w, true);
    } else {
      w = __builtin_amdgcn_cvt_pk_bf8_f32(g[0] * inv, g[1] * inv, w, false);
      w = __builtin_amdgcn_cvt_pk_bf8_f32(g[2] * inv, g[3] * inv, w, true);
    }
    r[i] = uint32_t(w);
  }
  return r;
}

// The values of eight bytes times their scale, exact.
template <Fp8 F>
__device__ __forceinline__ void unpack8(u32x2_t q, float scale, float f[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    f32x2_t a, b;
    if constexpr (F == Fp8::E4M3) {
      a = __builtin_amdgcn_cvt_pk_f32_fp8(int(q[i]), false);
      b = __builtin_amdgcn_cvt_pk_f32_fp8(int(q[i]), true);
    } else {
      a = __builtin_amdgcn_cvt_pk_f32_bf8(int(q[i]), false);
      b = __builtin_amdgcn_cvt_pk_f32_bf8(int(q[i]), true);
    }
    f[4 * i] = a[0] * scale;
    f[4 * i + 1] = a[1] * scale;
    f[4 * i + 2] = b[0] * scale;
    f[4 * i + 3] = b[1] * scale;
  }
}

// Four bytes times their scale as bf16, exact.
template <Fp8 F>
__device__ __forceinline__ u32x2_t widen4(uint32_t q, float scale) {
  bf16x2_t a, b;
  if constexpr (F == Fp8::E4M3) {
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q, scale, true);
  } else {
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(q, scale, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(q, scale, true);
  }
  return u32x2_t{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}

}  // namespace muonbp
