// Matrix products of 8-bit linear layers: C = A B^T of two 8-bit matrices, and
// the weight gradient dW = X^T dY of an 8-bit and a 16-bit one.
#include <type_traits>
#include <utility>

#include "linear_device.h"

namespace muonbp {

namespace {

// ---------------------------------------------------------------- shared pieces

typedef __attribute__((address_space(3))) void lds_void_t;

constexpr int kBufferWord3 = 0x00020000;  // raw buffer, 32-bit data format

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, int(bytes), kBufferWord3);
}

// s_waitcnt immediate: at most n vector-memory operations of this wave are
// outstanding.
constexpr int vmcnt_imm(int n) { return (n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14); }

// 16-byte LDS read issued without a compiler-inserted wait (which would wait
// for every copy into LDS still in flight); lgkm_wait and hold complete it.
template <int OFF>
__device__ __forceinline__ u32x4_t lds_read16(uint32_t addr) {
  u32x4_t v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
  return v;
}
template <int OFF>
__device__ __forceinline__ uint32_t lds_read4(uint32_t addr) {
  uint32_t v;
  asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
  return v;
}
// f(integral_constant 0), ..., f(integral_constant N - 1).
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}
__device__ __forceinline__ void lgkm_wait() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// No use of v may move above this point.
template <typename V>
__device__ __forceinline__ void hold(V& v) {
  asm volatile("" : "+v"(v));
}

// Workgroup barrier without the fence of __syncthreads(), which would wait
// for the copies that the pipeline keeps in flight.
__device__ __forceinline__ void barrier_no_fence() { asm volatile("s_barrier" ::: "memory"); }

// The wave's issue priority, 1 where `high`: in one block of assembly, because a
// branch in a K loop would let the compiler move MFMAs across it.
__device__ __forceinline__ void set_priority(int high) {
  asm volatile(
      "s_cmp_lg_u32 %0, 0\n\ts_cbranch_scc1 1f\n\ts_setprio 0\n\ts_branch 2f\n1:\n\ts_setprio 1\n2:" ::"s"(high)
      : "scc");
}

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const lds_void_t*)p));
}

// Which tile and part workgroup b runs.  Consecutive workgroups go to the 8 XCDs
// in turn; each XCD gets a contiguous run of tiles, taken `kGroupTall` tiles
// high, so that the tiles resident on one XCD share rows and columns in its L2.
struct TileAt {
  int ti, tj, part, parts;
  int split;  // its place among the tiles in parts
};
constexpr int kXcds = 8, kGroupTall = 8;
__device__ __forceinline__ int spread(int b, int total) {
  const int x = b % kXcds, q = total / kXcds, r = total % kXcds;
  return x * q + min(x, r) + b / kXcds;
}
__device__ __forceinline__ TileAt tile_at(int b, int total, int tall, int wide, const Shares& s) {
  TileAt t;
  int pos;
  if (b < s.whole) {
    pos = spread(b, s.whole);
    t.part = t.split = 0;
    t.parts = 1;
  } else {
    const int at = spread(b - s.whole, total - s.whole);
    t.split = at / s.parts;
    t.part = at - t.split * s.parts;
    t.parts = s.parts;
    pos = s.whole + t.split;
  }
  const int per = kGroupTall * wide, g = pos / per, in = pos - g * per;
  const int h = min(kGroupTall, tall - g * kGroupTall);
  t.ti = g * kGroupTall + in % h;
  t.tj = in / h;
  return t;
}

// Stores a wave's C block (TM x TN blocks of 32 x 32 whose first MFMA operand
// was the n side: lane l has row l % 32 and columns 8 q + 4 (l / 32) .. + 3 in
// acc[i][j][4 q .. 4 q + 3]) through `st`, 32 x (32 TN + 4) floats of LDS of the
// wave's own, so that rows are written in whole 8-element chunks.
template <typename T, int TM, int TN>
__device__ __forceinline__ void store_tile(f32x16_t (&acc)[TM][TN], float* st, const DenseRef& c, int64_t row0,
                                           int64_t col0, bool accumulate) {
  constexpr int P = 32 * TN + 4;
  constexpr int CH = 4 * TN;  // 8-element chunks of a row
  const int lane = threadIdx.x & 63;
  // Inside the matrix: stores without tests between them.
  const bool whole = !accumulate && row0 + 32 * TM <= c.rows && col0 + 32 * TN <= c.cols;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4_t*>(st + (lane & 31) * P + 32 * j + 8 * q + 4 * (lane >> 5)) =
            f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    if (whole) {
#pragma unroll
      for (int p = 0; p < 32 * CH / 64; ++p) {
        const int at = p * 64 + lane, r = at / CH, k = 8 * (at % CH);
        float f[8];
        *reinterpret_cast<f32x4_t*>(f) = *reinterpret_cast<const f32x4_t*>(st + r * P + k);
        *reinterpret_cast<f32x4_t*>(f + 4) = *reinterpret_cast<const f32x4_t*>(st + r * P + k + 4);
        store8(static_cast<T*>(c.ptr) + (row0 + 32 * i + r) * c.ld + col0 + k, 8, f);
      }
      continue;
    }
#pragma unroll
    for (int p = 0; p < 32 * CH / 64; ++p) {
      const int at = p * 64 + lane, r = at / CH, k = 8 * (at % CH);
      const int64_t row = row0 + 32 * i + r, col = col0 + k;
      const int64_t left = c.cols - col;
      const int n = row < c.rows ? int(left < 0 ? 0 : left > 8 ? 8 : left) : 0;
      if (n > 0) {
        float f[8];
        *reinterpret_cast<f32x4_t*>(f) = *reinterpret_cast<const f32x4_t*>(st + r * P + k);
        *reinterpret_cast<f32x4_t*>(f + 4) = *reinterpret_cast<const f32x4_t*>(st + r * P + k + 4);
        T* out = static_cast<T*>(c.ptr) + row * c.ld + col;
        if (accumulate) {
          float old[8];
          load8(out, n, old);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] += old[e];
        }
        store8(out, n, f);
      }
    }
  }
}

// The parts of a tile whose long axis is split: every workgroup stores its
// sums, the last to arrive adds them in the order of the parts (the result does
// not depend on which is last) and goes on; the others end, and none waits for
// another (false: this workgroup is done).  Sums are stored and loaded 16 bytes a
// lane with the policy of a relaxed atomic of device scope (sc1).  Why the last one reads what was stored:
//  - A store of that scope is complete (vmcnt 0) once it is at the device's point
//    of coherence, past the XCD's L2; each wave waits for its own, then the
//    workgroup for its waves, and only then is the part counted.
//  - The counts are read-modify-writes of device scope, one after another: who
//    gets parts - 1 comes after every other part's count, and its loads are
//    issued after that (the barrier).
//  - A load of that scope takes no line of the CU's cache, and none of its XCD's
//    L2 could be stale: a line of sums is touched by one part's stores and then by
//    these loads, once in a launch (parts are multiples of 16 KB, so no line
//    is shared), and what earlier launches left was invalidated at this one's start.
constexpr int kCoherent = 16;  // sc1
template <int TM, int TN, int W>
__device__ __forceinline__ bool join_parts(f32x16_t (&acc)[TM][TN], const SplitSpace& split, int tile, int part,
                                           int parts, int wave, int lane, int* last) {
  constexpr int WAVE = TM * TN * 16 * 64;  // sums of a wave
  float* const all = split.sums + size_t(tile) * parts * (WAVE * W) + wave * WAVE;
  auto span = [&](int p) { return buffer(all + size_t(p) * (WAVE * W), 4 * WAVE); };
  const __amdgpu_buffer_rsrc_t mine = span(part);
#pragma unroll
  for (int q = 0; q < TM * TN; ++q)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const f32x16_t& a = acc[q / TN][q % TN];
      __builtin_amdgcn_raw_buffer_store_b128(
          u32x4_t{f_bits(a[4 * v]), f_bits(a[4 * v + 1]), f_bits(a[4 * v + 2]), f_bits(a[4 * v + 3])}, mine,
          ((q * 4 + v) * 64 + lane) * 16, 0, kCoherent);
    }
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  __syncthreads();
  if (threadIdx.x == 0)
    *last = __hip_atomic_fetch_add(split.counts + tile, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
  __syncthreads();
  if (!*last) return false;
  for (int p = 0; p < parts; ++p) {
    const __amdgpu_buffer_rsrc_t from = span(p);
#pragma unroll
    for (int q = 0; q < TM * TN; ++q)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        f32x16_t& a = acc[q / TN][q % TN];
        const u32x4_t x = __builtin_amdgcn_raw_buffer_load_b128(from, ((q * 4 + v) * 64 + lane) * 16, 0, kCoherent);
#pragma unroll
        for (int e = 0; e < 4; ++e) a[4 * v + e] = p == 0 ? bits_f(x[e]) : a[4 * v + e] + bits_f(x[e]);
      }
  }
  if (threadIdx.x == 0) __hip_atomic_store(split.counts + tile, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}

// ---------------------------------------------------------------- product, ring of K slices
//
// A tile of BM x BN, K in slices of 64 bytes copied straight into a ring of 4
// slots in LDS (rows of 64 bytes; 16-byte chunk c of row r at c ^ swz(r), which
// spreads the 32 rows one fragment read touches over all banks).  WM x WN waves
// hold blocks of 32 TM x 32 TN.  While the MFMAs of slice kt run, its
// successor is read into the other set of fragment registers and the slot
// that kt came from is refilled with slice kt + 4: one barrier a slice, right
// after its first MFMA.
//
// The matrix instruction multiplies 32 x 64 by 64 x 32 in 8 bits and applies a
// power-of-two scale per row and 32 columns: with the block scales fed to it,
// the scaled product costs what an unscaled one does.  The words of scales of a
// tile's rows (4 blocks: 8 slices) are copied into LDS a group ahead, and read
// into registers when their group begins.
//
// EXACT (fp32 results, and bf16 ones on demand): the fragments are widened to
// bf16, scales included, which is exact, and multiplied by 16-bit instructions at
// half the rate: products exact, sums in fp32 (5e-8 off in the 2-norm).  The 8-bit
// instruction is not that good: of each 8 consecutive products it cuts off,
// toward zero, what lies below 2^-13 of the power of two of the largest, then adds
// the eights in fp32 (measured; the same in 32x32x64 and 16x16x128).  A result is off
// by at most the sum of min(|p|, 2^-13 |largest|) over the products p below 2^-6
// of the largest of their eight; in the 2-norm, at any K, 1.1e-5 to 1.6e-5 for normal
// values and 4e-5 to 1e-4 with outlier channels, where rounding to bf16 costs 1.7e-3.
//
// Tiles (chosen in linear_plan.h): 256 x 256 on 8 waves, two a SIMD, which take
// priority in turn (2-6% faster than equal priorities); 128 x 256 on 8 waves where
// that fills the chip and 256 x 256 does not; 128 x 128 and 64 x 128 on 4 waves,
// several workgroups a CU.  Large products are bound by the matrix cores (busy 64%
// of the clocks) at the clock that their power leaves (1.69 GHz), which differs by the
// card, and by the tiles' stores, 6 us of 60: 8192 x 4096 x 14336 414 to 443 us on four
// cards (2.17 to 2.32 PFLOP/s), 4096 x 8192 x 2048 62 to 67; EXACT 789 and 123.  The
// 4-wave tiles are bound by LDS: a slice of 128 x 128 is 48 KB through it, 384 clocks
// for 256 of MFMA.
__device__ __forceinline__ int swz(int row) { return ((row >> 1) & 3) ^ ((row >> 3) & 1); }

template <typename T, Fp8 F, bool EXACT, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_product(BlocksRef a, BlocksRef b, DenseRef c, bool accumulate,
                                                          Shares shares, SplitSpace split) {
  constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN, W = WM * WN, NS = 4, ROW = 64;
  constexpr int STAGE = (BM + BN) * ROW;
  constexpr int LP = (BM + BN) / 16 / W;  // 1 KB copies (16 rows) of a slice per wave
  constexpr int RS = (BM + BN) / 64;      // copies of 64 scale words
  constexpr int LS = (RS + W - 1) / W;
  static_assert(BM % (16 * W) == 0 && BN % (16 * W) == 0, "a wave's copy is all A or all B");
  constexpr int EPI = W * 32 * (32 * TN + 4) * 4;
  constexpr int RING = NS * STAGE > EPI ? NS * STAGE : EPI;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[RING + 2 * (BM + BN) * 4];
  __shared__ int last;
  uint32_t* const words = reinterpret_cast<uint32_t*>(lds + RING);

  const int tall = int((c.rows + BM - 1) / BM), wide = int((c.cols + BN - 1) / BN);
  const TileAt t = tile_at(blockIdx.x, gridDim.x, tall, wide, shares);
  const int64_t m0 = int64_t(t.ti) * BM, n0 = int64_t(t.tj) * BN;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int ma = int(min(int64_t(BM), a.rows - m0)), nb = int(min(int64_t(BN), b.rows - n0));
  const uint32_t kbytes = uint32_t((a.cols + kBlockCols - 1) / kBlockCols * kBlockCols);
  const uint32_t abytes = uint32_t(ma - 1) * uint32_t(a.ld) + kbytes;
  const uint32_t bbytes = uint32_t(nb - 1) * uint32_t(b.ld) + kbytes;
  const __amdgpu_buffer_rsrc_t ar = buffer(a.data + m0 * a.ld, abytes), br = buffer(b.data + n0 * b.ld, bbytes);

  // Slices of this part: whole blocks of 128.
  const int nblk = int(kbytes / kBlockCols);
  const int kb = 2 * (t.part * nblk / t.parts), ke = 2 * ((t.part + 1) * nblk / t.parts);

  uint32_t voff[LP];
#pragma unroll
  for (int j = 0; j < LP; ++j) {
    const int row = 16 * (wave + W * j) + (lane >> 2), col = 16 * ((lane & 3) ^ swz(row));
    if (W * j < BM / 16)
      voff[j] = row < ma ? uint32_t(row) * uint32_t(a.ld) + col : abytes;  // past the end: zeros
    else
      voff[j] = row - BM < nb ? uint32_t(row - BM) * uint32_t(b.ld) + col : bbytes;
  }
  // Copy j of slice kt into its slot.  Past the part's end the last slice is
  // copied again (never read), so that every wait is a constant count.
  auto copy = [&](int kt, int j) {
    lds_void_t* dst = (lds_void_t*)(lds + (kt & (NS - 1)) * STAGE + (wave + W * j) * 1024);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(W * j < BM / 16 ? ar : br, dst, 16, int(voff[j]),
                                             min(kt, ke - 1) * ROW, 0, 0);
  };
  const int groups = int((a.cols + kGroupCols - 1) / kGroupCols);
  auto copy_scales = [&](int g) {
#pragma unroll
    for (int j = 0; j < LS; ++j) {
      const int u = (wave + W * j) % RS;
      const bool of_a = u < BM / 64;
      const BlocksRef& m = of_a ? a : b;
      const int64_t r0 = of_a ? m0 : n0;
      const __amdgpu_buffer_rsrc_t r =
          buffer(m.scales + int64_t(min(g, groups - 1)) * m.scale_ld + r0, 4u * uint32_t(of_a ? ma : nb));
      lds_void_t* dst = (lds_void_t*)(words + (g & 1) * (BM + BN) + 64 * u);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 4, 4 * (64 * (of_a ? u : u - BM / 64) + lane), 0, 0, 0);
    }
  };

  f32x16_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x16_t{};

  constexpr int NF = TM + TN, NM = TM * TN, NR = 2 * NF;
  // A fragment is 32 rows, which leaves the swizzle as it is: lane addresses
  // of the first fragment of A and of B, half h, and constant offsets.
  uint32_t fa[2][2], wa[2];
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const int r = (side ? BM + wn * 32 * TN : wm * 32 * TM) + (lane & 31);
    wa[side] = lds_addr(words) + 4 * r;
#pragma unroll
    for (int h = 0; h < 2; ++h) fa[side][h] = lds_addr(lds) + r * ROW + (((2 * h + (lane >> 5)) ^ swz(r)) << 4);
  }
  u32x4_t fr[2][NF][2];
  uint32_t sw[NF];
  auto read_words = [&](int g) {
    const uint32_t base = (g & 1) * (4 * (BM + BN));
    each<NF>([&](auto o) {
      constexpr int f = o;
      sw[f] = lds_read4<128 * (f < TM ? f : f - TM)>(wa[f < TM ? 0 : 1] + base);
    });
  };
  auto read_frag = [&](auto o, u32x4_t (&to)[NF][2], uint32_t base) {
    constexpr int f = o / 2, h = o % 2, side = f < TM ? 0 : 1;
    to[f][h] = lds_read16<32 * ROW * (f < TM ? f : f - TM)>(fa[side][h] + base);
  };

#pragma unroll
  for (int s = 0; s < 2; ++s) copy_scales((kb >> 3) + s);
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int j = 0; j < LP; ++j) copy(kb + s, j);
  __builtin_amdgcn_s_waitcnt(vmcnt_imm((NS - 1) * LP));
  barrier_no_fence();
  each<NR>([&](auto o) { read_frag(o, fr[0], (kb & (NS - 1)) * STAGE); });
  read_words(kb >> 3);
  lgkm_wait();
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    hold(fr[0][f][0]);
    hold(fr[0][f][1]);
    hold(sw[f]);
  }

  auto slice = [&](auto set, int kt) {
    constexpr int P = decltype(set)::value;
    if constexpr (W == 8) set_priority((P + (wave >> 2)) & 1);
    const int shift = 8 * (kt >> 1 & 3);
    uint32_t sb[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f) sb[f] = sw[f] >> shift;
    u32x4_t wide_[EXACT ? NF : 1][4];
    if constexpr (EXACT) {
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        const float s = scale_of(sb[f] & 255u);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            u32x2_t x, y;
            if (f < TM) {
              x = widen4<F>(fr[P][f][h][2 * e], s);
              y = widen4<F>(fr[P][f][h][2 * e + 1], s);
            } else {
              x = widen4<Fp8::E4M3>(fr[P][f][h][2 * e], s);
              y = widen4<Fp8::E4M3>(fr[P][f][h][2 * e + 1], s);
            }
            wide_[f][2 * h + e] = u32x4_t{x[0], x[1], y[0], y[1]};
          }
      }
    }
    auto mfma = [&](int q) {
      const int i = q / TN, j = q % TN;
      if constexpr (EXACT) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, wide_[TM + j][e]),
                                                              __builtin_bit_cast(bf16x8_t, wide_[i][e]), acc[i][j], 0,
                                                              0, 0);
      } else {
        const u32x4_t *y = fr[P][TM + j], *x = fr[P][i];
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
            i32x8_t{int(y[0][0]), int(y[0][1]), int(y[0][2]), int(y[0][3]), int(y[1][0]), int(y[1][1]), int(y[1][2]),
                    int(y[1][3])},
            i32x8_t{int(x[0][0]), int(x[0][1]), int(x[0][2]), int(x[0][3]), int(x[1][0]), int(x[1][1]), int(x[1][2]),
                    int(x[1][3])},
            acc[i][j], 0, F == Fp8::E4M3 ? 0 : 1, 0, int(sb[TM + j]), 0, int(sb[i]));
      }
    };
    mfma(0);
    __builtin_amdgcn_sched_barrier(0);
    // Slice kt + 1 has landed for this wave, after the barrier for every wave;
    // and every wave holds slice kt in registers, so its slot takes kt + 4.
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((NS - 2) * LP));
    barrier_no_fence();
    constexpr int R = NM - 1, RR = R > 2 ? R - 1 : R;  // the last MFMA hides the last reads
    const uint32_t base = ((kt + 1) & (NS - 1)) * STAGE;
    each<R>([&](auto at) {
      mfma(at + 1);
      each<NR>([&](auto o) {
        if constexpr (o >= at * NR / RR && o < (at + 1) * NR / RR) read_frag(o, fr[P ^ 1], base);
      });
      each<LP>([&](auto o) {
        if constexpr (o >= at * LP / R && o < (at + 1) * LP / R) copy(kt + NS, o);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    lgkm_wait();
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      hold(fr[P ^ 1][f][0]);
      hold(fr[P ^ 1][f][1]);
    }
  };
  // A group of 8 slices shares its words of scales.  The inner loop has no
  // other branch, so that its MFMAs stay between its reads and copies.
  for (int kt = kb; kt < ke;) {
    const int g = kt >> 3, end = min(8 * g + 8, ke);
    for (; kt < end; kt += 2) {  // an even count: whole blocks
      slice(std::integral_constant<int, 0>{}, kt);
      slice(std::integral_constant<int, 1>{}, kt + 1);
    }
    // The words of group g + 1 were copied a whole group ago (or before the
    // first slice); every wave has read those of group g, so their place takes
    // the words of group g + 2.
    copy_scales(g + 2);
    read_words(g + 1);
    lgkm_wait();
#pragma unroll
    for (int f = 0; f < NF; ++f) hold(sw[f]);
  }
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));  // copies past the end land before the ring is reused
  if (t.parts > 1 && !join_parts<TM, TN, W>(acc, split, t.split, t.part, t.parts, wave, lane, &last)) return;
  __syncthreads();
  store_tile<T, TM, TN>(acc, reinterpret_cast<float*>(lds) + wave * 32 * (32 * TN + 4), c,
                        m0 + wm * 32 * TM, n0 + wn * 32 * TN, accumulate);
}

// ---------------------------------------------------------------- product, few rows
//
// C = A B^T for up to 16 rows of A (single tokens): bound by reading B once.
// One workgroup holds 16 rows of B; its waves take the groups of 512 columns in
// turn, straight from memory into registers (16 bytes a lane, 64 contiguous
// bytes of a row an instruction) with the next group on its way, and their sums
// meet in LDS.  Measured in a loop over the same operands (59 MB, which the last
// cache holds), one row: 14336 x 4096 12.5 us, 4096 x 14336 11.4 us; EXACT 13.0 and 11.8.
// 2 and 8 waves took 14.7 and 16.8 where 4 took 14.5, 12.5 and 11.1 where 4 took 11.2,
// and columns split over 2 or 4 workgroups 13.9 and 23 us, 13.1 and 14.1 us.  Few
// columns of C leave CUs without work: 1024 x 4096 4.5 us, 1024 x 14336 9.9.
constexpr int kFewWaves = 4;

template <typename T, Fp8 F, bool EXACT>
__global__ __launch_bounds__(64 * kFewWaves) void k_product_few(BlocksRef a, BlocksRef b, DenseRef c,
                                                                bool accumulate) {
  __shared__ __attribute__((aligned(16))) f32x4_t sums[kFewWaves][64];
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = int64_t(blockIdx.x) * 16;
  const int nr = int(min(int64_t(16), b.rows - n0)), mr = int(a.rows);
  const uint32_t kbytes = uint32_t((a.cols + kBlockCols - 1) / kBlockCols * kBlockCols);
  const int blocks = int(kbytes / kBlockCols), groups = (blocks + 3) / 4;
  const uint32_t bbytes = uint32_t(nr - 1) * uint32_t(b.ld) + kbytes;
  const uint32_t abytes = uint32_t(mr - 1) * uint32_t(a.ld) + kbytes;
  const __amdgpu_buffer_rsrc_t br = buffer(b.data + n0 * b.ld, bbytes), ar = buffer(a.data, abytes);
  const int row = lane & 15, col = 16 * (lane >> 4);
  const uint32_t boff = row < nr ? uint32_t(row) * uint32_t(b.ld) + col : bbytes;  // past the end: zeros
  const uint32_t aoff = row < mr ? uint32_t(row) * uint32_t(a.ld) + col : abytes;

  struct Group {
    u32x4_t y[4][2], x[4][2];
    uint32_t sy, sx;
  };
  auto load = [&](Group& r, int g) {
    const __amdgpu_buffer_rsrc_t sb = buffer(b.scales + int64_t(g) * b.scale_ld + n0, 4u * uint32_t(nr));
    const __amdgpu_buffer_rsrc_t sa = buffer(a.scales + int64_t(g) * a.scale_ld, 4u * uint32_t(mr));
    r.sy = __builtin_amdgcn_raw_buffer_load_b32(sb, 4 * row, 0, 0);
    r.sx = __builtin_amdgcn_raw_buffer_load_b32(sa, 4 * row, 0, 0);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = min(4 * g + k, blocks - 1) * kBlockCols;  // past the last block: it again, not used
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        r.y[k][h] = __builtin_amdgcn_raw_buffer_load_b128(br, int(boff), at + 64 * h, 0);
        r.x[k][h] = __builtin_amdgcn_raw_buffer_load_b128(ar, int(aoff), at + 64 * h, 0);
      }
    }
  };
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const Group& r, int g) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (4 * g + k >= blocks) break;
      const uint32_t sy = r.sy >> (8 * k) & 255u, sx = r.sx >> (8 * k) & 255u;
      const u32x4_t *y = r.y[k], *x = r.x[k];
      if constexpr (EXACT) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const u32x2_t p = widen4<Fp8::E4M3>(y[h][2 * e], scale_of(sy)),
                          q = widen4<Fp8::E4M3>(y[h][2 * e + 1], scale_of(sy));
            const u32x2_t u = widen4<F>(x[h][2 * e], scale_of(sx)), w = widen4<F>(x[h][2 * e + 1], scale_of(sx));
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8_t, u32x4_t{p[0], p[1], q[0], q[1]}),
                __builtin_bit_cast(bf16x8_t, u32x4_t{u[0], u[1], w[0], w[1]}), acc, 0, 0, 0);
          }
      } else {
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            i32x8_t{int(y[0][0]), int(y[0][1]), int(y[0][2]), int(y[0][3]), int(y[1][0]), int(y[1][1]), int(y[1][2]),
                    int(y[1][3])},
            i32x8_t{int(x[0][0]), int(x[0][1]), int(x[0][2]), int(x[0][3]), int(x[1][0]), int(x[1][1]), int(x[1][2]),
                    int(x[1][3])},
            acc, 0, F == Fp8::E4M3 ? 0 : 1, 0, int(sy), 0, int(sx));
      }
    }
  };
  int g = wave;
  if (g < groups) {
    Group r[2];
    load(r[0], g);
    for (; g < groups; g += 2 * waves) {
      if (g + waves < groups) load(r[1], g + waves);
      multiply(r[0], g);
      if (g + waves >= groups) break;
      if (g + 2 * waves < groups) load(r[0], g + 2 * waves);
      multiply(r[1], g + waves);
    }
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (wave > 0) return;
  f32x4_t v = sums[0][lane];
  for (int w = 1; w < waves; ++w) v += sums[w][lane];
  const int64_t n = n0 + 4 * (lane >> 4);
  if (row >= mr) return;
  T* out = static_cast<T*>(c.ptr) + row * c.ld + n;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (n + e < c.cols) {
      float f = v[e];
      if (accumulate) f += to_f(out[e]);
      out[e] = T(f);
    }
}

// ---------------------------------------------------------------- weight gradient
//
// dW = X^T dY over slices of 32 tokens.  A slice of X (8 bits) and of dY (16
// bits) is loaded into registers two slices ahead, X is widened to bf16 with
// its block's scale (exact; a thread's 16 values are one token's, so they share
// it, which they would not along the tokens), and both are written to one of two
// slots in LDS as they lie in memory: 32 rows (tokens) of BM or BN elements,
// 16-byte chunk c of row r at c ^ 4 (r % 4).  The operands of the 16-bit matrix
// instruction, 8 consecutive tokens of one feature a lane, come from LDS
// transpose reads.  One barrier a slice.
//
// Loads are of any alignment.  Only the last tokens, where a row's last 16 bytes
// may end past the matrix, are read an element at a time; a part begins with its
// last two slices, so that the loop's loads are the same for every slice (with a
// choice between them the compiler waits for all loads in flight at each: 940
// against 1130 TFLOP/s at 8192 tokens, 14336 x 4096).
//
// 256 x 256 tiles on 8 waves, 128 x 128 on 4 for matrices of fewer tiles.  Bound by
// the matrix cores (busy 65% of the clocks) at the clock that their power leaves
// (1.59 GHz), which differs by the card: 8192 tokens, 14336 x 4096 755 to 817 us on four
// cards (1.18 to 1.27 PFLOP/s); 8192^3 839 to 889.  Unaligned rows (8191) cost nothing.
__device__ __forceinline__ int row_swz(int r) { return 4 * (r & 3); }

// Each group of 16 lanes reads a 4 x 16 block of 16-bit elements; lane i gives
// the address of elements 4 (i % 4) .. + 3 of row i / 4 and receives column i.
template <int OFF>
__device__ __forceinline__ u32x2_t lds_read8_tr(uint32_t addr) {
  u32x2_t v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
  return v;
}

template <typename T, Fp8 F, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_weight_grad(BlocksRef x, DenseRef dy, DenseRef dw, bool accumulate,
                                                              Shares shares, SplitSpace split) {
  constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN, W = WM * WN, NT = 64 * W, KT = 32;
  constexpr int XP = 2 * BM, YP = 2 * BN, STAGE = KT * (XP + YP);  // bytes
  constexpr int XC = KT * BM / 16 / NT, YC = KT * BN / 8 / NT;     // 16-byte loads per thread and slice
  static_assert(XC * 16 * NT == KT * BM && YC * 8 * NT == KT * BN && BM % 128 == 0 && BN % 128 == 0, "tile");
  constexpr int EPI = W * 32 * (32 * TN + 4) * 4;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGE > EPI ? 2 * STAGE : EPI];
  __shared__ int last;

  const int tall = int((dw.rows + BM - 1) / BM), wide = int((dw.cols + BN - 1) / BN);
  const TileAt t = tile_at(blockIdx.x, gridDim.x, tall, wide, shares);
  const int64_t i0 = int64_t(t.ti) * BM, o0 = int64_t(t.tj) * BN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  // Slices of this part, in the order ke - 1, ke - 2, kb, kb + 1, ...
  const int64_t tokens = x.rows;
  const int nk = int((tokens + KT - 1) / KT);  // at most 2^21, times 8 parts
  const int kb = t.part * nk / t.parts, ke = (t.part + 1) * nk / t.parts, count = ke - kb;

  const int64_t padded = (x.cols + kBlockCols - 1) / kBlockCols * kBlockCols;
  uint32_t xoff[XC], xlds[XC], yoff[YC], ylds[YC];
  int xt[XC], yt[YC], ycol[YC];
  uint32_t xshift[XC];
#pragma unroll
  for (int j = 0; j < XC; ++j) {
    const int u = tid + NT * j, c = u % (BM / 16);
    xt[j] = u / (BM / 16);
    // Features past the padded columns: those of the first chunk instead
    // (rows of dW that are not stored).
    xoff[j] = uint32_t(xt[j]) * uint32_t(x.ld) + (i0 + 16 * c < padded ? 16 * c : 0);
    xshift[j] = 8 * uint32_t((i0 / kBlockCols + c / 8) % 4);
    xlds[j] = lds_addr(lds) + xt[j] * XP + (((2 * c) ^ row_swz(xt[j])) << 4);
  }
#pragma unroll
  for (int j = 0; j < YC; ++j) {
    const int u = tid + NT * j, c = u % (BN / 8);
    yt[j] = u / (BN / 8);
    ycol[j] = o0 + 8 * c < dy.cols ? 8 * c : 0;
    yoff[j] = 2 * (uint32_t(yt[j]) * uint32_t(dy.ld) + uint32_t(ycol[j]));
    ylds[j] = lds_addr(lds) + KT * XP + yt[j] * YP + ((c ^ row_swz(yt[j])) << 4);
  }
  const uint8_t* const xbase = x.data + i0;
  const uint32_t* const sbase = x.scales + i0 / kGroupCols * x.scale_ld;
  const uint16_t* const ybase = static_cast<const uint16_t*>(dy.ptr) + o0;

  constexpr int NF = TM + TN, NM = TM * TN, NR = 2 * NF;
  struct Set {
    u32x4_t x[XC], y[YC];
    uint32_t s[XC];
  };
  // Slices on their way: a small tile's take less time than a load from memory.
  constexpr int SETS = NM <= 4 ? 4 : 2;
  Set in[SETS];
  // Slice k: at least 8 tokens follow it, so a 16-byte load that passes the end
  // of its row stays inside the matrix.
  auto load_inner = [&](Set& r, int64_t k) {
    const int64_t t0 = k * KT;
#pragma unroll
    for (int j = 0; j < XC; ++j) {
      r.x[j] = gload<u32x4_t, 16>(xbase + t0 * x.ld + xoff[j]);
      r.s[j] = gload<uint32_t, 4>(sbase + t0 + xt[j]);
    }
#pragma unroll
    for (int j = 0; j < YC; ++j)
      r.y[j] = gload<u32x4_t, 2>(reinterpret_cast<const unsigned char*>(ybase + t0 * dy.ld) + yoff[j]);
  };
  // Any slice: tokens past the end as zeros, and where 16 bytes would pass the
  // end of a row, its elements one by one.
  auto load_any = [&](Set& r, int64_t k) {
    const int64_t t0 = k * KT;
    if (t0 + KT + 8 <= tokens) return load_inner(r, k);
#pragma unroll
    for (int j = 0; j < XC; ++j) {
      const int64_t row = t0 + xt[j];
      const int64_t at = row < tokens ? 0 : tokens - 1 - row;  // back to the last token
      r.x[j] = gload<u32x4_t, 16>(xbase + t0 * x.ld + at * x.ld + xoff[j]);
      r.s[j] = gload<uint32_t, 4>(sbase + row + at);
      if (at) r.x[j] = u32x4_t{0, 0, 0, 0};
    }
#pragma unroll
    for (int j = 0; j < YC; ++j) {
      const int64_t row = t0 + yt[j];
      const uint16_t* p = ybase + (row < tokens ? row : tokens - 1) * dy.ld + ycol[j];
      const int64_t n = dy.cols - o0 - ycol[j];
      if (n >= 8) {
        r.y[j] = gload<u32x4_t, 2>(p);
      } else {
        uint32_t h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = gload<uint16_t, 2>(p + (e < n ? e : 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) r.y[j][e] = h[2 * e] | h[2 * e + 1] << 16;
      }
      if (row >= tokens) r.y[j] = u32x4_t{0, 0, 0, 0};
    }
  };
  // Chunk j of the slice in r into a slot: X widened, dY as it is.
  auto write_x = [&](const Set& r, int j, uint32_t slot) {
    const float s = scale_of(r.s[j] >> xshift[j] & 255u);
    u32x4_t lo, hi;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const u32x2_t p = widen4<F>(r.x[j][e], s), q = widen4<F>(r.x[j][2 + e], s);
      lo[2 * e] = p[0];
      lo[2 * e + 1] = p[1];
      hi[2 * e] = q[0];
      hi[2 * e + 1] = q[1];
    }
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
    lds_u32x4_t* at = (lds_u32x4_t*)(uintptr_t)(xlds[j] + slot);
    at[0] = lo;
    at[1] = hi;
  };
  auto write_y = [&](const Set& r, int j, uint32_t slot) {
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
    *(lds_u32x4_t*)(uintptr_t)(ylds[j] + slot) = r.y[j];
  };

  f32x16_t acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = f32x16_t{};

  // Lane addresses of fragment f: 16 columns of 4 tokens per 16 lanes.
  uint32_t fa[NF];
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    const int si = lane & 15, g = lane >> 4;
    const int col = (f < TM ? wm * 32 * TM + 32 * f : wn * 32 * TN + 32 * (f - TM)) + 16 * (g & 1) + 4 * (si & 3);
    const int kr = 8 * (g >> 1) + (si >> 2);
    fa[f] = lds_addr(lds) + (f < TM ? kr * XP : KT * XP + kr * YP) + (((col >> 3) ^ row_swz(kr)) << 4) + 8 * (si & 1);
  }
  // Fragments of one step of 16 tokens, as halves until their wait.
  using Half = u32x2_t[NF][2];
  using Frag = u32x4_t[NF];
  auto read_half = [&](auto o, auto step, auto slot, Half& h) {
    constexpr int f = o / 2, r = o % 2;
    constexpr int off = slot * STAGE + (16 * step + 4 * r) * (f < TM ? XP : YP);
    h[f][r] = lds_read8_tr<off>(fa[f]);
  };
  auto landed = [&](Half& h, Frag& to) {
    lgkm_wait();
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      hold(h[f][0]);
      hold(h[f][1]);
      to[f] = __builtin_shufflevector(h[f][0], h[f][1], 0, 1, 2, 3);
    }
  };
  auto mfma = [&](const Frag& f, int q) {
    const int i = q / TN, j = q % TN;
    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, f[TM + j]),
                                                        __builtin_bit_cast(bf16x8_t, f[i]), acc[i][j], 0, 0, 0);
  };
  // Write o of slice r into a slot.
  auto write = [&](auto o, const Set& r, uint32_t slot) {
    if constexpr (o < XC)
      write_x(r, o, slot);
    else
      write_y(r, o - XC, slot);
  };
  using Zero = std::integral_constant<int, 0>;
  using One = std::integral_constant<int, 1>;
  constexpr int NW = XC + YC;
  // The n-th slice, n >= 2 (past the end: the last, unused).
  auto load_next = [&](Set& r, int n) { load_inner(r, kb + min(n, count - 1) - 2); };
  Half half[2];
  Frag fr[2];
  if (count > 0) {
    load_any(in[0], ke - 1);
    if (count > 1) load_any(in[1], ke - 2);
    if (count > 2)
      each<SETS - 2>([&](auto i) { load_next(in[i + 2], i + 2); });
    each<NW>([&](auto o) { write(o, in[0], 0); });
    if (count > 2) load_next(in[0], SETS);
    lgkm_wait();
    barrier_no_fence();
    each<NR>([&](auto o) { read_half(o, Zero{}, Zero{}, half[0]); });
    landed(half[0], fr[0]);
  }
  // Slice n, n % SETS = i, in slot n % 2, its step 0 in fr[0]; the next SETS - 1
  // slices are in registers or on their way there.
  auto slice = [&](auto i, auto more, int n) {
    constexpr int P = i % 2, Q = P ^ 1, S = (i + 1) % SETS;
    using Here = std::integral_constant<int, P>;
    using Next = std::integral_constant<int, Q>;
    // Step 0, with the reads of step 1 and the next slice on its way to LDS
    // (its slot was last read before the barrier of the slice before).
    each<NM>([&](auto q) {
      mfma(fr[0], q);
      each<NR>([&](auto o) {
        if constexpr (o >= q * NR / NM && o < (q + 1) * NR / NM) read_half(o, One{}, Here{}, half[1]);
      });
      each<NW>([&](auto o) {
        if constexpr (o >= q * NW / NM && o < (q + 1) * NW / NM) write(o, in[S], Q * STAGE);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    landed(half[1], fr[1]);
    mfma(fr[1], 0);
    __builtin_amdgcn_sched_barrier(0);
    barrier_no_fence();
    constexpr int R = NM - 1;
    each<R>([&](auto at) {
      mfma(fr[1], at + 1);
      each<NR>([&](auto o) {
        if constexpr (o >= at * NR / R && o < (at + 1) * NR / R) read_half(o, Zero{}, Next{}, half[0]);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (decltype(more)::value) load_next(in[S], n + 1 + SETS);
    landed(half[0], fr[0]);
  };
  int n = 0;
  if (count > 2) {
    for (; n + SETS <= count; n += SETS) each<SETS>([&](auto i) { slice(i, std::true_type{}, n + i); });
    each<SETS - 1>([&](auto i) {
      if (n + i < count) slice(i, std::false_type{}, n + i);
    });
  } else {
    if (count > 0) slice(Zero{}, std::false_type{}, 0);
    if (count > 1) slice(One{}, std::false_type{}, 1);
  }
  if (t.parts > 1 && !join_parts<TM, TN, W>(acc, split, t.split, t.part, t.parts, wave, lane, &last)) return;
  __syncthreads();
  store_tile<T, TM, TN>(acc, reinterpret_cast<float*>(lds) + wave * 32 * (32 * TN + 4), dw, i0 + wm * 32 * TM,
                        o0 + wn * 32 * TN, accumulate);
}

// ---------------------------------------------------------------- weight gradient, few tiles
//
// Tiles of 64 x 64 whose four waves share the slices: each takes every fourth
// one, of the whole tile, through 8 KB of LDS of its own.  One wave's LDS accesses
// are done in order, so the loop has no barrier and no wait but for the operands;
// the four sums then meet in LDS, each wave finishing one 32 x 32 quarter.  For
// matrices of few tiles, where a 128 x 128 tile leaves most CUs idle and takes four
// times the slices.  Measured against that tile, each in its best number of
// parts, us: 333 tokens, 650 x 975 6.8 against 10.9; 512, 1024 x 1024 6.4 against
// 9.9; 16384, 512 x 512 24 against 34; but 512, 2048 x 2048 15.5 against 11.0.
//
// Rows (tokens) of 64 elements, 128 bytes; 16-byte chunk c of row r at
// c ^ 4 (r / 2 % 2): the 4 rows x 64 bytes of a transpose read are on all banks.
template <typename T, Fp8 F>
__global__ __launch_bounds__(256) void k_weight_grad_waves(BlocksRef x, DenseRef dy, DenseRef dw, bool accumulate,
                                                           Shares shares, SplitSpace split) {
  constexpr int B = 64, W = 4, KT = 32, PITCH = 2 * B, SLOT = 2 * KT * PITCH, XC = 2, YC = 4;
  constexpr int SUMS = W * 3 * 32 * 32 * 4;  // three quarters of every wave
  __shared__ __attribute__((aligned(1024))) unsigned char lds[SUMS > W * SLOT ? SUMS : W * SLOT];
  __shared__ int last;

  const int tall = int((dw.rows + B - 1) / B), wide = int((dw.cols + B - 1) / B);
  const TileAt t = tile_at(blockIdx.x, gridDim.x, tall, wide, shares);
  const int64_t i0 = int64_t(t.ti) * B, o0 = int64_t(t.tj) * B;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t tokens = x.rows;
  const int nk = int((tokens + KT - 1) / KT);
  const int kb = t.part * nk / t.parts, ke = (t.part + 1) * nk / t.parts;
  // This wave's slices: ke - 1 - wave, then every fourth before it.
  const int first = ke - 1 - wave, count = first >= kb ? (first - kb) / W + 1 : 0;

  // Lane l has 32 features of token l / 2, and 8 columns of tokens l / 8 + 8 j.
  const int64_t padded = (x.cols + kBlockCols - 1) / kBlockCols * kBlockCols;
  const int xt = lane >> 1, xc = 32 * (lane & 1), yt = lane >> 3;
  const int ycol = o0 + 8 * (lane & 7) < dy.cols ? 8 * (lane & 7) : 0;
  const uint32_t xoff = uint32_t(xt) * uint32_t(x.ld) + (i0 + xc < padded ? xc : 0);
  const uint32_t xshift = 8 * uint32_t(i0 / kBlockCols % 4);
  const uint8_t* const xbase = x.data + i0;
  const uint32_t* const sbase = x.scales + i0 / kGroupCols * x.scale_ld;
  const uint16_t* const ybase = static_cast<const uint16_t*>(dy.ptr) + o0 + ycol;

  struct Set {
    u32x4_t x[XC], y[YC];
    uint32_t s;
  };
  // As in k_weight_grad: 8 tokens follow slice k, or any slice.
  auto load_inner = [&](Set& r, int k) {
    const int64_t t0 = int64_t(k) * KT;
#pragma unroll
    for (int j = 0; j < XC; ++j) r.x[j] = gload<u32x4_t, 16>(xbase + t0 * x.ld + xoff + 16 * j);
    r.s = gload<uint32_t, 4>(sbase + t0 + xt);
#pragma unroll
    for (int j = 0; j < YC; ++j) r.y[j] = gload<u32x4_t, 2>(ybase + (t0 + yt + 8 * j) * dy.ld);
  };
  auto load_any = [&](Set& r, int k) {
    const int64_t t0 = int64_t(k) * KT;
    if (t0 + KT + 8 <= tokens) return load_inner(r, k);
    const int64_t back = t0 + xt < tokens ? 0 : tokens - 1 - (t0 + xt);  // to the last token
#pragma unroll
    for (int j = 0; j < XC; ++j) {
      r.x[j] = gload<u32x4_t, 16>(xbase + (t0 + back) * x.ld + xoff + 16 * j);
      if (back) r.x[j] = u32x4_t{0, 0, 0, 0};
    }
    r.s = gload<uint32_t, 4>(sbase + t0 + xt + back);
    const int64_t n = dy.cols - o0 - ycol;
#pragma unroll
    for (int j = 0; j < YC; ++j) {
      const int64_t row = t0 + yt + 8 * j;
      const uint16_t* p = ybase + (row < tokens ? row : tokens - 1) * dy.ld;
      if (n >= 8) {
        r.y[j] = gload<u32x4_t, 2>(p);
      } else {
        uint32_t h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = gload<uint16_t, 2>(p + (e < n ? e : 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) r.y[j][e] = h[2 * e] | h[2 * e + 1] << 16;
      }
      if (row >= tokens) r.y[j] = u32x4_t{0, 0, 0, 0};
    }
  };

  const uint32_t mine = lds_addr(lds) + wave * SLOT;
  auto swz64 = [](int r) { return 4 * (r >> 1 & 1); };
  typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
  auto write = [&](const Set& r) {
    const float s = scale_of(r.s >> xshift & 255u);
#pragma unroll
    for (int j = 0; j < XC; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x2_t p = widen4<F>(r.x[j][2 * h], s), q = widen4<F>(r.x[j][2 * h + 1], s);
        *(lds_u32x4_t*)(uintptr_t)(mine + xt * PITCH + (((xc / 8 + 2 * j + h) ^ swz64(xt)) << 4)) =
            u32x4_t{p[0], p[1], q[0], q[1]};
      }
#pragma unroll
    for (int j = 0; j < YC; ++j) {
      const int row = yt + 8 * j;
      *(lds_u32x4_t*)(uintptr_t)(mine + KT * PITCH + row * PITCH + (((lane & 7) ^ swz64(row)) << 4)) = r.y[j];
    }
  };
  // Lane addresses of the four fragments (X 0, 1, dY 0, 1).
  uint32_t fa[4];
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    const int si = lane & 15, g = lane >> 4;
    const int col = 32 * (f & 1) + 16 * (g & 1) + 4 * (si & 3), kr = 8 * (g >> 1) + (si >> 2);
    fa[f] = mine + (f < 2 ? 0 : KT * PITCH) + kr * PITCH + (((col >> 3) ^ swz64(kr)) << 4) + 8 * (si & 1);
  }
  f32x16_t acc[2][2];
#pragma unroll
  for (int q = 0; q < 4; ++q) acc[q / 2][q % 2] = f32x16_t{};
  u32x2_t half[2][4][2];
  auto multiply = [&]() {
    asm volatile("" ::: "memory");  // the slice is written first; the hardware keeps the order
    each<16>([&](auto o) {
      constexpr int step = o / 8, f = o / 2 % 4, r = o % 2;
      half[step][f][r] = lds_read8_tr<(16 * step + 4 * r) * PITCH>(fa[f]);
    });
    each<2>([&](auto step) {
      if constexpr (step == 0)
        asm volatile("s_waitcnt lgkmcnt(8)" ::: "memory");  // the reads of step 1 are on their way
      else
        lgkm_wait();
      u32x4_t fr[4];
#pragma unroll
      for (int f = 0; f < 4; ++f) {
        hold(half[step][f][0]);
        hold(half[step][f][1]);
        fr[f] = __builtin_shufflevector(half[step][f][0], half[step][f][1], 0, 1, 2, 3);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q)
        acc[q / 2][q % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, fr[2 + q % 2]),
                                                                    __builtin_bit_cast(bf16x8_t, fr[q / 2]),
                                                                    acc[q / 2][q % 2], 0, 0, 0);
    });
  };
  if (count > 0) {
    Set in[2];
    load_any(in[0], first);
    if (count > 1) {
      load_inner(in[1], first - W);
      int n = 0;
      // Two slices ahead (past the end: the last again, unused).
      for (; n + 1 < count; n += 2) {
        write(in[0]);
        load_inner(in[0], first - W * min(n + 2, count - 1));
        multiply();
        write(in[1]);
        load_inner(in[1], first - W * min(n + 3, count - 1));
        multiply();
      }
      if (n < count) {
        write(in[0]);
        multiply();
      }
    } else {
      write(in[0]);
      multiply();
    }
  }
  // Quarter q goes to wave q; the sum is in the order of the waves.
  __syncthreads();
  f32x16_t own = {};
  typedef __attribute__((address_space(3))) f32x4_t lds_f32x4_t;
  auto at = [&](int q, int from) {  // the three other waves of quarter q
    return lds_addr(lds) + ((q * 3 + (from < q ? from : from - 1)) * 4 * 64 + lane) * 16;
  };
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const f32x16_t& a = acc[q / 2][q % 2];
    if (wave == q) {
      own = a;
    } else {
#pragma unroll
      for (int v = 0; v < 4; ++v)
        *(lds_f32x4_t*)(uintptr_t)(at(q, wave) + v * 1024) = f32x4_t{a[4 * v], a[4 * v + 1], a[4 * v + 2], a[4 * v + 3]};
    }
  }
  __syncthreads();
  f32x16_t total[1][1] = {};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w == wave) {
      total[0][0] += own;
    } else {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const f32x4_t p = *(const lds_f32x4_t*)(uintptr_t)(at(wave, w) + v * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) total[0][0][4 * v + e] += p[e];
      }
    }
  }
  if (t.parts > 1 && !join_parts<1, 1, W>(total, split, t.split, t.part, t.parts, wave, lane, &last)) return;
  __syncthreads();
  store_tile<T, 1, 1>(total, reinterpret_cast<float*>(lds) + wave * 32 * 36, dw, i0 + 32 * (wave >> 1),
                      o0 + 32 * (wave & 1), accumulate);
}

template <typename F>
hipError_t with_fp8(Fp8 v, F&& f) {
  return v == Fp8::E4M3 ? f(std::integral_constant<Fp8, Fp8::E4M3>{}) : f(std::integral_constant<Fp8, Fp8::E5M2>{});
}

}  // namespace

hipError_t launch_product(DType out_t, Fp8 a_fmt, const BlocksRef& a, const BlocksRef& b, const DenseRef& c,
                          bool accumulate, bool fp32_sums, const SplitSpace& split, int cus, hipStream_t s) {
  return with_fp8(a_fmt, [&](auto fmt) {
    constexpr Fp8 F = decltype(fmt)::value;
    auto go = [&](auto k, const Choice& p, int threads) {
      return launch(k, p.groups, threads, s, a, b, c, accumulate, p.shares, split);
    };
    auto run = [&](auto t, auto exact) {
      using T = decltype(t);
      constexpr bool EXACT = decltype(exact)::value;
      if (c.rows <= kFewRows) {
        const unsigned groups = unsigned((a.cols + kGroupCols - 1) / kGroupCols);
        const unsigned waves = groups < unsigned(kFewWaves) ? groups : unsigned(kFewWaves);
        return launch(k_product_few<T, F, EXACT>, unsigned((c.cols + 15) / 16), 64 * waves, s, a, b, c, accumulate);
      }
      const Choice p = product_choice(EXACT, c.rows, c.cols, a.cols, split.sum_floats, cus);
      if constexpr (EXACT) {
        if (p.tile == 0) return go(k_product<T, F, true, 2, 2, 2, 2>, p, 256);
        return go(k_product<T, F, true, 1, 2, 2, 2>, p, 256);
      } else {
        if (p.tile == 0) return go(k_product<T, F, false, 4, 2, 2, 4>, p, 512);
        if (p.tile == 1) return go(k_product<T, F, false, 2, 2, 2, 2>, p, 256);
        if (p.tile == 2) return go(k_product<T, F, false, 1, 2, 2, 2>, p, 256);
        return go(k_product<T, F, false, 2, 2, 2, 4>, p, 512);
      }
    };
    if (out_t == DType::F32) return run(float{}, std::true_type{});
    return fp32_sums ? run(bf16{}, std::true_type{}) : run(bf16{}, std::false_type{});
  });
}

hipError_t launch_weight_grad(DType out_t, Fp8 x_fmt, const BlocksRef& x, const DenseRef& dy, const DenseRef& dw,
                              bool accumulate, const SplitSpace& split, int cus, hipStream_t s) {
  const Choice p = weight_grad_choice(dw.rows, dw.cols, x.rows, split.sum_floats, cus);
  return with_fp8(x_fmt, [&](auto fmt) {
    constexpr Fp8 F = decltype(fmt)::value;
    auto go = [&](auto k, int threads) {
      return launch(k, p.groups, threads, s, x, dy, dw, accumulate, p.shares, split);
    };
    auto pick = [&](auto t) {
      using T = decltype(t);
      if (p.tile == 0) return go(k_weight_grad<T, F, 4, 2, 2, 4>, 512);
      if (p.tile == 1) return go(k_weight_grad<T, F, 2, 2, 2, 2>, 256);
      return go(k_weight_grad_waves<T, F>, 256);
    };
    return out_t == DType::BF16 ? pick(bf16{}) : pick(float{});
  });
}

}  // namespace muonbp
