// C ABI of the 8-bit linear-layer operators: argument checks, the context
// (stream and workspace) and the launches.
#include <hip/hip_runtime_api.h>

#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <new>

#include "../../include/muonbp.h"
#include "linear.h"

using namespace muonbp;

struct muonbp_linear_ctx {
  int device = 0;
  int cus = 256;
  hipStream_t stream = nullptr;
  SplitSpace split{};
  bool fp32_sums = false;
  bool poisoned = false;
  char err[256] = "";
};

namespace {

// Limits of the kernels' index arithmetic, 32-bit offsets inside a tile of 256
// rows, and of a launch, fewer than 2^32 threads: a wave for each row and 512
// columns, in workgroups of four.
constexpr int64_t kMaxCols = int64_t(1) << 22;
constexpr int64_t kMaxStrips = (int64_t(1) << 26) - 4;
static_assert((kMaxStrips + 3) / 4 * 256 < int64_t(1) << 32, "launch");

__attribute__((format(printf, 3, 4))) muonbp_status fail(muonbp_linear_ctx* c, muonbp_status st, const char* fmt,
                                                         ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(c->err, sizeof(c->err), fmt, ap);
  va_end(ap);
  return st;
}

muonbp_status launched(muonbp_linear_ctx* c, hipError_t e, const char* what) {
  if (e == hipSuccess) return MUONBP_OK;
  c->poisoned = true;
  return fail(c, MUONBP_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

muonbp_status usable(muonbp_linear_ctx* c) {
  if (!c) return MUONBP_E_INVALID;
  if (c->poisoned) return MUONBP_E_STATE;
  return MUONBP_OK;
}

struct Range {
  uintptr_t begin = 0, end = 0;
};

Range range_of(const DenseRef& m, size_t es) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(m.ptr);
  return m.rows > 0 ? Range{p, p + (size_t(m.rows - 1) * size_t(m.ld) + size_t(m.cols)) * es} : Range{};
}
int64_t groups_of(int64_t cols) { return (cols + kGroupCols - 1) / kGroupCols; }
int64_t padded(int64_t cols) { return (cols + kBlockCols - 1) / kBlockCols * kBlockCols; }
Range data_range(const BlocksRef& m) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(m.data);
  return m.data && m.rows > 0 ? Range{p, p + size_t(m.rows - 1) * size_t(m.ld) + size_t(padded(m.cols))} : Range{};
}

// The spans of memory of a call's operands: an output may not meet anything
// else.  (Column ranges of one dense matrix interleave, and so do the scale
// words of row ranges of one 8-bit matrix: these do not meet.)
struct Spans {
  struct Span {
    Range r;
    bool out;
    int64_t pitch, width;  // rows of `width` bytes, `pitch` apart
  };
  Span s[24];
  int n = 0;
  void add(Range r, bool out, int64_t pitch, int64_t width) {
    if (r.begin < r.end && n < 24) s[n++] = Span{r, out, pitch, width};
  }
  void dense(const DenseRef& m, size_t es, bool out) {
    if (m.ptr) add(range_of(m, es), out, m.ld * int64_t(es), m.cols * int64_t(es));
  }
  void blocks(const BlocksRef& m, bool out) {
    if (!m.data || m.rows == 0) return;
    add(data_range(m), out, m.ld, padded(m.cols));
    const uintptr_t p = reinterpret_cast<uintptr_t>(m.scales);
    add(Range{p, p + (size_t(groups_of(m.cols) - 1) * size_t(m.scale_ld) + size_t(m.rows)) * 4}, out,
        m.scale_ld * 4, m.rows * 4);
  }
  // Two strided sets of one pitch are apart where their rows pass each other.
  static bool meet(const Span& a, const Span& b) {
    if (b.r.begin < a.r.begin) return meet(b, a);
    if (b.r.begin >= a.r.end) return false;
    if (a.pitch != b.pitch || a.pitch <= 0) return true;
    const int64_t d = int64_t((b.r.begin - a.r.begin) % uint64_t(a.pitch));
    return d < a.width || a.pitch - d < b.width;
  }
  bool clash() const {
    for (int i = 0; i < n; ++i)
      for (int j = i + 1; j < n; ++j)
        if ((s[i].out || s[j].out) && meet(s[i], s[j])) return true;
    return false;
  }
};

muonbp_status check_dense(muonbp_linear_ctx* c, const muonbp_dense* m, const char* name, bool bf16_only,
                          DenseRef* out, DType* t) {
  if (!m) return fail(c, MUONBP_E_INVALID, "%s must not be NULL", name);
  if (m->dtype != MUONBP_BF16 && (bf16_only || m->dtype != MUONBP_F32))
    return fail(c, MUONBP_E_DTYPE, "%s: unsupported dtype", name);
  const int64_t es = m->dtype == MUONBP_F32 ? 4 : 2;
  if (m->rows < 0 || m->rows > kMaxStrips || m->cols < 1 || m->cols > kMaxCols)
    return fail(c, MUONBP_E_SHAPE, "%s: rows 0..2^26 - 4 and cols 1..2^22", name);
  if (m->ld < m->cols || m->ld > (int64_t(1) << 32) || m->rows * groups_of(m->cols) > kMaxStrips)
    return fail(c, MUONBP_E_SHAPE, "%s: ld below cols or over 2^32, or a matrix too large", name);
  if (m->rows > 0 && !m->ptr) return fail(c, MUONBP_E_INVALID, "%s: NULL pointer", name);
  if (reinterpret_cast<uintptr_t>(m->ptr) % uintptr_t(es))
    return fail(c, MUONBP_E_INVALID, "%s: pointer not element-aligned", name);
  *out = DenseRef{m->ptr, m->rows, m->cols, m->ld};
  *t = m->dtype == MUONBP_F32 ? DType::F32 : DType::BF16;
  return MUONBP_OK;
}

muonbp_status check_blocks(muonbp_linear_ctx* c, const muonbp_blocks* m, const char* name, BlocksRef* out, Fp8* f) {
  if (!m) return fail(c, MUONBP_E_INVALID, "%s must not be NULL", name);
  if (m->format != MUONBP_E4M3 && m->format != MUONBP_E5M2)
    return fail(c, MUONBP_E_INVALID, "%s: unknown format", name);
  if (m->rows < 0 || m->rows > kMaxStrips || m->cols < 1 || m->cols > kMaxCols)
    return fail(c, MUONBP_E_SHAPE, "%s: rows 0..2^26 - 4 and cols 1..2^22", name);
  if (m->ld < padded(m->cols) || m->ld % 16 || m->ld > kMaxCols || m->scale_ld < m->rows ||
      m->scale_ld > (int64_t(1) << 31) || m->rows * groups_of(m->cols) > kMaxStrips)
    return fail(c, MUONBP_E_SHAPE, "%s: ld below the padded cols, no multiple of 16 or too large, or scale_ld below rows",
                name);
  if (m->rows > 0 && (!m->data || !m->scales)) return fail(c, MUONBP_E_INVALID, "%s: NULL pointer", name);
  if (reinterpret_cast<uintptr_t>(m->data) % 16 || reinterpret_cast<uintptr_t>(m->scales) % 4)
    return fail(c, MUONBP_E_INVALID, "%s: data not 16-byte aligned, or scales not 4-byte aligned", name);
  *out = BlocksRef{static_cast<uint8_t*>(m->data), m->scales, m->rows, m->cols, m->ld, m->scale_ld};
  *f = m->format == MUONBP_E4M3 ? Fp8::E4M3 : Fp8::E5M2;
  return MUONBP_OK;
}

// Optional 8-bit operand: left as {} where NULL.
muonbp_status check_optional(muonbp_linear_ctx* c, const muonbp_blocks* m, const char* name, BlocksRef* out,
                             Fp8* f) {
  *out = BlocksRef{};
  return m ? check_blocks(c, m, name, out, f) : MUONBP_OK;
}

template <typename A, typename B>
bool same_shape(const A& a, const B& b) {
  return a.rows == b.rows && a.cols == b.cols;
}

size_t size_of(DType t) { return t == DType::F32 ? 4 : 2; }

}  // namespace

#define MUONBP_TRY(call)                               \
  do {                                                 \
    const muonbp_status st_ = (call);                  \
    if (st_ != MUONBP_OK) return st_;                  \
  } while (0)

extern "C" {

void muonbp_linear_options_default(muonbp_linear_options* o) {
  if (!o) return;
  std::memset(o, 0, sizeof(*o));
  o->workspace_bytes = int64_t(64) << 20;
}

muonbp_status muonbp_linear_create(const muonbp_linear_options* opt, void* hip_stream, muonbp_linear_ctx** out) {
  if (!out) return MUONBP_E_INVALID;
  *out = nullptr;
  muonbp_linear_options o;
  muonbp_linear_options_default(&o);
  if (opt) o = *opt;
  if (o.workspace_bytes < 0 || (o.fp32_sums != 0 && o.fp32_sums != 1)) return MUONBP_E_INVALID;
  muonbp_linear_ctx* c = new (std::nothrow) muonbp_linear_ctx();
  if (!c) return MUONBP_E_NOMEM;
  c->stream = static_cast<hipStream_t>(hip_stream);
  c->fp32_sums = o.fp32_sums == 1;
  auto bail = [&](hipError_t e) {
    if (c->split.sums) (void)hipFree(c->split.sums);
    if (c->split.counts) (void)hipFree(c->split.counts);
    delete c;
    (void)hipGetLastError();  // or the next launch of another context would report it
    return e == hipErrorOutOfMemory ? MUONBP_E_NOMEM : MUONBP_E_HIP;
  };
  hipError_t e;
  if ((e = hipGetDevice(&c->device)) != hipSuccess) return bail(e);
  if ((e = hipDeviceGetAttribute(&c->cus, hipDeviceAttributeMultiprocessorCount, c->device)) != hipSuccess)
    return bail(e);
  void* p = nullptr;
  if (o.workspace_bytes >= 4) {
    if ((e = hipMalloc(&p, size_t(o.workspace_bytes))) != hipSuccess) return bail(e);
    c->split.sums = static_cast<float*>(p);
    c->split.sum_floats = o.workspace_bytes / 4;
  }
  if ((e = hipMalloc(&p, kSplitCounts * sizeof(int))) != hipSuccess) return bail(e);
  c->split.counts = static_cast<int*>(p);
  if ((e = hipMemsetAsync(p, 0, kSplitCounts * sizeof(int), c->stream)) != hipSuccess) return bail(e);
  if ((e = hipStreamSynchronize(c->stream)) != hipSuccess) return bail(e);
  *out = c;
  return MUONBP_OK;
}

muonbp_status muonbp_linear_quantize(muonbp_linear_ctx* c, const muonbp_dense* x, const muonbp_blocks* out) {
  MUONBP_TRY(usable(c));
  DenseRef xr;
  BlocksRef o;
  DType t;
  Fp8 f;
  MUONBP_TRY(check_dense(c, x, "x", false, &xr, &t));
  MUONBP_TRY(check_blocks(c, out, "out", &o, &f));
  if (!same_shape(xr, o)) return fail(c, MUONBP_E_SHAPE, "x and out differ in shape");
  Spans sp;
  sp.dense(xr, size_of(t), false);
  sp.blocks(o, true);
  if (sp.clash()) return fail(c, MUONBP_E_INVALID, "out overlaps x");
  if (xr.rows == 0) return MUONBP_OK;
  return launched(c, launch_quantize(t, f, xr, o, c->stream), "quantize");
}

muonbp_status muonbp_linear_quantize_weight(muonbp_linear_ctx* c, const muonbp_dense* w, const muonbp_blocks* out,
                                            const muonbp_blocks* out_t) {
  MUONBP_TRY(usable(c));
  DenseRef wr;
  BlocksRef o, ot;
  DType t;
  Fp8 f = Fp8::E4M3, ft = Fp8::E4M3;
  MUONBP_TRY(check_dense(c, w, "w", false, &wr, &t));
  if (!out && !out_t) return fail(c, MUONBP_E_INVALID, "out and out_t are both NULL");
  MUONBP_TRY(check_optional(c, out, "out", &o, &f));
  MUONBP_TRY(check_optional(c, out_t, "out_t", &ot, &ft));
  if (wr.rows < 1) return fail(c, MUONBP_E_SHAPE, "w has no rows");
  if (out && !same_shape(wr, o)) return fail(c, MUONBP_E_SHAPE, "w and out differ in shape");
  if (out_t && (ot.rows != wr.cols || ot.cols != wr.rows))
    return fail(c, MUONBP_E_SHAPE, "out_t is not of the transposed shape");
  if (out && out_t && f != ft) return fail(c, MUONBP_E_INVALID, "out and out_t differ in format");
  Spans sp;
  sp.dense(wr, size_of(t), false);
  sp.blocks(o, true);
  sp.blocks(ot, true);
  if (sp.clash()) return fail(c, MUONBP_E_INVALID, "operands overlap");
  return launched(c, launch_quantize_weight(t, out ? f : ft, wr, o, ot, c->stream), "quantize_weight");
}

muonbp_status muonbp_linear_restore(muonbp_linear_ctx* c, const muonbp_blocks* x, const muonbp_dense* out) {
  MUONBP_TRY(usable(c));
  BlocksRef xr;
  DenseRef o;
  DType t;
  Fp8 f;
  MUONBP_TRY(check_blocks(c, x, "x", &xr, &f));
  MUONBP_TRY(check_dense(c, out, "out", false, &o, &t));
  if (!same_shape(xr, o)) return fail(c, MUONBP_E_SHAPE, "x and out differ in shape");
  Spans sp;
  sp.blocks(xr, false);
  sp.dense(o, size_of(t), true);
  if (sp.clash()) return fail(c, MUONBP_E_INVALID, "out overlaps x");
  if (xr.rows == 0) return MUONBP_OK;
  return launched(c, launch_restore(t, f, xr, o, c->stream), "restore");
}

muonbp_status muonbp_linear_product(muonbp_linear_ctx* c, const muonbp_blocks* a, const muonbp_blocks* b,
                                    const muonbp_dense* out, int32_t accumulate) {
  MUONBP_TRY(usable(c));
  BlocksRef ar, br;
  DenseRef o;
  DType t;
  Fp8 fa, fb;
  MUONBP_TRY(check_blocks(c, a, "a", &ar, &fa));
  MUONBP_TRY(check_blocks(c, b, "b", &br, &fb));
  MUONBP_TRY(check_dense(c, out, "c", false, &o, &t));
  if (accumulate != 0 && accumulate != 1) return fail(c, MUONBP_E_INVALID, "accumulate must be 0 or 1");
  if (fb != Fp8::E4M3) return fail(c, MUONBP_E_INVALID, "b must be e4m3");
  if (ar.cols != br.cols || o.rows != ar.rows || o.cols != br.rows)
    return fail(c, MUONBP_E_SHAPE, "c = a b^T: shapes do not match");
  Spans sp;
  sp.blocks(ar, false);
  sp.blocks(br, false);
  sp.dense(o, size_of(t), true);
  if (sp.clash()) return fail(c, MUONBP_E_INVALID, "c overlaps an operand");
  if (o.rows == 0) return MUONBP_OK;
  return launched(
      c, launch_product(t, fa, ar, br, o, accumulate == 1, c->fp32_sums, c->split, c->cus, c->stream), "product");
}

muonbp_status muonbp_linear_weight_grad(muonbp_linear_ctx* c, const muonbp_blocks* x, const muonbp_dense* dy,
                                        const muonbp_dense* dw, int32_t accumulate) {
  MUONBP_TRY(usable(c));
  BlocksRef xr;
  DenseRef g, o;
  DType tg, t;
  Fp8 f;
  MUONBP_TRY(check_blocks(c, x, "x", &xr, &f));
  MUONBP_TRY(check_dense(c, dy, "dy", true, &g, &tg));
  MUONBP_TRY(check_dense(c, dw, "dw", false, &o, &t));
  if (accumulate != 0 && accumulate != 1) return fail(c, MUONBP_E_INVALID, "accumulate must be 0 or 1");
  if (xr.rows != g.rows || o.rows != xr.cols || o.cols != g.cols)
    return fail(c, MUONBP_E_SHAPE, "dw = x^T dy: shapes do not match");
  if (g.ld > (int64_t(1) << 25)) return fail(c, MUONBP_E_SHAPE, "dy: ld over 2^25");
  Spans sp;
  sp.blocks(xr, false);
  sp.dense(g, size_of(tg), false);
  sp.dense(o, size_of(t), true);
  if (sp.clash()) return fail(c, MUONBP_E_INVALID, "dw overlaps an operand");
  return launched(c, launch_weight_grad(t, f, xr, g, o, accumulate == 1, c->split, c->cus, c->stream),
                  "weight_grad");
}

muonbp_status muonbp_linear_gated_forward(muonbp_linear_ctx* c, const muonbp_dense* gate, const muonbp_dense* up,
                                          const muonbp_dense* h, const muonbp_blocks* out8,
                                          const muonbp_blocks* gate_kept, const muonbp_blocks* up_kept) {
  MUONBP_TRY(usable(c));
  DenseRef g, u, o{};
  BlocksRef o8, g8, u8;
  DType t, tu, to;
  Fp8 f = Fp8::E4M3, fg = Fp8::E4M3, fu = Fp8::E4M3;
  MUONBP_TRY(check_dense(c, gate, "gate", false, &g, &t));
  MUONBP_TRY(check_dense(c, up, "up", false, &u, &tu));
  to = t;
  if (h) MUONBP_TRY(check_dense(c, h, "h", false, &o, &to));
  MUONBP_TRY(check_optional(c, out8, "out8", &o8, &f));
  MUONBP_TRY(check_optional(c, gate_kept, "gate_kept", &g8, &fg));
  MUONBP_TRY(check_optional(c, up_kept, "up_kept", &u8, &fu));
  if (!h && !out8) return fail(c, MUONBP_E_INVALID, "h and out8 are both NULL");
  if (!gate_kept != !up_kept) return fail(c, MUONBP_E_INVALID, "gate_kept and up_kept: both or neither");
  if (t != tu || t != to) return fail(c, MUONBP_E_DTYPE, "gate, up and h differ in dtype");
  if (fg != fu) return fail(c, MUONBP_E_INVALID, "gate_kept and up_kept differ in format");
  if (!same_shape(g, u) || (h && !same_shape(g, o)) || (out8 && !same_shape(g, o8)) ||
      (gate_kept && (!same_shape(g, g8) || !same_shape(g, u8))))
    return fail(c, MUONBP_E_SHAPE, "operands differ in shape");
  Spans sp;
  sp.dense(g, size_of(t), false);
  sp.dense(u, size_of(t), false);
  sp.dense(o, size_of(t), true);
  sp.blocks(o8, true);
  sp.blocks(g8, true);
  sp.blocks(u8, true);
  if (sp.clash()) return fail(c, MUONBP_E_INVALID, "operands overlap");
  if (g.rows == 0) return MUONBP_OK;
  return launched(c, launch_gated_forward(t, g, u, o, o8, f, g8, u8, fg, c->stream), "gated_forward");
}

muonbp_status muonbp_linear_gated_backward(muonbp_linear_ctx* c, const muonbp_dense* dh, const muonbp_blocks* gate,
                                           const muonbp_blocks* up, const muonbp_dense* dgate,
                                           const muonbp_dense* dup, const muonbp_blocks* dgate8,
                                           const muonbp_blocks* dup8) {
  MUONBP_TRY(usable(c));
  DenseRef d, dg{}, du{};
  BlocksRef g, u, dg8, du8;
  DType t, tg, tu;
  Fp8 fg, fu, f = Fp8::E4M3, f2 = Fp8::E4M3;
  MUONBP_TRY(check_dense(c, dh, "dh", false, &d, &t));
  MUONBP_TRY(check_blocks(c, gate, "gate", &g, &fg));
  MUONBP_TRY(check_blocks(c, up, "up", &u, &fu));
  tg = tu = t;
  if (dgate) MUONBP_TRY(check_dense(c, dgate, "dgate", false, &dg, &tg));
  if (dup) MUONBP_TRY(check_dense(c, dup, "dup", false, &du, &tu));
  MUONBP_TRY(check_optional(c, dgate8, "dgate8", &dg8, &f));
  MUONBP_TRY(check_optional(c, dup8, "dup8", &du8, &f2));
  if (!dgate != !dup || !dgate8 != !dup8)
    return fail(c, MUONBP_E_INVALID, "dgate and dup, dgate8 and dup8: both or neither");
  if (!dgate && !dgate8) return fail(c, MUONBP_E_INVALID, "no output given");
  if (t != tg || t != tu) return fail(c, MUONBP_E_DTYPE, "dh, dgate and dup differ in dtype");
  if (fg != fu || f != f2) return fail(c, MUONBP_E_INVALID, "a pair differs in format");
  if (!same_shape(d, g) || !same_shape(d, u) || (dgate && (!same_shape(d, dg) || !same_shape(d, du))) ||
      (dgate8 && (!same_shape(d, dg8) || !same_shape(d, du8))))
    return fail(c, MUONBP_E_SHAPE, "operands differ in shape");
  Spans sp;
  sp.dense(d, size_of(t), false);
  sp.blocks(g, false);
  sp.blocks(u, false);
  sp.dense(dg, size_of(t), true);
  sp.dense(du, size_of(t), true);
  sp.blocks(dg8, true);
  sp.blocks(du8, true);
  if (sp.clash()) return fail(c, MUONBP_E_INVALID, "operands overlap");
  if (d.rows == 0) return MUONBP_OK;
  return launched(c, launch_gated_backward(t, d, g, u, fg, dg, du, dg8, du8, f, c->stream), "gated_backward");
}

muonbp_status muonbp_linear_set_stream(muonbp_linear_ctx* c, void* hip_stream) {
  MUONBP_TRY(usable(c));
  MUONBP_TRY(launched(c, hipStreamSynchronize(c->stream), "hipStreamSynchronize"));
  c->stream = static_cast<hipStream_t>(hip_stream);
  return MUONBP_OK;
}

muonbp_status muonbp_linear_synchronize(muonbp_linear_ctx* c) {
  MUONBP_TRY(usable(c));
  return launched(c, hipStreamSynchronize(c->stream), "hipStreamSynchronize");
}

const char* muonbp_linear_last_error(const muonbp_linear_ctx* c) { return c ? c->err : "NULL context"; }

void muonbp_linear_destroy(muonbp_linear_ctx* c) {
  if (!c) return;
  (void)hipStreamSynchronize(c->stream);
  if (c->split.sums) (void)hipFree(c->split.sums);
  if (c->split.counts) (void)hipFree(c->split.counts);
  delete c;
}

}  // extern "C"
