// C ABI entry points of the learned blocks (include/gart.h): argument checks,
// then one launcher each.  No device memory is allocated here.
#include <hip/hip_runtime.h>

#include <cmath>

#include "blocks.h"
#include "orthogonalize.h"
#include "status.h"

using namespace gart;

namespace {

constexpr int64_t kMaxSize = (int64_t(1) << 31) - 1;
// Columns of an embedding's gradient: they span a launch's second dimension.
constexpr int64_t kMaxDim = int64_t(1) << 23;

gart_status check_dtype(gart_dtype t) {
  GART_REQUIRE(t >= GART_DTYPE_F32 && t <= GART_DTYPE_F16, "unknown dtype %d", int(t));
  return GART_OK;
}

gart_status check_act(gart_activation a) {
  GART_REQUIRE(a >= GART_ACT_NONE && a <= GART_ACT_GELU, "unknown activation %d", int(a));
  return GART_OK;
}

gart_status check_matrix(const char* name, const gart_matrix* m, gart_dtype t, bool output) {
  GART_REQUIRE(m != nullptr, "%s is NULL", name);
  GART_REQUIRE(m->rows >= 0 && m->rows <= kMaxSize && m->cols >= 0 && m->cols <= kMaxSize, "%s is %lld x %lld", name,
               (long long)m->rows, (long long)m->cols);
  if (m->rows == 0 || m->cols == 0) return GART_OK;
  GART_REQUIRE(m->data != nullptr, "%s data is NULL", name);
  GART_REQUIRE(reinterpret_cast<uintptr_t>(m->data) % dtype_bytes(t) == 0, "%s is not aligned to its elements", name);
  GART_REQUIRE(m->rows == 1 || m->stride >= m->cols || (m->stride == 0 && !output),
               "%s has row stride %lld for %lld columns", name, (long long)m->stride, (long long)m->cols);
  GART_REQUIRE(m->rows == 1 || m->stride <= (int64_t(1) << 60) / m->rows, "%s stride %lld", name,
               (long long)m->stride);
  return GART_OK;
}

gart_status check_vector(const char* name, const void* p, int64_t n, gart_dtype t) {
  GART_REQUIRE(p == nullptr || n == 0 || reinterpret_cast<uintptr_t>(p) % dtype_bytes(t) == 0,
               "%s is not aligned to its elements", name);
  return GART_OK;
}

// The bytes a matrix spans, and how its rows repeat in them.
struct Span {
  uintptr_t begin, end;
  uint64_t row, step;  // bytes of a row, bytes between rows (0: one row)
};

Span span_of(const gart_matrix* m, gart_dtype t) {
  if (m == nullptr || m->rows == 0 || m->cols == 0) return Span{0, 0, 0, 0};
  const uint64_t es = dtype_bytes(t), step = m->rows == 1 ? 0 : uint64_t(m->stride) * es;
  const uintptr_t b = reinterpret_cast<uintptr_t>(m->data);
  const uint64_t row = uint64_t(m->cols) * es;
  return Span{b, b + uint64_t(m->rows - 1) * step + row, row, step};
}

Span span_of(const void* p, int64_t bytes) {
  if (p == nullptr || bytes <= 0) return Span{0, 0, 0, 0};
  const uintptr_t b = reinterpret_cast<uintptr_t>(p);
  return Span{b, b + uint64_t(bytes), uint64_t(bytes), 0};
}

bool overlap(const Span& a, const Span& b) {
  if (a.begin >= b.end || b.begin >= a.end) return false;
  if (a.step == 0 || a.step != b.step) return true;  // interleaved only where rows step alike
  // columns of one wider buffer: disjoint if b's row fits beside a's in a step
  const uint64_t d = b.begin >= a.begin ? (b.begin - a.begin) % a.step
                                        : (a.step - (a.begin - b.begin) % a.step) % a.step;
  return !(d >= a.row && d + b.row <= a.step);
}

bool same(const gart_matrix* a, const gart_matrix* b) {
  return a->data == b->data && (a->rows <= 1 || a->stride == b->stride);
}

gart_status check_scratch(const void* scratch, size_t have, size_t need) {
  GART_REQUIRE(have >= need, "scratch_bytes %zu < required %zu", have, need);
  GART_REQUIRE(need == 0 || scratch != nullptr, "scratch is NULL");
  GART_REQUIRE(need == 0 || reinterpret_cast<uintptr_t>(scratch) % 16 == 0, "scratch must be 16-byte aligned");
  return GART_OK;
}

gart_status check_steps(const gart_newton_schulz& n) {
  GART_REQUIRE(std::isfinite(n.a) && std::isfinite(n.b) && std::isfinite(n.c), "coefficients must be finite");
  GART_REQUIRE(n.eps >= 0.0f && std::isfinite(n.eps), "eps must be at least 0 and finite");
  GART_REQUIRE(n.steps >= 1 && n.steps <= kMaxSteps, "steps must be in [1, %d]", kMaxSteps);
  Factors f;
  GART_REQUIRE(step_factors(n.a, n.b, n.c, n.steps, 1.0, &f.x, f.step), "singular values may pass 1024 in these steps");
  return GART_OK;
}

bool size_ok(int64_t v) { return v >= 0 && v <= kMaxSize; }

}  // namespace

#define GART_CHECK(expr)                            \
  do {                                              \
    const gart_status st_ = (expr);                 \
    if (st_ != GART_OK) return st_;                 \
  } while (0)

extern "C" {

gart_status gart_embedding(const gart_matrix* table, const void* ids, int32_t ids64, float scale, gart_dtype dtype,
                           const gart_matrix* out, void* stream) {
  clear_error();
  GART_CHECK(check_dtype(dtype));
  GART_CHECK(check_matrix("table", table, dtype, false));
  GART_CHECK(check_matrix("out", out, dtype, true));
  GART_REQUIRE(out->cols == table->cols, "out has %lld columns, table %lld", (long long)out->cols,
               (long long)table->cols);
  if (out->rows == 0 || out->cols == 0) return GART_OK;
  const size_t ids_bytes = ids64 ? 8 : 4;
  GART_REQUIRE(ids != nullptr, "ids is NULL");
  GART_REQUIRE(reinterpret_cast<uintptr_t>(ids) % ids_bytes == 0, "ids is not aligned to its elements");
  const Span o = span_of(out, dtype);
  GART_REQUIRE(!overlap(o, span_of(table, dtype)) && !overlap(o, span_of(ids, int64_t(ids_bytes) * out->rows)),
               "out overlaps an input");
  EmbeddingArgs a{};
  a.ids = ids;
  a.ids64 = ids64 != 0;
  a.n = out->rows;
  a.vocab = table->rows;
  a.dim = out->cols;
  a.scale = scale;
  a.table = table->data;
  a.table_ld = table->stride;
  a.out = out->data;
  a.out_ld = out->stride;
  GART_HIP(launch_embedding(a, dtype, static_cast<hipStream_t>(stream)));
  return GART_OK;
}

size_t gart_embedding_scratch_bytes(int64_t n, int64_t vocab, int64_t dim) {
  if (!size_ok(n) || !size_ok(vocab) || !size_ok(dim)) return 0;
  return embedding_scratch_bytes(n, vocab, dim);
}

gart_status gart_embedding_backward(const void* ids, int32_t ids64, const gart_matrix* dl_dout, float scale,
                                    gart_dtype dtype, const gart_matrix* g_table, void* scratch,
                                    size_t scratch_bytes, void* stream) {
  clear_error();
  GART_CHECK(check_dtype(dtype));
  GART_CHECK(check_matrix("dl_dout", dl_dout, dtype, false));
  GART_CHECK(check_matrix("g_table", g_table, dtype, true));
  GART_REQUIRE(g_table->cols == dl_dout->cols, "g_table has %lld columns, dl_dout %lld", (long long)g_table->cols,
               (long long)dl_dout->cols);
  if (g_table->rows == 0 || g_table->cols == 0) return GART_OK;
  if (g_table->cols > kMaxDim || !embedding_backward_launchable(dl_dout->rows, g_table->cols, dtype))
    return fail(GART_ERR_UNSUPPORTED, "%lld ids of %lld columns", (long long)dl_dout->rows, (long long)g_table->cols);
  const size_t ids_bytes = ids64 ? 8 : 4;
  GART_REQUIRE(dl_dout->rows == 0 || ids != nullptr, "ids is NULL");
  GART_REQUIRE(reinterpret_cast<uintptr_t>(ids) % ids_bytes == 0, "ids is not aligned to its elements");
  const size_t need = embedding_scratch_bytes(dl_dout->rows, g_table->rows, g_table->cols);
  GART_CHECK(check_scratch(scratch, scratch_bytes, need));
  const Span o = span_of(g_table, dtype);
  GART_REQUIRE(!overlap(o, span_of(dl_dout, dtype)) && !overlap(o, span_of(ids, int64_t(ids_bytes) * dl_dout->rows)),
               "g_table overlaps an input");
  const Span w = span_of(scratch, int64_t(need));
  GART_REQUIRE(!overlap(w, o) && !overlap(w, span_of(dl_dout, dtype)) &&
                   !overlap(w, span_of(ids, int64_t(ids_bytes) * dl_dout->rows)),
               "scratch overlaps an argument");
  EmbeddingArgs a{};
  a.ids = ids;
  a.ids64 = ids64 != 0;
  a.n = dl_dout->rows;
  a.vocab = g_table->rows;
  a.dim = g_table->cols;
  a.scale = scale;
  a.rows = dl_dout->data;
  a.rows_ld = dl_dout->stride;
  a.out = g_table->data;
  a.out_ld = g_table->stride;
  a.scratch = scratch;
  GART_HIP(launch_embedding_backward(a, dtype, static_cast<hipStream_t>(stream)));
  return GART_OK;
}

gart_status gart_dropout(const gart_matrix* x, const gart_matrix* residual, float p, uint64_t seed, uint64_t offset,
                         gart_dtype dtype, const gart_matrix* y, void* stream) {
  clear_error();
  GART_CHECK(check_dtype(dtype));
  GART_CHECK(check_matrix("x", x, dtype, false));
  GART_CHECK(check_matrix("y", y, dtype, true));
  GART_REQUIRE(x->rows == y->rows && x->cols == y->cols, "x and y differ in size");
  GART_REQUIRE(p >= 0.0f && p <= 1.0f, "p must be in [0, 1]");
  if (residual) {
    GART_CHECK(check_matrix("residual", residual, dtype, false));
    GART_REQUIRE(residual->rows == y->rows && residual->cols == y->cols, "residual and y differ in size");
  }
  if (y->rows == 0 || y->cols == 0) return GART_OK;
  const Span o = span_of(y, dtype);
  GART_REQUIRE(same(x, y) || !overlap(o, span_of(x, dtype)), "y overlaps x");
  GART_REQUIRE(!residual || same(residual, y) || !overlap(o, span_of(residual, dtype)), "y overlaps the residual");
  DropoutArgs a{};
  a.x = x->data;
  a.x_ld = x->stride;
  a.residual = residual ? residual->data : nullptr;
  a.residual_ld = residual ? residual->stride : 0;
  a.y = y->data;
  a.y_ld = y->stride;
  a.rows = y->rows;
  a.cols = y->cols;
  a.threshold = uint32_t(std::floor(double(p) * 65536.0 + 0.5));
  a.scale = a.threshold < 65536u ? float(65536.0 / double(65536u - a.threshold)) : 0.0f;
  a.seed = seed;
  a.offset = offset;
  GART_HIP(launch_dropout(a, dtype, static_cast<hipStream_t>(stream)));
  return GART_OK;
}

size_t gart_linear_scratch_bytes(int64_t rows, int64_t inputs, int64_t outputs, gart_dtype dtype) {
  clear_error();
  if (!size_ok(rows) || !size_ok(inputs) || !size_ok(outputs) || check_dtype(dtype) != GART_OK) return 0;
  const int64_t b = linear_scratch_bytes(rows, inputs, outputs, dtype);
  return b < 0 ? 0 : size_t(b);
}

size_t gart_linear_backward_scratch_bytes(int64_t rows, int64_t inputs, int64_t outputs, gart_dtype dtype,
                                          gart_activation act) {
  clear_error();
  if (!size_ok(rows) || !size_ok(inputs) || !size_ok(outputs) || check_dtype(dtype) != GART_OK ||
      check_act(act) != GART_OK)
    return 0;
  const int64_t b = linear_backward_scratch_bytes(rows, inputs, outputs, dtype, act);
  return b < 0 ? 0 : size_t(b);
}

gart_status gart_linear(const gart_matrix* x, const gart_matrix* weight, const void* bias,
                        const gart_matrix* residual, gart_activation act, gart_dtype dtype, const gart_matrix* y,
                        void* scratch, size_t scratch_bytes, void* stream) {
  clear_error();
  GART_CHECK(check_dtype(dtype));
  GART_CHECK(check_act(act));
  GART_CHECK(check_matrix("x", x, dtype, false));
  GART_CHECK(check_matrix("weight", weight, dtype, false));
  GART_CHECK(check_matrix("y", y, dtype, true));
  GART_REQUIRE(x->cols == weight->cols, "x has %lld columns, weight %lld", (long long)x->cols, (long long)weight->cols);
  GART_REQUIRE(y->rows == x->rows && y->cols == weight->rows, "y is %lld x %lld, not %lld x %lld", (long long)y->rows,
               (long long)y->cols, (long long)x->rows, (long long)weight->rows);
  GART_CHECK(check_vector("bias", bias, y->cols, dtype));
  if (residual) {
    GART_CHECK(check_matrix("residual", residual, dtype, false));
    GART_REQUIRE(residual->rows == y->rows && residual->cols == y->cols, "residual and y differ in size");
  }
  if (y->rows == 0 || y->cols == 0) return GART_OK;
  const int64_t need = linear_scratch_bytes(x->rows, x->cols, y->cols, dtype);
  if (need < 0) return fail(GART_ERR_UNSUPPORTED, "%lld x %lld outputs", (long long)y->rows, (long long)y->cols);
  GART_CHECK(check_scratch(scratch, scratch_bytes, size_t(need)));
  const Span o = span_of(y, dtype);
  GART_REQUIRE(!overlap(o, span_of(x, dtype)) && !overlap(o, span_of(weight, dtype)) &&
                   !overlap(o, span_of(bias, y->cols * int64_t(dtype_bytes(dtype)))),
               "y overlaps an input");
  GART_REQUIRE(!residual || same(residual, y) || !overlap(o, span_of(residual, dtype)), "y overlaps the residual");
  const Span s = span_of(scratch, need);
  GART_REQUIRE(!overlap(s, o) && !overlap(s, span_of(x, dtype)) && !overlap(s, span_of(weight, dtype)) &&
                   !overlap(s, span_of(bias, y->cols * int64_t(dtype_bytes(dtype)))) &&
                   !overlap(s, span_of(residual, dtype)),
               "scratch overlaps an argument");
  LinearArgs a{};
  a.m = x->rows;
  a.k = x->cols;
  a.n = y->cols;
  a.act = act;
  a.x = x->data;
  a.x_ld = x->stride;
  a.w = weight->data;
  a.w_ld = weight->stride;
  a.bias = bias;
  a.residual = residual ? residual->data : nullptr;
  a.residual_ld = residual ? residual->stride : 0;
  a.y = y->data;
  a.y_ld = y->stride;
  a.scratch = scratch;
  GART_HIP(launch_linear(a, dtype, static_cast<hipStream_t>(stream)));
  return GART_OK;
}

gart_status gart_linear_backward(const gart_matrix* x, const gart_matrix* weight, const void* bias,
                                 gart_activation act, const gart_matrix* dl_dy, gart_dtype dtype,
                                 const gart_matrix* g_x, const gart_matrix* g_weight, void* g_bias, void* scratch,
                                 size_t scratch_bytes, void* stream) {
  clear_error();
  GART_CHECK(check_dtype(dtype));
  GART_CHECK(check_act(act));
  GART_CHECK(check_matrix("x", x, dtype, false));
  GART_CHECK(check_matrix("weight", weight, dtype, false));
  GART_CHECK(check_matrix("dl_dy", dl_dy, dtype, false));
  GART_REQUIRE(x->cols == weight->cols, "x has %lld columns, weight %lld", (long long)x->cols, (long long)weight->cols);
  GART_REQUIRE(dl_dy->rows == x->rows && dl_dy->cols == weight->rows, "dl_dy is %lld x %lld, not %lld x %lld",
               (long long)dl_dy->rows, (long long)dl_dy->cols, (long long)x->rows, (long long)weight->rows);
  GART_CHECK(check_vector("bias", bias, weight->rows, dtype));
  GART_CHECK(check_vector("g_bias", g_bias, weight->rows, dtype));
  if (g_x) {
    GART_CHECK(check_matrix("g_x", g_x, dtype, true));
    GART_REQUIRE(g_x->rows == x->rows && g_x->cols == x->cols, "g_x and x differ in size");
  }
  if (g_weight) {
    GART_CHECK(check_matrix("g_weight", g_weight, dtype, true));
    GART_REQUIRE(g_weight->rows == weight->rows && g_weight->cols == weight->cols,
                 "g_weight and weight differ in size");
  }
  const int64_t need = linear_backward_scratch_bytes(x->rows, x->cols, weight->rows, dtype, act);
  if (need < 0)
    return fail(GART_ERR_UNSUPPORTED, "%lld rows of %lld inputs and %lld outputs", (long long)x->rows,
                (long long)x->cols, (long long)weight->rows);
  GART_CHECK(check_scratch(scratch, scratch_bytes, size_t(need)));
  const int64_t vec = weight->rows * int64_t(dtype_bytes(dtype));
  const Span out[3] = {span_of(g_x, dtype), span_of(g_weight, dtype), span_of(g_bias, vec)};
  const Span in[4] = {span_of(x, dtype), span_of(weight, dtype), span_of(dl_dy, dtype), span_of(bias, vec)};
  const Span s = span_of(scratch, need);
  for (int j = 0; j < 4; ++j) GART_REQUIRE(!overlap(s, in[j]), "scratch overlaps an input");
  for (int i = 0; i < 3; ++i) {
    GART_REQUIRE(!overlap(s, out[i]), "scratch overlaps a gradient");
    for (int j = 0; j < 4; ++j) GART_REQUIRE(!overlap(out[i], in[j]), "a gradient overlaps an input");
    for (int j = 0; j < i; ++j) GART_REQUIRE(!overlap(out[i], out[j]), "gradients overlap");
  }
  LinearArgs a{};
  a.m = x->rows;
  a.k = x->cols;
  a.n = weight->rows;
  a.act = act;
  a.x = x->data;
  a.x_ld = x->stride;
  a.w = weight->data;
  a.w_ld = weight->stride;
  a.bias = bias;
  a.dl = dl_dy->data;
  a.dl_ld = dl_dy->stride;
  a.g_x = g_x ? g_x->data : nullptr;
  a.g_x_ld = g_x ? g_x->stride : 0;
  a.g_w = g_weight ? g_weight->data : nullptr;
  a.g_w_ld = g_weight ? g_weight->stride : 0;
  a.g_bias = g_bias;
  a.scratch = scratch;
  GART_HIP(launch_linear_backward(a, dtype, static_cast<hipStream_t>(stream)));
  return GART_OK;
}

gart_status gart_layer_norm(const gart_matrix* x, const void* gain, const void* bias, float eps, gart_dtype dtype,
                            const gart_matrix* y, void* stream) {
  clear_error();
  GART_CHECK(check_dtype(dtype));
  GART_CHECK(check_matrix("x", x, dtype, false));
  GART_CHECK(check_matrix("y", y, dtype, true));
  GART_REQUIRE(x->rows == y->rows && x->cols == y->cols, "x and y differ in size");
  GART_REQUIRE(eps >= 0.0f && std::isfinite(eps), "eps must be at least 0 and finite");
  GART_CHECK(check_vector("gain", gain, y->cols, dtype));
  GART_CHECK(check_vector("bias", bias, y->cols, dtype));
  if (y->rows == 0 || y->cols == 0) return GART_OK;
  const Span o = span_of(y, dtype);
  const int64_t vec = y->cols * int64_t(dtype_bytes(dtype));
  GART_REQUIRE(same(x, y) || !overlap(o, span_of(x, dtype)), "y overlaps x");
  GART_REQUIRE(!overlap(o, span_of(gain, vec)) && !overlap(o, span_of(bias, vec)), "y overlaps gain or bias");
  LayerNormArgs a{};
  a.rows = x->rows;
  a.cols = x->cols;
  a.eps = eps;
  a.x = x->data;
  a.x_ld = x->stride;
  a.gain = gain;
  a.bias = bias;
  a.y = y->data;
  a.y_ld = y->stride;
  GART_HIP(launch_layer_norm(a, dtype, static_cast<hipStream_t>(stream)));
  return GART_OK;
}

size_t gart_layer_norm_backward_scratch_bytes(int64_t rows, int64_t cols, gart_dtype dtype) {
  clear_error();
  if (!size_ok(rows) || !size_ok(cols) || check_dtype(dtype) != GART_OK) return 0;
  return layer_norm_backward_scratch_bytes(rows, cols, dtype);
}

gart_status gart_layer_norm_backward(const gart_matrix* x, const gart_matrix* dl_dy, const void* gain, float eps,
                                     gart_dtype dtype, const gart_matrix* g_x, void* g_gain, void* g_bias,
                                     void* scratch, size_t scratch_bytes, void* stream) {
  clear_error();
  GART_CHECK(check_dtype(dtype));
  GART_CHECK(check_matrix("x", x, dtype, false));
  GART_CHECK(check_matrix("dl_dy", dl_dy, dtype, false));
  GART_REQUIRE(x->rows == dl_dy->rows && x->cols == dl_dy->cols, "x and dl_dy differ in size");
  GART_REQUIRE(eps >= 0.0f && std::isfinite(eps), "eps must be at least 0 and finite");
  GART_CHECK(check_vector("gain", gain, x->cols, dtype));
  GART_CHECK(check_vector("g_gain", g_gain, x->cols, dtype));
  GART_CHECK(check_vector("g_bias", g_bias, x->cols, dtype));
  if (g_x) {
    GART_CHECK(check_matrix("g_x", g_x, dtype, true));
    GART_REQUIRE(g_x->rows == x->rows && g_x->cols == x->cols, "g_x and x differ in size");
  }
  const size_t need = layer_norm_backward_scratch_bytes(x->rows, x->cols, dtype);
  GART_CHECK(check_scratch(scratch, scratch_bytes, need));
  const int64_t vec = x->cols * int64_t(dtype_bytes(dtype));
  const Span out[3] = {span_of(g_x, dtype), span_of(g_gain, vec), span_of(g_bias, vec)};
  const Span in[3] = {span_of(x, dtype), span_of(dl_dy, dtype), span_of(gain, vec)};
  const Span s = span_of(scratch, int64_t(need));
  for (int j = 0; j < 3; ++j) GART_REQUIRE(!overlap(s, in[j]), "scratch overlaps an input");
  for (int i = 0; i < 3; ++i) {
    GART_REQUIRE(!overlap(s, out[i]), "scratch overlaps a gradient");
    for (int j = 0; j < 3; ++j) GART_REQUIRE(!overlap(out[i], in[j]), "a gradient overlaps an input");
    for (int j = 0; j < i; ++j) GART_REQUIRE(!overlap(out[i], out[j]), "gradients overlap");
  }
  LayerNormArgs a{};
  a.rows = x->rows;
  a.cols = x->cols;
  a.eps = eps;
  a.x = x->data;
  a.x_ld = x->stride;
  a.gain = gain;
  a.dl = dl_dy->data;
  a.dl_ld = dl_dy->stride;
  a.g_x = g_x ? g_x->data : nullptr;
  a.g_x_ld = g_x ? g_x->stride : 0;
  a.g_gain = g_gain;
  a.g_bias = g_bias;
  a.scratch = scratch;
  GART_HIP(launch_layer_norm_backward(a, dtype, static_cast<hipStream_t>(stream)));
  return GART_OK;
}

size_t gart_orthogonalize_scratch_bytes(int64_t rows, int64_t cols, gart_dtype dtype) {
  clear_error();
  if (!size_ok(rows) || !size_ok(cols) || check_dtype(dtype) != GART_OK) return 0;
  const int64_t b = orthogonalize_scratch_bytes(rows, cols);
  return b < 0 ? 0 : size_t(b);
}

gart_status gart_orthogonalize(const gart_matrix* x, const gart_newton_schulz* how, gart_dtype dtype,
                               const gart_matrix* y, void* scratch, size_t scratch_bytes, void* stream) {
  clear_error();
  GART_CHECK(check_dtype(dtype));
  GART_REQUIRE(how != nullptr, "how is NULL");
  GART_CHECK(check_steps(*how));
  GART_CHECK(check_matrix("x", x, dtype, false));
  GART_CHECK(check_matrix("y", y, dtype, true));
  GART_REQUIRE(x->rows == y->rows && x->cols == y->cols, "x and y differ in size");
  if (y->rows == 0 || y->cols == 0) return GART_OK;
  const int64_t need = orthogonalize_scratch_bytes(x->rows, x->cols);
  if (need < 0) return fail(GART_ERR_UNSUPPORTED, "%lld x %lld", (long long)x->rows, (long long)x->cols);
  GART_CHECK(check_scratch(scratch, scratch_bytes, size_t(need)));
  const Span o = span_of(y, dtype), w = span_of(scratch, need);
  GART_REQUIRE(same(x, y) || !overlap(o, span_of(x, dtype)), "y overlaps x");
  GART_REQUIRE(!overlap(w, o) && !overlap(w, span_of(x, dtype)), "scratch overlaps an argument");
  OrthogonalizeArgs a{};
  a.rows = x->rows;
  a.cols = x->cols;
  a.a = how->a;
  a.b = how->b;
  a.c = how->c;
  a.eps = how->eps;
  a.steps = how->steps;
  a.x = x->data;
  a.x_ld = x->stride;
  a.y = y->data;
  a.y_ld = y->stride;
  a.scratch = scratch;
  GART_HIP(launch_orthogonalize(a, dtype, static_cast<hipStream_t>(stream)));
  return GART_OK;
}

size_t gart_muon_scratch_bytes(int64_t rows, int64_t cols, gart_dtype dtype) {
  return gart_orthogonalize_scratch_bytes(rows, cols, dtype);
}

gart_status gart_muon_step(const gart_matrix* param, const gart_matrix* grad, const gart_matrix* m,
                           const gart_muon* h, gart_dtype dtype, void* scratch, size_t scratch_bytes, void* stream) {
  clear_error();
  GART_CHECK(check_dtype(dtype));
  GART_REQUIRE(h != nullptr, "h is NULL");
  GART_REQUIRE(h->lr > 0.0f && std::isfinite(h->lr), "lr must be above 0 and finite");
  GART_REQUIRE(h->momentum >= 0.0f && h->momentum < 1.0f, "momentum must be in [0, 1)");
  GART_REQUIRE(h->weight_decay >= 0.0f && std::isfinite(h->weight_decay), "weight_decay must be at least 0 and finite");
  GART_REQUIRE(h->scale > 0.0f && std::isfinite(h->scale), "scale must be above 0 and finite");
  GART_CHECK(check_steps(h->how));
  GART_CHECK(check_matrix("param", param, dtype, true));
  GART_CHECK(check_matrix("grad", grad, dtype, false));
  GART_CHECK(check_matrix("m", m, GART_DTYPE_F32, true));
  GART_REQUIRE(grad->rows == param->rows && grad->cols == param->cols, "grad and param differ in size");
  GART_REQUIRE(m->rows == param->rows && m->cols == param->cols, "m and param differ in size");
  if (param->rows == 0 || param->cols == 0) return GART_OK;
  const int64_t need = orthogonalize_scratch_bytes(param->rows, param->cols);
  if (need < 0) return fail(GART_ERR_UNSUPPORTED, "%lld x %lld", (long long)param->rows, (long long)param->cols);
  GART_CHECK(check_scratch(scratch, scratch_bytes, size_t(need)));
  const Span t[4] = {span_of(param, dtype), span_of(grad, dtype), span_of(m, GART_DTYPE_F32), span_of(scratch, need)};
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i; ++j) GART_REQUIRE(!overlap(t[i], t[j]), "param, grad, m and scratch overlap");
  OrthogonalizeArgs a{};
  a.rows = param->rows;
  a.cols = param->cols;
  a.a = h->how.a;
  a.b = h->how.b;
  a.c = h->how.c;
  a.eps = h->how.eps;
  a.steps = h->how.steps;
  a.x = grad->data;
  a.x_ld = grad->stride;
  a.m = static_cast<float*>(m->data);
  a.m_ld = m->stride;
  a.momentum = h->momentum;
  a.nesterov = h->nesterov != 0;
  a.y = param->data;
  a.y_ld = param->stride;
  a.decay = float(double(h->lr) * double(h->weight_decay));
  a.step = float(double(h->lr) * double(h->scale));
  a.scratch = scratch;
  GART_HIP(launch_orthogonalize(a, dtype, static_cast<hipStream_t>(stream)));
  return GART_OK;
}

}  // extern "C"
