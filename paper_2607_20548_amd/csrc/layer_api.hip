// C ABI of the operators around an expert bank and of dense layers: argument checks and
// launches of layer norm, router, MXFP4, heads' norm, gated feed-forward and distillation.
// Everything is enqueued on the caller's stream; nothing here allocates.
#include "soap.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "internal.h"

namespace {

using soap::api_fail;
using soap::api_ok;

struct Buf {
  const void *p;
  size_t bytes;
  const char *name;
  bool written;
  bool required;
  size_t align;
};

// Scales of a matrix inside a packed bank start at any row's, of eight bytes at least.
constexpr size_t MX4_SCALE_ALIGN = 8;

size_t elem(int dtype) { return dtype == SOAP_BF16 ? 2 : 4; }

// Bytes from the first to the last element of a strided matrix.
size_t span(int64_t rows, int64_t cols, int64_t ld, size_t e) {
  return rows > 0 && cols > 0 ? e * ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) : 0;
}

int check_dtype(int dtype) {
  if (dtype != SOAP_F32 && dtype != SOAP_BF16)
    return api_fail(SOAP_ERR_HPARAM, "dtype %d is neither SOAP_F32 nor SOAP_BF16", dtype);
  return SOAP_OK;
}

int check_range(const char *name, int64_t v, int64_t lo, int64_t hi) {
  if (v < lo || v > hi)
    return api_fail(SOAP_ERR_SHAPE, "%s = %lld is outside [%lld, %lld]", name, (long long)v,
                    (long long)lo, (long long)hi);
  return SOAP_OK;
}

int check_ld(const char *name, int64_t ld, int64_t cols) {
  if (ld < cols || ld > INT32_MAX)
    return api_fail(SOAP_ERR_SHAPE, "%s = %lld is outside [%lld, 2^31)", name, (long long)ld,
                    (long long)cols);
  return SOAP_OK;
}

// Required pointers (an empty buffer may be NULL), alignment, and no written
// buffer over another one.
int check_bufs(std::initializer_list<Buf> bufs) {
  for (const Buf &b : bufs)
    if (!b.p && b.required && b.bytes) return api_fail(SOAP_ERR_NULL, "%s is NULL", b.name);
  for (const Buf &b : bufs)
    if (b.p && reinterpret_cast<uintptr_t>(b.p) % b.align != 0)
      return api_fail(SOAP_ERR_ALIGN, "%s is not %zu-byte aligned", b.name, b.align);
  for (const Buf *x = bufs.begin(); x != bufs.end(); ++x)
    for (const Buf *y = x + 1; y != bufs.end(); ++y) {
      if (!x->p || !y->p || !x->bytes || !y->bytes || !(x->written || y->written)) continue;
      const char *a = static_cast<const char *>(x->p), *b = static_cast<const char *>(y->p);
      if (a < b + y->bytes && b < a + x->bytes)
        return api_fail(SOAP_ERR_ALIAS, "%s overlaps %s", x->name, y->name);
    }
  return SOAP_OK;
}

int check_workspace(size_t have, size_t need) {
  if (have < need)
    return api_fail(SOAP_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
  return SOAP_OK;
}

int done(hipError_t e, const char *what) {
  if (e != hipSuccess) return api_fail(SOAP_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return api_ok();
}

#define SOAP_TRY(call)                      \
  do {                                      \
    const int rc_ = (call);                 \
    if (rc_ != SOAP_OK) return rc_;         \
  } while (0)

int check_router(int64_t tokens, int64_t experts, int64_t top_k, int dtype, int64_t ld, uint32_t flags,
                 float balance) {
  SOAP_TRY(check_range("tokens", tokens, 0, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("experts", experts, 1, SOAP_ROUTER_MAX_EXPERTS));
  SOAP_TRY(check_range("top_k", top_k, 1, experts < SOAP_ROUTER_MAX_TOP_K ? experts : SOAP_ROUTER_MAX_TOP_K));
  SOAP_TRY(check_range("tokens top_k", tokens * top_k, 0, 1 << 30));
  SOAP_TRY(check_dtype(dtype));
  SOAP_TRY(check_ld("ld", ld, experts));
  if (flags & ~(uint32_t)SOAP_ROUTER_RENORMALIZE)
    return api_fail(SOAP_ERR_HPARAM, "unknown flag bits 0x%x", flags);
  if (!std::isfinite(balance) || balance < 0.f)
    return api_fail(SOAP_ERR_HPARAM, "balance = %g must be finite and >= 0", (double)balance);
  return SOAP_OK;
}

// Shared by the products; tile_groups: groups that have all M rows each; c_bytes: the
// range of C.
int check_product(int64_t groups, int64_t tile_groups, int64_t M, int64_t N, int64_t K, bool grouped,
                  const int32_t *offsets,
                  const uint8_t *ad, const uint8_t *as, int64_t b_rows, const uint8_t *bd,
                  const uint8_t *bs, int dtype, void *C, size_t c_bytes) {
  SOAP_TRY(check_dtype(dtype));
  SOAP_TRY(check_range("tiles of 128 x 128", (M / 128 * tile_groups + 4 * groups + 64) * ((N + 127) / 128), 0, INT32_MAX));
  return check_bufs({{offsets, grouped ? 4 * (size_t)(groups + 1) : 0, "offsets", false, true, 4},
                     {ad, soap_mx4_data_bytes(M, K), "a_data", false, true, 16},
                     {as, soap_mx4_scale_bytes(M, K), "a_scale", false, true, MX4_SCALE_ALIGN},
                     {bd, soap_mx4_data_bytes(b_rows, K), "b_data", false, true, 16},
                     {bs, soap_mx4_scale_bytes(b_rows, K), "b_scale", false, true, MX4_SCALE_ALIGN},
                     {C, c_bytes, "C", true, true, elem(dtype)}});
}

// A side of heads (queries or keys): bytes from its first to its last element.
size_t head_span(int64_t tokens, int64_t heads, int64_t dim, int64_t token, int64_t head, size_t e) {
  return tokens > 0 && heads > 0 ? e * ((size_t)(tokens - 1) * (size_t)token + (size_t)(heads - 1) * (size_t)head + (size_t)dim)
                                 : 0;
}

int check_strides(const char *name, int64_t tokens, int64_t heads, int64_t dim, int64_t token, int64_t head, bool written) {
  if (token < 0 || head < 0 || token > INT32_MAX || head > INT32_MAX)
    return api_fail(SOAP_ERR_SHAPE, "%s: strides %lld, %lld are outside [0, 2^31)", name, (long long)token, (long long)head);
  // heads of tokens, or tokens of heads, one behind the other
  const bool by_token = (heads <= 1 || head >= dim) && (tokens <= 1 || token >= (heads - 1) * head + dim);
  const bool by_head = (tokens <= 1 || token >= dim) && (heads <= 1 || head >= (tokens - 1) * token + dim);
  if (written && tokens > 0 && heads > 0 && !by_token && !by_head)
    return api_fail(SOAP_ERR_ALIAS, "%s: heads lie over each other (strides %lld, %lld)", name, (long long)token,
                    (long long)head);
  return SOAP_OK;
}

// Whether a head of one side meets one of the other, heads being `width` bytes, d + v s + u step
// apart with v in [first, last] and u in (-tokens, tokens).
bool heads_meet(int64_t d, int64_t s, int64_t first, int64_t last, int64_t step, int64_t tokens, int64_t width) {
  for (int64_t v = first; v <= last; ++v) {
    const int64_t x = d + v * s, u = step ? -x / step : 0;   // the nearest u are this one and its neighbours
    for (int64_t i = u - 1; i <= u + 1; ++i) {
      const int64_t at = x + std::min(std::max(i, 1 - tokens), tokens - 1) * step;
      if (at < width && -at < width) return true;
    }
  }
  return false;
}

// Two sides whose heads may lie between each other's (as queries and keys of a fused row do, or of
// rows in which they take turns), but not over each other.
int check_sides(const char *an, const void *a, int64_t ah, int64_t at, int64_t ahead, const char *bn, const void *b,
                int64_t bh, int64_t bt, int64_t bhead, int64_t tokens, int64_t dim, size_t e) {
  const int64_t as = (int64_t)head_span(tokens, ah, dim, at, ahead, e), bs = (int64_t)head_span(tokens, bh, dim, bt, bhead, e);
  if (!a || !b || !as || !bs) return SOAP_OK;
  const int64_t d = (int64_t)(reinterpret_cast<intptr_t>(b) - reinterpret_cast<intptr_t>(a));
  if (d >= as || -d >= bs) return SOAP_OK;
  const int64_t step = (int64_t)e * at;
  if (at == bt && step > 0) {
    const int64_t ra = (int64_t)e * ((ah - 1) * ahead + dim), rb = (int64_t)e * ((bh - 1) * bhead + dim);
    const int64_t r = (d % step + step) % step;
    if (r >= ra && r + rb <= step) return SOAP_OK;
  }
  if ((at == bt || tokens == 1) && (ahead == bhead || ah == 1 || bh == 1)) {
    const int64_t s = (int64_t)e * (ah == 1 ? bhead : ahead);
    if (!heads_meet(d, s, 1 - ah, bh - 1, tokens == 1 ? 0 : step, tokens, (int64_t)e * dim)) return SOAP_OK;
  }
  return api_fail(SOAP_ERR_ALIAS, "%s overlaps %s", bn, an);
}

int check_heads(int64_t tokens, int64_t q_heads, int64_t k_heads, int64_t dim, int64_t rotary, int dtype, uint32_t flags,
                float eps) {
  SOAP_TRY(check_range("tokens", tokens, 0, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("q_heads", q_heads, 0, SOAP_HEAD_MAX_HEADS));
  SOAP_TRY(check_range("k_heads", k_heads, 0, SOAP_HEAD_MAX_HEADS));
  SOAP_TRY(check_range("dim", dim, 2, SOAP_HEAD_MAX_DIM));
  SOAP_TRY(check_range("rotary", rotary, 0, dim));
  if (dim % 2 || rotary % 2) return api_fail(SOAP_ERR_SHAPE, "dim = %lld and rotary = %lld must be even", (long long)dim, (long long)rotary);
  SOAP_TRY(check_dtype(dtype));
  if (flags & ~(uint32_t)SOAP_HEAD_INTERLEAVED) return api_fail(SOAP_ERR_HPARAM, "unknown flag bits 0x%x", flags);
  if (!std::isfinite(eps) || eps <= 0.f) return api_fail(SOAP_ERR_HPARAM, "eps = %g must be finite and > 0", (double)eps);
  return SOAP_OK;
}

int check_gated(int64_t tokens, int64_t m, int64_t n, int64_t p, int activation) {
  SOAP_TRY(check_range("tokens", tokens, 0, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("m", m, 8, SOAP_MAX_DIM));
  SOAP_TRY(check_range("n", n, 8, SOAP_GATED_MAX_HIDDEN));
  SOAP_TRY(check_range("p", p, 8, SOAP_MAX_DIM));
  if (m % 8 || n % 8 || p % 8)
    return api_fail(SOAP_ERR_SHAPE, "m = %lld, n = %lld and p = %lld must be multiples of 8", (long long)m, (long long)n, (long long)p);
  if (activation != SOAP_ACT_SILU && activation != SOAP_ACT_GELU)
    return api_fail(SOAP_ERR_HPARAM, "activation %d is neither SOAP_ACT_SILU nor SOAP_ACT_GELU", activation);
  return SOAP_OK;
}

// Rows that a product reads or writes 16 bytes at a time.
int check_ld8(const char *name, int64_t ld, int64_t cols) {
  if (ld < cols || ld > SOAP_GATED_MAX_LD || ld % 8)
    return api_fail(SOAP_ERR_SHAPE, "%s = %lld is no multiple of 8 in [%lld, %d]", name, (long long)ld, (long long)cols,
                    SOAP_GATED_MAX_LD);
  return SOAP_OK;
}

int check_distill(int64_t rows, int64_t classes, int64_t slots, int dtype, int64_t ld, int64_t ldi, int teacher_dtype,
                  int64_t ldt, uint32_t flags, float temperature) {
  SOAP_TRY(check_range("rows", rows, 0, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("classes", classes, 1, SOAP_DISTILL_MAX_CLASSES));
  SOAP_TRY(check_range("slots", slots, 1, SOAP_DISTILL_MAX_SLOTS));
  SOAP_TRY(check_dtype(dtype));
  SOAP_TRY(check_dtype(teacher_dtype));
  SOAP_TRY(check_ld("ld", ld, classes));
  SOAP_TRY(check_ld("ldi", ldi, slots));
  SOAP_TRY(check_ld("ldt", ldt, slots));
  if (flags & ~(uint32_t)(SOAP_DISTILL_TAIL | SOAP_DISTILL_SUMS)) return api_fail(SOAP_ERR_HPARAM, "unknown flag bits 0x%x", flags);
  if (!(temperature >= SOAP_DISTILL_MIN_TEMPERATURE && temperature <= SOAP_DISTILL_MAX_TEMPERATURE))
    return api_fail(SOAP_ERR_HPARAM, "temperature = %g is outside [%g, %g]", (double)temperature,
                    SOAP_DISTILL_MIN_TEMPERATURE, SOAP_DISTILL_MAX_TEMPERATURE);
  return SOAP_OK;
}

size_t stats_bytes(int64_t rows, uint32_t flags) { return (flags & SOAP_DISTILL_SUMS ? 24 : 8) * (size_t)rows; }

soap::DistillDesc distill_desc(int64_t rows, int64_t classes, int64_t slots, int dtype, const void *logits, int64_t ld,
                               const int32_t *index, int64_t ldi, int teacher_dtype, const void *teacher, int64_t ldt,
                               uint32_t flags, float temperature) {
  soap::DistillDesc d;
  d.rows = rows; d.classes = classes; d.slots = slots; d.ld = ld; d.ldi = ldi; d.ldt = ldt;
  d.bf16 = dtype == SOAP_BF16; d.teacher_bf16 = teacher_dtype == SOAP_BF16; d.tail = flags & SOAP_DISTILL_TAIL;
  d.sums = flags & SOAP_DISTILL_SUMS;
  d.tau = temperature; d.logits = logits; d.index = index; d.teacher = teacher;
  return d;
}

}  // namespace

extern "C" {

// ------------------------------------------------------------- layer norm
int soap_layer_norm_forward(int64_t rows, int64_t cols, int dtype, const void *x, int64_t ldx,
                            const float *weight, const float *bias, float eps, void *y, int64_t ldy,
                            float *mean, float *rstd, hipStream_t stream) {
  SOAP_TRY(check_range("rows", rows, 0, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("cols", cols, 1, SOAP_MAX_DIM));
  SOAP_TRY(check_dtype(dtype));
  SOAP_TRY(check_ld("ldx", ldx, cols));
  SOAP_TRY(check_ld("ldy", ldy, cols));
  if (!std::isfinite(eps) || eps <= 0.f)
    return api_fail(SOAP_ERR_HPARAM, "eps = %g must be finite and > 0", (double)eps);
  const size_t e = elem(dtype), pc = 4 * (size_t)cols, pr = 4 * (size_t)rows;
  SOAP_TRY(check_bufs({{x, span(rows, cols, ldx, e), "x", false, true, e},
                       {weight, pc, "weight", false, false, 4},
                       {bias, pc, "bias", false, false, 4},
                       {y, span(rows, cols, ldy, e), "y", true, true, e},
                       {mean, pr, "mean", true, false, 4},
                       {rstd, pr, "rstd", true, false, 4}}));
  soap::LayerNormDesc d;
  d.rows = rows; d.cols = cols; d.bf16 = dtype == SOAP_BF16;
  d.x = x; d.ldx = ldx; d.weight = weight; d.bias = bias; d.eps = eps;
  d.out = y; d.ldo = ldy; d.mean = mean; d.rstd = rstd;
  return done(soap::launch_layer_norm_fwd(d, stream), "layer norm");
}

size_t soap_layer_norm_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || rows > SOAP_MAX_ROWS || cols < 1 || cols > SOAP_MAX_DIM) return 0;
  return soap::layer_norm_part_bytes(rows, cols);
}

int soap_layer_norm_backward(int64_t rows, int64_t cols, int dtype, const void *dy, int64_t lddy,
                             const void *x, int64_t ldx, const float *weight, const float *mean,
                             const float *rstd, void *dx, int64_t lddx, float *dweight, float *dbias,
                             void *workspace, size_t workspace_bytes, hipStream_t stream) {
  SOAP_TRY(check_range("rows", rows, 0, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("cols", cols, 1, SOAP_MAX_DIM));
  SOAP_TRY(check_dtype(dtype));
  SOAP_TRY(check_ld("lddy", lddy, cols));
  SOAP_TRY(check_ld("ldx", ldx, cols));
  if (dx) SOAP_TRY(check_ld("lddx", lddx, cols));
  const size_t e = elem(dtype), pc = 4 * (size_t)cols, pr = 4 * (size_t)rows;
  const size_t need = dweight || dbias ? soap::layer_norm_part_bytes(rows, cols) : 0;
  SOAP_TRY(check_bufs({{dy, span(rows, cols, lddy, e), "dy", false, true, e},
                       {x, span(rows, cols, ldx, e), "x", false, true, e},
                       {weight, pc, "weight", false, false, 4},
                       {mean, pr, "mean", false, true, 4},
                       {rstd, pr, "rstd", false, true, 4},
                       {dx, dx ? span(rows, cols, lddx, e) : 0, "dx", true, false, e},
                       {dweight, pc, "dweight", true, false, 4},
                       {dbias, pc, "dbias", true, false, 4},
                       {workspace, need, "workspace", true, true, 16}}));
  SOAP_TRY(check_workspace(workspace_bytes, need));
  soap::LayerNormDesc d;
  d.rows = rows; d.cols = cols; d.bf16 = dtype == SOAP_BF16;
  d.dy = dy; d.lddy = lddy; d.x = x; d.ldx = ldx; d.weight = weight;
  d.mean = const_cast<float *>(mean); d.rstd = const_cast<float *>(rstd);
  d.out = dx; d.ldo = lddx; d.dweight = dweight; d.dbias = dbias;
  d.part = static_cast<float *>(workspace);
  return done(soap::launch_layer_norm_bwd(d, stream), "layer norm backward");
}

// ----------------------------------------------------------------- router
int64_t soap_router_rows(int64_t tokens, int64_t experts, int64_t top_k) {
  if (tokens < 0 || tokens > SOAP_MAX_ROWS || experts < 1 || experts > SOAP_ROUTER_MAX_EXPERTS ||
      top_k < 1 || top_k > experts || top_k > SOAP_ROUTER_MAX_TOP_K || tokens * top_k > 1 << 30)
    return 0;
  const int64_t n = tokens * top_k;
  return (n + 31 * (n < experts ? n : experts) + 31) / 32 * 32;
}

size_t soap_router_workspace_bytes(int64_t tokens, int64_t experts) {
  if (tokens < 0 || tokens > SOAP_MAX_ROWS || experts < 1 || experts > SOAP_ROUTER_MAX_EXPERTS) return 0;
  return soap::router_scratch_bytes(tokens, experts);
}

int soap_router_forward(int64_t tokens, int64_t experts, int64_t top_k, int dtype, const void *logits,
                        int64_t ld, const uint8_t *token_mask, uint32_t flags, float balance,
                        int32_t *index, float *gate, int32_t *counts, float *loss, int32_t *offsets,
                        int32_t *position, int32_t *row_token, void *workspace, size_t workspace_bytes,
                        hipStream_t stream) {
  SOAP_TRY(check_router(tokens, experts, top_k, dtype, ld, flags, balance));
  const int64_t rows = soap_router_rows(tokens, experts, top_k);
  const size_t e = elem(dtype), tk = 4 * (size_t)(tokens * top_k), pe = 4 * (size_t)(experts + 1);
  const bool plan = offsets || position || row_token;
  const size_t need = soap::router_scratch_bytes(tokens, experts);
  SOAP_TRY(check_bufs({{logits, span(tokens, experts, ld, e), "logits", false, true, e},
                       {token_mask, (size_t)tokens, "token_mask", false, false, 1},
                       {index, tk, "index", true, true, 4},
                       {gate, tk, "gate", true, true, 4},
                       {counts, pe, "counts", true, true, 4},
                       {loss, 4, "loss", true, false, 4},
                       {offsets, pe, "offsets", true, plan, 4},
                       {position, tk, "position", true, plan, 4},
                       {row_token, 4 * (size_t)rows, "row_token", true, plan, 4},
                       {workspace, need, "workspace", true, true, 16}}));
  SOAP_TRY(check_workspace(workspace_bytes, need));
  soap::RouterDesc d;
  d.tokens = tokens; d.experts = experts; d.top_k = top_k; d.ld = ld; d.rows = rows;
  d.bf16 = dtype == SOAP_BF16; d.renorm = flags & SOAP_ROUTER_RENORMALIZE ? 1 : 0;
  d.balance = balance; d.logits = logits; d.mask = token_mask;
  d.index = index; d.gate = gate; d.counts = counts; d.loss = loss;
  d.offsets = offsets; d.position = position; d.row_token = row_token;
  d.scratch = workspace;
  return done(soap::launch_router_fwd(d, stream), "router");
}

int soap_router_backward(int64_t tokens, int64_t experts, int64_t top_k, int dtype, const void *logits,
                         int64_t ld, const uint8_t *token_mask, uint32_t flags, float balance,
                         const int32_t *index, const int32_t *counts, const float *dgate,
                         const float *dloss, void *dlogits, int64_t ldd, hipStream_t stream) {
  SOAP_TRY(check_router(tokens, experts, top_k, dtype, ld, flags, balance));
  SOAP_TRY(check_ld("ldd", ldd, experts));
  const size_t e = elem(dtype), tk = 4 * (size_t)(tokens * top_k), pe = 4 * (size_t)(experts + 1);
  SOAP_TRY(check_bufs({{logits, span(tokens, experts, ld, e), "logits", false, true, e},
                       {token_mask, (size_t)tokens, "token_mask", false, false, 1},
                       {index, tk, "index", false, true, 4},
                       {counts, pe, "counts", false, true, 4},
                       {dgate, tk, "dgate", false, false, 4},
                       {dloss, 4, "dloss", false, false, 4},
                       {dlogits, span(tokens, experts, ldd, e), "dlogits", true, true, e}}));
  soap::RouterDesc d;
  d.tokens = tokens; d.experts = experts; d.top_k = top_k; d.ld = ld; d.ldd = ldd;
  d.bf16 = dtype == SOAP_BF16; d.renorm = flags & SOAP_ROUTER_RENORMALIZE ? 1 : 0;
  d.balance = balance; d.logits = logits; d.mask = token_mask;
  d.index = const_cast<int32_t *>(index); d.counts = const_cast<int32_t *>(counts);
  d.dgate = dgate; d.dloss = dloss; d.dlogits = dlogits;
  return done(soap::launch_router_bwd(d, stream), "router backward");
}

// ------------------------------------------------------------------ MXFP4
size_t soap_mx4_data_bytes(int64_t rows, int64_t k) {
  if (rows < 0 || k < 0) return 0;
  return (size_t)rows * (size_t)(soap::mx4_padded(k) / 2);
}

size_t soap_mx4_scale_bytes(int64_t rows, int64_t k) {
  if (rows < 0 || k < 0) return 0;
  return (size_t)rows * (size_t)(soap::mx4_padded(k) / 32);
}

int soap_mx4_quantize(int64_t batch, int64_t rows, int64_t cols, int dtype, const void *x, int64_t ldx,
                      const int32_t *row_index, int64_t x_rows, uint8_t *data, uint8_t *scale,
                      uint8_t *data_t, uint8_t *scale_t, hipStream_t stream) {
  SOAP_TRY(check_range("batch", batch, 1, SOAP_MAX_DIM));
  SOAP_TRY(check_range("rows", rows, 0, INT32_MAX));
  SOAP_TRY(check_range("cols", cols, 1, SOAP_MAX_ROWS));
  SOAP_TRY(check_dtype(dtype));
  SOAP_TRY(check_ld("ldx", ldx, cols));
  SOAP_TRY(check_range("tiles of 128 x 256", (rows + 255) / 128 * ((cols + 255) / 256), 0, INT32_MAX));
  if (row_index) {
    SOAP_TRY(check_range("batch with row_index", batch, 1, 1));
    SOAP_TRY(check_range("x_rows", x_rows, 0, SOAP_MAX_ROWS));
  } else {
    x_rows = rows;
  }
  if (!data != !scale || !data_t != !scale_t)
    return api_fail(SOAP_ERR_NULL, "data and scale (data_t and scale_t) come together");
  if (!data && !data_t && rows > 0) return api_fail(SOAP_ERR_NULL, "no output is wanted");
  const size_t e = elem(dtype), b = (size_t)batch;
  SOAP_TRY(check_bufs({{x, span(row_index ? x_rows : batch * rows, cols, ldx, e), "x", false, true, e},
                       {row_index, 4 * (size_t)rows, "row_index", false, false, 4},
                       {data, b * soap_mx4_data_bytes(rows, cols), "data", true, false, 16},
                       {scale, b * soap_mx4_scale_bytes(rows, cols), "scale", true, false, MX4_SCALE_ALIGN},
                       {data_t, b * soap_mx4_data_bytes(cols, rows), "data_t", true, false, 16},
                       {scale_t, b * soap_mx4_scale_bytes(cols, rows), "scale_t", true, false, MX4_SCALE_ALIGN}}));
  soap::Mx4QuantDesc d;
  d.batch = batch; d.rows = rows; d.cols = cols; d.ldx = ldx; d.x_rows = x_rows;
  d.bf16 = dtype == SOAP_BF16; d.x = x; d.row_index = row_index;
  d.data = data; d.scale = scale; d.data_t = data_t; d.scale_t = scale_t;
  return done(soap::launch_mx4_quantize(d, stream), "MXFP4 quantisation");
}

int soap_mx4_gather(int64_t rows, int64_t k, const int32_t *row_index, int64_t x_rows,
                    const uint8_t *x_data, const uint8_t *x_scale, uint8_t *data, uint8_t *scale,
                    hipStream_t stream) {
  SOAP_TRY(check_range("rows", rows, 0, INT32_MAX));
  SOAP_TRY(check_range("k", k, 1, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("x_rows", x_rows, 0, INT32_MAX));
  SOAP_TRY(check_bufs({{row_index, 4 * (size_t)rows, "row_index", false, true, 4},
                       {x_data, soap_mx4_data_bytes(x_rows, k), "x_data", false, true, 16},
                       {x_scale, soap_mx4_scale_bytes(x_rows, k), "x_scale", false, true, MX4_SCALE_ALIGN},
                       {data, soap_mx4_data_bytes(rows, k), "data", true, true, 16},
                       {scale, soap_mx4_scale_bytes(rows, k), "scale", true, true, MX4_SCALE_ALIGN}}));
  return done(soap::launch_mx4_gather({x_data, x_scale}, x_rows, row_index, rows, k, data, scale, stream),
              "MXFP4 rows");
}

int soap_mx4_dequantize(int64_t rows, int64_t k, const uint8_t *data, const uint8_t *scale, int dtype,
                        void *out, int64_t ldo, hipStream_t stream) {
  SOAP_TRY(check_range("rows", rows, 0, INT32_MAX));
  SOAP_TRY(check_range("k", k, 1, SOAP_MAX_ROWS));
  SOAP_TRY(check_dtype(dtype));
  SOAP_TRY(check_ld("ldo", ldo, k));
  const size_t e = elem(dtype);
  SOAP_TRY(check_bufs({{data, soap_mx4_data_bytes(rows, k), "data", false, true, 16},
                       {scale, soap_mx4_scale_bytes(rows, k), "scale", false, true, MX4_SCALE_ALIGN},
                       {out, span(rows, k, ldo, e), "out", true, true, e}}));
  return done(soap::launch_mx4_dequantize({data, scale}, rows, k, dtype == SOAP_BF16, out, ldo, stream),
              "MXFP4 values");
}

int soap_mx4_gemm(int64_t M, int64_t N, int64_t K, const uint8_t *a_data, const uint8_t *a_scale,
                  const uint8_t *b_data, const uint8_t *b_scale, int dtype, void *C, int64_t ldc,
                  hipStream_t stream) {
  SOAP_TRY(check_range("M", M, 0, INT32_MAX));
  SOAP_TRY(check_range("N", N, 1, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("K", K, 1, SOAP_MAX_ROWS));
  SOAP_TRY(check_ld("ldc", ldc, N));
  SOAP_TRY(check_product(1, 1, M, N, K, false, nullptr, a_data, a_scale, N, b_data, b_scale, dtype, C,
                         span(M, N, ldc, elem(dtype))));
  soap::Mx4GemmDesc d;
  d.M = M; d.N = N; d.K = K; d.ldc = ldc; d.bf16 = dtype == SOAP_BF16;
  d.A = {a_data, a_scale}; d.B = {b_data, b_scale}; d.C = C;
  return done(soap::launch_mx4_gemm(d, stream), "MXFP4 product");
}

int soap_mx4_gemm_rows(int64_t groups, int64_t M, int64_t N, int64_t K, const int32_t *offsets,
                       const uint8_t *a_data, const uint8_t *a_scale, const uint8_t *b_data,
                       const uint8_t *b_scale, int dtype, void *C, int64_t ldc, hipStream_t stream) {
  SOAP_TRY(check_range("groups", groups, 1, SOAP_MAX_DIM));
  SOAP_TRY(check_range("M", M, 0, INT32_MAX));
  SOAP_TRY(check_range("N", N, 1, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("K", K, 1, SOAP_MAX_ROWS));
  SOAP_TRY(check_ld("ldc", ldc, N));
  SOAP_TRY(check_product(groups, 1, M, N, K, true, offsets, a_data, a_scale, groups * N, b_data, b_scale,
                         dtype, C, span(M, N, ldc, elem(dtype))));
  soap::Mx4GemmDesc d;
  d.groups = groups; d.M = M; d.N = N; d.K = K; d.ldc = ldc; d.bf16 = dtype == SOAP_BF16;
  d.offsets = offsets; d.A = {a_data, a_scale}; d.B = {b_data, b_scale}; d.C = C;
  return done(soap::launch_mx4_gemm(d, stream), "MXFP4 product by rows");
}

int soap_mx4_gemm_k(int64_t groups, int64_t M, int64_t N, int64_t K, const int32_t *offsets,
                    const uint8_t *a_data, const uint8_t *a_scale, const uint8_t *b_data,
                    const uint8_t *b_scale, int dtype, void *C, hipStream_t stream) {
  SOAP_TRY(check_range("groups", groups, 1, SOAP_MAX_DIM));
  SOAP_TRY(check_range("M", M, 1, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("N", N, 1, SOAP_MAX_ROWS));
  SOAP_TRY(check_range("K", K, 0, 2 * SOAP_MAX_ROWS));
  SOAP_TRY(check_product(groups, groups, M, N, K, true, offsets, a_data, a_scale, N, b_data, b_scale, dtype, C,
                         elem(dtype) * (size_t)groups * (size_t)M * (size_t)N));
  soap::Mx4GemmDesc d;
  d.groups = groups; d.M = M; d.N = N; d.K = K; d.ldc = N; d.by_k = true; d.bf16 = dtype == SOAP_BF16;
  d.offsets = offsets; d.A = {a_data, a_scale}; d.B = {b_data, b_scale}; d.C = C;
  return done(soap::launch_mx4_gemm(d, stream), "MXFP4 product by k");
}

// ------------------------------------------------- heads' norm and rotation
int soap_head_norm_forward(int64_t tokens, int64_t q_heads, int64_t k_heads, int64_t dim, int64_t rotary, int dtype,
                           uint32_t flags, const void *q, int64_t q_token, int64_t q_head, const void *k,
                           int64_t k_token, int64_t k_head, const float *q_weight, const float *k_weight, float eps,
                           const int32_t *positions, const double *frequencies, void *q_out, int64_t q_out_token,
                           int64_t q_out_head, void *k_out, int64_t k_out_token, int64_t k_out_head,
                           hipStream_t stream) {
  SOAP_TRY(check_heads(tokens, q_heads, k_heads, dim, rotary, dtype, flags, eps));
  SOAP_TRY(check_strides("q", tokens, q_heads, dim, q_token, q_head, false));
  SOAP_TRY(check_strides("k", tokens, k_heads, dim, k_token, k_head, false));
  SOAP_TRY(check_strides("q_out", tokens, q_heads, dim, q_out_token, q_out_head, true));
  SOAP_TRY(check_strides("k_out", tokens, k_heads, dim, k_out_token, k_out_head, true));
  const size_t e = elem(dtype), pd = 4 * (size_t)dim;
  // queries and keys lie between each other in a token's row, as their outputs may: only a
  // side's own input and output are held apart by range, the others by their rows
  SOAP_TRY(check_bufs({{q, head_span(tokens, q_heads, dim, q_token, q_head, e), "q", false, true, e},
                       {q_weight, pd, "q_weight", false, false, 4},
                       {k_weight, pd, "k_weight", false, false, 4},
                       {positions, 4 * (size_t)tokens, "positions", false, false, 4},
                       {frequencies, 4 * (size_t)rotary, "frequencies", false, rotary > 0, 8},
                       {q_out, head_span(tokens, q_heads, dim, q_out_token, q_out_head, e), "q_out", true, true, e}}));
  SOAP_TRY(check_bufs({{k, head_span(tokens, k_heads, dim, k_token, k_head, e), "k", false, true, e},
                       {q_weight, pd, "q_weight", false, false, 4},
                       {k_weight, pd, "k_weight", false, false, 4},
                       {positions, 4 * (size_t)tokens, "positions", false, false, 4},
                       {frequencies, 4 * (size_t)rotary, "frequencies", false, rotary > 0, 8},
                       {k_out, head_span(tokens, k_heads, dim, k_out_token, k_out_head, e), "k_out", true, true, e}}));
  SOAP_TRY(check_sides("k", k, k_heads, k_token, k_head, "q_out", q_out, q_heads, q_out_token, q_out_head, tokens, dim, e));
  SOAP_TRY(check_sides("q", q, q_heads, q_token, q_head, "k_out", k_out, k_heads, k_out_token, k_out_head, tokens, dim, e));
  SOAP_TRY(check_sides("k_out", k_out, k_heads, k_out_token, k_out_head, "q_out", q_out, q_heads, q_out_token, q_out_head,
                       tokens, dim, e));
  soap::HeadNormDesc d;
  d.tokens = tokens; d.dim = dim; d.rotary = rotary; d.bf16 = dtype == SOAP_BF16; d.near = flags & SOAP_HEAD_INTERLEAVED;
  d.eps = eps; d.positions = positions; d.frequencies = frequencies;
  soap::HeadNormSide &a = d.side[0], &b = d.side[1];
  a.heads = q_heads; a.x = q; a.x_token = q_token; a.x_head = q_head; a.weight = q_weight;
  a.out = q_out; a.out_token = q_out_token; a.out_head = q_out_head;
  b.heads = k_heads; b.x = k; b.x_token = k_token; b.x_head = k_head; b.weight = k_weight;
  b.out = k_out; b.out_token = k_out_token; b.out_head = k_out_head;
  return done(soap::launch_head_norm_fwd(d, stream), "heads' norm");
}

size_t soap_head_norm_workspace_bytes(int64_t tokens, int64_t dim) {
  if (tokens < 0 || tokens > SOAP_MAX_ROWS || dim < 2 || dim > SOAP_HEAD_MAX_DIM) return 0;
  return soap::head_norm_part_bytes(tokens, dim);
}

int soap_head_norm_backward(int64_t tokens, int64_t q_heads, int64_t k_heads, int64_t dim, int64_t rotary, int dtype,
                            uint32_t flags, const void *dq_out, int64_t dq_out_token, int64_t dq_out_head,
                            const void *dk_out, int64_t dk_out_token, int64_t dk_out_head, const void *q, int64_t q_token,
                            int64_t q_head, const void *k, int64_t k_token, int64_t k_head, const float *q_weight,
                            const float *k_weight, float eps, const int32_t *positions, const double *frequencies,
                            void *dq, int64_t dq_token, int64_t dq_head, void *dk, int64_t dk_token, int64_t dk_head,
                            float *dq_weight, float *dk_weight, void *workspace, size_t workspace_bytes,
                            hipStream_t stream) {
  SOAP_TRY(check_heads(tokens, q_heads, k_heads, dim, rotary, dtype, flags, eps));
  SOAP_TRY(check_strides("dq_out", tokens, q_heads, dim, dq_out_token, dq_out_head, false));
  SOAP_TRY(check_strides("dk_out", tokens, k_heads, dim, dk_out_token, dk_out_head, false));
  SOAP_TRY(check_strides("q", tokens, q_heads, dim, q_token, q_head, false));
  SOAP_TRY(check_strides("k", tokens, k_heads, dim, k_token, k_head, false));
  if (dq) SOAP_TRY(check_strides("dq", tokens, q_heads, dim, dq_token, dq_head, true));
  if (dk) SOAP_TRY(check_strides("dk", tokens, k_heads, dim, dk_token, dk_head, true));
  const size_t e = elem(dtype), pd = 4 * (size_t)dim;
  const size_t need = dq_weight || dk_weight ? soap::head_norm_part_bytes(tokens, dim) : 0;
  for (int side = 0; side < 2; ++side) {
    const int64_t heads = side ? k_heads : q_heads;
    const size_t in = side ? head_span(tokens, heads, dim, k_token, k_head, e) : head_span(tokens, heads, dim, q_token, q_head, e);
    const size_t din = side ? head_span(tokens, heads, dim, dk_out_token, dk_out_head, e)
                            : head_span(tokens, heads, dim, dq_out_token, dq_out_head, e);
    const size_t out = side ? (dk ? head_span(tokens, heads, dim, dk_token, dk_head, e) : 0)
                            : (dq ? head_span(tokens, heads, dim, dq_token, dq_head, e) : 0);
    SOAP_TRY(check_bufs({{side ? dk_out : dq_out, din, side ? "dk_out" : "dq_out", false, true, e},
                         {side ? k : q, in, side ? "k" : "q", false, true, e},
                         {q_weight, pd, "q_weight", false, false, 4},
                         {k_weight, pd, "k_weight", false, false, 4},
                         {positions, 4 * (size_t)tokens, "positions", false, false, 4},
                         {frequencies, 4 * (size_t)rotary, "frequencies", false, rotary > 0, 8},
                         {side ? dk : dq, out, side ? "dk" : "dq", true, false, e},
                         {dq_weight, pd, "dq_weight", true, false, 4},
                         {dk_weight, pd, "dk_weight", true, false, 4},
                         {workspace, need, "workspace", true, true, 16}}));
  }
  SOAP_TRY(check_sides("k", k, k_heads, k_token, k_head, "dq", dq, q_heads, dq_token, dq_head, tokens, dim, e));
  SOAP_TRY(check_sides("dk_out", dk_out, k_heads, dk_out_token, dk_out_head, "dq", dq, q_heads, dq_token, dq_head, tokens, dim, e));
  SOAP_TRY(check_sides("q", q, q_heads, q_token, q_head, "dk", dk, k_heads, dk_token, dk_head, tokens, dim, e));
  SOAP_TRY(check_sides("dq_out", dq_out, q_heads, dq_out_token, dq_out_head, "dk", dk, k_heads, dk_token, dk_head, tokens, dim, e));
  SOAP_TRY(check_sides("dk", dk, k_heads, dk_token, dk_head, "dq", dq, q_heads, dq_token, dq_head, tokens, dim, e));
  SOAP_TRY(check_workspace(workspace_bytes, need));
  soap::HeadNormDesc d;
  d.tokens = tokens; d.dim = dim; d.rotary = rotary; d.bf16 = dtype == SOAP_BF16; d.near = flags & SOAP_HEAD_INTERLEAVED;
  d.eps = eps; d.positions = positions; d.frequencies = frequencies; d.part = static_cast<float *>(workspace);
  soap::HeadNormSide &a = d.side[0], &b = d.side[1];
  a.heads = q_heads; a.x = q; a.x_token = q_token; a.x_head = q_head; a.weight = q_weight; a.dweight = dq_weight;
  a.dy = dq_out; a.dy_token = dq_out_token; a.dy_head = dq_out_head; a.out = dq; a.out_token = dq_token; a.out_head = dq_head;
  b.heads = k_heads; b.x = k; b.x_token = k_token; b.x_head = k_head; b.weight = k_weight; b.dweight = dk_weight;
  b.dy = dk_out; b.dy_token = dk_out_token; b.dy_head = dk_out_head; b.out = dk; b.out_token = dk_token; b.out_head = dk_head;
  return done(soap::launch_head_norm_bwd(d, stream), "heads' norm backward");
}

// ------------------------------------------------- gated feed-forward block
size_t soap_gated_workspace_bytes(int64_t tokens, int64_t m, int64_t n, int64_t p, int backward) {
  if (check_gated(tokens, m, n, p, SOAP_ACT_SILU) != SOAP_OK) return 0;
  return soap::gated_workspace_bytes(tokens, m, n, p, backward != 0);
}

int soap_gated_forward(int64_t tokens, int64_t m, int64_t n, int64_t p, int activation, const void *x, int64_t ldx,
                       const void *w_gate, const void *w_up, const void *w_down, void *gate, void *up, void *y,
                       int64_t ldy, void *workspace, size_t workspace_bytes, hipStream_t stream) {
  SOAP_TRY(check_gated(tokens, m, n, p, activation));
  SOAP_TRY(check_ld8("ldx", ldx, m));
  SOAP_TRY(check_ld8("ldy", ldy, p));
  if (!gate != !up) return api_fail(SOAP_ERR_NULL, "gate and up come together");
  const size_t tn = 2 * (size_t)tokens * (size_t)n, need = soap::gated_workspace_bytes(tokens, m, n, p, false);
  SOAP_TRY(check_bufs({{x, span(tokens, m, ldx, 2), "x", false, true, 16},
                       {w_gate, 2 * (size_t)m * (size_t)n, "w_gate", false, true, 16},
                       {w_up, 2 * (size_t)m * (size_t)n, "w_up", false, true, 16},
                       {w_down, 2 * (size_t)n * (size_t)p, "w_down", false, true, 16},
                       {gate, tn, "gate", true, false, 16},
                       {up, tn, "up", true, false, 16},
                       {y, span(tokens, p, ldy, 2), "y", true, true, 16},
                       {workspace, need, "workspace", true, true, 16}}));
  SOAP_TRY(check_workspace(workspace_bytes, need));
  soap::GatedDesc d;
  d.tokens = tokens; d.m = m; d.n = n; d.p = p; d.ldx = ldx; d.ldy = ldy; d.act = activation;
  d.x = static_cast<const uint16_t *>(x); d.w_gate = static_cast<const uint16_t *>(w_gate);
  d.w_up = static_cast<const uint16_t *>(w_up); d.w_down = static_cast<const uint16_t *>(w_down);
  d.gate = static_cast<uint16_t *>(gate); d.up = static_cast<uint16_t *>(up); d.y = static_cast<uint16_t *>(y);
  d.workspace = workspace;
  return done(soap::launch_gated_fwd(d, stream), "gated feed-forward");
}

int soap_gated_backward(int64_t tokens, int64_t m, int64_t n, int64_t p, int activation, const void *dy, int64_t lddy,
                        const void *x, int64_t ldx, const void *w_gate, const void *w_up, const void *w_down,
                        const void *gate, const void *up, void *dx, int64_t lddx, int grad_dtype, void *dw_gate,
                        void *dw_up, void *dw_down, void *workspace, size_t workspace_bytes, hipStream_t stream) {
  SOAP_TRY(check_gated(tokens, m, n, p, activation));
  SOAP_TRY(check_dtype(grad_dtype));
  SOAP_TRY(check_ld8("lddy", lddy, p));
  SOAP_TRY(check_ld8("ldx", ldx, m));
  if (dx) SOAP_TRY(check_ld8("lddx", lddx, m));
  const size_t tn = 2 * (size_t)tokens * (size_t)n, need = soap::gated_workspace_bytes(tokens, m, n, p, true);
  const size_t mn = (size_t)m * (size_t)n, np = (size_t)n * (size_t)p, e = elem(grad_dtype);
  SOAP_TRY(check_bufs({{dy, span(tokens, p, lddy, 2), "dy", false, true, 16},
                       {x, span(tokens, m, ldx, 2), "x", false, true, 16},
                       {w_gate, 2 * mn, "w_gate", false, true, 16},
                       {w_up, 2 * mn, "w_up", false, true, 16},
                       {w_down, 2 * np, "w_down", false, true, 16},
                       {gate, tn, "gate", false, true, 16},
                       {up, tn, "up", false, true, 16},
                       {dx, dx ? span(tokens, m, lddx, 2) : 0, "dx", true, false, 16},
                       {dw_gate, e * mn, "dw_gate", true, false, 16},
                       {dw_up, e * mn, "dw_up", true, false, 16},
                       {dw_down, e * np, "dw_down", true, false, 16},
                       {workspace, need, "workspace", true, true, 16}}));
  SOAP_TRY(check_workspace(workspace_bytes, need));
  soap::GatedDesc d;
  d.tokens = tokens; d.m = m; d.n = n; d.p = p; d.lddy = lddy; d.ldx = ldx; d.lddx = lddx; d.act = activation;
  d.grad_bf16 = grad_dtype == SOAP_BF16;
  d.dy = static_cast<const uint16_t *>(dy); d.x = static_cast<const uint16_t *>(x);
  d.w_gate = static_cast<const uint16_t *>(w_gate); d.w_up = static_cast<const uint16_t *>(w_up);
  d.w_down = static_cast<const uint16_t *>(w_down);
  d.gate = static_cast<uint16_t *>(const_cast<void *>(gate)); d.up = static_cast<uint16_t *>(const_cast<void *>(up));
  d.dx = static_cast<uint16_t *>(dx); d.dw_gate = dw_gate; d.dw_up = dw_up; d.dw_down = dw_down;
  d.workspace = workspace;
  return done(soap::launch_gated_bwd(d, stream), "gated feed-forward backward");
}

// ----------------------------------------------------------- distillation
int soap_distill_forward(int64_t rows, int64_t classes, int64_t slots, int dtype, const void *logits, int64_t ld,
                         const int32_t *index, int64_t ldi, int teacher_dtype, const void *teacher, int64_t ldt,
                         uint32_t flags, float temperature, float *loss, float *stats, hipStream_t stream) {
  SOAP_TRY(check_distill(rows, classes, slots, dtype, ld, ldi, teacher_dtype, ldt, flags, temperature));
  const size_t e = elem(dtype), t = elem(teacher_dtype);
  SOAP_TRY(check_bufs({{logits, span(rows, classes, ld, e), "logits", false, true, e},
                       {index, span(rows, slots, ldi, 4), "index", false, true, 4},
                       {teacher, span(rows, slots, ldt, t), "teacher", false, true, t},
                       {loss, 4 * (size_t)rows, "loss", true, true, 4},
                       {stats, stats_bytes(rows, flags), "stats", true, false, 4}}));
  soap::DistillDesc d = distill_desc(rows, classes, slots, dtype, logits, ld, index, ldi, teacher_dtype, teacher, ldt, flags, temperature);
  d.loss = loss; d.stats = stats;
  return done(soap::launch_distill(d, stream), "distillation");
}

int soap_distill_backward(int64_t rows, int64_t classes, int64_t slots, int dtype, const void *logits, int64_t ld,
                          const int32_t *index, int64_t ldi, int teacher_dtype, const void *teacher, int64_t ldt,
                          uint32_t flags, float temperature, const float *stats, const float *dloss, void *dlogits,
                          int64_t ldd, hipStream_t stream) {
  SOAP_TRY(check_distill(rows, classes, slots, dtype, ld, ldi, teacher_dtype, ldt, flags, temperature));
  SOAP_TRY(check_ld("ldd", ldd, classes));
  const size_t e = elem(dtype), t = elem(teacher_dtype);
  SOAP_TRY(check_bufs({{logits, span(rows, classes, ld, e), "logits", false, true, e},
                       {index, span(rows, slots, ldi, 4), "index", false, true, 4},
                       {teacher, span(rows, slots, ldt, t), "teacher", false, true, t},
                       {stats, stats_bytes(rows, flags), "stats", false, true, 4},
                       {dloss, 4 * (size_t)rows, "dloss", false, false, 4},
                       {dlogits, span(rows, classes, ldd, e), "dlogits", true, true, e}}));
  soap::DistillDesc d = distill_desc(rows, classes, slots, dtype, logits, ld, index, ldi, teacher_dtype, teacher, ldt, flags, temperature);
  d.stats = const_cast<float *>(stats); d.dloss = dloss; d.dlogits = dlogits; d.ldd = ldd;
  return done(soap::launch_distill(d, stream), "distillation backward");
}

int soap_distill_forward_backward(int64_t rows, int64_t classes, int64_t slots, int dtype, const void *logits,
                                  int64_t ld, const int32_t *index, int64_t ldi, int teacher_dtype,
                                  const void *teacher, int64_t ldt, uint32_t flags, float temperature,
                                  const float *dloss, float *loss, float *stats, void *dlogits, int64_t ldd,
                                  hipStream_t stream) {
  SOAP_TRY(check_distill(rows, classes, slots, dtype, ld, ldi, teacher_dtype, ldt, flags, temperature));
  SOAP_TRY(check_ld("ldd", ldd, classes));
  const size_t e = elem(dtype), t = elem(teacher_dtype);
  SOAP_TRY(check_bufs({{logits, span(rows, classes, ld, e), "logits", false, true, e},
                       {index, span(rows, slots, ldi, 4), "index", false, true, 4},
                       {teacher, span(rows, slots, ldt, t), "teacher", false, true, t},
                       {dloss, 4 * (size_t)rows, "dloss", false, false, 4},
                       {loss, 4 * (size_t)rows, "loss", true, true, 4},
                       {stats, stats_bytes(rows, flags), "stats", true, false, 4},
                       {dlogits, span(rows, classes, ldd, e), "dlogits", true, true, e}}));
  soap::DistillDesc d = distill_desc(rows, classes, slots, dtype, logits, ld, index, ldi, teacher_dtype, teacher, ldt, flags, temperature);
  d.dloss = dloss; d.loss = loss; d.stats = stats; d.dlogits = dlogits; d.ldd = ldd;
  return done(soap::launch_distill(d, stream), "distillation forward and backward");
}

}  // extern "C"
