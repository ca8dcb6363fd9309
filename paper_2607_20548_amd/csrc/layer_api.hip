// C ABI of the operators around an expert bank: argument checks and launches of
// layer norm, router and MXFP4.  Everything is enqueued on the caller's stream;
// nothing here allocates.
#include "soap.h"

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

}  // extern "C"
