// C ABI of the training operators (include/lazymar.h, "Training a block with
// 8-bit activations"): argument checks and dispatch.
#include "block8.cuh"

using namespace lm;

namespace {

lazymar_status bad(const char* msg) { return report_error(LAZYMAR_ERR_INVALID_ARG, msg); }

#define TR_TRY(expr)                 \
  do {                               \
    lazymar_status s_ = (expr);      \
    if (s_ != LAZYMAR_OK) return s_; \
  } while (0)

// Rows and columns that the kernels count in 32 bits with room for a launch's strides.
constexpr int kMost = 1 << 30;
lazymar_status too_large() { return report_error(LAZYMAR_ERR_UNSUPPORTED, "at most 2^30 rows and columns"); }

bool float_type(int dtype) { return dtype == LAZYMAR_F32 || dtype == LAZYMAR_BF16; }
size_t elem(int dtype) { return dtype == LAZYMAR_F32 ? 4 : 2; }
bool at(const void* p, size_t align) { return reinterpret_cast<uintptr_t>(p) % align == 0; }

// An fp32 or bf16 tensor [rows, ld] of `cols` columns.
lazymar_status check_mat(const void* p, int dtype, int ld, int cols, const char* msg) {
  if (!float_type(dtype) || ld < cols || !at(p, elem(dtype)) || !is_device_ptr(p)) return bad(msg);
  return LAZYMAR_OK;
}
// Rows on boundaries of eight elements (absent tensors' are).
bool vec8(const void* p, int dtype, int ld) { return !p || (ld % 8 == 0 && at(p, 8 * elem(dtype))); }
Mat mat(const void* p, int ld, int dtype) { return Mat{p, ld, dtype, vec8(p, dtype, ld)}; }
MatOut mat_out(void* p, int ld, int dtype) { return MatOut{p, ld, dtype, vec8(p, dtype, ld)}; }

lazymar_status check_block8(const lazymar_block8* q, int cols, int scale_rows, const char* msg) {
  if (!q->q || !q->scale || q->ldq % 16 != 0 || q->ldq < cols || q->lds < scale_rows || !at(q->q, 16) ||
      !is_device_ptr(q->q) || !is_device_ptr(q->scale))
    return bad(msg);
  return LAZYMAR_OK;
}
lazymar_status check_f32(const float* p, const char* msg) {
  if (!at(p, 4) || !is_device_ptr(p)) return bad(msg);
  return LAZYMAR_OK;
}
lazymar_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return LAZYMAR_OK;
  if (bytes < need) return bad("workspace_bytes below the workspace function's result");
  if (!at(ws, 16) || !is_device_ptr(ws)) return bad("workspace must be a 16-byte aligned device pointer");
  return LAZYMAR_OK;
}
lazymar_block8 given(const lazymar_block8* q) { return q ? *q : lazymar_block8{nullptr, nullptr, 0, 0}; }
lazymar_status done(cudaError_t e, const char* what) { return e == cudaSuccess ? LAZYMAR_OK : report_cuda(e, what); }

}  // namespace

extern "C" lazymar_status lazymar_layernorm_forward(int x_dtype, const void* x, int ldx, const float* g, const float* b,
                                                    int y_dtype, void* y, int ldy, const lazymar_block8* y8,
                                                    const lazymar_block8* x8, float* mean, float* rstd, int M, int D,
                                                    float eps, void* stream) {
  if (M < 0 || D < 1 || !(eps > 0.f)) return bad("M >= 0, D >= 1, eps > 0 required");
  if (D > kLnMaxWidth) return report_error(LAZYMAR_ERR_UNSUPPORTED, "D <= 8192 required");
  if (M > kMost) return too_large();
  if (M == 0) return LAZYMAR_OK;  // (empty tensors have no address)
  if (!y && !y8 && !x8 && !mean && !rstd) return bad("no output given");
  if (y && x == y && M > 1 && (x_dtype != y_dtype || ldx != ldy))  // (as below)
    return bad("y in place of x: y_dtype = x_dtype and ldy = ldx required");
  TR_TRY(check_mat(x, x_dtype, ldx, D, "x: fp32 or bf16 device tensor, ldx >= D required"));
  if (y) TR_TRY(check_mat(y, y_dtype, ldy, D, "y: fp32 or bf16 device tensor, ldy >= D required"));
  if (y8) TR_TRY(check_block8(y8, D, M, "y8: device tensors, q 16-byte aligned, ldq % 16 == 0, ldq >= D, lds >= M"));
  if (x8) TR_TRY(check_block8(x8, D, M, "x8: device tensors, q 16-byte aligned, ldq % 16 == 0, ldq >= D, lds >= M"));
  const float* ps[] = {g, b, mean, rstd};
  for (const float* q : ps)
    if (q) TR_TRY(check_f32(q, "g, b, mean and rstd must be fp32 device pointers"));
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  LnForward p{};
  p.x = mat(x, ldx, x_dtype);
  p.g = g;
  p.b = b;
  p.params_vec = at(g, 32) && at(b, 32);
  p.y = mat_out(y, ldy, y_dtype);
  p.y8 = given(y8);
  p.x8 = given(x8);
  p.mean = mean;
  p.rstd = rstd;
  p.M = M;
  p.D = D;
  p.eps = eps;
  return done(launch_ln_forward(c, p), "LayerNorm forward kernel");
}

extern "C" size_t lazymar_layernorm_backward_workspace(int M, int D) { return ln_backward_workspace(M, D); }

extern "C" lazymar_status lazymar_layernorm_backward(int dy_dtype, const void* dy, int lddy, int x_dtype, const void* x,
                                                     int ldx, const lazymar_block8* x8, const float* mean,
                                                     const float* rstd, const float* g, const float* dres, int lddres,
                                                     int dx_dtype, void* dx, int lddx, float* dg, float* db,
                                                     int accumulate, int M, int D, void* workspace,
                                                     size_t workspace_bytes, void* stream) {
  if (M < 0 || D < 1) return bad("M >= 0, D >= 1 required");
  if (D > kLnMaxWidth) return report_error(LAZYMAR_ERR_UNSUPPORTED, "D <= 8192 required");
  if (M > kMost) return too_large();
  if ((dg == nullptr) != (db == nullptr)) return bad("dg and db: both or neither");
  if (M > 0) {
    if ((x == nullptr) == (x8 == nullptr)) return bad("exactly one of x and x8 required");
    // (rows are worked on side by side: in another layout dx would overwrite rows that are still to be read)
    if (dx && M > 1 && ((dx == dy && (dx_dtype != dy_dtype || lddx != lddy)) ||
                        (dx == x && (dx_dtype != x_dtype || lddx != ldx))))
      return bad("dx in place of dy or x: the same type and stride required");
    if (dres && dx == dres && (dx_dtype != LAZYMAR_F32 || (M > 1 && lddx != lddres)))
      return bad("dx in place of dres: fp32 with the same stride required");
    TR_TRY(check_mat(dy, dy_dtype, lddy, D, "dy: fp32 or bf16 device tensor, lddy >= D required"));
    if (x) TR_TRY(check_mat(x, x_dtype, ldx, D, "x: fp32 or bf16 device tensor, ldx >= D required"));
    if (x8) TR_TRY(check_block8(x8, D, M, "x8: device tensors, q 16-byte aligned, ldq % 16 == 0, ldq >= D, lds >= M"));
    TR_TRY(check_f32(mean, "mean must be an fp32 device pointer"));
    TR_TRY(check_f32(rstd, "rstd must be an fp32 device pointer"));
    if (g) TR_TRY(check_f32(g, "g must be an fp32 device pointer"));
    if (dres) TR_TRY(check_mat(dres, LAZYMAR_F32, lddres, D, "dres: fp32 device tensor, lddres >= D required"));
    TR_TRY(check_mat(dx, dx_dtype, lddx, D, "dx: fp32 or bf16 device tensor, lddx >= D required"));
  }
  if (dg) {
    TR_TRY(check_f32(dg, "dg must be an fp32 device pointer"));
    TR_TRY(check_f32(db, "db must be an fp32 device pointer"));
    TR_TRY(check_workspace(workspace, workspace_bytes, ln_backward_workspace(M, D)));
  }
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  LnBackward p{};
  p.dy = mat(dy, lddy, dy_dtype);
  p.x = mat(x, ldx, x_dtype);
  p.x8 = given(x8);
  p.mean = mean;
  p.rstd = rstd;
  p.g = g;
  p.dres = mat(dres, lddres, LAZYMAR_F32);
  p.dx = mat_out(dx, lddx, dx_dtype);
  p.dg = dg;
  p.db = db;
  p.accumulate = accumulate != 0;
  p.M = M;
  p.D = D;
  p.ws = static_cast<float*>(workspace);
  return done(launch_ln_backward(c, p), "LayerNorm backward kernel");
}

extern "C" lazymar_status lazymar_block8_pack(int dtype, const void* x, int ldx, const lazymar_block8* q, int rows,
                                              int cols, void* stream) {
  if (rows < 0 || cols < 1) return bad("rows >= 0, cols >= 1 required");
  if (rows > kMost || cols > kMost) return too_large();
  if (!q) return bad("q required");
  if (rows == 0) return LAZYMAR_OK;
  TR_TRY(check_mat(x, dtype, ldx, cols, "x: fp32 or bf16 device tensor, ldx >= cols required"));
  TR_TRY(check_block8(q, cols, rows, "q: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= cols, lds >= rows"));
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  Rows8 p{};
  p.in = mat(x, ldx, dtype);
  p.out = mat_out(nullptr, 0, dtype);
  p.out8 = *q;
  p.rows = rows;
  p.cols = cols;
  return done(launch_rows8(c, p), "8-bit pack kernel");
}

extern "C" lazymar_status lazymar_block8_unpack(const lazymar_block8* q, int dtype, void* x, int ldx, int rows,
                                                int cols, void* stream) {
  if (rows < 0 || cols < 1) return bad("rows >= 0, cols >= 1 required");
  if (rows > kMost || cols > kMost) return too_large();
  if (!q) return bad("q required");
  if (rows == 0) return LAZYMAR_OK;
  TR_TRY(check_block8(q, cols, rows, "q: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= cols, lds >= rows"));
  TR_TRY(check_mat(x, dtype, ldx, cols, "x: fp32 or bf16 device tensor, ldx >= cols required"));
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  return done(launch_unpack8(c, *q, mat_out(x, ldx, dtype), rows, cols), "8-bit unpack kernel");
}

extern "C" lazymar_status lazymar_block8_pack_weight(int dtype, const void* w, int ldw, const lazymar_block8* q,
                                                     const lazymar_block8* qt, int N, int K, void* stream) {
  if (N < 0 || K < 1 || N > 128 * 65535) return bad("0 <= N <= 8388480, K >= 1 required");
  if (K > kMost) return too_large();
  if (!q && !qt) return bad("q or qt required");
  if (N == 0) return LAZYMAR_OK;
  TR_TRY(check_mat(w, dtype, ldw, K, "w: fp32 or bf16 device tensor, ldw >= K required"));
  if (q)
    TR_TRY(check_block8(q, K, (N + 127) / 128,
                        "q: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= K, lds >= ceil(N / 128)"));
  if (qt)
    TR_TRY(check_block8(qt, N, (K + 127) / 128,
                        "qt: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= N, lds >= ceil(K / 128)"));
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  return done(launch_pack_weight8(c, mat(w, ldw, dtype), given(q), given(qt), N, K), "8-bit weight pack kernel");
}

extern "C" size_t lazymar_block8_gelu_backward_workspace(int rows, int cols) { return rows8_workspace(rows, cols); }

extern "C" lazymar_status lazymar_block8_gelu_backward(int dtype, const void* da, int ldda, const lazymar_block8* u,
                                                       int du_dtype, void* du, int lddu, const lazymar_block8* du8,
                                                       float* db, int accumulate, int rows, int cols, void* workspace,
                                                       size_t workspace_bytes, void* stream) {
  if (rows < 0 || cols < 1) return bad("rows >= 0, cols >= 1 required");
  if (rows > kMost || cols > kMost) return too_large();
  if (rows > 0) {
    if (!du && !du8 && !db) return bad("no output given");
    if (du && du == da && (du_dtype != dtype || (rows > 1 && lddu != ldda))) return bad("du in place of da: the same type and stride required");
    TR_TRY(check_mat(da, dtype, ldda, cols, "da: fp32 or bf16 device tensor, ldda >= cols required"));
    if (u)
      TR_TRY(check_block8(u, cols, rows, "u: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= cols, lds >= rows"));
    if (du) TR_TRY(check_mat(du, du_dtype, lddu, cols, "du: fp32 or bf16 device tensor, lddu >= cols required"));
    if (du8)
      TR_TRY(check_block8(du8, cols, rows,
                          "du8: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= cols, lds >= rows"));
  }
  if (db) {
    TR_TRY(check_f32(db, "db must be an fp32 device pointer"));
    TR_TRY(check_workspace(workspace, workspace_bytes, rows8_workspace(rows, cols)));
  }
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  Rows8 p{};
  p.in = mat(da, ldda, dtype);
  p.u = given(u);
  p.out = mat_out(du, lddu, du_dtype);
  p.out8 = given(du8);
  p.db = db;
  p.accumulate = accumulate != 0;
  p.rows = rows;
  p.cols = cols;
  p.ws = static_cast<float*>(workspace);
  return done(launch_rows8(c, p), "GELU gradient kernel");
}

extern "C" lazymar_status lazymar_block8_linear(int epilogue, const lazymar_block8* a, const lazymar_block8* w,
                                                const float* bias, const float* residual, int ldr, int out_dtype,
                                                void* out, int ldo, const lazymar_block8* out8,
                                                const lazymar_block8* u8, int M, int N, int K, void* stream) {
  if (epilogue != LAZYMAR_EPI_BIAS && epilogue != LAZYMAR_EPI_GELU && epilogue != LAZYMAR_EPI_RESIDUAL)
    return bad("epilogue: BIAS, GELU or RESIDUAL");
  if (M < 0 || N < 0 || K < 1) return bad("M >= 0, N >= 0, K >= 1 required");
  if (M > kMost || N > kMost || K > kMost) return too_large();
  if (!a || !w) return bad("a and w required");
  const bool empty = M == 0 || N == 0;  // (empty tensors have no address)
  if (!empty && !out && !out8) return bad("out or out8 required");
  if (epilogue == LAZYMAR_EPI_RESIDUAL) {
    if (out8 || (!out && !empty) || out_dtype != LAZYMAR_F32) return bad("RESIDUAL: out fp32 and no out8");
  } else if (residual) {
    return bad("residual is for LAZYMAR_EPI_RESIDUAL");
  }
  if (u8 && epilogue != LAZYMAR_EPI_GELU) return bad("u8 is for LAZYMAR_EPI_GELU");
  if (empty) return LAZYMAR_OK;
  if (residual && out == residual && M > 1 && ldo != ldr) return bad("out in place of residual: the same stride required");
  TR_TRY(check_block8(a, K, M, "a: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= K, lds >= M"));
  TR_TRY(check_block8(w, K, (N + 127) / 128,
                      "w: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= K, lds >= ceil(N / 128)"));
  if (bias) TR_TRY(check_f32(bias, "bias must be an fp32 device pointer"));
  if (epilogue == LAZYMAR_EPI_RESIDUAL)
    TR_TRY(check_mat(residual, LAZYMAR_F32, ldr, N, "residual: fp32 device tensor, ldr >= N required"));
  if (out) TR_TRY(check_mat(out, out_dtype, ldo, N, "out: fp32 or bf16 device tensor, ldo >= N required"));
  if (out8)
    TR_TRY(check_block8(out8, N, M, "out8: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= N, lds >= M"));
  if (u8) TR_TRY(check_block8(u8, N, M, "u8: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= N, lds >= M"));
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  Linear8 p{};
  p.epilogue = epilogue;
  p.a = *a;
  p.w = *w;
  p.bias = bias;
  p.residual = mat(residual, ldr, LAZYMAR_F32);
  p.out = mat_out(out, ldo, out_dtype);
  p.out8 = given(out8);
  p.u8 = given(u8);
  p.M = M;
  p.N = N;
  p.K = K;
  return done(launch_linear8(c, p), "8-bit linear kernel");
}

extern "C" size_t lazymar_block8_wgrad_workspace(int M, int N, int K) { return wgrad8_workspace(M, N, K); }

extern "C" lazymar_status lazymar_block8_wgrad(const void* dy, int lddy, const lazymar_block8* x, float* dw, int lddw,
                                               int accumulate, int M, int N, int K, void* workspace,
                                               size_t workspace_bytes, void* stream) {
  if (M < 0 || N < 0 || K < 1) return bad("M >= 0, N >= 0, K >= 1 required");
  if (M > kMost || N > kMost || K > kMost) return too_large();
  if (N == 0) return LAZYMAR_OK;
  TR_TRY(check_mat(dw, LAZYMAR_F32, lddw, K, "dw: fp32 device tensor, lddw >= K required"));
  if (M > 0) {
    if (!x) return bad("x required");
    TR_TRY(check_mat(dy, LAZYMAR_BF16, lddy, N, "dy: bf16 device tensor, lddy >= N required"));
    if (lddy % 8 != 0 || !at(dy, 16)) return bad("dy: 16-byte alignment and lddy % 8 == 0 required");
    TR_TRY(check_block8(x, K, M, "x: device tensors, 16-byte aligned, ldq % 16 == 0, ldq >= K, lds >= M"));
    TR_TRY(check_workspace(workspace, workspace_bytes, wgrad8_workspace(M, N, K)));
  }
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  Wgrad8 p{};
  p.dy = dy;
  p.lddy = lddy;
  p.x = given(x);
  p.dw = dw;
  p.lddw = lddw;
  p.accumulate = accumulate != 0;
  p.M = M;
  p.N = N;
  p.K = K;
  p.ws = static_cast<float*>(workspace);
  return done(launch_wgrad8(c, p), "weight gradient kernel");
}
