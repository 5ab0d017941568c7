// C ABI of the training operators (include/lazymar.h, "Training a block with
// 8-bit activations", "The residual join" and "The end of a training step"):
// argument checks and dispatch.
#include "block8.cuh"
#include "join.cuh"
#include "optim.cuh"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>
#include <new>
#include <utility>
#include <vector>

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

// ---------------------------------------------------------------------------
// The residual join
// ---------------------------------------------------------------------------
namespace {

// What a call may be given: [rows, cols] of fp32 or bf16, of E4M3 as well, of E4M3 alone.
enum { ROWS_FLOAT, ROWS_ANY, ROWS_8 };
lazymar_status check_rows(const lazymar_rows& r, int kind, int rows, int cols, const char* msg) {
  if (!r.p) return LAZYMAR_OK;
  if (r.dtype == LAZYMAR_E4M3 && kind != ROWS_FLOAT) {
    const lazymar_block8 q{r.p, r.scale, r.ld, r.lds};
    return check_block8(&q, cols, rows, msg);
  }
  if (kind == ROWS_8) return bad(msg);
  return check_mat(r.p, r.dtype, r.ld, cols, msg);
}
Rows rows_of(const lazymar_rows& r) {
  const bool e8 = r.dtype == LAZYMAR_E4M3;
  return Rows{r.p, r.scale, r.ld, r.lds, r.dtype, e8 || vec8(r.p, r.dtype, r.ld)};
}
MatOut out_of(const lazymar_rows& r) { return mat_out(r.p, r.ld, r.dtype); }
lazymar_block8 eight_of(const lazymar_rows& r) { return lazymar_block8{r.p, r.scale, r.ld, r.lds}; }

// An output in place of an input: rows are worked on side by side, so in another layout they
// would overwrite rows that are still to be read.
// (An 8-bit tensor's scales go with it: in place of those of another one they would leave its bytes without theirs.)
const uint8_t* scale_of(const lazymar_rows& r) { return r.p && r.dtype == LAZYMAR_E4M3 ? r.scale : nullptr; }
bool displaced(const lazymar_rows& out, const lazymar_rows& in, int M) {
  if (scale_of(out) && scale_of(out) == scale_of(in) && (out.p != in.p || out.lds != in.lds)) return true;
  return out.p && out.p == in.p && (out.dtype != in.dtype || (M > 1 && out.ld != in.ld));
}
// An output in place of an input that several rows, or several kernels, read.
bool shared(std::initializer_list<const void*> outputs, std::initializer_list<const void*> inputs) {
  for (const void* o : outputs)
    for (const void* i : inputs)
      if (o && o == i) return true;
  return false;
}
// Two outputs in one place.
bool twice(std::initializer_list<const void*> outputs) {
  for (auto a = outputs.begin(); a != outputs.end(); ++a)
    for (auto b = outputs.begin(); b != a; ++b)
      if (*a && *a == *b) return true;
  return false;
}
bool norm_kind(int k) { return k == LAZYMAR_NORM_NONE || k == LAZYMAR_NORM_LAYER || k == LAZYMAR_NORM_RMS; }
int mod_rows(int M, int group) { return group > 0 ? (int)(((long long)M + group - 1) / group) : 1; }

#define CHECK_ROWS(field, kind, rows)                                                                            \
  TR_TRY(check_rows(a->field, kind, rows, a->D,                                                                  \
                    kind == ROWS_8 ? #field ": E4M3 device tensor, 16-byte aligned, ld % 16 == 0, ld >= D, lds >= rows required" \
                    : kind == ROWS_ANY                                                                           \
                        ? #field ": fp32, bf16 or E4M3 device tensor, ld >= D (E4M3: 16-byte aligned, ld % 16 == 0, lds >= rows) required" \
                        : #field ": fp32 or bf16 device tensor, ld >= D required"))

}  // namespace

extern "C" lazymar_status lazymar_join(const lazymar_join_args* a, void* stream) {
  if (!a) return bad("a required");
  if (a->M < 0 || a->D < 1 || a->group < 0) return bad("M >= 0, D >= 1, group >= 0 required");
  if (!norm_kind(a->post) || !norm_kind(a->pre)) return bad("post and pre: LAZYMAR_NORM_NONE, _LAYER or _RMS");
  if (!(a->eps > 0.f) || !std::isfinite(a->eps) || !std::isfinite(a->res)) return bad("eps > 0 and a finite res required");
  if (a->D > kLnMaxWidth) return report_error(LAZYMAR_ERR_UNSUPPORTED, "D <= 8192 required");
  if (a->M > kMost) return too_large();
  if (a->M == 0) return LAZYMAR_OK;  // (empty tensors have no address)
  if (!a->z.p && !a->h.p && !a->h8.p && !a->z8.p && !a->y8.p && !a->y_mean && !a->y_rstd && !a->z_mean && !a->z_rstd)
    return bad("no output given");
  if (!a->y.p && (a->post || a->gate.p || a->post_g || a->post_b || a->y8.p || a->y_mean || a->y_rstd))
    return bad("post, gate, post_g, post_b, y8 and y's statistics need y");
  if (!a->post && (a->y_mean || a->y_rstd)) return bad("y_mean and y_rstd need post");
  if (!a->pre && (a->h.p || a->h8.p || a->scale.p || a->shift.p || a->pre_g || a->pre_b || a->z_mean || a->z_rstd))
    return bad("h, h8, scale, shift, pre_g, pre_b and z's statistics need pre");
  if (!a->x.p) return bad("x: fp32 or bf16 device tensor, ld >= D required");
  const uint8_t *const h8s = scale_of(a->h8), *const z8s = scale_of(a->z8), *const y8s = scale_of(a->y8);
  if (twice({a->z.p, a->h.p, a->h8.p, a->z8.p, a->y8.p, a->y_mean, a->y_rstd, a->z_mean, a->z_rstd, h8s, z8s, y8s}))
    return bad("two outputs in one place");
  for (const lazymar_rows* out : {&a->z, &a->h, &a->h8, &a->z8, &a->y8})
    for (const lazymar_rows* in : {&a->x, &a->y})
      if (displaced(*out, *in, a->M)) return bad("an output in place of x or y: the same type and stride required");
  if (shared({a->z.p, a->h.p, a->h8.p, a->z8.p, a->y8.p, a->y_mean, a->y_rstd, a->z_mean, a->z_rstd, h8s, z8s, y8s},
             {a->gate.p, a->scale.p, a->shift.p, a->post_g, a->post_b, a->pre_g, a->pre_b}) ||
      shared({a->y_mean, a->y_rstd, a->z_mean, a->z_rstd, h8s, z8s, y8s}, {a->x.p, a->y.p}) ||
      shared({a->z.p, a->h.p, a->h8.p, a->z8.p, a->y8.p, a->y_mean, a->y_rstd, a->z_mean, a->z_rstd}, {scale_of(a->y)}))
    return bad("an output in place of an input other than x or y");
  const int mods = mod_rows(a->M, a->group);
  CHECK_ROWS(x, ROWS_FLOAT, a->M);
  CHECK_ROWS(y, ROWS_ANY, a->M);
  CHECK_ROWS(gate, ROWS_FLOAT, mods);
  CHECK_ROWS(scale, ROWS_FLOAT, mods);
  CHECK_ROWS(shift, ROWS_FLOAT, mods);
  CHECK_ROWS(z, ROWS_FLOAT, a->M);
  CHECK_ROWS(h, ROWS_FLOAT, a->M);
  CHECK_ROWS(h8, ROWS_8, a->M);
  CHECK_ROWS(z8, ROWS_8, a->M);
  CHECK_ROWS(y8, ROWS_8, a->M);
  for (const float* q : {a->post_g, a->post_b, a->pre_g, a->pre_b, (const float*)a->y_mean, (const float*)a->y_rstd,
                         (const float*)a->z_mean, (const float*)a->z_rstd})
    if (q) TR_TRY(check_f32(q, "parameters and statistics must be fp32 device pointers"));
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  Join p{};
  p.M = a->M;
  p.D = a->D;
  p.group = a->group;
  p.post = a->post;
  p.pre = a->pre;
  p.res = a->res;
  p.eps = a->eps;
  p.x = rows_of(a->x);
  p.y = rows_of(a->y);
  p.gate = rows_of(a->gate);
  p.scale = rows_of(a->scale);
  p.shift = rows_of(a->shift);
  p.post_g = a->post_g;
  p.post_b = a->post_b;
  p.pre_g = a->pre_g;
  p.pre_b = a->pre_b;
  p.params_vec = at(p.post_g, 32) && at(p.post_b, 32) && at(p.pre_g, 32) && at(p.pre_b, 32);
  p.z = out_of(a->z);
  p.h = out_of(a->h);
  p.h8 = eight_of(a->h8);
  p.z8 = eight_of(a->z8);
  p.y8 = eight_of(a->y8);
  p.y_mean = a->y_mean;
  p.y_rstd = a->y_rstd;
  p.z_mean = a->z_mean;
  p.z_rstd = a->z_rstd;
  return done(launch_join(c, p), "residual join kernel");
}

extern "C" size_t lazymar_join_grad_workspace(int M, int D, int group) { return join_grad_workspace(M, D, group); }

extern "C" lazymar_status lazymar_join_grad(const lazymar_join_grad_args* a, void* stream) {
  if (!a) return bad("a required");
  if (a->M < 0 || a->D < 1 || a->group < 0) return bad("M >= 0, D >= 1, group >= 0 required");
  if (!norm_kind(a->post) || !norm_kind(a->pre)) return bad("post and pre: LAZYMAR_NORM_NONE, _LAYER or _RMS");
  if (!std::isfinite(a->res)) return bad("a finite res required");
  if (a->D > kLnMaxWidth) return report_error(LAZYMAR_ERR_UNSUPPORTED, "D <= 8192 required");
  if (a->M > kMost) return too_large();
  const bool sums = a->dgate.p || a->dscale.p || a->dshift.p || a->dpost_g || a->dpost_b || a->dpre_g || a->dpre_b;
  if (!sums && a->M == 0) return LAZYMAR_OK;
  if (!sums && !a->dx.p && !a->dy.p && !a->dy8.p) return bad("no output given");
  if (!a->pre && (a->scale.p || a->pre_g || a->pre_b || a->dscale.p || a->dshift.p || a->dpre_g || a->dpre_b))
    return bad("scale, pre_g, pre_b and the gradients of these and of shift need pre");
  const int mods = mod_rows(a->M, a->group);
  if (a->M > 0) {
    if ((a->dh.p != nullptr) != (a->pre != LAZYMAR_NORM_NONE)) return bad("dh: given exactly with pre");
    if (!a->dh.p && !a->dz.p) return bad("dh or dz required");
    if (a->pre && (!a->z.p || !a->z_rstd || (a->pre == LAZYMAR_NORM_LAYER && !a->z_mean)))
      return bad("pre needs z and its statistics");
    if ((a->post || a->dgate.p || a->dpost_g) && !a->y.p) return bad("post, dgate and dpost_g need y");
    if (a->post && (!a->y_rstd || (a->post == LAZYMAR_NORM_LAYER && !a->y_mean))) return bad("post needs y's statistics");
    const uint8_t* const dy8s = scale_of(a->dy8);
    if (twice({a->dx.p, a->dy.p, a->dy8.p, dy8s, a->dgate.p, a->dscale.p, a->dshift.p, a->dpost_g, a->dpost_b, a->dpre_g, a->dpre_b}))
      return bad("two outputs in one place");
    for (const lazymar_rows* out : {&a->dx, &a->dy, &a->dy8})
      for (const lazymar_rows* in : {&a->dh, &a->dz, &a->z, &a->y})
        if (displaced(*out, *in, a->M)) return bad("dx, dy or dy8 in place of an input: the same type and stride required");
    if (shared({a->dx.p, a->dy.p, a->dy8.p, dy8s, a->dgate.p, a->dscale.p, a->dshift.p, a->dpost_g, a->dpost_b, a->dpre_g, a->dpre_b},
               {a->gate.p, a->scale.p, a->post_g, a->post_b, a->pre_g, a->pre_b, a->y_mean, a->y_rstd, a->z_mean, a->z_rstd}) ||
        shared({dy8s, a->dgate.p, a->dscale.p, a->dshift.p, a->dpost_g, a->dpost_b, a->dpre_g, a->dpre_b},
               {a->dh.p, a->dz.p, a->z.p, a->y.p}) ||
        shared({a->dx.p, a->dy.p, a->dy8.p, a->dgate.p, a->dscale.p, a->dshift.p, a->dpost_g, a->dpost_b, a->dpre_g, a->dpre_b},
               {scale_of(a->z), scale_of(a->y)}))
      return bad("an output in place of an input, other than dx, dy and dy8 of dz, dh, z and y");
    CHECK_ROWS(dh, ROWS_FLOAT, a->M);
    CHECK_ROWS(dz, ROWS_FLOAT, a->M);
    CHECK_ROWS(z, ROWS_ANY, a->M);
    CHECK_ROWS(y, ROWS_ANY, a->M);
    CHECK_ROWS(gate, ROWS_FLOAT, mods);
    CHECK_ROWS(scale, ROWS_FLOAT, mods);
    CHECK_ROWS(dx, ROWS_FLOAT, a->M);
    CHECK_ROWS(dy, ROWS_FLOAT, a->M);
    CHECK_ROWS(dy8, ROWS_8, a->M);
    for (const float* q : {a->post_g, a->post_b, a->pre_g, a->pre_b, a->y_mean, a->y_rstd, a->z_mean, a->z_rstd})
      if (q) TR_TRY(check_f32(q, "parameters and statistics must be fp32 device pointers"));
  }
  if (mods > 0) {
    CHECK_ROWS(dgate, ROWS_FLOAT, mods);
    CHECK_ROWS(dscale, ROWS_FLOAT, mods);
    CHECK_ROWS(dshift, ROWS_FLOAT, mods);
  }
  for (const float* q : {a->dpost_g, a->dpost_b, a->dpre_g, a->dpre_b})
    if (q) TR_TRY(check_f32(q, "dpost_g, dpost_b, dpre_g and dpre_b must be fp32 device pointers"));
  if (sums) TR_TRY(check_workspace(a->workspace, a->workspace_bytes, join_grad_workspace(a->M, a->D, a->group)));
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  JoinGrad p{};
  p.M = a->M;
  p.D = a->D;
  p.group = a->group;
  p.post = a->post;
  p.pre = a->pre;
  p.res = a->res;
  p.accumulate = a->accumulate != 0;
  p.dh = rows_of(a->dh);
  p.dz = rows_of(a->dz);
  p.z = rows_of(a->z);
  p.y = rows_of(a->y);
  if (!a->post && !a->dgate.p && !a->dpost_g) p.y.p = nullptr;  // (nothing depends on it)
  p.gate = rows_of(a->gate);
  p.scale = rows_of(a->scale);
  p.y_mean = a->y_mean;
  p.y_rstd = a->y_rstd;
  p.z_mean = a->z_mean;
  p.z_rstd = a->z_rstd;
  p.post_g = a->post_g;
  p.post_b = a->post_b;
  p.pre_g = a->pre_g;
  p.pre_b = a->pre_b;
  p.params_vec = at(p.post_g, 32) && at(p.post_b, 32) && at(p.pre_g, 32) && at(p.pre_b, 32);
  p.dx = out_of(a->dx);
  p.dy = out_of(a->dy);
  p.dy8 = eight_of(a->dy8);
  p.dgate = out_of(a->dgate);
  p.dscale = out_of(a->dscale);
  p.dshift = out_of(a->dshift);
  p.dpost_g = a->dpost_g;
  p.dpost_b = a->dpost_b;
  p.dpre_g = a->dpre_g;
  p.dpre_b = a->dpre_b;
  p.ws = join_sums_at(a->workspace);
  return done(launch_join_grad(c, p), "residual join gradient kernel");
}

// ---------------------------------------------------------------------------
// The end of a training step
// ---------------------------------------------------------------------------
struct lazymar_params {
  int device = 0;
  bool has_weights = false;
  void* memory = nullptr;
  ParamList list{};
};

namespace {

constexpr int kMostParams = 1 << 20;

lazymar_status check_param(const lazymar_param& t, bool weights) {
  if (t.n < 0 || t.n > (1ll << 40)) return bad("n: 0 .. 2^40 elements");
  if (!float_type(t.g_dtype)) return bad("g_dtype: fp32 or bf16");
  if (t.out && !float_type(t.out_dtype)) return bad("out_dtype: fp32 or bf16");
  if (t.out && t.out == t.g && t.out_dtype != t.g_dtype) return bad("out in place of g: the same type required");
  if (!std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay)) return bad("finite lr_scale and weight_decay required");
  if (t.n == 0) return LAZYMAR_OK;  // (empty tensors have no address)
  if ((t.p != nullptr) != weights || (t.m != nullptr) != weights || (t.v != nullptr) != weights)
    return bad("p, m and v: all or none, alike for the whole list");
  if ((t.ema || t.copy) && !weights) return bad("ema and copy need p, m and v");
  const void* fs[] = {t.p, t.m, t.v, t.ema};
  for (const void* q : fs)
    if (q && (!at(q, 4) || !is_device_ptr(q))) return bad("p, m, v and ema must be fp32 device pointers");
  if (!at(t.g, elem(t.g_dtype)) || !is_device_ptr(t.g)) return bad("g must be a device pointer");
  if (t.out && (!at(t.out, elem(t.out_dtype)) || !is_device_ptr(t.out))) return bad("out must be a device pointer");
  if (t.copy && (!at(t.copy, 2) || !is_device_ptr(t.copy))) return bad("copy must be a bf16 device pointer");
  return LAZYMAR_OK;
}

// Elements of g in front of its first boundary of eight, where p lies on that boundary too.
int head_of(const lazymar_param& t) {
  const size_t e = elem(t.g_dtype);
  return (int)((8 - reinterpret_cast<uintptr_t>(t.g) / e % 8) % 8);
}
bool lies_alike(const void* p, size_t e, int head) { return !p || at(static_cast<const char*>(p) + head * e, 8 * e); }

Param param_of(const lazymar_param& t) {
  Param p{};
  p.g = t.g;
  p.out = t.out ? t.out : const_cast<void*>(t.g);
  p.p = t.p;
  p.m = t.m;
  p.v = t.v;
  p.ema = t.ema;
  p.copy = static_cast<bf16*>(t.copy);
  p.lr_scale = t.lr_scale;
  p.weight_decay = t.weight_decay;
  const int out_dtype = t.out ? t.out_dtype : t.g_dtype, head = head_of(t);
  p.flags = (t.g_dtype == LAZYMAR_BF16 ? PARAM_G_BF16 : 0u) | (out_dtype == LAZYMAR_BF16 ? PARAM_OUT_BF16 : 0u) |
            (lies_alike(p.out, elem(out_dtype), head) ? PARAM_VEC_OUT : 0u) |
            (lies_alike(t.p, 4, head) && lies_alike(t.m, 4, head) && lies_alike(t.v, 4, head) &&
                     lies_alike(t.ema, 4, head) && lies_alike(t.copy, 2, head)
                 ? PARAM_VEC_ALL
                 : 0u);
  return p;
}

// Whether tensors of a list overlap, other than an out that is its g. (A weight that is in it twice would be updated by
// two threads at once.)
bool overlaps(const lazymar_param* list, int count) {
  std::vector<std::pair<uintptr_t, uintptr_t>> spans;
  const auto add = [&](const void* p, long long n, size_t e) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    if (p) spans.emplace_back(at, at + (uintptr_t)n * e);
  };
  for (int i = 0; i < count; ++i) {
    const lazymar_param& t = list[i];
    if (t.n == 0) continue;
    add(t.g, t.n, elem(t.g_dtype));
    if (t.out != t.g) add(t.out, t.n, elem(t.out_dtype));
    for (const float* p : {t.p, t.m, t.v, t.ema}) add(p, t.n, 4);
    add(t.copy, t.n, 2);
  }
  std::sort(spans.begin(), spans.end());
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].first < spans[i - 1].second) return true;
  return false;
}

lazymar_status params_create(const lazymar_param* list, int count, lazymar_params** out) {
  bool weights = false;
  long long total = 0;
  for (int i = 0; i < count; ++i) weights |= list[i].n > 0 && list[i].p != nullptr;
  for (int i = 0; i < count; ++i) {
    TR_TRY(check_param(list[i], weights));
    total += list[i].n;
    if (total > (1ll << 40)) return report_error(LAZYMAR_ERR_UNSUPPORTED, "at most 2^40 elements");
  }
  if (overlaps(list, count)) return bad("tensors of a list overlap");
  // pieces of a multiple of kPiece, at most about kMostPieces of them
  const long long piece = kPiece * (1 + total / (kPiece * kMostPieces));
  std::vector<Param> params;
  std::vector<Piece> pieces;
  for (int i = 0; i < count; ++i) {
    const lazymar_param& t = list[i];
    if (t.n == 0) continue;
    const int head = head_of(t);
    for (long long from = 0; from < t.n;) {
      const long long most = piece + (from == 0 ? head : 0), n = t.n - from < most ? t.n - from : most;
      const int in_front = from > 0 ? 0 : n < head ? (int)n : head;
      pieces.push_back(piece_of(static_cast<const char*>(t.g) + from * (long long)elem(t.g_dtype), (unsigned)params.size(), (int)n,
                                in_front, t.g_dtype == LAZYMAR_BF16));
      from += n;
    }
    params.push_back(param_of(t));
  }
  Ctx c;
  TR_TRY(component_ctx(nullptr, &c));
  const size_t a = params.size() * sizeof(Param), b = pieces.size() * sizeof(Piece);
  const size_t at_pieces = (a + 255) / 256 * 256, at_partial = at_pieces + (b + 255) / 256 * 256 + 256;
  const size_t bytes = at_partial + (size_t)c.num_sms * kMostNormCtas * sizeof(double) + sizeof(unsigned);
  std::vector<char> image(bytes, 0);
  if (a) std::memcpy(image.data(), params.data(), a);
  if (b) std::memcpy(image.data() + at_pieces, pieces.data(), b);
  lazymar_params* h = new lazymar_params;
  cudaError_t e = cudaGetDevice(&h->device);
  if (e == cudaSuccess) e = cudaMalloc(&h->memory, bytes);
  char* m = static_cast<char*>(h->memory);
  if (e == cudaSuccess) e = cudaMemcpy(m, image.data(), bytes, cudaMemcpyHostToDevice);
  // (done before the calls on streams that do not wait for the default one)
  if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);
  if (e != cudaSuccess) {
    lazymar_params_destroy(h);
    return e == cudaErrorMemoryAllocation ? report_error(LAZYMAR_ERR_OOM, "device memory of the list") : report_cuda(e, "list");
  }
  h->has_weights = weights;
  h->list = ParamList{reinterpret_cast<Param*>(m), reinterpret_cast<Piece*>(m + at_pieces), reinterpret_cast<double*>(m + at_partial),
                      reinterpret_cast<unsigned*>(m + bytes - sizeof(unsigned)), (int)pieces.size()};
  *out = h;
  return LAZYMAR_OK;
}

// The list's call: its handle, the state, the device.
lazymar_status check_list(const lazymar_params* h, const lazymar_step_state* state, bool needed) {
  if (!h) return bad("a list required");
  if (!state && needed) return bad("state required");
  if (state && (!at(state, 4) || !is_device_ptr(state))) return bad("state must be a 4-byte aligned device pointer");
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return report_cuda(e, "cudaGetDevice");
  if (dev != h->device) return bad("the list was made on another device");
  return LAZYMAR_OK;
}

}  // namespace

extern "C" lazymar_status lazymar_params_create(const lazymar_param* list, int count, lazymar_params** out) {
  if (!out) return bad("out required");
  *out = nullptr;
  if (count < 0 || (count > 0 && !list)) return bad("count >= 0 and a list required");
  if (count > kMostParams) return report_error(LAZYMAR_ERR_UNSUPPORTED, "at most 2^20 tensors");
  try {
    return params_create(list, count, out);
  } catch (const std::bad_alloc&) {
    return report_error(LAZYMAR_ERR_OOM, "host memory of the list");
  }
}

extern "C" void lazymar_params_destroy(lazymar_params* h) {
  if (!h) return;
  cudaFree(h->memory);
  delete h;
}

extern "C" lazymar_status lazymar_grad_norm(lazymar_params* h, float scale, float max_norm, lazymar_step_state* state,
                                            void* stream) {
  if (!(scale > 0.f) || !std::isfinite(scale) || !(max_norm > 0.f)) return bad("scale > 0, finite, and max_norm > 0 required");
  TR_TRY(check_list(h, state, true));
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  return done(launch_grad_norm(c, h->list, scale, max_norm, state), "gradient norm kernel");
}

extern "C" lazymar_status lazymar_clip_grads(lazymar_params* h, const lazymar_step_state* state, void* stream) {
  TR_TRY(check_list(h, state, true));
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  return done(launch_clip_grads(c, h->list, state), "clipping kernel");
}

extern "C" lazymar_status lazymar_adamw(lazymar_params* h, const lazymar_adamw_args* a, const lazymar_step_state* state,
                                        void* stream) {
  if (!a) return bad("a required");
  if (!(a->beta1 >= 0 && a->beta1 < 1 && a->beta2 >= 0 && a->beta2 < 1)) return bad("0 <= beta < 1 required");
  if (!((float)a->eps > 0.f) || !std::isfinite((float)a->eps) || !std::isfinite((float)a->lr)) return bad("eps > 0 and a finite lr required");
  if (!(a->ema_decay >= 0 && a->ema_decay <= 1)) return bad("0 <= ema_decay <= 1 required");
  if (!state && (!((float)a->factor > 0.f) || !std::isfinite((float)a->factor) || a->steps < 1))
    return bad("without state: factor > 0, finite, and steps >= 1 required");
  if (a->lr_device) TR_TRY(check_f32(a->lr_device, "lr_device must be an fp32 device pointer"));
  TR_TRY(check_list(h, state, false));
  if (!h->has_weights && h->list.n_pieces > 0) return bad("the list has no weights");
  Ctx c;
  TR_TRY(component_ctx(stream, &c));
  AdamW p{};
  p.lr = (float)a->lr;
  p.eps = (float)a->eps;
  p.more1 = (float)(1 - a->beta1);
  p.more2 = (float)(1 - a->beta2);
  p.more_ema = (float)(1 - a->ema_decay);
  p.log1 = (float)std::log(a->beta1);
  p.log2 = (float)std::log(a->beta2);
  p.lr_device = a->lr_device;
  p.factor = (float)a->factor;
  p.steps = a->steps;
  return done(launch_adamw(c, h->list, p, state), "AdamW kernel");
}
