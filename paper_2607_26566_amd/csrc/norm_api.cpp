// Entry points of the residual's addition with an RMS norm: argument checks, then the
// launches.
#include <cmath>
#include <cstring>

#include "block_ops.h"

using namespace t2i;

namespace {

bool bad_dtype(int32_t d) { return d != T2I_F32 && d != T2I_BF16; }
bool off(const void* p, size_t n) { return (uintptr_t)p % n != 0; }
size_t bytes_of(int32_t d) { return d == T2I_BF16 ? 2 : 4; }
// (fewer than 2^32 threads: a wave per row up to K = 2048, up to 1024 threads for longer
// ones)
bool bad_sizes(int32_t rows, int32_t K) {
  return rows < 1 || K < 1 || K > 1 << 20 || rows >= (K <= 2048 ? (1 << 26) - 4 : 1 << 22);
}
t2i_status done(hipError_t e) {
  return e == hipSuccess ? T2I_OK : ops_fail(T2I_ERR_DEVICE, hipGetErrorString(e));
}

// y: the norm's output, or its codes (checked by the caller then)
t2i_status check_norm(int32_t dtype, int32_t resid_dtype, int32_t rows, int32_t K, const void* x, int32_t ldx,
                      const void* resid, int32_t ldr, const void* w, float eps, const void* h, int32_t ldh) {
  if (bad_dtype(dtype) || bad_dtype(resid_dtype)) return ops_fail(T2I_ERR_INVALID_ARG, "bad dtype");
  if (resid_dtype != dtype && (!resid || resid_dtype != T2I_F32))
    return ops_fail(T2I_ERR_INVALID_ARG, "the residual has the operands' type or fp32");
  if (bad_sizes(rows, K)) return ops_fail(T2I_ERR_SHAPE, "bad shape");
  if (!x || (resid && !h)) return ops_fail(T2I_ERR_INVALID_ARG, "NULL pointer");
  if (ldx < K || (resid && (ldr < K || ldh < K))) return ops_fail(T2I_ERR_SHAPE, "leading dimension < K");
  const size_t e = bytes_of(dtype), re = bytes_of(resid_dtype);
  if (off(x, e) || off(w, e) || off(resid, re) || (resid && off(h, re)))
    return ops_fail(T2I_ERR_INVALID_ARG, "operands need the alignment of their type");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return ops_fail(T2I_ERR_INVALID_ARG, "eps must be finite, >= 0");
  return T2I_OK;
}

NormFwd make_norm(int32_t rows, int32_t K, const void* x, int32_t ldx, const void* resid, int32_t ldr, const void* w,
                  float eps, void* h, int32_t ldh, void* y, int32_t ldy, float* scale) {
  NormFwd a;
  std::memset(&a, 0, sizeof(a));
  a.rows = rows;
  a.K = K;
  a.x = x;
  a.ldx = ldx;
  a.resid = resid;
  a.ldr = ldr;
  a.w = w;
  a.eps = eps;
  a.h = h;
  a.ldh = ldh;
  a.y = y;
  a.ldy = ldy;
  a.scale = scale;
  return a;
}

}  // namespace

extern "C" {

t2i_status t2i_op_add_rms_norm(int32_t dtype, int32_t resid_dtype, int32_t rows, int32_t K, const void* x,
                               int32_t ldx, const void* resid, int32_t ldr, const void* w, float eps, void* h,
                               int32_t ldh, void* y, int32_t ldy, void* stream) {
  const t2i_status s = check_norm(dtype, resid_dtype, rows, K, x, ldx, resid, ldr, w, eps, h, ldh);
  if (s != T2I_OK) return s;
  if (!y || off(y, bytes_of(dtype))) return ops_fail(T2I_ERR_INVALID_ARG, "y is NULL or off its type's alignment");
  if (ldy < K) return ops_fail(T2I_ERR_SHAPE, "leading dimension < K");
  return done(launch_add_rms_norm(dtype == T2I_BF16, resid_dtype == T2I_BF16, false,
                                  make_norm(rows, K, x, ldx, resid, ldr, w, eps, h, ldh, y, ldy, nullptr),
                                  (hipStream_t)stream));
}

t2i_status t2i_op_add_rms_norm_i8(int32_t dtype, int32_t resid_dtype, int32_t rows, int32_t K, const void* x,
                                  int32_t ldx, const void* resid, int32_t ldr, const void* w, float eps, void* h,
                                  int32_t ldh, int8_t* q, int32_t ldq, float* scale, void* stream) {
  const t2i_status s = check_norm(dtype, resid_dtype, rows, K, x, ldx, resid, ldr, w, eps, h, ldh);
  if (s != T2I_OK) return s;
  if (!q || !scale) return ops_fail(T2I_ERR_INVALID_ARG, "NULL pointer");
  if (ldq < i8_row(K) || ldq % 16)
    return ops_fail(T2I_ERR_SHAPE, "ldq must be a multiple of 16, at least K rounded up to 128");
  if (off(q, 16) || off(scale, 4)) return ops_fail(T2I_ERR_INVALID_ARG, "q needs 16-byte, scale 4-byte alignment");
  return done(launch_add_rms_norm(dtype == T2I_BF16, resid_dtype == T2I_BF16, true,
                                  make_norm(rows, K, x, ldx, resid, ldr, w, eps, h, ldh, q, ldq, scale),
                                  (hipStream_t)stream));
}

size_t t2i_op_add_rms_norm_backward_ws_bytes(int32_t rows, int32_t K) {
  return bad_sizes(rows, K) ? 0 : norm_bwd_ws_bytes(rows, K);
}

t2i_status t2i_op_add_rms_norm_backward(int32_t dtype, int32_t resid_dtype, int32_t rows, int32_t K, const void* dy,
                                        int32_t lddy, const void* h, int32_t ldh, const void* w, float eps,
                                        const void* dh, int32_t lddh, void* dx, int32_t lddx, void* dresid,
                                        int32_t lddr, void* dw, void* ws, size_t ws_bytes, void* stream) {
  if (bad_dtype(dtype) || bad_dtype(resid_dtype)) return ops_fail(T2I_ERR_INVALID_ARG, "bad dtype");
  if (resid_dtype != dtype && resid_dtype != T2I_F32)
    return ops_fail(T2I_ERR_INVALID_ARG, "the residual has the operands' type or fp32");
  if (bad_sizes(rows, K)) return ops_fail(T2I_ERR_SHAPE, "bad shape");
  if (!dy || !h || !dx) return ops_fail(T2I_ERR_INVALID_ARG, "NULL pointer");
  if (lddy < K || ldh < K || lddx < K || (dh && lddh < K) || (dresid && lddr < K))
    return ops_fail(T2I_ERR_SHAPE, "leading dimension < K");
  const size_t e = bytes_of(dtype), re = bytes_of(resid_dtype);
  if (off(dy, e) || off(w, e) || off(dx, e) || off(dw, e) || off(h, re) || off(dh, re) || off(dresid, re) ||
      (dw && off(ws, 256)))
    return ops_fail(T2I_ERR_INVALID_ARG, "operands need the alignment of their type, ws 256 bytes");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return ops_fail(T2I_ERR_INVALID_ARG, "eps must be finite, >= 0");
  const size_t need = dw ? norm_bwd_ws_bytes(rows, K) : 0;
  if (need && (!ws || ws_bytes < need)) return ops_fail(T2I_ERR_WORKSPACE, "workspace too small");
  NormBwd a;
  std::memset(&a, 0, sizeof(a));
  a.rows = rows;
  a.K = K;
  a.dy = dy;
  a.lddy = lddy;
  a.h = h;
  a.ldh = ldh;
  a.w = w;
  a.eps = eps;
  a.dh = dh;
  a.lddh = lddh;
  a.dx = dx;
  a.lddx = lddx;
  a.dresid = dresid;
  a.lddr = lddr;
  a.dw = dw;
  return done(launch_add_rms_norm_bwd(dtype == T2I_BF16, resid_dtype == T2I_BF16, a, dw ? (float*)ws : nullptr,
                                      (hipStream_t)stream));
}

}  // extern "C"
