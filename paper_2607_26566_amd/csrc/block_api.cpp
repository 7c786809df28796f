// Entry points of the block operators: argument checks, then the launches.
#include <cmath>
#include <cstring>

#include "block_ops.h"

using namespace t2i;

namespace {

bool bad_dtype(int32_t d) { return d != T2I_F32 && d != T2I_BF16; }
bool off(const void* p, size_t n) { return (uintptr_t)p % n != 0; }
// a launch holds fewer than 2^32 threads: the tiles that many outputs may take have at most
// 512 for 64 x 64 of them
bool too_large(int64_t M, int64_t N) { return ((M + 63) / 64) * ((N + 63) / 64) >= 1 << 23; }
// (fewer than 2^32 threads, of which a head takes less than a fourth of its elements)
bool too_many_heads(int64_t rows, int64_t hq, int64_t hk, int64_t d) {
  return rows * (hq + hk) > 0x7fffffff || rows * (hq + hk) * d >= 1LL << 34;
}
// the kernels address up to 256 rows of an operand with 32-bit byte offsets
bool far_rows(int32_t ld, size_t elem) { return (int64_t)ld * (int64_t)elem * 256 > 0x7fffffff; }
t2i_status done(hipError_t e) {
  return e == hipSuccess ? T2I_OK : ops_fail(T2I_ERR_DEVICE, hipGetErrorString(e));
}

t2i_status check_qk(int32_t dtype, int32_t rows, int32_t hq, int32_t hk, int32_t d, const void* q,
                    int32_t ldq, const void* k, int32_t ldk, const void* wq, const void* wk, float eps,
                    int32_t pairing, const float* table, int32_t n_pos, const int32_t* pos,
                    const void* oq, int32_t ldoq, const void* ok, int32_t ldok) {
  if (bad_dtype(dtype)) return ops_fail(T2I_ERR_INVALID_ARG, "bad dtype");
  if (pairing != T2I_ROPE_PAIRS && pairing != T2I_ROPE_HALVES)
    return ops_fail(T2I_ERR_INVALID_ARG, "bad pairing");
  if (rows < 1 || hq < 0 || hk < 0 || (int64_t)hq + hk < 1) return ops_fail(T2I_ERR_SHAPE, "no rows or no heads");
  if (d < 8 || d > 256 || d % 8) return ops_fail(T2I_ERR_SHAPE, "head_dim must be a multiple of 8 in 8 .. 256");
  if (pairing == T2I_ROPE_HALVES && d % 16)
    return ops_fail(T2I_ERR_SHAPE, "halves need head_dim % 16 == 0");
  if (too_many_heads(rows, hq, hk, d)) return ops_fail(T2I_ERR_SHAPE, "rows * heads past 2^31, or elements past 2^34");
  if ((hq && (!q || !oq)) || (hk && (!k || !ok))) return ops_fail(T2I_ERR_INVALID_ARG, "NULL pointer");
  if ((hq && (ldq < (int64_t)hq * d || ldoq < (int64_t)hq * d || ldq % 8 || ldoq % 8)) ||
      (hk && (ldk < (int64_t)hk * d || ldok < (int64_t)hk * d || ldk % 8 || ldok % 8)))
    return ops_fail(T2I_ERR_SHAPE, "bad leading dimension");
  if ((hq && (off(q, 16) || off(oq, 16))) || (hk && (off(k, 16) || off(ok, 16))) || off(wq, 16) ||
      off(wk, 16) || off(table, 16) || off(pos, 4))
    return ops_fail(T2I_ERR_INVALID_ARG, "pointers need 16-byte alignment (pos: 4)");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return ops_fail(T2I_ERR_INVALID_ARG, "eps must be finite, >= 0");
  if (table && (n_pos < 1 || (!pos && n_pos < rows)))
    return ops_fail(T2I_ERR_SHAPE, "the table is shorter than the rows");
  return T2I_OK;
}

QkNorm make_qk(int32_t rows, int32_t hq, int32_t hk, int32_t d, const void* q, int32_t ldq, const void* k,
               int32_t ldk, const void* wq, const void* wk, float eps, int32_t pairing,
               const float* table, int32_t n_pos, const int32_t* pos, void* oq, int32_t ldoq, void* ok,
               int32_t ldok) {
  QkNorm a;
  std::memset(&a, 0, sizeof(a));
  a.rows = rows;
  a.heads_q = hq;
  a.heads_k = hk;
  a.head_dim = d;
  a.q = q;
  a.k = k;
  a.ldq = ldq;
  a.ldk = ldk;
  a.wq = wq;
  a.wk = wk;
  a.eps = eps;
  a.halves = pairing == T2I_ROPE_HALVES;
  a.table = (const float2*)table;
  a.n_pos = n_pos;
  a.pos = pos;
  a.oq = oq;
  a.ok = ok;
  a.ldoq = ldoq;
  a.ldok = ldok;
  return a;
}

size_t gated_dgu_bytes(int32_t dtype, int32_t M, int32_t F) {
  return ((size_t)M * 2 * gated_cols(F) * (dtype == T2I_BF16 ? 2 : 4) + 255) / 256 * 256;
}

}  // namespace

extern "C" {

t2i_status t2i_op_quant_rows(int32_t dtype, int32_t rows, int32_t K, const void* x, int32_t ldx,
                             int8_t* q, int32_t ldq, float* scale, void* stream) {
  if (bad_dtype(dtype)) return ops_fail(T2I_ERR_INVALID_ARG, "bad dtype");
  // (fewer than 2^32 threads: a wave per row up to K = 2048, a workgroup for longer ones)
  if (rows < 1 || K < 1 || K > (1 << 30) || rows >= (K <= 2048 ? 1 << 26 : 1 << 24) - 4)
    return ops_fail(T2I_ERR_SHAPE, "bad shape");
  if (!x || !q || !scale) return ops_fail(T2I_ERR_INVALID_ARG, "NULL pointer");
  if (ldx < K) return ops_fail(T2I_ERR_SHAPE, "leading dimension < K");
  if (ldq < i8_row(K) || ldq % 16)
    return ops_fail(T2I_ERR_SHAPE, "ldq must be a multiple of 16, at least K rounded up to 128");
  if (off(x, dtype == T2I_BF16 ? 2 : 4) || off(q, 16) || off(scale, 4))
    return ops_fail(T2I_ERR_INVALID_ARG, "q needs 16-byte alignment, x and scale that of their type");
  return done(launch_quant_rows(dtype == T2I_BF16, rows, K, x, ldx, q, ldq, scale, (hipStream_t)stream));
}

t2i_status t2i_op_linear_i8(int32_t dtype, int32_t epilogue, int32_t M, int32_t N, int32_t K,
                            const int8_t* A, int32_t lda, const float* a_scale, const int8_t* W,
                            int32_t ldw, const float* w_scale, const void* bias, void* out,
                            int32_t ldo, float* resid, int32_t ldr, void* resid_copy,
                            const float* gate, void* stream) {
  if (bad_dtype(dtype)) return ops_fail(T2I_ERR_INVALID_ARG, "bad dtype");
  if (epilogue < T2I_EPI_STORE || epilogue > T2I_EPI_RESID_GATED)
    return ops_fail(T2I_ERR_INVALID_ARG, "bad epilogue");
  if (M < 1 || N < 1 || K < 1 || too_large(M, N)) return ops_fail(T2I_ERR_SHAPE, "bad shape");
  if (K > 131071) return ops_fail(T2I_ERR_SHAPE, "K past 131071: the sums would pass 32 bits");
  if (!A || !W || !a_scale || !w_scale) return ops_fail(T2I_ERR_INVALID_ARG, "NULL operand");
  if (lda < i8_row(K) || ldw < i8_row(K) || lda % 16 || ldw % 16)
    return ops_fail(T2I_ERR_SHAPE, "lda, ldw must be multiples of 16, at least K rounded up to 128");
  if (far_rows(lda, 1) || far_rows(ldw, 1)) return ops_fail(T2I_ERR_SHAPE, "rows more than 8 MiB apart");
  const bool res = epilogue >= T2I_EPI_RESID;
  if (res && (!resid || ldr < N)) return ops_fail(T2I_ERR_INVALID_ARG, "bad residual");
  if (!res && (!out || ldo < N)) return ops_fail(T2I_ERR_INVALID_ARG, "bad out");
  if (epilogue == T2I_EPI_RESID_GATED && !gate) return ops_fail(T2I_ERR_INVALID_ARG, "NULL gate");
  const size_t e = dtype == T2I_BF16 ? 2 : 4;
  if (off(A, 16) || off(W, 16) || off(a_scale, 4) || off(w_scale, 4) || off(bias, e) ||
      (!res && off(out, e)) ||
      (res && (off(resid, 4) || off(resid_copy, 2) || (epilogue == T2I_EPI_RESID_GATED && off(gate, 4)))))
    return ops_fail(T2I_ERR_INVALID_ARG, "A, W need 16-byte alignment, the others that of their type");
  I8Epi p;
  std::memset(&p, 0, sizeof(p));
  p.kind = epilogue;
  p.bf16_out = dtype == T2I_BF16;
  p.sa = a_scale;
  p.sw = w_scale;
  p.bias = bias;
  p.out = out;
  p.ldo = ldo;
  p.x = resid;
  p.ldx = ldr;
  p.xb = (bf16*)resid_copy;
  p.gate = gate;
  return done(launch_linear_i8(A, lda, W, ldw, M, N, K, p, (hipStream_t)stream));
}

t2i_status t2i_op_gated_linear(int32_t dtype, int32_t act, int32_t M, int32_t F, int32_t K,
                               const void* A, int32_t lda, const void* Wg, const void* Wu,
                               int32_t ldw, const void* bg, const void* bu, void* out, int32_t ldo,
                               float* pre, int32_t ldp, void* stream) {
  if (bad_dtype(dtype)) return ops_fail(T2I_ERR_INVALID_ARG, "bad dtype");
  if (act != T2I_EPI_GELU && act != T2I_EPI_SILU)
    return ops_fail(T2I_ERR_INVALID_ARG, "act must be T2I_EPI_GELU or T2I_EPI_SILU");
  if (M < 1 || F < 1 || K < 1 || K > (1 << 30) || F > (1 << 28) || too_large(M, 2LL * F))
    return ops_fail(T2I_ERR_SHAPE, "bad shape");
  if (!A || !Wg || !Wu || !out) return ops_fail(T2I_ERR_INVALID_ARG, "NULL operand");
  if (!bg != !bu) return ops_fail(T2I_ERR_INVALID_ARG, "bg and bu go together");
  if (lda < K || ldw < K || ldo < F || (pre && ldp < 2 * F))
    return ops_fail(T2I_ERR_SHAPE, "bad leading dimension");
  const bool bf = dtype == T2I_BF16;
  if (bf && (F % 8 || K % 8 || lda % 8 || ldw % 8 || ldo % 8 || (pre && ldp % 4)))
    return ops_fail(T2I_ERR_SHAPE, "bf16 needs F, K and strides % 8 == 0 (pre: 4)");
  if (far_rows(lda, bf ? 2 : 4) || far_rows(ldw, bf ? 2 : 4)) return ops_fail(T2I_ERR_SHAPE, "rows more than 8 MiB apart");
  const size_t al = bf ? 16 : 4;
  if (off(A, al) || off(Wg, al) || off(Wu, al) || off(bg, al) || off(bu, al) || off(out, al) || off(pre, al))
    return ops_fail(T2I_ERR_INVALID_ARG, "pointers need 16-byte (bf16) or 4-byte (fp32) alignment");
  GatedFwd g;
  std::memset(&g, 0, sizeof(g));
  g.act = act;
  g.A = A;
  g.Wg = Wg;
  g.Wu = Wu;
  g.bg = bg;
  g.bu = bu;
  g.lda = lda;
  g.ldw = ldw;
  g.out = out;
  g.ldo = ldo;
  g.pre = pre;
  g.ldp = ldp;
  return done(launch_gated_linear(bf, g, M, F, K, (hipStream_t)stream));
}

size_t t2i_op_gated_linear_backward_ws_bytes(int32_t dtype, int32_t M, int32_t F, int32_t K) {
  if (bad_dtype(dtype) || M < 1 || F < 1 || K < 1 || K > (1 << 30) || F > (1 << 28) || too_large(M, 2LL * F) ||
      too_large(M, K) || too_large(2LL * F, K))
    return 0;
  // dg | du, the bias gradients' column sums, the products' partial sums
  const size_t partial = ((size_t)gate_row_blocks(M, F) * 2 * gated_cols(F) * 4 + 255) / 256 * 256;
  return gated_dgu_bytes(dtype, M, F) + partial + gated_split_floats(dtype == T2I_BF16, M, F, K) * 4;
}

t2i_status t2i_op_gated_linear_backward(int32_t dtype, int32_t act, int32_t M, int32_t F, int32_t K,
                                        const void* A, int32_t lda, const void* Wg, const void* Wu,
                                        int32_t ldw, const float* pre, int32_t ldp, const void* dout,
                                        int32_t ldd, void* dA, int32_t ldda, void* dWg, void* dWu,
                                        int32_t lddw, void* dbg, void* dbu, void* ws, size_t ws_bytes,
                                        void* stream) {
  if (bad_dtype(dtype)) return ops_fail(T2I_ERR_INVALID_ARG, "bad dtype");
  if (act != T2I_EPI_GELU && act != T2I_EPI_SILU)
    return ops_fail(T2I_ERR_INVALID_ARG, "act must be T2I_EPI_GELU or T2I_EPI_SILU");
  if (M < 1 || F < 1 || K < 1 || K > (1 << 30) || F > (1 << 28) || too_large(M, 2LL * F) || too_large(M, K) ||
      too_large(2LL * F, K))
    return ops_fail(T2I_ERR_SHAPE, "bad shape");
  if (!A || !Wg || !Wu || !pre || !dout || !ws) return ops_fail(T2I_ERR_INVALID_ARG, "NULL operand");
  if (!dbg != !dbu) return ops_fail(T2I_ERR_INVALID_ARG, "dbg and dbu go together");
  if (!dA && !dWg && !dWu && !dbg) return ops_fail(T2I_ERR_INVALID_ARG, "no gradient asked for");
  const bool dw = dWg || dWu;
  if (lda < K || ldw < K || ldp < 2 * F || ldd < F || (dA && ldda < K) || (dw && lddw < K))
    return ops_fail(T2I_ERR_SHAPE, "bad leading dimension");
  const bool bf = dtype == T2I_BF16;
  if (bf && (F % 8 || K % 8 || lda % 8 || ldw % 8 || ldp % 4 || ldd % 8 || (dA && ldda % 8) ||
             (dw && lddw % 8)))
    return ops_fail(T2I_ERR_SHAPE, "bf16 needs F, K and strides % 8 == 0 (pre: 4)");
  if (far_rows(lda, bf ? 2 : 4) || far_rows(ldw, bf ? 2 : 4) || far_rows(gated_cols(F), bf ? 4 : 8))
    return ops_fail(T2I_ERR_SHAPE, "rows more than 8 MiB apart");
  const size_t al = bf ? 16 : 4;
  if (off(A, al) || off(Wg, al) || off(Wu, al) || off(pre, al) || off(dout, al) || off(dA, al) ||
      off(dWg, al) || off(dWu, al) || off(dbg, al) || off(dbu, al) || off(ws, 256))
    return ops_fail(T2I_ERR_INVALID_ARG,
                    "pointers need 16-byte (bf16) or 4-byte (fp32) alignment, ws 256-byte");
  if (ws_bytes < t2i_op_gated_linear_backward_ws_bytes(dtype, M, F, K))
    return ops_fail(T2I_ERR_WORKSPACE, "workspace too small");
  hipStream_t st = (hipStream_t)stream;
  float* partial = (float*)((char*)ws + gated_dgu_bytes(dtype, M, F));
  float* slices = partial + ((size_t)gate_row_blocks(M, F) * 2 * gated_cols(F) + 63) / 64 * 64;
  hipError_t e = launch_gate_grad(bf, act, M, F, pre, ldp, dout, ldd, ws, dbg ? partial : nullptr, st);
  if (e == hipSuccess && dbg) e = launch_gate_bias_grad(bf, M, F, partial, dbg, dbu, st);
  if (e == hipSuccess && dA) e = launch_gated_dx(bf, M, F, K, ws, Wg, Wu, ldw, dA, ldda, slices, st);
  if (e == hipSuccess && dw) e = launch_gated_dw(bf, M, F, K, ws, A, lda, dWg, dWu, lddw, slices, st);
  return done(e);
}

t2i_status t2i_op_qk_norm_rope(int32_t dtype, int32_t rows, int32_t heads_q, int32_t heads_k,
                               int32_t head_dim, const void* q, int32_t ldq, const void* k,
                               int32_t ldk, const void* wq, const void* wk, float eps,
                               int32_t pairing, const float* table, int32_t n_pos, const int32_t* pos,
                               void* q_out, int32_t ldqo, void* k_out, int32_t ldko, void* stream) {
  const t2i_status s = check_qk(dtype, rows, heads_q, heads_k, head_dim, q, ldq, k, ldk, wq, wk, eps,
                                pairing, table, n_pos, pos, q_out, ldqo, k_out, ldko);
  if (s != T2I_OK) return s;
  const QkNorm a = make_qk(rows, heads_q, heads_k, head_dim, q, ldq, k, ldk, wq, wk, eps, pairing, table,
                           n_pos, pos, q_out, ldqo, k_out, ldko);
  return done(launch_qk_norm_rope(dtype == T2I_BF16, a, (hipStream_t)stream));
}

size_t t2i_op_qk_norm_rope_backward_ws_bytes(int32_t rows, int32_t heads_q, int32_t heads_k,
                                             int32_t head_dim) {
  if (rows < 1 || heads_q < 0 || heads_k < 0 || (int64_t)heads_q + heads_k < 1 || head_dim < 8 ||
      head_dim > 256 || head_dim % 8 || too_many_heads(rows, heads_q, heads_k, head_dim))
    return 0;
  return (size_t)qk_bwd_blocks(rows, heads_q + heads_k, head_dim) * 2 * head_dim * 4;
}

t2i_status t2i_op_qk_norm_rope_backward(int32_t dtype, int32_t rows, int32_t heads_q, int32_t heads_k,
                                        int32_t head_dim, const void* dq, int32_t lddq, const void* dk,
                                        int32_t lddk, const void* q, int32_t ldq, const void* k,
                                        int32_t ldk, const void* wq, const void* wk, float eps,
                                        int32_t pairing, const float* table, int32_t n_pos,
                                        const int32_t* pos, void* dq_in, int32_t lddqi, void* dk_in,
                                        int32_t lddki, void* dwq, void* dwk, void* ws, size_t ws_bytes,
                                        void* stream) {
  const t2i_status s = check_qk(dtype, rows, heads_q, heads_k, head_dim, q, ldq, k, ldk, wq, wk, eps,
                                pairing, table, n_pos, pos, dq_in, lddqi, dk_in, lddki);
  if (s != T2I_OK) return s;
  if ((heads_q && !dq) || (heads_k && !dk)) return ops_fail(T2I_ERR_INVALID_ARG, "NULL gradient");
  if ((heads_q && (lddq < heads_q * head_dim || lddq % 8)) ||
      (heads_k && (lddk < heads_k * head_dim || lddk % 8)))
    return ops_fail(T2I_ERR_SHAPE, "bad leading dimension");
  const bool dw = dwq || dwk;
  const size_t e = dtype == T2I_BF16 ? 2 : 4;
  if ((heads_q && off(dq, 16)) || (heads_k && off(dk, 16)) || off(dwq, e) || off(dwk, e) ||
      (dw && off(ws, 256)))
    return ops_fail(T2I_ERR_INVALID_ARG, "gradients need 16-byte, ws 256-byte alignment");
  if (dw && (!ws || ws_bytes < t2i_op_qk_norm_rope_backward_ws_bytes(rows, heads_q, heads_k, head_dim)))
    return ops_fail(T2I_ERR_WORKSPACE, "workspace too small");
  QkNorm a = make_qk(rows, heads_q, heads_k, head_dim, q, ldq, k, ldk, wq, wk, eps, pairing, table, n_pos,
                     pos, dq_in, lddqi, dk_in, lddki);
  a.dq = dq;
  a.dk = dk;
  a.lddq = lddq;
  a.lddk = lddk;
  hipStream_t st = (hipStream_t)stream;
  const bool bf = dtype == T2I_BF16;
  hipError_t err = launch_qk_norm_rope_bwd(bf, a, dw ? (float*)ws : nullptr, st);
  if (err == hipSuccess && dw)
    err = launch_qk_weight_grad(bf, qk_bwd_blocks(rows, heads_q + heads_k, head_dim), head_dim,
                                (const float*)ws, dwq, dwk, st);
  return done(err);
}

}  // extern "C"
