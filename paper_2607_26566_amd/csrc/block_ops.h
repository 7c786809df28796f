// Block operators: 8-bit linear layer, gated feed-forward, query / key norm
// with rotation.  Launchers (asynchronous on `st`; arguments checked by the
// entry points in block_api.cpp).
#pragma once

#include "t2i_internal.h"
#include "../../include/t2i_ops.h"

namespace t2i {

// text of t2i_ops_last_error (per host thread); returns s
t2i_status ops_fail(t2i_status s, const char* msg) noexcept;

// ---- 8-bit linear layer

// bytes of a quantised row that hold data or the zeros behind it
inline int i8_row(int K) { return (K + 127) / 128 * 128; }

hipError_t launch_quant_rows(bool bf16_in, int rows, int K, const void* x, int ldx, int8_t* q,
                             int ldq, float* scale, hipStream_t st);

// Epilogue of the 8-bit product: y = acc sa[m] sw[n] + bias[n], then as the
// linear layer's epilogues.  `bf16_out` is the type of out and bias.
struct I8Epi {
  int kind;              // EPI_STORE .. EPI_RESID_GATED
  int bf16_out;
  const float* sa;
  const float* sw;
  const void* bias;      // or NULL
  void* out;
  int ldo;
  float* x;              // residual
  int ldx;
  bf16* xb;              // or NULL
  const float* gate;
};
hipError_t launch_linear_i8(const int8_t* A, int lda, const int8_t* W, int ldw, int M, int N, int K,
                            const I8Epi& e, hipStream_t st);

// ---- gated feed-forward

// F rounded up to whole 64-column pieces: columns of each half of the
// workspace's [dg | du] rows, zeros behind F
inline int gated_cols(int F) { return (F + 63) / 64 * 64; }

struct GatedFwd {
  int act;               // EPI_GELU or EPI_SILU
  const void *A, *Wg, *Wu, *bg, *bu;   // biases or NULL
  int lda, ldw;
  void* out;
  int ldo;
  float* pre;            // or NULL: [M, 2F] pre-activations g | u
  int ldp;
};
hipError_t launch_gated_linear(bool is_bf16, const GatedFwd& a, int M, int F, int K, hipStream_t st);

// dgu [M][2 gated_cols(F)] and, when partial != NULL, the column sums of every
// row block: partial [gate_row_blocks(M, F)][2 gated_cols(F)]
int gate_row_blocks(int M, int F);
hipError_t launch_gate_grad(bool is_bf16, int act, int M, int F, const float* pre, int ldp,
                            const void* dout, int ldd, void* dgu, float* partial, hipStream_t st);
// dbg[f] / dbu[f] = sum of the partials, in ascending block order
hipError_t launch_gate_bias_grad(bool is_bf16, int M, int F, const float* partial, void* dbg,
                                 void* dbu, hipStream_t st);
// fp32 room that the two products below need at `partial`
size_t gated_split_floats(bool is_bf16, int M, int F, int K);
// dx [M, K] = dg Wg + du Wu
hipError_t launch_gated_dx(bool is_bf16, int M, int F, int K, const void* dgu, const void* Wg,
                           const void* Wu, int ldw, void* dx, int ldx, float* partial, hipStream_t st);
// dWg, dWu [F, K] = dg^T A, du^T A (either may be NULL)
hipError_t launch_gated_dw(bool is_bf16, int M, int F, int K, const void* dgu, const void* A, int lda,
                           void* dWg, void* dWu, int lddw, float* partial, hipStream_t st);

// For the tests, which assert that a shape reaches the tile it is there for (host
// arithmetic only): the tile of a product, its workgroups per CU and slices.
extern "C" int t2i_test_block_tile(int op, int is_bf16, int M, int F, int K, int* rows, int* columns, int* per_cu,
                                   int* slices);
// also for the tests: heads that a group takes in the head norm's kernels, rows that a
// workgroup takes in the gate gradients'
extern "C" int t2i_test_head_norm_heads(int rows, int heads, int head_dim, int backward);
extern "C" int t2i_test_gate_rows(int M, int F);

// ---- query / key norm with rotation

struct QkNorm {
  int rows, heads_q, heads_k, head_dim;
  const void *q, *k, *wq, *wk;       // weights or NULL
  int ldq, ldk;
  float eps;
  int halves;                        // pairs (j, j + d/2) instead of (2j, 2j + 1)
  const float2* table;               // [n_pos][d/2] or NULL: no rotation
  int n_pos;
  const int32_t* pos;                // [rows] or NULL: row r at position r
  void *oq, *ok;                     // outputs (backward: gradients of q, k)
  int ldoq, ldok;
  const void *dq, *dk;               // backward: gradients of the outputs
  int lddq, lddk;
};
hipError_t launch_qk_norm_rope(bool is_bf16, const QkNorm& a, hipStream_t st);
// workgroups of the backward kernel: rows of its partial sums [blocks][2][head_dim]
int qk_bwd_blocks(int rows, int heads, int head_dim);
hipError_t launch_qk_norm_rope_bwd(bool is_bf16, const QkNorm& a, float* partial, hipStream_t st);
hipError_t launch_qk_weight_grad(bool is_bf16, int blocks, int head_dim, const float* partial,
                                 void* dwq, void* dwk, hipStream_t st);

}  // namespace t2i
