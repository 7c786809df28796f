// Block operators: 8-bit linear layer, gated feed-forward, query / key norm
// with rotation; the residual's addition with an RMS norm, low-rank adapters beside
// a shared layer, AdamW.  Launchers (asynchronous on `st`; arguments checked by the
// entry points in block_api.cpp; norm_api.cpp, adapter_api.cpp, adamw_api.cpp).
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

// ---- the residual's addition with an RMS norm

struct NormFwd {
  int rows, K;
  const void* x;
  int ldx;
  const void* resid;                 // or NULL: the norm of x
  int ldr;
  const void* w;                     // or NULL: ones
  float eps;
  void* h;                           // with resid
  int ldh;
  void* y;                           // or the codes
  int ldy;
  float* scale;                      // 8 bits
};
hipError_t launch_add_rms_norm(bool is_bf16, bool resid_bf16, bool to_i8, const NormFwd& a, hipStream_t st);

struct NormBwd {
  int rows, K;
  const void* dy;
  int lddy;
  const void* h;
  int ldh;
  const void* w;                     // or NULL
  float eps;
  const void* dh;                    // or NULL
  int lddh;
  void* dx;
  int lddx;
  void* dresid;                      // or NULL
  int lddr;
  void* dw;                          // or NULL
};
// workgroups of the kernel that walks the rows: rows of its partial sums [blocks][K]
int norm_bwd_blocks(bool is_bf16, int rows, int K);
size_t norm_bwd_ws_bytes(int rows, int K);
// ws: only with dw
hipError_t launch_add_rms_norm_bwd(bool is_bf16, bool resid_bf16, const NormBwd& a, float* ws, hipStream_t st);

// ---- low-rank adapters of many requests beside a shared linear layer

// columns of t and of the gradients' u: rank rounded up, zeros behind it
__host__ __device__ inline int adapter_cols(int rank) { return (rank + 31) / 32 * 32; }

// t = s x a^T: x [M, K], a [n][rank][K], t fp32 [M][ldt], ldt >= adapter_cols(rank)
struct AdapterDown {
  int M, K, n, rank;
  const void* x;
  int ldx;
  const void* a;
  const float* scale;                // [n] or NULL: ones
  const int32_t* index;              // [M] or NULL: adapter 0
  float* t;
  int ldt;
};
hipError_t launch_adapter_down(bool is_bf16, const AdapterDown& p, hipStream_t st);

// the product with the adapters' second matrices p [n][columns][stride], `rank` of which
// count
struct AdapterUp {
  const int32_t* index;
  int n, rank, stride;
  const void* p;
  const float* t;
  int ldt;
};
struct LinearEpi {
  int kind;                          // EPI_STORE .. EPI_RESID_GATED
  const void* bias;                  // or NULL
  void* out;
  int ldo;
  float* x;                          // residual
  int ldx;
  bf16* xb;                          // or NULL
  const float* gate;
};
hipError_t launch_adapter_linear(bool is_bf16, const void* x, int ldx, const void* w, int ldw, int M, int N, int K,
                                 const AdapterUp& up, const LinearEpi& e, hipStream_t st);
// dx = dy W + u A; fp32 room that it needs at `partial`
size_t adapter_dx_floats(bool is_bf16, int M, int N, int K);
hipError_t launch_adapter_dx(bool is_bf16, const void* dy, int lddy, const void* w, int ldw, int M, int N, int K,
                             const AdapterUp& up, void* dx, int ldx, float* partial, hipStream_t st);
// the gradients' first launch: the rows of every adapter, slices of at most `per` of them
// (groups = n, or 0 without an index), matrices turned: out [n][C][stride] = in
// [n][R][C], zeros behind R (in NULL: none), and u [M][adapter_cols(rank)] = s dy b (dy
// NULL: not)
int adapter_slice_rows(bool is_bf16, int M, int N, int K, int n, int rank);
struct AdapterTurn {
  const void* in;
  void* out;
  int R, C, stride, blocks;
};
struct AdapterPrepare {
  const int32_t* index;
  int M, n, per, groups;
  int32_t* order;
  int2* span;
  int4* slices;
  AdapterTurn turn[2];
  const void *dy, *b;
  const float* scale;
  float* u;
  int lddy, N, rank, rows;
};
bool adapter_few_rows(int M, int N, int rank);
hipError_t launch_adapter_prepare(bool is_bf16, AdapterPrepare p, hipStream_t st);
// dA, dB (either may be NULL)
struct AdapterSide {
  const void* z;                     // [M, cols]
  const float* v;                    // [M, ldv]
  int ldz, ldv, cols;
  float* partial;                    // [places][ranks][ldp]
  int ldp;                           // cols in whole pieces of eight
  void* grad;                        // set by the launch: dA, dB
};
struct AdapterOuter {
  AdapterSide side[2];               // dA: (x, u), dB: (dy, t)
  int M, per, rank, ranks;           // ranks: rank in whole pieces of four
  int blocks0;
  const int32_t* order;              // NULL: all rows are adapter 0's
  const int2* span;
  const int4* slices;
};
int adapter_slices(bool indexed, int M, int n, int per);
int adapter_places(int M, int per);
hipError_t launch_adapter_outer(bool is_bf16, const AdapterOuter& p, int n, void* dA, void* dB, hipStream_t st);

// ---- AdamW over many tensors

constexpr int kAdamTensors = 64;       // of a launch, by value
struct AdamGroup {
  void* p[kAdamTensors];
  const void* g[kAdamTensors];
  float *m[kAdamTensors], *v[kAdamTensors], *master[kAdamTensors];
  int64_t numel[kAdamTensors];
  int32_t first[kAdamTensors + 1];     // a tensor's first workgroup
  int32_t n;
};
struct AdamScalars {
  double beta1, beta2;
  float b1, b2, c1, c2;                // c = 1 - b
  float r1, r2;                        // 1 / (1 - beta^step), unless step is given
  float lr, eps, wd;
  const float* lr_dev;                 // or NULL
  const int32_t* step;                 // or NULL
  const float* grad_scale;             // or NULL
};
static_assert(sizeof(AdamGroup) + sizeof(AdamScalars) <= 4096, "kernel arguments");
// low: bf16 weights with masters
hipError_t launch_adamw(bool low, bool grad_bf16, const AdamGroup& a, const AdamScalars& s, hipStream_t st);

}  // namespace t2i
