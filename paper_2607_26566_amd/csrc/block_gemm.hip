// Matrix products of the block operators: the 8-bit linear layer, the gated
// feed-forward and its gradients.
//
// gemm_tile_kernel: one product C[m][n] = sum_k a(m, k) b(n, k) on 64 x 64
// tiles by 4 waves of 32 x 32 (v_mfma_f32_16x16x4_f32), 32 values of k at a
// time through LDS, the next step's operands fetched into registers under
// this step's MFMAs.  The operands are read by element through two functors,
// so any stride and size goes.
#include "block_ops.h"

namespace t2i {

// Elements of a row-major matrix, 0 outside [0, rows) x [0, cols).
// ALONG: the k axis runs along the rows (contiguous in memory).
template <typename T, bool ALONG>
struct Mat {
  static constexpr bool along = ALONG;
  const T* p;
  int ld, rows, cols;
  __device__ __forceinline__ float at(int r, int k) const {
    const int y = ALONG ? r : k, x = ALONG ? k : r;
    return y < rows && x < cols ? (float)p[(size_t)y * ld + x] : 0.f;
  }
};

// Gate and up weights side by side: of every 32 rows, 16 of the gate and the
// same 16 of the up projection, so that one lane ends up with both
template <typename T>
struct GateUp {
  static constexpr bool along = true;
  const T *g, *u;
  int ld, rows, cols;
  __device__ __forceinline__ float at(int r, int k) const {
    const int f = r / 32 * 16 + r % 16;
    return f < rows && k < cols ? (float)((r & 16) ? u : g)[(size_t)f * ld + k] : 0.f;
  }
};

// The gradients' operand [dg | du]^T... as rows of the contraction over both
// halves: k < Fp the gate's row k, else the up projection's row k - Fp
template <typename T>
struct TwoRows {
  static constexpr bool along = false;
  const T *g, *u;
  int ld, rows, cols, half;
  __device__ __forceinline__ float at(int n, int k) const {
    const int f = k < half ? k : k - half;
    return f < rows && n < cols ? (float)(k < half ? g : u)[(size_t)f * ld + n] : 0.f;
  }
};

template <bool INT, class LA, class LB, class EP>
__global__ __launch_bounds__(256) void gemm_tile_kernel(LA la, LB lb, EP ep, int tiles_n, int K) {
  constexpr int BK = 32, LD = 65;
  __shared__ float sA[BK][LD], sB[BK][LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1, fr = lane & 15, g = lane >> 4;
  const int m0 = (int)(blockIdx.x / (unsigned)tiles_n) * 64, n0 = (int)(blockIdx.x % (unsigned)tiles_n) * 64;
  float ra[8], rb[8];
  auto fetch = [&](int k0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int x = tid + i * 256;
      ra[i] = LA::along ? la.at(m0 + x / BK, k0 + x % BK) : la.at(m0 + x % 64, k0 + x / 64);
      rb[i] = LB::along ? lb.at(n0 + x / BK, k0 + x % BK) : lb.at(n0 + x % 64, k0 + x / 64);
    }
  };
  f32x4 acc[2][2];
  int iacc[2][2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int r = 0; r < 4; ++r) iacc[i][j][r] = 0;
    }
  fetch(0);
  for (int k0 = 0; k0 < K; k0 += BK) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int x = tid + i * 256;
      if (LA::along) sA[x % BK][x / BK] = ra[i]; else sA[x / 64][x % 64] = ra[i];
      if (LB::along) sB[x % BK][x / BK] = rb[i]; else sB[x / 64][x % 64] = rb[i];
    }
    __syncthreads();
    if (k0 + BK < K) fetch(k0 + BK);
#pragma unroll
    for (int kk = 0; kk < BK; kk += 4) {
      float a[2], b[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[i] = sA[kk + g][wm * 32 + i * 16 + fr];
        b[i] = sB[kk + g][wn * 32 + i * 16 + fr];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[j], a[i], acc[i][j], 0, 0, 0);
    }
    if (INT) {
      // 32 products of 8-bit values: below 2^24, exact in fp32
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            iacc[i][j][r] += (int)acc[i][j][r];
            acc[i][j][r] = 0.f;
          }
    }
  }
  // operands swapped: a lane holds row m0 + fr, four columns from g * 4
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float v[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) v[j] = INT ? (float)iacc[i][j][r] : acc[i][j][r];
      ep(m0 + wm * 32 + i * 16 + fr, n0 + wn * 32 + g * 4 + r, v);
    }
}

template <bool INT, class LA, class LB, class EP>
static hipError_t gemm_tile(const LA& la, const LB& lb, const EP& ep, int M, int N, int K, hipStream_t st) {
  const int tn = (N + 63) / 64;
  const long tiles = (long)((M + 63) / 64) * tn;
  hipLaunchKernelGGL((gemm_tile_kernel<INT, LA, LB, EP>), dim3((unsigned)tiles), dim3(256), 0, st, la, lb,
                     ep, tn, K);
  return hipGetLastError();
}

// ---- epilogues: v[0] column n, v[1] column n + 16

struct I8Store {
  I8Epi e;
  int M, N;
  __device__ __forceinline__ void one(int m, int n, float acc) const {
    if (m >= M || n >= N) return;
    float y = acc * e.sa[m] * e.sw[n];
    if (e.bias) y += e.bf16_out ? (float)((const bf16*)e.bias)[n] : ((const float*)e.bias)[n];
    if (e.kind == EPI_GELU) y = gelu_tanh(y);
    if (e.kind == EPI_SILU) y = silu(y);
    if (e.kind >= EPI_RESID) {
      const size_t i = (size_t)m * e.ldx + n;
      const float x = e.x[i] + (e.kind == EPI_RESID_GATED ? e.gate[n] : 1.f) * y;
      e.x[i] = x;
      if (e.xb) e.xb[i] = (bf16)x;
    } else if (e.bf16_out) {
      ((bf16*)e.out)[(size_t)m * e.ldo + n] = (bf16)y;
    } else {
      ((float*)e.out)[(size_t)m * e.ldo + n] = y;
    }
  }
  __device__ __forceinline__ void operator()(int m, int n, const float (&v)[2]) const {
    one(m, n, v[0]);
    one(m, n + 16, v[1]);
  }
};

template <typename T>
struct GatedStore {
  GatedFwd a;
  int M, F;
  __device__ __forceinline__ void operator()(int m, int n, const float (&v)[2]) const {
    const int f = n / 32 * 16 + n % 16;
    if (m >= M || f >= F) return;
    float g = v[0], u = v[1];
    if (a.bg) g += to_f32(((const T*)a.bg)[f]), u += to_f32(((const T*)a.bu)[f]);
    if (a.pre) {
      T* p = (T*)a.pre + (size_t)m * a.ldp + f;
      p[0] = from_f32<T>(g);
      p[F] = from_f32<T>(u);
    }
    ((T*)a.out)[(size_t)m * a.ldo + f] = from_f32<T>((a.act == EPI_GELU ? gelu_tanh(g) : silu(g)) * u);
  }
};

template <typename T>
struct PlainStore {
  T* p;
  int ld, rows, cols;
  __device__ __forceinline__ void operator()(int m, int n, const float (&v)[2]) const {
    if (m >= rows) return;
    if (n < cols) p[(size_t)m * ld + n] = from_f32<T>(v[0]);
    if (n + 16 < cols) p[(size_t)m * ld + n + 16] = from_f32<T>(v[1]);
  }
};

hipError_t launch_linear_i8(const int8_t* A, int lda, const int8_t* W, int ldw, int M, int N, int K,
                            const I8Epi& e, hipStream_t st) {
  return gemm_tile<true>(Mat<int8_t, true>{A, lda, M, K}, Mat<int8_t, true>{W, ldw, N, K}, I8Store{e, M, N},
                         M, N, K, st);
}

template <typename T>
static hipError_t gated_fwd(const GatedFwd& a, int M, int F, int K, hipStream_t st) {
  return gemm_tile<false>(Mat<T, true>{(const T*)a.A, a.lda, M, K},
                          GateUp<T>{(const T*)a.Wg, (const T*)a.Wu, a.ldw, F, K}, GatedStore<T>{a, M, F}, M,
                          (F + 15) / 16 * 32, K, st);
}

template <typename T>
static hipError_t gated_dx(int M, int F, int K, const void* dgu, const void* Wg, const void* Wu, int ldw,
                           void* dx, int ldx, hipStream_t st) {
  const int Fp = gated_cols(F);
  return gemm_tile<false>(Mat<T, true>{(const T*)dgu, 2 * Fp, M, 2 * Fp},
                          TwoRows<T>{(const T*)Wg, (const T*)Wu, ldw, F, K, Fp},
                          PlainStore<T>{(T*)dx, ldx, M, K}, M, K, 2 * Fp, st);
}

template <typename T>
static hipError_t gated_dw(int M, int F, int K, const void* dgu, const void* A, int lda, void* dWg,
                           void* dWu, int lddw, hipStream_t st) {
  const int Fp = gated_cols(F);
  for (int i = 0; i < 2; ++i) {
    T* o = (T*)(i ? dWu : dWg);
    if (!o) continue;
    const hipError_t e = gemm_tile<false>(Mat<T, false>{(const T*)dgu + i * Fp, 2 * Fp, M, F},
                                          Mat<T, false>{(const T*)A, lda, M, K},
                                          PlainStore<T>{o, lddw, F, K}, F, K, M, st);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_gated_linear(bool is_bf16, const GatedFwd& a, int M, int F, int K, hipStream_t st) {
  return is_bf16 ? gated_fwd<bf16>(a, M, F, K, st) : gated_fwd<float>(a, M, F, K, st);
}

hipError_t launch_gated_dx(bool is_bf16, int M, int F, int K, const void* dgu, const void* Wg,
                           const void* Wu, int ldw, void* dx, int ldx, hipStream_t st) {
  return is_bf16 ? gated_dx<bf16>(M, F, K, dgu, Wg, Wu, ldw, dx, ldx, st)
                 : gated_dx<float>(M, F, K, dgu, Wg, Wu, ldw, dx, ldx, st);
}

hipError_t launch_gated_dw(bool is_bf16, int M, int F, int K, const void* dgu, const void* A, int lda,
                           void* dWg, void* dWu, int lddw, hipStream_t st) {
  return is_bf16 ? gated_dw<bf16>(M, F, K, dgu, A, lda, dWg, dWu, lddw, st)
                 : gated_dw<float>(M, F, K, dgu, A, lda, dWg, dWu, lddw, st);
}

}  // namespace t2i
