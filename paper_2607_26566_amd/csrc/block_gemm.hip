// Matrix products of the block operators on the tiles of gemm_tile.h: the 8-bit
// linear layer, the gated feed-forward and its gradients.
#include <algorithm>

#include "block_gemm.h"

namespace t2i {

// ---- kernels

// one output of the 8-bit layer before the residual update
__device__ __forceinline__ float i8_value(int acc, float sa, float sw, float b, int kind) {
  const float y = fmaf((float)acc * sa, sw, b);
  return kind == EPI_GELU ? gelu_tanh(y) : kind == EPI_SILU ? silu(y) : y;
}

// The 8-bit linear layer: y = (sum of whole products) sa sw + b.  The sum is exact in
// 32 bits whatever the tile, so a row's result does not depend on the rows beside it.
// 7531 x 4608 x 1152 64 us, 66 with GELU (1.2 POP/s): nine k steps per tile, of which
// the first loads and 69 MB of stores take more than the products; 4096 x 4096 x 12288
// 156 - 177 us (2.3 - 2.6 POP/s).
template <class D, typename T, bool RES>
__global__ __launch_bounds__(D::THREADS, 1) void linear_i8_kernel(TileOperand a, TileOperand b, TileShape s,
                                                                  I8Epi e, int M, int N) {
  using P = TileProduct<D, ELEM_I8, false, false, false, false>;
  constexpr int THREADS = D::THREADS, NE = D::BM + (RES ? 3 : 2) * D::BN;
  __shared__ __attribute__((aligned(1024))) char smem[D::KG * D::RING + NE * 4];
  int tm, tn;
  tile_place(s, blockIdx.x, gridDim.x, tm, tn);
  const int m0 = tm * D::BM, n0 = tn * D::BN;
  auto value = [&](int x) -> float {
    if (x < D::BM) return e.sa[min(m0 + x, M - 1)];
    const int n = min(n0 + (x - D::BM) % D::BN, N - 1), which = (x - D::BM) / D::BN;
    if (which == 0) return e.sw[n];
    if (which == 1) return e.bias ? to_f32(((const T*)e.bias)[n]) : 0.f;
    return e.kind == EPI_RESID_GATED ? e.gate[n] : 1.f;
  };
  Staged<NE, THREADS, decltype(value)> st;
  st.fetch(value);
  typename P::Acc acc[D::TM][D::TN];
  const bool mine = P::run_groups(smem, a, b, s, m0, n0, acc);
  float* const ev = (float*)(smem + D::KG * D::RING);
  st.put(ev);
  tile_barrier();
  if (!mine) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, g = lane >> 4;
  const int mw = (wave / D::WGN) * D::WM, nw = (wave % D::WGN) * D::WN;
#pragma unroll
  for (int i = 0; i < D::TM; ++i) {
    const int ml = mw + i * 16 + fr, m = m0 + ml;
    if (m >= M) continue;
    const float sa = ev[ml];
#pragma unroll
    for (int j = 0; j < D::TN; ++j) {
      const int nl = nw + j * 16 + g * 4, n = n0 + nl, left = N - n;
      if (left <= 0) continue;
      const f32x4 sw = *(const f32x4*)(ev + D::BM + nl), bb = *(const f32x4*)(ev + D::BM + D::BN + nl);
      float y[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = i8_value(acc[i][j][r], sa, sw[r], bb[r], e.kind);
      if constexpr (RES) {
        float* x = e.x + (size_t)m * e.ldx + n;
        const f32x4 gt = *(const f32x4*)(ev + D::BM + 2 * D::BN + nl);
        float xv[4];
        if (left >= 4) {
          typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
          const any4 x4 = *(const any4*)x;
#pragma unroll
          for (int r = 0; r < 4; ++r) xv[r] = x4[r] + gt[r] * y[r];
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) xv[r] = r < left ? x[r] + gt[r] * y[r] : 0.f;
        }
        store4(x, left, xv);
        if (e.xb) store4(e.xb + (size_t)m * e.ldx + n, left, xv);
      } else {
        store4((T*)e.out + (size_t)m * e.ldo + n, left, y);
      }
    }
  }
}

// Both projections of the gated block on one tile of gate and up columns; a wave holds
// the same columns of both, so activation and product happen in registers and g and u
// go to memory only where the backward pass wants them.  8192 x 4608 x 1152 155 - 170
// us (1.0 - 1.1 PFLOP/s: 4.5 rounds of tiles in 5, 18 k steps each), 4096 x 10240 x 4096
// 515 - 530 us, one row of 10240 x 4096 33 us (the weights at 5.1 TB/s, a copy's rate).
template <class D, typename T, bool U>
__global__ __launch_bounds__(D::THREADS, 1) void gated_linear_kernel(TileOperand a, TileOperand b, TileShape s,
                                                                     GatedFwd p, int M, int F) {
  using P = TileProduct<D, elem_of<T>(), false, false, true, false, U>;
  constexpr int THREADS = D::THREADS, H = D::BN / 2, TH = D::TN / 2;
  __shared__ __attribute__((aligned(1024))) char smem[D::KG * D::RING + D::BN * 4];
  int tm, tn;
  tile_place(s, blockIdx.x, gridDim.x, tm, tn);
  const int m0 = tm * D::BM, f0 = tn * H;
  auto value = [&](int x) -> float {
    if (!p.bg) return 0.f;
    return to_f32(((const T*)(x < H ? p.bg : p.bu))[min(f0 + x % H, F - 1)]);
  };
  Staged<D::BN, THREADS, decltype(value)> st;
  st.fetch(value);
  typename P::Acc acc[D::TM][D::TN];
  const bool mine = P::run_groups(smem, a, b, s, m0, f0, acc);
  float* const ev = (float*)(smem + D::KG * D::RING);
  st.put(ev);
  tile_barrier();
  if (!mine) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, g = lane >> 4;
  const int mw = (wave / D::WGN) * D::WM, nw = (wave % D::WGN) * (D::WN / 2);
#pragma unroll
  for (int i = 0; i < D::TM; ++i) {
    const int m = m0 + mw + i * 16 + fr;
    if (m >= M) continue;
#pragma unroll
    for (int j = 0; j < TH; ++j) {
      const int fl = nw + j * 16 + g * 4, f = f0 + fl;
      const int left = sizeof(T) == 4 ? F - f : 4;   // (bf16: F % 8 == 0, four columns or none)
      if (f >= F) continue;
      const f32x4 bg = *(const f32x4*)(ev + fl), bu = *(const f32x4*)(ev + H + fl);
      float gv[4], uv[4], y[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        gv[r] = acc[i][j][r] + bg[r];
        uv[r] = acc[i][j + TH][r] + bu[r];
        y[r] = (p.act == EPI_GELU ? gelu_tanh(gv[r]) : silu(gv[r])) * uv[r];
      }
      if (p.pre) {
        float* q = p.pre + (size_t)m * p.ldp + f;
        store4(q, left, gv);
        store4(q + F, left, uv);
      }
      store4((T*)p.out + (size_t)m * p.ldo + f, left, y);
    }
  }
}

template <class D, typename T, bool U>
__global__ __launch_bounds__(D::THREADS, 1) void gated_dx_kernel(TileOperand a, TileOperand b, TileShape s, Split sp,
                                                                 T* dx, int ldx, int M, int K) {
  using P = TileProduct<D, elem_of<T>(), false, true, false, true, U>;
  __shared__ __attribute__((aligned(1024))) char smem[D::RING];
  int tm, tn;
  tile_place(s, blockIdx.x, gridDim.x, tm, tn);
  if (sp.partial) take_slice(sp, s);
  typename P::Acc acc[D::TM][D::TN];
  const int m0 = tm * D::BM, n0 = first_column<D, U>(tn, K);
  P::run(smem, a, b, s, m0, n0, acc);
  if (sp.partial)
    store_tile<D, P>(acc, sp.partial + (size_t)blockIdx.y * M * sp.ld, sp.ld, m0, n0, M, K);
  else
    store_tile<D, P>(acc, dx, ldx, m0, n0, M, K);
}

// row blocks [0, half) are the first output's, the others the second's (their
// operand lies `shift` bytes further)
template <class D, typename T, bool U>
__global__ __launch_bounds__(D::THREADS, 1) void gated_dw_kernel(TileOperand a, TileOperand b, TileShape s, Split sp,
                                                                 int half, int shift, T* d0, T* d1, int ldw,
                                                                 int F, int K) {
  using P = TileProduct<D, elem_of<T>(), true, true, false, false, U>;
  __shared__ __attribute__((aligned(1024))) char smem[D::RING];
  int tm, tn;
  tile_place(s, blockIdx.x, gridDim.x, tm, tn);
  if (sp.partial) take_slice(sp, s);
  const bool second = tm >= half;
  const int m0 = (second ? tm - half : tm) * D::BM;
  if (second) a.p += shift;
  typename P::Acc acc[D::TM][D::TN];
  const int n0 = first_column<D, U>(tn, K);
  P::run(smem, a, b, s, m0, n0, acc);
  if (sp.partial) {
    const size_t of = (size_t)blockIdx.y * (s.tiles_m / half) * F + (second ? F : 0);
    store_tile<D, P>(acc, sp.partial + of * sp.ld, sp.ld, m0, n0, F, K);
  } else {
    store_tile<D, P>(acc, second ? d1 : d0, ldw, m0, n0, F, K);
  }
}

// ---- launches
template <class D>
static void i8_launch(const TileOperand& a, const TileOperand& b, const I8Epi& e, int M, int N, int K, hipStream_t st) {
  const TileShape s = tile_shape<D>(M, N, i8_row(K) / 128, i8_row(K), 0);
  const dim3 grid((unsigned)(s.tiles_m * s.tiles_n));
  const bool res = e.kind >= EPI_RESID;
#define T2I_I8(T, RES)                                                                                         \
  hipLaunchKernelGGL((linear_i8_kernel<D, T, RES>), grid, dim3(D::THREADS), 0, st, a, b, s, e, M, N)
  if (e.bf16_out) {
    if (res) T2I_I8(bf16, true);
    else T2I_I8(bf16, false);
  } else {
    if (res) T2I_I8(float, true);
    else T2I_I8(float, false);
  }
#undef T2I_I8
}

hipError_t launch_linear_i8(const int8_t* A, int lda, const int8_t* W, int ldw, int M, int N, int K,
                            const I8Epi& e, hipStream_t st) {
  const TileOperand a{(const char*)A, nullptr, (uint32_t)lda, M, 0}, b{(const char*)W, nullptr, (uint32_t)ldw, N, 0};
  const int shape = tile_index(M, N, i8_row(K) / 128, 1.f);
  T2I_TILES_FWD(shape, i8_launch<D>(a, b, e, M, N, K, st))
  return hipGetLastError();
}

template <class D, typename T, bool U = false>
static void gated_fwd_launch(const GatedFwd& p, int M, int F, int K, hipStream_t st) {
  constexpr int e = sizeof(T), per = 128 / e;
  const TileOperand a{(const char*)p.A, nullptr, (uint32_t)e * p.lda, M, 0},
      b{(const char*)p.Wg, (const char*)p.Wu, (uint32_t)e * p.ldw, F, 0};
  const TileShape s = tile_shape<D>(M, 2 * F, (K + per - 1) / per, e * K, 0);
  hipLaunchKernelGGL((gated_linear_kernel<D, T, U>), dim3((unsigned)(s.tiles_m * s.tiles_n)), dim3(D::THREADS), 0, st, a,
                     b, s, p, M, F);
}

size_t gated_split_floats(bool is_bf16, int M, int F, int K) {
  auto floats = [](const SplitPick& p, long rows, long cols) -> size_t {
    return p.slices > 1 ? (size_t)p.slices * rows * whole4(cols) : 0;
  };
  return std::max({floats(split_dx(is_bf16, M, K, 2 * gated_cols(F)), M, K),
                   floats(split_dw(is_bf16, 2L * F, K, M), 2L * F, K), floats(split_dw(is_bf16, F, K, M), F, K)});
}

template <class D, typename T, bool U = false>
static void gated_dx_launch(int M, int F, int K, const void* dgu, const void* Wg, const void* Wu, int ldw, T* dx,
                            int ldx, const SplitPick& pick, const Split& sp, hipStream_t st) {
  constexpr int e = sizeof(T), per = 128 / e;
  const int Fp = gated_cols(F);
  const TileOperand a{(const char*)dgu, nullptr, 2u * e * Fp, M, 0},
      b{(const char*)Wg, (const char*)Wu, (uint32_t)e * ldw, F, K};
  const TileShape s = tile_shape<D>(M, K, 2 * Fp / per, 2 * e * Fp, Fp / per);
  hipLaunchKernelGGL((gated_dx_kernel<D, T, U>), dim3((unsigned)(s.tiles_m * s.tiles_n), pick.slices), dim3(D::THREADS), 0,
                     st, a, b, s, sp, dx, ldx, M, K);
  if (sp.partial) split_sum(sp, pick.slices, M, M, K, dx, dx, ldx, st);
}

template <class D, typename T, bool U = false>
static void gated_dw_launch(int M, int F, int K, const void* dgu, const void* A, int lda, T* dWg, T* dWu, int lddw,
                            const SplitPick& pick, const Split& sp, hipStream_t st) {
  constexpr int e = sizeof(T), per = 128 / e;
  const int Fp = gated_cols(F), n = dWg && dWu ? 2 : 1;
  T* const first = dWg ? dWg : dWu;
  const TileOperand a{(const char*)dgu + (dWg ? 0 : (size_t)e * Fp), nullptr, 2u * e * Fp, M, (F + 7) / 8 * 8},
      b{(const char*)A, nullptr, (uint32_t)e * lda, M, K};
  TileShape s = tile_shape<D>(F, K, (M + per - 1) / per, 0, 0);
  const int half = s.tiles_m;
  s.tiles_m *= n;
  hipLaunchKernelGGL((gated_dw_kernel<D, T, U>), dim3((unsigned)(s.tiles_m * s.tiles_n), pick.slices), dim3(D::THREADS), 0,
                     st, a, b, s, sp, half, e * Fp, first, dWu, lddw, F, K);
  if (sp.partial) split_sum(sp, pick.slices, (long)n * F, F, K, first, dWu, lddw, st);
}

hipError_t launch_gated_linear(bool is_bf16, const GatedFwd& p, int M, int F, int K, hipStream_t st) {
  const int shape = is_bf16 ? tile_index(M, 2L * F, (K + 63) / 64, 0.5f) : tile_index_f32(M, 2L * F, (K + 31) / 32);
  if (is_bf16) {
    T2I_TILES_FWD(shape, (gated_fwd_launch<D, bf16>(p, M, F, K, st)))
  } else if (f32_pieces({K, p.lda, p.ldw}, {p.A, p.Wg, p.Wu})) {
    T2I_TILES_F32_FWD(shape, (gated_fwd_launch<D, float>(p, M, F, K, st)))
  } else {
    T2I_TILES_F32_FWD(shape, (gated_fwd_launch<D, float, true>(p, M, F, K, st)))
  }
  return hipGetLastError();
}

hipError_t launch_gated_dx(bool is_bf16, int M, int F, int K, const void* dgu, const void* Wg, const void* Wu, int ldw,
                           void* dx, int ldx, float* partial, hipStream_t st) {
  const SplitPick pick = split_dx(is_bf16, M, K, 2 * gated_cols(F));
  const Split sp{pick.slices > 1 ? partial : nullptr, pick.per, (int)whole4(K)};
  if (is_bf16) {
    T2I_TILES(pick.shape, (gated_dx_launch<D, bf16>(M, F, K, dgu, Wg, Wu, ldw, (bf16*)dx, ldx, pick, sp, st)))
  } else if (f32_pieces({K, ldw}, {Wg, Wu})) {
    T2I_TILES_F32_DX(pick.shape, (gated_dx_launch<D, float>(M, F, K, dgu, Wg, Wu, ldw, (float*)dx, ldx, pick, sp, st)))
  } else {
    T2I_TILES_F32_DX(pick.shape,
                  (gated_dx_launch<D, float, true>(M, F, K, dgu, Wg, Wu, ldw, (float*)dx, ldx, pick, sp, st)))
  }
  return hipGetLastError();
}

hipError_t launch_gated_dw(bool is_bf16, int M, int F, int K, const void* dgu, const void* A, int lda, void* dWg,
                           void* dWu, int lddw, float* partial, hipStream_t st) {
  const long rows = (dWg && dWu ? 2L : 1L) * F;
  const SplitPick pick = split_dw(is_bf16, rows, K, M);
  const Split sp{pick.slices > 1 ? partial : nullptr, pick.per, (int)whole4(K)};
  if (is_bf16) {
    T2I_TILES(pick.shape,
              (gated_dw_launch<D, bf16>(M, F, K, dgu, A, lda, (bf16*)dWg, (bf16*)dWu, lddw, pick, sp, st)))
  } else if (f32_pieces({K, lda}, {A})) {
    T2I_TILES_F32_DW(pick.shape,
                  (gated_dw_launch<D, float>(M, F, K, dgu, A, lda, (float*)dWg, (float*)dWu, lddw, pick, sp, st)))
  } else {
    T2I_TILES_F32_DW(pick.shape, (gated_dw_launch<D, float, true>(M, F, K, dgu, A, lda, (float*)dWg, (float*)dWu, lddw,
                                                               pick, sp, st)))
  }
  return hipGetLastError();
}

// The tile and the slices (or groups of waves) that a product takes (op 0: 8-bit layer with F columns, 1:
// gated forward, 2: dx, 3: dWg and dWu, 4: adapters' forward of F columns, 5: their dx)
extern "C" int t2i_test_block_tile(int op, int is_bf16, int M, int F, int K, int* rows, int* columns, int* per_cu,
                                   int* slices) {
  if (M < 1 || F < 1 || K < 1 || op < 0 || op > 5) return 0;
  SplitPick p{0, 1, 0};
  const bool f32 = op != 0 && !is_bf16;
  if (op == 4) p.shape = adapter_tile(is_bf16, M, F, K);
  else if (op == 5) p = adapter_dx_pick(is_bf16, M, F, K);
  else if (op == 0) p.shape = tile_index(M, F, i8_row(K) / 128, 1.f);
  else if (op == 1) p.shape = f32 ? tile_index_f32(M, 2L * F, (K + 31) / 32) : tile_index(M, 2L * F, (K + 63) / 64, 0.5f);
  else p = op == 2 ? split_dx(is_bf16, M, K, 2 * gated_cols(F)) : split_dw(is_bf16, 2L * F, K, M);
  if (!f32 && p.shape == kTile16n) {
    *rows = *columns = 16;
    *per_cu = 1;
    *slices = 8;
    return 1;
  }
  if (!f32 && p.shape >= kTile192) {
    *rows = p.shape == kTile192 ? 192 : 256;
    *columns = p.shape == kTile192 ? 256 : 192;
    *per_cu = *slices = 1;
    return 1;
  }
  const bool stream = !f32 && p.shape == kStream;   // four stages, one workgroup per CU
  const TileChoice& c = f32 ? kTilesF32[p.shape] : kTiles[stream ? kTile32 : p.shape];
  *rows = c.bm;
  *columns = c.bn;
  *per_cu = stream ? 1 : c.per_cu;
  const int group = p.shape - (f32 ? kF32Groups : kTile32k);
  *slices = p.slices > 1 || op == 2 || op == 3 ? p.slices : group == 0 ? Tile32k::KG : group == 1 ? Tile16k::KG : 1;
  return 1;
}

}  // namespace t2i
