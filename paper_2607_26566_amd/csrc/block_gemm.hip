// Matrix products of the block operators on the tiles of gemm_tile.h: the 8-bit
// linear layer, the gated feed-forward and its gradients.
#include <algorithm>
#include <initializer_list>

#include "gemm_tile.h"

namespace t2i {

// ---- tile shapes.  `per_cu` workgroups of a shape share a CU.  A launch of n
// tiles takes rounds of 256 per_cu; a round takes `full` us per k step and `end` us
// for its first loads and its epilogue, the last one `alone` per step if it has 256
// tiles or fewer, and in between what lies between.
struct TileChoice { int bm, bn, per_cu; float alone, full, end; };
struct TilePick { int shape; float us; };
static TilePick choose_tile(const TileChoice* c, int shapes, long rows, long cols, int steps, float end_scale,
                            int slices = 1) {
  TilePick best{0, 0.f};
  for (int i = 0; i < shapes; ++i) {
    const long tiles = ((rows + c[i].bm - 1) / c[i].bm) * ((cols + c[i].bn - 1) / c[i].bn) * slices;
    const long slots = 256L * c[i].per_cu, rest = tiles % slots;
    const float end = c[i].end * end_scale, more = rest <= 256 ? 0.f : (float)(rest - 256) / (float)(slots - 256);
    const float us = (float)(tiles / slots) * (c[i].full * steps + end) +
                     (rest == 0 ? 0.f : (c[i].alone + (c[i].full - c[i].alone) * more) * steps + end);
    if (i == 0 || us < best.us) best = {i, us};
  }
  return best;
}

// ---- kernels

// rows of fp32 values that the epilogue needs, fetched into registers before the
// main loop (older than its loads, whose waits count younger ones) and put into
// LDS behind the ring after it: the epilogue's stores then wait for no load
template <int N, int THREADS, class F>
struct Staged {
  static constexpr int PER = (N + THREADS - 1) / THREADS;
  float v[PER];
  __device__ __forceinline__ void fetch(const F& f) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int x = (int)threadIdx.x + i * THREADS;
      v[i] = x < N ? f(x) : 0.f;
    }
  }
  __device__ __forceinline__ void put(float* lds) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int x = (int)threadIdx.x + i * THREADS;
      if (x < N) lds[x] = v[i];
    }
  }
};

// four consecutive values of a row, to memory as T: one store at any alignment of T
// (odd widths: fp32 dW of 9238 x 2385 82 -> 36 us, 8 bits 4032 x 9343 x 632 90 -> 66)
template <typename T>
__device__ __forceinline__ void store4(T* p, int left, const float (&v)[4]) {
  typedef T any4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  if (left >= 4) {
    *(any4*)p = any4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < left) p[r] = from_f32<T>(v[r]);
  }
}

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

template <typename T>
constexpr TileElem elem_of() { return sizeof(T) == 4 ? ELEM_F32 : ELEM_BF16; }

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

// The gradients' products.  b is a KR operand: a pair of fragments holds 8
// neighbouring columns of a row (bf16: all of them exist).  Stored in the operands'
// type (row stride ldc), or as fp32 partial sums (row stride Split::ld) where the
// contraction is split.
template <class D, class P, typename T>
__device__ __forceinline__ void store_tile(const typename P::Acc (&acc)[D::TM][D::TN], T* C, int ldc, int m0,
                                           int n0, int M, int N) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, g = lane >> 4;
  const int mw = m0 + (wave / D::WGN) * D::WM, nw = n0 + (wave % D::WGN) * D::WN;
#pragma unroll
  for (int i = 0; i < D::TM; ++i) {
    const int m = mw + P::row_of(i, fr);
    if (m >= M) continue;
#pragma unroll
    for (int j = 0; j < D::TN; j += 2) {
      const int n = nw + P::col_of(j, g * 4);
      if (n >= N) continue;
      T* p = C + (size_t)m * ldc + n;
      if constexpr (sizeof(T) == 2) {
        bf16x8 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[2 * r] = (bf16)acc[i][j][r], v[2 * r + 1] = (bf16)acc[i][j + 1][r];
        *(bf16x8*)p = v;
      } else {
        const float lo[4] = {acc[i][j][0], acc[i][j + 1][0], acc[i][j][1], acc[i][j + 1][1]};
        const float hi[4] = {acc[i][j][2], acc[i][j + 1][2], acc[i][j][3], acc[i][j + 1][3]};
        store4(p, N - n, lo);
        store4(p + 4, N - n - 4, hi);
      }
    }
  }
}

// First column of column block tn.  U: the last block ends with the matrix (if that is
// not narrower than a tile) and does some columns over again, the same sums in the
// same order, so that no load reaches past a row's end.
template <class D, bool U>
__device__ __forceinline__ int first_column(int tn, int cols) {
  return U && cols >= D::BN ? min(tn * D::BN, cols - D::BN) : tn * D::BN;
}

// A contraction split over gridDim.y slices of `per` steps: slice y writes fp32
// partial sums [rows][ld] behind those of the slices before it, which
// split_sum_kernel adds up in order.
struct Split {
  float* partial;   // NULL: not split
  int per, ld;      // ld: the output's columns in whole 16-byte pieces
};
__device__ __forceinline__ void take_slice(const Split& sp, TileShape& s) {
  s.first = (int)blockIdx.y * sp.per;
  s.steps = min(sp.per, s.steps - s.first);
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

// out (rows [0, half) to o0, the others to o1) = the sum of the slices' partials
// [rows][ldp], in ascending slice order; one thread per 4 columns
template <typename T>
__global__ __launch_bounds__(256) void split_sum_kernel(const float* __restrict__ partial, int slices, long rows,
                                                        long half, int cols, int ldp, T* o0, T* o1, int ld) {
  const long x = blockIdx.x * 256L + threadIdx.x, n4 = ldp / 4;
  if (x >= rows * n4) return;
  const long r = x / n4;
  const int c = (int)(x - r * n4) * 4;
  const float* p = partial + r * ldp + c;
  f32x4 a = *(const f32x4*)p;
#pragma unroll 4
  for (int i = 1; i < slices; ++i) a += *(const f32x4*)(p + i * rows * ldp);
  const float v[4] = {a[0], a[1], a[2], a[3]};
  store4((r < half ? o0 + r * ld : o1 + (r - half) * ld) + c, cols - c, v);
}

// ---- launches
// Shapes of the bf16 and 8-bit products: times measured on products of 4096 x 20480 x
// 4096 (full), 333 rows (alone) and K = 1152 (end; with bf16 outputs for every column
// of the tile, half of it for the gated block), then moved by up to a quarter to
// choose best for 104 drawn products (1.5 % above each one's fastest shape in the
// mean, 12 % at most).  Two stages and several workgroups per CU where the tiles fill
// the chip -- the epilogue of one then runs beside the loop of another --, three or
// four stages where they do not: 7531 x 4608 x 1152 in 8 bits 84 us on 256 x 256, 63 on
// 128 x 128 with two stages, 89 with four; 600 x 1152 x 4608 57, 28 and 21, 16 on 64 x
// 128 with three.  Three stages on 64 and 32 rows, two workgroups per CU, beat four
// where there are more than 256 tiles (gated 200 x 4608 x 1152 15.4 -> 11.2 us) and
// lose where the weights of few rows stream from memory (1 x 10240 x 4096 33.5 and 36.3
// us on 32 rows).
using Tile256 = TileDims<256, 256, 2, 4, 2>;
using Tile128 = TileDims<128, 128, 2, 4, 2>;
using Tile128d = TileDims<128, 128, 2, 4, 4>;
using Tile64 = TileDims<64, 128, 2, 4, 2>;
using Tile64d = TileDims<64, 128, 2, 4, 3>;
using Tile32 = TileDims<32, 128, 1, 4, 4>;
using Tile32d = TileDims<32, 128, 1, 4, 3>;
using Tile32k = TileDims<32, 64, 2, 2, 3, 2>;
using Tile16k = TileDims<16, 32, 1, 1, 3, 4>;
constexpr TileChoice kTiles[] = {{256, 256, 1, 1.60f, 1.60f, 13.f}, {128, 128, 2, 0.72f, 1.02f, 4.8f},
                                 {128, 128, 1, 0.55f, 0.55f, 5.f},  {64, 128, 3, 0.60f, 1.01f, 3.f},
                                 {64, 128, 2, 0.48f, 1.00f, 2.85f}, {32, 128, 2, 0.44f, 0.78f, 2.f},
                                 {32, 64, 2, 0.155f, 0.37f, 2.2f},  {16, 32, 2, 0.073f, 0.17f, 2.5f}};
// Shapes with groups of waves, for few tiles: their launch takes up to 2048 threads for 64
// x 64 outputs (the others at most 512), so that it stays below 2^32 only up to here.
static bool few_tiles(long rows, long cols) { return ((rows + 63) / 64) * ((cols + 63) / 64) < 1 << 21; }
constexpr int kGradTiles = 6, kTile32 = 5, kTile32k = 6, kTile16k = 7, kStream = 8;
// The products without slices (8-bit layer, gated forward) have two more shapes for few
// tiles of a long contraction: groups of waves share the steps of a tile.  us on the
// shapes before them, on Tile32k and on Tile16k: 8 bits 4 x 775 x 7447 20.5, 10.9, 9;
// F = 488 at 5 rows of K = 8896 35, 21, 11.7; F = 6488 at 21 rows of 2824 -, 13.4, 20.1.
// (Eight groups of 16 x 32 leave no room for a second workgroup: F = 1232 9.1 -> 8.2, F =
// 4256 17.0 -> 18.9.)  Tile32 takes one block of rows whose weights stream from memory.
static int tile_index(long rows, long cols, int steps, float end_scale) {
  const bool groups = steps >= 4 && few_tiles(rows, cols);
  const int shape = choose_tile(kTiles, groups ? kGradTiles + 2 : kGradTiles, rows, cols, steps, end_scale).shape;
  return shape >= kTile32 && rows <= 32 && cols > 128 * 128 ? kStream : shape;
}

// fp32 (sizes: rows x columns of g | u x K): bound by the matrix cores (154 TFLOP/s: 1.7
// us per step of 128 x 128), so that two stages are enough and several workgroups share
// a CU (4096 x 9216 x 1152: 143 TFLOP/s on 128 x 128, 139 on 64 x 64, 134 and 128 with
// four stages).  Costs from 36 to 9216 tiles of 36 steps: 22.7 us for up to 256 of 64 x
// 64, 17.1 for every 256 more; 70.5 and 67 on 128 x 128.  A wave's step is 32 MFMAs of
// 32 cycles on 64 x 64, 16 on 32 x 64, where a chain of steps is what takes the time: 33
// x 2304 x 1152 22.3 and 14.9 us (three stages; two stages of 32 x 32 per wave 4 - 10 us
// more, four stages 0.5 - 2); 517 x 2832 x 1152 38 and 32; 1024 x 9216 x 1152 160 and 174.
using Tile64s = TileDims<64, 64, 2, 2, 2>;
using Tile32s = TileDims<32, 64, 2, 2, 3>;
constexpr TileChoice kTilesF32[] = {{128, 128, 1, 1.88f, 1.79f, 3.f}, {64, 64, 1, 0.605f, 0.455f, 0.9f},
                                    {32, 64, 1, 0.404f, 0.25f, 0.7f}, {32, 64, 1, 0.32f, 0.25f, 1.2f},
                                    {16, 32, 2, 0.10f, 0.18f, 3.f}};
// dW: a's fragments are turned in twos at least, which 16 rows per wave do not have.
// The last two, with groups of waves, for the gated forward: a step of 16 x 32 is 16
// MFMAs instead of 64 of the CU (23 x 9238 x 2385 32.9 us on 32 x 64, 25.6 with two
// groups; 1 x 4608 x 7496 80, 69 and 26 on 16 x 32; 82 x 4512 x 1792 22, 19, 23).
constexpr int kF32DwTiles = 2, kF32DxTiles = 3, kF32Groups = 3;
static int tile_index_f32(long rows, long cols, int steps) {
  const bool groups = steps >= 4 && few_tiles(rows, cols);
  return choose_tile(kTilesF32, groups ? kF32Groups + 2 : kF32Groups, rows, cols, steps, 0.5f).shape;
}
constexpr int kMaxSlices = 16;

// group_m 8: eight row blocks share a column block's operand in an XCD's L2
template <class D>
static TileShape tile_shape(int rows, int cols, int steps, int kbytes, int half) {
  TileShape s;
  s.tiles_m = (rows + D::BM - 1) / D::BM;
  s.tiles_n = (cols + D::BN - 1) / D::BN;
  s.group_m = 8;
  s.steps = steps;
  s.kbytes = kbytes;
  s.half = half;
  s.first = 0;
  return s;
}

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

#define T2I_TILES(SHAPE, CALL)                    \
  switch (SHAPE) {                                \
    case 0: { using D = Tile256; CALL; break; }   \
    case 1: { using D = Tile128; CALL; break; }   \
    case 2: { using D = Tile128d; CALL; break; }  \
    case 3: { using D = Tile64; CALL; break; }    \
    case 4: { using D = Tile64d; CALL; break; }   \
    default: { using D = Tile32d; CALL; break; }  \
  }
#define T2I_TILES_FWD(SHAPE, CALL)                        \
  switch (SHAPE) {                                        \
    case kTile32k: { using D = Tile32k; CALL; break; }    \
    case kTile16k: { using D = Tile16k; CALL; break; }    \
    case kStream: { using D = Tile32; CALL; break; }      \
    default: T2I_TILES(SHAPE, CALL)                       \
  }

hipError_t launch_linear_i8(const int8_t* A, int lda, const int8_t* W, int ldw, int M, int N, int K,
                            const I8Epi& e, hipStream_t st) {
  const TileOperand a{(const char*)A, nullptr, (uint32_t)lda, M, 0}, b{(const char*)W, nullptr, (uint32_t)ldw, N, 0};
  const int shape = tile_index(M, N, i8_row(K) / 128, 1.f);
  T2I_TILES_FWD(shape, i8_launch<D>(a, b, e, M, N, K, st))
  return hipGetLastError();
}

#define T2I_TILES_F32_DW(SHAPE, CALL)            \
  switch (SHAPE) {                               \
    case 0: { using D = Tile128; CALL; break; }  \
    default: { using D = Tile64s; CALL; break; } \
  }
#define T2I_TILES_F32_DX(SHAPE, CALL)            \
  switch (SHAPE) {                               \
    case 2: { using D = Tile32s; CALL; break; }  \
    default: T2I_TILES_F32_DW(SHAPE, CALL)       \
  }
#define T2I_TILES_F32_FWD(SHAPE, CALL)                       \
  switch (SHAPE) {                                           \
    case kF32Groups: { using D = Tile32k; CALL; break; }     \
    case kF32Groups + 1: { using D = Tile16k; CALL; break; } \
    default: T2I_TILES_F32_DX(SHAPE, CALL)                   \
  }

// whether these sizes and strides of fp32 values, and pointers, are whole 16-byte pieces
static bool f32_pieces(std::initializer_list<int> sizes, std::initializer_list<const void*> ptrs) {
  uintptr_t bits = 0;
  for (int n : sizes) bits |= (uintptr_t)n * 4;
  for (const void* p : ptrs) bits |= (uintptr_t)p;
  return bits % 16 == 0;
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

// Tile shape and slices of a gradient's product: as few slices as keep the time
// least, counting 4 us for the second launch and the partial sums' way out and back
// at 4 TB/s (1024 x 9216 x 1152: 63 us on 144 64 x 128 tiles, 41 in slices).
struct SplitPick { int shape, slices, per; };
static SplitPick choose_split(const TileChoice* tiles, int shapes, long rows, long cols, int steps) {
  SplitPick best{0, 1, steps};
  float least = 0.f;
  for (int n = 1; n <= kMaxSlices; ++n) {
    const int per = (steps + n - 1) / n, slices = (steps + per - 1) / per;
    if (slices != n || (n > 1 && per < 4)) continue;
    const TilePick p = choose_tile(tiles, shapes, rows, cols, per, n > 1 ? 2.f : 1.f, n);
    const float us = p.us + (n > 1 ? 4.f + (float)n * rows * cols * 8 / 4e6f : 0.f);
    if (n == 1 || us < least) least = us, best = {p.shape, n, per};
  }
  return best;
}

static long whole4(long cols) { return (cols + 3) / 4 * 4; }
static SplitPick split_dx(bool is_bf16, long rows, long cols, int k) {
  return is_bf16 ? choose_split(kTiles, kGradTiles, rows, cols, (k + 63) / 64)
                 : choose_split(kTilesF32, kF32DxTiles, rows, cols, (k + 31) / 32);
}
static SplitPick split_dw(bool is_bf16, long rows, long cols, int k) {
  return is_bf16 ? choose_split(kTiles, kGradTiles, rows, cols, (k + 63) / 64)
                 : choose_split(kTilesF32, kF32DwTiles, rows, cols, (k + 31) / 32);
}

size_t gated_split_floats(bool is_bf16, int M, int F, int K) {
  auto floats = [](const SplitPick& p, long rows, long cols) -> size_t {
    return p.slices > 1 ? (size_t)p.slices * rows * whole4(cols) : 0;
  };
  return std::max({floats(split_dx(is_bf16, M, K, 2 * gated_cols(F)), M, K),
                   floats(split_dw(is_bf16, 2L * F, K, M), 2L * F, K), floats(split_dw(is_bf16, F, K, M), F, K)});
}

template <typename T>
static void split_sum(const Split& sp, int slices, long rows, long half, int cols, T* o0, T* o1, int ld,
                      hipStream_t st) {
  hipLaunchKernelGGL((split_sum_kernel<T>), dim3((unsigned)((rows * (sp.ld / 4) + 255) / 256)), dim3(256), 0, st,
                     sp.partial, slices, rows, half, cols, sp.ld, o0, o1, ld);
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
// gated forward, 2: dx, 3: dWg and dWu)
extern "C" int t2i_test_block_tile(int op, int is_bf16, int M, int F, int K, int* rows, int* columns, int* per_cu,
                                   int* slices) {
  if (M < 1 || F < 1 || K < 1 || op < 0 || op > 3) return 0;
  SplitPick p{0, 1, 0};
  const bool f32 = op != 0 && !is_bf16;
  if (op == 0) p.shape = tile_index(M, F, i8_row(K) / 128, 1.f);
  else if (op == 1) p.shape = f32 ? tile_index_f32(M, 2L * F, (K + 31) / 32) : tile_index(M, 2L * F, (K + 63) / 64, 0.5f);
  else p = op == 2 ? split_dx(is_bf16, M, K, 2 * gated_cols(F)) : split_dw(is_bf16, 2L * F, K, M);
  const bool stream = !f32 && p.shape == kStream;   // four stages, one workgroup per CU
  const TileChoice& c = f32 ? kTilesF32[p.shape] : kTiles[stream ? kTile32 : p.shape];
  *rows = c.bm;
  *columns = c.bn;
  *per_cu = stream ? 1 : c.per_cu;
  const int group = p.shape - (f32 ? kF32Groups : kTile32k);
  *slices = op > 1 ? p.slices : group == 0 ? Tile32k::KG : group == 1 ? Tile16k::KG : 1;
  return 1;
}

}  // namespace t2i
