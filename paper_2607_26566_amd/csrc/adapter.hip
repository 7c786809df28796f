// Low-rank adapters of many requests beside a shared linear layer, and the gradients of
// both (gfx950).  Row m takes adapter i = index[m], or none:
//   t = s_i x A_i^T,  y = x W^T + bias + t B_i^T.
// Three kinds of kernels: the narrow products with A (and, for the gradients, B) that make
// t, on tiles of 16 or 32 rows or, for few rows, one row and four ranks to a workgroup; the
// shared product on the tiles of gemm_tile.h, whose accumulators take t B^T before the
// epilogue; and the adapters' own gradients, sums over the rows of each.
//
// t (and the gradients' u) is fp32.  The matrix cores take it as three bf16 values, 8 of its
// 24 bits each and all of its sign: rounded once it would raise the error of dA and dB, whose
// operand it is, from 0.0017 to 0.0024, and parts of both signs would make a NaN of their
// products with an infinity.
//
// What bounds them: the layer is its tile product's (7531 x 4608 x 1152, rank 32, adapters
// in runs 100 - 118 us of 82.7 GFLOP, 4096 x 4096 x 4096, rank 16 105 of 137, dx 112), for
// few rows HBM and the ring's first loads (24 x 4096 x 4096 10.5 us); t and the gradients'
// sums are bound by reading x or dy once (33.6 MB: t 12.8 us, both sums 16.5).
//
// Adapters never meet: a row's sums hold nothing of another row's adapter, not even
// times zero (a NaN in one tenant's adapter stays in that tenant's rows).
#include <algorithm>

#include "block_gemm.h"
#include "row_ops.h"

namespace t2i {

// the adapter of a row, -1: none (an index out of range takes none)
__device__ __forceinline__ int adapter_of(const int32_t* index, int n, int row) {
  const int i = index ? index[row] : 0;
  return (unsigned)i < (unsigned)n ? i : -1;
}

// the least adapter above `now` of the rows of 16 neighbouring lanes (negative: none), or kNone:
// unsigned differences put those up to `now` last; ds_swizzle (lanes xor 8, 4, 2, 1) takes no
// registers for addresses
constexpr int kNone = 0x7fffffff;
template <int N>
__device__ __forceinline__ int least_above(int now, const int (&ids)[N]) {
  uint32_t v = ~0u;
#pragma unroll
  for (int i = 0; i < N; ++i) v = min(v, (uint32_t)(ids[i] - now - 1));
  v = min(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x201f));
  v = min(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x101f));
  v = min(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x081f));
  v = min(v, (uint32_t)__builtin_amdgcn_ds_swizzle((int)v, 0x041f));
  v = (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
  return v < 0x80000000u - (uint32_t)(now + 1) ? now + 1 + (int)v : kNone;
}

// elements of a lane's 16 bytes: consecutive k of an MFMA operand
template <typename T>
constexpr int kLaneK = 16 / (int)sizeof(T);

// 16 bytes at k of a row of `len` elements, `row` bytes behind base, 0 behind its end;
// whole: len is a multiple of a piece
template <typename T>
__device__ __forceinline__ i32x4 load_k(const void* base, uint32_t row, int k, int len, bool whole) {
  constexpr int L = kLaneK<T>;
  typedef T piece __attribute__((ext_vector_type(kLaneK<T>), aligned(sizeof(T))));
  const char* const p = (const char*)base;
  const uint32_t at = row + (uint32_t)k * (uint32_t)sizeof(T);
  i32x4 v = {0, 0, 0, 0};
  if (whole ? k < len : k + L <= len) {
    v = __builtin_bit_cast(i32x4, *(const piece*)(p + at));
  } else if (!whole) {
#pragma unroll
    for (int i = 0; i < L; ++i)
      if (k + i < len) {
        const T e = *(const T*)(p + at + i * sizeof(T));
        if constexpr (sizeof(T) == 2) v[i / 2] |= (int)((uint32_t)__builtin_bit_cast(uint16_t, e) << (16 * (i & 1)));
        else v[i] = __float_as_int(e);
      }
  }
  return v;
}
template <typename T>
__device__ __forceinline__ float element(const i32x4& v, int i) {
  if constexpr (sizeof(T) == 2)
    return __uint_as_float(i & 1 ? (uint32_t)v[i / 2] & 0xffff0000u : (uint32_t)v[i / 2] << 16);
  else
    return __int_as_float(v[i]);
}
// a lane's operand of t: L consecutive values, bf16 in three parts of t's sign, each the upper
// half of what the ones before it leave.  A part that would be 0 is 2^-40 t instead (t is off
// by 2^-39 of itself at most), so that an infinite factor makes an infinity of every part as it
// does of t, unless t is below 2^-86; t = 0 and infinities have equal parts.
template <typename T>
struct Exact {
  static constexpr int PARTS = sizeof(T) == 2 ? 3 : 1;
  i32x4 part[PARTS];
  __device__ __forceinline__ void set(const float (&v)[kLaneK<T>]) {
    if constexpr (sizeof(T) == 2) {
      auto top = [](float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); };
      // the upper halves of two values, with these signs
      auto pair = [](float x, float y) { return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302); };
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float mid[2], low[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float x = v[2 * i + e], least = fabsf(x) * 0x1p-40f;
          // (an infinity less itself is a NaN, which fmaxf leaves out)
          mid[e] = fmaxf(fabsf(x - top(x)), least);
          low[e] = fmaxf(mid[e] - top(mid[e]), least);
        }
        const uint32_t hi = pair(v[2 * i], v[2 * i + 1]), sign = hi & 0x80008000u;
        part[0][i] = (int)hi;
        part[1][i] = (int)(pair(mid[0], mid[1]) | sign);
        part[2][i] = (int)(pair(low[0], low[1]) | sign);
      }
    } else {
      part[0] = i32x4{__float_as_int(v[0]), __float_as_int(v[1]), __float_as_int(v[2]), __float_as_int(v[3])};
    }
  }
};
// c[j][m] += sum_k a[j][k] b[m][k], 32 (fp32: 16) of k: lane (x = lane & 15, g = lane >> 4)
// gives k = L g .. of row x of both; it holds c[4 g + r][x]
template <typename T>
__device__ __forceinline__ f32x4 narrow_mfma(const i32x4& a, const i32x4& b, f32x4 c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(a[k]), __int_as_float(b[k]), c, 0, 0, 0);
    return c;
  }
}

template <typename T>
__device__ __forceinline__ f32x4 narrow_mfma(const i32x4& a, const Exact<T>& b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < Exact<T>::PARTS; ++i) c = narrow_mfma<T>(a, b.part[i], c);
  return c;
}
template <typename T>
__device__ __forceinline__ f32x4 narrow_mfma(const Exact<T>& a, const i32x4& b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < Exact<T>::PARTS; ++i) c = narrow_mfma<T>(a.part[i], b, c);
  return c;
}

// ---------------------------------------------------------------------------
// t = s x A^T.  Few rows: a workgroup takes one row and four ranks, each wave a fourth of
// k.
template <typename T>
__global__ __launch_bounds__(256) void adapter_down_rows_kernel(AdapterDown p) {
  constexpr int RJ = 4;
  __shared__ float red[4][RJ];
  const int m = blockIdx.x, j0 = blockIdx.y * RJ, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int ad = adapter_of(p.index, p.n, m);
  float s[RJ] = {0.f, 0.f, 0.f, 0.f};
  if (ad >= 0 && j0 < p.rank) {
    const T* const x = (const T*)p.x + (size_t)m * p.ldx;
    const T* const a = (const T*)p.a + (size_t)ad * p.rank * p.K;
#pragma unroll 2
    for (int k = (wave * 64 + lane) * 8; k < p.K; k += 2048) {
      Piece<T> px, pa[RJ];
      load_piece(x, k, p.K, px);
#pragma unroll
      for (int j = 0; j < RJ; ++j) load_piece(a + (size_t)min(j0 + j, p.rank - 1) * p.K, k, p.K, pa[j]);
#pragma unroll
      for (int j = 0; j < RJ; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[j] = fmaf(px.get(e), pa[j].get(e), s[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < RJ; ++j) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s[j] += __shfl_xor(s[j], o, kWave);
    if (lane == 0) red[wave][j] = s[j];
  }
  __syncthreads();
  const int j = threadIdx.x;
  if (j >= RJ) return;
  const float v = (red[0][j] + red[1][j]) + (red[2][j] + red[3][j]);
  const float scale = ad >= 0 ? (p.scale ? p.scale[ad] : 1.f) : 0.f;
  p.t[(size_t)m * p.ldt + j0 + j] = ad >= 0 && j0 + j < p.rank ? v * scale : 0.f;
}

// Many rows: a tile of rows and all ranks (up to 64), whose groups of waves share k as
// in the products of few tiles; both operands come through LDS in whole lines (fragments
// straight from memory, 16 rows to an instruction, 19 us for 4096 rows of 4096 and 16
// ranks).
//
// A tile whose rows take several adapters does its product once for each of them.  Tiles of
// more than three in a window of rows share those rows anew instead, in the order of their
// adapters: each of them works out the same order from the window's index, which takes it
// about 5 us, and takes the part that is its turn (512 rows of 4096 with one of 32 adapters
// each, rank 16: 59 -> 25 us).
constexpr int kWindow = 4096, kSorted = 512, kOwn = 3;   // rows; adapters for that; adapters a tile takes as it is

template <int BM, int THREADS>
struct SharedRows {
  static constexpr int TILES = kWindow / BM, PER = kWindow / THREADS, NW = THREADS / 64;
  int16_t* ids;      // [kWindow] in LDS, as the others
  int* hist;         // [kSorted]
  uint8_t* several;  // [TILES] whether a tile's rows take more than kOwn adapters
  int* scratch;      // [NW + 4]
  int* row;          // [BM] the rows of this tile, counted from the window's first, -1: none
  int* adapter;      // [BM]

  // sum of v over the threads before this one; all of them in `sum`
  __device__ __forceinline__ int before(int v, int& sum) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(x, o, kWave);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) scratch[wave] = x;
    __syncthreads();
    int base = 0;
    sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      base += w < wave ? scratch[w] : 0;
      sum += scratch[w];
    }
    return base + x - v;
  }
  __device__ __forceinline__ void take(const AdapterDown& p, int first, int tile) const {
    const int t = threadIdx.x, rows = min(kWindow, p.M - first);
    for (int r = t; r < kWindow; r += THREADS) ids[r] = (int16_t)(r < rows ? adapter_of(p.index, p.n, first + r) : -1);
    for (int i = t; i < p.n; i += THREADS) hist[i] = 0;
    if (t < BM) row[t] = adapter[t] = -1;
    __syncthreads();
    for (int i = t; i < TILES; i += THREADS) {
      int seen[kOwn] = {-1, -1, -1}, count = 0;   // the first ones
      for (int r = 0; r < BM; ++r) {
        const int a = ids[i * BM + r];
        if (a < 0 || a == seen[0] || a == seen[1] || a == seen[2]) continue;
        if (count < kOwn) seen[count == 0 ? 0 : count == 1 ? 1 : 2] = a;
        ++count;
      }
      several[i] = count > kOwn;
    }
    __syncthreads();
    // this thread's rows, next to each other; those of no interest become -1
    int mine[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int r = t * PER + i;
      mine[i] = several[r / BM] ? ids[r] : -1;
      if (mine[i] >= 0) atomicAdd(&hist[mine[i]], 1);   // (counts: any order)
    }
    int turn = 0;
    for (int i = t & 63; i < tile; i += 64) turn += several[i];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) turn += __shfl_xor(turn, o, kWave);
    __syncthreads();
    // the adapter of the first row whose turn it is, and how many of its rows come before;
    // then row after row of it and the next ones
    int skip = turn * BM, got = 0;
    for (int a = 0; a < p.n && got < BM; ++a) {
      const int count = hist[a];
      if (count <= skip) {
        skip -= count;
        continue;
      }
      int here = 0, sum;
#pragma unroll
      for (int i = 0; i < PER; ++i) here += mine[i] == a;
      int at = before(here, sum) - skip + got;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (mine[i] == a) {
          if (at >= got && at < BM) row[at] = t * PER + i, adapter[at] = a;
          ++at;
        }
      got = min(BM, got + count - skip);
      skip = 0;
    }
    __syncthreads();
  }
};

template <class D, typename T, bool U>
__global__ __launch_bounds__(D::THREADS, 1) void adapter_down_kernel(AdapterDown p) {
  using P = TileProduct<D, elem_of<T>(), false, false, false, false, U>;
  using S = SharedRows<D::BM, D::THREADS>;
  constexpr int RING = D::KG * D::RING;
  static_assert(kWindow * 2 + kSorted * 4 + S::TILES + (S::NW + 4) * 4 <= RING, "room for a window's index");
  __shared__ __attribute__((aligned(1024))) char smem[RING];
  __shared__ int rows[2][D::BM];
  constexpr int EB = sizeof(T), TM = D::TM, TN = D::TN;
  const int lane = threadIdx.x & 63, fr = lane & 15, g = lane >> 4;
  int m0 = blockIdx.x * D::BM;
  const int j0 = blockIdx.y * D::BN, cols = adapter_cols(p.rank);
  const TileOperand a{(const char*)p.x, nullptr, (uint32_t)(EB * p.ldx), p.M, 0};
  TileShape s;
  s.tiles_m = s.tiles_n = s.group_m = 1;
  s.kbytes = EB * p.K;
  s.steps = (s.kbytes + 127) / 128;
  s.half = s.first = 0;
  int ad[TM], row[TM];   // adapter (-2: no row), row from m0
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    row[i] = i * 16 + fr;
    ad[i] = m0 + row[i] < p.M ? adapter_of(p.index, p.n, m0 + row[i]) : -2;
  }
  auto store = [&](int i, int j, const f32x4& v) {
    const int c = j0 + j * 16 + g * 4;
    f32x4 o;
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = c + r < p.rank ? v[r] : 0.f;
    if (c < cols) *(f32x4*)(p.t + (size_t)(m0 + row[i]) * p.ldt + c) = o;
  };
  const bool behind = j0 >= p.rank;   // the zeros behind the ranks
  if (threadIdx.x < 64) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
      if (ad[i] == -1 || (behind && ad[i] >= 0))
#pragma unroll
        for (int j = 0; j < TN; ++j) store(i, j, f32x4{0.f, 0.f, 0.f, 0.f});
  }
  if (behind) return;
  int next = least_above(-1, ad);
  int last = next;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) last = last == kNone ? last : least_above(last, ad);
  const bool several = last != kNone;   // more than kOwn
  if (several && p.n <= kSorted && (int64_t)kWindow * p.ldx * EB < 0x7fffffff) {
    const int first = m0 / kWindow * kWindow, tile = (m0 - first) / D::BM;
    const S sh{(int16_t*)smem, (int*)(smem + kWindow * 2), (uint8_t*)(smem + kWindow * 2 + kSorted * 4),
               (int*)(smem + kWindow * 2 + kSorted * 4 + S::TILES), rows[0], rows[1]};
    sh.take(p, first, tile);
    m0 = first;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      row[i] = max(rows[0][i * 16 + fr], 0);
      ad[i] = rows[0][i * 16 + fr] < 0 ? -2 : rows[1][i * 16 + fr];
    }
    next = least_above(-1, ad);
  } else {
    if (threadIdx.x < D::BM) rows[0][threadIdx.x] = min((int)threadIdx.x, p.M - 1 - m0);
    __syncthreads();
  }
  int now = -1;
  for (;;) {   // the adapters in ascending order, the same for every wave
    if (next == kNone) return;
    if (now >= 0) tile_barrier();   // (the sums of the adapter before are read)
    now = next;
    next = least_above(now, ad);
    const TileOperand b{(const char*)p.a + (size_t)now * p.rank * p.K * EB, nullptr, (uint32_t)(EB * p.K), p.rank, 0};
    typename P::Acc acc[TM][TN];
    if (!P::run_groups(smem, a, b, s, m0, j0, acc, FromZero(),
                       [&](int r, int, int) { return max(rows[0][r], 0); }))
      continue;
    const float scale = p.scale ? p.scale[now] : 1.f;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      if (ad[i] != now) continue;
#pragma unroll
      for (int j = 0; j < TN; ++j) store(i, j, acc[i][j] * scale);
    }
  }
}

// rows up to which the first kernel takes them (with a product of 8 columns behind it: 256
// of 4096, rank 16, 32 adapters 16 us, tiles 15.5; 512 18 and 13)
constexpr int kDownRows = 256;
template <class D, typename T, bool U>
static void down_launch(const AdapterDown& p, hipStream_t st) {
  hipLaunchKernelGGL((adapter_down_kernel<D, T, U>),
                     dim3((unsigned)((p.M + D::BM - 1) / D::BM), (unsigned)((adapter_cols(p.rank) + D::BN - 1) / D::BN)),
                     dim3(D::THREADS), 0, st, p);
}
template <typename T, bool U>
static void down_tiles(const AdapterDown& p, hipStream_t st) {
  const long steps = ((long)p.K * (int)sizeof(T) + 127) / 128;
  // Groups of waves have a step each at least.  Eight, one workgroup to a CU, while there
  // are no more tiles than CUs, else four and two (with a product of 8 columns behind it:
  // 7531 rows of 1152, rank 32 19.2 and 16.7 us, 16000 of 640, rank 8 19.7 and 14.3; 300 of
  // 4096, rank 16 16.5 and 17.6), and 32 rows to read the adapter half as often for many
  // ranks (8192 rows of 4608, rank 64 45 and 35.6).
  const bool many = p.M > 16 * 256;
  if (steps < 8) down_launch<TileDims<16, 32, 1, 1, 4>, T, U>(p, st);
  else if (p.rank <= 16 && !many) down_launch<TileDims<16, 16, 1, 1, 4, 8>, T, U>(p, st);
  else if (p.rank <= 16) down_launch<TileDims<16, 16, 1, 1, 3, 4>, T, U>(p, st);
  else if (p.rank <= 32 && !many) down_launch<TileDims<16, 32, 1, 1, 3, 8>, T, U>(p, st);
  else if (p.rank <= 32) down_launch<TileDims<16, 32, 1, 1, 3, 4>, T, U>(p, st);
  else if (!many) down_launch<TileDims<16, 64, 1, 1, 3, 4>, T, U>(p, st);
  else down_launch<TileDims<32, 64, 1, 1, 3, 4>, T, U>(p, st);
}
template <typename T>
static void down_any(const AdapterDown& p, hipStream_t st) {
  if (p.M <= kDownRows)
    hipLaunchKernelGGL((adapter_down_rows_kernel<T>), dim3((unsigned)p.M, (unsigned)(adapter_cols(p.rank) / 4)),
                       dim3(256), 0, st, p);
  else if constexpr (sizeof(T) == 2) down_tiles<T, false>(p, st);
  else if (f32_pieces({p.K, p.ldx}, {p.x, p.a})) down_tiles<T, false>(p, st);
  else down_tiles<T, true>(p, st);
}
hipError_t launch_adapter_down(bool is_bf16, const AdapterDown& p, hipStream_t st) {
  if (is_bf16) down_any<bf16>(p, st);
  else down_any<float>(p, st);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// acc += t P_i^T for the tile's rows, P_i [columns][stride] the adapter's second matrix
// (forward: B; gradients: A transposed), both operands straight from memory, while the
// ring's first loads are under way.  A wave whose rows have one adapter takes the matrix
// cores for all of them; rows of several take them once for every adapter, of whose
// results each row takes its own (the largest tile, whose accumulators leave few
// registers, after the last step, 16 rows at a time by way of LDS); in tiles of 16 rows,
// which are for few rows with an adapter each, a lane sums up its own row's products, all
// of whose loads are under way at once.
template <class P, class D, typename T>
struct Adapters {
  static constexpr int TM = D::TM, TN = D::TN, L = kLaneK<T>;
  const AdapterUp& u;
  int M, N, mw, nw, fr, g;
  static constexpr bool LATE = TM * TN > 16;
  int id[TM];   // a row's adapter, -2 (any) behind the last row

  __device__ __forceinline__ Adapters(const AdapterUp& up, int m0, int n0, int M_, int N_) : u(up), M(M_), N(N_) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % D::NW);
    fr = lane & 15, g = lane >> 4;
    mw = m0 + (wave / D::WGN) * D::WM, nw = n0 + (wave % D::WGN) * D::WN;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int m = mw + P::row_of(i, fr);
      const int a = adapter_of(u.index, u.n, min(m, M - 1));
      id[i] = m < M ? a : -2;
    }
  }
  // (t's and a matrix's rows of a wave span less than 2^31 bytes; t has whole steps)
  __device__ __forceinline__ void t_at(int i, int k, float (&v)[L]) const {
    const float* const t = u.t + (size_t)mw * u.ldt;
    const float* const p = t + (uint32_t)(min(P::row_of(i, fr), M - 1 - mw) * u.ldt + k);
#pragma unroll
    for (int q = 0; q < L / 4; ++q) {
      const f32x4 w = *(const f32x4*)(p + 4 * q);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * q + e] = w[e];
    }
  }
  __device__ __forceinline__ Exact<T> exact_t(int i, int k) const {
    float v[L];
    t_at(i, k, v);
    Exact<T> x;
    x.set(v);
    return x;
  }
  __device__ __forceinline__ i32x4 p_at(int ad, int j, int x, int k) const {
    const T* const p = (const T*)u.p + ((size_t)ad * N + nw) * u.stride;
    return load_k<T>(p, (uint32_t)(min(P::col_of(j, x), N - 1 - nw) * u.stride) * (uint32_t)sizeof(T), k, u.rank,
                     u.rank % L == 0);
  }
  __device__ __forceinline__ bool one_adapter() const {
    const int first = __builtin_amdgcn_readfirstlane(id[0]);
    bool same = true;
#pragma unroll
    for (int i = 0; i < TM; ++i) same = same && (id[i] == first || id[i] == -2);
    return __all(same);
  }
  __device__ __forceinline__ void operator()(f32x4 (&acc)[TM][TN]) const {
    if (mw >= M || nw >= N) return;
    if (one_adapter()) {
      const int first = __builtin_amdgcn_readfirstlane(id[0]);   // (row mw exists)
      if (first < 0) return;
#pragma unroll 1
      for (int k0 = 0; k0 < u.rank; k0 += 4 * L) {
        i32x4 pv[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) pv[j] = p_at(first, j, fr, k0 + g * L);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const Exact<T> tv = exact_t(i, k0 + g * L);
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = narrow_mfma<T>(pv[j], tv, acc[i][j]);
        }
      }
    } else if constexpr (LATE) {
    } else if constexpr (TM > 1) {
#pragma unroll 1
      for (int k0 = 0; k0 < u.rank; k0 += 4 * L) {
        Exact<T> tv[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) tv[i] = exact_t(i, k0 + g * L);
        // (one after the other: two at a time spill the accumulators of 128 x 128)
#pragma unroll 1
        for (int now = least_above(-1, id); now != kNone; now = least_above(now, id)) {
          i32x4 pv[TN];
#pragma unroll
          for (int j = 0; j < TN; ++j) pv[j] = p_at(now, j, fr, k0 + g * L);
#pragma unroll
          for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
              const f32x4 add = narrow_mfma<T>(pv[j], tv[i], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
              for (int r = 0; r < 4; ++r) acc[i][j][r] += id[i] == now ? add[r] : 0.f;
            }
        }
      }
    } else if (id[0] >= 0) {
#pragma unroll 1
      for (int k = 0; k < u.rank; k += L) {
        float tv[L];
        t_at(0, k, tv);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const i32x4 pv = p_at(id[0], j, g * 4 + r, k);
#pragma unroll
            for (int e = 0; e < L; ++e) acc[0][j][r] = fmaf(tv[e], element<T>(pv, e), acc[0][j][r]);
          }
      }
    }
  }
  // what the largest tile has left; smem: its ring, which no wave reads any more
  __device__ __forceinline__ void finish(char* smem, f32x4 (&acc)[TM][TN]) const {
    if constexpr (LATE) {
      if (mw >= M || nw >= N || one_adapter()) return;
      constexpr int HALF = TM / 2;
      static_assert(D::NW * HALF * TN * 1024 <= D::RING, "room for half of the results");
      const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % D::NW);
      f32x4* const part = (f32x4*)(smem + wave * HALF * TN * 1024) + lane;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int mine[HALF];
#pragma unroll
        for (int i = 0; i < HALF; ++i) {
          const int m = mw + P::row_of(h * HALF + i, fr);
          mine[i] = m < M ? adapter_of(u.index, u.n, m) : -2;
#pragma unroll
          for (int j = 0; j < TN; ++j) part[(i * TN + j) * 64] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll 1
        for (int k0 = 0; k0 < u.rank; k0 += 4 * L) {
          Exact<T> tv[HALF];
#pragma unroll
          for (int i = 0; i < HALF; ++i) {
            tv[i] = exact_t(h * HALF + i, k0 + g * L);
            __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll 1
          for (int now = least_above(-1, mine); now != kNone; now = least_above(now, mine)) {
            // (two fragments of P_i, and t's one after the other: all at once spill 20 registers more)
            i32x4 pv[2] = {p_at(now, 0, fr, k0 + g * L)};
#pragma unroll
            for (int j = 0; j < TN; ++j) {
              if (j + 1 < TN) pv[(j + 1) % 2] = p_at(now, j + 1, fr, k0 + g * L);
#pragma unroll
              for (int i = 0; i < HALF; ++i) {
                const f32x4 add = narrow_mfma<T>(pv[j % 2], tv[i], f32x4{0.f, 0.f, 0.f, 0.f});
                if (mine[i] == now) part[(i * TN + j) * 64] += add;
              }
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < HALF; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[h * HALF + i][j] += part[(i * TN + j) * 64];
      }
    }
  }
};

// waves per SIMD that a tile's LDS leaves room for, which the registers should, too (128 x
// 128 with 134 instead of 128 of them: 7531 x 4608 x 1152 148 instead of 105 us)
template <class D>
constexpr int waves_per_simd() {
  return (160 * 1024) / (D::KG * D::RING + 8 * D::BN) * D::THREADS / 256;
}

// y = x W^T + t B^T + bias, then the linear layer's epilogues
template <class D, typename T, bool RES, bool U>
__global__ __launch_bounds__(D::THREADS, waves_per_simd<D>()) void adapter_linear_kernel(TileOperand a, TileOperand b, TileShape s,
                                                                       AdapterUp up, LinearEpi e, int M, int N) {
  using P = TileProduct<D, elem_of<T>(), false, false, false, false, U>;
  constexpr int THREADS = D::THREADS, NE = (RES ? 2 : 1) * D::BN;
  __shared__ __attribute__((aligned(1024))) char smem[D::KG * D::RING + NE * 4];
  int tm, tn;
  tile_place(s, blockIdx.x, gridDim.x, tm, tn);
  const int m0 = tm * D::BM, n0 = tn * D::BN;
  auto value = [&](int x) -> float {
    const int n = min(n0 + x % D::BN, N - 1);
    if (x < D::BN) return e.bias ? to_f32(((const T*)e.bias)[n]) : 0.f;
    return e.kind == EPI_RESID_GATED ? e.gate[n] : 1.f;
  };
  Staged<NE, THREADS, decltype(value)> st;
  st.fetch(value);
  typename P::Acc acc[D::TM][D::TN];
  const Adapters<P, D, T> from(up, m0, n0, M, N);
  const bool mine = P::run_groups(smem, a, b, s, m0, n0, acc, from);
  float* const ev = (float*)(smem + D::KG * D::RING);
  st.put(ev);
  tile_barrier();
  if (!mine) return;
  from.finish(smem, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, g = lane >> 4;
  const int mw = (wave / D::WGN) * D::WM, nw = (wave % D::WGN) * D::WN;
#pragma unroll
  for (int i = 0; i < D::TM; ++i) {
    const int m = m0 + mw + i * 16 + fr;
    if (m >= M) continue;
#pragma unroll
    for (int j = 0; j < D::TN; ++j) {
      const int nl = nw + j * 16 + g * 4, n = n0 + nl, left = N - n;
      if (left <= 0) continue;
      const f32x4 bb = *(const f32x4*)(ev + nl);
      float y[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        y[r] = acc[i][j][r] + bb[r];
        if (!RES) y[r] = e.kind == EPI_GELU ? gelu_tanh(y[r]) : e.kind == EPI_SILU ? silu(y[r]) : y[r];
      }
      if constexpr (RES) {
        float* x = e.x + (size_t)m * e.ldx + n;
        const f32x4 gt = *(const f32x4*)(ev + D::BN + nl);
        float xv[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) xv[r] = r < left ? x[r] + gt[r] * y[r] : 0.f;
        store4(x, left, xv);
        if (e.xb) store4(e.xb + (size_t)m * e.ldx + n, left, xv);
      } else {
        store4((T*)e.out + (size_t)m * e.ldo + n, left, y);
      }
    }
  }
}

// dx = dy W + u A; where the contraction is split, the first slice takes the adapters
template <class D, typename T, bool U>
__global__ __launch_bounds__(D::THREADS, waves_per_simd<D>()) void adapter_dx_kernel(TileOperand a, TileOperand b, TileShape s, Split sp,
                                                                   AdapterUp up, T* dx, int ldx, int M, int K) {
  using P = TileProduct<D, elem_of<T>(), false, true, false, false, U>;
  __shared__ __attribute__((aligned(1024))) char smem[D::KG * D::RING];
  int tm, tn;
  tile_place(s, blockIdx.x, gridDim.x, tm, tn);
  if (sp.partial) take_slice(sp, s);
  typename P::Acc acc[D::TM][D::TN];
  const int m0 = tm * D::BM, n0 = first_column<D, U>(tn, K);
  const Adapters<P, D, T> from(up, m0, n0, M, K);
  const bool mine = P::run_groups(smem, a, b, s, m0, n0, acc, [&](f32x4 (&c)[D::TM][D::TN]) {
    if (blockIdx.y == 0) from(c);
  });
  if (!mine) return;
  if (from.LATE && blockIdx.y == 0) {
    tile_barrier();
    from.finish(smem, acc);
  }
  if (sp.partial)
    store_tile<D, P>(acc, sp.partial + (size_t)blockIdx.y * M * sp.ld, sp.ld, m0, n0, M, K);
  else
    store_tile<D, P>(acc, dx, ldx, m0, n0, M, K);
}

template <class D, typename T, bool U = false>
static void adapter_linear_launch(const void* x, int ldx, const void* w, int ldw, int M, int N, int K,
                                  const AdapterUp& up, const LinearEpi& e, hipStream_t st) {
  constexpr int eb = sizeof(T), per = 128 / eb;
  const TileOperand a{(const char*)x, nullptr, (uint32_t)eb * ldx, M, 0}, b{(const char*)w, nullptr, (uint32_t)eb * ldw, N, 0};
  const TileShape s = tile_shape<D>(M, N, (K + per - 1) / per, eb * K, 0);
  const dim3 grid((unsigned)(s.tiles_m * s.tiles_n));
  if (e.kind >= EPI_RESID)
    hipLaunchKernelGGL((adapter_linear_kernel<D, T, true, U>), grid, dim3(D::THREADS), 0, st, a, b, s, up, e, M, N);
  else
    hipLaunchKernelGGL((adapter_linear_kernel<D, T, false, U>), grid, dim3(D::THREADS), 0, st, a, b, s, up, e, M, N);
}

// Two more shapes of bf16 products, for sizes that 256 x 256 divides into too few tiles for
// the CUs: 8192 x 1152 x 4608 99 us on 256 x 256 (160 tiles), 83 on 256 x 192 (192); 2100 x
// 4608 x 4608 115 (162), 97 on 192 x 256 (198); 6000 x 2048 x 2048 68 and 60; 5000 x 4096 x
// 1152 59 on 128 x 128, 81.  Costs for choose_tile from these, as those of kTiles.
using Tile192 = TileDims<192, 256, 2, 4, 2>;
using Tile256n = TileDims<256, 192, 2, 4, 2>;
constexpr TileChoice kWideTiles[] = {{192, 256, 1, 1.30f, 1.30f, 14.f}, {256, 192, 1, 1.28f, 1.28f, 14.f}};
static int with_wide(int shape, float us, int wide, long rows, long cols, int steps) {
  const TilePick w = choose_tile(kWideTiles, wide, rows, cols, steps, 1.f);
  return w.us < us ? kTile192 + w.shape : shape;
}
// And one for few rows, whose weights stream from memory: 16 x 16 with eight groups of
// waves, one tile to a CU, where 16 x 32 leaves half of the CUs without one.  With t, 16 rows
// x 4096 x 4096 15.0 us instead of 17.5, x 10240 26.8 and 35.5, 64 x 1024 x 1024 8.0 and
// 9.4; more tiles than CUs take two rounds of it: 24 x 4096 x 4096 20.3 and 17.2.
using Tile16n = TileDims<16, 16, 1, 1, 4, 8>;
int adapter_tile(bool is_bf16, int M, int N, int K) {
  if (!is_bf16) return tile_index_f32(M, N, (K + 31) / 32);
  const int steps = (K + 63) / 64, shape = tile_index(M, N, steps, 1.f);
  if (steps >= Tile16n::KG && (M + 15L) / 16 * ((N + 15L) / 16) <= 256) return kTile16n;
  return shape < kGradTiles ? with_wide(shape, choose_tile(kTiles + shape, 1, M, N, steps, 1.f).us, 2, M, N, steps) : shape;
}
#define T2I_TILES_ADAPTER(SHAPE, CALL)                      \
  switch (SHAPE) {                                          \
    case kTile192: { using D = Tile192; CALL; break; }      \
    case kTile192 + 1: { using D = Tile256n; CALL; break; } \
    case kTile16n: { using D = Tile16n; CALL; break; }      \
    default: T2I_TILES_FWD(SHAPE, CALL)                     \
  }

hipError_t launch_adapter_linear(bool is_bf16, const void* x, int ldx, const void* w, int ldw, int M, int N, int K,
                                 const AdapterUp& up, const LinearEpi& e, hipStream_t st) {
  const int shape = adapter_tile(is_bf16, M, N, K);
  if (is_bf16) {
    T2I_TILES_ADAPTER(shape, (adapter_linear_launch<D, bf16>(x, ldx, w, ldw, M, N, K, up, e, st)))
  } else if (f32_pieces({K, ldx, ldw}, {x, w})) {
    T2I_TILES_F32_FWD(shape, (adapter_linear_launch<D, float>(x, ldx, w, ldw, M, N, K, up, e, st)))
  } else {
    T2I_TILES_F32_FWD(shape, (adapter_linear_launch<D, float, true>(x, ldx, w, ldw, M, N, K, up, e, st)))
  }
  return hipGetLastError();
}

// dx has the shapes with groups of waves, too, which need no second launch: taken where
// they are estimated to beat the best number of slices (fp32 333 x 1155 x 1153 20.5 -> 17.2
// us), and the wider of the two shapes above
SplitPick adapter_dx_pick(bool is_bf16, int M, int N, int K) {
  const SplitPick p = split_dx(is_bf16, M, K, N);
  const int steps = is_bf16 ? (N + 63) / 64 : (N + 31) / 32;
  const TileChoice* const tiles = is_bf16 ? kTiles : kTilesF32;
  const int first = is_bf16 ? kTile32k : kF32Groups;
  const TilePick split = choose_tile(tiles + p.shape, 1, M, K, p.per, p.slices > 1 ? 2.f : 1.f, p.slices);
  const float us = split.us + (p.slices > 1 ? 4.f + (float)p.slices * M * K * 8 / 4e6f : 0.f);
  if (steps >= 4 && few_tiles(M, K)) {
    // (bf16 with k across b's rows: a step takes twice as long as the forward product's)
    const TilePick g = choose_tile(tiles + first, 2, M, K, is_bf16 ? 2 * steps : steps, 1.f);
    if (g.us < us) return {first + g.shape, 1, steps};
  }
  return is_bf16 && with_wide(0, us, 1, M, K, steps) ? SplitPick{kTile192, 1, steps} : p;
}
size_t adapter_dx_floats(bool is_bf16, int M, int N, int K) {
  const SplitPick p = adapter_dx_pick(is_bf16, M, N, K);
  return p.slices > 1 ? (size_t)p.slices * M * whole4(K) : 0;
}
#define T2I_TILES_GRAD(SHAPE, CALL)                    \
  switch (SHAPE) {                                     \
    case kTile32k: { using D = Tile32k; CALL; break; } \
    case kTile16k: { using D = Tile16k; CALL; break; } \
    case kTile192: { using D = Tile192; CALL; break; } \
    default: T2I_TILES(SHAPE, CALL)                    \
  }

template <class D, typename T, bool U = false>
static void adapter_dx_launch(const void* dy, int lddy, const void* w, int ldw, int M, int N, int K, const AdapterUp& up,
                              T* dx, int ldx, const SplitPick& pick, const Split& sp, hipStream_t st) {
  constexpr int eb = sizeof(T), per = 128 / eb;
  const TileOperand a{(const char*)dy, nullptr, (uint32_t)eb * lddy, M, 0}, b{(const char*)w, nullptr, (uint32_t)eb * ldw, N, K};
  const TileShape s = tile_shape<D>(M, K, (N + per - 1) / per, eb * N, 0);
  hipLaunchKernelGGL((adapter_dx_kernel<D, T, U>), dim3((unsigned)(s.tiles_m * s.tiles_n), pick.slices), dim3(D::THREADS), 0,
                     st, a, b, s, sp, up, dx, ldx, M, K);
  if (sp.partial) split_sum(sp, pick.slices, M, M, K, dx, dx, ldx, st);
}

hipError_t launch_adapter_dx(bool is_bf16, const void* dy, int lddy, const void* w, int ldw, int M, int N, int K,
                             const AdapterUp& up, void* dx, int ldx, float* partial, hipStream_t st) {
  const SplitPick pick = adapter_dx_pick(is_bf16, M, N, K);
  const Split sp{pick.slices > 1 ? partial : nullptr, pick.per, (int)whole4(K)};
  if (is_bf16) {
    T2I_TILES_GRAD(pick.shape, (adapter_dx_launch<D, bf16>(dy, lddy, w, ldw, M, N, K, up, (bf16*)dx, ldx, pick, sp, st)))
  } else if (f32_pieces({N, K, lddy, ldw}, {dy, w})) {
    T2I_TILES_F32_FWD(pick.shape,
                      (adapter_dx_launch<D, float>(dy, lddy, w, ldw, M, N, K, up, (float*)dx, ldx, pick, sp, st)))
  } else {
    T2I_TILES_F32_FWD(pick.shape,
                      (adapter_dx_launch<D, float, true>(dy, lddy, w, ldw, M, N, K, up, (float*)dx, ldx, pick, sp, st)))
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// What the gradients need first, in one launch: the rows of every adapter, the adapters'
// matrices turned, and, of few rows, u = s dy B straight from B.
//
// Adapter i's rows, in ascending order, are order[start .. start + count), (start, count) =
// span[i].  Cut at every multiple of `per` they are the slices of the gradients' sums;
// slice b of adapter i has number b + i in `slices` (adapter, first, rows, place), so that
// each number below M / per + n is written by one workgroup, empty ones too.  An adapter's
// only slice, or its first if it has no rows, goes to the gradients (kWhole), a further empty
// one nowhere (kNowhere).  Of slices b at most one goes on from b - 1 and at most one begins
// and goes on to b + 1: their places among the partial sums are 2 b and 2 b + 1, however many
// adapters there are.  A workgroup per adapter reads the whole index twice.
constexpr int kWhole = -1, kNowhere = -2;
__device__ __forceinline__ int place_of(int b, int start, int count, int per) {
  const int b0 = start / per, b1 = count > 0 ? (start + count - 1) / per : b0;
  return b > b1 ? kNowhere : b0 == b1 ? kWhole : b == b0 ? 2 * b + 1 : 2 * b;
}
__device__ __forceinline__ void group_rows(const AdapterPrepare& p, int ad) {
  __shared__ int red[2][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, M = p.M;
  int before = 0, mine = 0;
#pragma unroll 4
  for (int m = threadIdx.x; m < M; m += 1024) {
    const int i = adapter_of(p.index, p.n, m);
    before += i >= 0 && i < ad;
    mine += i == ad;
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    before += __shfl_xor(before, o, kWave);
    mine += __shfl_xor(mine, o, kWave);
  }
  if (lane == 0) red[0][wave] = before, red[1][wave] = mine;
  __syncthreads();
  int start = 0, count = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) start += red[0][w], count += red[1][w];
  if (threadIdx.x == 0) p.span[ad] = int2{start, count};
  // (the last adapter's also write the numbers that rows without an adapter leave over)
  const int end = start + count, last = ad == p.n - 1 ? M / p.per : end / p.per;
  for (int b = start / p.per + (int)threadIdx.x; b <= last; b += 1024) {
    const int lo = max(start, b * p.per), hi = min(end, (b + 1) * p.per);
    p.slices[b + ad] = int4{ad, lo, max(hi - lo, 0), place_of(b, start, count, p.per)};
  }
  if (count == 0) return;
  int at = start;
  int next = (int)threadIdx.x < M ? adapter_of(p.index, p.n, threadIdx.x) : -1;
  for (int m0 = 0; m0 < M; m0 += 1024) {
    const int m = m0 + (int)threadIdx.x;
    const bool hit = next == ad;
    next = m + 1024 < M ? adapter_of(p.index, p.n, m + 1024) : -1;
    const uint64_t all = __ballot(hit);
    __syncthreads();   // (the counts of the round before, or of the sums, are read)
    if (lane == 0) red[0][wave] = __popcll(all);
    __syncthreads();
    int skip = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      skip += w < wave ? red[0][w] : 0;
      sum += red[0][w];
    }
    if (hit) p.order[at + skip + __popcll(all & ((1ULL << lane) - 1))] = m;
    at += sum;
  }
}

// out[i][c][r] = in[i][r][c] for rows r < R, 0 for R <= r < stride, thread x of all: 8
// values of a row of out
template <typename T>
__device__ __forceinline__ void turn_rows(const AdapterTurn& d, long x) {
  const long chunks = (d.stride + 7) / 8, per = chunks * d.C;
  const int ad = (int)(x / per);
  x -= ad * per;
  const int c = (int)(x % d.C), r0 = (int)(x / d.C) * 8;
  const T* const p = (const T*)d.in + (size_t)ad * d.R * d.C + c;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = r0 + i < d.R ? to_f32(p[(size_t)(r0 + i) * d.C]) : 0.f;
  store_piece((T*)d.out + ((size_t)ad * d.C + c) * d.stride + r0, d.stride - r0, v);
}

// u of few rows: a workgroup takes one row and 32 ranks, G lanes eight ranks each of a row of
// B, 64 / G rows side by side
template <typename T>
__device__ __forceinline__ void up_rows(const AdapterPrepare& p, int block) {
  __shared__ float red[16][32];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cols = adapter_cols(p.rank), per = cols / 32;
  const int m = block / per, first = block % per * 32;
  const int ranks = min(p.rank - first, 32), G = ranks <= 8 ? 1 : ranks <= 16 ? 2 : 4;
  const int ad = adapter_of(p.index, p.n, m), j0 = first + (lane & (G - 1)) * 8;
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (ad >= 0 && j0 < p.rank) {
    const T* const dy = (const T*)p.dy + (size_t)m * p.lddy;
    const T* const b = (const T*)p.b + (size_t)ad * p.N * p.rank;
    const int step = 64 / G;
#pragma unroll 4
    for (int c = wave * step + lane / G; c < p.N; c += 16 * step) {
      Piece<T> v;
      load_piece(b + (size_t)c * p.rank, j0, p.rank, v);
      const float d = to_f32(dy[c]);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = fmaf(d, v.get(j), s[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      const float y = __shfl_xor(s[j], o, kWave);
      s[j] += o >= G ? y : 0.f;
    }
    if (lane < 4) red[wave][lane * 8 + j] = lane < G ? s[j] : 0.f;
  }
  __syncthreads();
  if (threadIdx.x >= 32) return;
  float v = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) v += red[w][lane];
  const float scale = ad >= 0 ? (p.scale ? p.scale[ad] : 1.f) : 0.f;
  p.u[(size_t)m * cols + first + lane] = ad >= 0 && first + lane < p.rank ? v * scale : 0.f;
}

template <typename T>
__global__ __launch_bounds__(1024) void adapter_prepare_kernel(AdapterPrepare p) {
  int block = blockIdx.x;
  if (block < p.groups) {
    group_rows(p, block);
    return;
  }
  block -= p.groups;
  if (block < p.rows) {
    up_rows<T>(p, block);
    return;
  }
  block -= p.rows;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const AdapterTurn& d = p.turn[i];
    if (block < d.blocks) {
      const long x = block * 1024L + threadIdx.x;
      if (x < (long)((d.stride + 7) / 8) * d.C * p.n) turn_rows<T>(d, x);
      return;
    }
    block -= d.blocks;
  }
}
hipError_t launch_adapter_prepare(bool is_bf16, AdapterPrepare p, hipStream_t st) {
  p.rows = p.dy ? p.M * (adapter_cols(p.rank) / 32) : 0;
  long blocks = p.groups + p.rows;
  for (AdapterTurn& d : p.turn) {
    d.blocks = d.in ? (int)(((long)((d.stride + 7) / 8) * d.C * p.n + 1023) / 1024) : 0;
    blocks += d.blocks;
  }
  if (blocks == 0) return hipSuccess;
  if (is_bf16) hipLaunchKernelGGL((adapter_prepare_kernel<bf16>), dim3((unsigned)blocks), dim3(1024), 0, st, p);
  else hipLaunchKernelGGL((adapter_prepare_kernel<float>), dim3((unsigned)blocks), dim3(1024), 0, st, p);
  return hipGetLastError();
}

// u of up to so many products in the first launch: no second one, and B need not be
// turned (fp32 333 x 1155 x 1153, rank 5: 4.2 + 6.3 us in two launches, 7.9 in one)
bool adapter_few_rows(int M, int N, int rank) { return M <= 1024 && (int64_t)M * N * rank <= 1 << 23; }

constexpr int kSliceRows = 1024;
// rows of a slice: all of up to 768, whose sums are then done without a second launch;
// else the most, up to kSliceRows, that leave 384 workgroups (adapters cut the slices, too;
// up to 16 ranks, where a wave has one step's loads under way instead of two: 1024), at
// least a step of four waves.  dA and dB alone, 7531 x 4608 x 1152, rank 32, 8 adapters 67
// us with 1024 rows, 71 with 512, 87 with 128; 3320 x 224 x 4256, rank 32 36, 30, 36; 4096 x
// 4096 x 4096, rank 16 41, 35, 38, 34 with 256 (t in two bf16 parts; in three 35.5).
int adapter_slice_rows(bool is_bf16, int M, int N, int K, int n, int rank) {
  if (M <= 768) return kSliceRows;
  const int cols = is_bf16 ? 128 : 64;
  const long wide = (long)((K + cols - 1) / cols + (N + cols - 1) / cols) * ((rank + 31) / 32);
  int per = kSliceRows;
  while (per > 128 && ((M + per - 1) / per + n / 2) * wide < (rank <= 16 ? 1024 : 384)) per /= 2;
  return per;
}

// One slice's part of the gradients: partial[place][j][c] = sum over its rows of v[m, j]
// z[m, c], with (z, v) = (x, u) for dA and (dy, t) for dB, side by side in the grid.  A
// wave takes every fourth step of 32 (fp32: 16) of the slice's rows and 128 (64)
// columns: a lane reads 16 bytes of each of its 8 (4) rows and joins the halves of
// their dwords by v_perm, which gives it 8 (4) k of 8 (4) neighbouring columns, the
// operands of as many MFMAs; z is read once for 32 ranks.
template <typename T, int RT>
__global__ __launch_bounds__(256, RT == 1 ? 4 : 2) void adapter_outer_kernel(AdapterOuter p) {
  constexpr int L = kLaneK<T>, STEP = 4 * L, COLS = 16 * L;
  __shared__ f32x4 red[3][RT][64];
  __shared__ int order[kSliceRows];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, fr = lane & 15, g = lane >> 4;
  const bool second = (int)blockIdx.x >= p.blocks0;
  const AdapterSide& d = second ? p.side[1] : p.side[0];
  const int c0 = ((int)blockIdx.x - (second ? p.blocks0 : 0)) * COLS + fr * L, C = d.cols, j0 = blockIdx.z * RT * 16;
  int ad, first, rows, place;
  if (p.slices) {
    const int4 sl = p.slices[blockIdx.y];
    ad = sl.x, first = sl.y, rows = sl.z, place = sl.w;
  } else {   // (all rows are adapter 0's; if they are one slice, slice i is adapter i's)
    ad = p.M <= p.per ? blockIdx.y : 0;
    first = blockIdx.y * p.per, rows = max(0, min(p.per, p.M - first));
    place = p.M <= p.per ? kWhole : place_of(blockIdx.y, 0, p.M, p.per);
  }
  if (place == kNowhere) return;
  const T* const z = (const T*)d.z;
  const float* const v = d.v;
  const bool in = c0 < C, part = c0 + L > C;
  f32x4 acc[L][RT];
#pragma unroll
  for (int q = 0; q < L; ++q)
#pragma unroll
    for (int jt = 0; jt < RT; ++jt) acc[q][jt] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int r = threadIdx.x; r < rows; r += 256) order[r] = p.order ? p.order[first + r] : first + r;
  __syncthreads();
  // a step's operands, zeros behind the last row; of 32 ranks the next step's are under way
  // while one is multiplied
  struct Step {
    i32x4 raw[L];
    float e[RT][L];
  };
  auto load = [&](int r0, Step& x) {
    int row[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int at = r0 + g * L + i;
      row[i] = at < rows ? order[at] : -1;
    }
#pragma unroll
    for (int i = 0; i < L; ++i) {
      x.raw[i] = i32x4{0, 0, 0, 0};
      if (row[i] >= 0 && in) x.raw[i] = load_k<T>(z + (size_t)row[i] * d.ldz, 0, c0, C, !part);
    }
#pragma unroll
    for (int jt = 0; jt < RT; ++jt) {
      const int j = min(j0 + jt * 16 + fr, d.ldv - 1);
#pragma unroll
      for (int i = 0; i < L; ++i) x.e[jt][i] = row[i] >= 0 ? v[(size_t)row[i] * d.ldv + j] : 0.f;
    }
  };
  auto multiply = [&](const Step& x) {
    Exact<T> vv[RT];
#pragma unroll
    for (int jt = 0; jt < RT; ++jt) vv[jt].set(x.e[jt]);
#pragma unroll
    for (int q = 0; q < L; ++q) {
      i32x4 f;
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
          f[w] = __builtin_amdgcn_perm(x.raw[2 * w + 1][q / 2], x.raw[2 * w][q / 2], q & 1 ? 0x07060302 : 0x05040100);
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) f[w] = x.raw[w][q];
      }
#pragma unroll
      for (int jt = 0; jt < RT; ++jt) acc[q][jt] = narrow_mfma<T>(vv[jt], f, acc[q][jt]);
    }
  };
  Step even, odd;
  int r0 = wave * STEP;
  if constexpr (RT == 1) {   // (more waves instead)
#pragma unroll 1
    for (; r0 < rows; r0 += 4 * STEP) {
      load(r0, even);
      multiply(even);
    }
  } else {
    load(r0, even);
#pragma unroll 1
    for (; r0 < rows; r0 += 8 * STEP) {
      load(r0 + 4 * STEP, odd);   // (behind the last row: zeros)
      multiply(even);
      if (r0 + 4 * STEP >= rows) break;
      load(r0 + 8 * STEP, even);
      multiply(odd);
    }
  }
  // lane (fr, g) holds ranks 4 g + r of column c0 + q: the other waves' sums by way of LDS,
  // in ascending order (of one step only the first has any)
#pragma unroll
  for (int q = 0; q < L; ++q) {
    if (rows <= STEP) break;
    __syncthreads();
    if (wave > 0) {
#pragma unroll
      for (int jt = 0; jt < RT; ++jt) red[wave - 1][jt][lane] = acc[q][jt];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int jt = 0; jt < RT; ++jt) acc[q][jt] += red[w][jt][lane];
    }
  }
  if (wave > 0 || !in) return;
  if (place == kWhole) {
    T* const done = (T*)d.grad;
    const int left = C - c0;
#pragma unroll
    for (int jt = 0; jt < RT; ++jt) {
      const int j = j0 + jt * 16 + g * 4, ranks = p.rank - j;
      if (ranks <= 0) continue;
      if (second) {   // dB [N][rank]: four ranks of a column
#pragma unroll
        for (int q = 0; q < L; ++q) {
          const float w[4] = {acc[q][jt][0], acc[q][jt][1], acc[q][jt][2], acc[q][jt][3]};
          if (q < left) store4(done + ((size_t)ad * C + c0 + q) * p.rank + j, ranks, w);
        }
      } else {        // dA [rank][K]: neighbouring columns of a rank
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (r < ranks)
#pragma unroll
            for (int q = 0; q < L; q += 4) {
              const float w[4] = {acc[q][jt][r], acc[q + 1][jt][r], acc[q + 2][jt][r], acc[q + 3][jt][r]};
              if (q < left) store4(done + ((size_t)ad * p.rank + j + r) * C + c0 + q, left - q, w);
            }
      }
    }
    return;
  }
  float* const out = d.partial + (size_t)place * p.ranks * d.ldp + c0;
#pragma unroll
  for (int jt = 0; jt < RT; ++jt)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int j = j0 + jt * 16 + g * 4 + r;
      if (j >= p.ranks) continue;
#pragma unroll
      for (int q = 0; q < L; q += 4)   // (rows of ldp columns, a multiple of a lane's)
        *(f32x4*)(out + (size_t)j * d.ldp + q) = f32x4{acc[q][jt][r], acc[q + 1][jt][r], acc[q + 2][jt][r], acc[q + 3][jt][r]};
    }
}

// dA [n][rank][K] and dB [n][N][rank] of adapters of several slices: their parts, added up
// in fp64 in ascending order; zeros for the adapters that rows without an index do not take.
// A thread takes four columns of one rank (dA), or one column of four (dB).
template <typename T>
__global__ __launch_bounds__(256) void adapter_sum_kernel(AdapterOuter p, T* dA, T* dB, int per_a) {
  const int ad = blockIdx.y;
  const int2 span = p.span ? p.span[ad] : int2{0, ad == 0 ? p.M : 0};
  const int b0 = span.x / p.per, b1 = span.y > 0 ? (span.x + span.y - 1) / p.per + 1 : b0;
  if (p.span && b1 <= b0 + 1) return;
  const bool is_b = (int)blockIdx.x >= per_a;
  const long x = ((int)blockIdx.x - (is_b ? per_a : 0)) * 256L + threadIdx.x;
  const AdapterSide& d = is_b ? p.side[1] : p.side[0];
  const int per_row = is_b ? d.cols : (d.cols + 3) / 4;
  const int c = (int)(x % per_row) * (is_b ? 1 : 4), j0 = (int)(x / per_row) * (is_b ? 4 : 1);
  if (j0 >= p.rank) return;
  const size_t slice = (size_t)p.ranks * d.ldp;
  const float* const parts = d.partial + (size_t)j0 * d.ldp + c;
  auto part = [&](int b) { return parts + (size_t)(b == b0 ? 2 * b + 1 : 2 * b) * slice; };
  double s[4] = {0., 0., 0., 0.};
  if (!is_b) {
#pragma unroll 4
    for (int b = b0; b < b1; ++b) {
      const f32x4 v = *(const f32x4*)part(b);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += (double)v[e];
    }
  } else {
#pragma unroll 4
    for (int b = b0; b < b1; ++b) {
      const float* const at = part(b);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += (double)at[(size_t)e * d.ldp];
    }
  }
  const float v[4] = {(float)s[0], (float)s[1], (float)s[2], (float)s[3]};
  if (!is_b) store4(dA + ((size_t)ad * p.rank + j0) * d.cols + c, d.cols - c, v);
  else store4(dB + ((size_t)ad * d.cols + c) * p.rank + j0, p.rank - j0, v);
}

// slices of the launch: with an index M / per + n numbers; of up to one slice of rows one
// for every adapter, which need no sums
int adapter_slices(bool indexed, int M, int n, int per) {
  return (indexed ? M < per : M <= per) ? n : indexed ? M / per + n : (M + per - 1) / per;
}
// places of the partial sums
int adapter_places(int M, int per) { return M < per ? 0 : 2 * ((M - 1) / per + 1); }

template <typename T>
static void outer_any(AdapterOuter p, int n, T* dA, T* dB, hipStream_t st) {
  constexpr int COLS = 16 * kLaneK<T>;
  const int slices = adapter_slices(p.slices != nullptr, p.M, n, p.per);
  const bool direct = p.slices ? p.M < p.per : p.M <= p.per;
  p.side[0].grad = dA, p.side[1].grad = dB;
  const int blocks1 = dB ? (p.side[1].cols + COLS - 1) / COLS : 0;
  p.blocks0 = dA ? (p.side[0].cols + COLS - 1) / COLS : 0;
  if (p.rank <= 16)
    hipLaunchKernelGGL((adapter_outer_kernel<T, 1>), dim3((unsigned)(p.blocks0 + blocks1), (unsigned)slices, 1), dim3(256),
                       0, st, p);
  else
    hipLaunchKernelGGL((adapter_outer_kernel<T, 2>),
                       dim3((unsigned)(p.blocks0 + blocks1), (unsigned)slices, (unsigned)((p.rank + 31) / 32)), dim3(256), 0,
                       st, p);
  if (direct) return;
  const int a = dA ? (int)(((long)((p.side[0].cols + 3) / 4) * p.rank + 255) / 256) : 0;
  const int b = dB ? (int)(((long)p.side[1].cols * ((p.rank + 3) / 4) + 255) / 256) : 0;
  hipLaunchKernelGGL((adapter_sum_kernel<T>), dim3((unsigned)(a + b), (unsigned)n), dim3(256), 0, st, p, dA, dB, a);
}
hipError_t launch_adapter_outer(bool is_bf16, const AdapterOuter& p, int n, void* dA, void* dB, hipStream_t st) {
  if (is_bf16) outer_any(p, n, (bf16*)dA, (bf16*)dB, st);
  else outer_any(p, n, (float*)dA, (float*)dB, st);
  return hipGetLastError();
}

}  // namespace t2i
