// Row-wise block operators (gfx950): quantising rows to 8 bits, the gated
// feed-forward's elementwise gradients, RMS norm of query and key heads with
// the position rotation, and its gradients.  All of them are bound by HBM:
// each input is read once, 16 bytes per lane (the gate gradients in fp32: 4), held in
// registers, and each output written once.
#include <algorithm>

#include "block_ops.h"

namespace t2i {

// eight consecutive elements as fp32 (16 bytes of bf16, 32 of fp32)
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<bf16>(const bf16* p, float (&v)[8]) {
  const bf16x8 w = *(const bf16x8*)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)w[i];
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 w;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = (bf16)v[i];
    *(bf16x8*)p = w;
  } else {
    *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  }
}

// Groups of G lanes in a workgroup of 256: powers of two, or nine lanes (heads of 72),
// seven groups to a wave.
template <int G>
struct Groups {
  static constexpr int WAVE = 64 / G, ALL = 4 * WAVE;
  int lane, group;   // of the group; of the workgroup
  bool live;         // (nine: the 64th lane has no group)
  __device__ __forceinline__ Groups() {
    const int l = threadIdx.x & 63;
    lane = l % G, group = (threadIdx.x >> 6) * WAVE + l / G, live = l < WAVE * G;
  }
  // sum over the group's lanes, the same in each of them
  __device__ __forceinline__ float sum(float v) const {
    if constexpr ((G & (G - 1)) == 0) {
#pragma unroll
      for (int o = G / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, kWave);
      return v;
    } else {
      static_assert(G == 9, "lanes of a head");
      const int base = (threadIdx.x & 63) - lane;
      float s = v;
#pragma unroll
      for (int o = 1; o <= 4; o *= 2) s += __shfl(s, lane + o < G ? base + lane + o : base, kWave);
      // (the first lane's: eight lanes from it on, and the ninth)
      return __shfl(s, base, kWave) + __shfl(v, base + 8, kWave);
    }
  }
};

// ---------------------------------------------------------------------------
// Quantising rows: s = max(max |x| / 127, 2^-126) in fp32, q = x / s to the
// nearest whole number, ties to even, of the exact quotient.
//
// The rounding costs no division: m = fma(x, 1/s, 1.5 2^23) leaves the nearest
// whole number n in its low bits, wrong by one at most and only where x / s lies
// within the error of 1/s of a half.  r = fma(-n, s, x) is exact (|r| is at most
// about s / 2 and a multiple of s's last place over four), so |r| against s / 2
// says which pieces hold such a value; those (about one value in 10^5) are
// settled by comparing 2 r with s.
// A row with a NaN or an infinity gets s = NaN and q = 0: its outputs are NaN.
// 4096 rows of 12288 31 us (4.9 TB/s), 7531 of 1152 9.8 us (2.7 TB/s: one round of
// waves, whose loads, maximum and stores follow each other; fewer waves with the
// next row's loads ahead took 10.7 - 13.3).

__device__ __forceinline__ int quant1(float x, float s, float inv) {
  float n = rintf(x * inv);
  const float r2 = 2.f * fmaf(-n, s, x);
  const bool odd = ((int)n & 1) != 0;
  if (r2 > s || (r2 == s && odd)) n += 1.f;
  else if (r2 < -s || (r2 == -s && odd)) n -= 1.f;
  return (int)n;
}

// eight elements of a row as they lie in memory (at any address: one or two loads all
// the same), and the largest of their magnitudes' bits (which order as the magnitudes
// do, infinity and NaN above)
template <typename T>
struct Piece;
template <>
struct Piece<bf16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const bf16* p) {
    typedef uint32_t any4 __attribute__((ext_vector_type(4), aligned(2)));
    const any4 v = *(const any4*)p;
    w[0] = v[0], w[1] = v[1], w[2] = v[2], w[3] = v[3];
  }
  __device__ __forceinline__ void set(int i, bf16 v) {
    const uint32_t b = __builtin_bit_cast(uint16_t, v);
    w[i >> 1] |= b << (16 * (i & 1));
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 0;
  }
  __device__ __forceinline__ float get(int i) const {
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
  __device__ __forceinline__ uint32_t largest() const {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    return (uint32_t)max((uint32_t)m[0], (uint32_t)m[1]) << 16;
  }
};
template <>
struct Piece<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* p) {
    typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
    const any4 a = *(const any4*)p, b = *(const any4*)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
  __device__ __forceinline__ void set(int i, float x) { v[i] = x; }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  }
  __device__ __forceinline__ float get(int i) const { return v[i]; }
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
  }
};

// TPR threads per row, NV pieces per thread in registers; longer rows read their
// pieces again.
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(256) void quant_rows_kernel(const T* __restrict__ x, int ldx, int rows,
                                                         int K, int8_t* __restrict__ q, int ldq,
                                                         float* __restrict__ scale) {
  constexpr int RPB = 256 / TPR;
  __shared__ uint32_t red[RPB][TPR / 64];
  const int t = threadIdx.x % TPR, rl = threadIdx.x / TPR;
  const int row = blockIdx.x * RPB + rl;
  const bool live = row < rows;
  const T* xr = x + (size_t)(live ? row : 0) * ldx;
  Piece<T> v[NV];
  auto load = [&](int c, Piece<T>& p) {
    const int k = c * 8;
    if (k + 8 <= K) {
      p.load(xr + k);
    } else {
      p.clear();
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < K) p.set(i, xr[k + i]);
    }
  };
  const int chunks = (K + 127) / 128 * 16;   // the zeros behind K too
  uint32_t m = 0;
  const int rounds = (chunks + TPR * NV - 1) / (TPR * NV);
  for (int r = 0; r < rounds; ++r) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (r * NV + i) * TPR + t;
      if (c < chunks) load(c, v[i]);
      else v[i].clear();
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) m = max(m, v[i].largest());
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, kWave));
  if constexpr (TPR > 64) {
    if ((t & 63) == 0) red[rl][t >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) m = max(m, red[rl][i]);
  }
  const bool finite = m < 0x7f800000u;
  const float s = fmaxf(__uint_as_float(finite ? m : 0u) / 127.f, 1.17549435e-38f);
  const float inv = 1.f / s;
  // (below s / 2 by its last place: 0.5 s may be off by that where s is near 2^-126)
  const float near_half = 0.5f * s * (1.f - 2.4e-7f);
  if (live && t == 0) scale[row] = finite ? s : __uint_as_float(0x7fc00000u);
  if (!live) return;
  for (int r = 0; r < rounds; ++r) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (r * NV + i) * TPR + t;
      if (c >= chunks) break;
      if (rounds > 1) load(c, v[i]);
      uint32_t w[2] = {0, 0};
      if (finite) {
        constexpr float MAGIC = 12582912.f;   // 1.5 2^23
        uint32_t b[8];
        float far = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float xv = v[i].get(j), mg = fmaf(xv, inv, MAGIC);
          far = fmaxf(far, fabsf(fmaf(MAGIC - mg, s, xv)));
          b[j] = __float_as_uint(mg);
        }
        if (far >= near_half)
#pragma unroll
          for (int j = 0; j < 8; ++j) b[j] = (uint32_t)quant1(v[i].get(j), s, inv);
#pragma unroll
        for (int h = 0; h < 2; ++h)
          w[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x0c0c0400),
                                       __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x0c0c0400), 0x05040100);
      }
      *(uint2*)(q + (size_t)row * ldq + c * 8) = uint2{w[0], w[1]};
    }
  }
}

template <typename T>
static void quant_rows_any(int rows, int K, const T* x, int ldx, int8_t* q, int ldq, float* scale, hipStream_t st) {
#define T2I_Q(TPR, NV)                                                                                      \
  hipLaunchKernelGGL((quant_rows_kernel<T, TPR, NV>), dim3((unsigned)((rows + 256L / TPR - 1) / (256 / TPR))), \
                     dim3(256), 0, st, x, ldx, rows, K, q, ldq, scale)
  // one wave per row up to 2048 elements, a workgroup for longer rows; just the
  // pieces that the row has, up to what registers hold
  if (K <= 512) T2I_Q(64, 1);
  else if (K <= 1024) T2I_Q(64, 2);
  else if (K <= 1536) T2I_Q(64, 3);
  else if (K <= 2048) T2I_Q(64, 4);
  else if (K <= 4096) T2I_Q(256, 2);
  else if (K <= 8192) T2I_Q(256, 4);
  else T2I_Q(256, 8);
#undef T2I_Q
}

hipError_t launch_quant_rows(bool bf16_in, int rows, int K, const void* x, int ldx, int8_t* q,
                             int ldq, float* scale, hipStream_t st) {
  if (bf16_in) quant_rows_any(rows, K, (const bf16*)x, ldx, q, ldq, scale, st);
  else quant_rows_any(rows, K, (const float*)x, ldx, q, ldq, scale, st);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Query / key norm with rotation.  G lanes hold one head, 8 elements each (G = the
// power of two at or above head_dim / 8, or nine); a group keeps one row's rotation and
// takes HPG of its heads, all of whose loads are under way before the first norm.  The
// position, its table row and the two weights are loaded one after the other behind them,
// and two of the rotation's values pass through scratch memory (the branches of
// Rotor::load meet in one store): 12.6 of the 125.8 MB written below.  9216
// rows of 48 heads of 128 42 - 52 us (4.5 - 5.4 TB/s; a copy 5.1), 4451 rows of 32 heads
// of 72 10.8 us (3.8 TB/s; with 16 lanes of which nine work 13.0, 20000 rows of 28 heads
// 39.3 -> 31.9 and backward 75.2 -> 54.3).  72, the cross-attention models' head size, has
// the most to gain of the sizes between powers of two (7 heads to a wave instead of 4; 40
// would have 12 instead of 8, 80 6 instead of 4, 96 5 instead of 4, 160 3 instead of 2);
// those keep the power of two, and no other count was built or measured for them.

// The rotation of a lane's elements.  Pairs (2j, 2j + 1): four pairs in the lane.
// Halves (j, j + d/2): eight elements whose partners sit in another lane.
template <bool HALVES>
struct Rotor {
  static constexpr int N = HALVES ? 8 : 4;
  float c[N], s[N];
  bool turn;
  int partner;   // lane of the wave that holds the other half

  // lg: lane within the head, nl: lanes in use; inverse: the transposed rotation
  __device__ __forceinline__ void load(const QkNorm& a, int row, int lg, int nl, bool inverse) {
    turn = false;
    partner = threadIdx.x & 63;
    if (!a.table) return;
    const int pos = a.pos ? a.pos[row] : row;
    if (pos < 0) return;
    turn = true;
    float sg = inverse ? -1.f : 1.f;
    if (HALVES) {
      const int hl = nl / 2;
      partner += lg < hl ? hl : lg < nl ? -hl : 0;
      if (lg < hl) sg = -sg;
      lg -= lg < hl ? 0 : hl;
    }
    if (pos >= a.n_pos || lg * N >= a.head_dim / 2) {   // behind the table (or a spare lane)
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] = s[i] = __uint_as_float(0x7fc00000u);
      return;
    }
    const float4* t = (const float4*)(a.table + (size_t)pos * (a.head_dim / 2) + lg * N);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float4 p = t[i];
      c[2 * i] = p.x, s[2 * i] = sg * p.y, c[2 * i + 1] = p.z, s[2 * i + 1] = sg * p.w;
    }
  }
  __device__ __forceinline__ void apply(float (&v)[8]) const {
    if (HALVES) {
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = __shfl(v[i], partner, kWave);
      if (turn)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(o[i], s[i], v[i] * c[i]);
    } else if (turn) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = v[2 * i], y = v[2 * i + 1];
        v[2 * i] = fmaf(-y, s[i], x * c[i]);
        v[2 * i + 1] = fmaf(x, s[i], y * c[i]);
      }
    }
  }
};

template <typename T>
__device__ __forceinline__ void load_weight(const void* w, int lg, int nl, float (&v)[8]) {
  if (w && lg < nl) load8((const T*)w + lg * 8, v);
  else
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.f;
}

template <typename T, int G, bool HALVES, int HPG>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkNorm a, int upr) {
  const Groups<G> gr;
  const int lg = gr.lane, nl = a.head_dim / 8, H = a.heads_q + a.heads_k;
  const unsigned unit = blockIdx.x * Groups<G>::ALL + gr.group;
  const unsigned r = unit / (unsigned)upr;
  const int h0 = (int)(unit - r * (unsigned)upr);
  const bool live = r < (unsigned)a.rows && lg < nl && gr.live;
  const int row = r < (unsigned)a.rows ? (int)r : 0;
  float v[HPG][8];
#pragma unroll
  for (int i = 0; i < HPG; ++i) {
    const int h = h0 + i * upr;
    if (live && h < H) {
      const T* p = h < a.heads_q ? (const T*)a.q + (size_t)row * a.ldq + h * a.head_dim
                                 : (const T*)a.k + (size_t)row * a.ldk + (h - a.heads_q) * a.head_dim;
      load8(p + lg * 8, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
  }
  Rotor<HALVES> rot;
  rot.load(a, row, lg, nl, false);
  float wq[8], wk[8];
  load_weight<T>(a.wq, lg, nl, wq);
  load_weight<T>(a.wk, lg, nl, wk);
  const float rd = 1.f / (float)a.head_dim;
#pragma unroll
  for (int i = 0; i < HPG; ++i) {
    const int h = h0 + i * upr;
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) ss = fmaf(v[i][j], v[i][j], ss);
    const float rs = rsqrtf(fmaf(gr.sum(ss), rd, a.eps));
    const bool isq = h < a.heads_q;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * rs * (isq ? wq[j] : wk[j]);
    rot.apply(v[i]);
    if (live && h < H) {
      T* p = isq ? (T*)a.oq + (size_t)row * a.ldoq + h * a.head_dim
                 : (T*)a.ok + (size_t)row * a.ldok + (h - a.heads_q) * a.head_dim;
      store8(p + lg * 8, v[i]);
    }
  }
}

// lanes that hold one head, and groups of them in a workgroup
static int head_lanes(int head_dim) {
  if (head_dim == 9 * 8) return 9;
  int g = 1;
  while (g * 8 < head_dim) g *= 2;
  return g;
}
static int head_groups(int head_dim) { return 64 / head_lanes(head_dim) * 4; }

// heads per group of the forward kernel (two: 9216 rows of 48 heads of 128 54.3 us,
// four 51.9, six 51.4 but 22.0 instead of 20.5 for 16384 of 20 heads of 64)
constexpr int kFwdHeads = 4;
// several heads of a row per group where that still leaves workgroups enough
static int qk_fwd_hpg(int rows, int heads, int head_dim) {
  return (long)rows * ((heads + kFwdHeads - 1) / kFwdHeads) / head_groups(head_dim) >= 1024 ? kFwdHeads : 1;
}
template <typename T, int G, bool HALVES>
static void qk_launch(const QkNorm& a, hipStream_t st) {
  const int H = a.heads_q + a.heads_k;
  const int gr = Groups<G>::ALL;
  const int hpg = qk_fwd_hpg(a.rows, H, a.head_dim);
  const int upr = (H + hpg - 1) / hpg;
  const dim3 grid((unsigned)(((long)a.rows * upr + gr - 1) / gr));
  if (hpg > 1)
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, G, HALVES, kFwdHeads>), grid, dim3(256), 0, st, a, upr);
  else
    hipLaunchKernelGGL((qk_norm_rope_kernel<T, G, HALVES, 1>), grid, dim3(256), 0, st, a, upr);
}

// Backward.  With n = x r, r = (mean x^2 + eps)^-1/2, y = R (n w):
//   dn = (R^T dy) w,  dx = r (dn - n mean(dn n)),  dw = sum over rows and heads
//   of (R^T dy) n.
// 9216 rows of 48 heads of 128 86 us (4.0 TB/s), 4451 of 32 heads of 72 20.6 us with
// the second launch (16 lanes for a head of 72: 24.6).
// A fixed number of workgroups walks the (row, heads) units; dw adds up in fp32
// registers (a lane's own units: up to 28 of them at 9216 rows of 48 heads of 128), then
// in fp64 over the workgroup in LDS, whose sum is kept in fp32, and
// (qk_weight_grad_kernel) over the workgroups: a fixed order.
template <typename T, int G, bool HALVES, int HPG>
__global__ __launch_bounds__(256) void qk_norm_rope_bwd_kernel(QkNorm a, int upr, float* __restrict__ partial) {
  constexpr int GR = Groups<G>::ALL;
  __shared__ float red[2][GR][G * 8];
  const Groups<G> gr;
  const int lg = gr.lane, gi = gr.group, nl = a.head_dim / 8;
  const int H = a.heads_q + a.heads_k;
  const unsigned units = (unsigned)a.rows * (unsigned)upr, stride = gridDim.x * GR;
  float wq[8], wk[8], aq[8], ak[8];
  load_weight<T>(a.wq, lg, nl, wq);
  load_weight<T>(a.wk, lg, nl, wk);
#pragma unroll
  for (int j = 0; j < 8; ++j) aq[j] = ak[j] = 0.f;
  const float rd = 1.f / (float)a.head_dim;
  for (unsigned u0 = blockIdx.x * GR; u0 < units; u0 += stride) {
    const unsigned u = u0 + gi;
    const bool in = u < units && lg < nl && gr.live;
    const int row = u < units ? (int)(u / (unsigned)upr) : 0;
    const int h0 = u < units ? (int)(u - (unsigned)row * (unsigned)upr) : 0;
    float x[HPG][8], dy[HPG][8];
#pragma unroll
    for (int i = 0; i < HPG; ++i) {
      const int h = h0 + i * upr;
      const bool isq = h < a.heads_q;
      const int at = (isq ? h : h - a.heads_q) * a.head_dim + lg * 8;
      if (in && h < H) {
        load8((isq ? (const T*)a.q + (size_t)row * a.ldq : (const T*)a.k + (size_t)row * a.ldk) + at, x[i]);
        load8((isq ? (const T*)a.dq + (size_t)row * a.lddq : (const T*)a.dk + (size_t)row * a.lddk) + at, dy[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = dy[i][j] = 0.f;
      }
    }
    Rotor<HALVES> rot;
    rot.load(a, row, lg, nl, true);
#pragma unroll
    for (int i = 0; i < HPG; ++i) {
      const int h = h0 + i * upr;
      const bool isq = h < a.heads_q, live = in && h < H;
      float (&n)[8] = x[i], (&d)[8] = dy[i];
      rot.apply(d);
      if (!live)
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = 0.f;   // (a spare lane's rotation is NaN)
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(n[j], n[j], ss);
      const float r = rsqrtf(fmaf(gr.sum(ss), rd, a.eps));
      float dot = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        n[j] = live ? n[j] * r : 0.f;
        const float p = d[j] * n[j];
        if (isq) aq[j] += p;
        else ak[j] += p;
        d[j] *= isq ? wq[j] : wk[j];
        dot = fmaf(d[j], n[j], dot);
      }
      dot = gr.sum(dot) * rd;
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = r * fmaf(-n[j], dot, d[j]);
      if (live)
        store8((isq ? (T*)a.oq + (size_t)row * a.ldoq : (T*)a.ok + (size_t)row * a.ldok) +
                   (isq ? h : h - a.heads_q) * a.head_dim + lg * 8, d);
    }
  }
  if (!partial) return;
  if (gr.live)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      red[0][gi][lg * 8 + j] = aq[j];
      red[1][gi][lg * 8 + j] = ak[j];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * a.head_dim; i += 256) {
    const int w = i / a.head_dim, c = i - w * a.head_dim;
    double s = 0.;
#pragma unroll 4
    for (int g = 0; g < GR; ++g) s += (double)red[w][g][c];
    partial[(size_t)blockIdx.x * 2 * a.head_dim + i] = (float)s;
  }
}

// heads per group and step: two where that leaves every workgroup a step (9216 rows
// of 48 heads of 128: 93 us with one, 86 with two, 126 with four, whose registers
// halve the waves), 1024 workgroups (four per CU; 2048: 89 us, 768: 99)
constexpr int kBwdHeads = 2, kBwdBlocks = 1024;
static int qk_bwd_hpg(int rows, int heads, int head_dim) {
  const int gr = head_groups(head_dim);
  return (long)rows * ((heads + kBwdHeads - 1) / kBwdHeads) / gr >= kBwdBlocks ? kBwdHeads : 1;
}
int qk_bwd_blocks(int rows, int heads, int head_dim) {
  const int gr = head_groups(head_dim), hpg = qk_bwd_hpg(rows, heads, head_dim);
  return (int)std::min<long>(kBwdBlocks, ((long)rows * ((heads + hpg - 1) / hpg) + gr - 1) / gr);
}

extern "C" int t2i_test_head_norm_heads(int rows, int heads, int head_dim, int backward) {
  if (rows < 1 || heads < 1 || head_dim < 8 || head_dim > 256 || head_dim % 8) return 0;
  return backward ? qk_bwd_hpg(rows, heads, head_dim) : qk_fwd_hpg(rows, heads, head_dim);
}

template <typename T, int G, bool HALVES>
static void qk_bwd_launch(const QkNorm& a, float* partial, hipStream_t st) {
  const int H = a.heads_q + a.heads_k, hpg = qk_bwd_hpg(a.rows, H, a.head_dim), upr = (H + hpg - 1) / hpg;
  const dim3 grid((unsigned)qk_bwd_blocks(a.rows, H, a.head_dim));
  if (hpg > 1)
    hipLaunchKernelGGL((qk_norm_rope_bwd_kernel<T, G, HALVES, kBwdHeads>), grid, dim3(256), 0, st, a, upr, partial);
  else
    hipLaunchKernelGGL((qk_norm_rope_bwd_kernel<T, G, HALVES, 1>), grid, dim3(256), 0, st, a, upr, partial);
}

// (halves: head_dim % 16 == 0, so neither one lane nor nine)
#define T2I_QK(FN, ...)                                                             \
  switch (head_lanes(a.head_dim)) {                                                 \
    case 1: if constexpr (!HALVES) FN<T, 1, HALVES>(__VA_ARGS__); break;            \
    case 2: FN<T, 2, HALVES>(__VA_ARGS__); break;                                   \
    case 4: FN<T, 4, HALVES>(__VA_ARGS__); break;                                   \
    case 8: FN<T, 8, HALVES>(__VA_ARGS__); break;                                   \
    case 9: if constexpr (!HALVES) FN<T, 9, HALVES>(__VA_ARGS__); break;            \
    case 16: FN<T, 16, HALVES>(__VA_ARGS__); break;                                 \
    default: FN<T, 32, HALVES>(__VA_ARGS__); break;                                 \
  }
template <typename T, bool HALVES>
static void qk_any(const QkNorm& a, hipStream_t st) { T2I_QK(qk_launch, a, st) }
template <typename T, bool HALVES>
static void qk_bwd_any(const QkNorm& a, float* partial, hipStream_t st) {
  T2I_QK(qk_bwd_launch, a, partial, st)
}
#undef T2I_QK

hipError_t launch_qk_norm_rope(bool is_bf16, const QkNorm& a, hipStream_t st) {
  if (is_bf16) a.halves ? qk_any<bf16, true>(a, st) : qk_any<bf16, false>(a, st);
  else a.halves ? qk_any<float, true>(a, st) : qk_any<float, false>(a, st);
  return hipGetLastError();
}

hipError_t launch_qk_norm_rope_bwd(bool is_bf16, const QkNorm& a, float* partial, hipStream_t st) {
  if (is_bf16) a.halves ? qk_bwd_any<bf16, true>(a, partial, st) : qk_bwd_any<bf16, false>(a, partial, st);
  else a.halves ? qk_bwd_any<float, true>(a, partial, st) : qk_bwd_any<float, false>(a, partial, st);
  return hipGetLastError();
}

// Column sums of n rows of fp32 partials (row stride ld) in fp64: 16 columns
// per workgroup of 1024, each by 64 threads that take every 64th row (so that a
// sum's reads are all under way at once), joined in a fixed order.
__device__ __forceinline__ double column_sum(const float* p, int n, size_t ld, int c, bool in) {
  __shared__ double red[64][16];
  const int s = threadIdx.x / 16, l = threadIdx.x % 16;
  double v = 0.;
  if (in) {
#pragma unroll 4
    for (int i = s; i < n; i += 64) v += (double)p[(size_t)i * ld + c];
  }
  red[s][l] = v;
  __syncthreads();
  if (s < 4) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += red[s + 4 * i][l];
  }
  __syncthreads();
  if (s < 4) red[s][l] = v;
  __syncthreads();
  return (red[0][l] + red[1][l]) + (red[2][l] + red[3][l]);
}

template <typename T>
__global__ __launch_bounds__(1024) void qk_weight_grad_kernel(const float* __restrict__ partial,
                                                             int blocks, int d, T* __restrict__ dwq,
                                                             T* __restrict__ dwk) {
  const int c = blockIdx.x * 16 + threadIdx.x % 16;
  const double v = column_sum(partial, blocks, (size_t)2 * d, c, c < 2 * d);
  if (threadIdx.x < 16 && c < 2 * d) {
    T* o = c < d ? dwq : dwk;
    if (o) o[c < d ? c : c - d] = from_f32<T>((float)v);
  }
}

hipError_t launch_qk_weight_grad(bool is_bf16, int blocks, int head_dim, const float* partial,
                                 void* dwq, void* dwk, hipStream_t st) {
  const dim3 grid((unsigned)((2 * head_dim + 15) / 16));
  if (is_bf16)
    hipLaunchKernelGGL((qk_weight_grad_kernel<bf16>), grid, dim3(1024), 0, st, partial, blocks, head_dim,
                       (bf16*)dwq, (bf16*)dwk);
  else
    hipLaunchKernelGGL((qk_weight_grad_kernel<float>), grid, dim3(1024), 0, st, partial, blocks,
                       head_dim, (float*)dwq, (float*)dwk);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Gated feed-forward, elementwise gradients: with a = act(g),
//   dg = dh u act'(g),  du = dh a,
// rounded once to the operands' type for the products that follow (the matrix cores
// take nothing wider); the bias gradients' column sums take the unrounded values: up to
// 8 of a thread's rows in fp32, 8 threads in fp64, a workgroup's sum in fp32, these in fp64.
// 4096 x 10240 120 us (4.9 TB/s of a copy's 5.1), with the column sums 121.

struct ActGrad { float a, d; };   // act(g), act'(g)
__device__ __forceinline__ ActGrad act_grad(int act, float g) {
  if (act == EPI_GELU) {
    // g sigmoid(2 z), z = sqrt(2/pi) (g + 0.044715 g^3)
    constexpr float c0 = 2.0f * 0.7978845608028654f, c1 = -c0 * 1.4426950408889634f;
    const float g2 = g * g;
    const float s = __builtin_amdgcn_rcpf(
        1.f + __builtin_amdgcn_exp2f(g * fmaf(c1 * 0.044715f, g2, c1)));
    const float p = s * (1.f - s);
    // (p is 0 before g2 overflows)
    const float d = p == 0.f ? 0.f : p * g * c0 * fmaf(3.f * 0.044715f, g2, 1.f);
    return {g * s, s + d};
  }
  const float s = __builtin_amdgcn_rcpf(1.f + __expf(-g)), a = g * s;
  return {a, fmaf(a, 1.f - s, s)};
}

// rows per workgroup: 64, or down to the 8 that its threads take at a time while
// there are fewer than two workgroups of 256 columns (bf16's) per CU (333 rows of
// 1544: 13.9 -> 5.5 us)
static int gate_rows(int M, int F) {
  int rows = 64;
  while (rows > 8 && (long)((M + rows - 1) / rows) * ((gated_cols(F) + 255) / 256) < 512) rows /= 2;
  return rows;
}
int gate_row_blocks(int M, int F) {
  const int rows = gate_rows(M, F);
  return (M + rows - 1) / rows;
}

extern "C" int t2i_test_gate_rows(int M, int F) { return M < 1 || F < 1 ? 0 : gate_rows(M, F); }

// V columns per thread (bf16: 8, whose rows are whole 16-byte pieces; fp32, whose rows may
// lie anywhere: 1): 32 threads side by side, 8 rows at a time
template <typename T, int V>
__global__ __launch_bounds__(256) void gate_grad_kernel(int act, int M, int F, int Fp, int rows,
                                                        const float* __restrict__ pre, int ldp,
                                                        const T* __restrict__ dout, int ldd,
                                                        T* __restrict__ dgu, float* __restrict__ partial) {
  __shared__ float red[2][8][32 * V];
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
  const int f = (blockIdx.y * 32 + tx) * V;
  const int r0 = blockIdx.x * rows;
  float sg[V], su[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sg[j] = su[j] = 0.f;
  if (f < Fp)
    for (int r = r0 + ty; r < min(r0 + rows, M); r += 8) {
      float g[V], u[V], dh[V];
      if (f < F) {
        const float* p = pre + (size_t)r * ldp + f;
        if constexpr (V == 8) {
          load8(p, g);
          load8(p + F, u);
          load8(dout + (size_t)r * ldd + f, dh);
        } else {
          g[0] = p[0];
          u[0] = p[F];
          dh[0] = to_f32(dout[(size_t)r * ldd + f]);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const ActGrad ag = act_grad(act, g[j]);
          g[j] = dh[j] * u[j] * ag.d;
          u[j] = dh[j] * ag.a;
          sg[j] += g[j];
          su[j] += u[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) g[j] = u[j] = 0.f;
      }
      T* o = dgu + (size_t)r * 2 * Fp + f;
      if constexpr (V == 8) {
        store8(o, g);
        store8(o + Fp, u);
      } else {
        o[0] = from_f32<T>(g[0]);
        o[Fp] = from_f32<T>(u[0]);
      }
    }
  if (!partial) return;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    red[0][ty][tx * V + j] = sg[j];
    red[1][ty][tx * V + j] = su[j];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * 32 * V; i += 256) {
    const int w = i / (32 * V), c = i - w * 32 * V, col = blockIdx.y * 32 * V + c;
    if (col >= Fp) continue;
    double s = 0.;
#pragma unroll
    for (int y = 0; y < 8; ++y) s += (double)red[w][y][c];
    partial[(size_t)blockIdx.x * 2 * Fp + w * Fp + col] = (float)s;
  }
}

hipError_t launch_gate_grad(bool is_bf16, int act, int M, int F, const float* pre, int ldp,
                            const void* dout, int ldd, void* dgu, float* partial, hipStream_t st) {
  const int Fp = gated_cols(F), per = is_bf16 ? 256 : 32, rows = gate_rows(M, F);
  const dim3 grid((unsigned)gate_row_blocks(M, F), (unsigned)((Fp + per - 1) / per));
  if (is_bf16)
    hipLaunchKernelGGL((gate_grad_kernel<bf16, 8>), grid, dim3(256), 0, st, act, M, F, Fp, rows,
                       pre, ldp, (const bf16*)dout, ldd, (bf16*)dgu, partial);
  else
    hipLaunchKernelGGL((gate_grad_kernel<float, 1>), grid, dim3(256), 0, st, act, M, F, Fp, rows,
                       pre, ldp, (const float*)dout, ldd, (float*)dgu, partial);
  return hipGetLastError();
}

template <typename T>
__global__ __launch_bounds__(1024) void gate_bias_grad_kernel(const float* __restrict__ partial, int blocks,
                                                             int F, int Fp, T* __restrict__ dbg,
                                                             T* __restrict__ dbu) {
  const int c = blockIdx.x * 16 + threadIdx.x % 16, w = blockIdx.y;
  const double v = column_sum(partial + (size_t)w * Fp, blocks, (size_t)2 * Fp, c, c < F);
  if (threadIdx.x < 16 && c < F) (w ? dbu : dbg)[c] = from_f32<T>((float)v);
}

hipError_t launch_gate_bias_grad(bool is_bf16, int M, int F, const float* partial, void* dbg,
                                 void* dbu, hipStream_t st) {
  const dim3 grid((unsigned)((F + 15) / 16), 2);
  if (is_bf16)
    hipLaunchKernelGGL((gate_bias_grad_kernel<bf16>), grid, dim3(1024), 0, st, partial,
                       gate_row_blocks(M, F), F, gated_cols(F), (bf16*)dbg, (bf16*)dbu);
  else
    hipLaunchKernelGGL((gate_bias_grad_kernel<float>), grid, dim3(1024), 0, st, partial,
                       gate_row_blocks(M, F), F, gated_cols(F), (float*)dbg, (float*)dbu);
  return hipGetLastError();
}

}  // namespace t2i
