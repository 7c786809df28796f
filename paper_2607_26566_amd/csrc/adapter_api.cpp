// Entry points of the low-rank adapters beside a shared linear layer: argument checks,
// then the launches.
#include <algorithm>
#include <cstring>

#include "block_ops.h"

using namespace t2i;

namespace {

bool bad_dtype(int32_t d) { return d != T2I_F32 && d != T2I_BF16; }
bool off(const void* p, size_t n) { return (uintptr_t)p % n != 0; }
size_t bytes_of(int32_t d) { return d == T2I_BF16 ? 2 : 4; }
// (a launch holds fewer than 2^32 threads)
bool too_large(int64_t M, int64_t N) { return ((M + 63) / 64) * ((N + 63) / 64) >= 1 << 23; }
bool far_rows(int32_t ld, size_t elem) { return (int64_t)ld * (int64_t)elem * 256 > 0x7fffffff; }
size_t whole(size_t n) { return (n + 255) / 256 * 256; }
int32_t whole8(int32_t n) { return (n + 7) / 8 * 8; }
t2i_status done(hipError_t e) {
  return e == hipSuccess ? T2I_OK : ops_fail(T2I_ERR_DEVICE, hipGetErrorString(e));
}

bool bad_sizes(int32_t M, int32_t N, int32_t K, int32_t n, int32_t rank) {
  return M < 1 || N < 1 || K < 1 || n < 1 || rank < 1 || M > 1 << 24 || N > 1 << 28 || K > 1 << 28 || n > 32767 ||
         rank > 128 || too_large(M, N) || (int64_t)n * std::max(N, K) * whole8(rank) >= 1LL << 32;
}

// the gradients' workspace
struct Room {
  int per;                               // rows of a slice
  size_t u, at, bt, order, span, table, part_a, part_b, dx, all;   // offsets
};
Room room_of(bool bf, int32_t M, int32_t N, int32_t K, int32_t n, int32_t rank) {
  Room r;
  const size_t e = bf ? 2 : 4;
  r.per = adapter_slice_rows(bf, M, N, K, n, rank);
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t here = o;
    o += whole(bytes);
    return here;
  };
  const size_t ranks = (rank + 3) / 4 * 4, places = adapter_places(M, r.per);
  r.u = take((size_t)M * adapter_cols(rank) * 4);
  r.at = take((size_t)n * K * whole8(rank) * e);
  r.bt = take(adapter_few_rows(M, N, rank) ? 0 : (size_t)n * rank * N * e);
  r.order = take((size_t)M * 4);
  r.span = take((size_t)n * 8);
  r.table = take((size_t)(M / r.per + n) * 16);
  r.part_a = take(places * ranks * whole8(K) * 4);
  r.part_b = take(places * ranks * whole8(N) * 4);
  r.dx = take(adapter_dx_floats(bf, M, N, K) * 4);
  r.all = o;
  return r;
}
// whether the slices of the sums of so many columns pass a launch
bool too_many_slices(bool bf, int64_t slices, int64_t da_columns, int64_t db_columns, int32_t rank) {
  const int64_t cols = bf ? 128 : 64, blocks = (da_columns + cols - 1) / cols + (db_columns + cols - 1) / cols;
  return blocks * slices * ((rank + 31) / 32) >= 1 << 24 || slices > 65535;
}

t2i_status check_operands(int32_t dtype, int32_t M, int32_t N, int32_t K, const void* x, int32_t ldx, const void* w,
                          int32_t ldw, int32_t n, int32_t rank, const void* a, const void* b, const float* scale,
                          const int32_t* index, const float* t, int32_t ldt) {
  if (bad_dtype(dtype)) return ops_fail(T2I_ERR_INVALID_ARG, "bad dtype");
  if (bad_sizes(M, N, K, n, rank)) return ops_fail(T2I_ERR_SHAPE, "bad shape");
  if (!x || !w || !a || !b || !t) return ops_fail(T2I_ERR_INVALID_ARG, "NULL operand");
  if (ldx < K || ldw < K) return ops_fail(T2I_ERR_SHAPE, "leading dimension < K");
  if (ldt < adapter_cols(rank) || ldt % 8 || ldt > 1 << 20)
    return ops_fail(T2I_ERR_SHAPE, "ldt must be a multiple of 8, at least rank rounded up to 32");
  const bool bf = dtype == T2I_BF16;
  if (bf && (N % 8 || K % 8 || ldx % 8 || ldw % 8)) return ops_fail(T2I_ERR_SHAPE, "bf16 needs N, K, ldx and ldw % 8 == 0");
  if (far_rows(ldx, bytes_of(dtype)) || far_rows(ldw, bytes_of(dtype)))
    return ops_fail(T2I_ERR_SHAPE, "rows more than 8 MiB apart");
  const size_t al = bf ? 16 : 4;
  if (off(x, al) || off(w, al) || off(a, al) || off(b, bf ? 2 : 4) || off(scale, 4) || off(index, 4) || off(t, 16))
    return ops_fail(T2I_ERR_INVALID_ARG, "pointers need 16-byte (bf16; t) or 4-byte (fp32) alignment");
  return T2I_OK;
}

}  // namespace

extern "C" {

t2i_status t2i_op_adapter_linear(int32_t dtype, int32_t epilogue, int32_t M, int32_t N, int32_t K, const void* x,
                                 int32_t ldx, const void* w, int32_t ldw, const void* bias, int32_t n, int32_t rank,
                                 const void* a, const void* b, const float* scale, const int32_t* index, float* t,
                                 int32_t ldt, void* out, int32_t ldo, float* resid, int32_t ldr, void* resid_copy,
                                 const float* gate, void* stream) {
  if (epilogue < T2I_EPI_STORE || epilogue > T2I_EPI_RESID_GATED)
    return ops_fail(T2I_ERR_INVALID_ARG, "bad epilogue");
  const t2i_status s = check_operands(dtype, M, N, K, x, ldx, w, ldw, n, rank, a, b, scale, index, t, ldt);
  if (s != T2I_OK) return s;
  const bool res = epilogue >= T2I_EPI_RESID;
  if (res && (!resid || ldr < N)) return ops_fail(T2I_ERR_INVALID_ARG, "bad residual");
  if (!res && (!out || ldo < N)) return ops_fail(T2I_ERR_INVALID_ARG, "bad out");
  if (epilogue == T2I_EPI_RESID_GATED && !gate) return ops_fail(T2I_ERR_INVALID_ARG, "NULL gate");
  const size_t e = bytes_of(dtype);
  if (off(bias, e) || (!res && off(out, e)) ||
      (res && (off(resid, 4) || off(resid_copy, 2) || (epilogue == T2I_EPI_RESID_GATED && off(gate, 4)))))
    return ops_fail(T2I_ERR_INVALID_ARG, "bias and outputs need the alignment of their type");
  hipStream_t st = (hipStream_t)stream;
  AdapterDown d;
  std::memset(&d, 0, sizeof(d));
  d.M = M;
  d.K = K;
  d.n = n;
  d.rank = rank;
  d.x = x;
  d.ldx = ldx;
  d.a = a;
  d.scale = scale;
  d.index = index;
  d.t = t;
  d.ldt = ldt;
  const AdapterUp up{index, n, rank, rank, b, t, ldt};
  const LinearEpi p{epilogue, bias, out, ldo, resid, ldr, (bf16*)resid_copy, gate};
  const bool bf = dtype == T2I_BF16;
  hipError_t err = launch_adapter_down(bf, d, st);
  if (err == hipSuccess) err = launch_adapter_linear(bf, x, ldx, w, ldw, M, N, K, up, p, st);
  return done(err);
}

size_t t2i_op_adapter_linear_backward_ws_bytes(int32_t dtype, int32_t M, int32_t N, int32_t K, int32_t n,
                                               int32_t rank) {
  if (bad_dtype(dtype) || bad_sizes(M, N, K, n, rank) || too_large(M, K)) return 0;
  return room_of(dtype == T2I_BF16, M, N, K, n, rank).all;
}

t2i_status t2i_op_adapter_linear_backward(int32_t dtype, int32_t M, int32_t N, int32_t K, const void* dy, int32_t lddy,
                                          const void* x, int32_t ldx, const void* w, int32_t ldw, int32_t n,
                                          int32_t rank, const void* a, const void* b, const float* scale,
                                          const int32_t* index, const float* t, int32_t ldt, void* dx, int32_t lddx,
                                          void* da, void* db, void* ws, size_t ws_bytes, void* stream) {
  const t2i_status s = check_operands(dtype, M, N, K, x, ldx, w, ldw, n, rank, a, b, scale, index, t, ldt);
  if (s != T2I_OK) return s;
  const bool bf = dtype == T2I_BF16;
  if (too_large(M, K)) return ops_fail(T2I_ERR_SHAPE, "bad shape");
  if (!dy || !ws) return ops_fail(T2I_ERR_INVALID_ARG, "NULL operand");
  if (!dx && !da && !db) return ops_fail(T2I_ERR_INVALID_ARG, "no gradient asked for");
  if (lddy < N || (dx && lddx < K)) return ops_fail(T2I_ERR_SHAPE, "bad leading dimension");
  if (bf && (lddy % 8 || (dx && lddx % 8))) return ops_fail(T2I_ERR_SHAPE, "bf16 needs strides % 8 == 0");
  if (far_rows(lddy, bytes_of(dtype))) return ops_fail(T2I_ERR_SHAPE, "rows more than 8 MiB apart");
  const size_t al = bf ? 16 : 4;
  if (off(dy, al) || off(dx, al) || off(da, bytes_of(dtype)) || off(db, bytes_of(dtype)) || off(ws, 256))
    return ops_fail(T2I_ERR_INVALID_ARG, "pointers need 16-byte (bf16) or 4-byte (fp32) alignment, ws 256-byte");
  const Room r = room_of(bf, M, N, K, n, rank);
  if (too_many_slices(bf, adapter_slices(index != nullptr, M, n, r.per), da ? K : 0, db ? N : 0, rank))
    return ops_fail(T2I_ERR_SHAPE, "too many adapters for a launch");
  if (ws_bytes < r.all) return ops_fail(T2I_ERR_WORKSPACE, "workspace too small");
  hipStream_t st = (hipStream_t)stream;
  char* const at = (char*)ws;
  const int32_t ldu = adapter_cols(rank);
  const bool sums = da || db;
  AdapterPrepare pre;
  std::memset(&pre, 0, sizeof(pre));
  pre.index = index;
  pre.M = M;
  pre.n = n;
  pre.per = r.per;
  pre.groups = sums && index ? n : 0;
  pre.order = (int32_t*)(at + r.order);
  pre.span = (int2*)(at + r.span);
  pre.slices = (int4*)(at + r.table);
  const bool need_u = dx || da, few = adapter_few_rows(M, N, rank);
  pre.rank = rank;
  if (need_u && few) {
    pre.dy = dy;
    pre.lddy = lddy;
    pre.b = b;
    pre.N = N;
    pre.scale = scale;
    pre.u = (float*)(at + r.u);
  } else if (need_u) {
    pre.turn[0] = AdapterTurn{b, at + r.bt, N, rank, N, 0};
  }
  if (dx) pre.turn[1] = AdapterTurn{a, at + r.at, rank, K, whole8(rank), 0};
  hipError_t err = launch_adapter_prepare(bf, pre, st);
  if (err == hipSuccess && need_u && !few) {   // u = s dy B
    AdapterDown d;
    std::memset(&d, 0, sizeof(d));
    d.M = M;
    d.K = N;
    d.n = n;
    d.rank = rank;
    d.x = dy;
    d.ldx = lddy;
    d.a = at + r.bt;
    d.scale = scale;
    d.index = index;
    d.t = (float*)(at + r.u);
    d.ldt = ldu;
    err = launch_adapter_down(bf, d, st);
  }
  if (err == hipSuccess && dx) {
    const AdapterUp up{index, n, whole8(rank), whole8(rank), at + r.at, (const float*)(at + r.u), ldu};
    err = launch_adapter_dx(bf, dy, lddy, w, ldw, M, N, K, up, dx, lddx, (float*)(at + r.dx), st);
  }
  if (err == hipSuccess && sums) {
    AdapterOuter o;
    std::memset(&o, 0, sizeof(o));
    o.side[0] = AdapterSide{x, (const float*)(at + r.u), ldx, ldu, K, (float*)(at + r.part_a), whole8(K), nullptr};
    o.side[1] = AdapterSide{dy, t, lddy, ldt, N, (float*)(at + r.part_b), whole8(N), nullptr};
    o.M = M;
    o.per = r.per;
    o.rank = rank;
    o.ranks = (rank + 3) / 4 * 4;
    if (index) {
      o.order = (const int32_t*)(at + r.order);
      o.span = (const int2*)(at + r.span);
      o.slices = (const int4*)(at + r.table);
    }
    // (without an index only adapter 0 has rows)
    err = launch_adapter_outer(bf, o, n, da, db, st);
  }
  return done(err);
}

}  // extern "C"
