// C entry points of the operators around the fused nets: layer norm, dense
// layers of any width, and the vocabulary losses.  Argument checks,
// workspace layouts and launch sequences; host code only.
#include <cmath>
#include <limits>

#include "ffmlp.h"
#include "gemm.h"
#include "head.h"
#include "host.h"

using namespace ffmlp;

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 30, kMaxDim = MLP_MAX_DIM, kMaxHeadRows = (int64_t)1 << 24;

bool valid_type(int t) { return t == MLP_BF16 || t == MLP_FP32; }
size_t type_size(int t) { return t == MLP_FP32 ? 4 : 2; }

// Row stride of a matrix of `cols` columns.
bool valid_ld(int64_t ld, int64_t cols) { return ld >= cols && ld <= kMaxDim; }

SideArgs side(const void* p, int64_t ld, int64_t rows, int64_t cols) {
  return SideArgs{static_cast<const uint16_t*>(p), ld, rows, cols};
}

// ---- workspaces (byte offsets, 256-byte regions)

// Row stride of a buffer of the products' own: rows that start 128 bytes apart
// modulo 256 spread a tile's rows over the memory channels, which a stride with
// more factors of two does not.  8192 x 2048 over 65536 (P times W^T) with a
// stride of 65536: 1825 us, with 65600: 1785; over 65024: 2053 against 1809;
// 8192 x 4096 over 4096: 219 against 206.  Short rows only keep whole 16 bytes.
int64_t own_stride(int64_t cols) {
  return cols < 1024 ? (int64_t)round_up((size_t)cols, 8) : (cols + 63) / 128 * 128 + 64;
}

struct DenseWs {
  size_t dz, db, partial, total;
  int parts;
  int64_t ldz;
};
DenseWs dense_ws(int64_t M, int64_t K, int64_t N, int mode) {
  DenseWs w{};
  size_t o = 0;
  if (mode == MLP_MODE_TRAIN) {
    w.ldz = own_stride(N);
    w.dz = o; o = round_up(o + (size_t)M * w.ldz * 2, 256);
    w.parts = delta_parts(M, (int)N);
    w.db = o; o = round_up(o + (size_t)w.parts * N * 4, 256);
  }
  size_t p = M > 0 ? gemm_plan(GEMM_XW, M, N, K).partial_bytes : 0;
  if (mode == MLP_MODE_TRAIN) {
    const size_t dx = M > 0 ? gemm_plan(GEMM_DX, M, K, N).partial_bytes : 0, dw = gemm_plan(GEMM_DW, K, N, M).partial_bytes;
    p = p > dx ? p : dx;
    p = p > dw ? p : dw;
  }
  w.partial = o; o = round_up(o + p, 256);
  w.total = o;
  return w;
}

struct HeadWs {
  HeadPlan plan;
  size_t lse, row_loss, alpha, ok, part, pick, index, q, start, P, ref, acc, partial, total;
  int keys;
  int64_t ldp;
};
HeadWs head_ws(int64_t M, int64_t D, int64_t V, int top, int mode, bool teacher) {
  HeadWs w{};
  w.plan = head_plan(M, D, V);
  w.keys = (int)(round_up((size_t)V, 256) / kHeadKey) + 1;
  size_t o = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = o;
    o = round_up(o + bytes, 256);
    return at;
  };
  w.lse = take((size_t)M * 8);
  w.row_loss = take((size_t)M * 4);
  w.alpha = take(4);
  w.part = take((size_t)w.plan.parts * M * 8);
  w.pick = take((size_t)M * top * 4);
  if (teacher) {
    w.ok = take((size_t)M * 4);
    w.index = take((size_t)M * top * 4);
    w.q = take((size_t)M * top * 4);
    w.start = take((size_t)M * w.keys * 2);
  }
  if (mode == MLP_MODE_TRAIN) {
    w.ldp = own_stride(w.plan.piece);
    w.P = take((size_t)M * w.ldp * 2);
    w.ref = take((size_t)M * w.plan.refs * 4);
    w.acc = take(w.plan.pieces > 1 ? (size_t)M * D * 4 : 0);
    size_t p = 0;
    const int64_t last = V - (int64_t)(w.plan.pieces - 1) * w.plan.piece;
    for (const int64_t n : {(int64_t)w.plan.piece, last}) {
      const size_t dh = M > 0 ? gemm_plan(GEMM_DX, M, D, n).partial_bytes : 0, dw = gemm_plan(GEMM_DW, D, n, M).partial_bytes;
      p = p > dh ? p : dh;
      p = p > dw ? p : dw;
    }
    w.partial = take(p);
  }
  w.total = o;
  return w;
}

int check_head(const void* H, int64_t ldh, const void* W, int64_t ldw, const void* dH, int dh_type, int64_t lddh, const void* dW,
               int dw_type, int64_t lddw, const float* loss, const float* row_loss, int64_t M, int64_t D, int64_t V, const void* ws) {
  if (M < 0 || M > kMaxHeadRows) return fail(MLP_ERR_INVALID_ARG, "M = %lld outside [0, 2^24]", (long long)M);
  if (D < 1 || D > kMaxDim || V < 1 || V > kMaxDim)
    return fail(MLP_ERR_INVALID_ARG, "dim %lld or vocabulary %lld outside [1, %d]", (long long)D, (long long)V, (int)MLP_MAX_DIM);
  if (!ws || !W || (M > 0 && !H)) return fail(MLP_ERR_INVALID_ARG, "null H, W or workspace");
  if ((M > 0 && !valid_ld(ldh, D)) || !valid_ld(ldw, V)) return fail(MLP_ERR_INVALID_ARG, "row stride of H or W outside [columns, %d]", (int)MLP_MAX_DIM);
  if (!aligned(H, 2) || !aligned(W, 2) || !aligned(ws, 256) || !aligned(loss, 4) || !aligned(row_loss, 4))
    return fail(MLP_ERR_INVALID_ARG, "misaligned pointer (ws: 256 bytes; others: their elements)");
  if (!dH != !dW) return fail(MLP_ERR_INVALID_ARG, "dH and dW go together");
  if (dW) {
    if (!valid_type(dh_type) || !valid_type(dw_type)) return fail(MLP_ERR_UNSUPPORTED, "unknown type of dH or dW");
    if ((M > 0 && !valid_ld(lddh, D)) || !valid_ld(lddw, V)) return fail(MLP_ERR_INVALID_ARG, "row stride of dH or dW outside [columns, %d]", (int)MLP_MAX_DIM);
    if (!aligned(dH, type_size(dh_type)) || !aligned(dW, type_size(dw_type))) return fail(MLP_ERR_INVALID_ARG, "misaligned dH or dW");
  }
  return MLP_OK;
}

// The losses of the rows and, with dW, the gradients piece by piece.  `a` and
// `r` come with what tells cross entropy and distillation apart.
int run_head(bool distill, HeadArgs a, RowLossArgs r, const HeadWs& w, uint8_t* ws, void* dH, int dh_type, int64_t lddh, void* dW,
             int dw_type, int64_t lddw, hipStream_t s) {
  const int64_t M = a.M, D = a.D;
  const int V = a.V;
  const SideArgs all = a.w;
  const auto launch = distill ? launch_head_distill : launch_head_ce;
  a.pick = reinterpret_cast<float*>(ws + w.pick);
  a.partial = reinterpret_cast<f32x2*>(ws + w.part);
  a.lse = reinterpret_cast<const f32x2*>(ws + w.lse);
  a.mt = w.plan.mt;
  a.nt = w.plan.nt;
  a.runs = w.plan.runs;
  a.per_run = w.plan.per_run;
  uint16_t* P = reinterpret_cast<uint16_t*>(ws + w.P);
  if (dW) {
    a.P = P;
    a.ldp = w.ldp;
    a.keep = w.plan.piece;
    a.ref = reinterpret_cast<float*>(ws + w.ref);
    // Columns of a wave of the scaling pass, each of which merges its row's sums
    // anew: 4096, halved down to 1024 while fewer than 2048 waves come of it.  Steps
    // of hidden size 64 in us with 1024, 2048, 4096 and 8192: 16 rows over 131072
    // words 59.5, 60.4, 61.9 and 65.3; 64 over 65536 62.5, 59.6, 60.8 and 64.3; 256
    // over 50000 72.0, 66.2, 64.9 and 66.6; 2048 over 131072 726, 700, 707 and 707;
    // 65536 over 4096 723, 714, 689 and 689; hidden size 200, 513 over 10007 57.7,
    // 57.6, 59.0 and 63.1.
    a.chunk = 4096;
    while (a.chunk > 1024 && M * ((w.plan.piece + a.chunk - 1) / a.chunk) < 2048) a.chunk /= 2;
  }
  r.partial = a.partial;
  r.parts = w.plan.parts;
  r.pick = a.pick;
  r.M = M;
  r.V = V;
  r.lse = reinterpret_cast<f32x2*>(ws + w.lse);
  r.scale2 = a.scale2;
  if (!r.row_loss) r.row_loss = reinterpret_cast<float*>(ws + w.row_loss);
  r.alpha = reinterpret_cast<float*>(ws + w.alpha);
  hipError_t e;
  if (M > 0) {
    e = launch(w.plan.rows ? HEAD_ROWS : HEAD_LSE, w.plan.large, a, r, s);
    if (e != hipSuccess) return hip_fail(e, "log-sum-exp kernel launch");
    if (!w.plan.rows) {
      e = dW ? launch(HEAD_SCALE, w.plan.large, a, r, s) : launch_row_loss(r, s);
      if (e != hipSuccess) return hip_fail(e, "row loss kernel launch");
    }
  }
  e = launch_mean_loss(r, s);
  if (e != hipSuccess) return hip_fail(e, "mean loss kernel launch");
  if (!dW) return MLP_OK;
  float* partial = reinterpret_cast<float*>(ws + w.partial);
  float* acc = reinterpret_cast<float*>(ws + w.acc);
  const int n_pieces = w.plan.pieces;
  for (int k = 0; k < n_pieces; ++k) {
    const int v0 = k * w.plan.piece, n = V - v0 < w.plan.piece ? V - v0 : w.plan.piece;
    if (M > 0) {
      if (k > 0) {
        a.w = side(all.p + v0, all.ld, D, n);
        a.V = n;
        a.col0 = v0;
        a.nt = (int)((n + (w.plan.large ? 255 : 127)) / (w.plan.large ? 256 : 128));
        e = launch(HEAD_PROB, w.plan.large, a, r, s);
        if (e != hipSuccess) return hip_fail(e, "logit gradient kernel launch");
      }
      // dH: pieces before the last add up in fp32
      GemmArgs g{};
      g.m = side(P, w.ldp, M, n);
      g.n = side(all.p + v0, all.ld, D, n);
      g.M = M;
      g.N = (int)D;
      g.K = n;
      if (k > 0) {
        g.out.add = acc;
        g.out.ldadd = D;
      }
      if (k + 1 < n_pieces) {
        g.out.C = acc;
        g.out.ldc = D;
        g.out.c_fp32 = 1;
      } else {
        g.out.alpha = r.alpha;
        g.out.C = dH;
        g.out.ldc = lddh;
        g.out.c_fp32 = dh_type == MLP_FP32;
      }
      e = launch_gemm(GEMM_DX, g, partial, s);
      if (e != hipSuccess) return hip_fail(e, "dH product launch");
    }
    GemmArgs g{};
    g.m = side(a.h.p, a.h.ld, M, D);
    g.n = side(P, w.ldp, M, (int64_t)round_up((size_t)n, 8));
    g.M = D;
    g.N = n;
    g.K = M;
    g.out.alpha = r.alpha;
    g.out.C = static_cast<uint8_t*>(dW) + (size_t)v0 * type_size(dw_type);
    g.out.ldc = lddw;
    g.out.c_fp32 = dw_type == MLP_FP32;
    e = launch_gemm(GEMM_DW, g, partial, s);
    if (e != hipSuccess) return hip_fail(e, "dW product launch");
  }
  return MLP_OK;
}

// What an entry point returns for a C++ exception (host memory ran out): none
// leaves the library.
int entry_failed() noexcept {
  try {
    return fail(MLP_ERR_HIP, "out of host memory");
  } catch (...) {
    return MLP_ERR_HIP;
  }
}

}  // namespace

extern "C" {

// ------------------------------------------------------------- layer norm --

size_t mlp_layer_norm_workspace_bytes(int64_t M, int64_t N, int mode) {
  if (M < 0 || M > kMaxRows || N < 1 || N > kMaxDim || mode != MLP_MODE_TRAIN) return 0;
  return round_up((size_t)norm_parts(M, (int)N) * 2 * N * 4, 256);
}

int mlp_layer_norm_forward(const void* X, int x_type, int64_t ldx, const float* gamma, const float* beta, void* Y, int y_type,
                           int64_t ldy, float* stats, int64_t M, int64_t N, float eps, void* stream) try {
  clear_error();
  if (M < 0 || M > kMaxRows) return fail(MLP_ERR_INVALID_ARG, "M = %lld outside [0, 2^30]", (long long)M);
  if (N < 1 || N > kMaxDim) return fail(MLP_ERR_INVALID_ARG, "N = %lld outside [1, %d]", (long long)N, (int)MLP_MAX_DIM);
  if (!valid_type(x_type) || !valid_type(y_type)) return fail(MLP_ERR_UNSUPPORTED, "unknown type of X or Y");
  if (!(eps > 0.f) || !std::isfinite(eps)) return fail(MLP_ERR_INVALID_ARG, "eps must be positive and finite");
  if (M == 0) return MLP_OK;
  if (!X || !Y) return fail(MLP_ERR_INVALID_ARG, "null X or Y");
  if (!valid_ld(ldx, N) || !valid_ld(ldy, N)) return fail(MLP_ERR_INVALID_ARG, "row stride outside [N, %d]", (int)MLP_MAX_DIM);
  if (!aligned(X, type_size(x_type)) || !aligned(Y, type_size(y_type)) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(stats, 8))
    return fail(MLP_ERR_INVALID_ARG, "misaligned pointer (stats: 8 bytes; others: their elements)");
  NormArgs a{};
  a.X = X;
  a.x_fp32 = x_type == MLP_FP32;
  a.ldx = ldx;
  a.gamma = gamma;
  a.beta = beta;
  a.Y = Y;
  a.y_fp32 = y_type == MLP_FP32;
  a.ldy = ldy;
  a.stats = stats;
  a.eps = eps;
  a.M = M;
  a.N = (int)N;
  const hipError_t e = launch_norm_forward(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLP_OK : hip_fail(e, "layer norm kernel launch");
} catch (...) {
  return entry_failed();
}

int mlp_layer_norm_backward(const void* X, int x_type, int64_t ldx, const float* gamma, const float* stats, const void* dY, int dy_type,
                            int64_t lddy, void* dX, int dx_type, int64_t lddx, float* dgamma, float* dbeta, int64_t M, int64_t N,
                            void* ws, void* stream) try {
  clear_error();
  if (M < 0 || M > kMaxRows) return fail(MLP_ERR_INVALID_ARG, "M = %lld outside [0, 2^30]", (long long)M);
  if (N < 1 || N > kMaxDim) return fail(MLP_ERR_INVALID_ARG, "N = %lld outside [1, %d]", (long long)N, (int)MLP_MAX_DIM);
  if (!valid_type(x_type) || !valid_type(dy_type) || !valid_type(dx_type)) return fail(MLP_ERR_UNSUPPORTED, "unknown type of X, dY or dX");
  if (!dgamma || !dbeta || !ws) return fail(MLP_ERR_INVALID_ARG, "null dgamma, dbeta or workspace");
  if (M > 0 && (!X || !dY || !dX || !stats)) return fail(MLP_ERR_INVALID_ARG, "null X, dY, dX or stats");
  if (M > 0 && (!valid_ld(ldx, N) || !valid_ld(lddy, N) || !valid_ld(lddx, N)))
    return fail(MLP_ERR_INVALID_ARG, "row stride outside [N, %d]", (int)MLP_MAX_DIM);
  if (!aligned(X, type_size(x_type)) || !aligned(dY, type_size(dy_type)) || !aligned(dX, type_size(dx_type)) || !aligned(gamma, 4) ||
      !aligned(stats, 8) || !aligned(dgamma, 4) || !aligned(dbeta, 4) || !aligned(ws, 256))
    return fail(MLP_ERR_INVALID_ARG, "misaligned pointer (ws: 256 bytes; stats: 8; others: their elements)");
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (M == 0) {
    e = launch_column_reduce(static_cast<float*>(ws), 0, N, dgamma, dbeta, s);
  } else {
    NormArgs a{};
    a.X = X;
    a.x_fp32 = x_type == MLP_FP32;
    a.ldx = ldx;
    a.gamma = gamma;
    a.stats = const_cast<float*>(stats);
    a.dY = dY;
    a.dy_fp32 = dy_type == MLP_FP32;
    a.lddy = lddy;
    a.dX = dX;
    a.dx_fp32 = dx_type == MLP_FP32;
    a.lddx = lddx;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.partial = static_cast<float*>(ws);
    a.M = M;
    a.N = (int)N;
    a.parts = norm_parts(M, (int)N);
    e = launch_norm_backward(a, s);
  }
  return e == hipSuccess ? MLP_OK : hip_fail(e, "layer norm backward launch");
} catch (...) {
  return entry_failed();
}

// ------------------------------------------------------------------ dense --

size_t mlp_dense_workspace_bytes(int64_t M, int64_t K, int64_t N, int mode) {
  if (M < 0 || M > kMaxRows || K < 1 || K > kMaxDim || N < 1 || N > kMaxDim) return 0;
  if (mode != MLP_MODE_INFER && mode != MLP_MODE_TRAIN) return 0;
  return dense_ws(M, K, N, mode).total;
}

int mlp_dense_forward(const uint16_t* X, int64_t ldx, const uint16_t* W, int64_t ldw, const float* bias, int activation, const void* R,
                      int64_t ldr, void* Y, int y_type, int64_t ldy, float* stash, int64_t M, int64_t K, int64_t N, void* ws,
                      void* stream) try {
  clear_error();
  if (M < 0 || M > kMaxRows) return fail(MLP_ERR_INVALID_ARG, "M = %lld outside [0, 2^30]", (long long)M);
  if (K < 1 || K > kMaxDim || N < 1 || N > kMaxDim)
    return fail(MLP_ERR_INVALID_ARG, "K = %lld or N = %lld outside [1, %d]", (long long)K, (long long)N, (int)MLP_MAX_DIM);
  if (activation < MLP_ACT_LINEAR || activation > MLP_ACT_SILU) return fail(MLP_ERR_UNSUPPORTED, "unknown activation %d", activation);
  if (!valid_type(y_type)) return fail(MLP_ERR_UNSUPPORTED, "unknown type of Y");
  if (M == 0) return MLP_OK;
  if (!X || !W || !Y) return fail(MLP_ERR_INVALID_ARG, "null X, W or Y");
  if (!valid_ld(ldx, K) || !valid_ld(ldw, N) || !valid_ld(ldy, N) || (R && !valid_ld(ldr, N)))
    return fail(MLP_ERR_INVALID_ARG, "row stride outside [columns, %d]", (int)MLP_MAX_DIM);
  if (!aligned(X, 2) || !aligned(W, 2) || !aligned(bias, 4) || !aligned(stash, 4) || !aligned(Y, type_size(y_type)) ||
      !aligned(R, type_size(y_type)) || !aligned(ws, 256))
    return fail(MLP_ERR_INVALID_ARG, "misaligned pointer (ws: 256 bytes; others: their elements)");
  const DenseWs w = dense_ws(M, K, N, MLP_MODE_INFER);
  if (w.total > 0 && !ws) return fail(MLP_ERR_WORKSPACE, "this shape needs %zu workspace bytes", w.total);
  GemmArgs g{};
  g.m = side(X, ldx, M, K);
  g.n = side(W, ldw, K, N);
  g.M = M;
  g.N = (int)N;
  g.K = K;
  g.out.bias = bias;
  g.out.act = activation;
  g.out.stash = activation == MLP_ACT_LINEAR ? nullptr : stash;
  g.out.R = R;
  g.out.ldr = ldr;
  g.out.C = Y;
  g.out.ldc = ldy;
  g.out.c_fp32 = y_type == MLP_FP32;
  // Y is not read again here and would only displace X and W from the caches
  // (8192 x 2048 x 8192 with GELU: 274 -> 259 us); gradients showed no gain.
  g.out.nt = 1;
  const hipError_t e = launch_gemm(GEMM_XW, g, static_cast<float*>(ws), static_cast<hipStream_t>(stream));
  return e == hipSuccess ? MLP_OK : hip_fail(e, "dense product launch");
} catch (...) {
  return entry_failed();
}

int mlp_dense_backward(const uint16_t* X, int64_t ldx, const uint16_t* W, int64_t ldw, int activation, const float* stash,
                       const void* dY, int dy_type, int64_t lddy, void* dX, int dx_type, int64_t lddx, void* dW, int dw_type,
                       int64_t lddw, float* db, int64_t M, int64_t K, int64_t N, void* ws_, void* stream) try {
  clear_error();
  if (M < 0 || M > kMaxRows) return fail(MLP_ERR_INVALID_ARG, "M = %lld outside [0, 2^30]", (long long)M);
  if (K < 1 || K > kMaxDim || N < 1 || N > kMaxDim)
    return fail(MLP_ERR_INVALID_ARG, "K = %lld or N = %lld outside [1, %d]", (long long)K, (long long)N, (int)MLP_MAX_DIM);
  if (activation < MLP_ACT_LINEAR || activation > MLP_ACT_SILU) return fail(MLP_ERR_UNSUPPORTED, "unknown activation %d", activation);
  if (!valid_type(dy_type) || !valid_type(dx_type) || !valid_type(dw_type)) return fail(MLP_ERR_UNSUPPORTED, "unknown type of dY, dX or dW");
  if (!ws_) return fail(MLP_ERR_INVALID_ARG, "null workspace");
  if (M > 0 && (!dY || (dX && !W) || (dW && !X))) return fail(MLP_ERR_INVALID_ARG, "null dY, or W for dX, or X for dW");
  if (M > 0 && activation != MLP_ACT_LINEAR && !stash) return fail(MLP_ERR_INVALID_ARG, "null stash of a layer with an activation");
  if ((M > 0 && (!valid_ld(lddy, N) || (dX && (!valid_ld(lddx, K) || !valid_ld(ldw, N))) || (dW && !valid_ld(ldx, K)))) ||
      (dW && !valid_ld(lddw, N)))
    return fail(MLP_ERR_INVALID_ARG, "row stride outside [columns, %d]", (int)MLP_MAX_DIM);
  if (!aligned(X, 2) || !aligned(W, 2) || !aligned(stash, 4) || !aligned(dY, type_size(dy_type)) || !aligned(dX, type_size(dx_type)) ||
      !aligned(dW, type_size(dw_type)) || !aligned(db, 4) || !aligned(ws_, 256))
    return fail(MLP_ERR_INVALID_ARG, "misaligned pointer (ws: 256 bytes; others: their elements)");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const DenseWs w = dense_ws(M, K, N, MLP_MODE_TRAIN);
  uint8_t* ws = static_cast<uint8_t*>(ws_);
  if (activation == MLP_ACT_LINEAR) stash = nullptr;
  SideArgs dz = side(dY, lddy, M, N);
  const bool round = M > 0 && (dX || dW) && (stash || dy_type == MLP_FP32);  // dZ is not dY itself
  hipError_t e;
  if (round || db) {
    DeltaArgs d{};
    d.dY = dY;
    d.dy_fp32 = dy_type == MLP_FP32;
    d.lddy = lddy;
    d.stash = stash;
    d.relu = activation == MLP_ACT_RELU;
    d.dZ = round ? reinterpret_cast<uint16_t*>(ws + w.dz) : nullptr;
    d.ldz = w.ldz;
    d.partial = reinterpret_cast<float*>(ws + w.db);
    d.db = db;
    d.M = M;
    d.N = (int)N;
    d.parts = w.parts;
    e = launch_delta(d, s);
    if (e != hipSuccess) return hip_fail(e, "delta kernel launch");
    if (round) dz = side(d.dZ, w.ldz, M, N);
  }
  float* partial = reinterpret_cast<float*>(ws + w.partial);
  if (dX && M > 0) {
    GemmArgs g{};
    g.m = dz;
    g.n = side(W, ldw, K, N);
    g.M = M;
    g.N = (int)K;
    g.K = N;
    g.out.C = dX;
    g.out.ldc = lddx;
    g.out.c_fp32 = dx_type == MLP_FP32;
    e = launch_gemm(GEMM_DX, g, partial, s);
    if (e != hipSuccess) return hip_fail(e, "dX product launch");
  }
  if (dW) {
    GemmArgs g{};
    g.m = side(X, ldx, M, K);
    g.n = dz;
    if (round) g.n.cols = (int64_t)round_up((size_t)N, 8);
    g.M = K;
    g.N = (int)N;
    g.K = M;
    g.out.C = dW;
    g.out.ldc = lddw;
    g.out.c_fp32 = dw_type == MLP_FP32;
    e = launch_gemm(GEMM_DW, g, partial, s);
    if (e != hipSuccess) return hip_fail(e, "dW product launch");
  }
  return MLP_OK;
} catch (...) {
  return entry_failed();
}

// ------------------------------------------------------------------- head --

size_t mlp_head_workspace_bytes(int64_t M, int64_t D, int64_t V, int top, int mode) {
  if (M < 0 || M > kMaxHeadRows || D < 1 || D > kMaxDim || V < 1 || V > kMaxDim || top < 1 || top > kHeadMaxTop) return 0;
  if (mode != MLP_MODE_INFER && mode != MLP_MODE_TRAIN) return 0;
  return head_ws(M, D, V, top, mode, true).total;
}

int mlp_cross_entropy(const uint16_t* H, int64_t ldh, const uint16_t* W, int64_t ldw, const int64_t* target, int64_t ignore_index,
                      float* loss, float* row_loss, void* dH, int dh_type, int64_t lddh, void* dW, int dw_type, int64_t lddw,
                      int64_t M, int64_t D, int64_t V, void* ws, void* stream) try {
  clear_error();
  if (int rc = check_head(H, ldh, W, ldw, dH, dh_type, lddh, dW, dw_type, lddw, loss, row_loss, M, D, V, ws)) return rc;
  if (M > 0 && !target) return fail(MLP_ERR_INVALID_ARG, "null target");
  if (!aligned(target, 8)) return fail(MLP_ERR_INVALID_ARG, "target must be 8-byte aligned");
  const HeadWs w = head_ws(M, D, V, 1, dW ? MLP_MODE_TRAIN : MLP_MODE_INFER, false);
  HeadArgs a{};
  a.h = side(H, ldh, M, D);
  a.w = side(W, ldw, D, V);
  a.M = M;
  a.D = D;
  a.V = (int)V;
  a.scale2 = 1.44269504f;
  a.target = target;
  a.ignore = ignore_index;
  a.top = 1;
  RowLossArgs r{};
  r.target = target;
  r.ignore = ignore_index;
  r.top = 1;
  r.temperature = r.t2 = 1.f;
  r.loss = loss;
  r.row_loss = row_loss;
  return run_head(false, a, r, w, static_cast<uint8_t*>(ws), dH, dh_type, lddh, dW, dw_type, lddw, static_cast<hipStream_t>(stream));
} catch (...) {
  return entry_failed();
}

int mlp_distill(const uint16_t* H, int64_t ldh, const uint16_t* W, int64_t ldw, const int64_t* index, const void* logits,
                int logits_type, int top, float temperature, float* loss, float* row_loss, void* dH, int dh_type, int64_t lddh,
                void* dW, int dw_type, int64_t lddw, int64_t M, int64_t D, int64_t V, void* ws_, void* stream) try {
  clear_error();
  if (int rc = check_head(H, ldh, W, ldw, dH, dh_type, lddh, dW, dw_type, lddw, loss, row_loss, M, D, V, ws_)) return rc;
  if (top < 1 || top > kHeadMaxTop) return fail(MLP_ERR_INVALID_ARG, "top = %d outside [1, %d]", top, kHeadMaxTop);
  // its square and inverse, times a logit, stay well within fp32
  if (!(temperature >= 1e-4f && temperature <= 1e4f)) return fail(MLP_ERR_INVALID_ARG, "temperature outside [1e-4, 1e4]");
  if (!valid_type(logits_type)) return fail(MLP_ERR_UNSUPPORTED, "unknown type of the teacher's logits");
  if (M > 0 && (!index || !logits)) return fail(MLP_ERR_INVALID_ARG, "null index or logits");
  if (!aligned(index, 8) || !aligned(logits, type_size(logits_type))) return fail(MLP_ERR_INVALID_ARG, "misaligned index or logits");
  hipStream_t s = static_cast<hipStream_t>(stream);
  uint8_t* ws = static_cast<uint8_t*>(ws_);
  const HeadWs w = head_ws(M, D, V, top, dW ? MLP_MODE_TRAIN : MLP_MODE_INFER, true);
  TeacherArgs t{};
  t.index = index;
  t.logits = logits;
  t.logits_fp32 = logits_type == MLP_FP32;
  t.inv_t = 1.f / temperature;
  t.M = M;
  t.V = V;
  t.top = top;
  t.keys = w.keys;
  t.out_index = reinterpret_cast<int*>(ws + w.index);
  t.out_q = reinterpret_cast<float*>(ws + w.q);
  t.start = reinterpret_cast<uint16_t*>(ws + w.start);
  t.ok = reinterpret_cast<int*>(ws + w.ok);
  if (M > 0) {
    const hipError_t e = launch_teacher(t, s);
    if (e != hipSuccess) return hip_fail(e, "teacher list kernel launch");
  }
  HeadArgs a{};
  a.h = side(H, ldh, M, D);
  a.w = side(W, ldw, D, V);
  a.M = M;
  a.D = D;
  a.V = (int)V;
  a.scale2 = 1.44269504f / temperature;
  a.index = t.out_index;
  a.q = t.out_q;
  a.start = t.start;
  a.top = top;
  a.keys = w.keys;
  RowLossArgs r{};
  r.q = t.out_q;
  r.ok = t.ok;
  r.top = top;
  r.t2 = temperature * temperature;
  r.temperature = temperature;
  r.loss = loss;
  r.row_loss = row_loss;
  return run_head(true, a, r, w, ws, dH, dh_type, lddh, dW, dw_type, lddw, s);
} catch (...) {
  return entry_failed();
}

}  // extern "C"
