/* Host-only exercise of the entry points around the fused nets (layer norm,
 * dense layers, vocabulary losses) for the sanitizer build: workspace sizes
 * over many shapes and every argument check that fails before a launch.
 * Never launches a kernel.  Exit status 0 when every check holds. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "ffmlp.h"

#define CHECK(c)                                                      \
  do {                                                                \
    if (!(c)) {                                                       \
      fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c); \
      return 1;                                                       \
    }                                                                 \
  } while (0)

static const int64_t kRows[] = {0, 1, 15, 16, 17, 127, 1000, 4097, 1 << 20, 1 << 24};
static const int64_t kDims[] = {1, 7, 8, 100, 128, 1000, 4096, 65536, MLP_MAX_DIM};

static int sizes(void) {
  for (size_t i = 0; i < sizeof kRows / sizeof *kRows; ++i)
    for (size_t j = 0; j < sizeof kDims / sizeof *kDims; ++j) {
      const int64_t M = kRows[i], N = kDims[j];
      CHECK(mlp_layer_norm_workspace_bytes(M, N, MLP_MODE_INFER) == 0);
      CHECK(mlp_layer_norm_workspace_bytes(M, N, MLP_MODE_TRAIN) >= (size_t)N * 8);
      for (size_t k = 0; k < sizeof kDims / sizeof *kDims; ++k) {
        const int64_t K = kDims[k];
        const size_t inf = mlp_dense_workspace_bytes(M, K, N, MLP_MODE_INFER);
        const size_t trn = mlp_dense_workspace_bytes(M, K, N, MLP_MODE_TRAIN);
        CHECK(inf % 256 == 0 && trn % 256 == 0 && trn >= inf && trn >= (size_t)(2 * M * N));
        if (M > 1 << 20) continue;
        const size_t hi = mlp_head_workspace_bytes(M, K, N, 1, MLP_MODE_INFER);
        const size_t ht = mlp_head_workspace_bytes(M, K, N, 1, MLP_MODE_TRAIN);
        CHECK(hi > 0 && hi % 256 == 0 && ht >= hi);
        CHECK(mlp_head_workspace_bytes(M, K, N, 1024, MLP_MODE_TRAIN) >= ht);
      }
    }
  CHECK(mlp_layer_norm_workspace_bytes(-1, 8, MLP_MODE_TRAIN) == 0 && mlp_layer_norm_workspace_bytes(1, 0, MLP_MODE_TRAIN) == 0);
  CHECK(mlp_dense_workspace_bytes(1, 8, (int64_t)MLP_MAX_DIM + 1, MLP_MODE_TRAIN) == 0);
  CHECK(mlp_dense_workspace_bytes(1, 8, 8, 7) == 0);
  CHECK(mlp_head_workspace_bytes(1, 8, 8, 0, MLP_MODE_TRAIN) == 0 && mlp_head_workspace_bytes(1, 8, 8, 1025, MLP_MODE_TRAIN) == 0);
  return 0;
}

static int refusals(void) {
  void* p = (void*)(uintptr_t)0x1000; /* never dereferenced */
  void* q = (void*)(uintptr_t)0x1001;
  const int inv = MLP_ERR_INVALID_ARG, uns = MLP_ERR_UNSUPPORTED, b = MLP_BF16, f = MLP_FP32;
  const int64_t big = (int64_t)MLP_MAX_DIM + 1;
#define NF(X, xt, ldx, g, Y, yt, ldy, st, M, N, eps) mlp_layer_norm_forward(X, xt, ldx, g, NULL, Y, yt, ldy, st, M, N, eps, NULL)
  CHECK(NF(p, b, 8, NULL, p, b, 8, NULL, -1, 8, 1e-5f) == inv && NF(p, b, 8, NULL, p, b, 8, NULL, 4, 0, 1e-5f) == inv);
  CHECK(NF(p, b, 8, NULL, p, b, 8, NULL, ((int64_t)1 << 30) + 1, 8, 1e-5f) == inv && NF(p, b, big, NULL, p, b, 8, NULL, 4, 8, 1e-5f) == inv);
  CHECK(NF(p, 2, 8, NULL, p, b, 8, NULL, 4, 8, 1e-5f) == uns && NF(p, b, 8, NULL, p, -1, 8, NULL, 4, 8, 1e-5f) == uns);
  CHECK(NF(p, b, 8, NULL, p, b, 8, NULL, 4, 8, 0.f) == inv && NF(p, b, 8, NULL, p, b, 8, NULL, 4, 8, NAN) == inv);
  CHECK(NF(NULL, b, 8, NULL, p, b, 8, NULL, 4, 8, 1e-5f) == inv && NF(p, b, 7, NULL, p, b, 8, NULL, 4, 8, 1e-5f) == inv);
  CHECK(NF(q, b, 8, NULL, p, b, 8, NULL, 4, 8, 1e-5f) == inv && NF(p, f, 8, q, p, b, 8, NULL, 4, 8, 1e-5f) == inv);
  CHECK(NF(NULL, b, 0, NULL, NULL, b, 0, NULL, 0, 8, 1e-5f) == MLP_OK);
#define NB(X, st, dY, dX, ldx, dg, ws, M, N) mlp_layer_norm_backward(X, b, 8, NULL, st, dY, f, 8, dX, b, ldx, dg, p, M, N, ws, NULL)
  CHECK(NB(p, NULL, p, p, 8, p, p, 4, 8) == inv && NB(p, p, p, p, 8, NULL, p, 4, 8) == inv && NB(p, p, p, p, 8, p, NULL, 4, 8) == inv);
  CHECK(NB(p, p, p, p, 4, p, p, 4, 8) == inv && NB(p, p, p, NULL, 8, p, p, 4, 8) == inv && NB(p, p, p, p, 8, p, q, 4, 8) == inv);
#define DF(X, ldx, W, ldw, act, R, ldr, Y, yt, st, M, K, N, ws) mlp_dense_forward(X, ldx, W, ldw, NULL, act, R, ldr, Y, yt, N, st, M, K, N, ws, NULL)
  CHECK(DF(p, 8, p, 8, 6, NULL, 0, p, b, NULL, 4, 8, 8, p) == uns && DF(p, 8, p, 8, -1, NULL, 0, p, b, NULL, 4, 8, 8, p) == uns);
  CHECK(DF(p, 8, p, 8, 0, NULL, 0, p, 3, NULL, 4, 8, 8, p) == uns && DF(p, 8, p, 8, 0, NULL, 0, p, b, NULL, 4, 0, 8, p) == inv);
  CHECK(DF(p, 7, p, 8, 0, NULL, 0, p, b, NULL, 4, 8, 8, p) == inv && DF(p, 8, p, 7, 0, NULL, 0, p, b, NULL, 4, 8, 8, p) == inv);
  CHECK(DF(p, 8, p, 8, 0, p, 7, p, b, NULL, 4, 8, 8, p) == inv && DF(p, 8, p, 8, 0, q, 8, p, b, NULL, 4, 8, 8, p) == inv);
  CHECK(DF(NULL, 8, p, 8, 0, NULL, 0, p, b, NULL, 4, 8, 8, p) == inv && DF(p, 8, p, 8, 4, NULL, 0, p, b, q, 4, 8, 8, p) == inv);
  CHECK(DF(p, 4096, p, 64, 0, NULL, 0, p, b, NULL, 2, 4096, 64, NULL) == MLP_ERR_WORKSPACE); /* one row needs none */
  CHECK(DF(NULL, 0, NULL, 0, 0, NULL, 0, NULL, b, NULL, 0, 8, 8, NULL) == MLP_OK);
#define DB(X, W, act, st, dY, dyt, dX, dW, lddw, M, ws) mlp_dense_backward(X, 8, W, 8, act, st, dY, dyt, 8, dX, b, 8, dW, b, lddw, p, M, 8, 8, ws, NULL)
  CHECK(DB(p, p, 1, NULL, p, b, p, p, 8, 4, p) == inv && DB(p, p, 0, NULL, NULL, b, p, p, 8, 4, p) == inv);
  CHECK(DB(NULL, p, 0, NULL, p, b, p, p, 8, 4, p) == inv && DB(p, NULL, 0, NULL, p, b, p, p, 8, 4, p) == inv);
  CHECK(DB(p, p, 0, NULL, p, 5, p, p, 8, 4, p) == uns && DB(p, p, 0, NULL, p, b, p, p, 7, 4, p) == inv && DB(p, p, 0, NULL, p, b, p, p, 8, 4, NULL) == inv);
#define CE(H, ldh, W, ldw, t, dH, dW, M, D, V, ws) mlp_cross_entropy(H, ldh, W, ldw, t, -100, p, NULL, dH, f, D, dW, f, V, M, D, V, ws, NULL)
  CHECK(CE(NULL, 8, p, 9, p, NULL, NULL, 4, 8, 9, p) == inv && CE(p, 8, NULL, 9, p, NULL, NULL, 4, 8, 9, p) == inv);
  CHECK(CE(p, 8, p, 9, NULL, NULL, NULL, 4, 8, 9, p) == inv && CE(p, 8, p, 9, p, p, NULL, 4, 8, 9, p) == inv);
  CHECK(CE(p, 7, p, 9, p, NULL, NULL, 4, 8, 9, p) == inv && CE(p, 8, p, 8, p, NULL, NULL, 4, 8, 9, p) == inv);
  CHECK(CE(p, 8, p, 9, p, NULL, NULL, 4, 8, 9, NULL) == inv && CE(p, 8, p, 9, q, NULL, NULL, 4, 8, 9, p) == inv);
  CHECK(CE(p, 8, p, 9, p, NULL, NULL, ((int64_t)1 << 24) + 1, 8, 9, p) == inv && CE(p, 8, p, big, p, NULL, NULL, 4, 8, big, p) == inv);
#define KD(idx, z, zt, top, T, ws) mlp_distill(p, 8, p, 9, idx, z, zt, top, T, p, NULL, NULL, f, 8, NULL, f, 9, 4, 8, 9, ws, NULL)
  CHECK(KD(NULL, p, f, 3, 1.f, p) == inv && KD(p, NULL, f, 3, 1.f, p) == inv && KD(p, p, 2, 3, 1.f, p) == uns);
  CHECK(KD(p, p, f, 0, 1.f, p) == inv && KD(p, p, f, 1025, 1.f, p) == inv && KD(p, p, f, 3, 0.f, p) == inv);
  CHECK(KD(p, p, f, 3, -1.f, p) == inv && KD(p, p, f, 3, INFINITY, p) == inv && KD(p, p, f, 3, NAN, p) == inv && KD(p, q, f, 3, 1.f, p) == inv);
  CHECK(strlen(mlp_last_error()) > 0);
  return 0;
}

int main(void) {
  if (sizes() || refusals()) return 1;
  printf("layers ok\n");
  return 0;
}
