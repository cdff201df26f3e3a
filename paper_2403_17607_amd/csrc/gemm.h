// Arguments and launches of the wide products (gemm_kernel.h).
#pragma once

#include "common.h"

namespace ffmlp {

// A matrix operand: rows x cols elements, row-major with row stride ld.  Where
// k runs across the rows, columns past those of C may be named (they have to
// exist): a buffer of this library's own whose rows end with a whole piece.
struct SideArgs {
  const uint16_t* p;
  int64_t ld;
  int64_t rows, cols;
};

// What becomes of a product's fp32 sums z, in this order.
struct GemmOut {
  const float* add;    // z += add [M][ldadd], or null
  int64_t ldadd;
  const float* alpha;  // z *= *alpha (device), or null
  const float* bias;   // z += bias [N], or null
  int act;             // y = act(z)
  float* stash;        // act'(z) [M][N], or null
  const void* R;       // y += R [M][ldr], C's type, or null
  int64_t ldr;
  void* C;             // [M][ldc], bf16 or fp32
  int64_t ldc;
  int c_fp32;
  int nt;              // non-temporal stores of C
};

struct GemmArgs {
  SideArgs m, n;
  int64_t M, K;
  int N;
  GemmOut out;
  float* partial;  // [splits][M][N] fp32 when splits > 1
  int splits;
  int64_t kper;    // k of a split, a multiple of the tile's BK
  int mt, nt;
};

// Workgroup tiles (gemm_kernel.h) and which sides have k across their rows.
enum { GEMM_ROWS = 0, GEMM_SMALL = 1, GEMM_MEDIUM = 2, GEMM_HALF = 3, GEMM_LARGE = 4, GEMM_SQUARE = 5 };
enum { GEMM_XW = 0, GEMM_DX = 1, GEMM_DW = 2 };

struct GemmPlan {
  int tile, splits, mt, nt;
  int64_t kper;
  size_t partial_bytes;  // workspace of the splits' partial sums
};
// Tile and splits of an M x N product over K, from the sizes alone.
GemmPlan gemm_plan(int form, int64_t M, int64_t N, int64_t K);

// C = the product of the two sides as a.out says; fills in tiles and splits.
// `partial`: gemm_plan(...).partial_bytes of workspace.
hipError_t launch_gemm(int form, GemmArgs a, float* partial, hipStream_t s);

hipError_t launch_gemm_xw(int tile, const GemmArgs& a, hipStream_t s);
hipError_t launch_gemm_dx(int tile, const GemmArgs& a, hipStream_t s);
hipError_t launch_gemm_dw(int tile, const GemmArgs& a, hipStream_t s);

// dZ = bf16(dY * stash) [M][ldz] (dZ null: not stored; stash null: linear) and,
// for db, the column sums of the unrounded products: `parts` partial sums
// [parts][N] in `partial`, then db in a fixed order.
struct DeltaArgs {
  const void* dY;
  int dy_fp32;
  int64_t lddy;
  const float* stash;     // [M][N]
  int relu;               // a derivative of 0 gives 0 whatever dY is
  uint16_t* dZ;
  int64_t ldz;
  float* partial;
  float* db;
  int64_t M;
  int N, parts;
};
int delta_parts(int64_t M, int N);
hipError_t launch_delta(const DeltaArgs& a, hipStream_t s);

// out0[c], out1[c - C] (c < C, else) = sum over p of partial[p][c], c < 2 C (C if out1 is null).
hipError_t launch_column_reduce(const float* partial, int parts, int64_t C, float* out0, float* out1, hipStream_t s);

// ---- layer norm
struct NormArgs {
  const void* X;
  int x_fp32;
  int64_t ldx;
  const float *gamma, *beta;  // null: 1 and 0
  void* Y;
  int y_fp32;
  int64_t ldy;
  float* stats;  // [M][2] mean and 1 / std: written by the forward pass unless null
  float eps;
  const void* dY;
  int dy_fp32;
  int64_t lddy;
  void* dX;
  int dx_fp32;
  int64_t lddx;
  float *dgamma, *dbeta;
  float* partial;  // [parts][2][N]
  int64_t M;
  int N, parts;
};
int norm_parts(int64_t M, int N);
hipError_t launch_norm_forward(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s);

}  // namespace ffmlp
