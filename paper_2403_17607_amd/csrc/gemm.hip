// Wide products: the choice of tile and splits, the sum of the splits, and
// the pass over dY in front of a layer's backward products.
#include "gemm_kernel.h"
#include "rows.h"

namespace ffmlp {

namespace {

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// What a tile costs, in microseconds measured on an MI355X: a step of k of a
// workgroup that has a CU to itself and of one that shares it, and the rest of
// its life (first loads, epilogue), which shared CUs hide in part.  Shapes of
// 2048 .. 8192 rows, 1024 .. 8192 columns and 1024 .. 32768 of k, both ways:
//   8192 x 1024 over 4096 (X W): square 106, large 85, half 71, medium 89; with
//     two splits and their sum large 82
//   8192 x 8192 over 2048 (X W): square 265, large 240, half 285
//   4096 x 1024 over 8192 (X^T dZ): square 191, half 104, medium 90; half with
//     two splits and their sum 85
//   1024 x 1024 over 1024 (X W): large 25, half 16, medium 10.1, small 8.1
//   1111 x 771 over 1283 (dZ W^T): medium 13.5, small 10.8; 1111 x 1283 over 771
//     (X W): medium 10.1, small 12.4
// The costs are those of aligned rows and bf16 results; where rows start at odd
// elements or a result is fp32, every tile takes longer, in other proportions.
struct TileCost {
  int tile, bm, bn, bk, per_cu;
  double alone, shared, rest;
};
template <typename TL>
constexpr TileCost tile_cost(int tile, int per_cu, double alone, double shared, double rest) {
  return TileCost{tile, TL::BM, TL::BN, TL::BK, per_cu, alone, shared, rest};
}
constexpr TileCost kTiles[] = {
    tile_cost<GemmSquare>(GEMM_SQUARE, 1, 1.60, 1.60, 16.0),
    tile_cost<GemmLarge>(GEMM_LARGE, 2, 0.62, 0.90, 4.0),
    tile_cost<GemmHalf>(GEMM_HALF, 2, 0.75, 1.05, 5.0),
    tile_cost<GemmMedium>(GEMM_MEDIUM, 2, 0.42, 0.66, 4.0),
    tile_cost<GemmSmall>(GEMM_SMALL, 2, 0.28, 0.50, 3.5),
    tile_cost<GemmRows>(GEMM_ROWS, 2, 0.30, 0.40, 3.0),
};
constexpr int kCUs = 256;

// One side only: the large tile's short rows of k suit a side with k across
// its rows (X W); 16-row tiles need rows on the m side.
bool tile_suits(int tile, int form, int64_t M) {
  if (tile == GEMM_LARGE) return form == GEMM_XW;
  if (tile == GEMM_ROWS) return form != GEMM_DW && M <= GemmRows::BM;
  return true;
}

bool one_row(int form, int64_t M) { return form == GEMM_XW && M == 1; }

}  // namespace

GemmPlan gemm_plan(int form, int64_t M, int64_t N, int64_t K) {
  GemmPlan best{};
  if (one_row(form, M)) return best;
  double best_us = 0;
  for (const TileCost& t : kTiles) {
    if (!tile_suits(t.tile, form, M)) continue;
    const int64_t mt = cdiv(M, t.bm), nt = cdiv(N, t.bn), tiles = mt * nt, slots = (int64_t)kCUs * t.per_cu;
    const int64_t steps = cdiv(K > 0 ? K : 1, t.bk);
    for (int64_t want = 1; want == 1 || (want <= 64 && want * 4 <= steps && tiles * want <= slots); want *= 2) {
      const int64_t per = cdiv(steps, want), splits = cdiv(steps, per), n = tiles * splits;
      const double us = (double)cdiv(n, slots) * ((double)per * (n > kCUs ? t.shared : t.alone) + t.rest) +
                        (splits > 1 ? 5.0 + (double)(splits + 1) * (double)M * (double)N * 4e-6 / 4.5 : 0.0);
      if (best_us == 0 || us < best_us) {
        best_us = us;
        best.tile = t.tile;
        best.mt = (int)mt;
        best.nt = (int)nt;
        best.kper = per * t.bk;
        best.splits = (int)splits;
      }
    }
  }
  best.partial_bytes = best.splits > 1 ? (size_t)best.splits * M * N * 4 : 0;
  return best;
}

// The splits' partial sums added in order, then the epilogue; a thread has eight
// columns of a row.  Bound by the latency of its few loads: two splits of 4096 x
// 1024 to fp32 take 10 us for 50 MB.
__global__ __launch_bounds__(256) void split_sum_kernel(const float* partial, int splits, int64_t M, int N, const GemmOut o) {
  const int per = (N + 7) / 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= M * per) return;
  const int64_t m = i / per;
  const int n = (int)(i % per) * 8;
  const float* p = partial + m * N + n;
  float z[8] = {}, b[8];
  bias8(o, n, N, b);
  int s = 0;
  for (; s + 4 <= splits; s += 4, p += 4 * M * N) {  // four loads in flight, added in order
    float v[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k) load8(p + k * M * N, N - n, v[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int q = 0; q < 8; ++q) z[q] += v[k][q];
  }
  for (; s < splits; ++s, p += M * N) {
    float v[8];
    load8(p, N - n, v);
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] += v[q];
  }
  out8(o, m, n, N, z, b, o.alpha ? *o.alpha : 1.f);
}

hipError_t launch_one_row(const GemmArgs& a, hipStream_t s);

hipError_t launch_gemm(int form, GemmArgs a, float* partial, hipStream_t s) {
  if (a.M <= 0 || a.N <= 0) return hipSuccess;
  if (one_row(form, a.M)) return launch_one_row(a, s);
  const GemmPlan p = gemm_plan(form, a.M, a.N, a.K);
  a.mt = p.mt;
  a.nt = p.nt;
  a.splits = p.splits;
  a.kper = p.kper;
  a.partial = partial;
  const hipError_t e = form == GEMM_XW   ? launch_gemm_xw(p.tile, a, s)
                       : form == GEMM_DX ? launch_gemm_dx(p.tile, a, s)
                                         : launch_gemm_dw(p.tile, a, s);
  if (e != hipSuccess || p.splits <= 1) return e;
  const int64_t n = a.M * ((a.N + 7) / 8);
  hipLaunchKernelGGL(split_sum_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, partial, p.splits, a.M, a.N, a.out);
  return hipGetLastError();
}

// --------------------------------------------------------------- one row --

// Y = X W for one row: W is read once and its products are made on the vector
// units, so bandwidth and latency bound it (4096 x 4096: the 32 MiB of W, 6.5 us
// at the rate of a large copy).  A workgroup owns 8 LPR columns; LPR lanes hold
// them as 16-byte pieces, the wave's 64 / LPR groups take eight consecutive k
// each, the 16 waves every 16th such block.  Then the groups' sums are added by
// shuffles and the waves' in order through LDS.  LPR is chosen so that 256
// workgroups or more share an N of 4096 or more; those that share the 128 bytes of a line run on
// one chiplet.  4096 x 4096 with GELU: 11.3 us, against 13 of the matrix-core
// kernel with splits (two launches), which two rows take too.
template <int LPR>
__global__ __launch_bounds__(1024) void one_row_kernel(const GemmArgs a) {
  constexpr int COLS = 8 * LPR, PER = 64 / COLS, NW = 16;  // PER: workgroups of a line
  __shared__ __align__(16) float sums[NW][COLS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // workgroup b runs on chiplet b % 8: its neighbour there is b + 8
  const int b = blockIdx.x, at = (b / (8 * PER) * 8 + b % 8) * PER + b / 8 % PER;
  const int n = at * COLS + 8 * (lane % LPR);
  const int cols = a.N - n;  // of this lane
  float acc[8] = {};
  if (cols > 0) {
    for (int64_t k = (wave * (64 / LPR) + lane / LPR) * 8; k < a.K; k += NW * (64 / LPR) * 8) {
      const int kn = a.K - k < 8 ? (int)(a.K - k) : 8;
      u32x4 w[8];
      if (cols >= 8 && kn == 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = *reinterpret_cast<const u32x4_a2*>(a.n.p + (k + j) * a.n.ld + n);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          w[j] = u32x4{0u, 0u, 0u, 0u};
          if (j < kn) w[j] = load8_bits(a.n.p + (k + j) * a.n.ld + n, cols);
        }
      }
      float x[8];
      load8(a.m.p + k, kn, x);
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          acc[2 * q] += x[j] * bf16_lo(w[j][q]);
          acc[2 * q + 1] += x[j] * bf16_hi(w[j][q]);
        }
    }
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) {
#pragma unroll
    for (int d = LPR; d < 64; d *= 2) acc[q] += __shfl_xor(acc[q], d);
    if (lane < LPR) sums[wave][8 * lane + q] = acc[q];
  }
  __syncthreads();
  const int c = at * COLS + 8 * threadIdx.x;
  if (threadIdx.x >= LPR || c >= a.N) return;
  float z[8] = {}, bias[8], v[8];
  bias8(a.out, c, a.N, bias);
#pragma unroll 4
  for (int w = 0; w < NW; ++w) {
    lds8(&sums[w][8 * threadIdx.x], v);
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] += v[q];
  }
  out8(a.out, 0, c, a.N, z, bias, a.out.alpha ? *a.out.alpha : 1.f);
}

template <int LPR>
hipError_t launch_one_row_cols(const GemmArgs& a, hipStream_t s) {
  constexpr int COLS = 8 * LPR, PER = 64 / COLS;
  // whole lines on eight chiplets
  hipLaunchKernelGGL((one_row_kernel<LPR>), dim3((unsigned)(cdiv(a.N, COLS * 8 * PER) * 8 * PER)), dim3(1024), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_one_row(const GemmArgs& a, hipStream_t s) {
  return a.N >= 64 * 256 ? launch_one_row_cols<8>(a, s) : a.N >= 32 * 256 ? launch_one_row_cols<4>(a, s) : launch_one_row_cols<2>(a, s);
}

// ------------------------------------------------------------ column sums --

// Block (x, y): columns 512 x + 8 lane .. + 7, rows of part y, its four waves
// one row after the other.  Reads dY (and the stash) once, writes dZ; the
// column sums stay in registers until the block ends.  Bound by memory and, at
// sizes like 8192 x 1024 (8 us for the column sums of 17 MB of bf16), by the
// latency of the four rows that a wave has in flight.
template <bool F32>
__global__ __launch_bounds__(256) void delta_kernel(const DeltaArgs a) {
  __shared__ float sums[3][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.x * 512 + lane * 8;
  const int64_t per = (a.M + a.parts - 1) / a.parts;
  const int64_t r0 = per * blockIdx.y, r1 = r0 + per < a.M ? r0 + per : a.M;
  float db[8] = {};
  if (c < a.N) {
    const int n = a.N - c < 8 ? a.N - c : 8;
    for (int64_t r = r0 + wave; r < r1; r += 16) {  // four rows in flight
      float v[4][8], d[4][8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int nk = r + 4 * k < r1 ? n : 0;
        if constexpr (F32) load8(static_cast<const float*>(a.dY) + (r + 4 * k) * a.lddy + c, nk, v[k]);
        else load8(static_cast<const uint16_t*>(a.dY) + (r + 4 * k) * a.lddy + c, nk, v[k]);
        if (a.stash) load8(a.stash + (r + 4 * k) * a.N + c, nk, d[k]);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (a.stash)
#pragma unroll
          for (int q = 0; q < 8; ++q) v[k][q] = a.relu && d[k][q] == 0.f ? 0.f : v[k][q] * d[k][q];
#pragma unroll
        for (int q = 0; q < 8; ++q) db[q] += v[k][q];
        if (a.dZ && r + 4 * k < r1) store8(a.dZ + (r + 4 * k) * a.ldz + c, n, v[k]);
      }
    }
  }
  if (!a.db) return;
  if (wave)
#pragma unroll
    for (int q = 0; q < 8; ++q) sums[wave - 1][lane * 8 + q] = db[q];
  __syncthreads();
  if (wave == 0 && c < a.N)
#pragma unroll
    for (int q = 0; q < 8; ++q)
      if (c + q < a.N)
        a.partial[(int64_t)blockIdx.y * a.N + c + q] =
            ((db[q] + sums[0][lane * 8 + q]) + sums[1][lane * 8 + q]) + sums[2][lane * 8 + q];
}

int delta_parts(int64_t M, int N) {
  const int64_t want = cdiv(4 * kCUs, cdiv(N, 512)), most = cdiv(M, 16);
  return (int)(want < most ? want : most < 1 ? 1 : most);
}

hipError_t launch_delta(const DeltaArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)cdiv(a.N, 512), (unsigned)a.parts);
  if (a.dy_fp32) hipLaunchKernelGGL(delta_kernel<true>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(delta_kernel<false>, grid, dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.db) return e;
  return launch_column_reduce(a.partial, a.parts, a.N, a.db, nullptr, s);
}

// Block b: columns 64 b .. + 63; wave y of 16 adds the parts of slice y in
// order, then the slices are added in order.  3 to 5 us: a launch and three
// loads' latency.
__global__ __launch_bounds__(1024) void column_reduce_kernel(const float* partial, int parts, int64_t C, int64_t total,
                                                             float* out0, float* out1) {
  __shared__ float part[16][64];
  const int j = threadIdx.x & 63, y = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + j;
  float s = 0.f;
  if (c < total) {
    const int p0 = (int)((int64_t)parts * y / 16), p1 = (int)((int64_t)parts * (y + 1) / 16);
    const float* src = partial + c;
    int p = p0;
    for (; p + 8 <= p1; p += 8) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = src[(int64_t)(p + k) * total];
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
    }
    for (; p < p1; ++p) s += src[(int64_t)p * total];
  }
  part[y][j] = s;
  __syncthreads();
  if (threadIdx.x < 64 && c < total) {
    float g = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) g += part[k][threadIdx.x];
    float* o = c < C ? out0 + c : out1 + (c - C);
    *o = g;
  }
}

hipError_t launch_column_reduce(const float* partial, int parts, int64_t C, float* out0, float* out1, hipStream_t s) {
  const int64_t total = out1 ? 2 * C : C;
  hipLaunchKernelGGL(column_reduce_kernel, dim3((unsigned)cdiv(total, 64)), dim3(1024), 0, s, partial, parts, C, total, out0, out1);
  return hipGetLastError();
}

}  // namespace ffmlp
