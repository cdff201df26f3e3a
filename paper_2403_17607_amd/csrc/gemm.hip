// Wide products: the choice of tile and splits, the sum of the splits, and
// the pass over dY in front of a layer's backward products.
#include "gemm_kernel.h"
#include "rows.h"

namespace ffmlp {

namespace {

constexpr int kWorkgroups = 512;  // two per CU

struct TileSize { int bm, bn, bk; };
TileSize tile_size(int tile) {
  if (tile == GEMM_SQUARE) return {GemmSquare::BM, GemmSquare::BN, GemmSquare::BK};
  if (tile == GEMM_LARGE) return {GemmLarge::BM, GemmLarge::BN, GemmLarge::BK};
  if (tile == GEMM_MEDIUM) return {GemmMedium::BM, GemmMedium::BN, GemmMedium::BK};
  return {GemmRows::BM, GemmRows::BN, GemmRows::BK};
}
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

GemmPlan gemm_plan(int form, int64_t M, int64_t N, int64_t K) {
  GemmPlan p{};
  const int64_t large = cdiv(M, GemmLarge::BM) * cdiv(N, GemmLarge::BN);
  p.tile = form != GEMM_DW && M <= GemmRows::BM ? GEMM_ROWS
           : large < kWorkgroups / 4             ? GEMM_MEDIUM
           : form == GEMM_XW                     ? GEMM_LARGE
                                                 : GEMM_SQUARE;
  const TileSize t = tile_size(p.tile);
  p.mt = (int)cdiv(M, t.bm);
  p.nt = (int)cdiv(N, t.bn);
  const int64_t tiles = (int64_t)p.mt * p.nt;
  // Splits fill the chip when the tiles do not, each over at least 256 of k.
  int64_t s = (p.tile == GEMM_SQUARE ? kWorkgroups / 2 : kWorkgroups) / tiles, most = K / 256;
  if (s > most) s = most;
  if (s < 1) s = 1;
  p.kper = K > 0 ? cdiv(cdiv(K, s), t.bk) * t.bk : t.bk;
  p.splits = K > 0 ? (int)cdiv(K, p.kper) : 1;
  p.partial_bytes = p.splits > 1 ? (size_t)p.splits * M * N * 4 : 0;
  return p;
}

// The splits' partial sums added in order, then the epilogue.
__global__ __launch_bounds__(256) void split_sum_kernel(const float* partial, int splits, int64_t M, int N, const GemmOut o) {
  const int per = (N + 3) / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= M * per) return;
  const int64_t m = i / per;
  const int n = (int)(i % per) * 4;
  const float* p = partial + m * N + n;
  f32x4 z = {0.f, 0.f, 0.f, 0.f};
  if ((N & 3) == 0) {
    for (int s = 0; s < splits; ++s, p += M * N) z += *reinterpret_cast<const f32x4*>(p);
  } else {
    for (int s = 0; s < splits; ++s, p += M * N)
#pragma unroll
      for (int q = 0; q < 4; ++q) z[q] += n + q < N ? p[q] : 0.f;
  }
  out4(o, m, n, N, z);
}

hipError_t launch_gemm(int form, GemmArgs a, float* partial, hipStream_t s) {
  if (a.M <= 0 || a.N <= 0) return hipSuccess;
  const GemmPlan p = gemm_plan(form, a.M, a.N, a.K);
  a.mt = p.mt;
  a.nt = p.nt;
  a.tiles = p.mt * p.nt;
  a.splits = p.splits;
  a.kper = p.kper;
  a.partial = partial;
  hipError_t e = form == GEMM_XW   ? launch_gemm_xw(p.tile, a, s)
                 : form == GEMM_DX ? launch_gemm_dx(p.tile, a, s)
                                   : launch_gemm_dw(p.tile, a, s);
  if (e != hipSuccess || p.splits <= 1) return e;
  const int64_t n = a.M * ((a.N + 3) / 4);
  hipLaunchKernelGGL(split_sum_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, partial, p.splits, a.M, a.N, a.out);
  return hipGetLastError();
}

// ------------------------------------------------------------ column sums --

// Block (x, y): columns 512 x + 8 lane .. + 7, rows of part y, its four waves
// one row after the other.  Reads dY (and the stash) once, writes dZ; the
// column sums stay in registers until the block ends.
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
#pragma unroll 2
    for (int64_t r = r0 + wave; r < r1; r += 4) {
      float v[8];
      if constexpr (F32) load8(static_cast<const float*>(a.dY) + r * a.lddy + c, n, v);
      else load8(static_cast<const uint16_t*>(a.dY) + r * a.lddy + c, n, v);
      if (a.stash) {
        float d[8];
        load8(a.stash + r * a.N + c, n, d);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = a.relu && d[q] == 0.f ? 0.f : v[q] * d[q];
      }
#pragma unroll
      for (int q = 0; q < 8; ++q) db[q] += v[q];
      if (a.dZ) store8(a.dZ + r * a.ldz + c, n, v);
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
  const int64_t want = cdiv(2 * kWorkgroups, cdiv(N, 512)), most = cdiv(M, 16);
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
// order, then the slices are added in order.
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
