// Losses of the logits H W over a vocabulary, never stored whole.
//
//   x = log2(e) / T * (H W)                    (the logits in base-2 units)
//   lse = log2 sum_v 2^x
//   P = 2^(x - lse) - q                        (q: the target distribution)
//
// head_lse_kernel walks a run of column tiles with one row tile and keeps the
// running maximum and sum of every row in registers, so the logits live only
// in the matrix cores' results.  head_prob_kernel recomputes a piece of the
// vocabulary and stores P as bf16, from which two products make the gradients
// dH = P W^T and dW = H^T P.  q is sparse: the one target of a row, or the
// teacher's top entries sorted by index, with a table of where each block of
// 128 columns begins in a row's list.
#pragma once

#include "gemm_kernel.h"
#include "head.h"

namespace ffmlp {

constexpr float kLn2 = 0.69314718f;

// f(column within the wave's columns, position in the row's list) for row
// `row`'s entries among `cols` columns from c0 on, c0 a multiple of 64.
template <bool DISTILL, typename F>
__device__ __forceinline__ void head_hits(const HeadArgs& a, int64_t row, int c0, int cols, F&& f) {
  if (row >= a.M) return;
  if constexpr (DISTILL) {
    const uint16_t* st = a.start + row * a.keys + c0 / kHeadKey;
    const int e1 = st[1];
    for (int e = st[0]; e < e1; ++e) {
      const int c = a.index[row * a.top + e] - c0;
      if (c >= 0 && c < cols) f(c, e);
    }
  } else {
    const int64_t t = a.target[row];
    if (t != a.ignore && t >= c0 && t < (int64_t)c0 + cols) f((int)(t - c0), 0);
  }
}

// Row tile and run of a workgroup: a chiplet (blockIdx % 8) gets neighbouring
// row tiles with all their runs, so that its L2 holds its rows of H.
__device__ __forceinline__ int head_block(int b, int total) {
  const int q = total / 8, r = total % 8, x = b % 8, y = b / 8;
  return x * q + (x < r ? x : r) + y;
}

template <typename TL, bool DIRECT, bool DISTILL>
__global__ __launch_bounds__(TL::NTHR, 2) void head_lse_kernel(const HeadArgs a) {
  extern __shared__ __align__(16) uint8_t head_lds[];
  const int t = head_block(blockIdx.x, a.mt * a.runs);
  const int tm = t / a.runs, run = t % a.runs;
  const int64_t m0 = (int64_t)tm * TL::BM;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4;
  const int64_t mw = m0 + (wave / TL::WN) * TL::MB * 16 + (lane & 15);
  float mx[TL::MB], sum[TL::MB];
#pragma unroll
  for (int m = 0; m < TL::MB; ++m) {
    mx[m] = -__builtin_inff();
    sum[m] = 0.f;
  }
  const int t1 = (run + 1) * a.per_run < a.nt ? (run + 1) * a.per_run : a.nt;
  for (int tn = run * a.per_run; tn < t1; ++tn) {
    const int n0 = tn * TL::BN, nw = n0 + (wave % TL::WN) * TL::NB * 16;
    f32x4 acc[TL::MB][TL::NB];
#pragma unroll
    for (int m = 0; m < TL::MB; ++m)
#pragma unroll
      for (int n = 0; n < TL::NB; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    gemm_loop<TL, false, true, DIRECT>(a.h, a.w, m0, n0, 0, a.D, head_lds, acc);
    static_for<0, TL::MB>([&](auto mc) {
      constexpr int m = decltype(mc)::value;
      float top = mx[m];
#pragma unroll
      for (int n = 0; n < TL::NB; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float x = acc[m][n][q] * a.scale2;
          if (n0 + TL::BN > a.V) x = nw + 16 * n + 4 * g + q < a.V ? x : -__builtin_inff();
          acc[m][n][q] = x;
          top = __builtin_fmaxf(top, x);
        }
      const float at = top == -__builtin_inff() ? 0.f : top;
      float s = sum[m] * __builtin_amdgcn_exp2f(mx[m] - at);
#pragma unroll
      for (int n = 0; n < TL::NB; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) s += __builtin_amdgcn_exp2f(acc[m][n][q] - at);
      mx[m] = top;
      sum[m] = s;
      head_hits<DISTILL>(a, mw + 16 * m, nw, TL::NB * 16, [&](int c, int e) {
        if (((c >> 2) & 3) != g) return;
        float x = 0.f;
#pragma unroll
        for (int n = 0; n < TL::NB; ++n)
#pragma unroll
          for (int q = 0; q < 4; ++q) x = (c >> 4) == n && (c & 3) == q ? acc[m][n][q] : x;
        a.pick[(mw + 16 * m) * a.top + e] = x;
      });
    });
  }
  // the four lane groups hold the same rows
  f32x2* part = a.partial + (int64_t)(run * TL::WN + wave % TL::WN) * a.M;
#pragma unroll
  for (int m = 0; m < TL::MB; ++m) {
#pragma unroll
    for (int d = 16; d < 64; d *= 2) head_merge(mx[m], sum[m], __shfl_xor(mx[m], d), __shfl_xor(sum[m], d));
    if (g == 0 && mw + 16 * m < a.M) part[mw + 16 * m] = f32x2{mx[m], sum[m]};
  }
}

// P of the columns a.col0 .. a.col0 + a.V - 1 (a.w begins at the first).
template <typename TL, bool DIRECT, bool DISTILL>
__global__ __launch_bounds__(TL::NTHR, 2) void head_prob_kernel(const HeadArgs a) {
  extern __shared__ __align__(16) uint8_t head_lds[];
  int tm, tn;
  gemm_tile_of(blockIdx.x, a.mt, a.nt, tm, tn);
  const int64_t m0 = (int64_t)tm * TL::BM;
  const int n0 = tn * TL::BN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4;
  constexpr int COLS = TL::NB * 16, LD = COLS + 4, LPR = COLS / 4, RPI = 64 / LPR;
  const int64_t mw = m0 + (wave / TL::WN) * TL::MB * 16;
  const int nw = n0 + (wave % TL::WN) * COLS;
  f32x4 acc[TL::MB][TL::NB];
#pragma unroll
  for (int m = 0; m < TL::MB; ++m)
#pragma unroll
    for (int n = 0; n < TL::NB; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  gemm_loop<TL, false, true, DIRECT>(a.h, a.w, m0, n0, 0, a.D, head_lds, acc);
  float* part = reinterpret_cast<float*>(head_lds) + wave * 16 * LD;
  static_for<0, TL::MB>([&](auto mc) {
    constexpr int m = decltype(mc)::value;
    const int64_t row = mw + 16 * m + (lane & 15);
    const float lse = row < a.M ? a.lse2[row] : __builtin_inff();
    const bool live = lse != __builtin_inff();  // a row that does not count has none
#pragma unroll
    for (int n = 0; n < TL::NB; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        acc[m][n][q] = live ? __builtin_amdgcn_exp2f(acc[m][n][q] * a.scale2 - lse) : 0.f;
    head_hits<DISTILL>(a, row, a.col0 + nw, COLS, [&](int c, int e) {
      if (((c >> 2) & 3) != g) return;
      const float w = DISTILL ? a.q[row * a.top + e] : 1.f;
#pragma unroll
      for (int n = 0; n < TL::NB; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[m][n][q] -= (c >> 4) == n && (c & 3) == q ? w : 0.f;
    });
#pragma unroll
    for (int n = 0; n < TL::NB; ++n)
      *reinterpret_cast<f32x4*>(part + (lane & 15) * LD + 16 * n + 4 * g) = acc[m][n];
    __builtin_amdgcn_wave_barrier();
    const int n = nw + 4 * (lane % LPR);
#pragma unroll 1
    for (int r = lane / LPR; r < 16; r += RPI) {
      const int64_t out = mw + 16 * m + r;
      if (out >= a.M || n >= a.V) continue;
      const f32x4 p = *reinterpret_cast<const f32x4*>(part + r * LD + 4 * (lane % LPR));
      uint16_t* d = a.P + out * a.ldp + n;  // ldp is a multiple of 8, at least V rounded up
      *reinterpret_cast<u32x2*>(d) = u32x2{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3])};
    }
    __builtin_amdgcn_wave_barrier();
  });
}

template <typename TL, bool DIRECT, bool DISTILL>
hipError_t launch_head_tile(bool prob, const HeadArgs& a, hipStream_t s) {
  constexpr int lds = gemm_lds_bytes<TL, false, true, DIRECT>();
  const auto k = prob ? head_prob_kernel<TL, DIRECT, DISTILL> : head_lse_kernel<TL, DIRECT, DISTILL>;
  int occ;
  const hipError_t e = kernel_occupancy(reinterpret_cast<const void*>(k), TL::NTHR, lds, &occ);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k, dim3((unsigned)(prob ? a.mt * a.nt : a.mt * a.runs)), dim3(TL::NTHR), lds, s, a);
  return hipGetLastError();
}

template <bool DISTILL>
hipError_t launch_head(bool prob, bool large, bool direct, const HeadArgs& a, hipStream_t s) {
  if (large)
    return direct ? launch_head_tile<GemmLarge, true, DISTILL>(prob, a, s) : launch_head_tile<GemmLarge, false, DISTILL>(prob, a, s);
  return direct ? launch_head_tile<GemmMedium, true, DISTILL>(prob, a, s) : launch_head_tile<GemmMedium, false, DISTILL>(prob, a, s);
}

}  // namespace ffmlp
