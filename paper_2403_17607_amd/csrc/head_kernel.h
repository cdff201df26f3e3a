// Losses of the logits H W over a vocabulary, which are not stored themselves.
//
//   x = H W,  c = log2(e) / T                  (logits / T in base 2: x c)
//   m = max_v x,  ls = log2 sum_v 2^((x - m) c)
//   P = 2^((x - m) c - ls) - q                 (q: the target distribution)
//
// Products are subtracted before they are scaled: x c and m c themselves, at
// |x c| beyond 2^24, are rounded to whole numbers and more, and an exponent that
// is off by that much overflowed the fp16 below.
//
// head_lse_kernel walks a run of column tiles with one row tile and keeps the
// running maximum and sum of every row in registers; for the loss alone nothing
// else leaves it.  The gradients dH = P W^T and dW = H^T P take P as bf16, a piece
// of the vocabulary at a time.  For the first piece the same pass stores
// 2^((x - r) c + 15) as fp16, r the largest product of the row's columns in a
// wave's tile, and head_scale_kernel turns that into P in place once m and ls are
// known.  fp16 up to 2^15: half a step is 2^-11 of a value, or 2^-40 of the tile's
// largest, and P's own rounding to bf16 is 2^-8 of it, so a word outside the
// target distribution is rounded twice, the second time eight times as coarsely;
// in it, p is worked out again in fp32 from the word's product and p - q is rounded
// once, as everywhere in later pieces, whose products head_prob_kernel computes
// again.  q is sparse: the one target of a row, or the teacher's top entries
// sorted by index, with a table of where each block of 128 columns begins in a
// row's list.
//
// 8192 rows of 2048 over 65536 words: head_lse_kernel 2.1 ms (1050 TFLOP/s at
// 1.7 GHz, the matrix cores 54% busy: bound by power and by what feeds them),
// head_scale_kernel 0.44 ms (5.3 TB/s), the gradients' products 1.93 and 1.89 ms.
// Computing the logits again instead of the scaling pass would take 2.1 ms.
#pragma once

#include "gemm_kernel.h"
#include "head.h"
#include "lanes.h"

namespace ffmlp {

// f(column within the wave's columns, position in the row's list) for row
// `row`'s entries among `cols` columns from c0 on, c0 a multiple of 32.
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

// four results as fp16 (E), eight as bf16 (P)
__device__ __forceinline__ u32x2 pack4_f16(const f32x4& p) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  return u32x2{__builtin_bit_cast(uint32_t, f16x2{(_Float16)p[0], (_Float16)p[1]}),
               __builtin_bit_cast(uint32_t, f16x2{(_Float16)p[2], (_Float16)p[3]})};
}
__device__ __forceinline__ u32x4 pack8_bf16(const float* p) {
  return u32x4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
}

// A workgroup's row tile and run come in the products' order: a chiplet's 64
// workgroups have eight row tiles, which its L2 holds up to 2 KiB per row, and
// eight runs, which eight of them read together.  2047 rows of 1000 over 50021
// words take 251 us so and 308 with all runs of two row tiles on a chiplet.
template <typename TL, bool DISTILL>
__global__ __launch_bounds__(TL::NTHR, 2) void head_lse_kernel(const HeadArgs a) {
  extern __shared__ __align__(16) uint8_t head_lds[];
  int tm, run, one;
  gemm_tile_of(blockIdx.x, a.mt, a.runs, 1, tm, run, one);
  const int64_t m0 = (int64_t)tm * TL::BM;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int COLS = TL::NB * 16;
  const int64_t mw = m0 + (wave / TL::WN) * TL::MB * 16;
  float mx[TL::MB], sum[TL::MB];
#pragma unroll
  for (int m = 0; m < TL::MB; ++m) {
    mx[m] = -__builtin_inff();
    sum[m] = 0.f;
  }
  const int t1 = (run + 1) * a.per_run < a.nt ? (run + 1) * a.per_run : a.nt;
  for (int tn = run * a.per_run; tn < t1; ++tn) {
    const int n0 = tn * TL::BN, nw = n0 + (wave % TL::WN) * COLS;
    f32x4 acc[TL::MB][TL::NB];
#pragma unroll
    for (int m = 0; m < TL::MB; ++m)
#pragma unroll
      for (int n = 0; n < TL::NB; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    gemm_loop<TL, false, true>(a.h, a.w, m0, n0, 0, a.D, head_lds, acc);
    // Opaque copies: what follows from them is worked out here, per tile, and
    // not kept in registers across the products.
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int g = ln >> 4;
    const int64_t row0 = mw + (ln & 15);
    const bool keep = a.keep > n0;
    constexpr int LDE = COLS + 8;  // fp16: eight lanes write eight rows to different banks
    uint16_t* part = reinterpret_cast<uint16_t*>(head_lds) + wave * 16 * LDE;
    static_for<0, TL::MB>([&](auto mc) {
      constexpr int m = decltype(mc)::value;
      float top = -__builtin_inff();
#pragma unroll
      for (int n = 0; n < TL::NB; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (n0 + TL::BN > a.V) acc[m][n][q] = nw + 16 * n + 4 * g + q < a.V ? acc[m][n][q] : -__builtin_inff();
          top = __builtin_fmaxf(top, acc[m][n][q]);
        }
      // the four lane groups hold the same row
      top = lanes_max<64, 16>(top);
      head_hits<DISTILL>(a, row0 + 16 * m, nw, COLS, [&](int c, int e) {
        if (((c >> 2) & 3) != g) return;
        float x = 0.f;
#pragma unroll
        for (int n = 0; n < TL::NB; ++n)
#pragma unroll
          for (int q = 0; q < 4; ++q) x = (c >> 4) == n && (c & 3) == q ? acc[m][n][q] : x;
        a.pick[(row0 + 16 * m) * a.top + e] = x;
      });
      // a sum of 2^((x - top) c + 15), its largest term 2^15 exactly
      const float at = top == -__builtin_inff() ? 0.f : top;
      float s = 0.f;
#pragma unroll
      for (int n = 0; n < TL::NB; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          acc[m][n][q] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[m][n][q] - at, a.scale2, 15.f));
          s += acc[m][n][q];
        }
      head_merge(mx[m], sum[m], top, s, a.scale2);
      if (keep) {
        if (g == 0 && row0 + 16 * m < a.M) a.ref[(int64_t)(nw / COLS) * a.M + row0 + 16 * m] = top;
        constexpr int LPR = COLS / 8, RPI = 64 / LPR;
#pragma unroll
        for (int n = 0; n < TL::NB; ++n)
          *reinterpret_cast<u32x2*>(part + (ln & 15) * LDE + 16 * n + 4 * g) = pack4_f16(acc[m][n]);
        __builtin_amdgcn_wave_barrier();
        const int c = nw + 8 * (ln % LPR);
#pragma unroll
        for (int r = ln / LPR; r < 16; r += RPI) {
          const int64_t row = mw + 16 * m + r;
          if (c < a.keep && row < a.M)
            *reinterpret_cast<u32x4*>(a.P + row * a.ldp + c) = *reinterpret_cast<const u32x4*>(part + r * LDE + 8 * (ln % LPR));
        }
        __builtin_amdgcn_wave_barrier();
      }
    });
    if (keep) __syncthreads();  // the next tile's loads write where other waves read
  }
  const int g = lane >> 4;
  const int64_t row0 = mw + (lane & 15);
  f32x2* part = a.partial + (int64_t)(run * TL::WN + wave % TL::WN) * a.M;
#pragma unroll
  for (int m = 0; m < TL::MB; ++m) {
    // the lane groups' sums, the maximum being the same
    sum[m] = lanes_sum<64, 16>(sum[m]);
    if (g == 0 && row0 + 16 * m < a.M) part[row0 + 16 * m] = f32x2{mx[m], sum[m] * 0x1p-15f};
  }
}

// P of the columns a.col0 .. a.col0 + a.V - 1 (a.w begins at the first).
template <typename TL, bool DISTILL>
__global__ __launch_bounds__(TL::NTHR, 2) void head_prob_kernel(const HeadArgs a) {
  extern __shared__ __align__(16) uint8_t head_lds[];
  int tm, tn, one;
  gemm_tile_of(blockIdx.x, a.mt, a.nt, 1, tm, tn, one);
  const int64_t m0 = (int64_t)tm * TL::BM;
  const int n0 = tn * TL::BN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4;
  constexpr int COLS = TL::NB * 16;
  const int64_t mw = m0 + (wave / TL::WN) * TL::MB * 16, row0 = mw + (lane & 15);
  const int nw = n0 + (wave % TL::WN) * COLS;
  f32x4 acc[TL::MB][TL::NB];
#pragma unroll
  for (int m = 0; m < TL::MB; ++m)
#pragma unroll
    for (int n = 0; n < TL::NB; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  gemm_loop<TL, false, true>(a.h, a.w, m0, n0, 0, a.D, head_lds, acc);
  uint16_t* P = a.P + mw * a.ldp + nw + 8 * (lane % (COLS / 8));  // ldp: a multiple of 8, at least V
  const bool in = nw + 8 * (lane % (COLS / 8)) < a.V;
  out_rows<TL>(head_lds, acc, [&](auto mc) {
    constexpr int m = decltype(mc)::value;
    const int64_t row = row0 + 16 * m;
    RowLse lse = {0.f, __builtin_inff()};
    if (row < a.M) lse = RowLse{a.lse[row][0], a.lse[row][1]};
    const bool live = lse.live();  // a row that does not count has none
#pragma unroll
    for (int n = 0; n < TL::NB; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        acc[m][n][q] = live ? __builtin_amdgcn_exp2f(lse.log2_p(acc[m][n][q], a.scale2)) : 0.f;
    head_hits<DISTILL>(a, row, a.col0 + nw, COLS, [&](int c, int e) {
      if (((c >> 2) & 3) != g) return;
      const float w = DISTILL ? a.q[row * a.top + e] : 1.f;
#pragma unroll
      for (int n = 0; n < TL::NB; ++n)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[m][n][q] -= (c >> 4) == n && (c & 3) == q ? w : 0.f;
    });
  }, [&](int r, const float* p) {
    if (in && mw + r < a.M) *reinterpret_cast<u32x4*>(P + r * a.ldp) = pack8_bf16(p);
  });
}

// P of the first piece from what head_lse_kernel kept of it, in place; bound by
// memory (4096 rows of 32768, lists of 32: 120 us, 4.5 TB/s).  Wave
// w of block (x, y): row 4 x + w, columns `chunk` y on, 512 at a time; G: columns
// per reference.  Each wave merges its row's sums itself and those of y = 0 write
// the row's loss: one launch less.
template <bool DISTILL, int G>
__global__ __launch_bounds__(256) void head_scale_kernel(const HeadArgs a, const RowLossArgs rl) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.M) return;
  const int lane = threadIdx.x & 63;
  const RowLse lse = row_loss(rl, row, lane, blockIdx.y == 0);
  const bool live = lse.live();
  const int c1 = (int)(blockIdx.y + 1) * a.chunk < a.keep ? (int)(blockIdx.y + 1) * a.chunk : a.keep;
#pragma unroll 2
  for (int c0 = blockIdx.y * a.chunk; c0 < c1; c0 += 512) {
    const int c = c0 + 8 * lane;
    if (c >= c1) continue;
    uint16_t* p = a.P + row * a.ldp + c;
    const u32x4 u = *reinterpret_cast<const u32x4*>(p);
    const float f = live ? __builtin_amdgcn_exp2f(lse.log2_p(a.ref[(int64_t)(c / G) * a.M + row], a.scale2) - 15.f) : 0.f;
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float e = (float)__builtin_bit_cast(_Float16, (uint16_t)(u[q / 2] >> (16 * (q & 1))));
      v[q] = live ? e * f : 0.f;
    }
    // where q is taken off, p comes from the entry's product itself: with p near q
    // the fp16 rounding would be most of what is left
    head_hits<DISTILL>(a, row, c & ~(kHeadKey - 1), kHeadKey, [&](int at, int e) {
      const int k = at - (c & (kHeadKey - 1));
      if (k < 0 || k >= 8) return;
      const int64_t i = row * a.top + e;
      const float w = DISTILL ? a.q[i] : 1.f;
      const float p = live ? __builtin_amdgcn_exp2f(lse.log2_p(a.pick[i], a.scale2)) : 0.f;
      const bool again = DISTILL && e > 0 && a.index[i - 1] == a.index[i];  // equal indexes add up
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = k == q ? (again ? v[q] : p) - w : v[q];
    });
    *reinterpret_cast<u32x4*>(p) = pack8_bf16(v);
  }
}

// Few rows and a small vocabulary (the classes of a fused net): a workgroup
// makes all logits of 16 rows and is done with these rows in one pass: lse, loss
// and P.  Each of its eight waves has 128 columns and a ring of two slices of
// W, 32 of k, in LDS of its own, so no wave waits for another until all logits
// meet in LDS; H's rows are in registers.  Only M / 16 workgroups, and each reads
// all of W: hence few rows and columns.
constexpr int kRowsTile = 16, kRowsWaves = 8, kRowsVocab = 128 * kRowsWaves, kRowsDim = 256;

template <bool DISTILL>
__global__ __launch_bounds__(64 * kRowsWaves) void head_rows_kernel(const HeadArgs a, const RowLossArgs rl) {
  constexpr int BK = 32, NB = 8, LD = kRowsVocab + 4, ROWS = kRowsTile / kRowsWaves;
  typedef Side<true, 16 * NB, BK, 64> SW;
  __shared__ __align__(16) uint8_t lds[kRowsWaves * 2 * SW::BYTES];
  static_assert(sizeof(lds) >= kRowsTile * LD * 4, "the logits take the place of W's slices");
  float* logits = reinterpret_cast<float*>(lds);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t m0 = (int64_t)blockIdx.x * kRowsTile;
  const int nk = (int)((a.D + BK - 1) / BK), col0 = wave * 16 * NB;
  int64_t target[ROWS] = {};
  if constexpr (!DISTILL)
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if (m0 + r * kRowsWaves + wave < a.M) target[r] = a.target[m0 + r * kRowsWaves + wave];
  f32x4 acc[NB] = {};
  if (col0 < a.V) {
    uint8_t* own = lds + wave * 2 * SW::BYTES;
    const uint32_t l0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)own;
    Loader<SW, true, BK, 64> lw;
    lw.init(a.w, col0, 0, a.D, lane);
    const auto load = [&](int slot) {  // past D: zeros
      lw.begin(l0 + slot * SW::BYTES, 0);
#pragma unroll
      for (int j = 0; j < SW::PER; ++j) lw.piece(j, lane);
      lw.end();
    };
    u32x4 h[kRowsDim / BK];
    const int64_t row = m0 + (lane & 15);
    const uint16_t* hp = a.h.p + (row < a.M ? row : 0) * a.h.ld;
#pragma unroll
    for (int k = 0; k < kRowsDim / BK; ++k) {
      const int c = BK * k + 8 * (lane >> 4);
      h[k] = load8_bits(hp + c, row < a.M ? (int)a.D - c : 0);
    }
    load(0);
    load(1);
    // H has arrived before the first step, so no later one waits for it (which
    // would be for W's newer loads too)
#pragma unroll
    for (int k = 0; k < kRowsDim / BK; ++k) asm volatile("" : "+v"(h[k]));
    Frags<SW, true, NB> fw;
    fw.init(0, lane);
    static_for<0, kRowsDim / BK>([&](auto kc) {
      constexpr int k = decltype(kc)::value;
      if (k < nk) {
        uint8_t* s = own + (k & 1) * SW::BYTES;
        asm volatile("s_waitcnt vmcnt(%0)" :: "n"(SW::PER) : "memory");
        if (k == nk - 1 && lw.ragged()) {
          lw.fix(s, BK * k, lane);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[n] = mfma16(fw.read(s, 0, n), h[k], acc[n]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slice has been read
        load(k & 1);
      }
    });
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  if (col0 < a.V) {
    float* o = logits + (lane & 15) * LD + col0 + 4 * (lane >> 4);
#pragma unroll
    for (int n = 0; n < NB; ++n) *reinterpret_cast<f32x4*>(o + 16 * n) = acc[n];
  }
  __syncthreads();
  constexpr int J = kRowsVocab / 512;  // pieces of eight columns of a lane
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int64_t row = m0 + r * kRowsWaves + wave, t = target[r];
    if (row >= a.M) break;
    float* x = logits + (r * kRowsWaves + wave) * LD;
    float v[J][8], top = -__builtin_inff(), sum = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 512 * j + 8 * lane;
      lds8(x + c, v[j]);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        v[j][q] = c + q < a.V ? v[j][q] : -__builtin_inff();  // nothing was written past the last tile
        top = __builtin_fmaxf(top, v[j][q]);
      }
    }
    top = lanes_max<64>(top);
    const float at = top == -__builtin_inff() ? 0.f : top;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int q = 0; q < 8; ++q) sum += __builtin_amdgcn_exp2f((v[j][q] - at) * a.scale2);
    sum = lanes_sum<64>(sum);
    const RowLse lse = row_end(rl, row, lane, true, RowLse{top, __builtin_amdgcn_logf(sum)}, t, [&](int e) {
      return x[DISTILL ? a.index[row * a.top + e] : (int)t];
    });
    if (a.keep == 0) continue;
    const bool live = lse.live();  // a row that does not count has none
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int q = 0; q < 8; ++q) v[j][q] = live ? __builtin_amdgcn_exp2f(lse.log2_p(v[j][q], a.scale2)) : 0.f;
    if constexpr (DISTILL) {
      // through LDS: a lane takes a run of equal indexes
#pragma unroll
      for (int j = 0; j < J; ++j) {
        *reinterpret_cast<f32x4*>(x + 512 * j + 8 * lane) = f32x4{v[j][0], v[j][1], v[j][2], v[j][3]};
        *reinterpret_cast<f32x4*>(x + 512 * j + 8 * lane + 4) = f32x4{v[j][4], v[j][5], v[j][6], v[j][7]};
      }
      __builtin_amdgcn_wave_barrier();
      const int* index = a.index + row * a.top;
      for (int e = lane; e < a.top; e += 64) {
        const int c = index[e];
        if (c >= a.V || (e > 0 && index[e - 1] == c)) continue;  // absent ones are last
        float w = 0.f;
        for (int f = e; f < a.top && index[f] == c; ++f) w += a.q[row * a.top + f];
        x[c] -= w;
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < J; ++j) lds8(x + 512 * j + 8 * lane, v[j]);
    } else {
      if (t != a.ignore)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int q = 0; q < 8; ++q) v[j][q] -= t == 512 * j + 8 * lane + q ? 1.f : 0.f;
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 512 * j + 8 * lane;
      if (c < a.V) *reinterpret_cast<u32x4*>(a.P + row * a.ldp + c) = pack8_bf16(v[j]);
    }
  }
}

template <typename TL, bool DISTILL>
hipError_t launch_head_tile(HeadPass pass, const HeadArgs& a, const RowLossArgs& r, hipStream_t s) {
  if (pass == HEAD_SCALE) {
    hipLaunchKernelGGL((head_scale_kernel<DISTILL, TL::NB * 16>), dim3((unsigned)((a.M + 3) / 4), (unsigned)((a.keep + a.chunk - 1) / a.chunk)),
                       dim3(256), 0, s, a, r);
    return hipGetLastError();
  }
  if (pass == HEAD_ROWS) {
    hipLaunchKernelGGL(head_rows_kernel<DISTILL>, dim3((unsigned)((a.M + kRowsTile - 1) / kRowsTile)), dim3(64 * kRowsWaves), 0, s, a, r);
    return hipGetLastError();
  }
  constexpr int lds = gemm_lds_bytes<TL, false, true>();
  const auto k = pass == HEAD_PROB ? head_prob_kernel<TL, DISTILL> : head_lse_kernel<TL, DISTILL>;
  int occ;
  const hipError_t e = kernel_occupancy(reinterpret_cast<const void*>(k), TL::NTHR, lds, &occ);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k, dim3((unsigned)(pass == HEAD_PROB ? a.mt * a.nt : a.mt * a.runs)), dim3(TL::NTHR), lds, s, a);
  return hipGetLastError();
}

template <bool DISTILL>
hipError_t launch_head(HeadPass pass, bool large, const HeadArgs& a, const RowLossArgs& r, hipStream_t s) {
  return large ? launch_head_tile<GemmLarge, DISTILL>(pass, a, r, s) : launch_head_tile<GemmMedium, DISTILL>(pass, a, r, s);
}

}  // namespace ffmlp
