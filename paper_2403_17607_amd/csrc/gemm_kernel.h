// Matrix products of any size on the matrix cores, C = A B with bf16 operands
// and fp32 sums, as the wide layers and the vocabulary losses use them.
//
// The m side (rows of C) and the n side (columns of C) are each a row-major
// matrix, either with the contracted index k along its rows (T = false:
// [m][k], [n][k]) or across them (T = true: [k][m], [k][n]):
//     Y  = X W      X [m][k]  W [k][n]     m false, n true
//     dX = dZ W^T   dZ [m][k] W [n][k]     m false, n false
//     dW = X^T dZ   X [k][m]  dZ [k][n]    m true,  n true
// A workgroup owns a BM x BN tile of C and walks k in steps of BK.  Each step
// brings a BK slice of both sides to LDS as it lies in memory, without passing
// through registers (buffer_load ... lds); a side with k across its rows is
// transposed by the LDS read (ds_read_b64_tr_b16: 16 lanes read a 4 x 16 block
// and lane i gets its column i), so no operand is repacked.  The n side is the
// first MFMA operand: lane (i, g) of the result holds four consecutive columns
// 4 g .. 4 g + 3 of row i.
//
// LDS holds 16-byte pieces, [row][piece], the piece index XORed with a
// function of the row (below) so that the reads hit every bank once.
//
// Rows may start at any element: these loads take any address.  Measured per
// 64 KiB of 512-byte rows from L2: 0.62 us where rows start at a multiple of
// 4 bytes, 1.84 where none does, 1.22 where every second does.  What an
// unaligned or short row needs besides is the last step of k (Loader::fix).
#pragma once

#include "device.h"
#include "gemm.h"
#include "rows.h"

namespace ffmlp {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// One workgroup tile: BM x BN of C, WM x WN waves, BK of k per step, ST LDS
// buffers.
template <int BM_, int BN_, int BK_, int WM_, int WN_, int ST_>
struct GemmTile {
  static constexpr int BM = BM_, BN = BN_, BK = BK_, WM = WM_, WN = WN_, ST = ST_;
  static constexpr int NW = WM * WN, NTHR = NW * 64;
  static constexpr int MB = BM / WM / 16, NB = BN / WN / 16;  // 16 x 16 blocks of a wave
};

// One side's slice of a step: R rows or columns of C by BK of k.
template <bool T, int R, int BK, int NTHR>
struct Side {
  static constexpr int ROWS = T ? BK : R;        // rows of the slice in LDS
  static constexpr int CH = (T ? R : BK) / 8;    // 16-byte pieces of a row
  static constexpr int PIECES = ROWS * CH;
  static constexpr int PER = (PIECES + NTHR - 1) / NTHR;  // pieces a thread loads
  static constexpr int BYTES = PER * NTHR * 16;           // whole loads of the workgroup
  // Piece permutation of a row.  k along the rows: eight lanes read the same
  // piece of eight rows (128 bytes of banks).  k across: 16 lanes read 32
  // bytes of four rows, 32 lanes of rows r .. r + 3 and r + 8 .. r + 11.
  static __device__ __forceinline__ int swz(int row) {
    if constexpr (T) return (2 * ((row & 3) + 4 * ((row >> 3) & 1))) & (CH - 1);
    else if constexpr (CH >= 8) return row & 7;
    else return (row >> 1) & 3;
  }
};

// The global side of the loads of one thread, for a workgroup that owns the
// rows (T = false) or columns (T = true) from r0 on and contracts k0 .. kend - 1.
template <typename S, bool T, int BK, int NTHR>
struct Loader {
  SideArgs a;
  int64_t r0, kend;
  const uint8_t* p;       // the next step's first element,
  int64_t left;           // the bytes from it to the end of what may be read
  int krem;               // and the k from it on
  uint32_t voff[S::PER];  // byte offsets of the thread's pieces within a step

  static __device__ __forceinline__ int piece_row(int j, int tid) { return (j * NTHR + tid) / S::CH; }
  static __device__ __forceinline__ int piece_col(int j, int tid) {
    return 8 * (((j * NTHR + tid) % S::CH) ^ S::swz(piece_row(j, tid)));
  }
  static __device__ __forceinline__ bool piece_in(int j, int tid) {
    return S::PER * NTHR == S::PIECES || j * NTHR + tid < S::PIECES;
  }

  __device__ __forceinline__ void init(const SideArgs& args, int64_t first, int64_t k0, int64_t k1, int tid) {
    a = args;
    r0 = first;
    kend = k1;
    const int64_t row = T ? k0 : r0, col = T ? r0 : k0, last = T ? k1 - 1 : a.rows - 1;
    p = reinterpret_cast<const uint8_t*>(a.p + row * a.ld + col);
    left = ((last - row) * a.ld + a.cols - col) * 2;
    krem = (int)(k1 - k0);
#pragma unroll
    for (int j = 0; j < S::PER; ++j)
      voff[j] = piece_in(j, tid) ? (uint32_t)(((int64_t)piece_row(j, tid) * a.ld + piece_col(j, tid)) * 2) : kOOB;
  }
  // The next step to LDS at `lds`, piece by piece between begin and end.
  // Pieces that begin past kend or past the matrix are out of the descriptor's
  // range and arrive as zeros, so steps past the last one may be loaded too.
  // What follows a T side's row in memory (within the matrix) comes along in
  // its last tile: it only reaches columns of C that do not exist.
  u32x4 r;
  uint32_t dst;
  __device__ __forceinline__ void begin(uint32_t lds, int wave) {
    // (a buffer descriptor as make_rsrc builds it, in scalar registers)
    const uint64_t at = (uint64_t)p;
    const int64_t n = krem <= 0 || left <= 0 ? 0 : (left > 0x7fffffff ? 0x7fffffff : left);
    r = u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)n, 0x00020000u};
    dst = lds + (uint32_t)(wave * 64) * 16;
  }
  __device__ __forceinline__ void piece(int j, int tid) const {
    uint32_t o = voff[j];
    if (!T) o = piece_col(j, tid) < krem ? o : kOOB;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(dst + (uint32_t)(j * NTHR * 16)), "v"(o), "s"(r) : "memory");
  }
  __device__ __forceinline__ void end() {
    const int64_t step = T ? a.ld * (BK * 2) : BK * 2;
    p += step;
    left -= step;
    krem -= BK;
  }
  // Whether the step that ends with kend has pieces that are neither whole
  // nor empty: their rest would be of the next row (along k: nonzero), or they
  // end with the matrix, where the range check may drop the last element with
  // the dword it shares.
  __device__ __forceinline__ bool ragged() const {
    return T ? (a.cols & 7) != 0 && r0 + S::CH * 8 > a.cols : (kend & 7) != 0;
  }
  // That step's slice once more, exactly, through registers.
  __device__ __forceinline__ void fix(uint8_t* lds, int64_t k0, int tid) const {
    const int64_t rend = T ? kend : a.rows, cend = T ? a.cols : kend;
#pragma unroll 1
    for (int j = 0; j < S::PER; ++j) {
      const int64_t row = (T ? k0 : r0) + piece_row(j, tid), c = (T ? r0 : k0) + piece_col(j, tid);
      if (!piece_in(j, tid) || row >= rend || c >= cend || c + 8 <= cend) continue;
      const uint16_t* src = a.p + row * a.ld + c;
      uint32_t e[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) e[q] = c + q < cend ? (uint32_t)src[q] : 0u;
      *reinterpret_cast<u32x4*>(lds + (j * NTHR + tid) * 16) =
          u32x4{e[0] | (e[1] << 16), e[2] | (e[3] << 16), e[4] | (e[5] << 16), e[6] | (e[7] << 16)};
    }
  }
};

// A wave's operand fragments of one 32-wide block of k: block b holds rows
// (columns of C) w0 + 16 b + i, lane group g the positions 8 g .. 8 g + 7.
template <typename S, bool T, int NBLK>
struct Frags {
  uint32_t at[T ? NBLK : S::CH / 4];  // LDS byte offsets within the slice
  __device__ __forceinline__ void init(int w0, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (T) {
      const int row = 8 * g + (i >> 2), h = S::swz(row);
#pragma unroll
      for (int b = 0; b < NBLK; ++b) {
        const int piece = (w0 + 16 * b) / 8 + ((i & 3) >> 1);
        at[b] = (uint32_t)((row * S::CH + (piece ^ h)) * 16 + 8 * (i & 1));
      }
    } else {
      const int row = w0 + i;
#pragma unroll
      for (int kk = 0; kk < S::CH / 4; ++kk) at[kk] = (uint32_t)((row * S::CH + ((4 * kk + g) ^ S::swz(row))) * 16);
    }
  }
  // Block b of k-block kk; lds: the slice's first byte.
  __device__ __forceinline__ u32x4 read(const uint8_t* lds, int kk, int b) const {
    if constexpr (T) {
      typedef s16x4 __attribute__((address_space(3))) lds_s16x4;
      // rows + 4 keep swz(row) (it does not look at bit 2)
      const uint8_t* p = lds + at[b] + kk * 32 * S::CH * 16;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * S::CH * 16)));
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      return *reinterpret_cast<const u32x4*>(lds + at[kk] + b * 16 * S::CH * 16);
    }
  }
};

// Waits for all but the newest N of the wave's direct loads and for its LDS
// reads, then for the workgroup.
template <int N>
__device__ __forceinline__ void wait_loads_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

// acc += the BM x BN tile's products over k in [k0, k1), k0 a multiple of BK.
// `lds`: the workgroup's ST buffers of the two slices, free again when it
// returns.  The next loads are issued between the products of a step's first
// 32 k, a few at a time: issued together, they fill the memory queue and every
// wave waits there before its products (8192 x 4096 over 4096 of k, both sides'
// rows along k: 1215 TFLOP/s with the loads first, 1260 after the first reads,
// 1320 so; a library's product of this size 1110 to 1370).
template <typename TL, bool MT, bool NT>
__device__ __forceinline__ void gemm_loop(const SideArgs& ma, const SideArgs& na, int64_t m0, int64_t n0, int64_t k0,
                                          int64_t k1, uint8_t* lds, f32x4 (&acc)[TL::MB][TL::NB]) {
  typedef Side<MT, TL::BM, TL::BK, TL::NTHR> SM;
  typedef Side<NT, TL::BN, TL::BK, TL::NTHR> SN;
  constexpr int STAGE = SM::BYTES + SN::BYTES, LOADS = SM::PER + SN::PER;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / TL::WN, wn = wave % TL::WN;
  Loader<SM, MT, TL::BK, TL::NTHR> lm;
  Loader<SN, NT, TL::BK, TL::NTHR> ln;
  lm.init(ma, m0, k0, k1, tid);
  ln.init(na, n0, k0, k1, tid);
  Frags<SM, MT, TL::MB> fm;
  Frags<SN, NT, TL::NB> fn;
  fm.init(wm * TL::MB * 16, lane);
  fn.init(wn * TL::NB * 16, lane);
  const int nk = (int)((k1 - k0 + TL::BK - 1) / TL::BK);
  const uint32_t l0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
#pragma unroll
  for (int t = 0; t < TL::ST - 1; ++t) {
    lm.begin(l0 + t * STAGE, wave);
    ln.begin(l0 + t * STAGE + SM::BYTES, wave);
#pragma unroll
    for (int j = 0; j < SM::PER; ++j) lm.piece(j, tid);
#pragma unroll
    for (int j = 0; j < SN::PER; ++j) ln.piece(j, tid);
    lm.end();
    ln.end();
  }
  int slot = 0;
  for (int t = 0; t < nk; ++t) {
    wait_loads_barrier<(TL::ST - 2) * LOADS>();
    uint8_t* s = lds + slot * STAGE;
    if (t == nk - 1 && (lm.ragged() || ln.ragged())) {
      const int64_t k = k0 + (int64_t)t * TL::BK;
      lm.fix(s, k, tid);
      ln.fix(s + SM::BYTES, k, tid);
      __syncthreads();
    }
    // into the buffer of step t - 1, which every wave has read.  Steps past the
    // last load zeros, so that the count of loads in flight stays the same.
    const int next = slot == 0 ? TL::ST - 1 : slot - 1;
    lm.begin(l0 + next * STAGE, wave);
    ln.begin(l0 + next * STAGE + SM::BYTES, wave);
    static_for<0, TL::BK / 32>([&](auto kc) {
      constexpr int kk = decltype(kc)::value;
      u32x4 a[TL::MB], b[TL::NB];
#pragma unroll
      for (int n = 0; n < TL::NB; ++n) b[n] = fn.read(s + SM::BYTES, kk, n);
#pragma unroll
      for (int m = 0; m < TL::MB; ++m) a[m] = fm.read(s, kk, m);
      static_for<0, TL::MB>([&](auto mc) {
        constexpr int m = decltype(mc)::value;
#pragma unroll
        for (int n = 0; n < TL::NB; ++n) acc[m][n] = mfma16(b[n], a[m], acc[m][n]);
        constexpr int lo = LOADS * m / TL::MB, hi = LOADS * (m + 1) / TL::MB;
        if constexpr (kk == 0 && hi > lo) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int q = lo; q < hi; ++q) {
            if (q < SM::PER) lm.piece(q < SM::PER ? q : 0, tid);
            else ln.piece(q < SM::PER ? 0 : q - SM::PER, tid);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      });
    });
    lm.end();
    ln.end();
    slot = slot + 1 == TL::ST ? 0 : slot + 1;
  }
  wait_loads_barrier<0>();
}

// Results leave through LDS, ROWS = 16 G rows of a wave at a time in a part of
// its own, so that a wave's stores cover whole rows of its columns.  Row
// stride + 4 floats: eight lanes write eight rows' 16 bytes to different banks.
template <typename TL>
struct OutTile {
  static constexpr int G = TL::MB >= 2 ? 2 : 1, ROWS = 16 * G, COLS = TL::NB * 16, LD = COLS + 4;
  static constexpr int BYTES = TL::NW * ROWS * LD * 4;
};

template <typename TL, bool MT, bool NT>
constexpr int gemm_lds_bytes() {
  constexpr int loop = TL::ST * (Side<MT, TL::BM, TL::BK, TL::NTHR>::BYTES + Side<NT, TL::BN, TL::BK, TL::NTHR>::BYTES);
  return loop > OutTile<TL>::BYTES ? loop : OutTile<TL>::BYTES;
}

// f(r, p) for rows r of the wave's: p the lane's eight consecutive results of
// that row, columns 8 (lane % (COLS / 8)) on.  before(m): called before block m
// of acc is written.
template <typename TL, typename B, typename F>
__device__ __forceinline__ void out_rows(uint8_t* lds, f32x4 (&acc)[TL::MB][TL::NB], B&& before, F&& f) {
  typedef OutTile<TL> O;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float* part = reinterpret_cast<float*>(lds) + wave * O::ROWS * O::LD;
  constexpr int LPR = O::COLS / 8, RPI = 64 / LPR;
  static_for<0, TL::MB / O::G>([&](auto pc) {
    constexpr int ph = decltype(pc)::value;
    static_for<0, O::G>([&](auto gc) {
      constexpr int m = ph * O::G + decltype(gc)::value;
      before(std::integral_constant<int, m>{});
#pragma unroll
      for (int n = 0; n < TL::NB; ++n)
        *reinterpret_cast<f32x4*>(part + (16 * decltype(gc)::value + (lane & 15)) * O::LD + 16 * n + 4 * (lane >> 4)) = acc[m][n];
    });
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int r = lane / LPR; r < O::ROWS; r += RPI) f(ph * O::ROWS + r, part + r * O::LD + 8 * (lane % LPR));
    __builtin_amdgcn_wave_barrier();
  });
}

// The tile and the split of workgroup b of mt x nt tiles, `splits` each, in an
// order that keeps a chiplet's tiles together: the hardware deals workgroups out
// to the eight chiplets in turn, each with its own L2, so workgroup b takes item
// (b % 8) of eight equal runs.  A run stays within a split as far as it can (k is
// then shared by its tiles), and within the order, groups of eight tile rows
// share the n side's tiles.
__device__ __forceinline__ void gemm_tile_of(int b, int mt, int nt, int splits, int& tm, int& tn, int& split) {
  const int tiles = mt * nt, total = tiles * splits, q = total / 8, r = total % 8, x = b % 8, y = b / 8;
  int t = x * q + (x < r ? x : r) + y;
  split = t / tiles;
  t -= split * tiles;
  constexpr int G = 8;
  const int per = G * nt, grp = t / per, first = grp * G;
  const int rows = mt - first < G ? mt - first : G;
  const int in = t - grp * per;
  tm = first + in % rows;
  tn = in / rows;
}

// act(z) in y and act'(z) in d (which costs nothing where it is not used).  GELU is z Phi(z) with Phi from the rational
// approximation 7.1.26 of Abramowitz and Stegun (error of erf up to 1.5e-7),
// whose exponential the derivative needs too.
__device__ __forceinline__ void act_and_grad(int act, float z, float& y, float& d) {
  switch (act) {
    case ACT_RELU: y = z > 0.f ? z : (z != z ? z : 0.f); d = z > 0.f ? 1.f : 0.f; break;
    case ACT_SIGMOID: y = __builtin_amdgcn_rcpf(1.f + __expf(-z)); d = y * (1.f - y); break;
    case ACT_SINE: y = __sinf(z); d = __cosf(z); break;
    case ACT_GELU: {
      const float e = __expf(-0.5f * z * z), t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * 0.70710678f * __builtin_fabsf(z));
      const float q = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
      const float phi = z < 0.f ? q : 1.f - q;
      y = z * phi;
      d = phi + z * e * 0.39894228f;
      break;
    }
    case ACT_SILU: {
      const float p = __builtin_amdgcn_rcpf(1.f + __expf(-z));
      y = z * p;
      d = p + y * (1.f - p);
      break;
    }
    default: y = z; d = 1.f;
  }
}

// act(z) in place over eight values and, with GRAD, act'(z) in d.
template <bool GRAD>
__device__ __forceinline__ void act8(int act, float (&z)[8], float (&d)[8]) {
  const auto all = [&](auto kind) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      float y, g;
      act_and_grad(decltype(kind)::value, z[q], y, g);
      z[q] = y;
      if (GRAD) d[q] = g;
    }
  };
  switch (act) {
    case ACT_RELU: all(std::integral_constant<int, ACT_RELU>{}); break;
    case ACT_SIGMOID: all(std::integral_constant<int, ACT_SIGMOID>{}); break;
    case ACT_SINE: all(std::integral_constant<int, ACT_SINE>{}); break;
    case ACT_GELU: all(std::integral_constant<int, ACT_GELU>{}); break;
    case ACT_SILU: all(std::integral_constant<int, ACT_SILU>{}); break;
    default: all(std::integral_constant<int, ACT_LINEAR>{});
  }
}

// The bias of columns n .. n + 7 (zeros past N).
__device__ __forceinline__ void bias8(const GemmOut& o, int n, int N, float (&b)[8]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) b[q] = 0.f;
  if (o.bias && n < N) load8(o.bias + n, N - n, b);
}

// Columns n .. n + 7 of row m of a product's result (fewer where N ends), as `o`
// says: z the sums, b the bias of these columns.  Rows may start at any element;
// 16-byte accesses do (rows.h).
__device__ __forceinline__ void out8(const GemmOut& o, int64_t m, int n, int N, float (&z)[8], const float (&b)[8], float alpha) {
  const int left = N - n;
  float v[8];
  if (o.add) {
    load8(o.add + m * o.ldadd + n, left, v);
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] += v[q];
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) z[q] = z[q] * alpha + b[q];
  if (o.act != ACT_LINEAR) {
    float d[8];
    if (!o.stash) {
      act8<false>(o.act, z, d);
    } else {
      act8<true>(o.act, z, d);
      store8<true>(o.stash + m * (int64_t)N + n, left, d);
    }
  }
  if (o.R) {
    if (o.c_fp32) load8(static_cast<const float*>(o.R) + m * o.ldr + n, left, v);
    else load8(static_cast<const uint16_t*>(o.R) + m * o.ldr + n, left, v);
#pragma unroll
    for (int q = 0; q < 8; ++q) z[q] += v[q];
  }
  if (o.nt) {
    if (o.c_fp32) store8<true>(static_cast<float*>(o.C) + m * o.ldc + n, left, z);
    else store8<true>(static_cast<uint16_t*>(o.C) + m * o.ldc + n, left, z);
  } else {
    if (o.c_fp32) store8(static_cast<float*>(o.C) + m * o.ldc + n, left, z);
    else store8(static_cast<uint16_t*>(o.C) + m * o.ldc + n, left, z);
  }
}

// C = the product, or one split's share of it as fp32 partial sums.
template <typename TL, bool MT, bool NT>
__global__ __launch_bounds__(TL::NTHR, 2) void gemm_kernel(const GemmArgs a) {
  extern __shared__ __align__(16) uint8_t gemm_lds[];
  int tm, tn, split;
  gemm_tile_of(blockIdx.x, a.mt, a.nt, a.splits, tm, tn, split);
  const int64_t m0 = (int64_t)tm * TL::BM;
  const int n0 = tn * TL::BN;
  const int64_t k0 = split * a.kper, k1 = k0 + a.kper < a.K ? k0 + a.kper : a.K;
  f32x4 acc[TL::MB][TL::NB];
#pragma unroll
  for (int m = 0; m < TL::MB; ++m)
#pragma unroll
    for (int n = 0; n < TL::NB; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  gemm_loop<TL, MT, NT>(a.m, a.n, m0, n0, k0, k1, gemm_lds, acc);
  GemmOut o = a.out;
  if (a.splits > 1) {
    o = GemmOut{};
    o.C = a.partial + (int64_t)split * a.M * a.N;
    o.ldc = a.N;
    o.c_fp32 = 1;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int COLS = OutTile<TL>::COLS;
  const int64_t mw = m0 + (wave / TL::WN) * TL::MB * 16;
  const int nw = n0 + (wave % TL::WN) * COLS;
  const int n = nw + 8 * (lane % (COLS / 8));
  const float alpha = o.alpha ? *o.alpha : 1.f;
  float bias[8];
  bias8(o, n, a.N, bias);
  out_rows<TL>(gemm_lds, acc, [](auto) {}, [&](int r, const float* p) {
    if (mw + r >= a.M || n >= a.N) return;
    float z[8];
    lds8(p, z);
    out8(o, mw + r, n, a.N, z, bias, alpha);
  });
}

template <typename TL, bool MT, bool NT>
hipError_t launch_gemm_tile(GemmArgs a, hipStream_t s) {
  constexpr int lds = gemm_lds_bytes<TL, MT, NT>();
  const auto k = gemm_kernel<TL, MT, NT>;
  int occ;
  const hipError_t e = kernel_occupancy(reinterpret_cast<const void*>(k), TL::NTHR, lds, &occ);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k, dim3((unsigned)(a.mt * a.nt * a.splits)), dim3(TL::NTHR), lds, s, a);
  return hipGetLastError();
}

// Workgroup tiles.  GemmSquare: one workgroup per CU (128 KiB of LDS), fewest
// bytes per product, 128-byte rows of k.  The others: two per CU, so that one's
// epilogue hides behind the other's products.  gemm.hip chooses by what they cost.
// GemmMedium in eight waves: where tiles are few its waves wait for loads, and
// eight issue them sooner than four (1111 x 1283 over 771: 12.1 -> 10.1 us; of
// the larger tiles only those that are busy with products would lose by it).
typedef GemmTile<128, 256, 32, 2, 2, 3> GemmLarge;
typedef GemmTile<256, 256, 64, 2, 4, 2> GemmSquare;
typedef GemmTile<128, 128, 64, 2, 2, 2> GemmHalf;
typedef GemmTile<64, 128, 64, 2, 4, 3> GemmMedium;
typedef GemmTile<64, 64, 64, 2, 2, 3> GemmSmall;
typedef GemmTile<16, 128, 64, 1, 4, 4> GemmRows;

}  // namespace ffmlp
