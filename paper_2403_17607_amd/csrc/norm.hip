// Layer norm of the rows of a matrix, forward and backward.
//
//   mean = sum x / N,  var = sum (x - mean)^2 / N,  r = 1 / sqrt(var + eps)
//   xh = (x - mean) r,  y = xh gamma + beta
//   u = dy gamma,  dx = r (u - sum u / N - xh sum (u xh) / N)
//   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
//
// Bound by memory: each element is read once and written once.  A row is held
// in registers by G lanes (8 .. 64 of a wave, or 256 .. 1024 threads), J pieces
// of eight elements each, so the variance is taken about the mean itself, as a
// second pass over registers.  Sums, statistics and gradients are fp32.
// Measured, forward and backward: 16384 x 2048 bf16 30 us (4.4 TB/s) and 39 us
// (5.2 TB/s, the rate of a large copy); 3001 x 5003 from fp32 23 us (3.9 TB/s)
// and 38 us (4.0 TB/s), twelve rows one after the other on every CU.
#include "gemm.h"
#include "lanes.h"
#include "rows.h"

namespace ffmlp {

namespace {

template <bool F32> struct Elem { typedef uint16_t type; };
template <> struct Elem<true> { typedef float type; };

// Sums of K values over the G consecutive threads that hold a row, in a fixed
// order: within a wave by lanes_sum, and through LDS (K floats per wave) where they
// are several waves, which all of the workgroup then passes together.
template <int G, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float* lds) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = lanes_sum<(G < 64 ? G : 64)>(v[k]);
  if constexpr (G > 64) {
    constexpr int W = G / 64;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    __syncthreads();  // the last sums have been read
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) lds[K * wave + k] = v[k];
    __syncthreads();
    const float* of = lds + K * (threadIdx.x / G * W + lane % W);
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lanes_sum<W>(of[k]);
  }
}

// Mean and 1 / std of a row in registers; pieces past N hold zeros.
template <int G, int J>
__device__ __forceinline__ void row_stats(const float (&x)[J][8], int lane, int N, float eps, float* lds, float& mean,
                                          float& rstd) {
  float s[1] = {0.f}, v[1] = {0.f};
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int q = 0; q < 8; ++q) s[0] += x[j][q];
  row_sum<G>(s, lds);
  mean = s[0] / (float)N;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int n = N - 8 * (j * G + lane);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float d = x[j][q] - mean;
      v[0] += q < n ? d * d : 0.f;
    }
  }
  row_sum<G>(v, lds);
  rstd = 1.f / __builtin_sqrtf(v[0] / (float)N + eps);
}

// How a row may end: with a whole piece (or, one row to a wave, an even
// element); one row to a wave and an odd bf16 element; several rows to a wave
// and a piece that would run on into the next one.
enum { END_WHOLE, END_ODD, END_SHARED };

// Rows go through buffer descriptors that begin at a wave's first row: a lane's
// offsets stay the same from row to row, and what lies past the last row is out
// of range (reads as zeros, is not stored), so no branch and no address
// arithmetic stands between the loads of a row.  The range check works on
// dwords, so the last element of a bf16 row that does not end with one is loaded
// and stored by itself.
template <bool F32, int G, int J, int END>
struct BufRows {
  static constexpr int SIZE = F32 ? 4 : 2;
  static constexpr bool LAST = END != END_WHOLE && !F32;
  const uint8_t* p;
  int64_t ld;
  uint32_t voff[J];
  uint32_t last;  // offset of the last element of the lane's row
  int n;          // END_SHARED (J = 1): elements of the lane's piece
  rsrc_t r;
  __device__ __forceinline__ void init(const void* base, int64_t stride, int N) {
    p = static_cast<const uint8_t*>(base);
    ld = stride;
    const int lane = threadIdx.x % G, grp = (threadIdx.x & 63) / G;  // grp: 0 where G >= 64
    last = (uint32_t)((grp * stride + N - 1) * SIZE);
    n = N - 8 * lane;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * (j * G + lane);
      voff[j] = c < N ? (uint32_t)((grp * stride + c) * SIZE) : kOOB;
    }
  }
  // `row`: the wave's first row, wave-uniform; rows M and past it do not exist.
  __device__ __forceinline__ void at(int64_t row, int64_t M, int N) {
    constexpr int ROWS = G < 64 ? 64 / G : 1;
    const int64_t left = M - row, rows = left < ROWS ? left : ROWS;
    r = make_rsrc(p + row * ld * SIZE, rows <= 0 ? 0 : ((rows - 1) * ld + N) * SIZE);
  }
  struct Raw {
    u32x4 x[F32 ? 2 : 1];
    uint32_t end[1];
  };
  __device__ __forceinline__ Raw load(int j) const {
    Raw v;
    v.x[0] = bload128(r, voff[j], 0);
    if constexpr (F32) v.x[1] = bload128(r, voff[j] + 16, 0);
    if constexpr (LAST) v.end[0] = bload16(r, last, 0);
    return v;
  }
  __device__ __forceinline__ void widen(int j, const Raw& v, float (&f)[8]) const {
    if constexpr (F32) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f[q] = __uint_as_float(v.x[0][q]);
        f[q + 4] = __uint_as_float(v.x[1][q]);
      }
    } else {
      widen8(v.x[0], f);
      if constexpr (LAST)
#pragma unroll
        for (int q = 0; q < 8; q += END == END_ODD ? 2 : 1)
          f[q] = voff[j] + 2 * q == last ? __uint_as_float(v.end[0] << 16) : f[q];
    }
    if constexpr (END == END_SHARED)
#pragma unroll
      for (int q = 0; q < 8; ++q) f[q] = q < n ? f[q] : 0.f;
  }
  __device__ __forceinline__ void store(int j, const float (&f)[8]) const {
    if constexpr (END == END_SHARED) {
      if (n < 8) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if constexpr (F32) bstore32<false>(__float_as_uint(f[q]), r, q < n ? voff[j] + 4 * q : kOOB, 0);
          else bstore16<false>(pack_bf16x2(f[q], 0.f), r, q < n ? voff[j] + 2 * q : kOOB, 0);
        }
        return;
      }
    }
    if constexpr (F32) {
      bstore128<false>(__builtin_bit_cast(u32x4, f32x4{f[0], f[1], f[2], f[3]}), r, voff[j], 0);
      bstore128<false>(__builtin_bit_cast(u32x4, f32x4{f[4], f[5], f[6], f[7]}), r, voff[j] + 16, 0);
    } else {
      const u32x4 u = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
      bstore128<false>(u, r, voff[j], 0);
      if constexpr (END == END_ODD) {
        uint32_t e = u[0];
#pragma unroll
        for (int q = 1; q < 4; ++q) e = voff[j] + 4 * q == last ? u[q] : e;
        bstore16<false>(e, r, last - voff[j] < 16 ? last : kOOB, 0);
      }
    }
  }
};
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
// gamma (ones where it is NULL) or beta (zeros) in LDS, zeros past N.
__device__ __forceinline__ void fill_columns(float* dst, int cols, const float* src, int N, float missing) {
  for (int c = threadIdx.x; c < cols; c += blockDim.x) dst[c] = c < N ? (src ? src[c] : missing) : 0.f;
}
}  // namespace

// Threads of a forward workgroup.
template <int G> constexpr int norm_fwd_threads() { return G > 256 ? G : 256; }

template <int G, int J, int END, bool X32, bool Y32>
__global__ __launch_bounds__(norm_fwd_threads<G>()) void norm_fwd_buf_kernel(const NormArgs a) {
  __shared__ float lds[32];
  const int lane = threadIdx.x % G;
  constexpr int PER = norm_fwd_threads<G>() / G, WPR = G < 64 ? 64 / G : 1;  // rows of a workgroup, of a wave
  BufRows<X32, G, J, END> X;
  BufRows<Y32, G, J, END> Y;
  X.init(a.X, a.ldx, a.N);
  Y.init(a.Y, a.ldy, a.N);
  const rsrc_t rg = make_rsrc(a.gamma, a.gamma ? (int64_t)a.N * 4 : 0), rb = make_rsrc(a.beta, a.beta ? (int64_t)a.N * 4 : 0);
  const int wave_row = G <= 64 ? (int)(threadIdx.x >> 6) * WPR : 0;
  for (int64_t first = (int64_t)blockIdx.x * PER; first < a.M; first += (int64_t)gridDim.x * PER) {
    const int64_t row0 = uniform(first + wave_row), row = row0 + (threadIdx.x & 63) / G;
    X.at(row0, a.M, a.N);
    Y.at(row0, a.M, a.N);
    typename BufRows<X32, G, J, END>::Raw raw[J];
#pragma unroll
    for (int j = 0; j < J; ++j) raw[j] = X.load(j);
    float g[J][8], b[J][8], x[J][8];
#pragma unroll
    for (int j = 0; j < J; ++j) {  // in flight with the row
      const uint32_t c = 32 * (j * G + lane);
      *reinterpret_cast<u32x4*>(&g[j][0]) = bload128(rg, c, 0);
      *reinterpret_cast<u32x4*>(&g[j][4]) = bload128(rg, c + 16, 0);
      *reinterpret_cast<u32x4*>(&b[j][0]) = bload128(rb, c, 0);
      *reinterpret_cast<u32x4*>(&b[j][4]) = bload128(rb, c + 16, 0);
    }
#pragma unroll
    for (int j = 0; j < J; ++j) X.widen(j, raw[j], x[j]);
    float mean, rstd;
    row_stats<G, J>(x, lane, a.N, a.eps, lds, mean, rstd);
    if (a.stats && lane == 0 && row < a.M) *reinterpret_cast<f32x2*>(a.stats + 2 * row) = f32x2{mean, rstd};
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float y[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        y[q] = (x[j][q] - mean) * rstd * (a.gamma ? g[j][q] : 1.f) + b[j][q];  // no beta reads as zeros
      }
      Y.store(j, y);
    }
  }
}

// Threads of a backward workgroup, as many as its registers allow: they share
// one part of the sums for dgamma and dbeta.
template <int G, int J> constexpr int norm_bwd_threads() { return G == 64 && J == 2 ? 768 : 1024; }

// A workgroup's sums for dgamma and dbeta as one part: those of its waves (or
// of its groups of several waves) added in a fixed order.
template <int G, int J>
__device__ __forceinline__ void write_part(const NormArgs& a, float (&dg)[J][8], float (&db)[J][8], float* sums) {
  constexpr int UNIT = G < 64 ? 64 : G, UNITS = norm_bwd_threads<G, J>() / UNIT;
  const int lane = threadIdx.x % G, unit = threadIdx.x / UNIT;
  float* part = a.partial + (int64_t)blockIdx.x * 2 * a.N;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float(&v)[J][8] = w ? db : dg;
    if constexpr (UNITS > 1) {
#pragma unroll
      for (int m = G; m < 64; m *= 2)  // the groups of a wave
#pragma unroll
        for (int q = 0; q < 8; ++q) v[0][q] += __shfl_xor(v[0][q], m);
      for (int k = UNITS - 1; k >= 0; --k) {  // the last one first, the first adds and writes
        __syncthreads();
        if (unit == k && threadIdx.x % UNIT < G) {
#pragma unroll
          for (int j = 0; j < J; ++j)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              float& s = sums[8 * (j * G + lane) + q];
              v[j][q] += k == UNITS - 1 ? 0.f : s;
              s = v[j][q];
            }
        }
      }
      __syncthreads();
    }
    if (threadIdx.x < G)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int c = 8 * (j * G + lane);
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (c + q < a.N) part[(int64_t)w * a.N + c + q] = v[j][q];
      }
  }
}

// What a piece adds to the sums: of its row (s1 = sum u, s2 = sum u xh) and of
// its columns.  Past N dy is 0, and so is what it adds to a row's sums; the
// columns' own sums there are not written.
__device__ __forceinline__ void bwd_sums(const float (&x)[8], const float (&d)[8], const float (&g)[8], const f32x2& st, float (&dg)[8],
                                         float (&db)[8], float& s1, float& s2) {
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const float xh = (x[q] - st[0]) * st[1], u = d[q] * g[q];
    dg[q] += d[q] * xh;
    db[q] += d[q];
    s1 += u;
    s2 += u * xh;
  }
}
__device__ __forceinline__ void bwd_dx(const float (&x)[8], float (&d)[8], const float (&g)[8], const f32x2& st, float s1, float s2) {
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const float xh = (x[q] - st[0]) * st[1];
    d[q] = st[1] * (d[q] * g[q] - s1 - xh * s2);
  }
}

// Each group of G lanes takes rows blockIdx + k gridDim ... of its own and
// keeps the sums for dgamma and dbeta of its columns in registers, gamma being
// in LDS.  bf16 pieces stay packed until they are used; where registers allow,
// a group asks for its next rows (AHEAD of them) before it works on the current one.
template <int G, int J, int END, bool X32, bool DY32, bool DX32>
__global__ __launch_bounds__((norm_bwd_threads<G, J>())) void norm_bwd_buf_kernel(const NormArgs a) {
  constexpr int NTHR = norm_bwd_threads<G, J>(), PER = NTHR / G, COLS = 8 * J * G, WPR = G < 64 ? 64 / G : 1;
  constexpr int AHEAD = J == 1 ? 2 : J == 2 && G <= 64 && !X32 && !DY32 ? 1 : 0, BUFS = AHEAD ? AHEAD : 1;
  __shared__ float lds[32];
  __shared__ __align__(16) float gamma[COLS];
  __shared__ float sums[PER > 1 ? COLS : 1];
  const int lane = threadIdx.x % G;
  fill_columns(gamma, COLS, a.gamma, a.N, 1.f);
  __syncthreads();
  BufRows<X32, G, J, END> X;
  BufRows<DY32, G, J, END> D;
  BufRows<DX32, G, J, END> O;
  X.init(a.X, a.ldx, a.N);
  D.init(a.dY, a.lddy, a.N);
  O.init(a.dX, a.lddx, a.N);
  float dg[J][8] = {}, db[J][8] = {};
  struct Row {
    typename BufRows<X32, G, J, END>::Raw x[J];
    typename BufRows<DY32, G, J, END>::Raw d[J];
    f32x2 st;
  } next[BUFS];
  const int wave_row = G <= 64 ? (int)(threadIdx.x >> 6) * WPR : threadIdx.x / G, in_wave = G < 64 ? (threadIdx.x & 63) / G : 0;
  const auto fetch = [&](Row& to, int64_t row0) {
    X.at(row0, a.M, a.N);
    D.at(row0, a.M, a.N);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      to.x[j] = X.load(j);
      to.d[j] = D.load(j);
    }
    const int64_t row = row0 + in_wave;
    to.st = *reinterpret_cast<const f32x2*>(a.stats + 2 * (row < a.M ? row : a.M - 1));
  };
  const int64_t step = (int64_t)gridDim.x * PER;
  int64_t first = (int64_t)blockIdx.x * PER;
  static_for<0, AHEAD>([&](auto b) { fetch(next[decltype(b)::value], uniform(first + decltype(b)::value * step + wave_row)); });
  while (first < a.M) {
    static_for<0, BUFS>([&](auto b) {
      if (first >= a.M) return;
      Row& buf = next[decltype(b)::value];
      const int64_t row0 = uniform(first + wave_row);
      if (!AHEAD) fetch(buf, row0);
      const Row now = buf;
      if (AHEAD) fetch(buf, uniform(first + AHEAD * step + wave_row));
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float g[8], x[8], d[8];
        lds8(gamma + 8 * (j * G + lane), g);
        X.widen(j, now.x[j], x);
        D.widen(j, now.d[j], d);
        bwd_sums(x, d, g, now.st, dg[j], db[j], s[0], s[1]);
      }
      row_sum<G>(s, lds);
      s[0] /= (float)a.N;
      s[1] /= (float)a.N;
      O.at(row0, a.M, a.N);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float g[8], x[8], d[8];
        lds8(gamma + 8 * (j * G + lane), g);
        X.widen(j, now.x[j], x);
        D.widen(j, now.d[j], d);
        bwd_dx(x, d, g, now.st, s[0], s[1]);
        O.store(j, d);
      }
      first += step;
    });
  }
  write_part<G, J>(a, dg, db, sums);
}

// ---- rows that do not fit the registers of a workgroup: three passes over a
// row (two in the backward pass), which the caches hold in between.
template <bool X32, bool Y32>
__global__ __launch_bounds__(256) void norm_fwd_long_kernel(const NormArgs a) {
  typedef typename Elem<X32>::type TX;
  typedef typename Elem<Y32>::type TY;
  __shared__ float lds[8];
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    const TX* X = static_cast<const TX*>(a.X) + row * a.ldx;
    TY* Y = static_cast<TY*>(a.Y) + row * a.ldy;
    float s[1] = {0.f}, v[1] = {0.f}, x[8];
    for (int c = 8 * threadIdx.x; c < a.N; c += 2048) {
      load8(X + c, a.N - c, x);
      float t = 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) t += x[q];
      s[0] += t;
    }
    row_sum<256>(s, lds);
    const float mean = s[0] / (float)a.N;
    for (int c = 8 * threadIdx.x; c < a.N; c += 2048) {
      load8(X + c, a.N - c, x);
      float t = 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) t += c + q < a.N ? (x[q] - mean) * (x[q] - mean) : 0.f;
      v[0] += t;
    }
    row_sum<256>(v, lds);
    const float rstd = 1.f / __builtin_sqrtf(v[0] / (float)a.N + a.eps);
    if (a.stats && threadIdx.x == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * row) = f32x2{mean, rstd};
    for (int c = 8 * threadIdx.x; c < a.N; c += 2048) {
      const int n = a.N - c;
      float g[8], b[8];
      load8(X + c, n, x);
      if (a.gamma) load8(a.gamma + c, n, g);
      if (a.beta) load8(a.beta + c, n, b);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        x[q] = (x[q] - mean) * rstd;
        if (a.gamma) x[q] *= g[q];
        if (a.beta) x[q] += b[q];
      }
      store8(Y + c, n, x);
    }
  }
}

template <bool X32, bool DY32>
__global__ __launch_bounds__(256) void norm_bwd_long_kernel(const NormArgs a) {
  typedef typename Elem<X32>::type TX;
  typedef typename Elem<DY32>::type TD;
  __shared__ float lds[8];
  for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
    const TX* X = static_cast<const TX*>(a.X) + row * a.ldx;
    const TD* D = static_cast<const TD*>(a.dY) + row * a.lddy;
    const f32x2 st = *reinterpret_cast<const f32x2*>(a.stats + 2 * row);
    float s[2] = {0.f, 0.f}, x[8], d[8], g[8];
    auto load = [&](int c) {
      const int n = a.N - c;
      load8(X + c, n, x);
      load8(D + c, n, d);
      if (a.gamma) load8(a.gamma + c, n, g);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        x[q] = q < n ? (x[q] - st[0]) * st[1] : 0.f;
        if (a.gamma) d[q] *= g[q];
      }
    };
    for (int c = 8 * threadIdx.x; c < a.N; c += 2048) {
      load(c);
      float t1 = 0.f, t2 = 0.f;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        t1 += d[q];
        t2 += d[q] * x[q];
      }
      s[0] += t1;
      s[1] += t2;
    }
    row_sum<256>(s, lds);
    s[0] /= (float)a.N;
    s[1] /= (float)a.N;
    for (int c = 8 * threadIdx.x; c < a.N; c += 2048) {
      load(c);
#pragma unroll
      for (int q = 0; q < 8; ++q) d[q] = st[1] * (d[q] - s[0] - x[q] * s[1]);
      if (a.dx_fp32) store8(static_cast<float*>(a.dX) + row * a.lddx + c, a.N - c, d);
      else store8(static_cast<uint16_t*>(a.dX) + row * a.lddx + c, a.N - c, d);
    }
  }
}

// dgamma and dbeta of such rows: block (x, y) sums columns 512 x + 8 lane ..
// over the rows of part y.
template <bool X32, bool DY32>
__global__ __launch_bounds__(256) void norm_cols_long_kernel(const NormArgs a) {
  typedef typename Elem<X32>::type TX;
  typedef typename Elem<DY32>::type TD;
  __shared__ float sums[3][2][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.x * 512 + lane * 8, n = a.N - c;
  const int64_t per = (a.M + a.parts - 1) / a.parts;
  const int64_t r0 = per * blockIdx.y, r1 = r0 + per < a.M ? r0 + per : a.M;
  float v[2][8] = {};
  if (n > 0)
    for (int64_t r = r0 + wave; r < r1; r += 4) {
      float x[8], d[8];
      load8(static_cast<const TX*>(a.X) + r * a.ldx + c, n, x);
      load8(static_cast<const TD*>(a.dY) + r * a.lddy + c, n, d);
      const f32x2 st = *reinterpret_cast<const f32x2*>(a.stats + 2 * r);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        v[0][q] += q < n ? d[q] * ((x[q] - st[0]) * st[1]) : 0.f;
        v[1][q] += d[q];
      }
    }
  if (wave)
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      sums[wave - 1][0][lane * 8 + q] = v[0][q];
      sums[wave - 1][1][lane * 8 + q] = v[1][q];
    }
  __syncthreads();
  if (wave == 0)
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (q < n)
          a.partial[((int64_t)blockIdx.y * 2 + w) * a.N + c + q] =
              ((v[w][q] + sums[0][w][lane * 8 + q]) + sums[1][w][lane * 8 + q]) + sums[2][w][lane * 8 + q];
}

namespace {

// Workgroups of a pass over rows: a launch has fewer than 2^32 threads, whatever a
// workgroup's are (1024 at most); the kernels go on to further rows by themselves.
unsigned norm_grid(int64_t blocks) { return (unsigned)(blocks < (1 << 21) ? blocks : 1 << 21); }

template <typename F>
hipError_t by_types(bool a32, bool b32, F&& f) {
  if (a32) return b32 ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
  return b32 ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

// f(G, J): the lanes and pieces that hold a row of N; false if none do.  The
// backward pass spreads long rows over more lanes, for its two sums per column.
#define FFMLP_ROW(G, J) \
  if (N <= 8 * G * J) { f(std::integral_constant<int, G>{}, std::integral_constant<int, J>{}); return true; }
template <typename F>
bool by_row_forward(int N, F&& f) {
  FFMLP_ROW(8, 1) FFMLP_ROW(16, 1) FFMLP_ROW(32, 1) FFMLP_ROW(64, 1) FFMLP_ROW(64, 2) FFMLP_ROW(256, 1)
  FFMLP_ROW(512, 1) FFMLP_ROW(512, 2) FFMLP_ROW(512, 4)
  return false;
}
template <typename F>
bool by_row_backward(int N, F&& f) {
  FFMLP_ROW(8, 1) FFMLP_ROW(16, 1) FFMLP_ROW(32, 1) FFMLP_ROW(64, 1) FFMLP_ROW(64, 2) FFMLP_ROW(256, 1)
  FFMLP_ROW(512, 1) FFMLP_ROW(1024, 1) FFMLP_ROW(1024, 2)
  return false;
}
#undef FFMLP_ROW

}  // namespace

int norm_parts(int64_t M, int N) {
  int rows = 16;  // that a workgroup takes at a time
  by_row_backward(N, [&](auto g, auto j) {
    constexpr int G = decltype(g)::value;
    rows = norm_bwd_threads<G, decltype(j)::value>() / G;
  });
  const int64_t p = (M + rows - 1) / rows;
  return (int)(p < 1 ? 1 : p < 256 ? p : 256);  // one workgroup per CU
}

hipError_t launch_norm_forward(const NormArgs& a, hipStream_t s) {
  return by_types(a.x_fp32, a.y_fp32, [&](auto x32, auto y32) {
    constexpr bool X = decltype(x32)::value, Y = decltype(y32)::value;
    const bool held = by_row_forward(a.N, [&](auto g, auto j) {
      constexpr int G = decltype(g)::value, J = decltype(j)::value, T = norm_fwd_threads<G>(), R = T / G;
      const dim3 grid(norm_grid((a.M + R - 1) / R));
      constexpr int OTHER = G < 64 ? END_SHARED : END_ODD;
      if (a.N % (G < 64 ? 8 : 2) == 0) hipLaunchKernelGGL((norm_fwd_buf_kernel<G, J, END_WHOLE, X, Y>), grid, dim3(T), 0, s, a);
      else hipLaunchKernelGGL((norm_fwd_buf_kernel<G, J, OTHER, X, Y>), grid, dim3(T), 0, s, a);
    });
    if (!held) hipLaunchKernelGGL((norm_fwd_long_kernel<X, Y>), dim3(norm_grid(a.M)), dim3(256), 0, s, a);
    return hipGetLastError();
  });
}

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s) {
  const hipError_t e = by_types(a.x_fp32, a.dy_fp32, [&](auto x32, auto d32) {
    constexpr bool X = decltype(x32)::value, D = decltype(d32)::value;
    const bool held = by_row_backward(a.N, [&](auto g, auto j) {
      constexpr int G = decltype(g)::value, J = decltype(j)::value;
      const dim3 grid((unsigned)a.parts), block(norm_bwd_threads<G, J>());
      constexpr int OTHER = G < 64 ? END_SHARED : END_ODD;
      const auto run = [&](auto o32) {
        constexpr bool O = decltype(o32)::value;
        if (a.N % (G < 64 ? 8 : 2) == 0) hipLaunchKernelGGL((norm_bwd_buf_kernel<G, J, END_WHOLE, X, D, O>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((norm_bwd_buf_kernel<G, J, OTHER, X, D, O>), grid, block, 0, s, a);
      };
      if (a.dx_fp32) run(std::true_type{});
      else run(std::false_type{});
    });
    if (!held) {  // the columns first: dX may be dY
      hipLaunchKernelGGL((norm_cols_long_kernel<X, D>), dim3((unsigned)((a.N + 511) / 512), (unsigned)a.parts), dim3(256), 0, s, a);
      const hipError_t le = hipGetLastError();
      if (le != hipSuccess) return le;
      hipLaunchKernelGGL((norm_bwd_long_kernel<X, D>), dim3(norm_grid(a.M)), dim3(256), 0, s, a);
    }
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  return launch_column_reduce(a.partial, a.parts, a.N, a.dgamma, a.dbeta, s);
}

}  // namespace ffmlp
