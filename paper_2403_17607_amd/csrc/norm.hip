// Layer norm of the rows of a matrix, forward and backward.
//
//   mean = sum x / N,  var = sum (x - mean)^2 / N,  r = 1 / sqrt(var + eps)
//   xh = (x - mean) r,  y = xh gamma + beta
//   u = dy gamma,  dx = r (u - sum u / N - xh sum (u xh) / N)
//   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
//
// Bound by memory: each element is read once and written once.  A row is held
// in registers by G lanes (8 .. 64, or the 256 threads of a workgroup), J
// pieces of eight elements each, so the variance is taken about the mean
// itself, as a second pass over registers.  Sums, statistics and gradients
// are fp32.
#include "gemm.h"
#include "rows.h"

namespace ffmlp {

namespace {

constexpr int kNormParts = 256;  // one workgroup per CU in the backward pass

template <bool F32> struct Elem { typedef uint16_t type; };
template <> struct Elem<true> { typedef float type; };

// Sum over the G lanes (aligned groups of a wave) that hold a row, or over
// the workgroup (G = 256; `lds` has 8 floats, two per wave in turn).
template <int G>
__device__ __forceinline__ void row_sum2(float& a, float& b, float* lds) {
#pragma unroll
  for (int m = 1; m < (G < 64 ? G : 64); m *= 2) {
    a += __shfl_xor(a, m);
    b += __shfl_xor(b, m);
  }
  if constexpr (G == 256) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();  // the last sums have been read
    if ((threadIdx.x & 63) == 0) {
      lds[2 * wave] = a;
      lds[2 * wave + 1] = b;
    }
    __syncthreads();
    a = (lds[0] + lds[2]) + (lds[4] + lds[6]);
    b = (lds[1] + lds[3]) + (lds[5] + lds[7]);
  }
}

// Mean and 1 / std of a row in registers; pieces past N hold zeros.
template <int G, int J>
__device__ __forceinline__ void row_stats(const float (&x)[J][8], int lane, int N, float eps, float* lds, float& mean,
                                          float& rstd) {
  float s = 0.f, z = 0.f;
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int q = 0; q < 8; ++q) s += x[j][q];
  row_sum2<G>(s, z, lds);
  mean = s / (float)N;
  float v = 0.f;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int n = N - 8 * (j * G + lane);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float d = x[j][q] - mean;
      v += q < n ? d * d : 0.f;
    }
  }
  row_sum2<G>(v, z, lds);
  rstd = 1.f / __builtin_sqrtf(v / (float)N + eps);
}

}  // namespace

template <int G, int J, bool X32, bool Y32>
__global__ __launch_bounds__(256) void norm_fwd_kernel(const NormArgs a) {
  typedef typename Elem<X32>::type TX;
  typedef typename Elem<Y32>::type TY;
  __shared__ float lds[8];
  const int lane = threadIdx.x % G;
  // groups of lanes, or the whole workgroup, take rows of their own
  for (int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G; row < a.M; row += (int64_t)gridDim.x * (256 / G)) {
  const TX* X = static_cast<const TX*>(a.X) + row * a.ldx;
  float x[J][8];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = 8 * (j * G + lane);
    load8(X + c, a.N - c, x[j]);
  }
  float mean, rstd;
  row_stats<G, J>(x, lane, a.N, a.eps, lds, mean, rstd);
  if (a.stats && lane == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * row) = f32x2{mean, rstd};
  TY* Y = static_cast<TY*>(a.Y) + row * a.ldy;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = 8 * (j * G + lane), n = a.N - c;
    if (n <= 0) continue;
    float g[8], b[8], y[8];
    if (a.gamma) load8(a.gamma + c, n, g);
    if (a.beta) load8(a.beta + c, n, b);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      y[q] = (x[j][q] - mean) * rstd;
      if (a.gamma) y[q] *= g[q];
      if (a.beta) y[q] += b[q];
    }
    store8(Y + c, n, y);
  }
  }
}

// Each group of G lanes takes rows blockIdx + k gridDim ... of its own and
// keeps the sums for dgamma and dbeta of its columns in registers; at the end
// the workgroup's groups are added in a fixed order and written as one part.
template <int G, int J, bool X32, bool DY32>
__global__ __launch_bounds__(256) void norm_bwd_kernel(const NormArgs a) {
  typedef typename Elem<X32>::type TX;
  typedef typename Elem<DY32>::type TD;
  constexpr int GROUPS = 256 / G, COLS = 8 * J * G;
  __shared__ float lds[8];
  __shared__ float sums[GROUPS > 1 ? COLS : 1];
  const int lane = threadIdx.x % G, grp = threadIdx.x / G;
  float dg[J][8] = {}, db[J][8] = {};
  for (int64_t row = (int64_t)blockIdx.x * GROUPS + grp; row < a.M; row += (int64_t)gridDim.x * GROUPS) {
    const TX* X = static_cast<const TX*>(a.X) + row * a.ldx;
    const TD* D = static_cast<const TD*>(a.dY) + row * a.lddy;
    float x[J][8], d[J][8];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * (j * G + lane);
      load8(X + c, a.N - c, x[j]);
      load8(D + c, a.N - c, d[j]);
    }
    const f32x2 st = *reinterpret_cast<const f32x2*>(a.stats + 2 * row);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * (j * G + lane), n = a.N - c;
      float g[8];
      if (a.gamma && n > 0) load8(a.gamma + c, n, g);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float xh = (x[j][q] - st[0]) * st[1];
        dg[j][q] += q < n ? d[j][q] * xh : 0.f;
        db[j][q] += d[j][q];
        const float u = a.gamma ? (q < n ? d[j][q] * g[q] : 0.f) : d[j][q];
        x[j][q] = xh;
        d[j][q] = u;
        s1 += u;
        s2 += q < n ? u * xh : 0.f;
      }
    }
    row_sum2<G>(s1, s2, lds);
    s1 /= (float)a.N;
    s2 /= (float)a.N;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int c = 8 * (j * G + lane), n = a.N - c;
      if (n <= 0) continue;
#pragma unroll
      for (int q = 0; q < 8; ++q) d[j][q] = st[1] * (d[j][q] - s1 - x[j][q] * s2);
      if (a.dx_fp32) store8(static_cast<float*>(a.dX) + row * a.lddx + c, n, d[j]);
      else store8(static_cast<uint16_t*>(a.dX) + row * a.lddx + c, n, d[j]);
    }
  }
  float* part = a.partial + (int64_t)blockIdx.x * 2 * a.N;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float(&v)[J][8] = w ? db : dg;
    if constexpr (GROUPS > 1) {
      for (int k = GROUPS - 1; k >= 0; --k) {  // the last group first, group 0 adds and writes
        __syncthreads();
        if (grp == k) {
#pragma unroll
          for (int j = 0; j < J; ++j)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              float& s = sums[8 * (j * G + lane) + q];
              v[j][q] += k == GROUPS - 1 ? 0.f : s;
              s = v[j][q];
            }
        }
      }
      __syncthreads();
    }
    if (grp == 0)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int c = 8 * (j * G + lane);
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (c + q < a.N) part[(int64_t)w * a.N + c + q] = v[j][q];
      }
  }
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
  float s = 0.f, v = 0.f, z = 0.f, x[8];
  for (int c = 8 * threadIdx.x; c < a.N; c += 2048) {
    load8(X + c, a.N - c, x);
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) t += x[q];
    s += t;
  }
  row_sum2<256>(s, z, lds);
  const float mean = s / (float)a.N;
  for (int c = 8 * threadIdx.x; c < a.N; c += 2048) {
    load8(X + c, a.N - c, x);
    float t = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) t += c + q < a.N ? (x[q] - mean) * (x[q] - mean) : 0.f;
    v += t;
  }
  row_sum2<256>(v, z, lds);
  const float rstd = 1.f / __builtin_sqrtf(v / (float)a.N + a.eps);
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
  float s1 = 0.f, s2 = 0.f, x[8], d[8], g[8];
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
    s1 += t1;
    s2 += t2;
  }
  row_sum2<256>(s1, s2, lds);
  s1 /= (float)a.N;
  s2 /= (float)a.N;
  for (int c = 8 * threadIdx.x; c < a.N; c += 2048) {
    load(c);
#pragma unroll
    for (int q = 0; q < 8; ++q) d[q] = st[1] * (d[q] - s1 - x[q] * s2);
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

// Workgroups of a pass over rows: a launch has fewer than 2^32 threads.
unsigned norm_grid(int64_t blocks) { return (unsigned)(blocks < (1 << 23) ? blocks : 1 << 23); }

template <typename F>
hipError_t by_types(bool a32, bool b32, F&& f) {
  if (a32) return b32 ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
  return b32 ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

// f(G, J): the fewest lanes and pieces that hold a row of N; false if none does.
template <typename F>
bool by_row(int N, F&& f) {
  using std::integral_constant;
#define FFMLP_ROW(G, J) \
  if (N <= 8 * G * J) { f(integral_constant<int, G>{}, integral_constant<int, J>{}); return true; }
  FFMLP_ROW(8, 1)
  FFMLP_ROW(16, 1)
  FFMLP_ROW(32, 1)
  FFMLP_ROW(64, 1)
  FFMLP_ROW(64, 2)
  FFMLP_ROW(64, 4)
  FFMLP_ROW(256, 2)
  FFMLP_ROW(256, 4)
  FFMLP_ROW(256, 8)
#undef FFMLP_ROW
  return false;
}

}  // namespace

int norm_parts(int64_t M, int N) {
  int groups = 1;
  const bool held = by_row(N, [&](auto g, auto) { groups = 256 / decltype(g)::value; });
  const int64_t most = held ? (M + groups - 1) / groups : (M + 15) / 16;
  return (int)(most < 1 ? 1 : most < kNormParts ? most : kNormParts);
}

hipError_t launch_norm_forward(const NormArgs& a, hipStream_t s) {
  return by_types(a.x_fp32, a.y_fp32, [&](auto x32, auto y32) {
    constexpr bool X = decltype(x32)::value, Y = decltype(y32)::value;
    const bool held = by_row(a.N, [&](auto g, auto j) {
      constexpr int G = decltype(g)::value, J = decltype(j)::value, R = 256 / G;
      hipLaunchKernelGGL((norm_fwd_kernel<G, J, X, Y>), dim3(norm_grid((a.M + R - 1) / R)), dim3(256), 0, s, a);
    });
    if (!held) hipLaunchKernelGGL((norm_fwd_long_kernel<X, Y>), dim3(norm_grid(a.M)), dim3(256), 0, s, a);
    return hipGetLastError();
  });
}

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s) {
  const hipError_t e = by_types(a.x_fp32, a.dy_fp32, [&](auto x32, auto d32) {
    constexpr bool X = decltype(x32)::value, D = decltype(d32)::value;
    const bool held = by_row(a.N, [&](auto g, auto j) {
      constexpr int G = decltype(g)::value, J = decltype(j)::value;
      hipLaunchKernelGGL((norm_bwd_kernel<G, J, X, D>), dim3((unsigned)a.parts), dim3(256), 0, s, a);
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
