// Vocabulary losses: the plan, the teacher's lists, and the losses of the rows.
#include "head_kernel.h"

namespace ffmlp {

namespace {
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Logits whose exponentials are kept (as fp16, later P as bf16), and that a piece
// of P holds: 1 GiB, a bound on memory.  There is no knee in it: what is kept is
// not computed again.  Steps in ms with 2^27, 2^28, 2^29 and 2^30 of them, hidden
// size 2048: 16384 rows over 65536 words 14.96, 14.67, 13.81 and 12.19; 8192 over
// 131072 15.13, 14.52, 13.60 and 12.38; 12000 over 65536 12.48, 11.65, 10.97 and
// 9.87; hidden size 512, 16384 over 50021 4.18, 4.06, 3.90 and 3.71.
constexpr int64_t kPieceElems = (int64_t)1 << 29;
}  // namespace

HeadPlan head_plan(int64_t M, int64_t D, int64_t V) {
  HeadPlan p{};
  // One round of workgroups, one to a CU.  Whole calls with gradients in us in one
  // pass and in two, over 1000 words: 4096 rows of 64 34.2 and 42.8, of 128 35.3 and
  // 43.3, of 256 41.1 and 46.3; 8192 rows 48.4 and 49.3, 51.4 and 50.6, 62.5 and
  // 57.0; 16384 rows 69.3 and 62.7, 75.2 and 70.6, 100.1 and 88.2; over 200 words of
  // 128, 4096 rows 26.0 and 29.9, 6144 33.2 and 33.2, 16384 54.6 and 50.6.
  p.rows = V <= kRowsVocab && D <= kRowsDim && M <= 256 * kRowsTile;
  p.large = cdiv(M, GemmLarge::BM) * cdiv(V, GemmLarge::BN) >= 512;
  p.mt = (int)cdiv(M, p.large ? GemmLarge::BM : GemmMedium::BM);
  p.nt = (int)cdiv(V, p.large ? GemmLarge::BN : GemmMedium::BN);
  int64_t runs = 512 / (p.mt > 0 ? p.mt : 1);
  if (runs > p.nt) runs = p.nt;
  if (runs < 1) runs = 1;
  p.per_run = (int)cdiv(p.nt, runs);
  p.runs = (int)cdiv(p.nt, p.per_run);
  int64_t cols = kPieceElems / (M > 0 ? M : 1) / 256 * 256;
  if (cols < 1024) cols = 1024;
  // Where one piece does not do, the first is as large as it may be, so that few
  // logits too many cost few computed twice (8193 rows of 2048 over 65536 words:
  // 8.65 ms with equal pieces, 8.11 so).  A power of two of columns would put P's
  // rows 2^n + 128 bytes apart, where head_scale_kernel loses up to a quarter
  // (32768 rows over 16384 columns 587 us, over 16128 447); one piece more would
  // cost as much again.
  if (V > cols && (cols & (cols - 1)) == 0 && cdiv(V, cols - 256) == cdiv(V, cols)) cols -= 256;
  p.piece = (int)(V < cols ? V : cols);
  p.pieces = (int)cdiv(V, p.piece);
  const int across = p.large ? GemmLarge::WN : GemmMedium::WN;  // waves that share a row of a tile
  p.parts = p.runs * across;
  p.refs = (int)cdiv(p.piece, p.large ? GemmLarge::BN : GemmMedium::BN) * across;
  return p;
}

// One wave per row.  The list is sorted by counting, for every entry, the
// entries before it (index, then position): lists are short, and equal
// indexes keep their order.  4096 lists of 32: 11 us, most of it the latency of
// the searches for the 257 starts of a row.
__global__ __launch_bounds__(64) void teacher_kernel(const TeacherArgs a) {
  __shared__ int idx[kHeadMaxTop], sorted[kHeadMaxTop];
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x;
  const int64_t at = row * a.top;
  auto logit = [&](int e) {
    return a.logits_fp32 ? static_cast<const float*>(a.logits)[at + e]
                         : __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.logits)[at + e] << 16);
  };
  float mx = -__builtin_inff();
  int bad = 0;
  for (int e = lane; e < a.top; e += 64) {
    const int64_t i = a.index[at + e];
    bad |= i >= a.V;
    idx[e] = i < 0 || i >= a.V ? 0x7fffffff : (int)i;
    if (i >= 0) {
      const float z = logit(e);
      mx = z != z || mx != mx ? __builtin_nanf("") : __builtin_fmaxf(mx, z);
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const float o = __shfl_xor(mx, d);
    mx = o != o || mx != mx ? __builtin_nanf("") : __builtin_fmaxf(mx, o);
    bad |= __shfl_xor(bad, d);
  }
  const bool empty = mx == -__builtin_inff();
  // divided by T after the subtraction: a type's lowest value stays finite
  auto weight = [&](int e) { return __expf((logit(e) - mx) * a.inv_t); };
  float sum = 0.f;
  for (int e = lane; e < a.top; e += 64)
    if (a.index[at + e] >= 0 && !empty) sum += weight(e);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
  __syncthreads();
  for (int e = lane; e < a.top; e += 64) {
    const int me = idx[e];
    int rank = 0;
    for (int o = 0; o < a.top; ++o) rank += idx[o] < me || (idx[o] == me && o < e);
    sorted[rank] = me;
    a.out_index[at + rank] = me;
    // a denormal q is 0: the hardware's logarithm of it would be -inf, and q log q
    // is below 2^-119
    const float q = me != 0x7fffffff && !empty ? weight(e) / sum : 0.f;
    a.out_q[at + rank] = q < 0x1p-126f ? 0.f : q;
  }
  __syncthreads();
  for (int k = lane; k < a.keys; k += 64) {
    const int64_t first = (int64_t)k * kHeadKey;
    int lo = 0, hi = a.top;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (sorted[mid] != 0x7fffffff && sorted[mid] < first) lo = mid + 1; else hi = mid;
    }
    a.start[row * a.keys + k] = (uint16_t)lo;
  }
  if (lane == 0) a.ok[row] = bad ? -1 : empty ? 0 : 1;
}

hipError_t launch_teacher(const TeacherArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(teacher_kernel, dim3((unsigned)a.M), dim3(64), 0, s, a);
  return hipGetLastError();
}

// One wave per row.
__global__ __launch_bounds__(256) void row_loss_kernel(const RowLossArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row < a.M) row_loss(a, row, threadIdx.x & 63, true);
}

// One workgroup: thread t adds rows t, t + 1024, ... in order, then a tree.
// 4 us for 4096 rows, 7 for 8192: latency.
__global__ __launch_bounds__(1024) void mean_loss_kernel(const RowLossArgs a) {
  __shared__ float sums[1024];
  __shared__ int counts[1024];
  const int t = threadIdx.x;
  float s = 0.f;
  int n = 0;
  for (int64_t r = t; r < a.M; r += 1024) {
    s += a.row_loss[r];
    n += a.lse[r][1] != __builtin_inff();
  }
  sums[t] = s;
  counts[t] = n;
  __syncthreads();
  for (int h = 512; h > 0; h >>= 1) {
    if (t < h) {
      sums[t] += sums[t + h];
      counts[t] += counts[t + h];
    }
    __syncthreads();
  }
  if (t == 0) {
    const float inv = 1.f / (float)(counts[0] > 0 ? counts[0] : 1);
    if (a.loss) *a.loss = sums[0] * inv;
    *a.alpha = a.temperature * inv;
  }
}

hipError_t launch_row_loss(const RowLossArgs& a, hipStream_t s) {
  if (a.M == 0) return hipSuccess;
  hipLaunchKernelGGL(row_loss_kernel, dim3((unsigned)cdiv(a.M, 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_mean_loss(const RowLossArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(mean_loss_kernel, dim3(1), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace ffmlp
