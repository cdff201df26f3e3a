// Arguments and launches of the vocabulary losses (head_kernel.h, head.hip).
#pragma once

#include "gemm.h"

namespace ffmlp {

constexpr int kHeadKey = 128;     // columns per entry of the table of starts
constexpr int kHeadMaxTop = 1024; // teacher entries of a row

struct HeadArgs {
  SideArgs h, w;          // H [M][D]; W [D][V], or the piece's columns of it
  int64_t M, D;
  int V;                  // columns: the vocabulary, or the piece
  int col0;               // first column of the piece
  float scale2;           // log2(e) / T
  // cross entropy: one target per row
  const int64_t* target;
  int64_t ignore;
  // distillation: a row's entries sorted by index
  const int* index;       // [M][top], absent ones last
  const float* q;         // [M][top] teacher probabilities
  const uint16_t* start;  // [M][keys]: entries with index < 128 k
  int top, keys;
  float* pick;            // [M][top] products h w of the entries
  f32x2* partial;         // [parts][M] largest product, and sum relative to it
  int runs, per_run, mt, nt;
  const f32x2* lse;       // [M] (see RowLse)
  uint16_t* P;            // [M][ldp]
  int64_t ldp;
  int keep;               // columns of the first piece, or 0: no gradients
  float* ref;             // [keep / the columns of a wave's tile][M] largest products
  int chunk;              // columns of a row that a wave of HEAD_SCALE takes
};

// The teacher's entries: probabilities over a row's list, sorted by index,
// and the table of starts.  ok[m]: 1, 0 (an empty list) or -1 (an index past
// the vocabulary).
struct TeacherArgs {
  const int64_t* index;  // [M][top], negative: absent
  const void* logits;    // [M][top]
  int logits_fp32;
  float inv_t;
  int64_t M, V;
  int top, keys;
  int* out_index;
  float* out_q;
  uint16_t* start;
  int* ok;
};
hipError_t launch_teacher(const TeacherArgs& a, hipStream_t s);

// lse and the loss of every row, then the mean loss and the gradient's scale.
// Rows: launch_row_loss, or HEAD_SCALE on its way.
struct RowLossArgs {
  const f32x2* partial;
  int parts;
  const float* pick;
  const float* q;         // null: cross entropy
  const int* ok;          // distillation
  const int64_t* target;  // cross entropy
  int64_t ignore;
  int top;
  float t2;               // T^2
  float temperature;
  int64_t M, V;
  float scale2;           // log2(e) / T
  f32x2* lse;             // [M]
  float* row_loss;
  float *loss, *alpha;    // mean loss; T / rows that count
};
hipError_t launch_row_loss(const RowLossArgs& a, hipStream_t s);
hipError_t launch_mean_loss(const RowLossArgs& a, hipStream_t s);

struct HeadPlan {
  bool rows;                  // head_rows_kernel: whole rows of logits in LDS
  bool large;
  int mt, nt, runs, per_run;  // head_lse_kernel
  int parts;                  // its maxima and sums of a row
  int piece, pieces;          // columns of P, a multiple of 256 unless one piece holds all
  int refs;                   // references of a row in the first piece
};
HeadPlan head_plan(int64_t M, int64_t D, int64_t V);

// The passes over the logits: log-sum-exp; P of the first piece from what that
// kept, and the losses of the rows (r); P of a later piece; all of these at once.
enum HeadPass { HEAD_LSE, HEAD_SCALE, HEAD_PROB, HEAD_ROWS };
hipError_t launch_head_ce(HeadPass pass, bool large, const HeadArgs& a, const RowLossArgs& r, hipStream_t s);
hipError_t launch_head_distill(HeadPass pass, bool large, const HeadArgs& a, const RowLossArgs& r, hipStream_t s);

#ifdef __HIPCC__
// With a row's products x = h w (unscaled) and c = log2(e) / T, a row's
// log-sum-exp in base 2 is m c + ls, m its largest product and ls = log2 of
// sum 2^((x - m) c), kept apart: every exponent is then a difference of products
// times c, right to its last bits however large the logits are.
// ls = +inf: the row does not count (its probabilities are 0).  NaN: it has an
// index past the vocabulary.
struct RowLse {
  float m, ls;
  // log2 of the probability of a word with product x
  __device__ __forceinline__ float log2_p(float x, float c) const { return __builtin_fmaf(x - m, c, -ls); }
  __device__ __forceinline__ bool live() const { return ls != __builtin_inff(); }
};

// (m, s) and (m2, s2), each a largest product and a sum of 2^((x - it) c), as one.
__device__ __forceinline__ void head_merge(float& m, float& s, float m2, float s2, float c) {
  const float top = __builtin_fmaxf(m, m2), at = top == -__builtin_inff() ? 0.f : top;
  s = s * __builtin_amdgcn_exp2f((m - at) * c) + s2 * __builtin_amdgcn_exp2f((m2 - at) * c);
  m = top;
}

// A row's loss from its lse, its target (cross entropy) and the products of its
// entries, pick(e), by a wave.  Returns the lse as RowLse says; `write`: lse and
// loss to memory.
template <typename F>
__device__ __forceinline__ RowLse row_end(const RowLossArgs& a, int64_t row, int lane, bool write, RowLse lse, int64_t t, F&& pick) {
  constexpr float kLn2 = 0.69314718f;
  float loss = 0.f;
  int state;  // 1 counts, 0 does not, -1 has an index past the vocabulary
  if (a.q) {
    state = a.ok[row];
    if (write) {
      for (int e = lane; e < a.top; e += 64) {
        const float q = a.q[row * a.top + e];
        if (!(q == 0.f)) loss += q * (kLn2 * (__builtin_amdgcn_logf(q) - lse.log2_p(pick(e), a.scale2)));  // logf: base 2
      }
#pragma unroll
      for (int d = 1; d < 64; d *= 2) loss += __shfl_xor(loss, d);
      loss *= a.t2;
    }
  } else {
    state = t == a.ignore ? 0 : t >= 0 && t < a.V ? 1 : -1;
    if (state == 1) loss = -kLn2 * lse.log2_p(pick(0), a.scale2);
  }
  if (state == 0) {
    lse = RowLse{0.f, __builtin_inff()};
    loss = 0.f;
  } else if (state < 0) {
    lse.ls = loss = __builtin_nanf("");
  }
  if (write && lane == 0) {
    a.lse[row] = f32x2{lse.m, lse.ls};
    a.row_loss[row] = loss;
  }
  return lse;
}

// The same from the row's partial sums, merged in a fixed tree.
__device__ __forceinline__ RowLse row_loss(const RowLossArgs& a, int64_t row, int lane, bool write) {
  float m = -__builtin_inff(), s = 0.f;
  for (int p = lane; p < a.parts; p += 64) {
    const f32x2 v = a.partial[(int64_t)p * a.M + row];
    head_merge(m, s, v[0], v[1], a.scale2);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) head_merge(m, s, __shfl_xor(m, d), __shfl_xor(s, d), a.scale2);
  return row_end(a, row, lane, write, RowLse{m, __builtin_amdgcn_logf(s)}, a.q ? 0 : a.target[row],
                 [&](int e) { return a.pick[row * a.top + e]; });
}
#endif

}  // namespace ffmlp
