// Log-probabilities of given tokens, and the two losses that a draft (or a policy) is trained with on the logits of a head, with the
// gradient of those logits.
//
//   log p(a)  = (z_a - max z) - log sum_j exp(z_j - max z)
//   policy      r = exp(log p - old), row = -min(r A, clip(r, 1 - lo, 1 + hi) A) + beta (exp(ref - log p) - (ref - log p) - 1), L = sum w row
//   preference  margin = beta (S_chosen - S_rejected), S = sum of w (log p - ref) over an answer's rows,
//               pair = -(1 - e) log sigma(margin) - e log sigma(-margin), L = mean over the pairs
//   gradient    dL/dz_j = c ([j == a] - p_j) with c = dL/d(log p) of the row
//
// Everything but the passes over the logits is a few numbers a row, in 64 bits, added in a fixed order: the result is reproducible bit for bit.
// The passes: rows_stats_kernel reads each row once for its maximum and sum, a gradient pass reads the logits again and writes the gradient.  Between them one
// workgroup turns the sums into log-probabilities, losses and a coefficient per row (rows_grad_kernel), or every workgroup of the gradient pass does that for
// its row, a launch less (few_rows_grad_kernel).  A policy's coefficient depends on its row alone: from 128 long rows on one workgroup keeps a row between the two
// and reads it once (policy_fused_kernel).  All are bound by HBM where rows are many and by launches where they are few.
#include "common.h"

namespace nanospec {

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));           // rows start at any element: 16-byte loads at its alignment
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef uint16_t u16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));

constexpr int kRowThreads = 256;         // of a workgroup that takes a piece of a row
// log2 e lies between two fp32 numbers, 0.16 of their distance above the lower one.  With one of them for all exponents, every term of a row's sum is off by 1.3e-8 (or 7e-8) of
// its exponent to the same side, which does not average out (1e-7 of the sum; seen in the margin of two answers, where most of the log-probabilities cancel).  The sums
// therefore use both.  A gradient's entry is one probability, in which nothing cancels: it takes the lower one, whose 1.3e-8 is a fifth of the exponent's own rounding.
constexpr float kLog2e = 0x1.715476p+0f, kLog2eUp = 0x1.715478p+0f, kLog2eRest = 0x1.4ae0c0p-26f, kLn2 = 0.6931471805599453f;   // kLog2e + kLog2eRest: log2 e

// x <= 0, between two maxima, for the sums: the exponent rounded once
__device__ __forceinline__ float exp_neg(float x) {
  x = fmaxf(x, -1000.f);                                   // exp is 0 from -104 on; -inf would meet itself below
  const float y = x * kLog2e;
  return __builtin_amdgcn_exp2f(y + fmaf(x, kLog2eRest, fmaf(x, kLog2e, -y)));
}
__device__ __forceinline__ float exp_neg_short(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }      // of a logit; NaN stays NaN

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  typedef float Raw __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ Raw raw(const float* p) { return *reinterpret_cast<const f32x4_any*>(p); }
  static __device__ __forceinline__ void open(const Raw& v, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = v[i];
  }
  static __device__ __forceinline__ void load(const float* p, float (&x)[N]) { open(raw(p), x); }
  static __device__ __forceinline__ float one(const float* p) { return *p; }
};
template <>
struct Vec<uint16_t> {
  static constexpr int N = 8;
  typedef uint32_t Raw __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ Raw raw(const uint16_t* p) { return __builtin_bit_cast(Raw, (u16x8)*reinterpret_cast<const u16x8_any*>(p)); }
  static __device__ __forceinline__ void open(const Raw& v, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
  }
  static __device__ __forceinline__ void load(const uint16_t* p, float (&x)[N]) { open(raw(p), x); }
  static __device__ __forceinline__ float one(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
};

template <int N>
__device__ __forceinline__ void store_vec(float* p, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4_any*>(p + i) = f32x4_any{x[i], x[i + 1], x[i + 2], x[i + 3]};
}
template <int N>
__device__ __forceinline__ void store_vec(uint16_t* p, const float (&x)[N]) {       // rounded to nearest even, the only rounding of the gradient
  if constexpr (N == 8) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
    *reinterpret_cast<bf16x8_any*>(p) = v;
  } else {
    typedef __bf16 bf16x4_any __attribute__((ext_vector_type(4), aligned(2)));
    bf16x4_any v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (__bf16)x[i];
    *reinterpret_cast<bf16x4_any*>(p) = v;
  }
}
__device__ __forceinline__ void store_one(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_one(uint16_t* p, float x) { *p = __builtin_bit_cast(uint16_t, (__bf16)x); }

// a running maximum and the sum of exp(z - maximum); {-inf, 0} is nothing.  A NaN, or +inf, makes the sum NaN.
struct Stat {
  float m, s;
};

__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.f : m; }   // rows of -inf: exp(-inf - 0) = 0

__device__ __forceinline__ Stat join(Stat a, Stat b) {
  const float m = fmaxf(a.m, b.m), mm = finite_or_zero(m);
  return Stat{m, a.s * exp_neg(a.m - mm) + b.s * exp_neg(b.m - mm)};
}

// N more numbers: 2^(x l - c) with l one of the two neighbours of log2 e -- of sixteen numbers three take the upper one, which leaves the sum's bias a sixth --, c = fl(m l);
// what c is off by multiplies the sum.  A multiply-add, the exponential and an addition a number.
// That factor, 2^r with |r| at most half a step of c, is taken to first order, which is enough while r is small: below 2048 |c| < 2^12, |r| <= 2^-13, and what is dropped,
// (r ln 2)^2 / 2, is within 2^-28.  It is not for a row of -1e9, whose r may be 64.  Beyond, the maximum is subtracted first: one rounding of the difference, a subtraction a number more.
constexpr float kNearMax = 2048.f;

template <int N>
__device__ __forceinline__ void take(Stat& t, const float (&x)[N]) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
  const float m = fmaxf(t.m, top);
  float s = 0.f;
  if (fabsf(m) < kNearMax) {
    const float c = m * kLog2e, cu = m * kLog2eUp;
    float su = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i % 6 == 3) su += __builtin_amdgcn_exp2f(fmaf(x[i], kLog2eUp, -cu));
      else s += __builtin_amdgcn_exp2f(fmaf(x[i], kLog2e, -c));
    }
    s = fmaf(s, -kLn2 * fmaf(m, kLog2e, -c), s) + fmaf(su, -kLn2 * fmaf(m, kLog2eUp, -cu), su);
  } else {                                                 // far from zero, infinite, or nothing but -inf so far
    const float mm = finite_or_zero(m);
#pragma unroll
    for (int i = 0; i < N; ++i) s += __builtin_amdgcn_exp2f((x[i] - mm) * (i % 6 == 3 ? kLog2eUp : kLog2e));
  }
  t.s = t.s * exp_neg(t.m - finite_or_zero(m)) + s;
  t.m = m;
}

__device__ __forceinline__ Stat wave_join(Stat t) {
#pragma unroll
  for (int o = 32; o; o >>= 1) t = join(t, Stat{__shfl_xor(t.m, o), __shfl_xor(t.s, o)});
  return t;
}

// a token's column (-1: none) and logit (-inf: none)
struct Place {
  float z;
  int col;
};

// -inf where the token has no column, or its logit is -inf and the row's sum a number; both maximum and logit are exact, so only the sum carries a rounding
__device__ __forceinline__ double log_probability(const Place& a, const Stat& t) {
  if (a.z == -INFINITY) return a.col >= 0 && t.s != t.s ? (double)t.s : -INFINITY;
  return ((double)a.z - (double)t.m) - log((double)t.s);
}

// column of a row's token: the token itself, or its place in the ascending list; -1 if it has none.  One wavefront, every lane gets it.
__device__ __forceinline__ int token_column(const LogitRows& r, int row, int n) {
  const int t = r.tokens[row];
  if (!r.ids) return t >= 0 && t < n ? t : -1;
  const int32_t* ids = r.ids + (int64_t)(row / r.per_list) * r.V;
  const int lane = threadIdx.x & 63;
  int lo = 0, len = n;                                     // the places that may still hold it
  while (len > 0) {
    const int step = (len + 63) >> 6, at = lo + lane * step;
    const bool in = at < lo + len;
    const int v = in ? ids[at] : 0;
    const uint64_t hit = __ballot(in && v == t);
    if (hit) return lo + (__ffsll((unsigned long long)hit) - 1) * step;
    const uint64_t below = __ballot(in && v < t);
    if (!below || step == 1) return -1;
    const int k = __popcll(below) - 1, end = lo + len;     // behind the last probe below it
    lo += k * step + 1;
    len = (step - 1 < end - lo) ? step - 1 : end - lo;
  }
  return -1;
}

__device__ __forceinline__ int row_columns(const LogitRows& r, int row) {
  if (!r.n) return r.V;
  const int n = r.n[row / r.per_list];
  return n < 0 ? 0 : n < r.V ? n : r.V;
}

__device__ __forceinline__ bool row_counts(const LogitRows& r, int row) {
  return row >= r.first && row < r.last && (!r.weight || r.weight[row] != 0.f);
}

// Bound by HBM: 509 rows of 128256 in fp32 46 us (5.7 TB/s), 1021 of 152064 in bf16 64 us (4.9; a number costs 8 of the 64 lane-cycles a compute unit has, the exponential
// 2.5 of them), where the loads of the next step are on their way: left to itself the compiler waits for each load of a step before the next (49 and 82 us).
// Piece `blockIdx.x % pieces` of row `blockIdx.x / pieces`: maximum and sum of its columns to part[], and the token's column and logit, from
// the workgroup that has the row's first columns, to at[].  Rows that do not count are not read.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void rows_stats_kernel(const LogitRows r, int pieces, int span, Stat* __restrict__ part, Place* __restrict__ at,
                                                                 float* __restrict__ logprob) {
  constexpr int N = Vec<T>::N;
  const int row = blockIdx.x / pieces, piece = blockIdx.x - row * pieces, tid = threadIdx.x, w = tid >> 6;
  if (!row_counts(r, row)) return;
  const T* z = static_cast<const T*>(r.z) + (int64_t)row * r.ld;
  const int n = row_columns(r, row);
  const int c0 = piece * span, c1 = c0 + span < n ? c0 + span : n;
  Place a{-INFINITY, -1};
  if (piece == 0 && w == 0) {
    a.col = token_column(r, row, n);
    if (a.col >= 0) a.z = Vec<T>::one(z + a.col);
  }
  // whole steps of four pieces of 16 bytes a thread, the next step's on their way while one is taken
  constexpr int U = 4, STEP = NT * N * U;
  typedef typename Vec<T>::Raw Raw;
  Stat t{-INFINITY, 0.f};
  int c = c0;
  if (c0 + STEP <= c1) {
    Raw v[2][U];
    auto fetch = [&](int b, int at) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[b][u] = Vec<T>::raw(z + at + (u * NT + tid) * N);
    };
    auto use = [&](int b) {
#pragma unroll
      for (int u = 0; u < U; u += 16 / N) {
        float x[16];
#pragma unroll
        for (int i = 0; i < 16 / N; ++i) Vec<T>::open(v[b][u + i], *reinterpret_cast<float(*)[N]>(&x[i * N]));
        take(t, x);
      }
    };
    const int steps = (c1 - c0) / STEP, last = c0 + (steps - 1) * STEP;    // past the end the last step again, not used
    fetch(0, c0);
    for (int i = 0; i < steps; i += 2) {
      fetch(1, c + STEP < last ? c + STEP : last);
      __builtin_amdgcn_sched_barrier(0);
      use(0);
      fetch(0, c + 2 * STEP < last ? c + 2 * STEP : last);
      __builtin_amdgcn_sched_barrier(0);
      if (i + 1 < steps) use(1);
      c += 2 * STEP;
    }
    c = last + STEP;
  }
  // the rest, less than a step: its loads go out together as well
  if (c < c1) {
    const int whole = (c1 - c) / N * N;
    Raw v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = (u * NT + tid) * N;
      if (u * NT * N < whole) v[u] = Vec<T>::raw(z + c + (at < whole ? at : 0));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * NT * N >= whole) break;
      float x[N];
      Vec<T>::open(v[u], x);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = (u * NT + tid) * N < whole ? x[i] : -INFINITY;
      take(t, x);
    }
    const float x[1] = {tid < c1 - c - whole ? Vec<T>::one(z + c + whole + tid) : -INFINITY};
    take(t, x);
  }
  t = wave_join(t);
  __shared__ Stat red[NT / 64];
  if ((tid & 63) == 0) red[w] = t;
  __syncthreads();
  if (tid) return;
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) t = join(t, red[i]);
  if (logprob) {                                           // one piece and nothing else asked for
    logprob[row] = (float)log_probability(a, t);
    return;
  }
  part[(int64_t)row * pieces + piece] = t;
  if (piece == 0) at[row] = a;
}

struct RowResult {
  Stat t;
  double lp;
  int col;
  bool has;          // the token has a probability: lp is not -inf
};

__device__ __forceinline__ RowResult finish_row(int row, int pieces, const Stat* __restrict__ part, const Place* __restrict__ at) {
  RowResult q;
  const Place a = at[row];
  q.t = part[(int64_t)row * pieces];
  for (int i = 1; i < pieces; ++i) q.t = join(q.t, part[(int64_t)row * pieces + i]);
  q.lp = log_probability(a, q.t);
  q.col = a.col;
  q.has = !(q.lp == -INFINITY);
  return q;
}

__global__ __launch_bounds__(256) void rows_logprob_kernel(int rows, int pieces, const Stat* __restrict__ part, const Place* __restrict__ at, float* __restrict__ logprob) {
  const int row = blockIdx.x * 256 + threadIdx.x;
  if (row < rows) logprob[row] = (float)finish_row(row, pieces, part, at).lp;
}

// sum over a workgroup of NT in a fixed order, in thread 0
template <int NT>
__device__ __forceinline__ double block_sum(double x, double* red) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_down(x, o);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  double s = 0;
  if (threadIdx.x == 0)
    for (int i = 0; i < NT / 64; ++i) s += red[i];
  return s;
}

// what the gradient pass needs of a row: the maximum, -c / sum and c; c == 0: the row's gradient is zero
struct RowCoef {
  float m, scale, c;
  int col;
};

__device__ __forceinline__ RowCoef coef_of(const Stat& t, int col, double c, float grad_scale) {
  return RowCoef{t.m, (float)(-(c * grad_scale) / (double)t.s), (float)(c * grad_scale), col};
}

// A policy's ratio and KL term take exp of the log-probability: a row where that is 0 in 64 bits has no loss and no gradient.  A margin is a sum of log-probabilities, to which
// every finite one counts.
__device__ __forceinline__ bool policy_has(double lp) { return !(lp < -745.0); }

// a row's policy loss and its derivative by the log-probability
struct PolicyRow {
  double loss, c;
};

__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& a, int row, double lp) {
  const double adv = a.adv[row], ratio = exp(lp - (double)a.old[row]);
  const double lo = 1.0 - (double)a.clip_low, hi = 1.0 + (double)a.clip_high;
  // old may be -inf, or so low that the ratio does not fit: an advantage of 0 makes nothing of it
  auto times = [&](double x) { return adv == 0.0 && x == INFINITY ? 0.0 : x * adv; };
  const double held = times(ratio < lo ? lo : ratio > hi ? hi : ratio), free = times(ratio);
  PolicyRow r{-(free <= held ? free : held), free <= held ? -free : 0.0};
  if (free != free) r.loss = r.c = free;                   // NaN stays NaN
  if (a.ref) {
    const double gap = (double)a.ref[row] - lp, e = exp(gap);
    r.loss += (double)a.beta * (e - gap - 1.0);
    r.c += (double)a.beta * (1.0 - e);
  }
  return r;
}

__device__ __forceinline__ double weight_of(const LogitRows& r, int row) { return r.weight ? (double)r.weight[row] : 1.0; }

// all rows by one workgroup
template <int NT>
__device__ void policy_rows(const LogitRows& r, int pieces, const Stat* __restrict__ part, const Place* __restrict__ at, const PolicyArgs& a, RowCoef* __restrict__ coef) {
  __shared__ double red[NT / 64];
  double sum = 0;
  for (int row = threadIdx.x; row < r.rows; row += NT) {
    float lp_out = 0.f, loss_out = 0.f;
    RowCoef k{0.f, 0.f, 0.f, -1};
    if (row_counts(r, row)) {
      const RowResult q = finish_row(row, pieces, part, at);
      lp_out = (float)q.lp;
      if (policy_has(q.lp)) {
        const PolicyRow x = policy_row(a, row, q.lp);
        const double w = weight_of(r, row);
        loss_out = (float)x.loss;
        sum += w * x.loss;
        k = coef_of(q.t, q.col, w * x.c, a.grad_scale);
      }
    }
    if (a.row_loss) a.row_loss[row] = loss_out;
    if (a.logprob) a.logprob[row] = lp_out;
    if (coef) coef[row] = k;
  }
  sum = block_sum<NT>(sum, red);
  if (threadIdx.x == 0) a.loss[0] = (float)sum;
}

__global__ __launch_bounds__(1024) void policy_rows_kernel(const LogitRows r, int pieces, const Stat* __restrict__ part, const Place* __restrict__ at, const PolicyArgs a,
                                                           RowCoef* __restrict__ coef) {
  policy_rows<1024>(r, pieces, part, at, a, coef);
}

// the rows' weighted losses, added in a fixed order
__global__ __launch_bounds__(1024) void policy_sum_kernel(int rows, const double* __restrict__ term, float* __restrict__ loss) {
  __shared__ double red[16];
  double sum = 0;
  for (int row = threadIdx.x; row < rows; row += 1024) sum += term[row];
  sum = block_sum<1024>(sum, red);
  if (threadIdx.x == 0) loss[0] = (float)sum;
}

// A row's policy loss and its gradient by one workgroup, which keeps the row on the compute unit between the two: RC pieces of 16 bytes a thread in
// registers, LC in LDS, so that up to (RC + LC) 8 KB of a row are read from memory once; what is beyond is read a second time, from
// the caches.  Two launches over all rows instead read them twice from memory: 2048 rows of 128256, fp32 to bf16, 481 us apart, 330 so (4.8 TB/s read and written, near a
// copy; 512 KB of a row fit the compute unit's 672 of registers and LDS), bf16 to bf16 318 / 252, fp32 to fp32 420 so.  Eight wavefronts, not sixteen: 256 registers a lane instead of 128.
// A chunk is what the workgroup's threads hold in a piece each; a row's full chunks go to LDS first, then to registers, the others and the row's end are streamed.
template <typename T, typename G, int RC, int LC>
__global__ __launch_bounds__(512, 2) void policy_fused_kernel(const LogitRows r, const PolicyArgs a, double* __restrict__ term, G* grad, int64_t ld_grad) {
  constexpr int N = Vec<T>::N, CH = 512 * N, U = 16 / N;                  // U pieces: 16 numbers, what a step of the sums takes
  static_assert(RC % U == 0 && LC % U == 0 && LC <= RC, "whole steps");
  typedef typename Vec<T>::Raw Raw;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ Stat red[8];
  __shared__ RowCoef shared_k;
  __shared__ float shared_z;
  Raw* held = reinterpret_cast<Raw*>(smem);                               // [LC][512]
  const int row = blockIdx.x, tid = threadIdx.x, w = tid >> 6;
  const T* z = static_cast<const T*>(r.z) + (int64_t)row * r.ld;
  G* g = grad + (int64_t)row * ld_grad;
  const int n = row_columns(r, row);
  const int full = n / CH;
  if (!row_counts(r, row)) {
    const float x[N] = {};
    for (int c = tid * N; c < n; c += CH) {
      if (c + N <= n) store_vec(g + c, x);
      else
        for (int i = c; i < n; ++i) store_one(g + i, 0.f);
    }
    if (tid == 0) {
      if (a.row_loss) a.row_loss[row] = 0.f;
      if (a.logprob) a.logprob[row] = 0.f;
      term[row] = 0;
    }
    return;
  }
  // chunks: LDS 0 .. nl - 1, registers nl .. nl + nr - 1, streamed from there on
  const int nl = full < LC ? full / U * U : LC, nr = full - nl < RC ? (full - nl) / U * U : RC, from = nl + nr;
  Stat t{-INFINITY, 0.f};
  Raw v[RC];
  const T* zt = z + tid * N;
  // a load past the chunks there are is the last one's again: the number of loads in flight does not depend on the row
  auto chunk = [&](int c) { return Vec<T>::raw(zt + (int64_t)(c < from ? c : from - 1) * CH); };
  Place pl{-INFINITY, -1};
  if (from) {
#pragma unroll
    for (int c = 0; c < RC; ++c) v[c] = chunk(c < LC && LC ? (nl ? c : nl + c) : nl + c);
  }
  if (w == 0) {
    pl.col = token_column(r, row, n);
    if (pl.col >= 0) pl.z = Vec<T>::one(z + pl.col);
  }
  if (from) {
    if (LC && nl) {
#pragma unroll
      for (int c = 0; c < LC; c += U) {
        if (c < nl) {
          float x[16];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            held[(c + u) * 512 + tid] = v[c + u];
            Vec<T>::open(v[c + u], *reinterpret_cast<float(*)[N]>(&x[u * N]));
          }
          take(t, x);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) v[c + u] = chunk(nl + c + u);
      }
    }
#pragma unroll
    for (int c = 0; c < RC; c += U) {
      if (c < nr) {
        float x[16];
#pragma unroll
        for (int u = 0; u < U; ++u) Vec<T>::open(v[c + u], *reinterpret_cast<float(*)[N]>(&x[u * N]));
        take(t, x);
      }
    }
  }
  for (int c = from * CH + tid * N; c < n; c += CH) {
    float x[N];
    if (c + N <= n) {
      Vec<T>::load(z + c, x);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = c + i < n ? Vec<T>::one(z + c + i) : -INFINITY;
    }
    take(t, x);
  }
  t = wave_join(t);
  if ((tid & 63) == 0) red[w] = t;
  __syncthreads();
  if (tid == 0) {
#pragma unroll
    for (int i = 1; i < 8; ++i) t = join(t, red[i]);
    const double lp = log_probability(pl, t);
    RowCoef k{0.f, 0.f, 0.f, -1};
    double loss = 0, sum = 0;
    if (policy_has(lp)) {
      const PolicyRow x = policy_row(a, row, lp);
      const double wt = weight_of(r, row);
      loss = x.loss;
      sum = wt * x.loss;
      k = coef_of(t, pl.col, wt * x.c, a.grad_scale);
    }
    if (a.row_loss) a.row_loss[row] = (float)loss;
    if (a.logprob) a.logprob[row] = (float)lp;
    term[row] = sum;
    shared_k = k;
    shared_z = pl.z;
  }
  __syncthreads();
  const RowCoef k = shared_k;
  auto value = [&](float x) { return k.c == 0.f ? 0.f : k.scale * exp_neg_short(x - k.m); };
  G* gt = g + tid * N;
  auto put = [&](int c, const Raw& y) {
    float x[N];
    Vec<T>::open(y, x);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = value(x[i]);
    store_vec(gt + (int64_t)c * CH, x);
  };
#pragma unroll
  for (int c = 0; c < RC; ++c)
    if (c < nr) put(nl + c, v[c]);
  for (int c = 0; c < nl; ++c) put(c, held[c * 512 + tid]);
  for (int c = from * CH + tid * N; c < n; c += CH) {
    if (c + N <= n) {
      put(c / CH, Vec<T>::raw(z + c));
    } else {
      for (int i = c; i < n; ++i) store_one(g + i, value(Vec<T>::one(z + i)));
    }
  }
  // the token's own entry, by the thread that has just written its column
  if (k.c != 0.f && tid == k.col % CH / N) store_one(g + k.col, value(shared_z) + k.c);
}

// a pair's loss and its derivative by the margin
struct PairLoss {
  double loss, slope;
};

__device__ __forceinline__ PairLoss pair_loss(const PairArgs& a, double margin) {
  const double e = (double)a.smoothing, less = log1p(exp(-fabs(margin)));               // log(1 + exp(-m)) = max(-m, 0) + less
  const double up = 1.0 / (1.0 + exp(margin)), down = 1.0 / (1.0 + exp(-margin));       // sigma(-m), sigma(m)
  // a margin is infinite where a reference gives a token no probability: a term whose factor is 0 adds nothing then, not 0 * inf
  const double good = e == 1.0 ? 0.0 : (1.0 - e) * (fmax(-margin, 0.0) + less), bad = e == 0.0 ? 0.0 : e * (fmax(margin, 0.0) + less);
  PairLoss p{good + bad, (1.0 - e) * -up + e * down};
  if (margin != margin) p.loss = margin;
  return p;
}

// what a row adds to its answer's sum
__device__ __forceinline__ double pair_term(const LogitRows& r, const PairArgs& a, int row, const RowResult& q) {
  return q.has ? weight_of(r, row) * (q.lp - (a.ref ? (double)a.ref[row] : 0.0)) : 0.0;
}

// the derivative by a row's log-probability, from that by its pair's margin; rejected: the second answer of the pair
__device__ __forceinline__ double pair_coef(const LogitRows& r, const PairArgs& a, int row, double slope, bool rejected) {
  return (rejected ? -1.0 : 1.0) * slope * ((double)a.beta / a.pairs) * weight_of(r, row);
}

// the answer that holds a row: off[lo] <= row < off[lo + 1]
__device__ __forceinline__ int answer_of(const Offsets& off, int pairs, int row) {
  int lo = 0, hi = 2 * pairs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (off.v[mid] <= row) lo = mid;
    else hi = mid;
  }
  return lo;
}

// all rows by one workgroup
template <int NT>
__device__ void pair_rows(const LogitRows& r, int pieces, const Stat* __restrict__ part, const Place* __restrict__ at, const PairArgs& a, const Offsets& off,
                          double* __restrict__ term, RowCoef* __restrict__ coef) {
  __shared__ double red[NT / 64], sums[NANOSPEC_MAX_BATCH];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  for (int row = tid; row < r.rows; row += NT) {
    RowResult q{};
    const bool counts = row_counts(r, row);
    if (counts) q = finish_row(row, pieces, part, at);
    if (a.logprob) a.logprob[row] = counts ? (float)q.lp : 0.f;
    term[row] = counts ? pair_term(r, a, row, q) : 0.0;
    if (coef) coef[row] = RowCoef{q.t.m, q.t.s, 0.f, q.has ? q.col : -1};  // the coefficient follows
  }
  __threadfence_block();
  __syncthreads();
  for (int q = w; q < 2 * a.pairs; q += NT / 64) {         // a wavefront an answer
    double s = 0;
    for (int row = off.v[q] + lane; row < off.v[q + 1]; row += 64) s += term[row];
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) sums[q] = s;
  }
  __syncthreads();
  PairLoss p{0, 0};
  if (tid < a.pairs) {
    const double margin = (double)a.beta * (sums[2 * tid] - sums[2 * tid + 1]);
    p = pair_loss(a, margin);
    if (a.margin) a.margin[tid] = (float)margin;
  }
  __syncthreads();
  if (tid < a.pairs) sums[tid] = p.slope;
  const double loss = block_sum<NT>(p.loss, red);          // and a barrier behind sums[]
  if (tid == 0) a.loss[0] = (float)(loss / a.pairs);
  if (!coef) return;
  for (int row = tid; row < r.rows; row += NT) {           // written by this thread above
    RowCoef k = coef[row];
    if (k.col >= 0) {
      const int answer = answer_of(off, a.pairs, row);
      k = coef_of(Stat{k.m, k.scale}, k.col, pair_coef(r, a, row, sums[answer >> 1], answer & 1), a.grad_scale);
    }
    coef[row] = k;
  }
}

// the answers' first rows travel by value
__global__ __launch_bounds__(1024) void pair_rows_kernel(const LogitRows r, int pieces, const Stat* __restrict__ part, const Place* __restrict__ at, const PairArgs a, const Offsets off,
                                                         double* __restrict__ term, RowCoef* __restrict__ coef) {
  pair_rows<1024>(r, pieces, part, at, a, off, term, coef);
}

// dL/dz of the columns c0 .. c1 - 1 of a row; z may be the gradient's own memory: every element is read by the thread that writes it
template <typename T, typename G>
__device__ __forceinline__ void grad_piece(const T* z, G* g, const RowCoef& k, int c0, int c1) {
  constexpr int N = Vec<T>::N, U = 16 / N;
  const int tid = threadIdx.x;
  if (k.c == 0.f) {
    for (int c = c0 + tid * N; c < c1; c += kRowThreads * N) {
      const float x[N] = {};
      if (c + N <= c1) store_vec(g + c, x);
      else
        for (int i = c; i < c1; ++i) store_one(g + i, 0.f);
    }
    return;
  }
  auto one = [&](float x, int c) {
    const float p = k.scale * exp_neg_short(x - k.m);
    return c == k.col ? p + k.c : p;
  };
  int c = c0;
  for (; c + kRowThreads * N * U <= c1; c += kRowThreads * N * U) {
    float x[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) Vec<T>::load(z + c + (u * kRowThreads + tid) * N, x[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int b = c + (u * kRowThreads + tid) * N;
#pragma unroll
      for (int i = 0; i < N; ++i) x[u][i] = one(x[u][i], b + i);
      store_vec(g + b, x[u]);
    }
  }
  for (c += tid * N; c < c1; c += kRowThreads * N) {
    if (c + N <= c1) {
      float x[N];
      Vec<T>::load(z + c, x);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = one(x[i], c + i);
      store_vec(g + c, x);
    } else {
      for (int i = c; i < c1; ++i) store_one(g + i, one(Vec<T>::one(z + i), i));
    }
  }
}

// piece `blockIdx.x % pieces` of a row, the last rows first: of those the caches may still hold logits from the pass before (1021 rows of 152064 in bf16: 191 us for 194)
template <typename T, typename G>
__global__ __launch_bounds__(kRowThreads) void rows_grad_kernel(const LogitRows r, int pieces, int span, const RowCoef* __restrict__ coef, G* grad, int64_t ld_grad) {
  const int up = blockIdx.x / pieces, row = r.rows - 1 - up, piece = blockIdx.x - up * pieces;
  const int n = row_columns(r, row), c0 = piece * span, c1 = c0 + span < n ? c0 + span : n;
  grad_piece(static_cast<const T*>(r.z) + (int64_t)row * r.ld, grad + (int64_t)row * ld_grad, coef[row], c0, c1);
}

__device__ __forceinline__ void few_rows_total(const LogitRows& r, int pieces, const Stat* part, const Place* at, const PolicyArgs& a, double*) {
  policy_rows<kRowThreads>(r, pieces, part, at, a, nullptr);
}

__device__ __forceinline__ double few_rows_coef(const LogitRows& r, int, const Stat*, const Place*, const PolicyArgs& a, int row, const RowResult& q, double*) {
  return policy_has(q.lp) ? weight_of(r, row) * policy_row(a, row, q.lp).c : 0.0;
}

struct PairFew : PairArgs {
  Offsets off;
};

__device__ __forceinline__ void few_rows_total(const LogitRows& r, int pieces, const Stat* part, const Place* at, const PairFew& a, double* term) {
  pair_rows<kRowThreads>(r, pieces, part, at, a, a.off, term, nullptr);
}

// every thread a row of the pair, at most kRowThreads of them
__device__ __forceinline__ double few_rows_coef(const LogitRows& r, int pieces, const Stat* part, const Place* at, const PairFew& a, int row, const RowResult&, double* red) {
  const int answer = answer_of(a.off, a.pairs, row), first = a.off.v[answer & ~1], mid = a.off.v[answer | 1], last = a.off.v[(answer | 1) + 1];
  const int mine = first + (int)threadIdx.x;
  double s = 0;
  if (mine < last && row_counts(r, mine)) s = (mine < mid ? 1.0 : -1.0) * pair_term(r, a, mine, finish_row(mine, pieces, part, at));
  s = block_sum<kRowThreads>(s, red);
  return pair_coef(r, a, row, pair_loss(a, (double)a.beta * s).slope, answer & 1);       // of thread 0 only
}

// Bound by HBM where rows are many (1021 of 152064 in bf16 93 us, logits and gradient at 6.7 TB/s, some of the logits from the caches), else by the coefficients' 64-bit functions: 37 rows of 32000 7.4
// us, 7 rows of a policy 4.6.
// The coefficients by every workgroup for itself, from the sums of the pass before, in the launch that writes the gradient, and the totals by one workgroup more, the first: a launch less.
template <typename T, typename G, typename A>
__global__ __launch_bounds__(kRowThreads) void few_rows_grad_kernel(const LogitRows r, int pieces, int cut, int span, const Stat* part, const Place* at, const A a, double* term, G* grad,
                                                                    int64_t ld_grad) {
  __shared__ double red[kRowThreads / 64];
  __shared__ RowCoef shared_k;
  if (blockIdx.x == 0) {
    few_rows_total(r, pieces, part, at, a, term);
    return;
  }
  const int block = blockIdx.x - 1, up = block / cut, row = r.rows - 1 - up, piece = block - up * cut;
  const int n = row_columns(r, row), c0 = piece * span, c1 = c0 + span < n ? c0 + span : n;
  if (c0 >= c1) return;
  RowCoef k{0.f, 0.f, 0.f, -1};
  if (row_counts(r, row)) {
    const RowResult q = finish_row(row, pieces, part, at);
    const double c = few_rows_coef(r, pieces, part, at, a, row, q, red);
    if (threadIdx.x == 0) shared_k = q.has ? coef_of(q.t, q.col, c, a.grad_scale) : k;
    __syncthreads();
    k = shared_k;
  }
  grad_piece(static_cast<const T*>(r.z) + (int64_t)row * r.ld, grad + (int64_t)row * ld_grad, k, c0, c1);
}

// ---- host --------------------------------------------------------------------------------------------------------

// Threads of a workgroup that takes a whole row, where there are rows for half the compute units; 0: rows are cut into pieces until there are 2048 workgroups of
// kRowThreads, of no less than 4096 columns, and joined by a launch of its own (us, pieces / 256 / 512 / 1024 threads: 128 rows of 128256 in fp32 16.7 / 15.8 / 14.5 / 16.0, 509
// 53.8 / 53.4 / 53.1 / 52.5, 1021 of 152064 in bf16 67.5 / 66.1 / 64.6 / 63.2, 1500 of 17000 28.9 / 22.4 / 23.6 / 30.0, 3000 of 32000 in bf16 41.2 / 41.6 / 41.5 / 48.6; 300 of 128256,
// whose last 44 rows have the chip to themselves, 35 / 38 / 40 / 41).
static int whole_threads(int32_t rows, int32_t V) { return rows < 128 || V < 16384 ? 0 : V < 32768 ? 256 : 512; }

static RowCut row_cut(int32_t rows, int32_t V) {
  int64_t pieces = (2048 + (int64_t)rows - 1) / rows;
  const int64_t most = ((int64_t)V + 4095) / 4096;
  if (pieces > most) pieces = most;
  const int64_t span = ((V + pieces - 1) / pieces + 4095) / 4096 * 4096;
  return RowCut{(int32_t)((V + span - 1) / span), (int32_t)(span < V ? span : V)};
}

static RowCut stats_cut(int32_t rows, int32_t V) { return whole_threads(rows, V) ? RowCut{1, V} : row_cut(rows, V); }

static int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

// No less than rows * row_cut(rows, V).pieces, and no more for fewer rows or columns, so that a workspace of a program's largest batch is enough for the others (pieces fall as rows
// rise: 2047 rows have twice as many as 2048).
static int64_t most_pieces(int32_t rows, int32_t V) {
  const int64_t by_columns = (int64_t)rows * (((int64_t)V + 4095) / 4096), by_rows = (int64_t)rows + 2047;
  return by_columns < by_rows ? by_columns : by_rows;
}

struct LossSpace {
  Stat* part;
  Place* at;
  RowCoef* coef;
  double* term;
};

static LossSpace loss_space(char* p, int32_t rows, int32_t V) {
  LossSpace s;
  s.part = reinterpret_cast<Stat*>(p);
  p += up256(most_pieces(rows, V) * sizeof(Stat));
  s.coef = reinterpret_cast<RowCoef*>(p);
  p += up256((int64_t)rows * sizeof(RowCoef));
  s.term = reinterpret_cast<double*>(p);
  p += up256((int64_t)rows * sizeof(double));
  s.at = reinterpret_cast<Place*>(p);
  return s;
}

int64_t loss_workspace_bytes(int32_t rows, int32_t V) {
  return up256(most_pieces(rows, V) * sizeof(Stat)) + up256((int64_t)rows * sizeof(RowCoef)) + up256((int64_t)rows * sizeof(double)) +
         up256((int64_t)rows * sizeof(Place));
}

static hipError_t run_stats(const LogitRows& r, const LossSpace& s, float* logprob, hipStream_t stream) {
  const RowCut cut = stats_cut(r.rows, r.V);
  const unsigned grid = (unsigned)((int64_t)r.rows * cut.pieces);
#define NS_STATS(T, NT) rows_stats_kernel<T, NT><<<dim3(grid), NT, 0, stream>>>(r, cut.pieces, cut.span, s.part, s.at, logprob)
#define NS_STATS_T(NT)                                   \
  do {                                                   \
    if (r.type == NANOSPEC_F32) NS_STATS(float, NT);     \
    else NS_STATS(uint16_t, NT);                         \
  } while (0)
  switch (whole_threads(r.rows, r.V)) {
    case 512: NS_STATS_T(512); break;
    default: NS_STATS_T(kRowThreads);
  }
#undef NS_STATS_T
#undef NS_STATS
  return hipGetLastError();
}

static hipError_t run_grad(const LogitRows& r, const LossSpace& s, void* grad, int32_t type, int64_t ld, hipStream_t stream) {
  const RowCut cut = row_cut(r.rows, r.V);
  const unsigned grid = (unsigned)((int64_t)r.rows * cut.pieces);
#define NS_GRAD(T, G) rows_grad_kernel<T, G><<<dim3(grid), kRowThreads, 0, stream>>>(r, cut.pieces, cut.span, s.coef, static_cast<G*>(grad), ld)
  if (r.type == NANOSPEC_F32) {
    if (type == NANOSPEC_F32) NS_GRAD(float, float);
    else NS_GRAD(float, uint16_t);
  } else {
    if (type == NANOSPEC_F32) NS_GRAD(uint16_t, float);
    else NS_GRAD(uint16_t, uint16_t);
  }
#undef NS_GRAD
  return hipGetLastError();
}

// Whether few_rows_grad_kernel writes the gradient.  Pairs: a thread for every row of the longest one, and rows that the workgroup of the totals gets through while the others write
// (us, three launches / two: 37 rows of 32000 in fp32 14.4 / 11.5, 300 of 32000 29.2 / 26.3, 600 of 128256 155 / 150, 1021 of 152064 in bf16 184 / 178, 1000 of 8000 28.6 / 28.3).
static bool policy_few_rows(int32_t rows) { return rows <= 128; }
static bool pair_few_rows(int32_t rows, int32_t V, int32_t longest) { return longest <= kRowThreads && (rows <= 256 || (rows <= 2048 && V >= 8000)); }

template <typename A>
static hipError_t run_few_rows(const LogitRows& r, const LossSpace& s, const A& a, void* grad, int32_t type, int64_t ld, hipStream_t stream) {
  const RowCut cut = row_cut(r.rows, r.V);
  const unsigned grid = (unsigned)(r.rows * cut.pieces) + 1;
  const int pieces = stats_cut(r.rows, r.V).pieces;
#define NS_FEW(T, G) few_rows_grad_kernel<T, G, A><<<dim3(grid), kRowThreads, 0, stream>>>(r, pieces, cut.pieces, cut.span, s.part, s.at, a, s.term, static_cast<G*>(grad), ld)
  if (r.type == NANOSPEC_F32) {
    if (type == NANOSPEC_F32) NS_FEW(float, float);
    else NS_FEW(float, uint16_t);
  } else {
    if (type == NANOSPEC_F32) NS_FEW(uint16_t, float);
    else NS_FEW(uint16_t, uint16_t);
  }
#undef NS_FEW
  return hipGetLastError();
}

hipError_t launch_token_logprob(const LogitRows& r, float* logprob, char* ws, hipStream_t stream) {
  const LossSpace s = loss_space(ws, r.rows, r.V);
  const int pieces = stats_cut(r.rows, r.V).pieces;
  hipError_t e = run_stats(r, s, pieces == 1 ? logprob : nullptr, stream);
  if (e != hipSuccess || pieces == 1) return e;
  rows_logprob_kernel<<<dim3((unsigned)((r.rows + 255) / 256)), 256, 0, stream>>>(r.rows, pieces, s.part, s.at, logprob);
  return hipGetLastError();
}

// Chunks of 8 KB a row: what a workgroup of policy_fused_kernel holds.
template <typename T, typename G>
static hipError_t run_policy_fused(const LogitRows& r, const PolicyArgs& a, double* term, void* grad, int64_t ld_grad, hipStream_t s) {
  const int64_t bytes = (int64_t)r.V * sizeof(T);
  G* g = static_cast<G*>(grad);
  if (bytes <= 16 * 8192) policy_fused_kernel<T, G, 16, 0><<<dim3((unsigned)r.rows), 512, 0, s>>>(r, a, term, g, ld_grad);
  else if (bytes <= 32 * 8192) policy_fused_kernel<T, G, 32, 0><<<dim3((unsigned)r.rows), 512, 0, s>>>(r, a, term, g, ld_grad);
  else policy_fused_kernel<T, G, 48, 16><<<dim3((unsigned)r.rows), 512, 16 * 8192, s>>>(r, a, term, g, ld_grad);
  return hipGetLastError();
}

template <typename T, typename G>
static hipError_t configure_policy() {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(policy_fused_kernel<T, G, 48, 16>), hipFuncAttributeMaxDynamicSharedMemorySize, 16 * 8192);
}

hipError_t loss_configure_device() {
  hipError_t e = configure_policy<float, float>();
  if (e == hipSuccess) e = configure_policy<float, uint16_t>();
  if (e == hipSuccess) e = configure_policy<uint16_t, float>();
  if (e == hipSuccess) e = configure_policy<uint16_t, uint16_t>();
  return e;
}

static hipError_t launch_policy_fused(const LogitRows& r, const PolicyArgs& a, double* term, void* grad, int32_t type, int64_t ld, hipStream_t s) {
  hipError_t e;
  if (r.type == NANOSPEC_F32) e = type == NANOSPEC_F32 ? run_policy_fused<float, float>(r, a, term, grad, ld, s) : run_policy_fused<float, uint16_t>(r, a, term, grad, ld, s);
  else e = type == NANOSPEC_F32 ? run_policy_fused<uint16_t, float>(r, a, term, grad, ld, s) : run_policy_fused<uint16_t, uint16_t>(r, a, term, grad, ld, s);
  if (e != hipSuccess) return e;
  policy_sum_kernel<<<dim3(1), 1024, 0, s>>>(r.rows, term, a.loss);
  return hipGetLastError();
}

hipError_t launch_policy_loss(const LogitRows& r, const PolicyArgs& a, void* grad, int32_t grad_type, int64_t ld_grad, char* ws, hipStream_t stream) {
  const LossSpace s = loss_space(ws, r.rows, r.V);
  if (grad && policy_fuses(r.rows, r.V)) return launch_policy_fused(r, a, s.term, grad, grad_type, ld_grad, stream);
  hipError_t e = run_stats(r, s, nullptr, stream);
  if (e != hipSuccess) return e;
  if (grad && policy_few_rows(r.rows)) return run_few_rows(r, s, a, grad, grad_type, ld_grad, stream);
  policy_rows_kernel<<<dim3(1), 1024, 0, stream>>>(r, stats_cut(r.rows, r.V).pieces, s.part, s.at, a, grad ? s.coef : nullptr);
  e = hipGetLastError();
  return e == hipSuccess && grad ? run_grad(r, s, grad, grad_type, ld_grad, stream) : e;
}

hipError_t launch_preference_loss(const LogitRows& r, const PairArgs& a, const Offsets& off, void* grad, int32_t grad_type, int64_t ld_grad, char* ws, hipStream_t stream) {
  const LossSpace s = loss_space(ws, r.rows, r.V);
  hipError_t e = run_stats(r, s, nullptr, stream);
  if (e != hipSuccess) return e;
  int most = 0;
  for (int p = 0; p < a.pairs; ++p) most = off.v[2 * p + 2] - off.v[2 * p] > most ? off.v[2 * p + 2] - off.v[2 * p] : most;
  if (grad && pair_few_rows(r.rows, r.V, most)) return run_few_rows(r, s, PairFew{a, off}, grad, grad_type, ld_grad, stream);
  pair_rows_kernel<<<dim3(1), 1024, 0, stream>>>(r, stats_cut(r.rows, r.V).pieces, s.part, s.at, a, off, s.term, grad ? s.coef : nullptr);
  e = hipGetLastError();
  return e == hipSuccess && grad ? run_grad(r, s, grad, grad_type, ld_grad, stream) : e;
}

}  // namespace nanospec
