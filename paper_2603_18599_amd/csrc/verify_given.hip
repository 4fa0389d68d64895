// Verification of drafted tokens against given probabilities with the caller's
// uniforms (definition: sjd.h).
//
// Bound by memory: only a row that is drawn from needs more than two of its
// entries, and it needs p and q once. One workgroup takes a drawn row: each of 16
// waves sums a contiguous stretch of it in 64 bits, the stretch that holds r *
// total is summed again in 16 parts (it lies in the cache), and a wave finds the
// token in its part. Differences and products of floats are exact or rounded
// once in 64 bits, so another summation order moves a draw only where r * total
// lies within some 1e-15 of the total from a border.
#include "device.h"
#include "ops.h"

namespace sjd {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;

struct GivenArgs {
  sjd_given_params p;
  sjd_given_io io;
};

SJD_DEV double wave_sum64(double v) { return wave_sum_d_dpp(v); }

// The weights of a row
struct Row {
  const float *p, *q;  // q NULL: p alone, but for entry `skip`
  int V, skip;
  SJD_DEV double at(int x) const {
    double d = p[x];
    if (q) d -= (double)q[x];
    else if (x == skip) d = 0.0;
    return d > 0.0 ? d : 0.0;  // (NaN: 0)
  }
};

// Sum of w over [lo, hi) by one wave, and the largest x with mass (-1: none)
SJD_DEV double stretch_sum(const Row& w, int lo, int hi) {
  double s = 0.0;
  for (int x = lo + (threadIdx.x & 63); x < hi; x += kWave) s += w.at(x);
  return wave_sum64(s);
}

struct DrawSmem {
  double seg[kWaves];
  int tok;
};

// Least x with cum(x) > r * total, or -1 for a row without mass (every thread
// gets the result).
SJD_DEV int draw(const Row& w, float r, DrawSmem& sm) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int seg = ((w.V + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;  // entries per wave
  auto sums = [&](int base, int end, int len) {
    const int lo = min(base + wave * len, end), hi = min(lo + len, end);
    const double s = stretch_sum(w, lo, hi);
    __syncthreads();  // (the last round's sums have been read)
    if (lane == 0) sm.seg[wave] = s;
    __syncthreads();
  };
  sums(0, w.V, seg);
  double total = 0.0;
  for (int i = 0; i < kWaves; ++i) total += sm.seg[i];
  if (!(total > 0.0)) return -1;
  const double target = (double)r * total;
  // the part that holds the target: the first whose end lies above it, else
  // (r * total rounded up to the total) the last one with mass
  auto find = [&](double& before) {
    double cum = before, at = before;
    int pick = -1, last = 0;
    double last_before = before;
    for (int i = 0; i < kWaves; ++i) {
      const double s = sm.seg[i];
      if (s > 0.0) { last = i; last_before = cum; }
      if (pick < 0 && cum + s > target && s > 0.0) { pick = i; at = cum; }
      cum += s;
    }
    if (pick < 0) { pick = last; at = last_before; }
    before = at;
    return pick;
  };
  double before = 0.0;
  int base = find(before) * seg, end = min(base + seg, w.V), len = seg;
  while (len > kWave) {
    len = ((len + kWaves - 1) / kWaves + kWave - 1) / kWave * kWave;
    sums(base, end, len);
    base += find(before) * len;
    end = min(base + len, end);
  }
  if (wave == 0) {  // at most 64 entries, in lane order
    const int x = base + lane;
    const double v = x < end ? w.at(x) : 0.0;
    double cum = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const double u = __shfl_up(cum, o, kWave);
      if (lane >= o) cum += u;
    }
    const uint64_t above = __ballot(v > 0.0 && before + cum > target), some = __ballot(v > 0.0);
    if (lane == 0) sm.tok = base + (above ? __builtin_ctzll(above) : 63 - __builtin_clzll(some));
  }
  __syncthreads();
  return sm.tok;
}

// Draft j of window b: accepted?  (*x: its entry, -1 if it is no token of the row)
SJD_DEV bool accepts(const GivenArgs& a, int b, int j, int* x) {
  const int64_t at = (int64_t)b * a.p.L + j;
  const int64_t e = (int64_t)a.io.d_draft[at] - a.p.vis_lo;
  if (e < 0 || e >= a.p.V) {
    *x = -1;
    return false;
  }
  *x = (int)e;
  const double p = a.io.d_p[b * a.p.p_win + j * a.p.p_row + e], u = a.io.d_u[at];
  const double q = a.io.d_q ? (double)a.io.d_q[b * a.p.q_win + j * a.p.q_row + e] : 1.0;
  return u * q < p;
}

// Token drawn at row j (drafts: the residual; x < 0 or row n: p itself)
SJD_DEV int draw_row(const GivenArgs& a, int b, int j, bool residual, int x, DrawSmem& sm) {
  Row w{a.io.d_p + b * a.p.p_win + j * a.p.p_row, nullptr, a.p.V, -1};
  const float r = a.io.d_r[(int64_t)b * (a.p.L + 1) + j];
  int t = -1;
  if (residual) {
    w.q = a.io.d_q ? a.io.d_q + b * a.p.q_win + j * a.p.q_row : nullptr;
    w.skip = x;
    t = draw(w, r, sm);
    w.q = nullptr;
    w.skip = -1;
  }
  if (t < 0) t = draw(w, r, sm);
  return t < 0 ? -1 : t + a.p.vis_lo;
}

SJD_DEV int drafts_of(const GivenArgs& a, int b) {
  const int n = a.io.d_n ? a.io.d_n[b] : a.p.L;
  return n >= 0 && n <= a.p.L ? n : -1;
}

// One window: up to its first rejection.
__global__ __launch_bounds__(kThreads) void k_given_chain(GivenArgs a) {
  __shared__ DrawSmem sm;
  __shared__ int s_first, s_x;
  const int b = blockIdx.x, L = a.p.L, n = drafts_of(a, b);
  int32_t* meta = a.io.d_meta + 4 * (int64_t)b;
  if (n < 0) {
    if (threadIdx.x < 4) meta[threadIdx.x] = threadIdx.x < 2 ? -1 : 0;
    return;
  }
  const int j = threadIdx.x;
  if (j < kWave) {  // (L <= 64: one wave tests every draft)
    int x = -1;
    const bool bad = j < n && !accepts(a, b, j, &x);
    const uint64_t m = __ballot(bad);
    const int first = m ? __builtin_ctzll(m) : n;
    if (bad && j == first) s_x = x;
    if (j == 0) s_first = first;
  }
  __syncthreads();
  const int first = s_first;
  const bool drawn = first < n || (a.p.flags & SJD_BONUS);
  const int t = drawn ? draw_row(a, b, first, first < n && s_x >= 0, s_x, sm) : -1;
  const int n_c = first + (drawn ? 1 : 0);
  if (j <= L)
    a.io.d_tok[(int64_t)b * (L + 1) + j] = j < first ? a.io.d_draft[(int64_t)b * L + j] : j < n_c ? t : -1;
  if (j < L && a.io.d_next) a.io.d_next[(int64_t)b * L + j] = -1;
  if (j == 0) *(int4*)meta = make_int4(n_c, first < n ? first : -1, first, 0);
}

// Adaptive continuation: every row by itself, its token (the draft, or what was
// drawn) into d_tok.
__global__ __launch_bounds__(kThreads) void k_given_rows(GivenArgs a) {
  __shared__ DrawSmem sm;
  const int rows = a.p.L + (a.p.flags & SJD_BONUS ? 1 : 0);
  const int b = blockIdx.x / rows, j = blockIdx.x % rows, n = drafts_of(a, b);
  if (j > n || (j == n && rows == a.p.L)) return;
  int x = -1, t;
  if (j < n && accepts(a, b, j, &x)) t = a.io.d_draft[(int64_t)b * a.p.L + j];
  else t = draw_row(a, b, j, j < n && x >= 0, x, sm);
  if (threadIdx.x == 0) a.io.d_tok[(int64_t)b * (a.p.L + 1) + j] = t;
}
// The rows' tokens into committed ones and next drafts (the accept tests, two
// reads each, are made again rather than stored).
__global__ __launch_bounds__(128) void k_given_end(GivenArgs a) {
  __shared__ int row[65];
  __shared__ int s_first;
  const int b = blockIdx.x, L = a.p.L, n = drafts_of(a, b), j = threadIdx.x;
  int32_t* meta = a.io.d_meta + 4 * (int64_t)b;
  if (n < 0) {
    if (j < 4) meta[j] = j < 2 ? -1 : 0;
    return;
  }
  int32_t* tok = a.io.d_tok + (int64_t)b * (L + 1);
  const int bonus = a.p.flags & SJD_BONUS ? 1 : 0;
  if (j < kWave) {
    int x;
    const uint64_t m = __ballot(j < n && !accepts(a, b, j, &x));
    if (j == 0) s_first = m ? __builtin_ctzll(m) : n;
  }
  if (j < n + bonus) row[j] = tok[j];
  __syncthreads();
  const int first = s_first;
  const int n_c = first < n ? first + 1 : n + bonus;
  if (j <= L) tok[j] = j < n_c ? row[j] : -1;
  const int carried = n + bonus - n_c;
  if (j < L) a.io.d_next[(int64_t)b * L + j] = j < carried ? row[n_c + j] : -1;
  if (j == 0) *(int4*)meta = make_int4(n_c, first < n ? first : -1, first, carried);
}

}  // namespace

hipError_t launch_verify_given(const sjd_given_params& p, const sjd_given_io& io, hipStream_t s) {
  const GivenArgs a{p, io};
  if (p.flags & SJD_AC) {
    const int rows = p.L + (p.flags & SJD_BONUS ? 1 : 0);
    hipLaunchKernelGGL(k_given_rows, dim3(p.B * rows), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(k_given_end, dim3(p.B), dim3(128), 0, s, a);
  } else {
    hipLaunchKernelGGL(k_given_chain, dim3(p.B), dim3(kThreads), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace sjd
