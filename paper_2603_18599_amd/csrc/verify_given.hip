// Verification of drafted tokens against given probabilities with the caller's
// uniforms (definition: sjd.h).
//
// Bound by memory: only a row that is drawn from needs more than two of its
// entries, and it needs p and q once. One workgroup of W waves takes a drawn row:
// each wave sums a contiguous stretch of it in 64 bits, with 8 16-byte loads per
// lane in flight; the stretch that holds r * total is read again (it lies in the
// cache), 4 entries to a lane, and a wave finds the token in its 256. Differences
// and products of floats are exact or rounded once in 64 bits, so another summation
// order moves a draw only where r * total lies within some 1e-15 of the total from
// a border.
#include "device.h"
#include "ops.h"

namespace sjd {

namespace {

struct GivenArgs {
  sjd_given_params p;
  sjd_given_io io;
};

SJD_DEV double wave_sum64(double v) { return wave_sum_d_dpp(v); }

// Four entries of a row, which may start on any float (16-byte loads need 4-byte
// alignment only)
struct Four {
  float x, y, z, w;
};

// The weights of a row
struct Row {
  const float *p, *q;  // q NULL: p alone, but for entry `skip`
  int V, skip;
  SJD_DEV double weight(int x, float pv, float qv) const {
    const double d = q ? (double)pv - (double)qv : x == skip ? 0.0 : (double)pv;
    return d > 0.0 ? d : 0.0;  // (NaN: 0)
  }
  // entries x .. x + 3, those from `end` on as zeros
  SJD_DEV void four(int x, int end, Four& a, Four& b) const {
    a = b = Four{0, 0, 0, 0};
    if (x + 4 <= end) {
      a = *(const Four*)(p + x);
      if (q) b = *(const Four*)(q + x);
    } else {
      float* u = &a.x;
      float* v = &b.x;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (x + i < end) {
          u[i] = p[x + i];
          if (q) v[i] = q[x + i];
        }
    }
  }
  SJD_DEV void weights(int x, const Four& a, const Four& b, double (&w)[4]) const {
    w[0] = weight(x, a.x, b.x);
    w[1] = weight(x + 1, a.y, b.y);
    w[2] = weight(x + 2, a.z, b.z);
    w[3] = weight(x + 3, a.w, b.w);
  }
  // sum over [lo, hi) by one wave
  SJD_DEV double sum(int lo, int hi) const {
    double s = 0.0;
    for (int x0 = lo + 4 * (int)(threadIdx.x & 63); x0 < hi; x0 += 16 * kWave) {
      Four a[4], b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) four(x0 + 4 * kWave * i, hi, a[i], b[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        double w[4];
        weights(x0 + 4 * kWave * i, a[i], b[i], w);
        s += (w[0] + w[1]) + (w[2] + w[3]);
      }
    }
    return wave_sum64(s);
  }
};

template <int W>
struct DrawSmem {
  double part[2][W];
  int tok;
};

// The first of n parts whose end lies above the target (parts from `before` on), else
// (r * total rounded up to the total) the last one with mass; `before` becomes what
// lies before it.
template <int N>
SJD_DEV int find(const double* part, double target, double& before) {
  double cum = before, at = before, last_at = before;
  int pick = -1, last = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const double s = part[i];
    if (s > 0.0) {
      last = i;
      last_at = cum;
      if (pick < 0 && cum + s > target) {
        pick = i;
        at = cum;
      }
    }
    cum += s;
  }
  before = pick < 0 ? last_at : at;
  return pick < 0 ? last : pick;
}

// Least x with cum(x) > r * total, or -1 for a row without mass (every thread
// gets the result). Rounds of sums narrow the row down to what the waves can hold in
// registers, 1024 entries each; that round ends in one wave.
template <int W>
SJD_DEV int draw(const Row& w, float r, DrawSmem<W>& sm) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  constexpr int kGroup = 4 * kWave, kGroups = 4, kPart = kGroups * kGroup;
  // entries per wave; a round leaves at most the W-th part of what it began with, or
  // kPart (a row for one wave has no more than that)
  auto split = [](int len) { return ((len + W - 1) / W + kPart - 1) / kPart * kPart; };
  int round = 0;
  double target = 0.0, before = 0.0;
  int base = 0, end = w.V, len = split(w.V);
  // (two buffers: a round's sums are read while the next one writes its own, and the
  // barrier between them is enough)
  for (;; len = split(len)) {
    const int lo = min(base + wave * len, end), hi = min(lo + len, end);
    double* part = sm.part[round & 1];
    double x[kGroups][4], own[kGroups], group[kGroups], s = 0.0;
    if (len > kPart) {
      s = w.sum(lo, hi);
    } else {
      Four a[kGroups], b[kGroups];
#pragma unroll
      for (int i = 0; i < kGroups; ++i) w.four(lo + kGroup * i + 4 * lane, hi, a[i], b[i]);
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        w.weights(lo + kGroup * i + 4 * lane, a[i], b[i], x[i]);
        own[i] = (x[i][0] + x[i][1]) + (x[i][2] + x[i][3]);
        group[i] = lo + kGroup * i < hi ? wave_sum64(own[i]) : 0.0;
        s += group[i];
      }
    }
    if (lane == 0) part[wave] = s;
    __syncthreads();
    if (round++ == 0) {
      double total = 0.0;
      for (int i = 0; i < W; ++i) total += part[i];
      if (!(total > 0.0)) {
        __syncthreads();  // (a draw that follows writes the same buffer)
        return -1;
      }
      target = (double)r * total;
    }
    const int pick = find<W>(part, target, before);
    if (len > kPart) {
      base += pick * len;
      end = min(base + len, end);
      continue;
    }
    if (wave == pick) {
      const int g = find<kGroups>(group, target, before);
      double y[4] = {}, mine = 0.0;
#pragma unroll
      for (int i = 0; i < kGroups; ++i)
        if (i == g) {
          mine = own[i];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = x[i][e];
        }
      double cum = mine;
#pragma unroll
      for (int o = 1; o < kWave; o <<= 1) {
        const double u = __shfl_up(cum, o, kWave);
        if (lane >= o) cum += u;
      }
      const uint64_t above = __ballot(mine > 0.0 && before + cum > target), some = __ballot(mine > 0.0);
      if (lane == (above ? __builtin_ctzll(above) : 63 - __builtin_clzll(some))) {
        double c = before + (cum - mine);
        int t = -1, last = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          c += y[i];
          if (y[i] > 0.0) last = i;
          if (t < 0 && y[i] > 0.0 && c > target) t = i;
        }
        sm.tok = lo + kGroup * g + 4 * lane + (t < 0 ? last : t);
      }
    }
    __syncthreads();
    return sm.tok;
  }
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
template <int W>
SJD_DEV int draw_row(const GivenArgs& a, int b, int j, bool residual, int x, DrawSmem<W>& sm) {
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
template <int W>
__global__ __launch_bounds__(W * kWave) void k_given_chain(GivenArgs a) {
  __shared__ DrawSmem<W> sm;
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
  const int t = drawn ? draw_row<W>(a, b, first, first < n && s_x >= 0, s_x, sm) : -1;
  const int n_c = first + (drawn ? 1 : 0);
  for (int i = j; i <= L; i += W * kWave) {  // (L + 1 may be one more than a wave)
    a.io.d_tok[(int64_t)b * (L + 1) + i] = i < first ? a.io.d_draft[(int64_t)b * L + i] : i < n_c ? t : -1;
    if (i < L && a.io.d_next) a.io.d_next[(int64_t)b * L + i] = -1;
  }
  if (j == 0) *(int4*)meta = make_int4(n_c, first < n ? first : -1, first, 0);
}

// Adaptive continuation: every row by itself, its token (the draft, or what was
// drawn) into d_tok.
template <int W>
__global__ __launch_bounds__(W * kWave) void k_given_rows(GivenArgs a) {
  __shared__ DrawSmem<W> sm;
  const int rows = gridDim.x, b = blockIdx.y, j = blockIdx.x, n = drafts_of(a, b);
  if (j > n || (j == n && rows == a.p.L)) return;
  int x = -1, t;
  if (j < n && accepts(a, b, j, &x)) t = a.io.d_draft[(int64_t)b * a.p.L + j];
  else t = draw_row<W>(a, b, j, j < n && x >= 0, x, sm);
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

template <int W>
void launch(const GivenArgs& a, hipStream_t s) {
  if (a.p.flags & SJD_AC) {
    const int rows = a.p.L + (a.p.flags & SJD_BONUS ? 1 : 0);
    // (in two dimensions: all rows' threads in one may pass 2^32)
    hipLaunchKernelGGL(k_given_rows<W>, dim3(rows, a.p.B), dim3(W * kWave), 0, s, a);
    hipLaunchKernelGGL(k_given_end, dim3(a.p.B), dim3(128), 0, s, a);
  } else {
    hipLaunchKernelGGL(k_given_chain<W>, dim3(a.p.B), dim3(W * kWave), 0, s, a);
  }
}

}  // namespace

hipError_t launch_verify_given(const sjd_given_params& p, const sjd_given_io& io, hipStream_t s) {
  const GivenArgs a{p, io};
  // Waves per row: 1024 entries each are one round. us with 1 / 4 / 16 of them: 6475
  // rows of 236 entries 9.5 / 15 / 62; 3190 of 5795 - / 17 / 37; 1000 of 12000 - / 27 /
  // 34; 32 of 16384 - / 11.6 / 9.6; 256 of 65536 - / 44 / 27 (134 MB: 5.0 TB/s).
  if (p.V <= 1024) launch<1>(a, s);
  else if (p.V <= 12288) launch<4>(a, s);
  else launch<16>(a, s);
  return hipGetLastError();
}

}  // namespace sjd
