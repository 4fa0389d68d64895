// Rows placed and appended in one call (definition: sjd.h): keys turned by their
// angles on the way into their pages, values beside them, queries turned into the rows
// that the attention reads.
//
// Bound by memory: rows of q, k and v once in, rows of q, codes and exponents once out; as two
// calls k passes through memory twice more, and a short window pays a second launch. An angle
// costs 30 instructions and every head of a row shares it, so a workgroup keeps its rows' (cos,
// sin) in LDS. Keys and values go by tiles of 32 positions as sjd_kv_append's do, queries by
// themselves beside them: one after the other in a workgroup they took 7.3 us for four tokens,
// side by side 4.9 (two calls: 3.7 + 4.2). 10432 rows of 32 and 8 heads of 128 into e4m3 pages
// (234 MB): 55 us from memory, 4.3 TB/s; 43 where calls follow each other on rows that the last
// cache still holds in part (two calls 49); of 32 and 32 heads into bf16 pages 107 (120).
#include "paged_rows.h"

namespace sjd {

namespace {

constexpr int kThreads = 256;

struct PlaceArgs {
  PoolView pv;
  sjd_windows w;
  sjd_kv_rows r;
  const void* q;
  void* out;
  int64_t q_row, out_row;
  const int32_t* pos;
  int H, pairs, axes;
  int HP, YK;      // key / value heads to a workgroup, workgroups of them to a tile
  int R;           // positions of a workgroup of queries
  uint64_t rev[64];       // revolutions per position, their fraction in 2^-64
  uint8_t axis[64];
};

template <class E>
SJD_DEV float elem(E v) {
  if constexpr (sizeof(E) == 2) return bf16_to_f32(v);
  else return v;
}

// (cos, sin) of pos * rev / 2^64 revolutions. A position being whole, the fraction of a
// revolution is what 64 bits keep of the product (a revolution per position that a 64-bit float
// holds is exact in them to 2^-64, which a position multiplies to 2^-33 at most). The nearest
// quarter comes off, and the rest, at most pi / 4, goes through the Taylor series of both (first
// terms left out: t^11 / 11! and t^12 / 12!, below 2^-29). A third of the instructions of 64-bit
// floats and the library's function.
SJD_DEV float2 turn_of(int pos, uint64_t rev) {
  const uint32_t lo = (uint32_t)rev, hi = (uint32_t)(rev >> 32);
  uint32_t ph = __umulhi((uint32_t)pos, lo) + (uint32_t)pos * hi;  // 32 bits of the fraction
  if (pos < 0) ph -= lo;                                           // (pos + 2^32 above)
  const uint32_t quarter = (ph + 0x20000000u) >> 30;
  const int g = (int)(ph - (quarter << 30));
  constexpr float k = 0x1p-32f * 6.283185307179586f;
  const float f = (float)g;
  const float t = __builtin_fmaf(f, k, (float)(g - (int)f) * k), u = t * t;
  float s = __builtin_fmaf(u, 1.0f / 362880.0f, -1.0f / 5040.0f);
  s = __builtin_fmaf(u, s, 1.0f / 120.0f);
  s = __builtin_fmaf(u, s, -1.0f / 6.0f);
  s = __builtin_fmaf(u * t, s, t);
  float c = __builtin_fmaf(u, -1.0f / 3628800.0f, 1.0f / 40320.0f);
  c = __builtin_fmaf(u, c, -1.0f / 720.0f);
  c = __builtin_fmaf(u, c, 1.0f / 24.0f);
  c = __builtin_fmaf(u, c, -0.5f);
  c = __builtin_fmaf(u, c, 1.0f);
  const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -x : x, quarter & 2 ? -y : y);
}

// N consecutive elements as they lie in memory (16-byte aligned): loads that nothing waits for
// until the floats are asked for
template <bool F32, int N>
struct Raw {
  uint4 r[N * (F32 ? 4 : 2) / 16];
  SJD_DEV void load(const void* base, int64_t at) {
    const uint4* p = (const uint4*)((const char*)base + at * (F32 ? 4 : 2));
#pragma unroll
    for (int i = 0; i < N * (F32 ? 4 : 2) / 16; ++i) r[i] = p[i];
  }
  SJD_DEV void get(float (&v)[N]) const {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int w = F32 ? e : e / 2;
      const uint32_t u = w % 4 == 0 ? r[w / 4].x : w % 4 == 1 ? r[w / 4].y : w % 4 == 2 ? r[w / 4].z : r[w / 4].w;
      v[e] = __uint_as_float(F32 ? u : e & 1 ? u & 0xFFFF0000u : u << 16);
    }
  }
};
// The turns of dims j .. j + N - 1 from those of their row's pairs: x, with the other of its pair o,
// becomes x * cos + o * sin, the sine's sign being the first's or the second's of a pair.
// WIDE: pairs is a multiple of 8
template <bool WIDE, int N>
SJD_DEV void turns_of(const float2* cs, int j, int pairs, float2 (&t)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int d = WIDE ? j + (e & ~7) : j + e;  // (of a piece of 8, or each by itself)
    const bool low = d < pairs;
    t[e] = make_float2(1.0f, 0.0f);
    if (d >= 2 * pairs) continue;  // (passes through)
    t[e] = cs[j + e - (low ? 0 : pairs)];
    if (low) t[e].y = -t[e].y;
  }
}
// (the roundings are rotate_pair's). The first `turned` dims; those behind them pass through as they
// are: a product with 0 would make NaN of infinities, and a sum with it +0 of -0
template <int N>
SJD_DEV void turn(const float2 (&t)[N], int turned, float (&x)[N], const float (&o)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) x[e] = e < turned ? __builtin_fmaf(x[e], t[e].x, o[e] * t[e].y) : x[e];
}

template <class E>
SJD_DEV void put(void* out, int64_t at, float v) {
  if constexpr (sizeof(E) == 2) ((uint16_t*)out)[at] = f32_to_bf16(v);
  else ((float*)out)[at] = v;
}

// The angles of positions [lo, hi) of a tile (rows from t0 + lo on), entry of position i, pair p
// at cs[i * turn_row(pairs) + p]: a thread keeps to one pair. (16 bytes more in a row of them:
// eight rows that are read together lie in different banks.)
SJD_DEV int turn_row(int pairs) { return pairs + 2; }
SJD_DEV void angles(const PlaceArgs& a, int64_t t0, int lo, int hi, float2* cs) {
  const int per = kThreads / a.pairs, r0 = threadIdx.x / a.pairs, p = threadIdx.x - r0 * a.pairs;
  if (r0 >= per) return;
  const uint64_t rev = a.rev[p];
  const int32_t* const pos = a.pos + a.axis[p];
  for (int r = lo + r0; r < hi; r += per) cs[r * turn_row(a.pairs) + p] = turn_of(pos[(t0 + r) * a.axes], rev);
}

// grid (tile of 32 positions, YK groups of HP key / value heads and then parts of R of the tile's
// queries, sequence)
template <int HD, bool FP8, bool F32, bool OUT32, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_append_rope(PlaceArgs a) {
  constexpr int ES = FP8 ? 1 : 2, N = HD / 8, W = WIDE ? 8 : 1;
  using E = std::conditional_t<F32, float, uint16_t>;
  using O = std::conditional_t<OUT32, float, uint16_t>;
  __shared__ __align__(16) char vs[32 * HD * ES * 17 / 16];
  __shared__ __align__(16) float2 cs[32 * (HD / 2 + 2)];
  const int z = blockIdx.z;
  const Seq sq = load_seq(a.w, a.pv, z);
  const int p0 = ((sq.cached >> 5) + (int)blockIdx.x) << 5;
  if (sq.rows == 0 || p0 >= sq.cached + sq.rows) return;
  int lo = max(0, sq.cached - p0), hi = min(32, sq.cached + sq.rows - p0);  // positions that the window holds
  const int64_t t0 = sq.row0 + (p0 - sq.cached);                            // row of the tile's position 0

  if ((int)blockIdx.y < a.YK) {  // keys and values
    char* const page = page_of(a.w, a.pv, z, p0);
    if (!page) return;
    const int i = threadIdx.x >> 3, c = threadIdx.x & 7;
    const bool ok = i >= lo && i < hi;
    const int64_t t = t0 + i;
    const int end = min((int)(blockIdx.y + 1) * a.HP, a.pv.Hkv);
    int h = blockIdx.y * a.HP;
    // a head's rows, and of WIDE rows the other of each pair (in pieces of 8), ahead of their use:
    // the first ones before the angles, which cover the latency
    Raw<F32, N> kr, vr;
    Raw<F32, 8> ko[N / 8];
    auto load = [&] {
      if (!ok) return;
      const int64_t at = t * a.r.k_row + h * HD;
      kr.load(a.r.d_k, at + c * N);
      vr.load(a.r.d_v, t * a.r.v_row + h * HD + c * N);
      if constexpr (WIDE) {
#pragma unroll
        for (int g = 0; g < N / 8; ++g) {
          const int j = c * N + 8 * g;
          ko[g].load(a.r.d_k, at + (j < a.pairs ? j + a.pairs : j < 2 * a.pairs ? j - a.pairs : j));
        }
      }
    };
    load();
    angles(a, t0, lo, hi, cs);
    __syncthreads();
    float2 turns[N];  // the same for every head
    if (ok) turns_of<WIDE, N>(cs + i * turn_row(a.pairs), c * N, a.pairs, turns);
    for (;;) {
      float kf[N] = {}, vf[N] = {};
      if (ok) {
        float o[N];
        kr.get(kf);
        vr.get(vf);
        if constexpr (WIDE) {
#pragma unroll
          for (int g = 0; g < N / 8; ++g) {
            float v[8];
            ko[g].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[8 * g + e] = v[e];
          }
        } else {
          const E* k = (const E*)a.r.d_k + t * a.r.k_row + h * HD;
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const int j = c * N + e;
            o[e] = j < 2 * a.pairs ? elem(k[j < a.pairs ? j + a.pairs : j - a.pairs]) : 0.0f;
          }
        }
        turn<N>(turns, 2 * a.pairs - c * N, kf, o);
      }
      const int now = h;
      if (++h < end) load();
      store_tile<HD, FP8>(a.pv, page, now, p0 & ((1 << a.pv.plen_log2) - 1), lo, hi, ok, kf, vf, vs);
      if (h >= end) return;
      __syncthreads();  // (the values' tile in LDS is read until here)
    }
  }

  // Queries of R positions: a piece is W pairs, or dims that pass through (rows turned in place keep
  // them): eight, or one up to the first aligned eight; a thread keeps to one place of the heads
  const int part = (int)blockIdx.y - a.YK;
  lo = max(lo, a.R * part);
  hi = min(hi, a.R * part + a.R);
  if (lo >= hi) return;
  const int np = a.pairs / W, ones = -2 * a.pairs & 7, rest = a.out == a.q ? 0 : ones + (HD - 2 * a.pairs) / 8;
  const int per = np + rest;
  const int step = kThreads / per, g0 = threadIdx.x / per, place = threadIdx.x - g0 * per;
  const int total = g0 < step ? (hi - lo) * a.H : 0;
  const bool eight = place >= np + ones;  // (WIDE: ones is 0)
  const int j = place < np ? place * W : 2 * a.pairs + (eight ? ones + (place - np - ones) * 8 : place - np);
  if constexpr (WIDE) {
    // two pieces at a time, ahead of their use, the first ones before the angles (one, loaded when
    // it is needed: 62 us for the rows above; four: 58)
    constexpr int U = 2;
    Raw<F32, 8> x[U], y[U];
    int r[U], h[U];
    const int other = place < np ? a.pairs : 0;
    // (no branches: a wait would be for all that is under way. Items past the last read it again)
    auto load = [&](int g) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = min(g + u * step, (hi - lo) * a.H - 1);
        r[u] = at / a.H;
        h[u] = at - r[u] * a.H;
        r[u] += lo;
        const int64_t src = (t0 + r[u]) * a.q_row + h[u] * HD + j;
        x[u].load(a.q, src);
        y[u].load(a.q, src + other);
      }
    };
    load(g0);
    angles(a, t0, lo, hi, cs);
    __syncthreads();
    for (int g = g0; g < total; g += U * step) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (g + u * step >= total) break;
        const int64_t dst = (t0 + r[u]) * a.out_row + h[u] * HD + j;
        const float2* const turns = cs + r[u] * turn_row(a.pairs) + place * W;
        float p[8], q[8];
        x[u].get(p);
        if (place < np) {
          y[u].get(q);
#pragma unroll
          for (int e = 0; e < 8; ++e) rotate_pair(p[e], q[e], turns[e], p[e], q[e]);
          store_row<OUT32, 8>(a.out, dst + a.pairs, q);
        }
        store_row<OUT32, 8>(a.out, dst, p);
      }
      if (g + U * step < total) load(g + U * step);
    }
  } else {
    angles(a, t0, lo, hi, cs);
    __syncthreads();
    for (int g = g0; g < total; g += step) {
      const int r = lo + g / a.H, h = g % a.H;
      const int64_t src = (t0 + r) * a.q_row + h * HD, dst = (t0 + r) * a.out_row + h * HD;
      if (eight) {
        float x[8];
        load_row<F32, 8>(a.q, src + j, x);
        store_row<OUT32, 8>(a.out, dst + j, x);
        continue;
      }
      const E* q = (const E*)a.q + src;
      float u = elem(q[j]), v;
      if (place < np) {
        rotate_pair(u, elem(q[a.pairs + j]), cs[r * turn_row(a.pairs) + place * W], u, v);
        put<O>(a.out, dst + a.pairs + j, v);
      }
      put<O>(a.out, dst + j, u);
    }
  }
}

}  // namespace

hipError_t launch_kv_append_rope(const sjd_pages& p, const sjd_windows& w, const sjd_kv_rows& r, const sjd_append_rope& o,
                                 hipStream_t s) {
  PlaceArgs a{};
  a.pv = pool_view(p); a.w = w; a.r = r;
  a.q = o.d_q; a.out = o.d_out_q; a.q_row = o.q_row; a.out_row = o.out_q_row; a.pos = o.d_pos;
  a.H = o.H; a.pairs = o.pairs; a.axes = o.axes;
  for (int i = 0; i < o.pairs; ++i) {
    // (of the size: a fraction of a negative number would round)
    const double v = std::fabs(o.h_freq[i] / 6.283185307179586476925286766559);
    const uint64_t u = (uint64_t)((v - std::floor(v)) * 0x1p64);
    a.rev[i] = o.h_freq[i] < 0 ? 0 - u : u;
    a.axis[i] = o.h_axis[i];
  }
  // Up to four heads share a tile's angles, and four positions' queries theirs, where that leaves
  // two workgroups of either kind to a compute unit (10432 rows of 32 and 8 heads, us: one head 63,
  // two 58, four 55, and with queries of eight positions 58, of sixteen 61; of 32 and 32 heads:
  // four 107, sixteen, which follow each other, 126)
  const int64_t tiles = (w.max_rows + 62) / 32;
  a.HP = 1;
  while (a.HP < 4 && a.HP < p.n_kv_heads && tiles * w.B * ((p.n_kv_heads + 2 * a.HP - 1) / (2 * a.HP)) >= 512) a.HP *= 2;
  a.YK = (p.n_kv_heads + a.HP - 1) / a.HP;
  for (a.R = 4; a.R > 1 && tiles * w.B * (32 / a.R) < 512;) a.R /= 2;
  const dim3 grid(tiles, a.YK + (o.H ? 32 / a.R : 0), w.B), block(kThreads);
  auto go = [&](auto hd, auto fp8, auto f32, auto out32, auto wide) {
    hipLaunchKernelGGL((k_append_rope<decltype(hd)::value, decltype(fp8)::value, decltype(f32)::value,
                                      decltype(out32)::value, decltype(wide)::value>),
                       grid, block, 0, s, a);
  };
  auto pick = [](bool b, auto f) { b ? f(std::true_type{}) : f(std::false_type{}); };
  pick(p.head_dim == 128, [&](auto big) {
    const std::integral_constant<int, decltype(big)::value ? 128 : 64> hd;
    pick(p.dtype == SJD_E4M3, [&](auto fp8) {
      pick(r.dtype == SJD_F32, [&](auto f32) {
        pick(o.out_dtype == SJD_F32, [&](auto out32) {
          pick(o.pairs % 8 == 0, [&](auto wide) { go(hd, fp8, f32, out32, wide); });
        });
      });
    });
  });
  return hipGetLastError();
}

}  // namespace sjd
