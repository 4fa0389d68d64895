// Rows placed and appended in one call (definition: sjd.h): keys turned by their
// angles on the way into their pages, values beside them, queries turned into the rows
// that the attention reads.
#include "paged_rows.h"

namespace sjd {

namespace {

struct PlaceArgs {
  PoolView pv;
  sjd_windows w;
  sjd_kv_rows r;
  const void* q;
  void* out;
  int64_t q_row, out_row;
  const int32_t* pos;
  int H, G, pairs, axes;  // G query heads to a workgroup
  double rev[64];         // revolutions per position
  uint8_t axis[64];
};

template <class E>
SJD_DEV float elem(E v) {
  if constexpr (sizeof(E) == 2) return bf16_to_f32(v);
  else return v;
}

// (cos, sin) of v revolutions, v reduced to [-1/2, 1/2] in 64 bits; what a float loses
// of it turns the result by its first order (an angle would be 2^-24 off otherwise,
// twice a rounding of the result)
SJD_DEV float2 turn_of(double v) {
  v -= rint(v);
  const float f = (float)v, d = (float)(v - (double)f) * 6.283185307179586f;
  float s, c;
  sincospif(2.0f * f, &s, &c);
  return make_float2(__builtin_fmaf(-d, s, c), __builtin_fmaf(d, c, s));
}

// N dims of a row from dim j, turned. cs: of the row's pairs. WIDE: pairs is a multiple of 8
template <bool F32, bool WIDE, int N>
SJD_DEV void turned(const void* base, int64_t at, int j, int pairs, const float2* cs, float (&x)[N]) {
  using E = std::conditional_t<F32, float, uint16_t>;
  load_row<F32, N>(base, at + j, x);
#pragma unroll
  for (int g = 0; g < N; g += 8) {
    const int jg = j + g;
    if constexpr (WIDE) {
      if (jg >= 2 * pairs) continue;
      const bool low = jg < pairs;
      const int p = low ? jg : jg - pairs;
      float o[8];
      load_row<F32, 8>(base, at + (low ? jg + pairs : p), o);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float u, v;
        rotate_pair(low ? x[g + e] : o[e], low ? o[e] : x[g + e], cs[p + e], u, v);
        x[g + e] = low ? u : v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int je = jg + e;
        if (je >= 2 * pairs) continue;
        const bool low = je < pairs;
        const int p = low ? je : je - pairs;
        const float o = elem(((const E*)base)[at + (low ? je + pairs : p)]);
        float u, v;
        rotate_pair(low ? x[g + e] : o, low ? o : x[g + e], cs[p], u, v);
        x[g + e] = low ? u : v;
      }
    }
  }
}

template <class E>
SJD_DEV void put(void* out, int64_t at, float v) {
  if constexpr (sizeof(E) == 2) ((uint16_t*)out)[at] = f32_to_bf16(v);
  else ((float*)out)[at] = v;
}

// grid (tile, key / value head, sequence)
template <int HD, bool FP8, bool F32, bool OUT32, bool WIDE>
__global__ __launch_bounds__(256) void k_append_rope(PlaceArgs a) {
  constexpr int ES = FP8 ? 1 : 2, N = HD / 8;
  using E = std::conditional_t<F32, float, uint16_t>;
  using O = std::conditional_t<OUT32, float, uint16_t>;
  __shared__ __align__(16) char vs[32 * HD * ES * 17 / 16];
  __shared__ float2 cs[32 * (HD / 2)];
  const int z = blockIdx.z, h = blockIdx.y;
  const Seq sq = load_seq(a.w, a.pv, z);
  const int p0 = ((sq.cached >> 5) + (int)blockIdx.x) << 5;
  if (sq.rows == 0 || p0 >= sq.cached + sq.rows) return;
  const int lo = max(0, sq.cached - p0), hi = min(32, sq.cached + sq.rows - p0);  // positions that the window holds
  const int64_t t0 = sq.row0 + (p0 - sq.cached);                                  // row of the tile's position 0
  for (int i = threadIdx.x; i < (hi - lo) * a.pairs; i += 256) {
    const int r = i / a.pairs, p = i - r * a.pairs;
    cs[(lo + r) * a.pairs + p] = turn_of((double)a.pos[(t0 + lo + r) * a.axes + a.axis[p]] * a.rev[p]);
  }
  __syncthreads();
  char* page = page_of(a.w, a.pv, z, p0);
  if (page) {
    const int i = threadIdx.x >> 3, c = threadIdx.x & 7;
    const bool ok = i >= lo && i < hi;
    float kf[N] = {}, vf[N] = {};
    if (ok) {
      const int64_t t = t0 + i;
      turned<F32, WIDE, N>(a.r.d_k, t * a.r.k_row + h * HD, c * N, a.pairs, cs + i * a.pairs, kf);
      load_row<F32, N>(a.r.d_v, t * a.r.v_row + h * HD + c * N, vf);
    }
    store_tile<HD, FP8>(a.pv, page, h, p0 & ((1 << a.pv.plen_log2) - 1), lo, hi, ok, kf, vf, vs);
  }
  // queries: a piece is W pairs, or W dims that pass through (rows turned in place keep them)
  constexpr int W = WIDE ? 8 : 1;
  const int h0 = h * a.G, heads = min(a.G, a.H - h0);
  if (heads <= 0) return;
  const int np = a.pairs / W, rest = a.out == a.q ? 0 : (HD - 2 * a.pairs) / W, per = np + rest;
  for (int u = threadIdx.x; u < (hi - lo) * heads * per; u += 256) {
    const int c = u % per, rh = u / per, i = lo + rh / heads, hq = h0 + rh % heads;
    const int64_t t = t0 + i, src = t * a.q_row + hq * HD, dst = t * a.out_row + hq * HD;
    float x[W], y[W];
    if constexpr (WIDE) {
      if (c >= np) {
        const int j = 2 * a.pairs + (c - np) * 8;
        load_row<F32, 8>(a.q, src + j, x);
        store_row<OUT32, 8>(a.out, dst + j, x);
        continue;
      }
      load_row<F32, 8>(a.q, src + c * 8, x);
      load_row<F32, 8>(a.q, src + a.pairs + c * 8, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float p, q;
        rotate_pair(x[e], y[e], cs[i * a.pairs + c * 8 + e], p, q);
        x[e] = p;
        y[e] = q;
      }
      store_row<OUT32, 8>(a.out, dst + c * 8, x);
      store_row<OUT32, 8>(a.out, dst + a.pairs + c * 8, y);
    } else {
      const E* q = (const E*)a.q + src;
      if (c >= np) {
        const int j = 2 * a.pairs + c - np;
        put<O>(a.out, dst + j, elem(q[j]));
        continue;
      }
      float p, v;
      rotate_pair(elem(q[c]), elem(q[a.pairs + c]), cs[i * a.pairs + c], p, v);
      put<O>(a.out, dst + c, p);
      put<O>(a.out, dst + a.pairs + c, v);
    }
  }
}

}  // namespace

hipError_t launch_kv_append_rope(const sjd_pages& p, const sjd_windows& w, const sjd_kv_rows& r, const sjd_append_rope& o,
                                 hipStream_t s) {
  PlaceArgs a{};
  a.pv = pool_view(p); a.w = w; a.r = r;
  a.q = o.d_q; a.out = o.d_out_q; a.q_row = o.q_row; a.out_row = o.out_q_row; a.pos = o.d_pos;
  a.H = o.H; a.G = (o.H + p.n_kv_heads - 1) / p.n_kv_heads; a.pairs = o.pairs; a.axes = o.axes;
  for (int i = 0; i < o.pairs; ++i) {
    a.rev[i] = o.h_freq[i] / 6.283185307179586476925286766559;
    a.axis[i] = o.h_axis[i];
  }
  const dim3 grid((w.max_rows + 62) / 32, p.n_kv_heads, w.B), block(256);
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
