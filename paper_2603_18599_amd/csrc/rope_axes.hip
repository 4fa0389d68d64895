// Rotary positions with several axes: rows of q and k, a pair (dims i and pairs
// + i of a head) turned by the angle pos[axis_i] * freq_i.
//
// Bound by memory: each row is read and written once (at 2 bytes an element, 6
// operations per pair of 8 bytes). An angle costs more than a turn, 40
// instructions with the reduction to one revolution in 64 bits, and every head of
// a row shares it, so a workgroup first fills a table in LDS with the (cos, sin)
// of its rows' pairs, one entry per thread, and then streams the heads in 16-byte
// pieces. 8190 rows of 32 + 8 heads of 128 (168 MB): 35 us, 4.8 TB/s, a copy's rate; one
// row 4.1 us.
#include "device.h"
#include "ops.h"

namespace sjd {

namespace {

struct RopeArgs {
  const void *q, *k;
  const int32_t* pos;
  void *oq, *ok;
  int64_t q_row, k_row, oq_row, ok_row;
  int T, H, Hkv, hd, pairs, axes, R;
  float sign;
  double rev[128];  // revolutions per position
  uint8_t axis[128];
};

template <class E>
SJD_DEV float to_f32(E v) {
  if constexpr (sizeof(E) == 2) return bf16_to_f32(v);
  else return v;
}
template <class E>
SJD_DEV E from_f32(float v) {
  if constexpr (sizeof(E) == 2) return f32_to_bf16(v);
  else return v;
}

template <class E, int W>
struct alignas(sizeof(E) * W) Piece {
  E v[W];
};

// E: element (uint16_t bf16, float); W elements per access (1, or 16 bytes)
template <class E, int W>
__global__ __launch_bounds__(256) void k_rope_axes(RopeArgs a) {
  __shared__ __align__(16) float2 cs[256];  // rows * pairs <= 256
  using P = Piece<E, W>;
  const int t0 = blockIdx.x * a.R, rows = min(a.R, a.T - t0);
  for (int i = threadIdx.x; i < rows * a.pairs; i += 256) {
    const int r = i / a.pairs, p = i - r * a.pairs;
    // revolutions, reduced to [-1/2, 1/2] before they leave 64 bits
    const double v = (double)a.pos[(int64_t)(t0 + r) * a.axes + a.axis[p]] * a.rev[p];
    float s, c;
    sincospif(2.0f * (float)(v - rint(v)), &s, &c);
    cs[i] = make_float2(c, a.sign * s);
  }
  __syncthreads();
  // a head: its pairs in W at a time, then (unless the tensor is turned in
  // place) the dims that pass through
  const int np = a.pairs / W, rest = (a.hd - 2 * a.pairs) / W, heads = a.H + a.Hkv;
  const int per = np + rest, total = rows * heads * per;
  for (int i = threadIdx.x; i < total; i += 256) {
    const int c = i % per, rh = i / per, h = rh % heads, r = rh / heads;
    const bool isq = h < a.H;
    const int64_t t = t0 + r;
    const int hh = isq ? h : h - a.H;
    const E* src = (const E*)(isq ? a.q : a.k) + t * (isq ? a.q_row : a.k_row) + hh * a.hd;
    E* dst = (E*)(isq ? a.oq : a.ok) + t * (isq ? a.oq_row : a.ok_row) + hh * a.hd;
    if (c >= np) {
      if (src != dst) {
        const int j = 2 * a.pairs + (c - np) * W;
        *(P*)(dst + j) = *(const P*)(src + j);
      }
      continue;
    }
    const int j = c * W;
    const P x = *(const P*)(src + j), y = *(const P*)(src + a.pairs + j);
    P o0, o1;
#pragma unroll
    for (int e = 0; e < W; ++e) {
      float u, v;
      rotate_pair(to_f32<E>(x.v[e]), to_f32<E>(y.v[e]), cs[r * a.pairs + j + e], u, v);
      o0.v[e] = from_f32<E>(u);
      o1.v[e] = from_f32<E>(v);
    }
    *(P*)(dst + j) = o0;
    *(P*)(dst + a.pairs + j) = o1;
  }
}

}  // namespace

hipError_t launch_rope_axes(const sjd_rope_params& p, const sjd_rope_io& io, hipStream_t s) {
  RopeArgs a{};
  a.q = io.d_q; a.k = io.d_k; a.pos = io.d_pos; a.oq = io.d_out_q; a.ok = io.d_out_k;
  a.q_row = p.q_row; a.k_row = p.k_row; a.oq_row = p.out_q_row; a.ok_row = p.out_k_row;
  a.T = p.T; a.H = p.H; a.Hkv = p.Hkv; a.hd = p.head_dim; a.pairs = p.pairs; a.axes = p.axes;
  a.sign = p.inverse ? -1.0f : 1.0f;
  for (int i = 0; i < p.pairs; ++i) {
    a.rev[i] = p.h_freq[i] / 6.283185307179586476925286766559;
    a.axis[i] = p.h_axis[i];
  }
  // rows per workgroup: as many as give each thread one angle, unless that
  // leaves compute units without rows
  a.R = 256 / p.pairs < 1 ? 1 : 256 / p.pairs > 8 ? 8 : 256 / p.pairs;
  if (p.T < 256 * a.R) a.R = 1;
  const int grid = (p.T + a.R - 1) / a.R;
  // 16-byte accesses where every part of every head starts on one
  auto fine = [&](const void* x, int64_t row, int W) { return ((uintptr_t)x & 15) == 0 && row % W == 0; };
  const int W = p.dtype == SJD_F32 ? 4 : 8;
  const bool wide = p.pairs % W == 0 && p.head_dim % W == 0 &&
                    (!p.H || (fine(io.d_q, p.q_row, W) && fine(io.d_out_q, p.out_q_row, W))) &&
                    (!p.Hkv || (fine(io.d_k, p.k_row, W) && fine(io.d_out_k, p.out_k_row, W)));
  if (p.dtype == SJD_F32) {
    if (wide) hipLaunchKernelGGL((k_rope_axes<float, 4>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_rope_axes<float, 1>), dim3(grid), dim3(256), 0, s, a);
  } else {
    if (wide) hipLaunchKernelGGL((k_rope_axes<uint16_t, 8>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_rope_axes<uint16_t, 1>), dim3(grid), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace sjd
