// Rows as 8-bit integers with a scale each (definition: sjd.h), the input of the
// products in matmul_i8.hip, with what stands in front of a projection: an RMSNorm or
// the gate of a gated layer.
//
// Bound by memory: a row is read once, stays in registers while its norm and its largest value
// are found, and leaves as codes. A wave has a row of up to 2048 inputs, which needs no barrier, a
// workgroup a longer one or one of few; many rows fill the card by themselves, few are bound by the launch and
// the chain load - sum - largest - store (a row of 4096: 2.4 us, 128 gated rows of 11008: 5.4; 2000
// rows of 20000 behind a norm 42, more than 32768 inputs pass through scratch in part). Calls in a row
// on rows that the last cache holds in part: 4096 gated rows of 11008 42 us, 5.4 TB/s, 4096 x 4096 behind a
// norm 12.5; between other work the latter takes 15.4 to 18.6.
#include <algorithm>
#include <type_traits>

#include "device.h"
#include "ops.h"
#include "rows_i8.h"

namespace sjd {

namespace {

template <int N>
using Int = std::integral_constant<int, N>;

struct QuantArgs {
  const void *x, *norm, *gate;
  int8_t* code;
  float* scale;
  int64_t x_row, gate_row, code_row;
  int T, K;
  int norm_f32;
  float inv_k, eps;
};

// Elements k .. k + 7 of a row, zeros behind K. Rows may start at any element: a piece is
// loaded at the alignment of one.
template <class E>
SJD_DEV void load8(const E* row, int k, int K, float (&v)[8]) {
  if (k + 8 <= K) {
    E x[8];
    __builtin_memcpy(x, row + k, sizeof x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = elem_f32(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k + e < K ? elem_f32(row[k + e]) : 0.0f;
  }
}

// NT threads hold a row in P pieces of 8 elements each; a wave per row (four to a
// workgroup) needs no barrier. E: element (uint16_t bf16, float)
template <class E, int NT, int P, bool NORM, bool GATE>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void k_quantise(QuantArgs a) {
  __shared__ float red[NT / kWave];
  __shared__ uint32_t redu[NT / kWave];
  const int64_t g = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, t = NT == kWave ? g * 4 + (threadIdx.x >> 6) : g;
  if (t >= a.T) return;
  const int tid = threadIdx.x % NT, cols = (a.K + 15) & ~15;
  const E* x = (const E*)a.x + t * a.x_row;
  float y[P][8];
#pragma unroll
  for (int i = 0; i < P; ++i) load8(x, (tid + i * NT) * 8, a.K, y[i]);
  bool bad = false;
  if constexpr (NORM) {
    float ss = 0.0f;
    if constexpr (NT == kWave) {  // (in the order of a workgroup with a piece a thread)
#pragma unroll
      for (int i = 0; i < P; ++i) {
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) part = __builtin_fmaf(y[i][e], y[i][e], part);
        ss += wave_sum(part);
      }
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(y[i][e], y[i][e], ss);
      ss = block_sum<NT>(ss, red);
    }
    bad = !(ss < INFINITY);
    const float rinv = 1.0f / sqrtf(ss * a.inv_k + a.eps);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int k = (tid + i * NT) * 8;
      float g[8];
      if (a.norm_f32) load8((const float*)a.norm, k, a.K, g);
      else load8((const uint16_t*)a.norm, k, a.K, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[i][e] = y[i][e] * rinv * g[e];
    }
  }
  if constexpr (GATE) {
    const E* gate = (const E*)a.gate + t * a.gate_row;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      float g[8];
      load8(gate, (tid + i * NT) * 8, a.K, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[i][e] *= silu(g[e]);
    }
  }
  uint32_t m = 0;  // (as bits: NaN is above infinity)
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(y[i][e]) & 0x7FFFFFFFu);
  m = NT == kWave ? wave_max_u32(m) : block_max<NT>(m, redu);
  const RowScale rs = row_scale(m, bad);
  if (tid == 0) a.scale[t] = rs.scale;
  int8_t* code = a.code + t * a.code_row;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int k = (tid + i * NT) * 8;
    if (k >= cols) break;
    uint32_t w[2] = {};
    if (rs.inv > 0.0f)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e / 4] |= code_of(y[i][e], rs.inv) << (8 * (e & 3));
    *(uint2*)(code + k) = make_uint2(w[0], w[1]);
  }
}

}  // namespace

hipError_t launch_quantise_rows(const sjd_quantise_params& p, const sjd_quantise_io& io, hipStream_t s) {
  const QuantArgs a{io.d_x, io.d_norm, io.d_gate, io.d_code, io.d_scale, p.x_row, p.gate_row, p.code_row, p.T, p.K,
                    p.norm_dtype == SJD_F32, (float)(1.0 / p.K), p.eps};
  auto go = [&](auto e, auto nt, auto pieces) {
    using E = decltype(e);
    constexpr int NT = decltype(nt)::value, P = decltype(pieces)::value;
    // (two dimensions: one has less than 2^32 threads)
    const int wgs = NT == kWave ? (p.T + 3) / 4 : p.T, gx = std::min(wgs, 1 << 20);
    const dim3 grid(gx, (wgs + gx - 1) / gx), block(NT < 256 ? 256 : NT);
    if (io.d_norm) hipLaunchKernelGGL((k_quantise<E, NT, P, true, false>), grid, block, 0, s, a);
    else if (io.d_gate) hipLaunchKernelGGL((k_quantise<E, NT, P, false, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_quantise<E, NT, P, false, false>), grid, block, 0, s, a);
  };
  // (The order of a row's sum is by K alone: it does not depend on the rows beside it. Of 512 to 2048
  // inputs a workgroup to a row takes 3.1 us for 32 rows of 1024 behind a norm, a wave 3.8; for 4096
  // rows 7.1 and 5.5)
  auto pick = [&](auto e) {
    if (p.K <= 512) go(e, Int<64>{}, Int<1>{});
    else if (p.K <= 2048 && p.T <= 1024) go(e, Int<256>{}, Int<1>{});
    else if (p.K <= 2048) go(e, Int<64>{}, Int<4>{});
    else if (p.K <= 4096) go(e, Int<256>{}, Int<2>{});
    else if (p.K <= 16384) go(e, Int<1024>{}, Int<2>{});
    else if (p.K <= 32768) go(e, Int<1024>{}, Int<4>{});
    else go(e, Int<1024>{}, Int<8>{});
  };
  if (p.dtype == SJD_F32) pick(float{});
  else pick(uint16_t{});
  return hipGetLastError();
}

}  // namespace sjd
