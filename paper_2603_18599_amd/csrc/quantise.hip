// Rows as 8-bit integers with a scale each (definition: sjd.h), the input of the
// products in matmul_i8.hip, with what stands in front of a projection: an RMSNorm or
// the gate of a gated layer.
#include "device.h"
#include "ops.h"
#include "rows_i8.h"

namespace sjd {

namespace {

struct QuantArgs {
  const void *x, *norm, *gate;
  int8_t* code;
  float* scale;
  int64_t x_row, gate_row, code_row;
  int K;
  int norm_f32;
  float inv_k, eps;
};

constexpr int kThreads = 256;

// E: element (uint16_t bf16, float)
template <class E, bool NORM, bool GATE>
__global__ __launch_bounds__(kThreads) void k_quantise(QuantArgs a) {
  __shared__ float red[kThreads / kWave];
  __shared__ uint32_t redu[kThreads / kWave];
  const int64_t t = blockIdx.x;
  const E* x = (const E*)a.x + t * a.x_row;
  const E* gate = (const E*)a.gate + t * a.gate_row;
  float rinv = 0.0f;
  bool bad = false;
  if constexpr (NORM) {
    float ss = 0.0f;
    for (int k = threadIdx.x; k < a.K; k += kThreads) {
      const float v = elem_f32(x[k]);
      ss += v * v;
    }
    ss = block_sum<kThreads>(ss, red);
    bad = !(ss < INFINITY);
    rinv = 1.0f / sqrtf(ss * a.inv_k + a.eps);
  }
  auto y = [&](int k) {
    const float v = elem_f32(x[k]);
    if constexpr (NORM) return v * rinv * (a.norm_f32 ? ((const float*)a.norm)[k] : bf16_to_f32(((const uint16_t*)a.norm)[k]));
    if constexpr (GATE) return v * silu(elem_f32(gate[k]));
    return v;
  };
  uint32_t m = 0;  // (as bits: NaN is above infinity)
  for (int k = threadIdx.x; k < a.K; k += kThreads) m = max(m, __float_as_uint(y(k)) & 0x7FFFFFFFu);
  m = block_max<kThreads>(m, redu);
  const RowScale rs = row_scale(m, bad);
  if (threadIdx.x == 0) a.scale[t] = rs.scale;
  int8_t* code = a.code + t * a.code_row;
  const int cols = (a.K + 15) & ~15;
  for (int k = threadIdx.x; k < cols; k += kThreads) code[k] = k < a.K && rs.inv > 0.0f ? code_of(y(k), rs.inv) : 0;
}

}  // namespace

hipError_t launch_quantise_rows(const sjd_quantise_params& p, const sjd_quantise_io& io, hipStream_t s) {
  const QuantArgs a{io.d_x, io.d_norm, io.d_gate, io.d_code, io.d_scale, p.x_row, p.gate_row, p.code_row, p.K,
                    p.norm_dtype == SJD_F32, (float)(1.0 / p.K), p.eps};
  const dim3 grid(p.T), block(kThreads);
  auto go = [&](auto e) {
    using E = decltype(e);
    if (io.d_norm) hipLaunchKernelGGL((k_quantise<E, true, false>), grid, block, 0, s, a);
    else if (io.d_gate) hipLaunchKernelGGL((k_quantise<E, false, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_quantise<E, false, false>), grid, block, 0, s, a);
  };
  if (p.dtype == SJD_F32) go(float{});
  else go(uint16_t{});
  return hipGetLastError();
}

}  // namespace sjd
