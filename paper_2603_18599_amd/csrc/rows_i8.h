// Rows of 8-bit integers with a scale: the rule that makes one, and the layout of
// packed weights, shared by the quantiser, the packer and the product.
#pragma once
#include "device.h"

namespace sjd {

constexpr float kLeastRow = 0x1p-100f;  // rows below it count as zeros (127 / max stays finite)

SJD_DEV float elem_f32(uint16_t v) { return bf16_to_f32(v); }
SJD_DEV float elem_f32(float v) { return v; }
// x / (1 + e^-x) by the hardware's power of two and reciprocal. The argument p of the power rounds, by up to
// 2^-24 of |x| log2 e, which far below zero is many steps of the result: what it lost comes back as a
// factor, 1 - r with r = x + p ln 2 (below 2^-17, so its square is nothing; ln 2 as a float is 2^-28.4 of
// itself off, which moves the power by |x| 2^-28.4). All of it in quarters, so that the reciprocal, which
// flushes below 2^-126, keeps every gate whose power is a float. A power beyond the largest float
// (x below -88.72) is infinite and gives 0. Without the correction gates near -60 are up to 60 units of
// 2^-24 off, with it 6; it costs 4096 gated rows of 11008 42 us instead of 38.
SJD_DEV float silu(float x) {
  const float a = __builtin_amdgcn_fmed3f(x, -200.0f, 128.0f);  // (no infinity in r; the limits are those of x)
  const float p = a * -1.44269504f, r = __builtin_fmaf(p, 0.693147181f, a);
  const float power = __builtin_amdgcn_exp2f(p) * __builtin_fmaf(r, -0.25f, 0.25f);
  return 0.25f * x * __builtin_amdgcn_rcpf(0.25f + power);
}

struct RowScale {
  float scale, inv;  // inv 0: the codes are zeros
};
// bits: the largest |y| of the row, as bits
SJD_DEV RowScale row_scale(uint32_t bits, bool bad) {
  if (bad || bits >= 0x7F800000u) return {__uint_as_float(0x7FC00000u), 0.0f};
  const float m = __uint_as_float(bits);
  if (m < kLeastRow) return {0.0f, 0.0f};
  return {m / 127.0f, 127.0f / m};
}
// The code of y (|y| * inv <= 127 + 2^-16): the sum with 1.5 * 2^23 rounds once, to the nearest
// whole number, ties to even, and holds it in its low bits
SJD_DEV uint32_t code_of(float y, float inv) { return __float_as_uint(__builtin_fmaf(y, inv, 12582912.0f)) & 0xFFu; }

// over a workgroup of N threads (scratch: a word per wave)
template <int N>
SJD_DEV float block_sum(float v, float* scratch) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0f;
#pragma unroll
  for (int w = 0; w < N / kWave; ++w) v += scratch[w];
  return v;
}
SJD_DEV uint32_t wave_max_u32(uint32_t v) {
  return wave_reduce32(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int N>
SJD_DEV uint32_t block_max(uint32_t v, uint32_t* scratch) {
  v = wave_max_u32(v);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < N / kWave; ++w) v = max(v, scratch[w]);
  return v;
}

// Packed weights: tiles of 32 channels x 32 inputs, 1 KB, channels and inputs (up to a
// multiple of 128) padded with zeros. Channel n, input k of a tile: byte 16 * (n + 32 *
// (k / 16)) + k % 16, so a wave reads a tile as an operand of the 32x32x32 MFMA with
// one contiguous load. Tiles of a row block lie one behind the other.
struct I8Shape {
  int nb, ks;  // row blocks, tiles of a row block
};
__host__ __device__ inline I8Shape i8_shape(int N, int K) { return {(N + 31) / 32, (K + 127) / 128 * 4}; }

}  // namespace sjd
