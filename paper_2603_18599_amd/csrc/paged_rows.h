// Rows of keys and values on their way into pages: wide loads and stores, the rule of an
// e4m3 row's power of two, and the write of one tile. Shared by the kernels that append.
#pragma once
#include "device.h"
#include "forward.h"
#include "ops.h"

namespace sjd {

// N consecutive elements as floats (16-byte aligned)
template <bool F32, int N>
SJD_DEV void load_row(const void* base, int64_t at, float (&v)[N]) {
  if constexpr (F32) {
    const float4* p = (const float4*)((const float*)base + at);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const float4 x = p[i];
      v[4 * i] = x.x; v[4 * i + 1] = x.y; v[4 * i + 2] = x.z; v[4 * i + 3] = x.w;
    }
  } else {
    const uint4* p = (const uint4*)((const uint16_t*)base + at);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      const uint4 x = p[i];
      const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[8 * i + 2 * e] = __uint_as_float(u[e] << 16);
        v[8 * i + 2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
      }
    }
  }
}
template <bool F32, int N>
SJD_DEV void store_row(void* base, int64_t at, const float (&v)[N]) {
  if constexpr (F32) {
    float4* p = (float4*)((float*)base + at);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) p[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  } else {
    uint4* p = (uint4*)((uint16_t*)base + at);
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      uint32_t u[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        u[e] = (uint32_t)f32_to_bf16(v[8 * i + 2 * e]) | ((uint32_t)f32_to_bf16(v[8 * i + 2 * e + 1]) << 16);
      p[i] = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
}

// Exponent byte of a row whose largest finite magnitude is amax: the smallest E
// with amax <= 448 * 2^(E - 127). 448 = 1.75 * 2^8, so the mantissa decides
// whether the row's own exponent less 8 is enough.
SJD_DEV int row_exp(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int E = (int)(u >> 23) - ((u & 0x7FFFFFu) <= 0x600000u ? 8 : 7);
  return amax == 0.0f ? 127 : min(max(E, kMinExp), kMaxExp);
}
SJD_DEV float exp_scale(uint32_t E) { return __uint_as_float(E << 23); }

// N elements of a row (8 lanes hold it) as e4m3 codes; returns the exponent byte
template <int N>
SJD_DEV int quantise_row(const float (&v)[N], uint32_t (&code)[N / 4]) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float a = fabsf(v[i]);
    m = fmaxf(m, a < INFINITY ? a : 0.0f);
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
  const int E = row_exp(m);
  const float inv = exp_scale(254 - E);
  auto fit = [&](float x) {
    const float y = x * inv;
    return y != y ? y : fminf(fmaxf(y, -448.0f), 448.0f);  // (infinities, and rows past kMaxExp)
  };
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(fit(v[4 * i]), fit(v[4 * i + 1]), 0, false);
    code[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fit(v[4 * i + 2]), fit(v[4 * i + 3]), w, true);
  }
  return E;
}
SJD_DEV void decode4(uint32_t w, float f, float* v) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  v[0] = a[0] * f; v[1] = a[1] * f; v[2] = b[0] * f; v[3] = b[1] * f;
}

// A value tile's place in LDS: 16 bytes more every 256, which spreads the 8 threads of a
// row (256 and 1024 bytes apart) over the banks
SJD_DEV int pad(int b) { return b + ((b >> 8) << 4); }
// The first position (see val_byte) of the 16-byte piece u of a value tile; e4m3's second
// 8 bytes are 16 positions on
template <bool FP8>
SJD_DEV int piece_pos(int u) {
  const int hi = ((u & 63) >> 5) * 8;
  return FP8 ? hi : hi + 16 * ((u >> 6) & 1);
}

// Writes the rows of one tile (32 positions from `in` of a page, head h) that a workgroup of
// 256 (or each 256 threads of one) holds: thread 8 i + c has dims c * N .. of position i, `ok` where that is one of the
// positions [lo, hi) that the window holds. vs: the values' tile in LDS.
template <int HD, bool FP8>
SJD_DEV void store_tile(const PoolView& pv, char* page, int h, int in, int lo, int hi, bool ok, const float (&kf)[HD / 8],
                        const float (&vf)[HD / 8], char* vs) {
  constexpr int ES = FP8 ? 1 : 2, N = HD / 8;
  const int tid = threadIdx.x & 255, i = tid >> 3, c = tid & 7;
  // (of the row's first 8 dims; a second chunk, 128-dim heads: 8 bytes on in e4m3, 1024 in bf16)
  char* kt = page + tile_off<HD, ES>(pv, h, in, 0) + key_byte<HD, FP8>(i, c * N);
  char* vt = page + tile_off<HD, ES>(pv, h, in, 1);
  if constexpr (FP8) {
    uint32_t kc[N / 4], vc[N / 4];
    const int ke = quantise_row<N>(kf, kc), ve = quantise_row<N>(vf, vc);
    if (ok) {
      if constexpr (N == 16) *(uint4*)kt = make_uint4(kc[0], kc[1], kc[2], kc[3]);
      else *(uint2*)kt = make_uint2(kc[0], kc[1]);
      if (c == 0) {
        page[exp_off<HD>(pv, h, 0) + in + i] = (char)ke;
        page[exp_off<HD>(pv, h, 1) + in + i] = (char)ve;
      }
    }
#pragma unroll
    for (int e = 0; e < N; ++e) vs[pad(val_byte<true>(i, c * N + e))] = (char)(vc[e / 4] >> (8 * (e & 3)));
  } else {
#pragma unroll
    for (int g = 0; g < N / 8; ++g) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = kf[8 * g + e];
      if (ok) store_row<false, 8>(kt + 1024 * g, 0, x);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) *(uint16_t*)(vs + pad(val_byte<false>(i, c * N + e))) = f32_to_bf16(vf[e]);
  }
  __syncthreads();
  for (int u = tid; u < 2 * HD * ES; u += 256) {
    const uint4 x = *(const uint4*)(vs + pad(16 * u));
    const int p = piece_pos<FP8>(u);
    char* d = vt + 16 * u;
    if (lo == 0 && hi == 32) {
      *(uint4*)d = x;
      continue;
    }
    const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 16 / ES; ++e) {
      const int pe = FP8 ? p + 16 * (e >> 3) + (e & 7) : p + e;
      if (pe < lo || pe >= hi) continue;
      if constexpr (FP8) d[e] = (char)(y[e / 4] >> (8 * (e & 3)));
      else ((uint16_t*)d)[e] = (uint16_t)(y[e / 2] >> (16 * (e & 1)));
    }
  }
}

}  // namespace sjd
