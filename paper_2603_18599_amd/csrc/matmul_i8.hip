// Products in 8-bit integers (definition: sjd.h): rows of codes with packed weights,
// exact in 32-bit integers, then the scales of row and channel.
#include "device.h"
#include "ops.h"
#include "rows_i8.h"

namespace sjd {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

struct MatArgs {
  const char* w;
  const float* wscale;
  const int8_t* code;
  const float* cscale;
  void* out;
  const void* add;
  int64_t code_row, out_row, add_row;
  int T, N, cols;  // cols: codes of a row that are there
  int nb, ks;
  int f32;
};

// C rows (channels) of register i: 8 (i / 4) + 4 half + i % 4; column (row of codes) lane % 32
SJD_DEV void finish(const MatArgs& a, const i32x16& c, int n0, int t) {
  if (t >= a.T) return;
  const float cs = a.cscale[t];
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int n = n0 + 8 * (i >> 2) + 4 * half + (i & 3);
    if (n >= a.N) continue;
    float v = (float)c[i] * a.wscale[n] * cs;
    if (a.f32) {
      if (a.add) v += ((const float*)a.add)[t * a.add_row + n];
      ((float*)a.out)[t * a.out_row + n] = v;
    } else {
      if (a.add) v += bf16_to_f32(((const uint16_t*)a.add)[t * a.add_row + n]);
      ((uint16_t*)a.out)[t * a.out_row + n] = f32_to_bf16(v);
    }
  }
}

// A wave: 32 channels x 32 rows, operands straight from memory. Rows past T read the last
// row, codes past the row's end its first ones (against weights of zero).
__global__ __launch_bounds__(256) void k_matmul_i8(MatArgs a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  const int nb = blockIdx.y * 4 + wave;
  if (nb >= a.nb) return;
  const int t = blockIdx.x * 32 + (lane & 31);
  const int8_t* code = a.code + min(t, a.T - 1) * a.code_row;
  const char* w = a.w + (int64_t)nb * a.ks * 1024 + lane * 16;
  i32x16 c = {};
  for (int ks = 0; ks < a.ks; ++ks) {
    const int k = ks * 32 + 16 * half;
    const i32x4 x = *(const i32x4*)(w + (int64_t)ks * 1024), y = *(const i32x4*)(code + (k < a.cols ? k : 0));
    c = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, y, c, 0, 0, 0);
  }
  finish(a, c, nb * 32, t);
}

struct PackArgs {
  const void* src;
  int64_t row;
  char* w;
  float* scale;
  int N, K, ks;
};

// A workgroup: a row block. Channels' scales, then its tiles in 16-byte pieces.
template <class E>
__global__ __launch_bounds__(256) void k_pack_i8(PackArgs a) {
  __shared__ float inv[32];
  const int n0 = blockIdx.x * 32, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  constexpr bool kCodes = sizeof(E) == 1;
  if constexpr (!kCodes) {
    for (int i = wave; i < 32; i += 4) {
      const int n = n0 + i;
      uint32_t m = 0;
      if (n < a.N)
        for (int k = lane; k < a.K; k += kWave)
          m = max(m, __float_as_uint(elem_f32(((const E*)a.src)[n * a.row + k])) & 0x7FFFFFFFu);
      m = wave_reduce32(m, [](uint32_t p, uint32_t q) { return p > q ? p : q; });
      const RowScale rs = row_scale(m, false);
      if (lane == 0) {
        inv[i] = rs.inv;
        if (n < a.N) a.scale[n] = rs.scale;
      }
    }
    __syncthreads();
  }
  for (int p = threadIdx.x; p < a.ks * 64; p += 256) {
    const int i = p & 31, n = n0 + i, k0 = (p >> 6) * 32 + 16 * (p >> 5 & 1);
    uint32_t v[4] = {};
    if (n < a.N)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int k = k0 + e;
        if (k >= a.K) continue;
        const E s = ((const E*)a.src)[n * a.row + k];
        int8_t c = 0;
        if constexpr (kCodes) c = s;
        else if (inv[i] > 0.0f) c = code_of(elem_f32(s), inv[i]);
        v[e / 4] |= (uint32_t)(uint8_t)c << (8 * (e & 3));
      }
    *(uint4*)(a.w + ((int64_t)blockIdx.x * a.ks * 64 + p) * 16) = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

}  // namespace

int64_t matmul_i8_ws(const sjd_i8_weights& w, int T) { return 0; }

hipError_t launch_matmul_i8(const sjd_i8_weights& w, const sjd_matmul_io& io, void* ws, hipStream_t s) {
  const I8Shape sh = i8_shape(w.N, w.K);
  const MatArgs a{(const char*)w.d_w, w.d_scale, io.d_code, io.d_code_scale, io.d_out, io.d_add, io.code_row, io.out_row,
                  io.add_row, io.T, w.N, (w.K + 15) & ~15, sh.nb, sh.ks, io.dtype == SJD_F32};
  hipLaunchKernelGGL(k_matmul_i8, dim3((io.T + 31) / 32, (sh.nb + 3) / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_pack_i8(const sjd_i8_weights& w, const void* src, int dtype, int64_t row, hipStream_t s) {
  const I8Shape sh = i8_shape(w.N, w.K);
  const PackArgs a{src, row, (char*)w.d_w, w.d_scale, w.N, w.K, sh.ks};
  const dim3 grid(sh.nb), block(256);
  if (dtype == SJD_I8) hipLaunchKernelGGL(k_pack_i8<int8_t>, grid, block, 0, s, a);
  else if (dtype == SJD_F32) hipLaunchKernelGGL(k_pack_i8<float>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(k_pack_i8<uint16_t>, grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace sjd
