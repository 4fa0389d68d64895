// Products in 8-bit integers (definition: sjd.h): rows of codes with packed weights,
// exact in 32-bit integers, then the scales of row and channel.
#include <type_traits>

#include "device.h"
#include "ops.h"
#include "rows_i8.h"

namespace sjd {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

template <int N>
using Int = std::integral_constant<int, N>;

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
  int pair;  // bf16 outputs may be stored two channels at a time
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
SJD_DEV uint32_t pk_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

SJD_DEV void put(const MatArgs& a, int t, int n, int sum, float ws, float cs) {
  float v = (float)sum * ws * cs;
  if (a.f32) {
    if (a.add) v += ((const float*)a.add)[t * a.add_row + n];
    ((float*)a.out)[t * a.out_row + n] = v;
  } else {
    if (a.add) v += bf16_to_f32(((const uint16_t*)a.add)[t * a.add_row + n]);
    ((uint16_t*)a.out)[t * a.out_row + n] = f32_to_bf16(v);
  }
}

// C rows (channels) of register i: 8 (i / 4) + 4 half + i % 4; column (row of codes) lane % 32
SJD_DEV void finish(const MatArgs& a, const i32x16& c, int n0, int t) {
  if (t >= a.T) return;
  const float cs = a.cscale[t];
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int n = n0 + 8 * (i >> 2) + 4 * half + (i & 3);
    if (n < a.N) put(a, t, n, c[i], a.wscale[n], cs);
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

// Few rows: the weights pass once. A workgroup has CH channels and TT tiles of CH rows;
// its eight waves share the inputs, units of 128 of them with DEPTH units' loads in
// flight, and add their sums up in LDS.
template <int CH>
struct FewMfma;
template <>
struct FewMfma<32> {
  using C = i32x16;
  static constexpr int kRegs = 16, kSteps = 4;  // of a unit
  static SJD_DEV C mma(i32x4 x, i32x4 y, C c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(x, y, c, 0, 0, 0); }
  static SJD_DEV int k(int lane) { return 16 * (lane >> 5); }
  static SJD_DEV int w(int lane, int) { return lane * 16; }
  // channel of registers 4 i ..
  static SJD_DEV int n(int lane, int i) { return 8 * i + 4 * (lane >> 5); }
};
template <>
struct FewMfma<16> {
  using C = i32x4;
  static constexpr int kRegs = 4, kSteps = 2;
  static SJD_DEV C mma(i32x4 x, i32x4 y, C c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(x, y, c, 0, 0, 0); }
  static SJD_DEV int k(int lane) { return 16 * (lane >> 4); }
  static SJD_DEV int w(int lane, int odd) { return (lane >> 5) * 1024 + 16 * ((lane & 15) + 16 * odd + 32 * (lane >> 4 & 1)); }
  static SJD_DEV int n(int lane, int) { return 4 * (lane >> 4); }
};

constexpr int kFewWaves = 8;

// STAGE: codes are loaded eight lanes to a row's 128 bytes and pass through the wave's own
// part of LDS, 16-byte pieces exchanged so that rows eight apart share banks; else
// each lane loads its operand, which touches a line per row.
template <int CH, int TT, int DEPTH, bool STAGE>
__global__ __launch_bounds__(64 * kFewWaves, 2) void k_matmul_few(MatArgs a) {
  using M = FewMfma<CH>;
  constexpr int S = M::kSteps, ROW = CH + 4;  // (ints of a row of sums: 16 bytes more spread them over the banks)
  constexpr int kSums = kFewWaves * CH * ROW, kStage = STAGE ? kFewWaves * TT * CH * 32 : 0;
  __shared__ __align__(16) int lds[kSums > kStage ? kSums : kStage];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int t0 = blockIdx.y * (CH * TT), n0 = blockIdx.x * CH;
  const char* w = a.w + (int64_t)(n0 >> 5) * a.ks * 1024 + M::w(lane, (n0 >> 4) & 1);
  // STAGE: a load is rows 8 p .. + 7 of a tile, piece lane % 8 ^ row
  const int k0 = STAGE ? 16 * ((lane & 7) ^ (lane >> 3)) : M::k(lane);
  constexpr int ROWS = STAGE ? TT * S : TT;
  const int8_t* code[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i)
    code[i] = a.code + min(t0 + (STAGE ? 8 * i + (lane >> 3) : CH * i + lane % CH), a.T - 1) * a.code_row;
  int* const mine = lds + wave * (TT * CH * 32);
  const int units = a.ks >> 2, u0 = units * wave / kFewWaves, u1 = units * (wave + 1) / kFewWaves;
  i32x4 x[DEPTH][S], y[DEPTH][TT][S];
  auto load = [&](int d, int u) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      x[d][s] = *(const i32x4*)(w + (int64_t)u * 4096 + s * (4096 / S));
      const int k = u * 128 + (STAGE ? 0 : s * (128 / S)) + k0;
#pragma unroll
      for (int i = 0; i < TT; ++i) y[d][i][s] = *(const i32x4*)(code[STAGE ? i * S + s : i] + (k < a.cols ? k : 0));
    }
  };
  typename M::C c[TT] = {};
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (u0 + d < u1) load(d, u0 + d);
  for (int u = u0; u < u1; u += DEPTH)
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      if (u + d >= u1) break;
      if constexpr (STAGE) {
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
          for (int s = 0; s < S; ++s) *(i32x4*)(mine + (i * S + s) * 256 + lane * 4) = y[d][i][s];
      }
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < TT; ++i) {
          if constexpr (STAGE) {
            const int row = lane % CH, piece = s * (8 / S) + lane / CH;
            const i32x4 v = *(const i32x4*)(mine + i * (CH * 32) + row * 32 + 4 * (piece ^ (row & 7)));
            c[i] = M::mma(x[d][s], v, c[i]);
          } else {
            c[i] = M::mma(x[d][s], y[d][i][s], c[i]);
          }
        }
      if (u + d + DEPTH < u1) load(d, u + d + DEPTH);
    }
  int(*const sums)[CH * ROW] = (int(*)[CH * ROW])lds;
#pragma unroll
  for (int i = 0; i < TT; ++i) {
    if (STAGE || i) __syncthreads();
#pragma unroll
    for (int r = 0; r < M::kRegs; r += 4)
      *(i32x4*)&sums[wave][(lane % CH) * ROW + M::n(lane, r / 4)] = i32x4{c[i][r], c[i][r + 1], c[i][r + 2], c[i][r + 3]};
    __syncthreads();
    for (int e = threadIdx.x; e < CH * CH; e += 64 * kFewWaves) {
      const int t = t0 + CH * i + e / CH, n = n0 + e % CH;
      if (t >= a.T || n >= a.N) continue;
      int sum = 0;
#pragma unroll
      for (int v = 0; v < kFewWaves; ++v) sum += sums[v][e / CH * ROW + e % CH];
      put(a, t, n, sum, a.wscale[n], a.cscale[t]);
    }
  }
}

// Scales, addend and stores of a wave's FT x FN blocks from row t0, channel n0. Register r of
// a block: row 8 (r / 4) + 4 (lane / 32) + r % 4, channel lane % 32. bf16: two lanes
// exchange halves of two rows, so that each stores two channels of one.
template <bool F32, bool ADD, int FT, int FN>
SJD_DEV void finish_many(const MatArgs& a, const i32x16 (&c)[FT][FN], int t0, int n0) {
  using E = std::conditional_t<F32, float, uint16_t>;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < FT; ++i) {
    const int tb = t0 + 32 * i + 4 * (lane >> 5);
    float cs[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) cs[r] = a.cscale[min(tb + 8 * (r >> 2) + (r & 3), a.T - 1)];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int n = n0 + 32 * j + (lane & 31);
      const float ws = a.wscale[min(n, a.N - 1)];
      float v[16];
      if constexpr (ADD) {
        const E* add = (const E*)a.add + min(n, a.N - 1);
        E x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = add[min(tb + 8 * (r >> 2) + (r & 3), a.T - 1) * a.add_row];
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = (float)c[i][j][r] * ws * cs[r] + elem_f32(x[r]);
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) v[r] = (float)c[i][j][r] * ws * cs[r];
      }
      if constexpr (F32) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int t = tb + 8 * (r >> 2) + (r & 3);
          if (t < a.T && n < a.N) ((float*)a.out)[t * a.out_row + n] = v[r];
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const uint32_t p = pk_bf16(v[r], v[r + 1]);
          const int t = tb + 8 * (r >> 2) + (r & 3);
          if (a.pair) {
            const uint32_t o = dpp::mov<dpp::kXor1>(p);
            const bool odd = lane & 1;
            const uint32_t q = odd ? (o >> 16) | (p & 0xFFFF0000u) : (p & 0xFFFFu) | (o << 16);
            const int tq = t + odd, nq = n & ~1;
            if (tq < a.T && nq < a.N) *(uint32_t*)((uint16_t*)a.out + tq * a.out_row + nq) = q;
          } else {
            if (t < a.T && n < a.N) ((uint16_t*)a.out)[t * a.out_row + n] = (uint16_t)p;
            if (t + 1 < a.T && n < a.N) ((uint16_t*)a.out)[(t + 1) * a.out_row + n] = (uint16_t)(p >> 16);
          }
        }
      }
    }
  }
}

// Many rows: a workgroup of 2 x 2 waves has BT rows and BN channels, in steps of 128 inputs
// through two buffers of LDS, filled from memory directly.
typedef const void __attribute__((address_space(1)))* GlobalPtr;
typedef void __attribute__((address_space(3)))* LdsPtr;

template <int BT, int BN, int VT, int VN>
__global__ __launch_bounds__(64 * VT * VN, VT * VN / 4) void k_matmul_many(MatArgs a, int nt, int nn) {
  constexpr int WT = BT / VT, WN = BN / VN, FT = WT / 32, FN = WN / 32;
  __shared__ __align__(16) char lds0[(BT + BN) * 128];
  __shared__ __align__(16) char lds1[(BT + BN) * 128];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // eight dies take workgroups in turn: each has a run of tiles, four tiles of rows by all
  // the channels at a time
  int tt, tn;
  {
    const int total = nt * nn, id = blockIdx.x, per = total >> 3, more = total & 7, die = id & 7;
    const int tile = die * per + min(die, more) + (id >> 3);
    const int g = tile / (4 * nn), r = tile - g * 4 * nn, rows = min(4, nt - 4 * g);
    tt = 4 * g + r % rows;
    tn = r / rows;
  }
  const int t0 = tt * BT, b0 = tn * (BN / 32);
  // this wave's loads of a step: rows of codes 8 at a time, tiles of weights
  constexpr int LT = BT / 8 / (VT * VN), LN = BN / 8 / (VT * VN);
  const int8_t* code[LT];
  const char* w[LN];
  const int kl = 16 * ((lane & 7) ^ (lane >> 3));
#pragma unroll
  for (int i = 0; i < LT; ++i) code[i] = a.code + min(t0 + 8 * (wave * LT + i) + (lane >> 3), a.T - 1) * a.code_row;
#pragma unroll
  for (int i = 0; i < LN; ++i) {
    const int q = wave * LN + i;  // row block q / 4, tile q % 4 of the step
    w[i] = a.w + ((int64_t)min(b0 + q / 4, a.nb - 1) * a.ks + (q & 3)) * 1024 + lane * 16;
  }
  auto fill = [&](char* lds, int u) {
    const int k = u * 128 + kl;
#pragma unroll
    for (int i = 0; i < LT; ++i)
      __builtin_amdgcn_global_load_lds((GlobalPtr)(code[i] + (k < a.cols ? k : 0)), (LdsPtr)(lds + (wave * LT + i) * 1024), 16,
                                       0, 0);
#pragma unroll
    for (int i = 0; i < LN; ++i)
      __builtin_amdgcn_global_load_lds((GlobalPtr)(w[i] + (int64_t)u * 4096),
                                       (LdsPtr)(lds + BT * 128 + (wave * LN + i) * 1024), 16, 0, 0);
  };
  const int wt = wave % VT * WT, wn = wave / VT * FN;
  i32x16 c[FT][FN] = {};
  auto compute = [&](const char* lds) {
    i32x4 x[2][FT], y[2][FN];
    auto frags = [&](int s, int p) {
#pragma unroll
      for (int i = 0; i < FT; ++i) {
        const int row = wt + 32 * i + (lane & 31);
        x[p][i] = *(const i32x4*)(lds + row * 128 + 16 * ((2 * s + (lane >> 5)) ^ (row & 7)));
      }
#pragma unroll
      for (int j = 0; j < FN; ++j) y[p][j] = *(const i32x4*)(lds + BT * 128 + ((wn + j) * 4 + s) * 1024 + lane * 16);
    };
    frags(0, 0);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s < 3) frags(s + 1, (s + 1) & 1);
#pragma unroll
      for (int i = 0; i < FT; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) c[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[s & 1][i], y[s & 1][j], c[i][j], 0, 0, 0);
    }
  };
  const int units = a.ks >> 2;
  auto step = [&](char* now, char* next, int u) {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's part of the step is in LDS
    __syncthreads();                     // .. and the others'; nobody reads the other buffer
    if (u + 1 < units) fill(next, u + 1);
    compute(now);
  };
  fill(lds0, 0);
  for (int u = 0; u < units; u += 2) {
    step(lds0, lds1, u);
    if (u + 1 < units) step(lds1, lds0, u + 1);
  }
  auto finish = [&](auto f32, auto add) { finish_many<decltype(f32)::value, decltype(add)::value, FT, FN>(a, c, t0 + wt, (b0 + wn) * 32); };
  if (a.f32) a.add ? finish(std::true_type{}, std::true_type{}) : finish(std::true_type{}, std::false_type{});
  else a.add ? finish(std::false_type{}, std::true_type{}) : finish(std::false_type{}, std::false_type{});
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
      m = wave_max_u32(m);
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
                  io.add_row, io.T, w.N, (w.K + 15) & ~15, sh.nb, sh.ks, io.dtype == SJD_F32,
                  ((uintptr_t)io.d_out & 3) == 0 && io.out_row % 2 == 0 && w.N % 2 == 0};
  if (io.T <= 128) {
    auto few = [&](auto ch, auto tt, auto depth, auto stage) {
      constexpr int CH = decltype(ch)::value, TT = decltype(tt)::value;
      hipLaunchKernelGGL((k_matmul_few<CH, TT, decltype(depth)::value, decltype(stage)::value>),
                         dim3((w.N + CH - 1) / CH, (io.T + CH * TT - 1) / (CH * TT)), dim3(64 * kFewWaves), 0, s, a);
    };
    const std::false_type direct;
    const std::true_type stage;
    const bool narrow = w.N <= 8192;
    if (narrow && io.T <= 8) few(Int<16>{}, Int<1>{}, Int<8>{}, direct);
    else if (narrow && io.T <= 16) few(Int<16>{}, Int<1>{}, Int<8>{}, stage);
    else if (narrow && io.T <= 32) few(Int<16>{}, Int<2>{}, Int<6>{}, stage);
    else if (narrow && io.T <= 64) few(Int<16>{}, Int<4>{}, Int<4>{}, stage);
    else if (io.T <= 8) few(Int<32>{}, Int<1>{}, Int<4>{}, direct);
    else if (io.T <= 32) few(Int<32>{}, Int<1>{}, Int<4>{}, stage);
    else if (io.T <= 64) few(Int<32>{}, Int<2>{}, Int<3>{}, stage);
    else few(Int<32>{}, Int<4>{}, Int<2>{}, stage);
    return hipGetLastError();
  }
  auto many = [&](auto bt, auto bn, auto vt, auto vn) {
    constexpr int BT = decltype(bt)::value, BN = decltype(bn)::value, VT = decltype(vt)::value, VN = decltype(vn)::value;
    const int nt = (io.T + BT - 1) / BT, nn = (w.N + BN - 1) / BN;
    hipLaunchKernelGGL((k_matmul_many<BT, BN, VT, VN>), dim3(nt * nn), dim3(64 * VT * VN), 0, s, a, nt, nn);
  };
  if (io.T > 1024) many(Int<256>{}, Int<256>{}, Int<2>{}, Int<4>{});
  else many(Int<128>{}, Int<128>{}, Int<2>{}, Int<2>{});
  return hipGetLastError();
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
