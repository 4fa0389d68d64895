// Products in 8-bit integers (definition: sjd.h): rows of codes with packed weights,
// exact in 32-bit integers, then the scales of row and channel.
#include <algorithm>
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
  int wide;  // four channels of a row are aligned for one access
  int splits;      // of the inputs; with more than one
  int32_t* sums;   // .. sums of their parts, [splits][T][32 nb]
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
SJD_DEV uint32_t pk_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// A sum with its scales, plus an addend: alike in every kernel, so that a row's bits do not
// depend on which one it meets
SJD_DEV float scaled(int sum, float ws, float cs) { return (float)sum * ws * cs; }
SJD_DEV float scaled(int sum, float ws, float cs, float add) { return __builtin_fmaf((float)sum * ws, cs, add); }

// Channels n .. n + 3 of row t, from their sums
SJD_DEV void put(const MatArgs& a, int t, int n, const i32x4& sum, const float4& scales, float cs) {
  const float ws[4] = {scales.x, scales.y, scales.z, scales.w};
  float v[4];
  const int64_t at = t * a.out_row + n, from = t * a.add_row + n;
  if (a.wide && n + 4 <= a.N) {
    float add[4];
    if (a.add && a.f32) {
      const float4 x = *(const float4*)((const float*)a.add + from);
      add[0] = x.x; add[1] = x.y; add[2] = x.z; add[3] = x.w;
    } else if (a.add) {
      const uint2 x = *(const uint2*)((const uint16_t*)a.add + from);
      add[0] = __uint_as_float(x.x << 16); add[1] = __uint_as_float(x.x & 0xFFFF0000u);
      add[2] = __uint_as_float(x.y << 16); add[3] = __uint_as_float(x.y & 0xFFFF0000u);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = a.add ? scaled(sum[e], ws[e], cs, add[e]) : scaled(sum[e], ws[e], cs);
    if (a.f32) *(float4*)((float*)a.out + at) = make_float4(v[0], v[1], v[2], v[3]);
    else *(uint2*)((uint16_t*)a.out + at) = make_uint2(pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3]));
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (n + e >= a.N) break;
    float x = scaled(sum[e], ws[e], cs);
    if (a.add) {
      const float add = a.f32 ? ((const float*)a.add)[from + e] : bf16_to_f32(((const uint16_t*)a.add)[from + e]);
      x = scaled(sum[e], ws[e], cs, add);
    }
    if (a.f32) ((float*)a.out)[at + e] = x;
    else ((uint16_t*)a.out)[at + e] = f32_to_bf16(x);
  }
}
SJD_DEV float4 channel_scales(const MatArgs& a, int n) {
  return make_float4(a.wscale[min(n, a.N - 1)], a.wscale[min(n + 1, a.N - 1)], a.wscale[min(n + 2, a.N - 1)],
                     a.wscale[min(n + 3, a.N - 1)]);
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

// Where a row of P pieces of 16 bytes in LDS has piece p, and which piece lies at place p: the
// 16 rows that a read takes at a time cover all 64 banks
template <int P>
SJD_DEV int swizzle(int row, int p) {
  static_assert(P == 4 || P == 8, "16 rows of P pieces: P times all banks");
  return p ^ (P == 8 ? row >> 1 & 7 : row >> 2 & 3);
}

constexpr int kFewWaves = 8;

// STAGE: codes are loaded eight lanes to a row's 128 bytes and pass through the wave's own
// part of LDS; else each lane loads its operand, which touches a line per row.
template <int CH, int TT, int DEPTH, bool STAGE>
__global__ __launch_bounds__(64 * kFewWaves) void k_matmul_few(MatArgs a) {
  using M = FewMfma<CH>;
  constexpr int S = M::kSteps, ROW = CH + 4;  // (ints of a row of sums: 16 bytes more spread them over the banks)
  constexpr int kSums = kFewWaves * CH * ROW, kStage = STAGE ? kFewWaves * TT * CH * 32 : 0;
  __shared__ __align__(16) int lds[kSums > kStage ? kSums : kStage];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int t0 = blockIdx.y * (CH * TT), n0 = blockIdx.x * CH;
  const char* w = a.w + (int64_t)(n0 >> 5) * a.ks * 1024 + M::w(lane, (n0 >> 4) & 1);
  // STAGE: a load is rows 8 p .. + 7 of a tile
  const int k0 = STAGE ? 0 : M::k(lane);
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
      const int k = u * 128 + (STAGE ? 16 * swizzle<8>(8 * s + (lane >> 3), lane & 7) : s * (128 / S)) + k0;
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
            const i32x4 v = *(const i32x4*)(mine + i * (CH * 32) + row * 32 + 4 * swizzle<8>(row, piece));
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
    if (threadIdx.x >= CH * CH / 4) continue;
    const int row = threadIdx.x / (CH / 4), col = threadIdx.x % (CH / 4) * 4, t = t0 + CH * i + row, n = n0 + col;
    if (t >= a.T || n >= a.N) continue;
    i32x4 sum = {};
#pragma unroll
    for (int v = 0; v < kFewWaves; ++v) sum += *(const i32x4*)&sums[v][row * ROW + col];
    put(a, t, n, sum, channel_scales(a, n), a.cscale[t]);
  }
}

typedef const void __attribute__((address_space(1)))* GlobalPtr;
typedef void __attribute__((address_space(3)))* LdsPtr;
SJD_DEV void load_lds(const void* src, char* lds) {
  __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)lds, 16, 0, 0);
}
// Waits until this wave's reads of LDS are done and at most N of its loads are outstanding, then
// for the other waves. (A plain barrier: a fence would wait for every load.)
template <int N>
SJD_DEV void wait_barrier() {
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);  // vmcnt(N) lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Rows q0 + i * STEP (i < U) of a wave's block of sums in LDS, scaled and stored: four
// channels a lane
template <bool F32, bool ADD, int U, int STEP, int OUT>
SJD_DEV void put_rows(const MatArgs& a, const int* sums, const float* scales, int t0, int q0, int n, const float4& ws) {
  using P = std::conditional_t<F32, float4, uint2>;
  constexpr int ES = F32 ? 4 : 2;
  i32x4 c[U];
  P add[U];
  float cs[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int q = q0 + i * STEP;
    c[i] = *(const i32x4*)(sums + q * OUT);
    cs[i] = scales[q];
    if constexpr (ADD) add[i] = *(const P*)((const char*)a.add + (min(t0 + q, a.T - 1) * a.add_row + n) * ES);
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int t = t0 + q0 + i * STEP;
    float v[4], x[4] = {};
    if constexpr (ADD && F32) {
      x[0] = add[i].x, x[1] = add[i].y, x[2] = add[i].z, x[3] = add[i].w;
    } else if constexpr (ADD) {
      x[0] = __uint_as_float(add[i].x << 16), x[1] = __uint_as_float(add[i].x & 0xFFFF0000u);
      x[2] = __uint_as_float(add[i].y << 16), x[3] = __uint_as_float(add[i].y & 0xFFFF0000u);
    }
    const float w[4] = {ws.x, ws.y, ws.z, ws.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = ADD ? scaled(c[i][e], w[e], cs[i], x[e]) : scaled(c[i][e], w[e], cs[i]);
    P* const out = (P*)((char*)a.out + (t * a.out_row + n) * ES);
    if constexpr (F32) {
      if (t < a.T) *out = make_float4(v[0], v[1], v[2], v[3]);
    } else {
      if (t < a.T) *out = make_uint2(pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3]));
    }
  }
}

// Many rows: a workgroup of VT x VN waves has BT rows and BN channels, a wave FT x FN blocks of
// 32 x 32. Steps of 64 inputs pass through four buffers of LDS, filled from memory directly.
// Half-way through a step its operands are all in registers: its buffer is filled again, with
// the step four on.
template <int BT, int BN, int VT, int VN>
__global__ __launch_bounds__(64 * VT * VN, 2) void k_matmul_many(MatArgs a, int nt, int nn) {
  constexpr int WT = BT / VT, WN = BN / VN, FT = WT / 32, FN = WN / 32, WAVES = VT * VN;
  constexpr int kBuf = (BT + BN) * 64;
  __shared__ __align__(256) float scales[BT];
  // (an object each: the compiler then knows that a step's reads do not touch what is being filled)
  __shared__ __align__(16) char lds0[kBuf], lds1[kBuf], lds2[kBuf], lds3[kBuf];
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
  const int wt = wave % VT * WT, wn = wave / VT * FN;
  const int units = a.ks >> 1, u0 = units * (int)blockIdx.y / a.splits, u1 = units * ((int)blockIdx.y + 1) / a.splits;
  // this wave's loads of a step: rows of codes 16 at a time (64 bytes of each; rows past T read
  // the last one), tiles of weights
  constexpr int LT = BT / 16 / WAVES, LN = BN / 16 / WAVES, L = LT + LN, L0 = L / 2;
  const int8_t* code[LT];
  const char* w[LN];
  const int kl = 16 * swizzle<4>(lane >> 2, lane & 3);
#pragma unroll
  for (int i = 0; i < LT; ++i)
    code[i] = a.code + min(t0 + 16 * (wave * LT + i) + (lane >> 2), a.T - 1) * a.code_row + (int64_t)u0 * 64 + kl;
#pragma unroll
  for (int i = 0; i < LN; ++i) {
    const int q = wave * LN + i;  // row block q / 2, tile q % 2 of the step
    w[i] = a.w + ((int64_t)min(b0 + q / 2, a.nb - 1) * a.ks + 2 * u0 + q % 2) * 1024;
  }
  // load p of step u (its pointer then is at the next step's). FULL: no code lies behind its row;
  // else such a piece reads the row's first, against weights of zero
  auto fill = [&](auto full, char* lds, int u, int p) __attribute__((always_inline)) {
    if (p < LT) {
      const int k = u * 64 + kl;
      load_lds(decltype(full)::value || k < a.cols ? code[p] : code[p] - k, lds + (wave * LT + p) * 1024);
      code[p] += 64;
    } else {
      load_lds(w[p - LT] + (uint32_t)(lane * 16), lds + BT * 64 + (wave * LN + p - LT) * 1024);
      w[p - LT] += 2048;
    }
  };
  i32x16 c[FT][FN] = {};
  i32x4 x[2][FT], y[2][FN];
  auto frags = [&](const char* lds, int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FT; ++i) {
      const int row = wt + 32 * i + (lane & 31);
      x[s][i] = *(const i32x4*)(lds + row * 64 + 16 * swizzle<4>(row, 2 * s + (lane >> 5)));
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) y[s][j] = *(const i32x4*)(lds + BT * 64 + ((wn + j) * 2 + s) * 1024 + lane * 16);
  };
  // Products of half a step, `more`: with loads P0 .. P1 - 1 of step u between them. They go out one
  // at a time, over a whole step: the waves' loads of half of it would wait for each other.
  auto multiply = [&](auto full, int s, bool more, char* lds, int u, auto p0, auto p1) __attribute__((always_inline)) {
    constexpr int P0 = decltype(p0)::value, N = decltype(p1)::value - P0;
#pragma unroll
    for (int i = 0; i < FT; ++i) {
      if (more) {
#pragma unroll
        for (int p = 0; p < N; ++p)
          if (p * FT / N == i) fill(full, lds, u, P0 + p);
      }
#pragma unroll
      for (int j = 0; j < FN; ++j) c[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(y[s][j], x[s][i], c[i][j], 0, 0, 0);
    }
  };
  // FULL: there are eight steps behind it
  auto step = [&](auto full, char* now, const char* next, char* last, int u) __attribute__((always_inline)) {
    constexpr bool FULL = decltype(full)::value;
    if (!FULL && u >= u1) return;
    frags(now, 1);
    multiply(full, 0, FULL || u + 3 < u1, last, u + 3, Int<L0>{}, Int<L>{});
    // the next step is there, and no wave reads this one's buffer any more
    if (FULL || u + 3 < u1) wait_barrier<2 * L>();
    else if (u + 2 < u1) wait_barrier<L>();
    else wait_barrier<0>();
    if (FULL || u + 1 < u1) frags(next, 0);
    multiply(full, 1, FULL || u + 4 < u1, now, u + 4, Int<0>{}, Int<L0>{});
  };
  const float cs = threadIdx.x < BT ? a.cscale[min(t0 + (int)threadIdx.x, a.T - 1)] : 0.0f;
  const std::false_type checked;
#pragma unroll
  for (int p = 0; p < 3 * L + L0; ++p) {
    const int i = p / L;
    if (i == 0 || u0 + i < u1) fill(checked, i == 0 ? lds0 : i == 1 ? lds1 : i == 2 ? lds2 : lds3, u0 + i, p % L);
  }
  if (u0 + 3 < u1) wait_barrier<2 * L + L0>();
  else wait_barrier<0>();
  frags(lds0, 0);
  int u = u0;
  auto four = [&](auto full) __attribute__((always_inline)) {
    step(full, lds0, lds1, lds3, u);
    step(full, lds1, lds2, lds0, u + 1);
    step(full, lds2, lds3, lds1, u + 2);
    step(full, lds3, lds0, lds2, u + 3);
  };
  for (; u + 12 <= u1; u += 4) four(std::true_type{});
  for (; u < u1; u += 4) four(checked);

  // Blocks of 32 rows pass through a part of LDS of the wave's own, to leave in whole rows
  // (register r of a block: channel 8 (r / 4) + 4 (lane / 32) + r % 4, row lane % 32)
  constexpr int OUT = WN + 4, kParts = kBuf / (32 * OUT * 4), LPR = WN / 4, RPI = 64 / LPR, U = 32 / RPI < 8 ? 32 / RPI : 8;
  static_assert(kParts * 4 >= WAVES && BT <= 64 * WAVES, "a part for each wave, a scale for each thread");
  if (threadIdx.x < BT) scales[threadIdx.x] = cs;
  __syncthreads();
  const int part = wave / kParts;
  int* const mine = (int*)(part == 0 ? lds0 : part == 1 ? lds1 : part == 2 ? lds2 : lds3) + wave % kParts * (32 * OUT);
  const int col = lane % LPR * 4, n = (b0 + wn) * 32 + col, q0 = lane / LPR;
  const float4 ws = channel_scales(a, n);
  const int64_t row = a.nb * 32LL;
  int32_t* const sums = a.sums + (int64_t)blockIdx.y * a.T * row + n;
#pragma unroll
  for (int i = 0; i < FT; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *(i32x4*)(mine + (lane & 31) * OUT + 32 * j + 2 * r + 4 * (lane >> 5)) =
            i32x4{c[i][j][r], c[i][j][r + 1], c[i][j][r + 2], c[i][j][r + 3]};
    const int tb = t0 + wt + 32 * i;
    const float* const sc = scales + wt + 32 * i;
    if (a.splits > 1) {
#pragma unroll
      for (int q = 0; q < 32; q += RPI) {
        const i32x4 v = *(const i32x4*)(mine + (q0 + q) * OUT + col);
        if (tb + q0 + q < a.T && n < row) *(i32x4*)(sums + (tb + q0 + q) * row) = v;
      }
    } else if (a.wide && n + 4 <= a.N) {
      for (int q = q0; q < 32; q += U * RPI) {
        if (a.f32) {
          if (a.add) put_rows<true, true, U, RPI, OUT>(a, mine + col, sc, tb, q, n, ws);
          else put_rows<true, false, U, RPI, OUT>(a, mine + col, sc, tb, q, n, ws);
        } else {
          if (a.add) put_rows<false, true, U, RPI, OUT>(a, mine + col, sc, tb, q, n, ws);
          else put_rows<false, false, U, RPI, OUT>(a, mine + col, sc, tb, q, n, ws);
        }
      }
    } else if (n < a.N) {
      for (int q = q0; q < 32; q += RPI)
        if (tb + q < a.T) put(a, tb + q, n, *(const i32x4*)(mine + q * OUT + col), ws, sc[q]);
    }
  }
}

// Sums of the parts of split inputs, scaled: a thread has four channels of a row
__global__ __launch_bounds__(256) void k_matmul_join(MatArgs a) {
  const int n0 = (blockIdx.y * 256 + threadIdx.x) * 4, t = blockIdx.x;
  if (n0 >= a.N) return;
  const int64_t row = a.nb * 32LL;
  const int32_t* p = a.sums + t * row + n0;
  i32x4 c = *(const i32x4*)p;
  for (int s = 1; s < a.splits; ++s) c += *(const i32x4*)(p + s * (a.T * row));
  put(a, t, n0, c, channel_scales(a, n0), a.cscale[t]);
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
        uint32_t c = 0;
        if constexpr (kCodes) c = (uint8_t)s;
        else if (inv[i] > 0.0f) c = code_of(elem_f32(s), inv[i]);
        v[e / 4] |= c << (8 * (e & 3));
      }
    *(uint4*)(a.w + ((int64_t)blockIdx.x * a.ks * 64 + p) * 16) = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

}  // namespace

// Which kernel, tile and split of the inputs a product takes: the cheapest by an estimate in
// us, fitted to some 2000 timings of them all (24 to 8190 rows, 512 to 32768 channels, 1024 to
// 14336 inputs). Over 88 sizes of 256 rows and more its choice took 0.9% more than the best of
// them on average, 13% at most. The results do not depend on it.
struct MatPlan {
  int bt, bn;  // rows and channels of a workgroup; bt 0: few rows
  int splits;
};
static MatPlan matmul_plan(const sjd_i8_weights& w, int T) {
  if (T <= 32) return {0, 0, 1};
  struct Tile {
    int bt, bn, fit;             // .. workgroups on a compute unit
    double fixed, alone, shared;  // start and end; a step of 64 inputs, of one and of each of several on a unit
  };
  static constexpr Tile kTiles[] = {{64, 64, 4, 2.4, 0.195, 0.20},     {64, 128, 2, 4.8, 0.26, 0.225},
                                    {128, 128, 2, 7.1, 0.32, 0.315},   {128, 256, 1, 5.8, 0.475, 0.55},
                                    {256, 256, 1, 10.0, 0.86, 0.91}};
  const int64_t bytes = (int64_t)w.N * w.K;
  MatPlan best{0, 0, 1};
  double least = T <= 128 ? 3.6 + bytes * (w.N > 8192 ? 0.29e-6 : 0.37e-6) * ((T + 63) / 64) : 1e30;
  for (const Tile& t : kTiles)
    for (int s = 1; s <= 8; s *= 2) {
      const int64_t wgs = (int64_t)((w.N + t.bn - 1) / t.bn) * ((T + t.bt - 1) / t.bt) * s;
      if (s > 1 && (wgs > 640 || w.K < 512 * s)) break;
      const int64_t per = (wgs + 255) / 256, rounds = (per + t.fit - 1) / t.fit;
      double us = t.fixed + (rounds - 1) * 1.2 + (w.K + 127) / 128 * 2.0 / s * (per == 1 ? t.alone : per * t.shared);
      us = std::max(us, 4 + bytes * 0.25e-6);                           // the weights from memory
      if (s > 1) us += 3.3 + (double)s * T * w.N * 2.5e-6;              // the parts' sums, and a launch
      if (us < least) least = us, best = MatPlan{t.bt, t.bn, s};
    }
  return best;
}

int64_t i8_weight_bytes(int N, int K) {
  const I8Shape s = i8_shape(N, K);
  return (int64_t)s.nb * s.ks * 1024;
}

int64_t matmul_i8_ws(const sjd_i8_weights& w, int T) {
  const MatPlan p = matmul_plan(w, T);
  return p.splits > 1 ? (int64_t)p.splits * T * i8_shape(w.N, w.K).nb * 128 : 0;
}

hipError_t launch_matmul_i8(const sjd_i8_weights& w, const sjd_matmul_io& io, void* ws, hipStream_t s) {
  const I8Shape sh = i8_shape(w.N, w.K);
  const MatPlan p = matmul_plan(w, io.T);
  const uintptr_t es = io.dtype == SJD_F32 ? 4 : 2;
  auto fine = [&](const void* q, int64_t row) { return ((uintptr_t)q & (4 * es - 1)) == 0 && row % 4 == 0; };
  const MatArgs a{(const char*)w.d_w, w.d_scale, io.d_code, io.d_code_scale, io.d_out, io.d_add, io.code_row, io.out_row,
                  io.add_row, io.T, w.N, (w.K + 15) & ~15, sh.nb, sh.ks, io.dtype == SJD_F32,
                  fine(io.d_out, io.out_row) && (!io.d_add || fine(io.d_add, io.add_row)), p.splits, (int32_t*)ws};
  if (!p.bt) {
    auto few = [&](auto ch, auto tt, auto depth, auto stage) {
      constexpr int CH = decltype(ch)::value, TT = decltype(tt)::value;
      hipLaunchKernelGGL((k_matmul_few<CH, TT, decltype(depth)::value, decltype(stage)::value>),
                         dim3((w.N + CH - 1) / CH, (io.T + CH * TT - 1) / (CH * TT)), dim3(64 * kFewWaves), 0, s, a);
    };
    const std::false_type direct;
    const std::true_type stage;
    // (16 channels to a workgroup where 32 leave compute units without one, or each with so few that
    // their ends show: us, 16 and 32 channels, of 16 rows 4096 x 4096 5.5 and 6.0, 12288 12.3 and
    // 13.5, 22016 22.6 and 21.1; of 32 rows 4096 x 11008 15.1 and 17.9, 12288 x 4096 15.5 and 14.8. More
    // loads in flight cost workgroups: depths 2, 3 and 4 of 32 rows, 22016 x 4096: 22.6, 24.5, 25.8)
    if (io.T <= 8) few(Int<16>{}, Int<1>{}, Int<4>{}, direct);
    else if (io.T <= 16 && w.N <= 16384) few(Int<16>{}, Int<1>{}, Int<3>{}, stage);
    else if (io.T <= 32 && w.N > 8192) few(Int<32>{}, Int<1>{}, Int<2>{}, stage);
    else if (io.T <= 32) few(Int<16>{}, Int<2>{}, Int<2>{}, stage);
    else if (w.N > 8192) few(Int<32>{}, Int<2>{}, Int<1>{}, stage);
    else few(Int<16>{}, Int<4>{}, Int<4>{}, stage);
    return hipGetLastError();
  }
  auto many = [&](auto bt, auto bn, auto vt, auto vn) {
    constexpr int BT = decltype(bt)::value, BN = decltype(bn)::value, VT = decltype(vt)::value, VN = decltype(vn)::value;
    if (p.bt != BT || p.bn != BN) return;
    const int nt = (io.T + BT - 1) / BT, nn = (w.N + BN - 1) / BN;
    hipLaunchKernelGGL((k_matmul_many<BT, BN, VT, VN>), dim3(nt * nn, p.splits), dim3(64 * VT * VN), 0, s, a, nt, nn);
  };
  many(Int<256>{}, Int<256>{}, Int<2>{}, Int<4>{});
  many(Int<128>{}, Int<256>{}, Int<2>{}, Int<4>{});
  many(Int<128>{}, Int<128>{}, Int<2>{}, Int<2>{});
  many(Int<64>{}, Int<128>{}, Int<2>{}, Int<2>{});
  many(Int<64>{}, Int<64>{}, Int<2>{}, Int<2>{});
  if (p.splits > 1) hipLaunchKernelGGL(k_matmul_join, dim3(io.T, (w.N + 1023) / 1024), dim3(256), 0, s, a);
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
