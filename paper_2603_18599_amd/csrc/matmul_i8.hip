// Products in 8-bit integers (definition: sjd.h): out[t][n] = cs[t] ws[n] sum_k code[t][k] w[n][k]
// (+ add[t][n]). The sums are exact in 32-bit integers (65536 products of 2^14 at most), so tiles,
// splits and their order are free choices, and a row's bits never depend on them. One product of a
// whole number and two scales is rounded three times, then the addend joins in one fused step.
//
// Few rows: the weights pass once through memory, which bounds them (one row, 32768 x 4096: 20 us,
// 6.8 TB/s where the last cache holds part of the 134 MB; 25 in a row of other work, 5.4). Many
// rows: bound by the matrix units and by the clock that they leave (bf16 outputs, no addend: 8190 rows
// of 4096 x 14336 402 us, 2390 TOP/s, the matrix units busy in 70% of the cycles at 1.63 GHz; 4096^3 66 us,
// 2090 TOP/s, 51% at 1.95 GHz). Between, loads on their way bound them (128 rows of 4096 x 11008, 64 x
// 128 tiles in four parts: 13.4 us, 43 steps of 0.24 us in a workgroup to each unit, three steps of 12
// KB under way, 136 MB from the dies' caches, the matrix units busy in 16%).
//
// The rows' codes are the second operand: a lane then owns one row and 16 channels of a 32 x 32
// block, four of them one behind the other, so sums and outputs move 16 and 8 bytes at a time.
#include <algorithm>
#include <cmath>
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

// Four channels of an output row, which may start at any element: one access of the size of
// four elements at the alignment of one. (Where a row is aligned for no more, such an access
// passes lane by lane: 2748 rows of 779 channels in large tiles take 25 us, of 780 15. Elements
// of a row one behind the other take 24, but in small tiles 18% longer than these.)
template <bool F32>
struct Four {
  using E = std::conditional_t<F32, float, uint16_t>;
  E v[4];
  SJD_DEV void load(const void* base, int64_t at) { __builtin_memcpy(v, (const E*)base + at, sizeof v); }
  SJD_DEV float get(int e) const {
    if constexpr (F32) return v[e];
    else return bf16_to_f32(v[e]);
  }
};
template <bool F32>
SJD_DEV void store_four(void* base, int64_t at, const float (&v)[4]) {
  if constexpr (F32) {
    __builtin_memcpy((float*)base + at, v, sizeof v);
  } else {
    const uint32_t u[2] = {pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
    __builtin_memcpy((uint16_t*)base + at, u, sizeof u);
  }
}

// Channels n .. n + 3 of row t, from their sums
template <bool F32>
SJD_DEV void put(const MatArgs& a, int t, int n, const i32x4& sum, const float4& scales, float cs) {
  using E = typename Four<F32>::E;
  const float ws[4] = {scales.x, scales.y, scales.z, scales.w};
  const int64_t at = t * a.out_row + n, from = t * a.add_row + n;
  Four<F32> x = {};
  float v[4];
  if (n + 4 <= a.N) {
    if (a.add) x.load(a.add, from);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = a.add ? scaled(sum[e], ws[e], cs, x.get(e)) : scaled(sum[e], ws[e], cs);
    store_four<F32>(a.out, at, v);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (n + e >= a.N) break;
    if (a.add) x.v[e] = ((const E*)a.add)[from + e];
    v[e] = a.add ? scaled(sum[e], ws[e], cs, x.get(e)) : scaled(sum[e], ws[e], cs);
    if constexpr (F32) ((E*)a.out)[at + e] = v[e];
    else ((E*)a.out)[at + e] = f32_to_bf16(v[e]);
  }
}
SJD_DEV void put(const MatArgs& a, int t, int n, const i32x4& sum, const float4& scales, float cs) {
  a.f32 ? put<true>(a, t, n, sum, scales, cs) : put<false>(a, t, n, sum, scales, cs);
}
SJD_DEV float4 channel_scales(const MatArgs& a, int n) {
  return make_float4(a.wscale[min(n, a.N - 1)], a.wscale[min(n + 1, a.N - 1)], a.wscale[min(n + 2, a.N - 1)],
                     a.wscale[min(n + 3, a.N - 1)]);
}

// Between one lane's writes of LDS and another's reads in the same wave: no instruction (a wave's accesses
// of LDS keep their order), the compiler's order alone
SJD_DEV void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
}

// Few rows: a workgroup has CH channels and TT tiles of CH rows. Its eight waves share the inputs,
// units of 128 of them with DEPTH units' loads in flight, straight from memory into the registers
// of the matrix operand, and add their sums up in LDS: 4096 channels would else be 128 waves. One
// row of 4096 x 4096: 3.8 us; 32 rows of 12288 x 4096: 9.8 us, 5.1 TB/s, launches in a row on the same
// weights, which the last cache holds (5.6 and 14.3 us where they come from memory).
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
        wave_order();
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
      if constexpr (STAGE) wave_order();
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

// A wave's block of sums in LDS, 32 rows of WN channels (n0 ..), scaled and stored, four
// channels a lane
template <bool F32, bool ADD, int WN, int OUT>
SJD_DEV void put_block(const MatArgs& a, const int* sums, const float* scales, int t0, int n0, const float4& ws) {
  constexpr int LPR = WN / 4, STEP = 64 / LPR, U = 32 / STEP < 8 ? 32 / STEP : 8;
  const int lane = threadIdx.x & 63, q0 = lane / LPR, col = lane % LPR * 4, n = n0 + col;
  if (n >= a.N) return;
  sums += col;
  if (n + 4 > a.N) {
    for (int q = q0; q < 32; q += STEP)
      if (t0 + q < a.T) put<F32>(a, t0 + q, n, *(const i32x4*)(sums + q * OUT), ws, scales[q]);
    return;
  }
  const float w[4] = {ws.x, ws.y, ws.z, ws.w};
  for (int qu = q0; qu < 32; qu += U * STEP) {
    i32x4 c[U];
    Four<F32> add[U];
    float cs[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int q = qu + i * STEP;
      c[i] = *(const i32x4*)(sums + q * OUT);
      cs[i] = scales[q];
      if constexpr (ADD) add[i].load(a.add, min(t0 + q, a.T - 1) * a.add_row + n);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int t = t0 + qu + i * STEP;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (ADD) v[e] = scaled(c[i][e], w[e], cs[i], add[i].get(e));
        else v[e] = scaled(c[i][e], w[e], cs[i]);
      }
      if (t < a.T) store_four<F32>(a.out, t * a.out_row + n, v);
    }
  }
}

// Many rows: a workgroup of VT x VN waves has BT rows and BN channels, a wave FT x FN blocks of
// 32 x 32 in registers. Steps of 64 inputs pass through four buffers of LDS, filled from memory
// directly (no register holds them, and three steps are on their way). Half-way through a step its
// operands are all in registers: its buffer is filled again, with the step four on, and one barrier
// a step is enough. Eight waves of 128 x 64 cover each other's waits in a tile of 256 x 256: 4096
// rows of 22016 x 4096 took 398 us with four of 128 x 128, 366 with them, 4096^3 71 and 65. (Three
// buffers, for two workgroups of 128 x 256 on a unit: 1024 rows of 22016 x 4096 110 us instead of
// 115, but single rounds slower.)
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
  for (int i = 0; i < LT; ++i) code[i] = a.code + min(t0 + 16 * (wave * LT + i) + (lane >> 2), a.T - 1) * a.code_row;
#pragma unroll
  for (int i = 0; i < LN; ++i) {
    const int q = wave * LN + i;  // row block q / 2, tile q % 2 of the step
    w[i] = a.w + ((int64_t)min(b0 + q / 2, a.nb - 1) * a.ks + q % 2) * 1024;
  }
  // Load p of step u. Steps behind the last read it once more, and codes behind a row its last 16,
  // against weights of zero: without a branch the compiler knows which loads are under way (with
  // one for each it waited for all of them in a call's last 8 to 11 steps, 2 us at a time).
  auto fill = [&](char* lds, int u, int p) __attribute__((always_inline)) {
    const int at = min(u, u1 - 1);
    if (p < LT) load_lds(code[p] + min(at * 64 + kl, a.cols - 16), lds + (wave * LT + p) * 1024);
    else load_lds(w[p - LT] + at * 2048 + (uint32_t)(lane * 16), lds + BT * 64 + (wave * LN + p - LT) * 1024);
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
  // Products of half a step, with loads P0 .. P1 - 1 of step u between them. They go out one
  // at a time, over a whole step: the waves' loads of half of it would wait for each other.
  auto multiply = [&](int s, char* lds, int u, auto p0, auto p1) __attribute__((always_inline)) {
    constexpr int P0 = decltype(p0)::value, N = decltype(p1)::value - P0;
#pragma unroll
    for (int i = 0; i < FT; ++i) {
#pragma unroll
      for (int p = 0; p < N; ++p)
        if (p * FT / N == i) fill(lds, u, P0 + p);
#pragma unroll
      for (int j = 0; j < FN; ++j) c[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(y[s][j], x[s][i], c[i][j], 0, 0, 0);
    }
  };
  auto step = [&](char* now, const char* next, char* last, int u) __attribute__((always_inline)) {
    frags(now, 1);
    multiply(0, last, u + 3, Int<L0>{}, Int<L>{});
    // the next step is there, and no wave reads this one's buffer any more
    wait_barrier<2 * L>();
    frags(next, 0);
    multiply(1, now, u + 4, Int<0>{}, Int<L0>{});
  };
  const float cs = threadIdx.x < BT ? a.cscale[min(t0 + (int)threadIdx.x, a.T - 1)] : 0.0f;
#pragma unroll
  for (int p = 0; p < 3 * L + L0; ++p) {
    const int i = p / L;
    fill(i == 0 ? lds0 : i == 1 ? lds1 : i == 2 ? lds2 : lds3, u0 + i, p % L);
  }
  wait_barrier<2 * L + L0>();
  frags(lds0, 0);
  int u = u0;
  for (; u + 4 <= u1; u += 4) {
    step(lds0, lds1, lds3, u);
    step(lds1, lds2, lds0, u + 1);
    step(lds2, lds3, lds1, u + 2);
    step(lds3, lds0, lds2, u + 3);
  }
  if (u < u1) {
    step(lds0, lds1, lds3, u);
    if (u + 1 < u1) step(lds1, lds2, lds0, u + 1);
    if (u + 2 < u1) step(lds2, lds3, lds1, u + 2);
  }
  wait_barrier<0>();  // (loads of steps behind the last)

  // Blocks of 32 rows pass through a part of LDS of the wave's own, to leave in whole rows
  // (register r of a block: channel 8 (r / 4) + 4 (lane / 32) + r % 4, row lane % 32)
  constexpr int OUT = WN + 4, kParts = kBuf / (32 * OUT * 4), LPR = WN / 4;
  static_assert(kParts * 4 >= WAVES && BT <= 64 * WAVES, "a part for each wave, a scale for each thread");
  if (threadIdx.x < BT) scales[threadIdx.x] = cs;
  __syncthreads();
  const int part = wave / kParts;
  int* const mine = (int*)(part == 0 ? lds0 : part == 1 ? lds1 : part == 2 ? lds2 : lds3) + wave % kParts * (32 * OUT);
  const int n0 = (b0 + wn) * 32;
  const float4 ws = channel_scales(a, n0 + lane % LPR * 4);
  auto blocks = [&](auto leave) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FT; ++i) {
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          *(i32x4*)(mine + (lane & 31) * OUT + 32 * j + 2 * r + 4 * (lane >> 5)) =
              i32x4{c[i][j][r], c[i][j][r + 1], c[i][j][r + 2], c[i][j][r + 3]};
      wave_order();
      leave(wt + 32 * i);
      wave_order();
    }
  };
  auto rows = [&](auto f32, auto add) __attribute__((always_inline)) {
    blocks([&](int t) __attribute__((always_inline)) {
      put_block<decltype(f32)::value, decltype(add)::value, WN, OUT>(a, mine, scales + t, t0 + t, n0, ws);
    });
  };
  const std::true_type yes;
  const std::false_type no;
  if (a.splits > 1) {
    const int64_t row = a.nb * 32LL;
    const int col = lane % LPR * 4, n = n0 + col;
    int32_t* const sums = a.sums + (int64_t)blockIdx.y * a.T * row + n;
    blocks([&](int t) __attribute__((always_inline)) {
#pragma unroll
      for (int q = 0; q < 32; q += 64 / LPR) {
        const int r = q + lane / LPR;
        const i32x4 v = *(const i32x4*)(mine + r * OUT + col);
        if (t0 + t + r < a.T && n < row) *(i32x4*)(sums + (t0 + t + r) * row) = v;
      }
    });
  } else {
    if (a.f32) a.add ? rows(yes, yes) : rows(yes, no);
    else a.add ? rows(no, yes) : rows(no, no);
  }
}

// Sums of the parts of split inputs, scaled: a thread has four channels of a row. Bound by memory
// that the parts' sums have just passed into (128 rows of 4096 channels, four parts: 4.1 us, 3.8 at
// the least).
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

// A workgroup: a row block. Channels' scales, then its tiles in 16-byte pieces. Bound by its loads, of an
// element each (22016 x 4096 codes 174 us, from bf16 340, fp32 447; 4096 x 11008, 128 workgroups with 2.7
// times the inputs each: 177, 619, 639): it runs once for a program's weights.
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
// us, fitted to 5170 timings of them all (33 to 5569 rows, 272 to 30197 channels, 289 to 14336
// inputs; 10% off, root mean square). Over their 480 sizes its choice took 1.5% more than the
// best of them on average, 43% at most (384 rows of 5572 x 8391; 64 rows of 5120 x 5120 37%, of 6144 x 4096
// 31%, the others below 28%). The results do not depend on it.
struct MatPlan {
  int bt, bn;  // rows and channels of a workgroup; bt 0: few rows
  int splits;
  double us;
};
static MatPlan plan_of(int N, int K, int T) {
  // a step of 64 inputs takes `half` where half of the compute units have a workgroup, `whole`
  // where all have, `shared` for each of several; one more round of workgroups takes `gap`, the
  // outputs of a workgroup whose rows are not aligned `odd`
  struct Tile {
    int bt, bn, fit;  // .. workgroups that share a unit
    double fixed, half, whole, shared, gap, odd;
  };
  static constexpr Tile kTiles[] = {{64, 64, 4, 3.1, 0.138, 0.150, 0.102, 0.1, 0.7},
                                    {64, 128, 2, 3.5, 0.161, 0.099, 0.127, 0.3, 1.7},
                                    {128, 128, 2, 4.3, 0.238, 0.227, 0.247, 2.8, 3.2},
                                    {128, 256, 1, 4.9, 0.347, 0.372, 0.371, 4.5, 3.4},
                                    {256, 256, 1, 7.0, 0.597, 0.740, 0.814, 4.2, 7.7}};
  const double bytes = (double)N * K;
  auto both = [](double a, double b) { return std::sqrt(a * a + b * b); };  // (two that overlap in part)
  MatPlan best{0, 0, 1, 1e30};
  if (T <= 128) {
    const int more = (T + 63) / 64 - 1;
    best.us = 4.1 + both(bytes * (N > 8192 ? 0.28e-6 + 0.155e-6 * more : 0.352e-6 + 0.338e-6 * more), K * 0.58e-3);
  }
  if (T <= 32) return best;
  for (const Tile& t : kTiles)
    for (int s = 1; s <= 8; s *= 2) {
      const int64_t nt = (T + t.bt - 1) / t.bt, wgs = (N + t.bn - 1) / t.bn * nt * s;
      if (s > 1 && (wgs > 640 || K < 512 * s)) break;
      if (wgs >= 1 << 23) continue;  // (a launch has less than 2^32 threads)
      const int64_t per = (wgs + 255) / 256, last = t.fit > 1 ? wgs : wgs - (per - 1) * 256;
      const double steps = (K + 127) / 128 * 2.0 / s;
      double work;
      if (per == 1 || t.fit == 1)
        work = steps * (t.half + (t.whole - t.half) * std::clamp(last / 128.0 - 1, 0.0, 1.0)) +
               (per - 1) * (t.gap + steps * t.shared);
      else
        work = steps * per * t.shared + ((per + t.fit - 1) / t.fit - 1) * t.gap;
      if (N % 4 && s == 1) work += per * t.odd;
      // (the weights pass from memory, and once more for every row of tiles, beside the work)
      double us = t.fixed + both(work, bytes * (0.235e-6 + 0.073e-6 * (nt - 1)));
      if (s > 1) us += 2.0 + 1.43e-6 * s * T * N;  // the parts' sums, and a launch
      if (us < best.us) best = MatPlan{t.bt, t.bn, s, us};
    }
  return best;
}

// Rows [t0, t0 + T) and channels [n0, n0 + N) of a product, one launch
struct MatPart {
  int t0, T, n0, N;
  MatPlan plan;
};
// The last round of large tiles may leave most compute units without one: where the estimate
// gains by it, whole rounds are one launch, and the rows or channels that are left another, of
// tiles that suit them. Returns the number of parts.
static int matmul_parts(int N, int K, int T, MatPart (&part)[2]) {
  part[0] = {0, T, 0, N, plan_of(N, K, T)};
  if (T <= 128 || part[0].plan.splits > 1) return 1;
  double least = part[0].plan.us * 0.98;
  int parts = 1;
  auto consider = [&](int T1, int N1) {
    if (T1 <= 0 || N1 <= 0 || (T1 >= T && N1 >= N)) return;
    const MatPart a{0, std::min(T1, T), 0, std::min(N1, N), plan_of(std::min(N1, N), K, std::min(T1, T))};
    const MatPart b = a.T < T ? MatPart{a.T, T - a.T, 0, N, plan_of(N, K, T - a.T)}
                              : MatPart{0, T, a.N, N - a.N, plan_of(N - a.N, K, T)};
    const double us = a.plan.us + b.plan.us + 1;
    if (us < least) least = us, part[0] = a, part[1] = b, parts = 2;
  };
  for (int bt : {128, 256}) {
    const int64_t nt = (T + bt - 1) / bt, nn = (N + 255) / 256, full = nt * nn / 256 * 256;
    if (full) {
      consider(T, (int)std::min<int64_t>(full / nt, nn - 1) * 256);
      consider((int)std::min<int64_t>(full / nn, nt - 1) * bt, N);
    }
  }
  return parts;
}

int64_t i8_weight_bytes(int N, int K) {
  const I8Shape s = i8_shape(N, K);
  return (int64_t)s.nb * s.ks * 1024;
}

static int64_t sums_bytes(const MatPart& p) {
  return p.plan.splits > 1 ? (int64_t)p.plan.splits * p.T * ((p.N + 31) / 32) * 128 : 0;
}
int64_t matmul_i8_ws(const sjd_i8_weights& w, int T) {
  MatPart p[2];
  return matmul_parts(w.N, w.K, T, p) == 1 ? sums_bytes(p[0]) : std::max(sums_bytes(p[0]), sums_bytes(p[1]));
}

static void launch_part(const sjd_i8_weights& w, const sjd_matmul_io& io, const MatPart& part, void* ws, hipStream_t s) {
  const MatPlan& p = part.plan;
  const int T = part.T, N = part.N;
  const I8Shape sh = i8_shape(N, w.K);
  const uintptr_t es = io.dtype == SJD_F32 ? 4 : 2;
  auto from = [&](const void* q, int64_t row) { return (char*)q + (part.t0 * row + part.n0) * es; };
  const MatArgs a{(const char*)w.d_w + i8_weight_bytes(part.n0, w.K), w.d_scale + part.n0,
                  io.d_code + part.t0 * io.code_row, io.d_code_scale + part.t0, from(io.d_out, io.out_row),
                  io.d_add ? from(io.d_add, io.add_row) : nullptr, io.code_row, io.out_row, io.add_row, T, N,
                  (w.K + 15) & ~15, sh.nb, sh.ks, io.dtype == SJD_F32, p.splits, (int32_t*)ws};
  if (!p.bt) {
    auto few = [&](auto ch, auto tt, auto depth, auto stage) {
      constexpr int CH = decltype(ch)::value, TT = decltype(tt)::value;
      hipLaunchKernelGGL((k_matmul_few<CH, TT, decltype(depth)::value, decltype(stage)::value>),
                         dim3((N + CH - 1) / CH, (T + CH * TT - 1) / (CH * TT)), dim3(64 * kFewWaves), 0, s, a);
    };
    const std::false_type direct;
    const std::true_type stage;
    // (16 channels to a workgroup where 32 leave compute units without one, or each with so few that
    // their ends show: us with weights from memory, several in turn, 16 and 32 channels, of 16 rows 4096 x
    // 4096 5.5 and 6.0, 12288 12.3 and 13.5, 22016 22.6 and 21.1; of 32 rows 4096 x 11008 15.1 and 17.9, 12288
    // x 4096 15.5 and 14.8. More loads in flight cost workgroups: depths 2, 3 and 4 of 32 rows, 22016 x 4096:
    // 22.6, 24.5, 25.8)
    if (T <= 8) few(Int<16>{}, Int<1>{}, Int<4>{}, direct);
    else if (T <= 16 && N <= 16384) few(Int<16>{}, Int<1>{}, Int<3>{}, stage);
    else if (T <= 32 && N > 8192) few(Int<32>{}, Int<1>{}, Int<2>{}, stage);
    else if (T <= 32) few(Int<16>{}, Int<2>{}, Int<2>{}, stage);
    else if (N > 8192) few(Int<32>{}, Int<2>{}, Int<1>{}, stage);
    else few(Int<16>{}, Int<4>{}, Int<4>{}, stage);
    return;
  }
  auto many = [&](auto bt, auto bn, auto vt, auto vn) {
    constexpr int BT = decltype(bt)::value, BN = decltype(bn)::value, VT = decltype(vt)::value, VN = decltype(vn)::value;
    if (p.bt != BT || p.bn != BN) return;
    const int nt = (T + BT - 1) / BT, nn = (N + BN - 1) / BN;
    hipLaunchKernelGGL((k_matmul_many<BT, BN, VT, VN>), dim3(nt * nn, p.splits), dim3(64 * VT * VN), 0, s, a, nt, nn);
  };
  many(Int<256>{}, Int<256>{}, Int<2>{}, Int<4>{});
  many(Int<128>{}, Int<256>{}, Int<2>{}, Int<4>{});
  many(Int<128>{}, Int<128>{}, Int<2>{}, Int<2>{});
  many(Int<64>{}, Int<128>{}, Int<2>{}, Int<2>{});
  many(Int<64>{}, Int<64>{}, Int<2>{}, Int<2>{});
  if (p.splits > 1) hipLaunchKernelGGL(k_matmul_join, dim3(T, (N + 1023) / 1024), dim3(256), 0, s, a);
}

hipError_t launch_matmul_i8(const sjd_i8_weights& w, const sjd_matmul_io& io, void* ws, hipStream_t s) {
  MatPart part[2];
  const int parts = matmul_parts(w.N, w.K, io.T, part);
  for (int i = 0; i < parts; ++i) launch_part(w, io, part[i], ws, s);
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
