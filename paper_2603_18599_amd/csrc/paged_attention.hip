// Attention of windows of new rows over a cache in pages (definition: sjd.h).
//
// The query heads of a key / value head and the rows of a window are one list of
// query slots (slot f: row f / G, head f % G), taken 32 at a time. Scores are
// formed transposed, S^T = K . Q^T, so a lane owns one slot and the softmax is
// lane-local but for one exchange between the wave's halves; the key rows that the
// tile layout feeds to the MFMA leave the probabilities in the order that O^T =
// V^T . P^T takes them in, so they never leave registers (v_mfma_f32_32x32x16_bf16).
// e4m3 codes become bf16 without rounding, times the key's power of two (an operand
// of the conversion); a value row's power multiplies its probability.
// 64 tokens over up to 8190 keys (8 heads, e4m3, 647 MB): 127 us, 5.1 TB/s, bound by
// memory (bf16 pages: 235). A prompt of 4096 rows over 4172 keys (bf16, 417 GFLOP): 434 to
// 463 us on several cards, 900 to 960 TFLOP/s (a library product: 1207). MFMAs keep the
// matrix units busy for 44% of its cycles and the softmax the vector units for about 40%;
// two waves per SIMD overlap them in part (waves wait 32% of their cycles, LDS is active
// in 22%).
#include <cmath>
#include <type_traits>

#include "device.h"
#include "forward.h"
#include "ops.h"

namespace sjd {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kMostSplits = 32;

struct PagedArgs {
  PoolView pv;
  sjd_windows w;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_row, out_row;
  const uint64_t* anc;
  int H, G;
  float scale;  // |scale| * log2(e);
  int negate;   // scale < 0: q changes sign
  int chunk, splits;
  int ws_rows;  // rows of a split in the workspace, see split_rows
  int ws_seq;   // .. of a sequence of them, or 0: rows of the tensors
  float* ws_o;  // [splits][ws_rows][H][HD] unnormalised outputs (splits > 1)
  float* ws_ml; // [splits][ws_rows][H][2] reference (log2 domain), sum
};
// The workspace has a place for each row of the tensors, or, where that is less, for
// each row that the windows can have: a few of them may lie anywhere in large tensors.
inline int split_rows(const sjd_windows& w) {
  const int64_t n = (int64_t)w.B * w.max_rows;
  return n < w.T ? (int)n : w.T;
}
SJD_DEV int split_row0(const PagedArgs& a, const Seq& sq, int z) { return a.ws_seq ? z * a.ws_seq : sq.row0; }

SJD_DEV uint32_t pk_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
template <bool HI>
SJD_DEV uint32_t pk_bf16_of_e4m3(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
}
SJD_DEV bf16x8 bf16_of_e4m3(uint2 c, float scale) {
  return __builtin_bit_cast(bf16x8, make_uint4(pk_bf16_of_e4m3<false>(c.x, scale), pk_bf16_of_e4m3<true>(c.x, scale),
                                               pk_bf16_of_e4m3<false>(c.y, scale), pk_bf16_of_e4m3<true>(c.y, scale)));
}

// One lane's part of a 32-position tile's keys, or of its values, as it lies in
// memory, and the MFMA operands that it makes: of keys step t, 8 dims of a key row;
// of values (d, jj), 8 positions from 16 jj of a column of dims block d.
template <int HD, bool FP8>
struct RawKeys {
  static constexpr int N = FP8 ? HD / 32 : HD / 16;
  static constexpr bool kCodes = FP8;
  uint4 x[N];
  uint32_t e;  // e4m3: exponent byte of the lane's key row, position swap23(lane % 32)
  SJD_DEV void load(const PagedArgs& a, const char* page, int h, int p0) {
    const int in = p0 & ((1 << a.pv.plen_log2) - 1), lane = threadIdx.x & 63;
    const char* p = page + tile_off<HD, FP8 ? 1 : 2>(a.pv, h, in, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = *(const uint4*)(p + (uint32_t)(16 * lane) + 1024 * i);
    if constexpr (FP8) e = (uint8_t)(page + exp_off<HD>(a.pv, h, 0) + in)[(uint32_t)swap23(lane & 31)];
  }
  SJD_DEV bf16x8 key(int t) const {
    if constexpr (FP8) {
      const uint4 y = x[t >> 1];
      return bf16_of_e4m3(t & 1 ? make_uint2(y.z, y.w) : make_uint2(y.x, y.y), __uint_as_float(e << 23));
    } else {
      return __builtin_bit_cast(bf16x8, x[t]);
    }
  }
};
template <int HD, bool FP8>
struct RawValues {
  static constexpr int N = FP8 ? HD / 32 : HD / 16;
  static constexpr bool kCodes = FP8;  // (and the operands lack their rows' powers of two)
  uint4 x[N];
  uint2 e[2];  // e4m3: exponent bytes of positions 16 jj + 8 half + 0 .. 7, the score registers'
  SJD_DEV void load(const PagedArgs& a, const char* page, int h, int p0) {
    const int in = p0 & ((1 << a.pv.plen_log2) - 1), lane = threadIdx.x & 63;
    const char* p = page + tile_off<HD, FP8 ? 1 : 2>(a.pv, h, in, 1);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = *(const uint4*)(p + (uint32_t)(16 * lane) + 1024 * i);
    if constexpr (FP8) {
      const char* q = page + exp_off<HD>(a.pv, h, 1) + in;
      e[0] = *(const uint2*)(q + (uint32_t)((lane & 32) >> 2));
      e[1] = *(const uint2*)(q + (uint32_t)((lane & 32) >> 2) + 16);
    }
  }
  SJD_DEV bf16x8 val(int d, int jj) const {
    if constexpr (FP8) {
      const uint4 y = x[d];
      return bf16_of_e4m3(jj ? make_uint2(y.z, y.w) : make_uint2(y.x, y.y), 1.0f);
    } else {
      return __builtin_bit_cast(bf16x8, x[d * 2 + jj]);
    }
  }
  SJD_DEV float power(int i) const {  // of score register i's value row
    const uint32_t w = (i & 7) < 4 ? e[i >> 3].x : e[i >> 3].y;
    return __uint_as_float(((w >> (8 * (i & 3))) & 0xFFu) << 23);
  }
};

// Both of a tile in LDS, widened to bf16: [key steps, then value blocks][lane]
template <int HD>
struct LdsTile {
  static constexpr bool kCodes = false;
  const uint4* at;
  SJD_DEV bf16x8 key(int t) const { return __builtin_bit_cast(bf16x8, at[64 * t + (threadIdx.x & 63)]); }
  SJD_DEV bf16x8 val(int d, int jj) const {
    return __builtin_bit_cast(bf16x8, at[64 * (HD / 16 + 2 * d + jj) + (threadIdx.x & 63)]);
  }
  SJD_DEV float power(int) const { return 1.0f; }
};

// Largest magnitude bits (of each half of a dword) of value operands seen so far;
// from kNotFinite on one of them is infinite or NaN
constexpr uint32_t kNotFinite = 0x7F80u;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
SJD_DEV uint32_t largest(uint32_t seen, bf16x8 v) {
  const uint4 u = __builtin_bit_cast(uint4, v);
  auto top = [](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
  };
  constexpr uint32_t kMag = 0x7FFF7FFFu;
  return top(top(seen, u.x & kMag), top(top(u.y & kMag, u.z & kMag), u.w & kMag));
}
SJD_DEV bool not_finite(uint32_t seen) { return (seen & 0xFFFFu) >= kNotFinite || (seen >> 16) >= kNotFinite; }
// Value operand (positions pos ..) with the positions from `lim` on cleared
SJD_DEV bf16x8 clear_from(bf16x8 v, int pos, int lim) {
  uint4 u = __builtin_bit_cast(uint4, v);
  uint32_t* w = (uint32_t*)&u;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] &= (pos + 2 * e < lim ? 0xFFFFu : 0u) | (pos + 2 * e + 1 < lim ? 0xFFFF0000u : 0u);
  return __builtin_bit_cast(bf16x8, u);
}

// The larger of v in lanes l and l ^ 32
SJD_DEV float max_of_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// One wave's state: 32 slots. m is the reference that probabilities are relative
// to: the largest score when it was last moved (log2 domain).
template <int HD>
struct WaveState {
  f32x16 o[HD / 32];
  float m, l;
};

// S^T of 32 keys. vis (MASKED): bit i says that register i's key is visible.
template <int HD, bool MASKED, class Keys, class Q>
SJD_DEV void scores(f32x16& c, const Keys& k, const Q& q, uint32_t vis) {
#pragma unroll
  for (int i = 0; i < 16; ++i) c[i] = 0.0f;
#pragma unroll
  for (int t = 0; t < HD / 16; ++t) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.key(t), q(t), c, 0, 0, 0);
  }
  if (MASKED)
#pragma unroll
    for (int i = 0; i < 16; ++i) c[i] = (vis >> i) & 1 ? c[i] : -INFINITY;
}

// The reference lies kLag above the largest score of the time when it was last moved,
// and moves when a score passes it. Most tiles so skip the rescaling of HD / 2 output
// registers, and probabilities stay between 2^-8 (a slot's largest) and 1: bf16 and
// float are relative, so a factor loses nothing, and neither a probability times an
// e4m3 row's power of two (up to 2^127) nor the sum of N of them, each times its
// value, passes N of the largest value. (A reference kLag below its ceiling let
// probabilities reach 2^8, and values 256 times smaller overflow.)
constexpr float kLag = 8.0f;
// A reference of this size is rounded to 2^-4 and larger ones to more, which the
// exact product under an exponent would show: past 2^31 as infinity or as zero.
constexpr float kHuge = 0x1p20f;

// Moves the reference if these scores ask for it, makes them probabilities and adds
// them to the sum.
template <int HD, int N, bool MASKED>
SJD_DEV void weigh(WaveState<HD>& s, f32x16 (&c)[N], float scale, const uint32_t (&vis)[N]) {
  float mx = c[0][0];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, c[n][i]);
  mx = max_of_halves(mx);
  mx = mx == -INFINITY ? mx : mx * scale;
  const bool move = mx > s.m;
  if (__any(move)) {
    // (each slot by itself: what its wave's other slots hold changes no bit of it)
    const float m = mx + kLag, alpha = move ? __builtin_amdgcn_exp2f(s.m - m) : 1.0f;
    s.m = move ? m : s.m;
    s.l *= alpha;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) s.o[d][i] *= alpha;
  }
  const float base = s.m == -INFINITY ? 0.0f : s.m;
  const bool huge = fabsf(base) >= kHuge;
  if (__any(huge)) {  // (products rounded as the reference's was)
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) c[n][i] = huge ? c[n][i] * scale : c[n][i];
    scale = huge ? 1.0f : scale;
  }
  float sum[4] = {};
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(c[n][i], scale, -base));
      c[n][i] = MASKED && !((vis[n] >> i) & 1) ? 0.0f : e;
      sum[i & 3] += c[n][i];
    }
  s.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// O^T += V^T . P^T for the 32 keys of c. MASKED: `lim` positions of the tile hold
// anything.
template <int HD, bool MASKED, class Values>
SJD_DEV void collect(WaveState<HD>& s, f32x16& c, const Values& r, uint32_t vis, int lim) {
  if constexpr (Values::kCodes)
#pragma unroll
    for (int i = 0; i < 16; ++i)  // (a masked position's exponent byte may be anything)
      c[i] = MASKED && !((vis >> i) & 1) ? 0.0f : c[i] * r.power(i);
  bf16x8 p[2];
#pragma unroll
  for (int jj = 0; jj < 2; ++jj)
    p[jj] = __builtin_bit_cast(bf16x8, make_uint4(pk_bf16(c[8 * jj], c[8 * jj + 1]), pk_bf16(c[8 * jj + 2], c[8 * jj + 3]),
                                                  pk_bf16(c[8 * jj + 4], c[8 * jj + 5]),
                                                  pk_bf16(c[8 * jj + 6], c[8 * jj + 7])));
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) {
    bf16x8 v[2] = {r.val(d, 0), r.val(d, 1)};
    uint32_t seen = 0;
    if (MASKED) {
      if (lim < kTile) {
        v[0] = clear_from(v[0], 8 * half, lim);
        v[1] = clear_from(v[1], 16 + 8 * half, lim);
      }
      seen = largest(largest(0, v[0]), v[1]);
    }
    if (MASKED && __any(not_finite(seen))) {
      // A value that is not finite: 0 * it would reach slots that do not attend
      // to its position. It is taken out, and each slot that attends to one of
      // its kind gets one added.
      auto kind_of = [](float x) { return x != x ? 2 : x == INFINITY ? 0 : x == -INFINITY ? 1 : 3; };
#pragma unroll 1
      for (int kind = 0; kind < 3; ++kind) {
        f32x16 cnt;
#pragma unroll
        for (int i = 0; i < 16; ++i) cnt[i] = 0.0f;
#pragma unroll
        for (int jj = 0; jj < 2; ++jj) {
          bf16x8 w, see;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            w[e] = (__bf16)(kind_of((float)v[jj][e]) == kind ? 1.0f : 0.0f);
            see[e] = (__bf16)((vis >> (8 * jj + e)) & 1 ? 1.0f : 0.0f);
          }
          cnt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, see, cnt, 0, 0, 0);
        }
        const float add = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : __builtin_nanf("");
#pragma unroll
        for (int i = 0; i < 16; ++i) s.o[d][i] += cnt[i] > 0.0f ? add : 0.0f;
      }
#pragma unroll
      for (int jj = 0; jj < 2; ++jj)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[jj][e] = kind_of((float)v[jj][e]) == 3 ? v[jj][e] : (__bf16)0.0f;
    }
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) s.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[jj], p[jj], s.o[d], 0, 0, 0);

  }
}

// A lane's slot: row f / G of the window, query head f % G of the group
struct Slot {
  int row, head;
  bool ok;
  int64_t t;  // row of the tensors
  uint64_t mask;
};
SJD_DEV Slot slot_of(const PagedArgs& a, const Seq& sq, int h, int f) {
  Slot s;
  s.ok = f < sq.rows * a.G;
  s.row = f / a.G;
  s.head = h * a.G + f % a.G;
  s.t = sq.row0 + (s.ok ? s.row : 0);
  s.mask = a.anc && s.ok ? a.anc[s.t] : 0;
  return s;
}
// Piece i of a slot's q: dims half * HD / 2 + 8 i .. (zeros for a slot that is not there)
template <int HD>
SJD_DEV uint4 load_q(const PagedArgs& a, const Slot& sl, int i) {
  const int half = (threadIdx.x & 63) >> 5;
  const uint32_t sign = a.negate ? 0x80008000u : 0u;
  // (a slot that is not there reads the window's first row: no branch, no wait)
  const uint4 x = ((const uint4*)(a.q + sl.t * a.q_row + (sl.ok ? sl.head : 0) * HD + half * (HD / 2)))[i];
  const uint32_t keep = sl.ok ? ~0u : 0u;
  return make_uint4((x.x ^ sign) & keep, (x.y ^ sign) & keep, (x.z ^ sign) & keep, (x.w ^ sign) & keep);
}
template <int HD>
SJD_DEV void start(WaveState<HD>& s) {
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) s.o[d][i] = 0.0f;
  s.m = -INFINITY;
  s.l = 0.0f;
}

// Visible score registers of a lane with slot sl, for the tile of positions p0 ..:
// first as a mask of the tile's positions, which are visible up to the slot's own
// row, or where the ancestor mask, moved to the window's place in the tile, says so
SJD_DEV uint32_t visible(const PagedArgs& a, const Seq& sq, int p0, const Slot& sl) {
  auto below = [](int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; };  // positions 0 .. n - 1
  const int d = sq.cached - p0;  // the window's first row is position d of the tile
  uint32_t m;
  if (a.anc) {
    const uint32_t moved = d >= 32 ? 0u : d >= 0 ? (uint32_t)sl.mask << d : d > -64 ? (uint32_t)(sl.mask >> -d) : 0u;
    m = (below(d) | moved) & below(d + sq.rows);
  } else {
    m = below(d + min(sl.row + 1, sq.rows));
  }
  if (!sl.ok) m = 0;
  // register i holds position 16 (i / 8) + 8 half + i % 8
  m >>= 8 * ((threadIdx.x & 63) >> 5);
  return (m & 0xFFu) | (m >> 8 & 0xFF00u);
}

// Few slots: 32 of one key / value head of one sequence per workgroup; its four
// waves take every fourth tile of the split's keys, straight from memory to
// registers with the next tile's loads behind this one's arithmetic, and merge in
// LDS.
constexpr int kRound = 4 * kTile;  // keys of the four waves

template <int HD>
struct MergeSmem {
  uint4 q[HD / 16][kWave];
  float o[4][32][HD + 1];
  float m[4][32], l[4][32];
};

template <int HD, bool FP8>
__global__ __launch_bounds__(256, 2) void k_paged_attn(PagedArgs a) {
  constexpr int ND = HD / 32;
  __shared__ MergeSmem<HD> sm;
  const int h = blockIdx.x % a.pv.Hkv, sp = blockIdx.x / a.pv.Hkv, z = blockIdx.z;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int beg = sp * a.chunk;
  int p0 = beg + kTile * wave;
  // (page ids do not wait for the sequence: inside the table there is something to read)
  auto id_of = [&](int p) { return (p >> a.pv.plen_log2) < a.w.table_len ? page_id(a.w, a.pv, z, p) : -1; };
  const int id = id_of(p0);
  int id_next = id_of(p0 + kRound);
  const Seq sq = load_seq(a.w, a.pv, z);
  const int slots = sq.rows * a.G, f0 = blockIdx.y * 32;
  if (f0 >= slots) return;
  // causal: the last row of these slots bounds their keys
  const int total = sq.cached + sq.rows, last = min(sq.rows - 1, (f0 + 31) / a.G);
  const int end = min(a.anc ? total : sq.cached + last + 1, beg + a.chunk), full = min(sq.cached, end);
  if (beg >= total) return;
  const Slot sl = slot_of(a, sq, h, f0 + (lane & 31));
  RawKeys<HD, FP8> k;
  RawValues<HD, FP8> v;
  bool ok;  // (a tile that is left out holds the pool's first one: loads without a branch)
  auto source = [&](bool inside, int page) {
    const char* pg = inside ? page_at(a.pv, page) : nullptr;
    ok = pg != nullptr;
    return ok ? pg : a.pv.pool;
  };
  {
    const char* pg = source(p0 < end, id);
    k.load(a, pg, h, p0);
    v.load(a, pg, h, p0);
  }
#pragma unroll
  for (int i = wave; i < HD / 16; i += 4) sm.q[i][lane] = load_q<HD>(a, sl, i);
  WaveState<HD> s;
  start(s);
  __syncthreads();
  const auto q = [&](int t) { return __builtin_bit_cast(bf16x8, sm.q[t][lane]); };
  // One tile, and the loads of the next one into its registers: the keys' once the
  // scores are formed, the values' once they are used up. (A second set of registers
  // for them is no faster at 64 dims and spills at 128.)
  auto step = [&](auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    const bool now = ok;
    const int p = p0, np = p0 + kRound;
    const char* next = source(np < end, id_next);
    id_next = id_of(np + kRound);
    p0 = np;
    if (!now) {
      k.load(a, next, h, np);
      v.load(a, next, h, np);
      return;
    }
    const uint32_t vis[1] = {MASKED ? visible(a, sq, p, sl) : 0xFFFFu};
    f32x16 c[1];
    scores<HD, MASKED>(c[0], k, q, vis[0]);
    k.load(a, next, h, np);
    weigh<HD, 1, MASKED>(s, c, a.scale, vis);
    collect<HD, MASKED>(s, c[0], v, vis[0], total - p);
    v.load(a, next, h, np);
  };
  while (p0 + kTile <= full) step(std::false_type{});
  while (p0 < end) step(std::true_type{});
  s.l += __shfl_xor(s.l, 32, kWave);
  // register i of block d holds dim 32 d + 8 (i / 4) + 4 half + i % 4
  if (sl.ok)
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) sm.o[wave][lane & 31][d * 32 + 8 * (i >> 2) + 4 * half + (i & 3)] = s.o[d][i];
  if (half == 0) {
    sm.m[wave][lane] = s.m;
    sm.l[wave][lane] = s.l;
  }
  __syncthreads();
  constexpr int DPT = HD / 8;
  const int sn = threadIdx.x >> 3, d0 = (threadIdx.x & 7) * DPT;
  const int g = f0 + sn;
  if (g >= slots) return;
  float mx = -INFINITY;
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm.m[w][sn]);
  float y[DPT] = {}, l = 0.0f;
  for (int w = 0; w < 4; ++w) {
    const float fw = mx == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(sm.m[w][sn] - mx);
    l += sm.l[w][sn] * fw;
#pragma unroll
    for (int i = 0; i < DPT; ++i) y[i] += sm.o[w][sn][d0 + i] * fw;
  }
  const int64_t tt = sq.row0 + g / a.G;
  const int hh = h * a.G + g % a.G;
  if (a.splits == 1) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // (no key at all: zeros)
    uint4* o = (uint4*)(a.out + tt * a.out_row + hh * HD + d0);
#pragma unroll
    for (int i = 0; i < DPT / 8; ++i)
      o[i] = make_uint4(pk_bf16(y[8 * i] * inv, y[8 * i + 1] * inv), pk_bf16(y[8 * i + 2] * inv, y[8 * i + 3] * inv),
                        pk_bf16(y[8 * i + 4] * inv, y[8 * i + 5] * inv), pk_bf16(y[8 * i + 6] * inv, y[8 * i + 7] * inv));
    return;
  }
  const int64_t at = ((int64_t)sp * a.ws_rows + split_row0(a, sq, z) + g / a.G) * a.H + hh;
#pragma unroll
  for (int i = 0; i < DPT; i += 4)
    *(float4*)(a.ws_o + at * HD + d0 + i) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
  if ((threadIdx.x & 7) == 0) *(float2*)(a.ws_ml + at * 2) = make_float2(mx, l);
}

// Many slots: 128 of them per workgroup, 32 per wave, and every wave takes every
// key. Steps of 64 keys pass through LDS, widened to bf16 by the threads that load
// them (once for the four waves), in two buffers: a step's loads are issued before
// the arithmetic of the step before it and stored behind it.
constexpr int kStep = 64, kStepTiles = kStep / kTile;

template <int HD, bool FP8>
struct Stage {
  static constexpr int HP = FP8 ? HD * 2 : HD * 4;     // 16-byte pieces of a tile's keys
  static constexpr int N = kStepTiles * 2 * HP / 256;  // pieces per thread
  static constexpr int TILE = 2 * (HD / 16) * 64;      // uint4 of a tile in LDS
  uint4 x[FP8 ? N : 1];
  uint2 e[FP8 ? N : 1][2];  // exponent bytes: a key row's, or those of 16 positions
  // piece i of this thread: tile, key or value, place in its part
  static SJD_DEV void where(int i, int& tile, int& kv, int& u) {
    static_assert(2 * HP % 256 == 0, "a round of the workgroup stays inside a tile");
    int tid = (int)threadIdx.x;
    const int n = i * 256;
    asm volatile("" : "+v"(tid));  // (lane offsets are made anew: kept across the step they cost registers that it lacks)
    tile = n / (2 * HP);
    kv = HP >= 256 ? n / HP & 1 : __builtin_amdgcn_readfirstlane(tid / HP);
    u = HP >= 256 ? n % HP + tid : tid % HP;
  }
  // Starts the loads of positions p0 .. (a page that is NULL: its tile is not read;
  // nor is what LDS holds there used)
  SJD_DEV void load(const PagedArgs& a, const char* const (&page)[kStepTiles], int h, int p0, uint4* lds) {
    constexpr int ES = FP8 ? 1 : 2;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int tile, kv, u;
      where(i, tile, kv, u);
      const char* pg = tile ? page[1] : page[0];
      if (!pg) continue;
      const int in = (p0 + 32 * tile) & ((1 << a.pv.plen_log2) - 1);
      const uint4* src = (const uint4*)(pg + tile_off<HD, ES>(a.pv, h, in, kv)) + (uint32_t)u;
      if constexpr (FP8) {
        x[i] = *src;
        const char* ep = pg + exp_off<HD>(a.pv, h, kv) + in;
        if (kv) {
          const uint2* e2 = (const uint2*)ep + (uint32_t)(u >> 5 & 1);
          e[i][0] = e2[0];
          e[i][1] = e2[2];
        } else {
          e[i][0].x = (uint8_t)ep[(uint32_t)swap23(u & 31)];
        }
      } else {
        // a wave's 1 KB lands in lane order behind a uniform address
        uint4* d = lds + tile * TILE + kv * (TILE / 2) + (u & ~63);
        __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)src,
                                         (void __attribute__((address_space(3)))*)d, 16, 0, 0);
      }
    }
  }
  // Ends them: what was loaded is in LDS (of this wave's pieces)
  SJD_DEV void store(uint4* lds) const {
    if constexpr (!FP8) {
      __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        int tile, kv, u;
        where(i, tile, kv, u);
        uint4* d = lds + tile * TILE + kv * (TILE / 2) + (u >> 6) * 128 + (u & 63);
        if (kv) {
          d[0] = widen(make_uint2(x[i].x, x[i].y), e[i][0]);
          d[64] = widen(make_uint2(x[i].z, x[i].w), e[i][1]);
        } else {
          const float f = __uint_as_float(e[i][0].x << 23);
          d[0] = __builtin_bit_cast(uint4, bf16_of_e4m3(make_uint2(x[i].x, x[i].y), f));
          d[64] = __builtin_bit_cast(uint4, bf16_of_e4m3(make_uint2(x[i].z, x[i].w), f));
        }
      }
    }
  }
  // 8 codes, each with its own exponent byte
  static SJD_DEV uint4 widen(uint2 c, uint2 e) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t cc = j < 2 ? c.x : c.y, ee = (j < 2 ? e.x : e.y) >> (16 * (j & 1));
      const f32x2 v = j & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)cc, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)cc, false);
      w[j] = pk_bf16(v[0] * __uint_as_float((ee & 0xFFu) << 23), v[1] * __uint_as_float((ee >> 8 & 0xFFu) << 23));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

template <int HD, bool FP8>
__global__ __launch_bounds__(256, 2) void k_paged_chunk(PagedArgs a) {
  constexpr int ND = HD / 32;
  using St = Stage<HD, FP8>;
  __shared__ uint4 lds[2][kStepTiles * St::TILE];
  const int h = blockIdx.x, z = blockIdx.z;
  const Seq sq = load_seq(a.w, a.pv, z);
  // (the last slots of a causal window have the most keys: they start first)
  const int slots = sq.rows * a.G, f0 = ((int)gridDim.y - 1 - (int)blockIdx.y) * 128;
  if (f0 >= slots) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int total = sq.cached + sq.rows;
  const int end = a.anc ? total : sq.cached + min(sq.rows - 1, (f0 + 127) / a.G) + 1;
  const int w0 = f0 + 32 * wave;
  const Slot sl = slot_of(a, sq, h, w0 + (lane & 31));
  uint4 qr[HD / 16];
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) qr[i] = load_q<HD>(a, sl, i);
  const auto q = [&](int t) { return __builtin_bit_cast(bf16x8, qr[t]); };
  WaveState<HD> s;
  start(s);
  // keys that every slot of the workgroup sees, and that any slot of this wave sees
  const int all = a.anc ? sq.cached : sq.cached + f0 / a.G + 1;
  const int any = w0 >= slots ? 0 : a.anc ? total : sq.cached + min(sq.rows - 1, (w0 + 31) / a.G) + 1;

  // page ids are read two steps ahead of their use, loads of the pages one
  auto ids = [&](int p0, int (&id)[kStepTiles]) {
#pragma unroll
    for (int n = 0; n < kStepTiles; ++n) id[n] = p0 + 32 * n < end ? page_id(a.w, a.pv, z, p0 + 32 * n) : -1;
  };
  auto pages = [&](const int (&id)[kStepTiles], const char* (&pg)[kStepTiles]) {
#pragma unroll
    for (int n = 0; n < kStepTiles; ++n) pg[n] = page_at(a.pv, id[n]);
  };
  St st;
  const char* pg[kStepTiles];
  int id[kStepTiles];
  ids(0, id);
  pages(id, pg);
  ids(kStep, id);
  st.load(a, pg, h, 0, lds[0]);
  st.store(lds[0]);
  __syncthreads();
  int buf = 0, p0 = 0;
  // One step: the next one's loads, `work` on this one, and the loads' end
  auto step = [&](auto work) {
    const char* next[kStepTiles];
    const bool more = p0 + kStep < end;
    if (more) {
      pages(id, next);
      ids(p0 + 2 * kStep, id);
      st.load(a, next, h, p0 + kStep, lds[buf ^ 1]);
    }
    work();
    if (more) {
      st.store(lds[buf ^ 1]);
      pg[0] = next[0];
      pg[1] = next[1];
    }
    __syncthreads();
    buf ^= 1;
    p0 += kStep;
  };
  // keys without a mask (in a loop of its own: it needs fewer registers), then the rest
  while (p0 + kStep <= min(all, end) && pg[0] && pg[1])
    step([&] {
      const uint32_t vis[kStepTiles] = {0xFFFFu, 0xFFFFu};
      f32x16 c[kStepTiles];
#pragma unroll
      for (int n = 0; n < kStepTiles; ++n) scores<HD, false>(c[n], LdsTile<HD>{lds[buf] + n * St::TILE}, q, vis[n]);
      weigh<HD, kStepTiles, false>(s, c, a.scale, vis);
#pragma unroll
      for (int n = 0; n < kStepTiles; ++n) collect<HD, false>(s, c[n], LdsTile<HD>{lds[buf] + n * St::TILE}, vis[n], 32);
    });
  while (p0 < end)
    step([&] {
#pragma unroll 1
      for (int n = 0; n < kStepTiles; ++n) {
        const int p = p0 + 32 * n;
        if (!pg[n] || p >= any) continue;
        const LdsTile<HD> t{lds[buf] + n * St::TILE};
        const uint32_t vis[1] = {visible(a, sq, p, sl)};
        f32x16 c[1];
        scores<HD, true>(c[0], t, q, vis[0]);
        weigh<HD, 1, true>(s, c, a.scale, vis);
        collect<HD, true>(s, c[0], t, vis[0], total - p);
      }
    });
  s.l += __shfl_xor(s.l, 32, kWave);
  if (!sl.ok) return;
  // register i of block d holds dim 32 d + 8 (i / 4) + 4 half + i % 4
  const float inv = s.l == 0.0f ? 0.0f : 1.0f / s.l;  // (no key at all: zeros)
  uint16_t* o = a.out + sl.t * a.out_row + sl.head * HD + 4 * half;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *(uint2*)(o + d * 32 + 2 * i) = make_uint2(pk_bf16(s.o[d][i] * inv, s.o[d][i + 1] * inv),
                                                 pk_bf16(s.o[d][i + 2] * inv, s.o[d][i + 3] * inv));
}

// Joins the splits of a row: one wave per (row, head).
template <int HD>
__global__ __launch_bounds__(256) void k_paged_join(PagedArgs a) {
  const int z = blockIdx.y, i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const Seq sq = load_seq(a.w, a.pv, z);
  if (i >= sq.rows * a.H) return;
  const int64_t t = sq.row0 + i / a.H;
  const int hh = i % a.H;
  const int n = (sq.cached + sq.rows + a.chunk - 1) / a.chunk;
  // (place i of the sequence's (row, head) pairs)
  const int64_t at = (int64_t)split_row0(a, sq, z) * a.H + i, step = (int64_t)a.ws_rows * a.H;
  // A lane reads one split's statistics and every lane its dims of each split, the
  // first 8 before anything waits for the statistics
  constexpr int W = HD / 64, kBatch = 8;
  static_assert(kMostSplits <= kWave, "one lane per split");
  const float2 ml = lane < n ? *(const float2*)(a.ws_ml + (at + lane * step) * 2) : make_float2(-INFINITY, 0.0f);
  float x[kBatch][W], v[W] = {};
  auto read = [&](int k) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
#pragma unroll
      for (int e = 0; e < W; ++e) x[u][e] = k + u < n ? a.ws_o[(at + (k + u) * step) * HD + lane * W + e] : 0.0f;
  };
  read(0);
  const float mx = wave_max_dpp(ml.x);
  const float f = mx == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml.x - mx);
  const float l = wave_sum(lane < n ? ml.y * f : 0.0f);
  for (int k = 0;;) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (k + u < n) {
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), k + u));
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] += x[u][e] * w;
      }
    k += kBatch;
    if (k >= n) break;
    read(k);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t* o = a.out + t * a.out_row + hh * HD + lane * (HD / 64);
  if constexpr (HD == 128) *(uint32_t*)o = pk_bf16(v[0] * inv, v[1] * inv);
  else *o = (uint16_t)pk_bf16(v[0] * inv, 0.0f);
}

template <int HD, bool FP8>
void launch_head(const PagedArgs& a, const AttnPlan& pl, dim3 grid, hipStream_t s) {
  if (pl.few) hipLaunchKernelGGL((k_paged_attn<HD, FP8>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_paged_chunk<HD, FP8>), grid, dim3(256), 0, s, a);
}

}  // namespace

// Up to this many tiles of 32 slots the waves of a workgroup share out the keys;
// more are many slots for one sequence and head, whose keys are worth sharing. us,
// 32 query and 8 key / value heads of 128, e4m3 (bf16), keys shared out -> shared:
//   1536 tiles (24 windows of 64 rows, 1239 cached)    39 (38) -> 78 (72)
//   2048 tiles (32 of 64, 1239)                        52 (50) -> 50 (44)
//   2048 tiles (32 of 64, 4172)                       117 (148) -> 139 (127)
//   16384 tiles (1 of 4096, 4172)                     618 (656) -> 466 (436)
// With up to 64 slots half of a 128-slot workgroup idles (64 of 16 rows, 4172: 115
// -> 139).
constexpr int kFewTiles = 1536;
// Splits: as many as give two workgroups to each of 256 compute units, of one tile
// per wave at least. More even out ragged sequences, but their partial outputs and
// the second launch cost more: 64 single tokens over up to 8190 keys, 512 / 1024
// workgroups: 127 / 131 us; 8 windows of 64 rows over 2000, 23 / 38. Past 32 the join's
// rounds cost more than the splits save (a token of one key / value head over 8190
// keys, 64 splits -> 32: 13.2 -> 11.3 us; over 30000, 235 -> 32: 29.7 -> 15.4).
constexpr int kSplitWgs = 512;
AttnPlan paged_attention_plan(const sjd_pages& p, const sjd_windows& w, int H) {
  const int64_t most = (int64_t)w.max_cached + w.max_rows;
  const int64_t slots = (int64_t)w.max_rows * (H / p.n_kv_heads);
  const int64_t tiles = (int64_t)w.B * p.n_kv_heads * ((slots + 31) / 32);
  const bool few = slots <= 64 || tiles <= kFewTiles;
  int64_t S = few ? (kSplitWgs + tiles - 1) / tiles : 1;
  if (S > (most + kRound - 1) / kRound) S = (most + kRound - 1) / kRound;
  if (S > kMostSplits) S = kMostSplits;
  const int64_t chunk = ((most + S - 1) / S + kRound - 1) / kRound * kRound;
  return AttnPlan{(int)chunk, (int)((most + chunk - 1) / chunk), few};
}

int64_t paged_attention_ws(const sjd_pages& p, const sjd_windows& w, int H) {
  const AttnPlan pl = paged_attention_plan(p, w, H);
  if (pl.splits <= 1) return 0;
  return (int64_t)pl.splits * split_rows(w) * H * (p.head_dim + 2) * 4;
}

hipError_t launch_paged_attention(const sjd_pages& p, const sjd_windows& w, const sjd_attention_io& io, void* ws,
                                  hipStream_t s) {
  const AttnPlan pl = paged_attention_plan(p, w, io.H);
  PagedArgs a{};
  a.pv = pool_view(p); a.w = w; a.q = (const uint16_t*)io.d_q; a.out = (uint16_t*)io.d_out;
  a.q_row = io.q_row; a.out_row = io.out_row; a.anc = io.d_anc; a.H = io.H; a.G = io.H / p.n_kv_heads;
  a.scale = log2_scale(io.scale);
  a.negate = io.scale < 0.0f ? 1 : 0;
  a.chunk = pl.chunk; a.splits = pl.splits;
  a.ws_rows = split_rows(w);
  a.ws_seq = a.ws_rows < w.T ? w.max_rows : 0;
  a.ws_o = (float*)ws;
  a.ws_ml = ws ? (float*)ws + (int64_t)pl.splits * a.ws_rows * io.H * p.head_dim : nullptr;
  const int slots = w.max_rows * a.G, per = pl.few ? 32 : 128;
  const dim3 grid(p.n_kv_heads * pl.splits, (slots + per - 1) / per, w.B);
  const bool f8 = p.dtype == SJD_E4M3;
  if (p.head_dim == 128) f8 ? launch_head<128, true>(a, pl, grid, s) : launch_head<128, false>(a, pl, grid, s);
  else f8 ? launch_head<64, true>(a, pl, grid, s) : launch_head<64, false>(a, pl, grid, s);
  if (pl.splits > 1) {
    const dim3 jg((unsigned)(((int64_t)w.max_rows * io.H + 3) / 4), w.B);
    if (p.head_dim == 128) hipLaunchKernelGGL(k_paged_join<128>, jg, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(k_paged_join<64>, jg, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace sjd
