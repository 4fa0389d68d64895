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
#include "device.h"
#include "ops.h"

namespace sjd {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct PagedArgs {
  PoolView pv;
  sjd_windows w;
  const uint16_t* q;
  uint16_t* out;
  int64_t q_row, out_row;
  const uint64_t* anc;
  int H, G;
  float scale;  // times log2(e)
  int chunk, splits;
  float* ws_o;  // [splits][T][H][HD] unnormalised outputs (splits > 1)
  float* ws_ml; // [splits][T][H][2] maximum (log2 domain), sum
};

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

// One lane's part of a 32-position tile as it lies in memory
template <int HD, bool FP8>
struct RawTile {
  static constexpr int NK = FP8 ? HD / 32 : HD / 16;  // 16-byte pieces of keys, and of values
  uint4 k[NK], v[NK];
  uint32_t ke;   // e4m3: exponent byte of the lane's key row,
  uint2 ve[2];   // and of the 16 positions that its score registers hold
};

// MFMA operand of 8 dims of a key row (step t), of 8 positions of a value column
// (dims block d, positions 16 jj ..)
template <int HD, bool FP8>
SJD_DEV bf16x8 key_frag(const RawTile<HD, FP8>& r, int t, float ks) {
  if constexpr (FP8) {
    const uint4 x = r.k[t >> 1];
    return bf16_of_e4m3(t & 1 ? make_uint2(x.z, x.w) : make_uint2(x.x, x.y), ks);
  } else {
    return __builtin_bit_cast(bf16x8, r.k[t]);
  }
}
template <int HD, bool FP8>
SJD_DEV bf16x8 val_frag(const RawTile<HD, FP8>& r, int d, int jj) {
  if constexpr (FP8) {
    const uint4 x = r.v[d];
    return bf16_of_e4m3(jj ? make_uint2(x.z, x.w) : make_uint2(x.x, x.y), 1.0f);
  } else {
    return __builtin_bit_cast(bf16x8, r.v[d * 2 + jj]);
  }
}

// Loads the tile of positions p0 .. p0 + 31 (page: its page)
template <int HD, bool FP8>
SJD_DEV void load_tile(RawTile<HD, FP8>& r, const PagedArgs& a, const char* page, int h, int p0) {
  constexpr int ES = FP8 ? 1 : 2;
  const int in = p0 & ((1 << a.pv.plen_log2) - 1), lane = threadIdx.x & 63;
  const uint4* k = (const uint4*)(page + tile_off<HD, ES>(a.pv, h, in, 0)) + lane;
  const uint4* v = (const uint4*)(page + tile_off<HD, ES>(a.pv, h, in, 1)) + lane;
#pragma unroll
  for (int i = 0; i < RawTile<HD, FP8>::NK; ++i) r.k[i] = k[64 * i];
#pragma unroll
  for (int i = 0; i < RawTile<HD, FP8>::NK; ++i) r.v[i] = v[64 * i];
  if constexpr (FP8) {
    // a lane's MFMA key row is position swap23(lane % 32); its score registers 8 jj
    // + e hold positions 16 jj + 8 half + e
    const int i = lane & 31, sw = (i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1);
    r.ke = (uint8_t)page[exp_off<HD>(a.pv, h, 0) + in + sw];
    const char* e = page + exp_off<HD>(a.pv, h, 1) + in + 8 * (lane >> 5);
    r.ve[0] = *(const uint2*)e;
    r.ve[1] = *(const uint2*)(e + 16);
  }
}

// Clears the values of positions from `lim` of the tile on, and says whether any
// other value of this lane is not finite
template <int HD, bool FP8>
SJD_DEV bool clean_values(RawTile<HD, FP8>& r, int lim) {
  const int half = (threadIdx.x & 63) >> 5;
  bool bad = false;
  auto fix = [&](uint32_t w, int pos) {  // 4 codes or 2 bf16 from position pos on
    constexpr int PER = FP8 ? 4 : 2, BITS = 32 / PER;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const uint32_t m = (FP8 ? 0xFFu : 0xFFFFu) << (BITS * e);
      if (pos + e >= lim) w &= ~m;
      const uint32_t x = (w >> (BITS * e)) & (FP8 ? 0x7Fu : 0x7F80u);
      bad |= x == (FP8 ? 0x7Fu : 0x7F80u);
    }
    return w;
  };
#pragma unroll
  for (int i = 0; i < RawTile<HD, FP8>::NK; ++i) {
    const int p = 8 * half + (FP8 ? 0 : 16 * (i & 1));
    r.v[i].x = fix(r.v[i].x, p);
    r.v[i].y = fix(r.v[i].y, p + (FP8 ? 4 : 2));
    r.v[i].z = fix(r.v[i].z, p + (FP8 ? 16 : 4));
    r.v[i].w = fix(r.v[i].w, p + (FP8 ? 20 : 6));
  }
  return bad;
}

// One wave's state: 32 slots
template <int HD>
struct WaveState {
  bf16x8 q[HD / 16];
  f32x16 o[HD / 32];
  float m, l;
};

// Bit r of a lane's mask: its score register r is visible
template <int HD, bool FP8, bool MASKED>
SJD_DEV void attend_tile(WaveState<HD>& s, RawTile<HD, FP8>& r, float scale, uint32_t vis, int lim) {
  constexpr int ND = HD / 32;
  f32x16 c;
#pragma unroll
  for (int i = 0; i < 16; ++i) c[i] = 0.0f;
  const float ks = FP8 ? __uint_as_float(r.ke << 23) : 1.0f;
#pragma unroll
  for (int t = 0; t < HD / 16; ++t)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_frag<HD, FP8>(r, t, ks), s.q[t], c, 0, 0, 0);
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    c[i] = !MASKED || ((vis >> i) & 1) ? c[i] * scale : -INFINITY;
    mx = fmaxf(mx, c[i]);
  }
  mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
  const float m = fmaxf(s.m, mx), base = m == -INFINITY ? 0.0f : m;
  const float alpha = __builtin_amdgcn_exp2f(s.m - base);
  s.m = m;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    c[i] = __builtin_amdgcn_exp2f(c[i] - base);
    sum += c[i];
  }
  s.l = s.l * alpha + sum;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) s.o[d][i] *= alpha;
  if constexpr (FP8) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = (i & 7) < 4 ? r.ve[i >> 3].x : r.ve[i >> 3].y;
      const float f = __uint_as_float(((w >> (8 * (i & 3))) & 0xFFu) << 23);
      // (a masked position's exponent may be anything)
      c[i] = MASKED && !((vis >> i) & 1) ? 0.0f : c[i] * f;
    }
  }
  bf16x8 p[2];
#pragma unroll
  for (int jj = 0; jj < 2; ++jj)
    p[jj] = __builtin_bit_cast(bf16x8, make_uint4(pk_bf16(c[8 * jj], c[8 * jj + 1]), pk_bf16(c[8 * jj + 2], c[8 * jj + 3]),
                                                  pk_bf16(c[8 * jj + 4], c[8 * jj + 5]),
                                                  pk_bf16(c[8 * jj + 6], c[8 * jj + 7])));
  if constexpr (MASKED) {
    if (__any(clean_values<HD, FP8>(r, lim))) {
      // A value that is not finite: 0 * it would reach slots that do not attend
      // to its position. It is taken out, and each slot that attends to one of its
      // kind gets one added.
      auto kind_of = [](float x) { return x != x ? 2 : x == INFINITY ? 0 : x == -INFINITY ? 1 : 3; };
      bf16x8 see[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) see[i >> 3][i & 7] = (__bf16)((vis >> i) & 1 ? 1.0f : 0.0f);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        for (int kind = 0; kind < 3; ++kind) {
          f32x16 n;
#pragma unroll
          for (int i = 0; i < 16; ++i) n[i] = 0.0f;
#pragma unroll
          for (int jj = 0; jj < 2; ++jj) {
            const bf16x8 v = val_frag<HD, FP8>(r, d, jj);
            bf16x8 w;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = (__bf16)(kind_of((float)v[e]) == kind ? 1.0f : 0.0f);
            n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, see[jj], n, 0, 0, 0);
          }
          const float add = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : __builtin_nanf("");
#pragma unroll
          for (int i = 0; i < 16; ++i) s.o[d][i] += n[i] > 0.0f ? add : 0.0f;
        }
#pragma unroll
        for (int jj = 0; jj < 2; ++jj) {
          bf16x8 v = val_frag<HD, FP8>(r, d, jj);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = kind_of((float)v[e]) == 3 ? v[e] : (__bf16)0.0f;
          s.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[jj], s.o[d], 0, 0, 0);
        }
      }
      return;
    }
  }
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int jj = 0; jj < 2; ++jj)
      s.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(val_frag<HD, FP8>(r, d, jj), p[jj], s.o[d], 0, 0, 0);
}

// Visible score registers of a lane whose slot is window row `row` (ok: there is
// such a row), for the tile of positions p0 ..
SJD_DEV uint32_t visible(const Seq& sq, int p0, int row, bool ok, const uint64_t* anc, uint64_t mask) {
  const int half = (threadIdx.x & 63) >> 5, nk = sq.cached + sq.rows;
  uint32_t v = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int p = p0 + 16 * (i >> 3) + 8 * half + (i & 7), w = p - sq.cached;
    const bool see = p < nk && (w < 0 || (anc ? (mask >> (w & 63)) & 1 : w <= row));
    v |= (uint32_t)(ok && see) << i;
  }
  return v;
}

// 32 slots of one key / value head of one sequence per workgroup; the four waves
// take every fourth tile of the split's keys and merge in LDS.
template <int HD>
struct MergeSmem {
  float o[4][32][HD + 1];
  float m[4][32], l[4][32];
};

template <int HD, bool FP8>
__global__ __launch_bounds__(256) void k_paged_attn(PagedArgs a) {
  constexpr int ND = HD / 32;
  __shared__ MergeSmem<HD> sm;
  const int h = blockIdx.x % a.pv.Hkv, sp = blockIdx.x / a.pv.Hkv, z = blockIdx.z;
  const Seq sq = load_seq(a.w, a.pv, z);
  const int slots = sq.rows * a.G, f0 = blockIdx.y * 32;
  if (f0 >= slots) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, half = lane >> 5;
  // causal: the last row of these slots bounds their keys
  const int last = min(sq.rows - 1, (f0 + 31) / a.G);
  const int nk = sq.cached + (a.anc ? sq.rows : last + 1);
  const int beg = sp * a.chunk, end = min(nk, beg + a.chunk);
  if (beg >= sq.cached + sq.rows) return;
  const int f = f0 + (lane & 31), row = f / a.G, head = h * a.G + f % a.G;
  const bool ok = f < slots;
  const int64_t t = sq.row0 + (ok ? row : 0);
  WaveState<HD> s;
  {
    const uint4* q = (const uint4*)(a.q + t * a.q_row + (ok ? head : 0) * HD + half * (HD / 2));
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) s.q[i] = __builtin_bit_cast(bf16x8, ok ? q[i] : make_uint4(0, 0, 0, 0));
  }
  const uint64_t mask = a.anc && ok ? a.anc[t] : 0;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) s.o[d][i] = 0.0f;
  s.m = -INFINITY;
  s.l = 0.0f;
  for (int p0 = beg + 32 * wave; p0 < end; p0 += 128) {
    const char* page = page_of(a.w, a.pv, z, p0);
    if (!page) continue;
    RawTile<HD, FP8> r;
    load_tile<HD, FP8>(r, a, page, h, p0);
    if (p0 + 32 <= sq.cached) attend_tile<HD, FP8, false>(s, r, a.scale, 0xFFFFu, 32);
    else attend_tile<HD, FP8, true>(s, r, a.scale, visible(sq, p0, row, ok, a.anc, mask), sq.cached + sq.rows - p0);
  }
  s.l += __shfl_xor(s.l, 32, kWave);
  // register i of block d holds dim 32 d + 8 (i / 4) + 4 half + i % 4
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
  const int sl = threadIdx.x >> 3, d0 = (threadIdx.x & 7) * DPT;
  const int g = f0 + sl;
  if (g >= slots) return;
  float mx = -INFINITY;
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm.m[w][sl]);
  float v[DPT] = {}, l = 0.0f;
  for (int w = 0; w < 4; ++w) {
    const float fw = mx == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(sm.m[w][sl] - mx);
    l += sm.l[w][sl] * fw;
#pragma unroll
    for (int i = 0; i < DPT; ++i) v[i] += sm.o[w][sl][d0 + i] * fw;
  }
  const int64_t tt = sq.row0 + g / a.G;
  const int hh = h * a.G + g % a.G;
  if (a.splits == 1) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // (no key at all: zeros)
    uint4* o = (uint4*)(a.out + tt * a.out_row + hh * HD + d0);
#pragma unroll
    for (int i = 0; i < DPT / 8; ++i)
      o[i] = make_uint4(pk_bf16(v[8 * i] * inv, v[8 * i + 1] * inv), pk_bf16(v[8 * i + 2] * inv, v[8 * i + 3] * inv),
                        pk_bf16(v[8 * i + 4] * inv, v[8 * i + 5] * inv), pk_bf16(v[8 * i + 6] * inv, v[8 * i + 7] * inv));
    return;
  }
  const int64_t at = ((int64_t)sp * a.w.T + tt) * a.H + hh;
#pragma unroll
  for (int i = 0; i < DPT; i += 4)
    *(float4*)(a.ws_o + at * HD + d0 + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  if ((threadIdx.x & 7) == 0) *(float2*)(a.ws_ml + at * 2) = make_float2(mx, l);
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
  const int64_t at = t * a.H + hh, step = (int64_t)a.w.T * a.H;
  float mx = -INFINITY;
  for (int k = lane; k < n; k += kWave) mx = fmaxf(mx, a.ws_ml[(at + k * step) * 2]);
  mx = wave_max(mx);
  float l = 0.0f, v[HD / 64] = {};
  for (int k = 0; k < n; ++k) {
    const int64_t j = at + k * step;
    const float2 ml = *(const float2*)(a.ws_ml + j * 2);
    const float f = mx == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml.x - mx);
    l += ml.y * f;
#pragma unroll
    for (int e = 0; e < HD / 64; ++e) v[e] += a.ws_o[j * HD + lane * (HD / 64) + e] * f;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t* o = a.out + t * a.out_row + hh * HD + lane * (HD / 64);
  if constexpr (HD == 128) *(uint32_t*)o = pk_bf16(v[0] * inv, v[1] * inv);
  else *o = (uint16_t)pk_bf16(v[0] * inv, 0.0f);
}

}  // namespace

// Keys per split: one split where sequences, heads and slots fill the compute
// units twice, else as many as do that, of 256 keys at least.
AttnPlan paged_attention_plan(const sjd_pages& p, const sjd_windows& w, int H) {
  const int64_t most = (int64_t)w.max_cached + w.max_rows;
  const int64_t slots = (int64_t)w.max_rows * (H / p.n_kv_heads);
  const int64_t wgs = (int64_t)w.B * p.n_kv_heads * ((slots + 31) / 32);
  int64_t S = wgs >= 512 ? 1 : (512 + wgs - 1) / wgs;
  const int64_t cap = (most + 255) / 256;
  if (S > cap) S = cap;
  if (S < 1) S = 1;
  const int64_t chunk = ((most + S - 1) / S + 127) / 128 * 128;
  return AttnPlan{(int)chunk, (int)((most + chunk - 1) / chunk)};
}

int64_t paged_attention_ws(const sjd_pages& p, const sjd_windows& w, int H) {
  const AttnPlan pl = paged_attention_plan(p, w, H);
  if (pl.splits <= 1) return 0;
  return (int64_t)pl.splits * w.T * H * (p.head_dim + 2) * 4;
}

hipError_t launch_paged_attention(const sjd_pages& p, const sjd_windows& w, const sjd_attention_io& io, void* ws,
                                  hipStream_t s) {
  const AttnPlan pl = paged_attention_plan(p, w, io.H);
  PagedArgs a{};
  a.pv = pool_view(p); a.w = w; a.q = (const uint16_t*)io.d_q; a.out = (uint16_t*)io.d_out;
  a.q_row = io.q_row; a.out_row = io.out_row; a.anc = io.d_anc; a.H = io.H; a.G = io.H / p.n_kv_heads;
  a.scale = (float)(1.4426950408889634 * (double)io.scale);
  a.chunk = pl.chunk; a.splits = pl.splits;
  a.ws_o = (float*)ws;
  a.ws_ml = ws ? (float*)ws + (int64_t)pl.splits * w.T * io.H * p.head_dim : nullptr;
  const dim3 grid(p.n_kv_heads * pl.splits, (w.max_rows * a.G + 31) / 32, w.B);
  const bool f8 = p.dtype == SJD_E4M3;
  if (p.head_dim == 128) {
    if (f8) hipLaunchKernelGGL((k_paged_attn<128, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_paged_attn<128, false>), grid, dim3(256), 0, s, a);
  } else {
    if (f8) hipLaunchKernelGGL((k_paged_attn<64, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_paged_attn<64, false>), grid, dim3(256), 0, s, a);
  }
  if (pl.splits > 1) {
    const dim3 jg((unsigned)(((int64_t)w.max_rows * io.H + 3) / 4), w.B);
    if (p.head_dim == 128) hipLaunchKernelGGL(k_paged_join<128>, jg, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(k_paged_join<64>, jg, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace sjd
