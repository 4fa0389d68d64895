// Internal interface of the standalone operators (not part of the C ABI):
// rotary axes, caches in pages, their attention, given verification.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "forward.h"
#include "sjd.h"

namespace sjd {

// ---- pages (layout: sjd.h). page_len is a power of two of at least a tile.
constexpr int kTile = 32;          // positions per tile, the attention's MFMA key rows
constexpr int kMinExp = 27, kMaxExp = 246;  // exponent bytes that the quantiser writes

struct PoolView {
  char* pool;
  int n_pages, Hkv;
  int plen_log2;
  int64_t page_bytes;
};

inline int64_t page_data_bytes(const sjd_pages& p) {
  return 2LL * p.n_kv_heads * p.page_len * p.head_dim * (p.dtype == SJD_E4M3 ? 1 : 2);
}
inline int64_t page_bytes(const sjd_pages& p) {
  const int64_t b = page_data_bytes(p) + (p.dtype == SJD_E4M3 ? 2LL * p.n_kv_heads * p.page_len : 0);
  return (b + 255) / 256 * 256;
}
inline PoolView pool_view(const sjd_pages& p) {
  int lg = 0;
  while ((1 << lg) < p.page_len) ++lg;
  return PoolView{(char*)p.d_pool, p.n_pages, p.n_kv_heads, lg, page_bytes(p)};
}

#ifdef __HIPCC__
// A sequence of a call, or rows = 0 where its numbers break the call's bounds
// (sjd.h: it is left out).
struct Seq {
  int row0, rows, cached;
};
__device__ __forceinline__ Seq load_seq(const sjd_windows& w, const PoolView& pv, int z) {
  const int4 v = ((const int4*)w.d_seq)[z];
  Seq s{v.x, v.y, v.z};
  // (unsigned: negative numbers are large)
  const bool ok = (uint32_t)s.rows <= (uint32_t)w.max_rows && (uint32_t)s.cached <= (uint32_t)w.max_cached && s.row0 >= 0 &&
                  s.row0 <= w.T - s.rows && (int64_t)s.cached + s.rows <= ((int64_t)w.table_len << pv.plen_log2);
  if (!ok) s.rows = 0;
  return s;
}
// Page id of position p of sequence z (scalar load: the table does not change
// during a call, and every caller asks for one position per wave), and the start of
// a page, NULL for an id outside the pool
__device__ __forceinline__ int page_id(const sjd_windows& w, const PoolView& pv, int z, int p) {
  const auto* t = (const int32_t __attribute__((address_space(4)))*)w.d_table;
  return __builtin_amdgcn_readfirstlane(t[(int64_t)z * w.table_len + (p >> pv.plen_log2)]);
}
__device__ __forceinline__ char* page_at(const PoolView& pv, int id) {
  return (uint32_t)id < (uint32_t)pv.n_pages ? pv.pool + (int64_t)id * pv.page_bytes : nullptr;
}
__device__ __forceinline__ char* page_of(const sjd_windows& w, const PoolView& pv, int z, int p) {
  return page_at(pv, page_id(w, pv, z, p));
}
// Byte offsets inside a page, head h: the tile of position `in` (of the page), and
// the exponent bytes of the page's positions 0 ..
template <int HD, int ES>
__device__ __forceinline__ int64_t tile_off(const PoolView& pv, int h, int in, int kv) {
  return (((int64_t)(2 * h + kv) << pv.plen_log2) + (in & ~(kTile - 1))) * (HD * ES);
}
template <int HD>
__device__ __forceinline__ int64_t exp_off(const PoolView& pv, int h, int kv) {
  return ((int64_t)2 * pv.Hkv * HD + 2 * h + kv) << pv.plen_log2;
}
// Byte of position i (of 32) and dim j inside a key tile and inside a value tile: the
// layout of sjd.h, which the attention reads as its matrix operands without these
template <int HD, bool FP8>
__device__ __forceinline__ int key_byte(uint32_t i, uint32_t j) {
  const uint32_t lane = swap23(i) + 32 * (j / (HD / 2)), t = j % (HD / 2) / 8;
  return FP8 ? (64 * (t / 2) + lane) * 16 + 8 * (t % 2) + j % 8 : (64 * t + lane) * 16 + 2 * (j % 8);
}
template <bool FP8>
__device__ __forceinline__ int val_byte(uint32_t i, uint32_t j) {
  const uint32_t lane = j % 32 + 32 * (i / 8 % 2);
  return FP8 ? (64 * (j / 32) + lane) * 16 + 8 * (i / 16) + i % 8
             : ((j / 32 * 2 + i / 16) * 64 + lane) * 16 + 2 * (i % 8);
}
#endif

hipError_t launch_kv_append(const sjd_pages& p, const sjd_windows& w, const sjd_kv_rows& r, hipStream_t s);
hipError_t launch_kv_read(const sjd_pages& p, const sjd_windows& w, const sjd_kv_rows& r, hipStream_t s);

// ---- attention over pages
// Scores are formed in the log2 domain: |scale| * log2(e)
inline float log2_scale(float scale) { return (float)(1.4426950408889634 * std::fabs((double)scale)); }
struct AttnPlan {
  int chunk;   // keys per split, a multiple of the workgroup's keys per round
  int splits;  // most splits of a sequence
  bool few;    // few slots per window: waves split the keys, not the slots
};
AttnPlan paged_attention_plan(const sjd_pages& p, const sjd_windows& w, int H);
int64_t paged_attention_ws(const sjd_pages& p, const sjd_windows& w, int H);
hipError_t launch_paged_attention(const sjd_pages& p, const sjd_windows& w, const sjd_attention_io& io, void* ws,
                                  hipStream_t s);

// ---- decoder contexts with e4m3 pages or a grid (paged_step.hip)
// A window's sequences (of pages) and places: seq[z] = { row0, rows, cached, 0 } of stream z,
// pos[m] = the row's position, or with grid { time, row, column } of it: a text
// token's position three times; image token g (the first one at position n_p): n_p,
// n_p + g / (row_len + 1), n_p + g % (row_len + 1).
struct PageWindow {
  const Window* win;
  const DevState* st;  // NULL: rows of a prompt from position `start` on, all of them text
  int start, M, L, grid, row_len;
  Streams sm;
  int32_t* seq;
  int32_t* pos;
};
hipError_t launch_page_window(const PageWindow& a, hipStream_t s);
// rows[m][0 .. N) = bf16 of the sum of S fp32 partial planes (N a multiple of 4)
hipError_t launch_plane_rows(const float* part, int S, size_t plane, int M, int N, uint16_t* rows, hipStream_t s);
// bf16 rows [M][K] into activation tiles (K a multiple of 64; the lo planes are zero)
hipError_t launch_row_tiles(const uint16_t* rows, int M, int K, uint16_t* y, int mtiles, hipStream_t s);
// An accepted sibling's key and value move to their place in the sequence, in every
// layer's pool (launch_step_end's move, for pages). pool_bytes: from layer to layer.
hipError_t launch_page_commit(const DevState* st, const Window* win, const sjd_pages& p, int64_t pool_bytes, int layers,
                              const int32_t* table, int table_len, int K, int nstreams, bool guided, hipStream_t s);

hipError_t launch_rope_axes(const sjd_rope_params& p, const sjd_rope_io& io, hipStream_t s);
hipError_t launch_verify_given(const sjd_given_params& p, const sjd_given_io& io, hipStream_t s);

}  // namespace sjd
