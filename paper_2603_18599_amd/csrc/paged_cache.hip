// A cache in pages: rows of keys and values quantised (e4m3 with a power of two
// per row and head) or rounded to bf16 as they are written, and read back.
//
// Both directions are bound by memory: a row of a head is hd input elements in
// and hd codes and an exponent out. A workgroup takes one tile, 32 positions of
// one head (whose part of a page is contiguous), 8 threads to a row. Keys go from
// a thread's registers to their place; values lie transposed, so they cross LDS
// in the tile's own order and move to and from memory in 16-byte pieces. 10432 rows of
// 32 heads of 128 written and 15363 read back (636 MB): 62 + 88 us, 4.2 TB/s; a copy
// runs at 4.9.
#include "paged_rows.h"

namespace sjd {

namespace {

struct CacheArgs {
  PoolView pv;
  sjd_windows w;
  sjd_kv_rows r;
};

template <int HD, bool FP8, bool F32>
__global__ __launch_bounds__(256) void k_kv_append(CacheArgs a) {
  constexpr int ES = FP8 ? 1 : 2, N = HD / 8;
  __shared__ __align__(16) char vs[32 * HD * ES * 17 / 16];
  const int z = blockIdx.z, h = blockIdx.y;
  const Seq sq = load_seq(a.w, a.pv, z);
  const int p0 = ((sq.cached >> 5) + (int)blockIdx.x) << 5;
  if (sq.rows == 0 || p0 >= sq.cached + sq.rows) return;
  char* page = page_of(a.w, a.pv, z, p0);
  if (!page) return;
  const int in = p0 & ((1 << a.pv.plen_log2) - 1);
  const int i = threadIdx.x >> 3, c = threadIdx.x & 7;
  const int r = p0 + i - sq.cached;
  const bool ok = (uint32_t)r < (uint32_t)sq.rows;
  const int lo = max(0, sq.cached - p0), hi = min(32, sq.cached + sq.rows - p0);  // positions that the window holds
  float kf[N] = {}, vf[N] = {};
  if (ok) {
    const int64_t t = sq.row0 + r;
    load_row<F32, N>(a.r.d_k, t * a.r.k_row + h * HD + c * N, kf);
    load_row<F32, N>(a.r.d_v, t * a.r.v_row + h * HD + c * N, vf);
  }
  store_tile<HD, FP8>(a.pv, page, h, in, lo, hi, ok, kf, vf, vs);
}

template <int HD, bool FP8, bool F32>
__global__ __launch_bounds__(256) void k_kv_read(CacheArgs a) {
  constexpr int ES = FP8 ? 1 : 2, N = HD / 8;
  __shared__ __align__(16) char vs[32 * HD * ES * 17 / 16];
  const int z = blockIdx.z, h = blockIdx.y;
  const Seq sq = load_seq(a.w, a.pv, z);
  const int p0 = ((sq.cached >> 5) + (int)blockIdx.x) << 5;
  if (sq.rows == 0 || p0 >= sq.cached + sq.rows) return;
  const char* page = page_of(a.w, a.pv, z, p0);
  const int in = p0 & ((1 << a.pv.plen_log2) - 1);
  const int i = threadIdx.x >> 3, c = threadIdx.x & 7;
  const int r = p0 + i - sq.cached;
  const bool ok = (uint32_t)r < (uint32_t)sq.rows;
  const int64_t t = sq.row0 + r;
  float kf[N] = {}, vf[N] = {};
  if (page) {
    const char* kt = page + tile_off<HD, ES>(a.pv, h, in, 0) + key_byte<HD, FP8>(i, c * N);
    const char* vt = page + tile_off<HD, ES>(a.pv, h, in, 1);
    for (int u = threadIdx.x; u < 2 * HD * ES; u += 256) *(uint4*)(vs + pad(16 * u)) = *(const uint4*)(vt + 16 * u);
    if constexpr (FP8) {
      const float ks = exp_scale((uint8_t)page[exp_off<HD>(a.pv, h, 0) + in + i]);
      const float vsc = exp_scale((uint8_t)page[exp_off<HD>(a.pv, h, 1) + in + i]);
#pragma unroll
      for (int g = 0; g < N / 8; ++g) {
        const uint2 x = *(const uint2*)(kt + 8 * g);
        decode4(x.x, ks, kf + 8 * g);
        decode4(x.y, ks, kf + 8 * g + 4);
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < N; e += 4) {
        uint32_t w = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) w |= (uint32_t)(uint8_t)vs[pad(val_byte<true>(i, c * N + e + b))] << (8 * b);
        decode4(w, vsc, vf + e);
      }
    } else {
#pragma unroll
      for (int g = 0; g < N / 8; ++g) {
        float x[8];
        load_row<false, 8>(kt + 1024 * g, 0, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) kf[8 * g + e] = x[e];
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < N; ++e) vf[e] = bf16_to_f32(*(const uint16_t*)(vs + pad(val_byte<false>(i, c * N + e))));
    }
  }
  if (!ok) return;
  store_row<F32, N>(a.r.d_k, t * a.r.k_row + h * HD + c * N, kf);
  store_row<F32, N>(a.r.d_v, t * a.r.v_row + h * HD + c * N, vf);
}

template <template <int, bool, bool> class K>
hipError_t launch(const sjd_pages& p, const sjd_windows& w, const sjd_kv_rows& r, hipStream_t s) {
  const CacheArgs a{pool_view(p), w, r};
  // tiles of a window: it may start and end inside one
  const dim3 grid((w.max_rows + 62) / 32, p.n_kv_heads, w.B);
  const bool f32 = r.dtype == SJD_F32;
  if (p.head_dim == 128) {
    if (p.dtype == SJD_E4M3) f32 ? K<128, true, true>::go(a, grid, s) : K<128, true, false>::go(a, grid, s);
    else f32 ? K<128, false, true>::go(a, grid, s) : K<128, false, false>::go(a, grid, s);
  } else {
    if (p.dtype == SJD_E4M3) f32 ? K<64, true, true>::go(a, grid, s) : K<64, true, false>::go(a, grid, s);
    else f32 ? K<64, false, true>::go(a, grid, s) : K<64, false, false>::go(a, grid, s);
  }
  return hipGetLastError();
}

template <int HD, bool FP8, bool F32>
struct Append {
  static void go(const CacheArgs& a, dim3 grid, hipStream_t s) {
    hipLaunchKernelGGL((k_kv_append<HD, FP8, F32>), grid, dim3(256), 0, s, a);
  }
};
template <int HD, bool FP8, bool F32>
struct Read {
  static void go(const CacheArgs& a, dim3 grid, hipStream_t s) {
    hipLaunchKernelGGL((k_kv_read<HD, FP8, F32>), grid, dim3(256), 0, s, a);
  }
};

}  // namespace

hipError_t launch_kv_append(const sjd_pages& p, const sjd_windows& w, const sjd_kv_rows& r, hipStream_t s) {
  return launch<Append>(p, w, r, s);
}
hipError_t launch_kv_read(const sjd_pages& p, const sjd_windows& w, const sjd_kv_rows& r, hipStream_t s) {
  return launch<Read>(p, w, r, s);
}

}  // namespace sjd
