// What a decoder context with e4m3 pages runs around the standalone operators: its
// window's sequences and places (these with a grid, too), rows from GEMM planes and
// back into activation tiles, and the move of an accepted sibling's cache row. All of
// it small beside the projections (a window is at most 128 rows).
#include "device.h"
#include "ops.h"

namespace sjd {

namespace {

__global__ __launch_bounds__(kWinRows) void k_page_window(PageWindow a) {
  const int m = threadIdx.x;
  const bool multi = a.sm.mode != kStreamsOne;
  const int nz = multi ? a.sm.nz : 1;
  if (m < nz) {
    const int n = a.st ? (multi ? stream_rows(a.sm, 0, m) : a.st->n) : a.start;
    ((int4*)a.seq)[m] = make_int4(32 * m, a.st ? a.L : a.M, n, 0);
  }
  if (m >= a.M) return;
  const int z = multi ? m >> 5 : 0;
  const bool row = !multi || (m & 31) < a.L;  // (else padding between two streams)
  const int pos = row ? a.win->pos[m] : 0;
  if (!a.grid) {
    a.pos[m] = pos;
    return;
  }
  int t = pos, y = pos, x = pos;
  if (a.st && row) {
    const DevState& d = a.st[multi ? stream_image(a.sm, z) : 0];
    // the prompt's length: cached rows less generated ones, and the pending token
    const int n_p = d.n - d.g0 + 1 + (multi && stream_uncond(a.sm, z) ? d.delta_u : 0);
    const int g = pos - n_p;
    if (g >= 0) {
      t = n_p;
      y = n_p + g / (a.row_len + 1);
      x = n_p + g % (a.row_len + 1);
    }
  }
  a.pos[3 * m] = t;
  a.pos[3 * m + 1] = y;
  a.pos[3 * m + 2] = x;
}

__global__ __launch_bounds__(256) void k_plane_rows(const float* part, int S, size_t plane, int N, uint16_t* rows) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= N) return;
  const size_t at = (size_t)blockIdx.y * N + c;
  float4 v = *(const float4*)(part + at);
  for (int s = 1; s < S; ++s) {
    const float4 u = *(const float4*)(part + s * plane + at);
    v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
  }
  *(uint2*)(rows + at) = make_uint2((uint32_t)f32_to_bf16(v.x) | ((uint32_t)f32_to_bf16(v.y) << 16),
                                    (uint32_t)f32_to_bf16(v.z) | ((uint32_t)f32_to_bf16(v.w) << 16));
}

__global__ __launch_bounds__(256) void k_row_tiles(const uint16_t* rows, int K, uint16_t* y, int mtiles) {
  const int k = (blockIdx.x * 256 + threadIdx.x) * 8, m = blockIdx.y;
  if (k >= K) return;
  uint16_t* d = y + act_off(m, k, mtiles);
  *(uint4*)d = *(const uint4*)(rows + (size_t)m * K + k);
  *(uint4*)(d + kActLo) = make_uint4(0, 0, 0, 0);
}

// grid (layer, key / value head, stream), one thread per dim
template <int HD>
__global__ __launch_bounds__(HD) void k_page_commit(const DevState* st, const Window* win, PoolView pv,
                                                    int64_t pool_bytes, const int32_t* table, int table_len, int K,
                                                    int guided) {
  const int z = blockIdx.z, h = blockIdx.y, j = threadIdx.x, b = guided ? z >> 1 : z;
  const DevState* s = st + b;
  const int acc_k = s->meta[5];
  if (acc_k < 2) return;
  const int n = win->n[b] + (guided && (z & 1) ? s->delta_u : 0), r = s->meta[1];
  const int src = n + win->n_s[b] + r * (K - 1) + (acc_k - 2), dst = n + r + 1;
  char* pool = pv.pool + blockIdx.x * pool_bytes;
  auto page = [&](int p) { return pool + table[z * table_len + (p >> pv.plen_log2)] * pv.page_bytes; };
  char *ps = page(src), *pd = page(dst);
  const int mask = (1 << pv.plen_log2) - 1, is = src & mask, id = dst & mask;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const int es = kv ? val_byte<true>(is & 31, j) : key_byte<HD, true>(is & 31, j);
    const int ed = kv ? val_byte<true>(id & 31, j) : key_byte<HD, true>(id & 31, j);
    pd[tile_off<HD, 1>(pv, h, id, kv) + ed] = ps[tile_off<HD, 1>(pv, h, is, kv) + es];
    if (j == 0) pd[exp_off<HD>(pv, h, kv) + id] = ps[exp_off<HD>(pv, h, kv) + is];
  }
}

}  // namespace

hipError_t launch_page_window(const PageWindow& a, hipStream_t s) {
  const bool multi = a.sm.mode != kStreamsOne;
  if (a.M < 1 || a.M > kWinRows || (multi && (a.sm.nz < 1 || a.sm.nz > kMaxStreams)) || (a.grid && a.st && a.row_len < 1))
    return hipErrorInvalidValue;
  hipLaunchKernelGGL(k_page_window, dim3(1), dim3(kWinRows), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_plane_rows(const float* part, int S, size_t plane, int M, int N, uint16_t* rows, hipStream_t s) {
  hipLaunchKernelGGL(k_plane_rows, dim3((N + 1023) / 1024, M), dim3(256), 0, s, part, S, plane, N, rows);
  return hipGetLastError();
}

hipError_t launch_row_tiles(const uint16_t* rows, int M, int K, uint16_t* y, int mtiles, hipStream_t s) {
  hipLaunchKernelGGL(k_row_tiles, dim3((K + 2047) / 2048, M), dim3(256), 0, s, rows, K, y, mtiles);
  return hipGetLastError();
}

hipError_t launch_page_commit(const DevState* st, const Window* win, const sjd_pages& p, int64_t pool_bytes, int layers,
                              const int32_t* table, int table_len, int K, int nstreams, bool guided, hipStream_t s) {
  if (p.dtype != SJD_E4M3) return hipErrorInvalidValue;
  const auto k = p.head_dim == 128 ? k_page_commit<128> : k_page_commit<64>;
  hipLaunchKernelGGL(k, dim3(layers, p.n_kv_heads, nstreams), dim3(p.head_dim), 0, s, st, win, pool_view(p), pool_bytes,
                     table, table_len, K, guided ? 1 : 0);
  return hipGetLastError();
}

}  // namespace sjd
