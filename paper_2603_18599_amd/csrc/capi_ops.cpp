// C ABI of the standalone operators: argument checks, before anything is
// enqueued.
#include <hip/hip_runtime.h>

#include <cmath>

#include "ops.h"
#include "sjd.h"

namespace {

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

int status(hipError_t e) { return e == hipSuccess ? SJD_OK : SJD_EHIP; }

int check_given(const sjd_given_params* p, const sjd_given_io* io) {
  if (!p || !io) return SJD_EINVAL;
  if (p->B < 1 || p->B > 65535 || p->L < 1 || p->L > 64 || p->V < 1 || p->V > (1 << 24)) return SJD_EINVAL;
  if (p->flags & ~(SJD_AC | SJD_BONUS)) return SJD_EINVAL;
  if (!io->d_p || !io->d_draft || !io->d_u || !io->d_r || !io->d_meta || !io->d_tok) return SJD_EINVAL;
  if ((p->flags & SJD_AC) && !io->d_next) return SJD_EINVAL;
  for (const void* b : {(const void*)io->d_p, (const void*)io->d_q, (const void*)io->d_draft, (const void*)io->d_n,
                        (const void*)io->d_u, (const void*)io->d_r, (const void*)io->d_tok, (const void*)io->d_next})
    if (!aligned(b, 4)) return SJD_EINVAL;
  if (!aligned(io->d_meta, 16)) return SJD_EINVAL;
  // (windows may overlap or share their rows: any stride between them but a negative one)
  if (p->p_row < p->V || p->p_win < 0 || (io->d_q && (p->q_row < p->V || p->q_win < 0))) return SJD_EINVAL;
  return SJD_OK;
}

int check_rope(const sjd_rope_params* p, const sjd_rope_io* io) {
  if (!p || !io) return SJD_EINVAL;
  if (p->T < 0 || p->T > (1 << 24) || p->H < 0 || p->Hkv < 0 || p->H > 1024 || p->Hkv > 1024 || p->H + p->Hkv < 1)
    return SJD_EINVAL;
  if (p->head_dim < 2 || p->head_dim > 256 || (p->head_dim & 1) || p->pairs < 1 || p->pairs > p->head_dim / 2)
    return SJD_EINVAL;
  if (p->axes < 1 || p->axes > 4 || (p->inverse != 0 && p->inverse != 1)) return SJD_EINVAL;
  if (p->dtype != SJD_F32 && p->dtype != SJD_BF16) return SJD_EINVAL;
  if (!p->h_freq || !p->h_axis) return SJD_EINVAL;
  for (int i = 0; i < p->pairs; ++i)
    if (p->h_axis[i] >= p->axes || !std::isfinite(p->h_freq[i])) return SJD_EINVAL;
  if (p->T == 0) return SJD_OK;
  const uintptr_t es = p->dtype == SJD_F32 ? 4 : 2;
  if (!io->d_pos || !aligned(io->d_pos, 4)) return SJD_EINVAL;
  const int64_t nq = (int64_t)p->H * p->head_dim, nk = (int64_t)p->Hkv * p->head_dim;
  if (p->H && (!io->d_q || !io->d_out_q || p->q_row < nq || p->out_q_row < nq || !aligned(io->d_q, es) ||
               !aligned(io->d_out_q, es) || (io->d_q == io->d_out_q && p->q_row != p->out_q_row)))
    return SJD_EINVAL;
  if (p->Hkv && (!io->d_k || !io->d_out_k || p->k_row < nk || p->out_k_row < nk || !aligned(io->d_k, es) ||
                 !aligned(io->d_out_k, es) || (io->d_k == io->d_out_k && p->k_row != p->out_k_row)))
    return SJD_EINVAL;
  return SJD_OK;
}

int check_page_shape(const sjd_pages* p) {
  if (!p || p->n_pages < 1 || p->n_kv_heads < 1 || p->n_kv_heads > 1024) return SJD_EINVAL;
  if (p->page_len < 32 || p->page_len > 1024 || (p->page_len & (p->page_len - 1))) return SJD_EINVAL;
  if (p->dtype != SJD_BF16 && p->dtype != SJD_E4M3) return SJD_EINVAL;
  if (p->head_dim != 64 && p->head_dim != 128) return SJD_ENOTSUP;
  return SJD_OK;
}

int check_pages(const sjd_pages* p) {
  const int st = check_page_shape(p);
  if (st != SJD_OK) return st;
  return p->d_pool && aligned(p->d_pool, 256) ? SJD_OK : SJD_EINVAL;
}

// (counts only; the device pointers are looked at where something is launched)
int check_windows_shape(const sjd_pages* p, const sjd_windows* w) {
  if (!w || w->B < 0 || w->B > 65535 || w->T < 0 || w->T > (1 << 24) || w->max_rows < 0 || w->max_rows > w->T ||
      w->max_cached < 0 || w->table_len < 0)
    return SJD_EINVAL;
  // positions are 32-bit numbers
  if ((int64_t)w->max_cached + w->max_rows > (1 << 30)) return SJD_EINVAL;
  return SJD_OK;
}
bool nothing(const sjd_windows* w) { return w->B == 0 || w->max_rows == 0; }

int check_windows(const sjd_pages* p, const sjd_windows* w) {
  const int st = check_windows_shape(p, w);
  if (st != SJD_OK || nothing(w)) return st;
  if (w->table_len < 1 || !w->d_seq || !w->d_table || !aligned(w->d_seq, 16) || !aligned(w->d_table, 4))
    return SJD_EINVAL;
  return SJD_OK;
}

int check_rows(const sjd_pages* p, const sjd_windows* w, const sjd_kv_rows* r) {
  if (!r || (r->dtype != SJD_F32 && r->dtype != SJD_BF16)) return SJD_EINVAL;
  if (nothing(w)) return SJD_OK;
  const int64_t n = (int64_t)p->n_kv_heads * p->head_dim;
  if (!r->d_k || !r->d_v || !aligned(r->d_k, 16) || !aligned(r->d_v, 16)) return SJD_EINVAL;
  if (r->k_row < n || r->v_row < n || (r->k_row & 7) || (r->v_row & 7)) return SJD_EINVAL;
  return SJD_OK;
}

#define TRY(e)                     \
  do {                             \
    const int _rc = (e);           \
    if (_rc != SJD_OK) return _rc; \
  } while (0)

int check_heads(const sjd_pages* p, const sjd_windows* w, int32_t H) {
  if (H < 1 || H > 1024 || H % p->n_kv_heads) return SJD_EINVAL;
  // query slots of a window: a launch has 65535 blocks of 128 of them
  return (int64_t)w->max_rows * (H / p->n_kv_heads) <= 65535LL * 128 ? SJD_OK : SJD_ENOTSUP;
}

}  // namespace

extern "C" int sjd_verify_given(const sjd_given_params* p, const sjd_given_io* io, void* stream) {
  TRY(check_given(p, io));
  return status(sjd::launch_verify_given(*p, *io, (hipStream_t)stream));
}

extern "C" int sjd_rope_axes(const sjd_rope_params* p, const sjd_rope_io* io, void* stream) {
  TRY(check_rope(p, io));
  if (p->T == 0) return SJD_OK;
  return status(sjd::launch_rope_axes(*p, *io, (hipStream_t)stream));
}

extern "C" int64_t sjd_page_bytes(const sjd_pages* p) {
  return check_page_shape(p) == SJD_OK ? sjd::page_bytes(*p) : 0;
}

extern "C" int sjd_kv_append(const sjd_pages* p, const sjd_windows* w, const sjd_kv_rows* r, void* stream) {
  TRY(check_pages(p));
  TRY(check_windows(p, w));
  TRY(check_rows(p, w, r));
  if (nothing(w)) return SJD_OK;
  return status(sjd::launch_kv_append(*p, *w, *r, (hipStream_t)stream));
}

extern "C" int sjd_kv_read(const sjd_pages* p, const sjd_windows* w, const sjd_kv_rows* r, void* stream) {
  TRY(check_pages(p));
  TRY(check_windows(p, w));
  TRY(check_rows(p, w, r));
  if (nothing(w)) return SJD_OK;
  return status(sjd::launch_kv_read(*p, *w, *r, (hipStream_t)stream));
}

extern "C" int64_t sjd_paged_attention_workspace(const sjd_pages* p, const sjd_windows* w, int32_t H) {
  if (check_page_shape(p) != SJD_OK || check_windows_shape(p, w) != SJD_OK || check_heads(p, w, H) != SJD_OK) return 0;
  return nothing(w) ? 0 : sjd::paged_attention_ws(*p, *w, H);
}

extern "C" int sjd_paged_attention(const sjd_pages* p, const sjd_windows* w, const sjd_attention_io* io, void* d_ws,
                                   int64_t ws_bytes, void* stream) {
  TRY(check_pages(p));
  TRY(check_windows(p, w));
  if (!io || !std::isfinite(sjd::log2_scale(io->scale))) return SJD_EINVAL;
  TRY(check_heads(p, w, io->H));
  if (nothing(w)) return SJD_OK;
  const int64_t n = (int64_t)io->H * p->head_dim;
  if (!io->d_q || !io->d_out || !aligned(io->d_q, 16) || !aligned(io->d_out, 16) || io->q_row < n || io->out_row < n ||
      (io->q_row & 7) || (io->out_row & 7))
    return SJD_EINVAL;
  if (io->d_anc && (w->max_rows > 64 || !aligned(io->d_anc, 8))) return SJD_EINVAL;
  const int64_t need = sjd::paged_attention_ws(*p, *w, io->H);
  if (need && (!d_ws || ws_bytes < need || !aligned(d_ws, 256))) return SJD_EINVAL;
  return status(sjd::launch_paged_attention(*p, *w, *io, d_ws, (hipStream_t)stream));
}
