"""MI355X (gfx950) speculative-Jacobi step library for SJD-PAC.

The compute path lives in libsjd.so (hand-written HIP); this package only
marshals arguments to its C ABI (include/sjd.h). Importing it does not need a
GPU, but every call that reaches the library needs the built libsjd.so and
fails loudly without it.
"""
from .sjd import (SJD_AC, SJD_BONUS, SJD_KV_E4M3, SJD_PD, SJD_ROPE_GRID, SJD_W8A8, Engine, I8Weights, Pages, SjdError,  # noqa: F401
                  Windows, attention_workspace, code_columns, lib_path, load_library, matmul_workspace, page_bytes, sjd_kv_append,
                  sjd_kv_append_rope, sjd_kv_read, sjd_matmul_i8, sjd_pack_i8, sjd_paged_attention, sjd_quantise_rows,
                  sjd_rope_axes, sjd_status_str, sjd_verify, sjd_verify_given)
