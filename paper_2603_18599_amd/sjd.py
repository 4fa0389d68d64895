"""ctypes binding of libsjd.so (include/sjd.h): argument marshalling only.

Device buffers are torch tensors on the current HIP device; their data
pointers and the current torch stream are handed to the C entry points.
Every step of the computation runs in the library's HIP kernels; there is no
fallback path.
"""
import ctypes as C
import os
from array import array

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libsjd.so"

SJD_AC = 1
SJD_PD = 2
SJD_EAGER = 4
SJD_NO_TUNE = 8
SJD_TUNE = 16
SJD_CHECK_FINITE = 32
SJD_FULL_SELECT = 64
SJD_KV_E4M3 = 128
SJD_ROPE_GRID = 256
SJD_BONUS = 512
SJD_VERIFY_NOALLOC_MAX_ROWS = 131072

_STATUS = {0: "SJD_OK", -1: "SJD_EINVAL", -2: "SJD_ENOMEM", -3: "SJD_EHIP", -4: "SJD_ESTATE", -5: "SJD_ENOTSUP",
           -6: "SJD_ENONFINITE"}


class SjdError(RuntimeError):
    def __init__(self, fn, code):
        super().__init__(f"{fn} failed: {_STATUS.get(code, code)}")
        self.code = code


class VerifyParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("L", C.c_int32), ("V", C.c_int32), ("K", C.c_int32), ("D", C.c_int32),
                ("top_k", C.c_int32), ("temperature", C.c_float), ("flags", C.c_uint32), ("seed", C.c_uint64),
                ("step", C.c_uint32), ("vis_lo", C.c_int32), ("eol_id", C.c_int32), ("row_len", C.c_int32)]


class VerifyIO(C.Structure):
    _fields_ = [("d_cur", C.c_void_p), ("d_draft", C.c_void_p), ("d_draft_tok", C.c_void_p),
                ("d_sib", C.c_void_p), ("d_in_meta", C.c_void_p), ("d_out_meta", C.c_void_p),
                ("d_out_tok", C.c_void_p), ("d_out_next", C.c_void_p), ("d_out_sib", C.c_void_p),
                ("d_out_rows", C.c_void_p), ("d_dbg_p", C.c_void_p)]


class Config(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn_dim", C.c_int32),
                ("vocab_size", C.c_int32), ("vis_lo", C.c_int32), ("V", C.c_int32), ("max_seq", C.c_int32),
                ("L", C.c_int32), ("K", C.c_int32), ("D", C.c_int32), ("flags", C.c_uint32),
                ("rms_eps", C.c_float), ("rope_theta", C.c_float), ("eol_id", C.c_int32),
                ("row_len", C.c_int32), ("weights_f32", C.c_int32), ("cfg_w", C.c_float),
                ("batch", C.c_int32)]


class Weights(C.Structure):
    _fields_ = [("d_embed", C.c_void_p), ("h_layer", C.c_void_p), ("d_final_norm", C.c_void_p),
                ("d_lm_head", C.c_void_p)]


class GivenParams(C.Structure):
    _fields_ = [("B", C.c_int32), ("L", C.c_int32), ("V", C.c_int32), ("flags", C.c_uint32), ("vis_lo", C.c_int32),
                ("p_row", C.c_int64), ("p_win", C.c_int64), ("q_row", C.c_int64), ("q_win", C.c_int64)]


class GivenIO(C.Structure):
    _fields_ = [("d_p", C.c_void_p), ("d_q", C.c_void_p), ("d_draft", C.c_void_p), ("d_n", C.c_void_p),
                ("d_u", C.c_void_p), ("d_r", C.c_void_p), ("d_meta", C.c_void_p), ("d_tok", C.c_void_p),
                ("d_next", C.c_void_p)]


class RopeParams(C.Structure):
    _fields_ = [("T", C.c_int32), ("H", C.c_int32), ("Hkv", C.c_int32), ("head_dim", C.c_int32),
                ("pairs", C.c_int32), ("axes", C.c_int32), ("dtype", C.c_int32), ("inverse", C.c_int32),
                ("q_row", C.c_int64), ("k_row", C.c_int64), ("out_q_row", C.c_int64), ("out_k_row", C.c_int64),
                ("h_freq", C.c_void_p), ("h_axis", C.c_char_p)]


class RopeIO(C.Structure):
    _fields_ = [("d_q", C.c_void_p), ("d_k", C.c_void_p), ("d_pos", C.c_void_p), ("d_out_q", C.c_void_p),
                ("d_out_k", C.c_void_p)]


class PagesDesc(C.Structure):
    _fields_ = [("d_pool", C.c_void_p), ("n_pages", C.c_int32), ("page_len", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class WindowsDesc(C.Structure):
    _fields_ = [("B", C.c_int32), ("T", C.c_int32), ("max_rows", C.c_int32), ("max_cached", C.c_int32),
                ("table_len", C.c_int32), ("d_seq", C.c_void_p), ("d_table", C.c_void_p)]


class KvRows(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("k_row", C.c_int64), ("v_row", C.c_int64),
                ("dtype", C.c_int32)]


class AttentionIO(C.Structure):
    _fields_ = [("H", C.c_int32), ("scale", C.c_float), ("d_q", C.c_void_p), ("d_out", C.c_void_p),
                ("q_row", C.c_int64), ("out_row", C.c_int64), ("d_anc", C.c_void_p)]


EXPORTS = ["sjd_status_str", "sjd_verify", "sjd_verify_noalloc", "sjd_init", "sjd_prefill", "sjd_prefill_image",
           "sjd_prefill_cfg", "sjd_prefill_image_cfg", "sjd_set_drafts", "sjd_step", "sjd_forward_window",
           "sjd_get_plan", "sjd_destroy", "sjd_verify_given", "sjd_rope_axes", "sjd_page_bytes", "sjd_kv_append",
           "sjd_kv_read", "sjd_paged_attention_workspace", "sjd_paged_attention"]

_lib = None


def lib_path():
    """The in-tree library, or the one SJD_LIBRARY names (another build of
    the same sources, e.g. to compare two builds in one process tree)."""
    return os.environ.get("SJD_LIBRARY") or os.path.join(HERE, _LIB_NAME)


def load_library():
    """Loads libsjd.so (built in-tree by __graft_entry__.build()); raises if
    it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build the HIP library first (python -c "
                           "'import __graft_entry__ as g; g.build()')")
    lib = C.CDLL(path)
    lib.sjd_status_str.restype = C.c_char_p
    lib.sjd_status_str.argtypes = [C.c_int]
    lib.sjd_verify.restype = C.c_int
    lib.sjd_verify.argtypes = [C.POINTER(VerifyParams), C.POINTER(VerifyIO), C.c_void_p]
    lib.sjd_verify_noalloc.restype = C.c_int
    lib.sjd_verify_noalloc.argtypes = [C.POINTER(VerifyParams), C.POINTER(VerifyIO), C.c_void_p]
    lib.sjd_init.restype = C.c_int
    lib.sjd_init.argtypes = [C.POINTER(Config), C.POINTER(Weights), C.c_void_p, C.POINTER(C.c_void_p)]
    lib.sjd_prefill.restype = C.c_int
    lib.sjd_prefill.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_uint64, C.c_void_p]
    lib.sjd_get_plan.restype = C.c_int
    lib.sjd_get_plan.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.c_int32]
    lib.sjd_prefill_image.restype = C.c_int
    lib.sjd_prefill_image.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_uint64, C.c_void_p]
    lib.sjd_prefill_cfg.restype = C.c_int
    lib.sjd_prefill_cfg.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_uint64,
                                    C.c_void_p]
    lib.sjd_prefill_image_cfg.restype = C.c_int
    lib.sjd_prefill_image_cfg.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32,
                                          C.c_uint64, C.c_void_p]
    lib.sjd_step.restype = C.c_int
    lib.sjd_step.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_int32,
                             C.c_uint64, C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.sjd_set_drafts.restype = C.c_int
    lib.sjd_set_drafts.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.sjd_forward_window.restype = C.c_int
    lib.sjd_forward_window.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
    lib.sjd_destroy.restype = None
    lib.sjd_destroy.argtypes = [C.c_void_p]
    lib.sjd_verify_given.restype = C.c_int
    lib.sjd_verify_given.argtypes = [C.POINTER(GivenParams), C.POINTER(GivenIO), C.c_void_p]
    lib.sjd_rope_axes.restype = C.c_int
    lib.sjd_rope_axes.argtypes = [C.POINTER(RopeParams), C.POINTER(RopeIO), C.c_void_p]
    lib.sjd_page_bytes.restype = C.c_int64
    lib.sjd_page_bytes.argtypes = [C.POINTER(PagesDesc)]
    for name in ("sjd_kv_append", "sjd_kv_read"):
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = [C.POINTER(PagesDesc), C.POINTER(WindowsDesc), C.POINTER(KvRows), C.c_void_p]
    lib.sjd_paged_attention_workspace.restype = C.c_int64
    lib.sjd_paged_attention_workspace.argtypes = [C.POINTER(PagesDesc), C.POINTER(WindowsDesc), C.c_int32]
    lib.sjd_paged_attention.restype = C.c_int
    lib.sjd_paged_attention.argtypes = [C.POINTER(PagesDesc), C.POINTER(WindowsDesc), C.POINTER(AttentionIO),
                                        C.c_void_p, C.c_int64, C.c_void_p]
    _lib = lib
    return lib


def sjd_status_str(code):
    return load_library().sjd_status_str(code).decode()


def _ptr(t):
    if t is None:
        return None
    return t.data_ptr()


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _check(fn, rc):
    if rc != 0:
        raise SjdError(fn, rc)


def sjd_verify(cur, draft, draft_tok, in_meta, out, *, K, D, top_k, temperature=1.0, flags=SJD_AC | SJD_PD,
               seed=0, step=0, sib=None, vis_lo=0, eol_id=-1, row_len=0, out_rows=None, dbg_p=None, stream=None,
               noalloc=False):
    """Standalone verification (sjd_verify in include/sjd.h; noalloc:
    sjd_verify_noalloc). cur/draft: float32 [B,L,V] device tensors; draft_tok
    int32 [B,L]; in_meta int32 [B,4]; out: dict of int32 device tensors meta
    [B,8], tok [B,L], next [B,L], sib [B,D,K-1]."""
    B, L, V = cur.shape
    p = VerifyParams(B, L, V, K, D, top_k, temperature, flags, seed, step, vis_lo, eol_id, row_len)
    io = VerifyIO(_ptr(cur), _ptr(draft), _ptr(draft_tok), _ptr(sib), _ptr(in_meta), _ptr(out["meta"]),
                  _ptr(out["tok"]), _ptr(out["next"]), _ptr(out["sib"]), _ptr(out_rows), _ptr(dbg_p))
    lib = load_library()
    fn = "sjd_verify_noalloc" if noalloc else "sjd_verify"
    _check(fn, getattr(lib, fn)(C.byref(p), C.byref(io), _stream(stream)))


def verify_outputs(B, L, K, D, device="cuda"):
    import torch
    return {"meta": torch.zeros(B, 8, dtype=torch.int32, device=device),
            "tok": torch.zeros(B, L, dtype=torch.int32, device=device),
            "next": torch.zeros(B, L, dtype=torch.int32, device=device),
            "sib": torch.zeros(B, max(D, 0), max(K - 1, 0), dtype=torch.int32, device=device)}


# ---- the standalone operators. A call costs some microseconds on the GPU, so the
# checks here are kept to comparisons of what a tensor already holds.
_DTYPES = {"float32": 0, "bfloat16": 1, "fp32": 0, "bf16": 1, "e4m3": 2}


def _types():
    """torch and {torch type: sjd_dtype}, once torch is needed."""
    global _types
    import torch
    t = (torch, {torch.float32: 0, torch.bfloat16: 1})
    _types = lambda: t  # noqa: E731
    return t


def _expect(fn, ok):
    """The library reads device memory by the sizes that it is told: a tensor of
    another type, shape, layout or device is refused like any other bad
    argument."""
    if not ok:
        raise SjdError(fn, -1)


def _launch(fn, stream, device, *args):
    """The call on `stream`, or the device's current one. Its tensors lie on
    `device`, which must be the current GPU (the library launches there)."""
    torch = _types()[0]
    _expect(fn, device >= 0 and device == torch.cuda.current_device())
    raw = stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(device)
    rc = getattr(_lib or load_library(), fn)(*args, raw)
    if rc != 0:
        raise SjdError(fn, rc)


def _row_stride(fn, t, T, heads, hd):
    """Row stride of [T, heads, hd] rows whose heads lie one behind the other."""
    if t.shape != (T, heads, hd):
        raise SjdError(fn, -1)
    if t.is_contiguous():  # (a single row whatever its stride, which separates nothing)
        return heads * hd
    s = t.stride()
    _expect(fn, T > 1 and s[2] == 1 and (heads == 1 or s[1] == hd))
    return s[0]


def _dense(fn, t, shape, dtype, device):
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous() or t.get_device() != device:
        raise SjdError(fn, -1)
    return t.data_ptr()


def sjd_verify_given(p, q, draft, n, u, r, meta, tok, next=None, *, flags=0, vis_lo=0, stream=None):
    """Verification against given probabilities with given uniforms
    (sjd_verify_given in include/sjd.h). p: float32 [B, L (SJD_BONUS: L + 1),
    V], q: float32 [B, L, V] or None (certain drafts), entries one behind the
    other; draft int32 [B, L]; n int32 [B] or None; u float32 [B, L]; r
    float32 [B, L + 1]; outputs int32 meta [B, 4], tok [B, L + 1], next [B, L]
    (None without SJD_AC)."""
    fn = "sjd_verify_given"
    torch = _types()[0]
    i32, f32 = torch.int32, torch.float32
    _expect(fn, draft.dim() == 2 and p.dim() == 3)
    (B, L), V, dev = draft.shape, p.shape[2], p.get_device()

    def rows(t, count):
        _expect(fn, t.shape == (B, count, V) and t.dtype is f32 and t.get_device() == dev)
        s = t.stride()
        _expect(fn, V == 1 or s[2] == 1)
        # (a stride that separates nothing may be anything)
        return t.data_ptr(), max(s[1], V) if count <= 1 else s[1], s[0]

    pp, p_row, p_win = rows(p, L + 1 if flags & SJD_BONUS else L)
    qp, q_row, q_win = (None, 0, 0) if q is None else rows(q, L)
    io = GivenIO(pp, qp, _dense(fn, draft, (B, L), i32, dev), None if n is None else _dense(fn, n, (B,), i32, dev),
                 _dense(fn, u, (B, L), f32, dev), _dense(fn, r, (B, L + 1), f32, dev),
                 _dense(fn, meta, (B, 4), i32, dev), _dense(fn, tok, (B, L + 1), i32, dev),
                 None if next is None else _dense(fn, next, (B, L), i32, dev))
    par = GivenParams(B, L, V, flags, vis_lo, p_row, p_win, q_row, q_win)
    _launch(fn, stream, dev, C.byref(par), C.byref(io))


def sjd_rope_axes(q, k, pos, freq, axis, *, out_q=None, out_k=None, inverse=False, stream=None):
    """Rotary positions with several axes (sjd_rope_axes in include/sjd.h) on
    rows q [T, H, hd] and k [T, Hkv, hd] (either may be None; bfloat16 or
    float32), in place unless out_q / out_k are given. pos int32 [T, axes]; freq
    and axis: one frequency and one axis for each pair of dims."""
    fn = "sjd_rope_axes"
    torch, types = _types()
    x = q if q is not None else k
    _expect(fn, x is not None and x.dim() == 3 and pos.dim() == 2 and len(axis) == len(freq))
    (T, _, hd), dt, dev, axes = x.shape, x.dtype, x.get_device(), pos.shape[1]
    f, ax = array("d", freq), bytes(axis)

    def rows(t, out):  # heads, strides and addresses of a tensor and of what it becomes
        if t is None:
            return 0, 0, 0, None, None
        if t.dim() != 3 or t.dtype is not dt or t.get_device() != dev:
            raise SjdError(fn, -1)
        H, at = t.shape[1], t.data_ptr()
        row = _row_stride(fn, t, T, H, hd)
        if out is None or out is t:
            return H, row, row, at, at
        if out.dtype is not dt or out.get_device() != dev:
            raise SjdError(fn, -1)
        return H, row, _row_stride(fn, out, T, H, hd), at, out.data_ptr()

    H, q_row, out_q_row, qp, out_qp = rows(q, out_q)
    Hkv, k_row, out_k_row, kp, out_kp = rows(k, out_k)
    par = RopeParams(T, H, Hkv, hd, len(f), axes, types.get(dt, -1), 1 if inverse else 0, q_row, k_row, out_q_row,
                     out_k_row, f.buffer_info()[0], ax)
    io = RopeIO(qp, kp, _dense(fn, pos, (T, axes), torch.int32, dev), out_qp, out_kp)
    _launch(fn, stream, dev, C.byref(par), C.byref(io))


def page_bytes(page_len, n_kv_heads, head_dim, dtype):
    """Bytes of a page (dtype "bf16" or "e4m3"); 0 for sizes that no page has."""
    d = PagesDesc(None, 1, page_len, n_kv_heads, head_dim, _DTYPES.get(dtype, -1))
    return load_library().sjd_page_bytes(C.byref(d))


class Pages:
    """A pool of pages (sjd_pages) in the caller's uint8 tensor."""

    def __init__(self, pool, n_pages, page_len, n_kv_heads, head_dim, dtype):
        size = page_bytes(page_len, n_kv_heads, head_dim, dtype)
        _expect("sjd_pages", size > 0 and n_pages >= 1 and pool.dtype is _types()[0].uint8 and pool.is_contiguous() and
                pool.numel() >= n_pages * size)
        self.pool, self.n_kv_heads, self.head_dim, self.device = pool, n_kv_heads, head_dim, pool.get_device()
        self.desc = PagesDesc(pool.data_ptr(), n_pages, page_len, n_kv_heads, head_dim, _DTYPES[dtype])


class Windows:
    """Windows of new rows (sjd_windows): seq int32 [B, 4] = (row0, rows, cached,
    0), table int32 [B, pages], over row tensors of T rows."""

    def __init__(self, seq, table, T, max_rows, max_cached):
        fn, i32, self.device = "sjd_windows", _types()[0].int32, seq.get_device()
        _expect(fn, seq.dim() == 2 and table.dim() == 2)
        B, cols = seq.shape[0], table.shape[1]
        self.seq, self.table, self.T = seq, table, T
        self.desc = WindowsDesc(B, T, max_rows, max_cached, cols, _dense(fn, seq, (B, 4), i32, self.device),
                                _dense(fn, table, (B, cols), i32, self.device))


def _kv_call(fn, pages, win, k, v, stream):
    T, H, hd, dev = win.T, pages.n_kv_heads, pages.head_dim, pages.device
    _expect(fn, k.dtype is v.dtype and win.device == dev and k.get_device() == dev and v.get_device() == dev)
    rows = KvRows(k.data_ptr(), v.data_ptr(), _row_stride(fn, k, T, H, hd), _row_stride(fn, v, T, H, hd),
                  _types()[1].get(k.dtype, -1))
    _launch(fn, stream, dev, C.byref(pages.desc), C.byref(win.desc), C.byref(rows))


def sjd_kv_append(pages, win, k, v, stream=None):
    """Writes rows k, v [T, Hkv, hd] (bfloat16 or float32) into the windows'
    pages (sjd_kv_append in include/sjd.h)."""
    _kv_call("sjd_kv_append", pages, win, k, v, stream)


def sjd_kv_read(pages, win, k, v, stream=None):
    """Reads the windows' positions back into rows k, v [T, Hkv, hd]
    (sjd_kv_read in include/sjd.h)."""
    _kv_call("sjd_kv_read", pages, win, k, v, stream)


def attention_workspace(pages, win, H):
    """Scratch for sjd_paged_attention with these pages and windows (calls that
    overlap in time need one each)."""
    n = load_library().sjd_paged_attention_workspace(C.byref(pages.desc), C.byref(win.desc), H)
    return _types()[0].empty(n, dtype=_types()[0].uint8, device=pages.pool.device)


def sjd_paged_attention(pages, win, q, out, ws, *, scale, anc=None, stream=None):
    """Attention of rows q [T, H, hd] over the windows' pages into out
    (sjd_paged_attention in include/sjd.h); bfloat16. ws: attention_workspace;
    anc: int64 [T] ancestor masks of tree windows, or None (causal)."""
    fn = "sjd_paged_attention"
    torch = _types()[0]
    dev, hd, T = pages.device, pages.head_dim, win.T
    _expect(fn, q.dim() == 3 and q.dtype is torch.bfloat16 and out.dtype is torch.bfloat16 and win.device == dev and
            q.get_device() == dev and out.get_device() == dev)
    H, size = q.shape[1], ws.numel()
    _expect(fn, ws.dtype is torch.uint8 and ws.is_contiguous() and (size == 0 or ws.get_device() == dev))
    io = AttentionIO(H, scale, q.data_ptr(), out.data_ptr(), _row_stride(fn, q, T, H, hd), _row_stride(fn, out, T, H, hd),
                     None if anc is None else _dense(fn, anc, (T,), torch.int64, dev))
    _launch(fn, stream, dev, C.byref(pages.desc), C.byref(win.desc), C.byref(io), ws.data_ptr(), size)


class Engine:
    """A decoder context (sjd_init .. sjd_destroy)."""

    def __init__(self, cfg: dict, weights: dict, stream=None):
        lib = load_library()
        self.cfg = cfg
        c = Config(cfg["n_layers"], cfg["d_model"], cfg["n_heads"], cfg["n_kv_heads"], cfg["head_dim"],
                   cfg["ffn_dim"], cfg["vocab_size"], cfg["vis_lo"], cfg["V"], cfg["max_seq"], cfg["L"], cfg["K"],
                   cfg["D"], cfg.get("flags", SJD_AC | SJD_PD), cfg.get("rms_eps", 1e-5),
                   cfg.get("rope_theta", 1e4), cfg.get("eol_id", -1), cfg.get("row_len", 0),
                   1 if cfg.get("weights_f32", False) else 0, cfg.get("cfg_w", 0.0), cfg.get("batch", 1))
        names = ["attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "wg", "wu", "wd"]
        self._layer_ptrs = (C.c_void_p * (9 * cfg["n_layers"]))()
        for l in range(cfg["n_layers"]):
            for i, nm in enumerate(names):
                self._layer_ptrs[9 * l + i] = weights["layers"][l][nm].data_ptr()
        self._weights = weights  # keep alive
        w = Weights(weights["embed"].data_ptr(), C.cast(self._layer_ptrs, C.c_void_p).value,
                    weights["final_norm"].data_ptr(), weights["lm_head"].data_ptr())
        h = C.c_void_p()
        _check("sjd_init", lib.sjd_init(C.byref(c), C.byref(w), _stream(stream), C.byref(h)))
        self.h = h

    def prefill(self, prompt, seed, stream=None):
        _check("sjd_prefill", load_library().sjd_prefill(self.h, _ptr(prompt), prompt.numel(), seed,
                                                          _stream(stream)))

    def plan(self, rows64=False):
        """GEMM plan chosen at init for windows of up to 32 rows (or, rows64,
        of more): splits [qkv, o, gate|up, down, head] followed by the column
        blocks per workgroup of each."""
        out = (C.c_int32 * 20)()
        _check("sjd_get_plan", load_library().sjd_get_plan(self.h, out, 20))
        return list(out)[10:] if rows64 else list(out)[:10]

    def plan_pin(self):
        """The plan for windows of up to 32 rows as an SJD_SPLITS value."""
        p = self.plan()
        return ",".join(f"{p[i]}:{p[5 + i]}" for i in range(4))

    def prefill_image(self, image, prompt, seed, stream=None):
        """Batched contexts: (re)starts image `image` with `prompt`."""
        _check("sjd_prefill_image", load_library().sjd_prefill_image(self.h, image, _ptr(prompt), prompt.numel(), seed,
                                                                      _stream(stream)))

    def prefill_cfg(self, prompt, uncond, seed, stream=None, image=None):
        """Guided contexts (cfg_w != 0): text prompt and unconditional prompt
        (of image `image` of a guided batch; None: sjd_prefill_cfg)."""
        lib = load_library()
        if image is None:
            _check("sjd_prefill_cfg", lib.sjd_prefill_cfg(self.h, _ptr(prompt), prompt.numel(), _ptr(uncond),
                                                          uncond.numel(), seed, _stream(stream)))
        else:
            _check("sjd_prefill_image_cfg", lib.sjd_prefill_image_cfg(self.h, image, _ptr(prompt), prompt.numel(),
                                                                      _ptr(uncond), uncond.numel(), seed,
                                                                      _stream(stream)))

    def set_drafts(self, draft_tok, draft_logits=None, image=0, stream=None):
        """The next step verifies draft_tok (int32 [L], vocabulary ids) against
        draft_logits (float32 [L][V] logits over the sampled range, or None)."""
        _check("sjd_set_drafts", load_library().sjd_set_drafts(self.h, image, _ptr(draft_tok), _ptr(draft_logits),
                                                                _stream(stream)))

    def step(self, temperature, top_k, seed, step, out_meta=None, out_tok=None, out_next=None, stream=None,
             draft_tok=None, draft_logits=None):
        """One iteration. draft_tok (int32 [batch, L] vocabulary ids) and
        draft_logits (float32 [batch, L, V] or None) replace the context's
        own drafts for this step (None: the context's)."""
        _check("sjd_step", load_library().sjd_step(self.h, _ptr(draft_tok), _ptr(draft_logits), 0, 0, temperature,
                                                    top_k, seed, step, _ptr(out_meta), _ptr(out_tok),
                                                    _ptr(out_next), _stream(stream)))

    def forward_window(self, logits, stream=None):
        _check("sjd_forward_window", load_library().sjd_forward_window(self.h, _ptr(logits), _stream(stream)))

    def close(self):
        if getattr(self, "h", None):
            load_library().sjd_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
