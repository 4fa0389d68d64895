"""Rows and weights in 8-bit integers and their products, against plain 64-bit
forms, at the sizes, strides and values where they can go wrong."""
import numpy as np
import pytest
import torch

import paper_2603_18599_amd as sjd

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
ULP = 2.0 ** -24  # half a step of fp32, relative
EPS = 1e-5


def rows_reference(x, norm=None, gate=None):
    """y in 64 bits, and how far 32 bits may be off it, relative to max |y| of the row.
    Norm: the squares' sum is off by a step for each addend that a thread adds up and
    some twenty more (its root by half of that), then four roundings. Gate: e^-x within
    a step, then a sum, a quotient and two products."""
    y, K = x.double(), x.shape[1]
    if norm is not None:
        y = y / torch.sqrt((y * y).mean(1, keepdim=True) + EPS) * norm.double()
        return y, (0.5 * (K / 256 + 20) + 4) * ULP
    if gate is not None:
        z = gate.double()
        return y * z / (1 + torch.exp(-z)), 7 * ULP
    return y, 0.0


def check_rows(y, off, code, scale, cols):
    """A code is off by half a unit, by what y is off, and by the roundings of the row's
    factor, of the product and of the maximum (all relative to at most 127 units)."""
    top = y.abs().max(1).values
    assert ((scale.double() - top / 127).abs() <= top / 127 * (off + 2 * ULP)).all()
    unit = (top / 127).clamp(min=1e-300)[:, None]
    err = (code[:, :y.shape[1]].double() - y / unit).abs().max().item()
    assert err <= 0.5 + 127 * (2 * off + 4 * ULP), err
    assert (code[:, y.shape[1]:cols] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("form", ["rows", "norm", "gate"])
@pytest.mark.parametrize("T,K", [(1, 1), (3, 15), (2, 16), (5, 17), (1, 255), (4, 257), (7, 1000), (1, 4096), (33, 2811),
                                 (3, 4097), (2, 8192), (5, 11008), (3, 16384), (2, 16385), (2, 40001), (1, 65536),
                                 (300, 640), (2050, 264)])
def test_quantise(T, K, form, dtype):
    g = torch.Generator(device="cuda").manual_seed(T * 100003 + K)
    x = (torch.randn(T, K, generator=g, device="cuda") * 3).to(DT[dtype])
    norm = (1 + 0.3 * torch.randn(K, generator=g, device="cuda")).to(DT[dtype]) if form == "norm" else None
    gate = (2 * torch.randn(T, K, generator=g, device="cuda")).to(DT[dtype]) if form == "gate" else None
    code = torch.full((T, sjd.code_columns(K)), 77, dtype=torch.int8, device="cuda")
    scale = torch.full((T,), -1.0, device="cuda")
    sjd.sjd_quantise_rows(x, code, scale, norm=norm, gate=gate, eps=EPS)
    y, off = rows_reference(x, norm, gate)
    check_rows(y, off, code, scale, code.shape[1])


@pytest.mark.parametrize("form", ["rows", "norm", "gate"])
@pytest.mark.parametrize("K", [40, 4096, 20000])
def test_quantise_strides_types_and_neighbours(K, form):
    """Rows inside wider tensors, off every alignment, gains of the other type; bytes
    beside the codes are left as they are."""
    T, cols = 9, sjd.code_columns(K)
    for dtype, off, wide in (("bf16", 1, 5), ("bf16", 8, 16), ("fp32", 3, 7), ("fp32", 4, 8), ("bf16", 4, 8)):
        x = torch.randn(T, K + wide, device="cuda").to(DT[dtype])[:, off:off + K] if wide > off else None
        gate = torch.randn(T, K + 9, device="cuda").to(DT[dtype])[:, 1:1 + K] if form == "gate" else None
        norm = torch.randn(K, device="cuda").to(DT["fp32" if dtype == "bf16" else "bf16"]) if form == "norm" else None
        buf = torch.full((T, cols + 48), 55, dtype=torch.int8, device="cuda")
        code, scale = buf[:, 16:16 + cols], torch.empty(T, device="cuda")
        sjd.sjd_quantise_rows(x, code, scale, norm=norm, gate=gate, eps=EPS)
        y, o = rows_reference(x, norm, gate)
        check_rows(y, o, code, scale, cols)
        assert (buf[:, :16] == 55).all() and (buf[:, 16 + cols:] == 55).all()


@pytest.mark.parametrize("K", [300, 700, 1024, 2047, 4096])
@pytest.mark.parametrize("form", ["rows", "norm", "gate"])
def test_quantised_rows_do_not_depend_on_their_company(form, K):
    """A row's codes and scale have the same bits alone, among a few and among many."""
    T = 1500
    x, g = torch.randn(T, K, device="cuda"), torch.randn(T, K, device="cuda")

    def rows(lo, n):
        code, scale = torch.empty(n, sjd.code_columns(K), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        kw = dict(norm=g[0]) if form == "norm" else dict(gate=g[lo:lo + n]) if form == "gate" else {}
        sjd.sjd_quantise_rows(x[lo:lo + n], code, scale, **kw)
        return code, scale

    code, scale = rows(0, T)
    for lo, n in ((0, 1), (700, 64), (3, 1024), (4, 1025)):
        c, s = rows(lo, n)
        assert torch.equal(c, code[lo:lo + n]) and torch.equal(s, scale[lo:lo + n]), (lo, n)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K", [70, 4096, 30000])
def test_quantise_rows_of_special_values(K, dtype):
    """Zeros, values that are too small to scale, the largest ones, infinities and NaN:
    each keeps to its own row."""
    x = torch.randn(9, K, device="cuda")
    x[1] = 0
    x[2] *= 2.0 ** -110
    x[3] = x[3].clamp(-1, 1) * 3e38
    x[4, K - 1] = float("inf")
    x[5, K // 2] = float("nan")
    x[6, 0] = -float("inf")
    x[7] *= 2.0 ** -90
    x = x.to(DT[dtype])
    code, scale = torch.empty(9, sjd.code_columns(K), dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    sjd.sjd_quantise_rows(x, code, scale)
    fine = [0, 3, 7, 8]
    y, off = rows_reference(x[fine])
    check_rows(y, off, code[fine], scale[fine], code.shape[1])
    assert (code[[1, 2, 4, 5, 6]] == 0).all()
    assert (scale[[1, 2]] == 0).all() and torch.isnan(scale[[4, 5, 6]]).all()
    # behind a norm a row whose squares overflow is one of these, and zeros and tiny rows are fine
    sjd.sjd_quantise_rows(x, code, scale, norm=torch.ones(K, device="cuda"), eps=EPS)
    assert torch.isnan(scale[[3, 4, 5, 6]]).all() and (code[[1, 3, 4, 5, 6]] == 0).all() and scale[1] == 0
    assert torch.isfinite(scale[[0, 1, 2, 7, 8]]).all()
    # gates far from zero on both sides: silu's limits, and no NaN from an exponential that overflows
    gate = torch.zeros(9, K, device="cuda", dtype=DT[dtype])
    gate[0], gate[8] = -200.0, 200.0
    sjd.sjd_quantise_rows(x, code, scale, gate=gate)
    assert scale[0] == 0 and torch.isfinite(scale[8]) and torch.isnan(scale[[4, 5, 6]]).all()
    y, off = rows_reference(x[8:], None, gate[8:])
    check_rows(y, off, code[8:], scale[8:], code.shape[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lo,hi,size", [(-5, -1, 1.0), (-12, -6, 1.0), (-30, -20, 1e3), (-60, -10, 1e6), (-62, -58, 1e10),
                                        (-87, -80, 1e25), (-88.6, -87.5, 1e27), (20, 30, 1.0), (80, 200, 1.0),
                                        (1e-20, 1e-10, 1.0), (-1e-3, 1e-3, 1.0), (3e37, 3e38, 1e-20)])
def test_gates_of_one_size(lo, hi, size, dtype):
    """Rows whose gates are all far below zero, or far above, or near it: no moderate gate covers for
    what they lose. In steps of 2^-24: the power is within 2 and its correction, their product, the
    sum with 1 and the gate's product round by one each, the reciprocal is within 2, and the last
    product rounds by one: 9. ln 2 as a float moves e^-gate by another 0.047 |gate|."""
    T, K = 6, 3000
    g = torch.Generator(device="cuda").manual_seed(int(min(lo, 1000)) + 100)
    x = (torch.randn(T, K, generator=g, device="cuda") * size).to(DT[dtype])
    gate = (lo + (hi - lo) * torch.rand(T, K, generator=g, device="cuda")).to(DT[dtype])
    code = torch.empty(T, sjd.code_columns(K), dtype=torch.int8, device="cuda")
    scale = torch.empty(T, device="cuda")
    sjd.sjd_quantise_rows(x, code, scale, gate=gate)
    z = gate.double()
    check_rows(x.double() * z / (1 + torch.exp(-z)), (9 + 0.047 * max(-lo, 0)) * ULP, code, scale, code.shape[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("K", [100, 4096, 20000])
def test_gates_of_special_values(K, dtype):
    """A gate that is no number or has no limit makes its row, and no other, NaN, at whatever x; the largest
    finite ones are themselves above zero and 0 below it."""
    inf, nan = float("inf"), float("nan")
    x, gate = torch.ones(8, K, device="cuda"), torch.ones(8, K, device="cuda")
    gate[0, K - 1], gate[1, 0], gate[2, K // 2], gate[3, 1], gate[4], gate[5, 3] = inf, -inf, nan, 3e38, -3e38, -3e38
    x[1, 0], x[3] = 0.0, 1e-3
    x, gate = x.to(DT[dtype]), gate.to(DT[dtype])
    code, scale = torch.empty(8, sjd.code_columns(K), dtype=torch.int8, device="cuda"), torch.empty(8, device="cuda")
    sjd.sjd_quantise_rows(x, code, scale, gate=gate)
    assert torch.isnan(scale[:3]).all() and (code[:3] == 0).all() and scale[4] == 0 and (code[4] == 0).all()
    assert (code[[5, 6, 7], :K] == torch.where(gate[[5, 6, 7]] < 0, 0, 127)).all() and torch.isfinite(scale[5:]).all()
    y = (x[3].double() * gate[3].double()).max()
    assert abs(scale[3].double() - y / 127) <= y / 127 * 11 * ULP and code[3, 1] == 127 and (code[3, 2:] == 0).all()


def weights(N, K, seed, low=-127):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randint(low, 128, (N, K), generator=g, device="cuda", dtype=torch.int8)
    h = sjd.I8Weights(N, K, 1e-3 * (0.5 + torch.rand(N, generator=g, device="cuda")))
    sjd.sjd_pack_i8(h, w)
    return h, w


def codes(T, K, seed, low=-127):
    """Codes and scales; what lies behind K is there to be ignored."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    a = torch.randint(low, 128, (T, sjd.code_columns(K)), generator=g, device="cuda", dtype=torch.int8)
    return a, 0.01 * (0.5 + torch.rand(T, generator=g, device="cuda"))


def product(a, a_scale, w, w_scale, add=None):
    """In 64 bits (sums of integers below 2^53: exact), and how far 32 bits may be off: the
    sum becomes a float, two products, and the addition round by half a step each."""
    x = (a[:, :w.shape[1]].double() @ w.double().t()) * a_scale.double()[:, None] * w_scale.double()
    tol = 3.01 * ULP * x.abs()
    if add is not None:
        x = x + add.double()
        tol = tol + ULP * (x.abs() + tol)
    return x, tol


def check_product(out, x, tol):
    err = (out.double() - x).abs()
    if out.dtype is torch.bfloat16:
        tol = tol + 2.0 ** -8 * (x.abs() + tol)
    assert (err <= tol).all(), ((err - tol).max().item(), err.max().item())


def run(h, a, s, dtype, add=None, out=None):
    out = torch.full((a.shape[0], h.N), float("nan"), device="cuda").to(DT[dtype]) if out is None else out
    ws = sjd.matmul_workspace(h, a.shape[0])
    ws.fill_(0xFF)  # (nothing is expected of it)
    sjd.sjd_matmul_i8(h, a, s, out, ws, add=add)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,N,K", [
    (1, 1, 1), (2, 31, 15), (1, 33, 16), (3, 40, 17), (5, 64, 127), (16, 100, 128), (17, 96, 129), (1, 4096, 4096),
    (31, 1000, 640), (32, 256, 4096), (33, 257, 1000), (63, 1024, 256), (64, 4096, 1024), (65, 130, 11008), (77, 1003, 2811),
    (127, 255, 384), (128, 4096, 512), (129, 33, 2816), (200, 1500, 1025), (256, 512, 512), (257, 513, 513), (1, 20, 65536),
    (40, 70, 65536), (513, 1029, 200), (1000, 300, 96), (2049, 520, 320), (300, 12288, 130)])
def test_product(T, N, K, dtype):
    h, w = weights(N, K, T + N)
    a, s = codes(T, K, K)
    add = torch.randn(T, N, device="cuda").to(DT[dtype]) if (T + N + K) % 2 else None
    out = run(h, a, s, dtype, add)
    check_product(out, *product(a, s, w, h.scale, add))


def test_product_of_the_largest_codes():
    """-128 everywhere: sums of 2^30 for the longest rows."""
    for T in (1, 40, 300):
        K, N = 65536, 35
        h, w = sjd.I8Weights(N, K, torch.ones(N, device="cuda")), torch.full((N, K), -128, dtype=torch.int8, device="cuda")
        sjd.sjd_pack_i8(h, w)
        a, s = torch.full((T, K), -128, dtype=torch.int8, device="cuda"), torch.ones(T, device="cuda")
        assert (run(h, a, s, "fp32") == 2.0 ** 30).all()


@pytest.mark.parametrize("T", [1, 20, 90, 400])
def test_product_strides_and_neighbours(T):
    """Codes inside wider rows, outputs at odd places of wider ones (no wide stores), an addend
    of another stride, in place; what lies beside is left as it was."""
    N, K = 203, 300
    h, w = weights(N, K, 5)
    a, s = codes(T, K, 6)
    wide = torch.full((T, 512), 99, dtype=torch.int8, device="cuda")
    wide[:, 32:32 + a.shape[1]] = a
    for dtype in ("bf16", "fp32"):
        for off, more in ((0, 5), (1, 1), (8, 24), (3, 8)):
            buf = torch.full((T, N + off + more), 7.0, device="cuda").to(DT[dtype])
            add = torch.randn(T, N + 3, device="cuda").to(DT[dtype])[:, 2:2 + N]
            out = buf[:, off:off + N]
            run(h, wide[:, 32:32 + a.shape[1]], s, dtype, add, out)
            check_product(out, *product(a, s, w, h.scale, add))
            assert (buf[:, :off] == 7).all() and (buf[:, off + N:] == 7).all()
            before = out.clone()
            run(h, a, s, dtype, out, out)
            check_product(out, *product(a, s, w, h.scale, before))


def test_rows_do_not_depend_on_their_company():
    """A row's product has the same bits in any batch and at any place in it."""
    N, K = 1100, 1536
    h, w = weights(N, K, 1)
    a, s = codes(700, K, 2)
    whole = run(h, a, s, "fp32")
    for lo, n in ((0, 1), (699, 1), (5, 16), (100, 33), (30, 65), (7, 129), (200, 300)):
        assert torch.equal(run(h, a[lo:lo + n].contiguous(), s[lo:lo + n].contiguous(), "fp32"), whole[lo:lo + n])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,K", [(1100, 1536), (1101, 1537), (512, 8192)])
def test_rows_with_addends_do_not_depend_on_their_company(N, K, dtype):
    """The addend joins by the same steps in the kernels of few and of many rows, where
    the inputs are split and where channels do not come by fours."""
    h, w = weights(N, K, 1)
    a, s = codes(1500, K, 2)
    add = torch.randn(1500, N, device="cuda").to(DT[dtype])
    whole = run(h, a, s, dtype, add)
    assert len({sjd.matmul_workspace(h, n).numel() > 0 for n in (1, 100, 300, 700, 1500)}) == (2 if K == 8192 else 1)
    for lo, n in ((0, 1), (699, 1), (5, 16), (100, 33), (30, 100), (7, 300), (200, 700)):
        assert torch.equal(run(h, a[lo:lo + n].contiguous(), s[lo:lo + n].contiguous(), dtype, add[lo:lo + n].contiguous()),
                           whole[lo:lo + n]), (lo, n)


@pytest.mark.parametrize("T,N,K,dtype", [(4171, 4096, 4096, "bf16"), (4116, 4096, 4096, "fp32"),
                                         (4171, 4096, 11008, "fp32"), (1500, 12288, 4096, "bf16"),
                                         (4096, 5001, 4096, "bf16"), (1500, 22016, 1000, "fp32")])
def test_products_in_two_parts(T, N, K, dtype):
    """Sizes whose last rows or channels are a launch of their own, with outputs and
    addends in wider tensors whose other elements stay as they were."""
    h, w = weights(N, K, 5)
    a, s = codes(T, K, 6)
    out = torch.full((T, N + 3), 7.0, device="cuda", dtype=DT[dtype])
    add = torch.randn(T, N + 1, device="cuda").to(DT[dtype])[:, :N]
    run(h, a, s, dtype, add, out[:, 1:1 + N])
    check_product(out[:, 1:1 + N], *product(a, s, w, h.scale, add))
    assert (out[:, 0] == 7).all() and (out[:, 1 + N:] == 7).all()
    for lo, n in ((T - 1, 1), (T - 80, 80), (0, 200)):
        assert torch.equal(run(h, a[lo:lo + n].contiguous(), s[lo:lo + n].contiguous(), dtype, add[lo:lo + n]),
                           out[lo:lo + n, 1:1 + N]), (lo, n)


def test_nan_scales_and_addends_stay_in_their_rows():
    N, K, T = 150, 256, 70
    h, w = weights(N, K, 3)
    a, s = codes(T, K, 4)
    s[3], s[40] = float("nan"), float("inf")
    add = torch.zeros(T, N, device="cuda")
    add[5, 7] = float("nan")
    add[6, 8] = float("inf")
    out = run(h, a, s, "fp32", add)
    ok = torch.ones(T, N, dtype=torch.bool, device="cuda")
    ok[3], ok[40], ok[5, 7], ok[6, 8] = False, False, False, False
    assert torch.isfinite(out[ok]).all() and torch.isnan(out[3]).all() and torch.isnan(out[5, 7]) and out[6, 8] == float("inf")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_weights_are_quantised_like_rows(dtype):
    """Packed from float weights: the products are those of the rows' rule."""
    for N, K in ((1, 5), (50, 333), (300, 1024), (70, 2816)):
        x = torch.randn(N, K + 3, device="cuda").to(DT[dtype])[:, 1:1 + K]
        if N > 10:
            x[4] = 0
            x[7, 2] = float("inf")
        h = sjd.I8Weights(N, K)
        sjd.sjd_pack_i8(h, x)
        code, scale = torch.empty(N, sjd.code_columns(K), dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
        sjd.sjd_quantise_rows(x, code, scale)
        assert torch.equal(torch.nan_to_num(h.scale, nan=-1), torch.nan_to_num(scale, nan=-1))
        g = sjd.I8Weights(N, K, scale)
        sjd.sjd_pack_i8(g, code[:, :K])
        assert torch.equal(h.w, g.w)


def test_offsets_past_32_bits():
    """Codes, outputs and weights of more than 2^31 bytes and elements."""
    N, K = 64, 1024
    h, w = weights(N, K, 8)
    T, row = 40, 1 << 26  # 2.6 GB of codes; outputs of 2.6 G elements
    a, s = codes(T, K, 9)
    wide = torch.empty(T * row, dtype=torch.int8, device="cuda").as_strided((T, K), (row, 1))
    wide.copy_(a)
    out = torch.empty(T * row, dtype=torch.bfloat16, device="cuda").as_strided((T, N), (row, 1))
    run(h, wide, s, "bf16", None, out)
    check_product(out, *product(a, s, w, h.scale))
    x = torch.empty(T * row, dtype=torch.bfloat16, device="cuda").as_strided((T, K), (row, 1))
    x.copy_(torch.randn(T, K, device="cuda"))
    scale = torch.empty(T, device="cuda")
    wide.zero_()
    sjd.sjd_quantise_rows(x, wide, scale)
    check_rows(x.double(), 0.0, wide, scale, K)
    del wide, out, x
    N, K = 33000, 65536
    h, w = weights(N, K, 10)
    for T in (1, 300):
        a, s = codes(T, K, 11)
        out = run(h, a, s, "fp32")
        pick = torch.tensor([0, 31, 16000, 32767, 32768, 32999], device="cuda")
        want, tol = product(a, s, w[pick], h.scale[pick])
        check_product(out[:, pick], want, tol)


def test_no_rows():
    h, _ = weights(40, 50, 1)
    a, s = codes(0, 50, 1)
    assert run(h, a, s, "fp32").shape == (0, 40)
    sjd.sjd_quantise_rows(torch.empty(0, 50, device="cuda"), a, s)


def test_two_streams_and_graphs():
    """Calls that overlap in time on streams of their own, and captured ones replayed
    between eager work, with a workspace each."""
    N, K = 4096, 2816
    h, w = weights(N, K, 20)
    sets = []
    for T in (3, 100):
        x = torch.randn(T, K, device="cuda")
        sets.append(dict(x=x, code=torch.empty(T, sjd.code_columns(K), dtype=torch.int8, device="cuda"),
                         scale=torch.empty(T, device="cuda"), out=torch.empty(T, N, device="cuda"),
                         ws=sjd.matmul_workspace(h, T)))

    def go(d, stream=None):
        sjd.sjd_quantise_rows(d["x"], d["code"], d["scale"], stream=stream)
        sjd.sjd_matmul_i8(h, d["code"], d["scale"], d["out"], d["ws"], stream=stream)

    for d in sets:
        go(d)
    want = [d["out"].clone() for d in sets]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for d in sets:
        d["out"].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for d, st in zip(sets, streams):
            go(d, st)
    torch.cuda.synchronize()
    for d, v in zip(sets, want):
        assert torch.equal(d["out"], v)
    graphs = []
    for d in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            go(d)
    for i in range(4):
        xs = [torch.randn_like(d["x"]) for d in sets]
        for d, x, g in zip(sets, xs, graphs):
            d["x"].copy_(x)
            g.replay()
        torch.cuda.synchronize()
        got = [d["out"].clone() for d in sets]
        for d, v in zip(sets, got):
            go(d)
            assert torch.equal(d["out"], v)


def test_captured_products_that_share_a_workspace():
    """Split inputs and a product in two parts, captured with one workspace and replayed
    in turn on one stream: nothing in it outlives a call."""
    calls = []
    for T, N, K in ((128, 4096, 11008), (1500, 12288, 4096), (4171, 4096, 4096)):
        h, _ = weights(N, K, T)
        a, s = codes(T, K, T + 1)
        calls.append((h, a, s, torch.empty(T, N, device="cuda", dtype=torch.bfloat16)))
    ws = max((sjd.matmul_workspace(h, a.shape[0]) for h, a, _, _ in calls), key=torch.Tensor.numel)
    assert ws.numel() > 0
    graphs = []
    for h, a, s, out in calls:
        sjd.sjd_matmul_i8(h, a, s, out, ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            sjd.sjd_matmul_i8(h, a, s, out, ws)
    for i in range(4):
        for h, a, s, out in calls:
            a.random_(-127, 128)
            out.zero_()
        for g in graphs:
            g.replay()
        ws.fill_(0xFF)
        graphs[i % 3].replay()
        torch.cuda.synchronize()
        for h, a, s, out in calls:
            assert torch.equal(out, run(h, a, s, "bf16"))
