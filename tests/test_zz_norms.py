"""RMS norms with a residual, their rows in 8 bits and their gradients on the GPU, each against its definition in 64 bits on the host.

Tolerances, u = 2^-24 being half an ulp of fp32 and v that of the output type (2^-24, 2^-8, 2^-11):
  a sum over a row  at least 64 lanes share a row that fills them, a lane adds width / 64 + 8 terms one after the other and the lanes meet in 6 + 3 steps: L = width / 64 + 17 roundings of each term
  1 / rms           the mean's (L + 2) u counts half, its root, the sum with eps and the quotient once each: i_err = (L / 2 + 4) u
  y                 i_err, two products and the output: (i_err + 2u + v) |y|
  scale             i_err and three operations: (i_err + 3u) scale;  q: exactly 127 v / a rounded, but where it is within 127 * 4 * 2^-53 of a tie (fp64's roundings)
  dx                with the exact i rounded to fp32: of A = i |w dy| and B = i^3 |s| mean |w dy s| each at most L + 12 roundings (their operations, and i's in all its powers), of dsum one: (L + 12) u (A + B) + u |dsum| + v |dx|
  dweight           `rows` terms at the most one after the other, each with three roundings: (rows + 4) u sum |dy s i|
and 2^-25 for fp16 outputs, half of its smallest number.  The sum x + residual is the same two roundings on either side: exactly.
"""
import ctypes

import numpy as np
import pytest

import paper_2006_05664_amd as P
from test_zz_experts import CODE, TINY, U, V, Matrix, _activations, _torch, _words, gpu

EPS = 1e-5


def _narrow(v, dtype):
    torch, types = _torch()
    return torch.from_numpy(np.asarray(v, dtype=np.float32)).to(types[dtype]).float().numpy()


def _sum(xv, rv, dtype):
    return xv if rv is None else _narrow(xv + rv, dtype)


def _terms(width):
    return width / 64 + 17


def _i_err(width):
    return (_terms(width) / 2 + 4) * U


def _inv(s, eps=EPS):
    return 1.0 / np.sqrt((s.astype(np.float64) ** 2).mean(axis=1, keepdims=True) + eps)


def _weights(rng, width, dtype):
    return _narrow(1.0 + 0.3 * rng.standard_normal(width), dtype)


# rows, width, dtype, extra between rows, shift
SIZES = [
    (1, 1, "bf16", 0, 0), (1, 7, "f32", 0, 0), (1, 4096, "bf16", 0, 0), (2, 8, "f16", 0, 0), (3, 9, "f16", 2, 1), (5, 64, "bf16", 0, 0), (33, 130, "f32", 3, 1),
    (300, 24, "f16", 0, 0), (70, 1000, "f32", 0, 0), (13, 1001, "bf16", 0, 3), (9, 2048, "f16", 0, 0), (31, 3000, "f32", 0, 0), (7, 8192, "bf16", 8, 0),
    (6, 16384, "f16", 0, 0), (5, 20011, "bf16", 0, 1), (4, 12000, "f32", 0, 0), (9000, 512, "bf16", 0, 0), (4200, 1030, "f16", 0, 0), (2100, 2056, "f32", 0, 0),
    (1030, 4100, "bf16", 0, 0), (20000, 3, "f32", 0, 0),
]


@gpu
@pytest.mark.parametrize("residual,weighted", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("rows,width,dtype,pad,shift", SIZES)
def test_norms(rows, width, dtype, pad, shift, residual, weighted):
    rng = np.random.default_rng(rows * 31 + width)
    xv = _activations(rng, rows, width, dtype) * np.float32(4)
    rv = _activations(rng, rows, width, dtype) if residual else None
    wv = _weights(rng, width, dtype) if weighted else None
    x, y = Matrix(rows, width, dtype, width + pad, shift, values=xv), Matrix(rows, width, dtype, width + pad, shift)
    r = Matrix(rows, width, dtype, width + 2 * pad, shift, values=rv) if residual else None
    w = Matrix(1, width, dtype, None, shift, values=wv[None]) if weighted else None
    s = Matrix(rows, width, dtype, width + pad, shift)
    inv = _words(np.full(rows + 1, -7), np.float32)
    P.opevo_norm_rows(x.ptr, x.ld, r.ptr if r else 0, r.ld if r else 0, w.ptr if w else 0, EPS, CODE[dtype], rows, width, s.ptr if residual else 0, s.ld, y.ptr, y.ld, inv.data_ptr())
    got, want_s = y.host(), _sum(xv, rv, dtype)
    if residual:
        assert np.array_equal(s.host(), want_s)
    want_i = _inv(want_s)
    got_i = inv.cpu().numpy()
    assert got_i[-1] == -7
    assert np.all(np.abs(got_i[:-1, None] - want_i) <= _i_err(width) * want_i)
    want = want_s.astype(np.float64) * want_i * (wv if weighted else 1.0)
    assert np.all(np.abs(got - want) <= (_i_err(width) + 2 * U + V[dtype] * (1 + 1e-3)) * np.abs(want) + TINY[dtype])


def _check_8(q, scale, s, w, width, eps=EPS):
    v = s.astype(np.float64) * (w.astype(np.float64) if w is not None else 1.0)
    with np.errstate(all="ignore"):
        a = np.abs(v).max(axis=1)
        finite = np.isfinite(v).all(axis=1)
        want_scale = a * _inv(s, eps)[:, 0] / 127.0
    assert np.array_equal(np.isnan(scale), ~finite)
    assert np.all(np.abs(scale - want_scale)[finite] <= (_i_err(width) + 3 * U) * want_scale[finite])
    on = finite & (a > 0)
    assert not q[~on].any()
    exact = 127.0 * v[on] / a[on][:, None]
    off = q[on] != np.rint(exact)
    near = np.abs(np.abs(exact - np.floor(exact)) - 0.5) <= 127 * 4 * 2.0 ** -53
    assert not (off & ~near).any()


@gpu
@pytest.mark.parametrize("residual,weighted", [(True, True), (False, True), (False, False)])
@pytest.mark.parametrize("rows,width,dtype,pad,shift", SIZES)
def test_norms_in_8_bits(rows, width, dtype, pad, shift, residual, weighted):
    rng = np.random.default_rng(rows * 37 + width)
    xv = _activations(rng, rows, width, dtype)
    if weighted and rows > 3:
        xv[1] = 0.0                                            # nothing but zeros
        xv[2] = (np.arange(width) % 255 - 127) / 2.0           # ties, where the weight is 1
        xv[3] = 2.0 ** -20
    rv = _activations(rng, rows, width, dtype) if residual else None
    if residual and rows > 3:
        rv[1:4] = 0.0
    wv = _weights(rng, width, dtype) if weighted else None
    if weighted and rows % 2:
        wv[:] = 1.0
    x, q = Matrix(rows, width, dtype, width + pad, shift, values=xv), Matrix(rows, width, "i8", width + pad, shift)
    r = Matrix(rows, width, dtype, width + pad, shift, values=rv) if residual else None
    w = Matrix(1, width, dtype, None, shift, values=wv[None]) if weighted else None
    s = Matrix(rows, width, dtype, width + 2 * pad, shift)
    scale = _words(np.full(rows + 1, -7), np.float32)
    P.opevo_norm_rows_i8(x.ptr, x.ld, r.ptr if r else 0, r.ld if r else 0, w.ptr if w else 0, EPS, CODE[dtype], rows, width, s.ptr, s.ld, q.ptr, q.ld, scale.data_ptr())
    want_s = _sum(xv, rv, dtype)
    assert np.array_equal(s.host(), want_s)
    assert scale[-1].item() == -7
    _check_8(q.host(), scale[:-1].cpu().numpy(), want_s, wv, width)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [5, 700, 20000])
def test_rows_that_hold_no_number(dtype, width):
    """Infinities and NaNs stay in their row; a NaN's neighbours are what they are without it."""
    rng = np.random.default_rng(width)
    xv = _activations(rng, 6, width, dtype)
    xv[1, width // 2], xv[2, 0], xv[3, width - 1], xv[4, 0] = np.inf, -np.inf, np.nan, np.nan
    x, y, q = Matrix(6, width, dtype, values=xv), Matrix(6, width, dtype, fill=0.0), Matrix(6, width, "i8")
    scale = _words(np.zeros(6), np.float32)
    w = Matrix(1, width, dtype, values=_weights(rng, width, dtype)[None])
    P.opevo_norm_rows(x.ptr, width, 0, 0, w.ptr, EPS, CODE[dtype], 6, width, 0, 0, y.ptr, width)
    P.opevo_norm_rows_i8(x.ptr, width, 0, 0, w.ptr, EPS, CODE[dtype], 6, width, 0, 0, q.ptr, width, scale.data_ptr())
    got = y.host()
    assert np.isfinite(got[[0, 5]]).all()
    assert np.isnan(got[3]).all() and np.isnan(got[4]).all()
    assert np.isnan(got[1, width // 2]) and not got[1, np.arange(width) != width // 2].any()        # an infinite square: i = 0
    assert np.array_equal(np.isnan(scale.cpu().numpy()), [False, True, True, True, True, False])
    assert not q.host()[1:5].any() and q.host()[[0, 5]].any(axis=1).all()


@gpu
@pytest.mark.parametrize("width", [9, 4096, 20011])
def test_sum_in_place_of_an_input_and_norm_in_place_of_the_other(width):
    torch, _ = _torch()
    rng = np.random.default_rng(width)
    rows, dtype = 17, "bf16"
    xv, rv, wv = _activations(rng, rows, width, dtype), _activations(rng, rows, width, dtype), _weights(rng, width, dtype)
    w = Matrix(1, width, dtype, values=wv[None])
    x, r, s, y = (Matrix(rows, width, dtype, width + 3, 1, values=v) for v in (xv, rv, xv, xv))
    P.opevo_norm_rows(x.ptr, x.ld, r.ptr, r.ld, w.ptr, EPS, P.OPEVO_BF16, rows, width, s.ptr, s.ld, y.ptr, y.ld)
    for into_x, into_r in ((False, True), (True, False)):
        a, b = Matrix(rows, width, dtype, width + 3, 1, values=xv), Matrix(rows, width, dtype, width + 3, 1, values=rv)
        to_s, to_y = (b, a) if into_r else (a, b)
        P.opevo_norm_rows(a.ptr, a.ld, b.ptr, b.ld, w.ptr, EPS, P.OPEVO_BF16, rows, width, to_s.ptr, to_s.ld, to_y.ptr, to_y.ld)
        assert np.array_equal(to_s.host(), s.host()) and np.array_equal(to_y.host(), y.host())
        a = Matrix(rows, width, dtype, width + 3, 1, values=xv)
        b, q = Matrix(rows, width, dtype, width + 3, 1, values=rv), Matrix(rows, width, "i8")
        scale = _words(np.zeros(rows), np.float32)
        to = b if into_r else a
        P.opevo_norm_rows_i8(a.ptr, a.ld, b.ptr, b.ld, w.ptr, EPS, P.OPEVO_BF16, rows, width, to.ptr, to.ld, q.ptr, width, scale.data_ptr())
        assert np.array_equal(to.host(), s.host())
        _check_8(q.host(), scale.cpu().numpy(), _sum(xv, rv, dtype), wv, width)


def _gradients(s, w, dy, dsum, inv):
    """dx, what bounds its error, dweight and what bounds that, in 64 bits."""
    s, dy, inv = s.astype(np.float64), dy.astype(np.float64), inv.astype(np.float64)
    w = 1.0 if w is None else w.astype(np.float64)
    dx = inv * (w * dy - s * inv ** 2 * (w * dy * s).mean(axis=1, keepdims=True))
    size = inv * np.abs(w * dy) + inv ** 3 * np.abs(s) * np.abs(w * dy * s).mean(axis=1, keepdims=True)
    if dsum is not None:
        dx = dx + dsum
    terms = dy * s * inv
    return dx, size, terms.sum(axis=0), np.abs(terms).sum(axis=0)


@gpu
@pytest.mark.parametrize("past,weighted", [(True, True), (False, True), (False, False)])
@pytest.mark.parametrize("rows,width,dtype,pad,shift", SIZES)
def test_gradients(rows, width, dtype, pad, shift, past, weighted):
    torch, _ = _torch()
    rng = np.random.default_rng(rows * 41 + width)
    sv, gv = _activations(rng, rows, width, dtype) * np.float32(2), _activations(rng, rows, width, dtype)
    pv = _activations(rng, rows, width, dtype) if past else None
    wv = _weights(rng, width, dtype) if weighted else None
    iv = _inv(sv).astype(np.float32)
    s, g, dx = Matrix(rows, width, dtype, width + pad, shift, values=sv), Matrix(rows, width, dtype, width + 2 * pad, shift, values=gv), Matrix(rows, width, dtype, width + pad, shift)
    p = Matrix(rows, width, dtype, width + pad, shift, values=pv) if past else None
    w = Matrix(1, width, dtype, None, shift, values=wv[None]) if weighted else None
    inv, dw = _words(iv[:, 0], np.float32), _words(np.full(width + 1, -7), np.float32)
    size = P.opevo_norm_rows_grad_workspace(rows, width)
    ws = torch.full((size + 64,), 255, dtype=torch.uint8, device="cuda")
    P.opevo_norm_rows_grad(g.ptr, g.ld, p.ptr if p else 0, p.ld if p else 0, s.ptr, s.ld, w.ptr if w else 0, inv.data_ptr(), CODE[dtype], rows, width, dx.ptr, dx.ld,
                           dw.data_ptr(), ws.data_ptr(), size)
    got, got_w = dx.host(), dw.cpu().numpy()
    assert got_w[-1] == -7 and bool((ws[size:] == 255).all())
    want, bound, want_w, bound_w = _gradients(sv, wv, gv, pv, iv)
    assert np.all(np.abs(got - want) <= (_terms(width) + 12) * U * bound * (1 + 1e-3) + (U * np.abs(pv) if past else 0) + V[dtype] * (1 + 1e-3) * np.abs(want) + TINY[dtype])
    assert np.all(np.abs(got_w[:-1] - want_w) <= (rows + 4) * U * bound_w)
    # without the weight's gradient, in place of what comes in
    for into in (g, p):
        if into:
            P.opevo_norm_rows_grad(g.ptr, g.ld, p.ptr if p else 0, p.ld if p else 0, s.ptr, s.ld, w.ptr if w else 0, inv.data_ptr(), CODE[dtype], rows, width, into.ptr, into.ld)
            assert np.array_equal(into.host(), got)
            into.view.copy_(torch.from_numpy(gv if into is g else pv).cuda())


@gpu
def test_gradients_against_differences():
    """The derivative of <y, dy> + <s, dsum> along each input, by a step into the imaginary numbers, which leaves no difference of two near values."""
    torch, _ = _torch()
    rng = np.random.default_rng(3)
    rows, width = 5, 19
    s, w, dy, dsum = rng.standard_normal((rows, width)), 1 + 0.3 * rng.standard_normal(width), rng.standard_normal((rows, width)), rng.standard_normal((rows, width))
    s, w, dy, dsum = (v.astype(np.float32).astype(np.float64) for v in (s, w, dy, dsum))

    def loss(s, w):
        y = s / np.sqrt((s * s).mean(axis=1, keepdims=True) + EPS) * w
        return (y * dy).sum() + (s * dsum).sum()

    h, x, want_x, want_w = 1e-30, Matrix(rows, width, "f32", values=s), np.zeros((rows, width)), np.zeros(width)
    for i in range(rows):
        for j in range(width):
            step = np.zeros((rows, width), dtype=complex)
            step[i, j] = 1j * h
            want_x[i, j] = loss(s + step, w.astype(complex)).imag / h
    for j in range(width):
        step = np.zeros(width, dtype=complex)
        step[j] = 1j * h
        want_w[j] = loss(s.astype(complex), w + step).imag / h
    y, dx, g, p, wm = Matrix(rows, width, "f32"), Matrix(rows, width, "f32"), Matrix(rows, width, "f32", values=dy), Matrix(rows, width, "f32", values=dsum), Matrix(1, width, "f32", values=w[None])
    inv, dw = _words(np.zeros(rows), np.float32), _words(np.zeros(width), np.float32)
    size = P.opevo_norm_rows_grad_workspace(rows, width)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    P.opevo_norm_rows(x.ptr, width, 0, 0, wm.ptr, EPS, P.OPEVO_F32, rows, width, 0, 0, y.ptr, width, inv.data_ptr())
    P.opevo_norm_rows_grad(g.ptr, width, p.ptr, width, x.ptr, width, wm.ptr, inv.data_ptr(), P.OPEVO_F32, rows, width, dx.ptr, width, dw.data_ptr(), ws.data_ptr(), size)
    _, bound, _, bound_w = _gradients(s, w, dy, dsum, _inv(s))
    # i of the forward pass carries i_err in place of one rounding, three times in B
    assert np.all(np.abs(dx.host() - want_x) <= ((_terms(width) + 12) * U + 3 * _i_err(width)) * bound + U * np.abs(dsum) + U * np.abs(want_x))
    assert np.all(np.abs(dw.cpu().numpy() - want_w) <= ((rows + 4) * U + _i_err(width)) * bound_w)


@gpu
def test_no_rows():
    torch, _ = _torch()
    for width in (1, 40, 20011):
        dw = torch.full((width + 1,), -7.0, device="cuda")
        P.opevo_norm_rows(0, 0, 0, 0, 0, EPS, P.OPEVO_BF16, 0, width, 0, 0, 0, 0)
        P.opevo_norm_rows_i8(0, 0, 0, 0, 0, EPS, P.OPEVO_BF16, 0, width, 0, 0, 0, 0, 0)
        assert P.opevo_norm_rows_grad_workspace(0, width) == 0
        P.opevo_norm_rows_grad(0, 0, 0, 0, 0, 0, 0, 0, P.OPEVO_BF16, 0, width, 0, 0, dw.data_ptr())
        torch.cuda.synchronize()
        assert not dw[:-1].any() and dw[-1].item() == -7.0


@gpu
def test_rows_more_than_32_bits_apart():
    """The last row beyond 2^32 bytes from the first."""
    torch, _ = _torch()
    rows, width, far = 3, 40, (1 << 30) + 8
    rng = np.random.default_rng(0)
    xv, rv, wv = _activations(rng, rows, width, "bf16"), _activations(rng, rows, width, "bf16"), _weights(rng, width, "bf16")
    buf = torch.zeros(2 * far + 2 * width, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (rows, width), (far, 1))
    r = torch.as_strided(buf, (rows, width), (far, 1), width)
    x.copy_(torch.from_numpy(xv).cuda())
    r.copy_(torch.from_numpy(rv).cuda())
    w, y = Matrix(1, width, "bf16", values=wv[None]), Matrix(rows, width, "bf16")
    inv = _words(np.zeros(rows), np.float32)
    P.opevo_norm_rows(x.data_ptr(), far, r.data_ptr(), far, w.ptr, EPS, P.OPEVO_BF16, rows, width, r.data_ptr(), far, y.ptr, width, inv.data_ptr())
    s = _sum(xv, rv, "bf16")
    assert np.array_equal(r.float().cpu().numpy(), s)
    want = s * _inv(s) * wv
    assert np.all(np.abs(y.host() - want) <= (_i_err(width) + 2 * U + V["bf16"] * (1 + 1e-3)) * np.abs(want))
    P.opevo_norm_rows_grad(y.ptr, width, r.data_ptr(), far, r.data_ptr(), far, w.ptr, inv.data_ptr(), P.OPEVO_BF16, rows, width, x.data_ptr(), far)
    dx, bound, _, _ = _gradients(s, wv, y.host(), s, inv.cpu().numpy()[:, None])
    assert np.all(np.abs(x.float().cpu().numpy() - dx) <= (_terms(width) + 12) * U * bound + U * np.abs(s) + V["bf16"] * (1 + 1e-3) * np.abs(dx))


def test_refusals():
    """Arguments that a kernel is never started with (no GPU needed)."""
    p, big = 1 << 20, 1 << 41
    ok = dict(x=p, ld_x=8, residual=p, ld_residual=8, weight=p, eps=EPS, dtype=P.OPEVO_BF16, rows=2, width=8, sum=p, ld_sum=8)
    bad = [dict(x=0), dict(x=p + 1), dict(ld_x=7), dict(ld_x=big), dict(residual=p + 1), dict(ld_residual=7), dict(weight=p + 1), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
           dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=(1 << 24) + 1, ld_x=1 << 25, ld_residual=1 << 25, ld_sum=1 << 25), dict(sum=0),
           dict(sum=p + 1), dict(ld_sum=7)]

    def refused(call, *args):
        with pytest.raises(P.OpevoError) as e:
            call(*args)
        assert e.value.status == P.OPEVO_E_ARG

    for change in bad:
        a = {**ok, **change}
        wide = max(8, a["width"])
        refused(P.opevo_norm_rows, *a.values(), p, wide)
        refused(P.opevo_norm_rows_i8, *a.values(), p, wide, p)
    refused(P.opevo_norm_rows, *ok.values(), 0, 8)
    refused(P.opevo_norm_rows, *ok.values(), p + 1, 8)
    refused(P.opevo_norm_rows, *ok.values(), p, 7)
    refused(P.opevo_norm_rows, *ok.values(), p, 8, p + 2)
    refused(P.opevo_norm_rows_i8, *ok.values(), 0, 8, p)
    refused(P.opevo_norm_rows_i8, *ok.values(), p, 7, p)
    refused(P.opevo_norm_rows_i8, *ok.values(), p, 8, 0)
    refused(P.opevo_norm_rows_i8, *ok.values(), p, 8, p + 2)
    grad = dict(dy=p, ld_dy=8, dsum=p, ld_dsum=8, sum=p, ld_sum=8, weight=p, inv=p, dtype=P.OPEVO_F16, rows=600, width=8, dx=p, ld_dx=8, dweight=p, ws=p, size=600 * 32)
    for change in [dict(dy=0), dict(dy=p + 1), dict(ld_dy=7), dict(dsum=p + 1), dict(ld_dsum=7), dict(sum=0), dict(ld_sum=7), dict(weight=p + 1), dict(inv=0), dict(inv=p + 2), dict(dtype=7),
                   dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(dx=0), dict(ld_dx=7), dict(dweight=p + 2), dict(ws=0), dict(ws=p + 1), dict(size=512 * 32 - 1)]:
        refused(P.opevo_norm_rows_grad, *{**grad, **change}.values())
    refused(P.opevo_norm_rows_grad_workspace, -1, 8)
    refused(P.opevo_norm_rows_grad_workspace, 1 << 31, 8)
    refused(P.opevo_norm_rows_grad_workspace, 8, 0)
    refused(P.opevo_norm_rows_grad_workspace, 8, (1 << 24) + 1)
    assert P.binding.lib.opevo_norm_rows_grad_workspace(1, 1, ctypes.POINTER(ctypes.c_size_t)()) == P.OPEVO_E_ARG
    assert P.opevo_norm_rows_grad_workspace(1, 100) == 0 and P.opevo_norm_rows_grad_workspace(1 << 20, 100) == 512 * 400


@gpu
def test_captured_and_replayed():
    """A norm, its 8-bit form and a gradient in one graph: every replay, with eager calls between, gives what the eager calls give."""
    torch, _ = _torch()
    rows, width = 700, 1000
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r, dy, ds = (torch.randn(rows, width, generator=g, device="cuda").bfloat16() for _ in range(4))
    w = torch.rand(width, generator=g, device="cuda").bfloat16()
    size = P.opevo_norm_rows_grad_workspace(rows, width)

    def buffers():
        return dict(s=torch.empty_like(x), y=torch.empty_like(x), inv=torch.empty(rows, device="cuda"), q=torch.empty(rows, width, dtype=torch.int8, device="cuda"), scale=torch.empty(rows, device="cuda"),
                    dx=torch.empty_like(x), dw=torch.empty(width, device="cuda"), ws=torch.empty(size, dtype=torch.uint8, device="cuda"))

    def calls(b, stream):
        at = {k: v.data_ptr() for k, v in b.items()}
        P.opevo_norm_rows(x.data_ptr(), width, r.data_ptr(), width, w.data_ptr(), EPS, P.OPEVO_BF16, rows, width, at["s"], width, at["y"], width, at["inv"], stream)
        P.opevo_norm_rows_i8(x.data_ptr(), width, r.data_ptr(), width, w.data_ptr(), EPS, P.OPEVO_BF16, rows, width, at["s"], width, at["q"], width, at["scale"], stream)
        P.opevo_norm_rows_grad(dy.data_ptr(), width, ds.data_ptr(), width, at["s"], width, w.data_ptr(), at["inv"], P.OPEVO_BF16, rows, width, at["dx"], width, at["dw"], at["ws"], size, stream)

    eager, captured = buffers(), buffers()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(captured, torch.cuda.current_stream().cuda_stream)
    for turn in range(3):
        x.normal_(generator=g)
        for v in captured.values():
            v.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        calls(eager, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for k in eager:
            if k != "ws":
                assert torch.equal(eager[k], captured[k]), (turn, k)
