"""Norms of rows at the ends of their numbers' range, where a step on the way leaves fp32 and the result does not.  Tolerances are those of the norms' other tests."""
import numpy as np
import pytest

import paper_2006_05664_amd as P
import test_zz_norms as N
from test_zz_experts import CODE, U, V, Matrix, _activations, _torch, _words, gpu


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [2e-20, 1e-12, 1e15, 8e18])
@pytest.mark.parametrize("width", [7, 300, 4099, 20011])
def test_gradients_of_small_and_large_rows(width, size, dtype):
    """eps = 0 and 1 / rms up to 5e19 or down to 1e-19, whose square fp32 does not hold, or not in 24 bits.  The gradient is about dy / rms."""
    rng = np.random.default_rng(width)
    rows = 9
    sv = N._narrow(_activations(rng, rows, width, dtype) * np.float32(size), dtype)
    gv, wv = _activations(rng, rows, width, dtype), N._weights(rng, width, dtype)
    iv = N._inv(sv, 0.0).astype(np.float32)
    assert np.isfinite(iv).all()
    s, g, dx = Matrix(rows, width, dtype, values=sv), Matrix(rows, width, dtype, values=gv), Matrix(rows, width, dtype)
    w, inv, dw = Matrix(1, width, dtype, values=wv[None]), _words(iv[:, 0], np.float32), _words(np.zeros(width), np.float32)
    torch, _ = _torch()
    bytes_ = P.opevo_norm_rows_grad_workspace(rows, width)
    ws = torch.empty(max(bytes_, 4), dtype=torch.uint8, device="cuda")
    P.opevo_norm_rows_grad(g.ptr, width, 0, 0, s.ptr, width, w.ptr, inv.data_ptr(), CODE[dtype], rows, width, dx.ptr, width, dw.data_ptr(), ws.data_ptr(), bytes_)
    want, bound, want_w, bound_w = N._gradients(sv, wv, gv, None, iv)
    assert np.all(np.abs(dx.host() - want) <= (N._terms(width) + 12) * U * bound * (1 + 1e-3) + V[dtype] * (1 + 1e-3) * np.abs(want))
    assert np.all(np.abs(dw.cpu().numpy() - want_w) <= (rows + 4) * U * bound_w)


def _in_8_bits(xv, wv, dtype, eps, rv=None, in_place=False):
    rows, width = xv.shape
    x, q = Matrix(rows, width, dtype, values=xv), Matrix(rows, width, "i8")
    r = Matrix(rows, width, dtype, values=rv) if rv is not None else None
    s = x if in_place else Matrix(rows, width, dtype)
    w, scale = Matrix(1, width, dtype, values=wv[None]), _words(np.full(rows + 1, -7), np.float32)
    P.opevo_norm_rows_i8(x.ptr, width, r.ptr if r else 0, width if r else 0, w.ptr, eps, CODE[dtype], rows, width, s.ptr, width, q.ptr, width, scale.data_ptr())
    got, scales = q.host(), scale.cpu().numpy()
    assert scales[-1] == -7
    assert np.array_equal(s.host(), N._sum(xv, rv, dtype))
    return got, scales[:-1]


def _check_q(q, s, w):
    v = s.astype(np.float64) * w.astype(np.float64)
    a = np.abs(v).max(axis=1, keepdims=True)
    exact = 127.0 * v / np.where(a > 0, a, 1.0)
    near = np.abs(np.abs(exact - np.floor(exact)) - 0.5) <= 127 * 4 * 2.0 ** -53
    assert not ((q != np.rint(exact)) & ~near).any()
    return a[:, 0]


@gpu
@pytest.mark.parametrize("width", [3, 130, 700, 1500, 4096, 5001, 20011])
def test_rows_in_8_bits_whose_factor_leaves_fp32(width):
    """fp32 rows and weights whose product is 1e-68 and less, down to the product of two subnormal numbers: q as ever.  (The scale is below fp32: 0.)"""
    rng = np.random.default_rng(width)
    sizes = np.array([1e-31, 1e-35, 1e-38, 1e-42, 1.0, 0.0], dtype=np.float32)
    wv = (1 + rng.random(width)).astype(np.float32) * np.float32(1e-37)
    xv = ((1 + rng.random((len(sizes), width))) * np.where(rng.random((len(sizes), width)) < 0.5, -1, 1) * sizes[:, None]).astype(np.float32)
    q, scale = _in_8_bits(xv, wv, "f32", N.EPS)
    _check_q(q, xv, wv)
    assert not scale[[0, 1, 2, 3, 5]].any() and np.isfinite(scale).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_scale_that_fp32_holds_and_its_127_fold_not(dtype):
    """One number among 4096: i = 64, so that a i = 64 * 3e38 is beyond fp32 and scale = a i / 127 is not."""
    rng = np.random.default_rng(1)
    rows, width = 3, 4096
    xv, wv = np.zeros((rows, width), dtype=np.float32), N._narrow(np.full(width, 3e38), dtype)
    xv[np.arange(rows), rng.integers(0, width, rows)] = [1.0, -0.5, 1.0]
    q, scale = _in_8_bits(xv, wv, dtype, 0.0)
    a = _check_q(q, xv, wv)
    want = a * N._inv(xv, 0.0)[:, 0] / 127.0
    assert np.all(np.abs(scale - want) <= (N._i_err(width) + 3 * U) * want)


# a row of every way a workgroup holds rows in: in one wave, in two of its four, in the whole of it; held and not
@gpu
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,width", [(1, 3), (40, 130), (41, 700), (9, 1500), (8, 4096), (5, 5001), (7, 20011), (3, 8192)])
def test_rows_in_8_bits_whose_products_fp32_does_not_hold(rows, width, residual):
    """bf16 rows of 1e-18 under weights of 1e-22 to 1e-36, with eps = 0: the products are below fp32, where they lose bits and then all of them, and what they make of the row is not.  Rows of other sizes,
    and of zeros, stand between them."""
    rng = np.random.default_rng(width)
    for size in (1e-22, 1e-25, 1e-30, 1e-36):
        wv = N._narrow((1 + rng.random(width)) * size, "bf16")
        xv = _activations(rng, rows, width, "bf16") + 0.1
        xv = N._narrow(xv * np.array([1e-18, 1e-17, 1.0, 1e12])[np.arange(rows) % 4][:, None], "bf16")
        rv = N._narrow(0.3 * rng.standard_normal((rows, width)) * 1e-18, "bf16") if residual else None
        xv[rows // 2] = 0 if rows > 1 else xv[rows // 2]
        if residual:
            rv[rows // 2] = 0
        s = N._sum(xv, rv, "bf16")
        q, scale = _in_8_bits(xv, wv, "bf16", 0.0, rv, in_place=residual)
        a = _check_q(q, s, wv)
        on = a > 0
        want = a[on] * N._inv(s[on], 0.0)[:, 0] / 127.0
        assert np.all(np.abs(scale[on] - want) <= (N._i_err(width) + 3 * U) * want + 2.0 ** -150)
