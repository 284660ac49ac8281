"""Layers of experts for few tokens at the ends of their numbers' range: factors that stand for no number, for 2^-127 and for 2^127, and activations whose last bit is the smallest number of bf16.  Tolerances
are those of the layers' other tests."""
import numpy as np
import pytest

import paper_2006_05664_amd as P
import test_zz_expert_layer as L
from test_zz_expert_layer_numbers import Rows
from test_zz_experts import CODE, U, V, Matrix, _activations, _torch, _words, gpu
from test_zz_mx4 import VALUES


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("width,inner", [(512, 256), (300, 333), (20, 17), (1040, 1024)])
def test_a_factor_that_is_no_number(width, inner, dtype):
    """255 in a row of w_in makes h of its channel NaN and with it all that its expert's tokens get; in a row of w_out it makes that channel NaN.  Everything else is what it is without."""
    torch, _ = _torch()
    g, rng = torch.Generator(device="cuda").manual_seed(width), np.random.default_rng(inner)
    tokens, k, experts = 8, 2, 6
    win, wout = L.Weights(g, experts * 2 * inner, width, "mx4"), L.Weights(g, experts * width, inner, "mx4")
    ids = np.array([[0, 1], [2, 3], [4, 5], [3, 1], [5, 4], [2, 0], [1, 1], [5, 3]], dtype=np.int32)
    x = Matrix(tokens, width, dtype, values=_activations(rng, tokens, width, dtype))
    y, z = Matrix(tokens, width, dtype), Matrix(tokens, width, dtype, fill=77.0)
    size = P.opevo_expert_layer_workspace(tokens, k, CODE[dtype], inner)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    d_ids = _words(ids, np.int32)
    L._call("mx4", x, dtype, d_ids, None, tokens, k, experts, width, inner, win, wout, y, ws, size)
    clean = y.host()
    assert np.isfinite(clean).all()
    win.f.view[0 * 2 * inner + 3, 0] = 255              # a gate row of expert 0, its first block
    win.f.view[2 * 2 * inner + inner + 5, -1] = 255     # an up row of expert 2, its last block
    wout.f.view[4 * width + 7, 0] = 255                 # channels 7 and 9 of expert 4
    wout.f.view[4 * width + 9, -1] = 255
    L._call("mx4", x, dtype, d_ids, None, tokens, k, experts, width, inner, win, wout, z, ws, size)
    got, none = z.host(), np.zeros((tokens, width), dtype=bool)
    none[((ids == 0) | (ids == 2)).any(axis=1)] = True
    none[np.ix_((ids == 4).any(axis=1), [7, 9])] = True
    assert np.array_equal(np.isnan(got), none)
    assert np.array_equal(got[~none], clean[~none])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width,inner", [(256, 256), (300, 333)])
@pytest.mark.parametrize("into,low", [("win", True), ("win", False), ("wout", True), ("wout", False)])
def test_the_smallest_and_largest_factors(width, inner, into, low, dtype):
    """2^-127 under activations of 2^60, and 2^127 (codes up to 1.5, which fp32 holds) under those of 2^-60."""
    torch, _ = _torch()
    g, rng = torch.Generator(device="cuda").manual_seed(width), np.random.default_rng(inner)
    tokens, k, experts = 5, 1, 2
    win, wout = L.Weights(g, experts * 2 * inner, width, "mx4"), L.Weights(g, experts * width, inner, "mx4")
    up = win.f.view.reshape(experts, 2, inner, -1)
    far = 60 if low else -60
    xv = _activations(rng, tokens, width, dtype) * np.float32(1.0 if into == "wout" else 2.0 ** far)
    if into == "wout":
        up[:, 1] += far                             # h of 2^60, or of 2^-60
        wide = wout
    else:
        up[:, 0] -= far                             # gates of some size all the same
        wide = win
    end = wide.f.view if into == "wout" else up[:, 1]
    end.copy_(torch.randint(0, 3, end.shape, generator=g, device="cuda", dtype=torch.uint8) if low else torch.randint(253, 255, end.shape, generator=g, device="cuda", dtype=torch.uint8))
    for w, K in ((win, width), (wout, inner)):
        if not low and w is wide:
            w.q.view.bitwise_and_(0xBB)             # codes 0, 0.5, 1, 1.5 and their negatives: within fp32 under any factor
        code = torch.stack([w.q.view & 15, w.q.view >> 4], dim=2).reshape(w.q.view.shape[0], -1)[:, :K].long()
        w.values = torch.from_numpy(VALUES).cuda()[code] * torch.exp2(w.f.view.double() - 127).repeat_interleave(32, 1)[:, :K]
    ids = rng.integers(0, experts, (tokens, k)).astype(np.int32)
    x, y = Matrix(tokens, width, dtype, values=xv), Matrix(tokens, width, dtype)
    size = P.opevo_expert_layer_workspace(tokens, k, CODE[dtype], inner)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    L._call("mx4", x, dtype, _words(ids, np.int32), None, tokens, k, experts, width, inner, win, wout, y, ws, size)
    L._layer.dtype = dtype
    want, err = (v.cpu().numpy() for v in L._layer(x.view.double(), ids, None, win, wout, experts, inner))
    assert np.abs(want).max() < 2.0 ** 120 and np.abs(want).max() > 2.0 ** -120
    assert np.all(np.abs(y.host() - want) <= err + V[dtype] * (1 + 1e-3) * np.abs(want) + 2.0 ** -134)


@gpu
@pytest.mark.parametrize("kind", ["i8", "mx4"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_activations(dtype, kind):
    """x down to 2^-109, whose last bit in fp32 is the smallest number of bf16: all of it counts."""
    torch, _ = _torch()
    g, rng = torch.Generator(device="cuda").manual_seed(3), np.random.default_rng(3)
    tokens, k, experts, width, inner = 6, 1, 2, 256, 64
    win, wout = L.Weights(g, experts * 2 * inner, width, kind), L.Weights(g, experts * width, inner, kind)
    xv = _activations(rng, tokens, width, dtype)
    xv = np.where(np.abs(xv) < 2.0 ** -9, np.float32(0), xv) * np.float32(2.0 ** -100)
    if kind == "i8":
        win.scale *= 2.0 ** 100
        win.values *= 2.0 ** 100
    else:
        win.f.view += 100
        win.values *= 2.0 ** 100
    ids = rng.integers(0, experts, (tokens, k)).astype(np.int32)
    x, y = Matrix(tokens, width, dtype, values=xv), Matrix(tokens, width, dtype)
    size = P.opevo_expert_layer_workspace(tokens, k, CODE[dtype], inner)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    L._call(kind, x, dtype, _words(ids, np.int32), None, tokens, k, experts, width, inner, win, wout, y, ws, size)
    L._layer.dtype = dtype
    want, err = (v.cpu().numpy() for v in L._layer(x.view.double(), ids, None, win, wout, experts, inner))
    assert np.all(np.abs(y.host() - want) <= err + V[dtype] * (1 + 1e-3) * np.abs(want))


@gpu
@pytest.mark.parametrize("kind", ["i8", "mx4"])
@pytest.mark.parametrize("exponent", [-100, -109])
def test_the_last_bit_of_a_small_activation(kind, exponent):
    """One number of x counts, and its gate and up are 2^-exponent of it: y = silu(g) g with g in [1, 2), whose roundings (the sum of x's three parts 2u and the factor u for either, twice that through silu's slope of
    at most 2 g sigmoid(g) relative to itself; exp, quotient and products 8u; the sum of h's three parts 2u and the output u) make less than 24 u; without the last of the three parts, 2^-16 of x, it would be 256 u and more."""
    torch, _ = _torch()
    rng = np.random.default_rng(-exponent)
    tokens, width, inner = 64, 256, 128
    xv = np.zeros((tokens, width), dtype=np.float32)
    g = 1 + rng.random(tokens).astype(np.float32).astype(np.float64)
    g = g.astype(np.float32)
    xv[:, 0] = g * np.float32(2.0 ** exponent)
    assert np.array_equal(xv[:, 0].astype(np.float64) * 2.0 ** -exponent, g.astype(np.float64))
    ones_in, ones_out = np.zeros((2 * inner, width)), np.zeros((width, inner))
    ones_in[:, 0] = 1
    ones_out[:, 5] = 1
    win, wout = Rows(ones_in, kind), Rows(ones_out, kind)
    if kind == "i8":
        win.scale *= 2.0 ** -exponent
    else:
        win.f.view += -exponent
    x, y = Matrix(tokens, width, "f32", values=xv), Matrix(tokens, width, "f32")
    size = P.opevo_expert_layer_workspace(tokens, 1, CODE["f32"], inner)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    L._call(kind, x, "f32", _words(np.zeros((tokens, 1)), np.int32), None, tokens, 1, 1, width, inner, win, wout, y, ws, size)
    g = g.astype(np.float64)
    want = (g / (1 + np.exp(-g)) * g)[:, None]
    assert np.all(np.abs(y.host() - want) <= 24 * U * want), (np.abs(y.host() / want - 1) / U).max()
