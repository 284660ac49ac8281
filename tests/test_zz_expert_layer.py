"""Layers of experts for few tokens on the GPU, against the definition in 64 bits on the host.

Tolerance.  u = 2^-24, v half an ulp of the output type, and the products of bf16 numbers are exact.  A sum of K products meets in at most K / 32 + 8 additions of a matrix instruction and 4 of the waves, three of
the parts, each right to 2u of the magnitudes it adds (a sum within the instruction may be cut off, not rounded): E(K) = 2u (K / 32 + 16).  In 64 bits let
  G, U = the two first products, |G|, |U| the same of magnitudes, h = silu(G) U, Y = the second product, weighted, |Y| that of magnitudes
  dG = (E(width) + 2u) |G| (the scale: two roundings; none for factors), dU likewise
  silu' is at most 1.1, silu(G) <= |G|: dh = 1.1 dG |U| + |silu(G)| dU + dG dU + (10u + d) |h|   with d = 2^-16 for the two bf16 that keep h (2^-17 and its first half's bits), 2^-23 for three; exp, the quotient and two products are 8u
  dY = sum_j weight_j sum_k (dh |Wo|) + (E(inner) + 4u + (k + 2) u) |Y|
and |y - Y| <= dY + v |Y| (1 + 1e-3) + half the smallest number.
"""
import numpy as np
import pytest

import paper_2006_05664_amd as P
from test_zz_experts import CODE, TINY, U, V, Matrix, _activations, _torch, _words, gpu
from test_zz_mx4 import VALUES, Bytes


def _e(k):
    return 2 * U * (k / 32 + 16)


class Weights:
    """Rows of weights on the device, and their values in fp64 there (the integers apart from their scales)."""

    def __init__(self, g, rows, K, kind, pad=0, shift=0):
        torch, _ = _torch()
        self.kind = kind
        if kind == "i8":
            self.q = Matrix(rows, K, "i8", K + pad, shift)
            self.q.view.copy_(torch.randint(-128, 128, (rows, K), generator=g, device="cuda", dtype=torch.int8))
            self.scale = (torch.rand(rows, generator=g, device="cuda") + 0.5) / (74 * K ** 0.5)
            self.values = self.q.view.double() * self.scale.double()[:, None]
            self.args = (self.q.ptr, self.q.ld, self.scale.data_ptr())
        else:
            half, blocks = (K + 1) // 2, (K + 31) // 32
            self.q = Bytes(rows, half, half + pad, shift, values=torch.randint(0, 256, (rows, half), generator=g, device="cuda", dtype=torch.uint8))
            middle = 127 - int(round(np.log2(3 * K ** 0.5)))
            self.f = Bytes(rows, blocks, blocks + pad, shift, values=torch.randint(middle - 1, middle + 2, (rows, blocks), generator=g, device="cuda", dtype=torch.uint8))
            code = torch.stack([self.q.view & 15, self.q.view >> 4], dim=2).reshape(rows, -1)[:, :K].long()
            self.values = torch.from_numpy(VALUES).cuda()[code] * torch.exp2(self.f.view.double() - 127).repeat_interleave(32, 1)[:, :K]
            self.args = (self.q.ptr, self.q.ld, self.f.ptr, self.f.ld)


def _layer(x, ids, weight, win, wout, experts, inner):
    """(Y, what bounds the error but for the output's rounding) in fp64 on the device; `x` (tokens, width) in fp64."""
    import torch
    tokens, width = x.shape
    y, err = torch.zeros_like(x), torch.zeros_like(x)
    extra = 2 * U if win.kind == "i8" else 0.0
    k = ids.shape[1]
    keep = 2.0 ** -16 if _layer.dtype != "f32" else 2.0 ** -23
    for e in range(experts):
        t, j = np.nonzero(ids == e)
        if not len(t):
            continue
        a, b = win.values[e * 2 * inner:(e + 1) * 2 * inner], wout.values[e * width:(e + 1) * width]
        xs = x[torch.from_numpy(t).cuda()]
        up, size = torch.matmul(xs, a.t().contiguous()), torch.matmul(xs.abs(), a.abs().t().contiguous())
        d = (_e(width) + extra) * size
        G, Up, dG, dU = up[:, :inner], up[:, inner:], d[:, :inner], d[:, inner:]
        silu = G * torch.sigmoid(G)
        h = silu * Up
        dh = 1.1 * dG * Up.abs() + silu.abs() * dU + 1.1 * dG * dU + (10 * U + keep) * h.abs()
        w = torch.ones(len(t), 1, dtype=torch.float64, device="cuda") if weight is None else torch.from_numpy(weight[t, j].astype(np.float64)).cuda()[:, None]
        bt = b.t().contiguous()
        y.index_add_(0, torch.from_numpy(t).cuda(), w * torch.matmul(h, bt))
        err.index_add_(0, torch.from_numpy(t).cuda(), w.abs() * (torch.matmul(dh, bt.abs()) + (_e(inner) + extra + (k + 6) * U) * torch.matmul(h.abs() + dh, bt.abs())))
    return y, err


def _call(kind, x, dtype, d_ids, d_weight, tokens, k, experts, width, inner, win, wout, y, ws, size, stream=0):
    call = P.opevo_expert_layer_i8 if kind == "i8" else P.opevo_expert_layer_mx4
    call(x.ptr, x.ld, CODE[dtype], d_ids.data_ptr(), d_weight.data_ptr() if d_weight is not None else 0, tokens, k, experts, width, inner, *win.args, *wout.args, y.ptr, y.ld, ws.data_ptr(), size, stream)


# tokens, k, experts, width, inner, held, extra between rows, shift
SIZES = [
    (1, 1, 1, 1, 1, 1.0, 0, 0), (1, 2, 8, 1024, 512, 1.0, 0, 0), (1, 2, 8, 64, 40, 0.0, 0, 0), (3, 2, 4, 17, 33, 0.7, 3, 1), (2, 3, 5, 256, 256, 1.0, 0, 0), (5, 4, 16, 320, 128, 0.9, 0, 0),
    (8, 64, 1024, 32, 24, 0.9, 0, 0), (17, 1, 3, 300, 1001, 1.0, 1, 1), (32, 4, 64, 512, 256, 1.0, 0, 0), (64, 8, 40, 256, 200, 0.8, 0, 0), (100, 5, 2, 128, 384, 1.0, 16, 0), (512, 1, 7, 96, 64, 0.9, 0, 0),
    (256, 2, 300, 130, 65, 1.0, 0, 0), (9, 1, 1, 2048, 31, 1.0, 0, 0), (1, 8, 128, 2560, 768, 1.0, 0, 0), (40, 1, 2, 33, 4096, 1.0, 0, 0), (4, 2, 1000, 1000, 77, 0.9, 5, 3),
    (3, 2, 4, 1030, 512, 1.0, 0, 0), (20, 2, 3, 2050, 1024, 0.9, 0, 0), (1, 1, 2, 7, 2048, 1.0, 0, 0), (50, 3, 5, 1280, 1536, 1.0, 0, 0),
]


@gpu
@pytest.mark.parametrize("kind", ["i8", "mx4"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,k,experts,width,inner,held,pad,shift", SIZES)
def test_layers(tokens, k, experts, width, inner, held, pad, shift, dtype, kind):
    torch, _ = _torch()
    rng = np.random.default_rng(tokens * 7 + width)
    g = torch.Generator(device="cuda").manual_seed(width + inner)
    ids = rng.integers(0, experts, (tokens, k)) if experts < k else np.argsort(rng.random((tokens, experts)), axis=1)[:, :k]
    away = rng.random((tokens, k)) >= held
    ids = np.where(away, np.where(rng.random((tokens, k)) < 0.5, -1 - ids, experts + ids), ids).astype(np.int32)
    weight = rng.random((tokens, k)).astype(np.float32) if tokens % 2 else None
    if weight is not None:
        weight[away] = np.nan                   # a slot that is not held adds nothing, whatever its weight
    xv = _activations(rng, tokens, width, dtype)
    win, wout = Weights(g, experts * 2 * inner, width, kind, pad, shift), Weights(g, experts * width, inner, kind, pad, shift)
    x, y = Matrix(tokens, width, dtype, width + pad, shift, values=xv), Matrix(tokens, width, dtype, width + 2 * pad, shift)
    d_ids, d_weight = _words(ids, np.int32), None if weight is None else _words(weight, np.float32)
    size = P.opevo_expert_layer_workspace(tokens, k, CODE[dtype], inner)
    ws = torch.full((size + 64,), 255, dtype=torch.uint8, device="cuda")
    _call(kind, x, dtype, d_ids, d_weight, tokens, k, experts, width, inner, win, wout, y, ws, size)
    got = y.host()
    assert bool((ws[size:] == 255).all())
    _layer.dtype = dtype
    want, err = (v.cpu().numpy() for v in _layer(x.view.double(), ids, weight, win, wout, experts, inner))
    assert not got[(away.all(axis=1))].any()
    assert np.all(np.abs(got - want) <= err + V[dtype] * (1 + 1e-3) * np.abs(want) + TINY[dtype]), (np.abs(got - want) / (err + V[dtype] * np.abs(want) + 1e-300)).max()
    # again, over what is left in the workspace and the output
    before = y.view.clone()
    y.view.fill_(3.0)
    _call(kind, x, dtype, d_ids, d_weight, tokens, k, experts, width, inner, win, wout, y, ws, size)
    torch.cuda.synchronize()
    assert torch.equal(before, y.view)


@gpu
@pytest.mark.parametrize("kind", ["i8", "mx4"])
def test_the_same_expert_twice(kind):
    """A token that names an expert twice gets it twice."""
    torch, _ = _torch()
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens, k, experts, width, inner = 6, 4, 3, 128, 96
    win, wout = Weights(g, experts * 2 * inner, width, kind), Weights(g, experts * width, inner, kind)
    rng = np.random.default_rng(1)
    xv = _activations(rng, tokens, width, "bf16")
    ids = np.array([[0, 0, 0, 0], [1, 2, 1, 2], [2, 2, 0, 1], [0, 1, 2, 0], [-1, 1, 1, 5], [1, 1, 1, 0]], dtype=np.int32)
    weight = rng.random((tokens, k)).astype(np.float32)
    x, y = Matrix(tokens, width, "bf16", values=xv), Matrix(tokens, width, "bf16")
    d_ids, d_weight = _words(ids, np.int32), _words(weight, np.float32)
    size = P.opevo_expert_layer_workspace(tokens, k, P.OPEVO_BF16, inner)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    _call(kind, x, "bf16", d_ids, d_weight, tokens, k, experts, width, inner, win, wout, y, ws, size)
    _layer.dtype = "bf16"
    want, err = (v.cpu().numpy() for v in _layer(x.view.double(), ids, weight, win, wout, experts, inner))
    assert np.all(np.abs(y.host() - want) <= err + V["bf16"] * (1 + 1e-3) * np.abs(want))


@gpu
@pytest.mark.parametrize("kind", ["i8", "mx4"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_numbers_that_are_none_stay_with_their_token(dtype, kind):
    """The largest numbers and infinities of a type go through its parts; what is no number comes out for that token alone."""
    torch, types = _torch()
    g = torch.Generator(device="cuda").manual_seed(6)
    tokens, k, experts, width, inner = 7, 2, 2, 160, 64
    win, wout = Weights(g, experts * 2 * inner, width, kind), Weights(g, experts * width, inner, kind)
    rng = np.random.default_rng(2)
    xv = _activations(rng, tokens, width, dtype)
    xv[1, 3], xv[3, 7], xv[5, 159] = np.nan, np.inf, -np.inf
    clean = Matrix(tokens, width, dtype, values=np.where(np.isfinite(xv), xv, 0))
    ids = np.tile(np.array([[0, 1]], dtype=np.int32), (tokens, 1))
    x, y, z = Matrix(tokens, width, dtype, values=xv), Matrix(tokens, width, dtype, fill=0.0), Matrix(tokens, width, dtype)
    d_ids = _words(ids, np.int32)
    size = P.opevo_expert_layer_workspace(tokens, k, CODE[dtype], inner)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    _call(kind, x, dtype, d_ids, None, tokens, k, experts, width, inner, win, wout, y, ws, size)
    _call(kind, clean, dtype, d_ids, None, tokens, k, experts, width, inner, win, wout, z, ws, size)
    got, rest = y.host(), z.host()
    assert np.isnan(got[1]).all() and not np.isfinite(got[[3, 5]]).any()
    assert np.array_equal(got[[0, 2, 4, 6]], rest[[0, 2, 4, 6]])


@gpu
def test_captured_and_replayed_beside_eager_calls():
    torch, _ = _torch()
    g = torch.Generator(device="cuda").manual_seed(7)
    tokens, k, experts, width, inner = 12, 3, 9, 256, 130
    win, wout = Weights(g, experts * 2 * inner, width, "mx4"), Weights(g, experts * width, inner, "mx4")
    x, y, z = Matrix(tokens, width, "bf16"), Matrix(tokens, width, "bf16"), Matrix(tokens, width, "bf16")
    ids = torch.zeros(tokens, k, dtype=torch.int32, device="cuda")
    weight = torch.rand(tokens, k, generator=g, device="cuda")
    size = P.opevo_expert_layer_workspace(tokens, k, P.OPEVO_BF16, inner)
    ws = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _call("mx4", x, "bf16", ids, weight, tokens, k, experts, width, inner, win, wout, y, ws[0], size, torch.cuda.current_stream().cuda_stream)
    for turn in range(4):                       # other tokens and other experts, down to none, in the buffers that were captured
        x.view.normal_(generator=g)
        ids.copy_(torch.randint(-turn, experts, (tokens, k), generator=g, device="cuda") if turn < 3 else torch.full((tokens, k), -1, device="cuda"))
        y.view.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _call("mx4", x, "bf16", ids, weight, tokens, k, experts, width, inner, win, wout, z, ws[1], size, torch.cuda.current_stream().cuda_stream)
        assert np.array_equal(y.host(), z.host()), turn
    assert not y.host().any()


@gpu
def test_rows_more_than_32_bits_apart():
    torch, _ = _torch()
    rng = np.random.default_rng(4)
    tokens, k, experts, width, inner, far = 2, 1, 1, 40, 33, (1 << 27) + 16
    ids = _words(np.zeros((tokens, k)), np.int32)
    near = Weights(torch.Generator(device="cuda").manual_seed(1), 2 * inner, width, "i8"), Weights(torch.Generator(device="cuda").manual_seed(2), width, inner, "i8")
    buf = torch.empty(2 * inner * far, dtype=torch.int8, device="cuda")
    apart = torch.as_strided(buf, (2 * inner, width), (far, 1))
    apart.copy_(near[0].q.view)
    out = torch.as_strided(buf, (width, inner), (far, 1), 64)
    out.copy_(near[1].q.view)
    x, y, z = Matrix(tokens, width, "bf16", values=_activations(rng, tokens, width, "bf16")), Matrix(tokens, width, "bf16"), Matrix(tokens, width, "bf16")
    size = P.opevo_expert_layer_workspace(tokens, k, P.OPEVO_BF16, inner)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    _call("i8", x, "bf16", ids, None, tokens, k, experts, width, inner, *near, y, ws, size)
    P.opevo_expert_layer_i8(x.ptr, x.ld, P.OPEVO_BF16, ids.data_ptr(), 0, tokens, k, experts, width, inner, buf.data_ptr(), far, near[0].scale.data_ptr(), buf.data_ptr() + 64, far,
                            near[1].scale.data_ptr(), z.ptr, z.ld, ws.data_ptr(), size)
    assert np.array_equal(y.host(), z.host())


@gpu
def test_a_norm_and_a_layer_as_a_block_uses_them():
    """The residual's addition and the norm, the layer, and the next norm with the layer's output as its residual, against each one's definition."""
    torch, _ = _torch()
    g = torch.Generator(device="cuda").manual_seed(8)
    rng = np.random.default_rng(8)
    tokens, k, experts, width, inner = 5, 2, 6, 320, 96
    win, wout = Weights(g, experts * 2 * inner, width, "mx4"), Weights(g, experts * width, inner, "mx4")
    x, r = (Matrix(tokens, width, "bf16", values=_activations(rng, tokens, width, "bf16")) for _ in range(2))
    ids, weight = rng.integers(0, experts, (tokens, k)).astype(np.int32), rng.random((tokens, k)).astype(np.float32)
    s, n, y, s2, n2 = (Matrix(tokens, width, "bf16") for _ in range(5))
    d_ids, d_weight = _words(ids, np.int32), _words(weight, np.float32)
    size = P.opevo_expert_layer_workspace(tokens, k, P.OPEVO_BF16, inner)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    P.opevo_norm_rows(x.ptr, width, r.ptr, width, 0, 1e-6, P.OPEVO_BF16, tokens, width, s.ptr, width, n.ptr, width)
    _call("mx4", n, "bf16", d_ids, d_weight, tokens, k, experts, width, inner, win, wout, y, ws, size)
    P.opevo_norm_rows(y.ptr, width, s.ptr, width, 0, 1e-6, P.OPEVO_BF16, tokens, width, s2.ptr, width, n2.ptr, width)
    assert torch.equal(s.view, (x.view.float() + r.view.float()).bfloat16())
    _layer.dtype = "bf16"
    want, err = (v.cpu().numpy() for v in _layer(n.view.double(), ids, weight, win, wout, experts, inner))
    assert np.all(np.abs(y.host() - want) <= err + V["bf16"] * (1 + 1e-3) * np.abs(want))
    assert torch.equal(s2.view, (y.view.float() + s.view.float()).bfloat16())
    total = s2.host()
    exact = total / np.sqrt((total ** 2).mean(axis=1, keepdims=True) + 1e-6)
    assert np.all(np.abs(n2.host() - exact) <= (V["bf16"] + 40 * U) * (1 + 1e-3) * np.abs(exact))


def test_refusals():
    """Arguments that a kernel is never started with (no GPU needed)."""
    p = 1 << 20

    def refused(call, *args):
        with pytest.raises(P.OpevoError) as e:
            call(*args)
        assert e.value.status == P.OPEVO_E_ARG

    head = dict(x=p, ld_x=40, dtype=P.OPEVO_BF16, expert=p, weight=p, tokens=4, k=2, experts=3, width=40, inner=33)
    tail = dict(y=p, ld_y=40, ws=p, size=P.opevo_expert_layer_workspace(4, 2, P.OPEVO_BF16, 33))
    in8 = dict(w_in=p, ld_in=40, scale_in=p, w_out=p, ld_out=33, scale_out=p)
    in4 = dict(w_in=p, ld_in=20, scale_in=p, ld_scale_in=2, w_out=p, ld_out=17, scale_out=p, ld_scale_out=2)
    for change in [dict(x=0), dict(x=p + 1), dict(ld_x=39), dict(dtype=3), dict(expert=0), dict(expert=p + 2), dict(weight=p + 1), dict(tokens=-1), dict(tokens=257), dict(k=0), dict(k=65),
                   dict(tokens=9, k=64), dict(experts=0), dict(experts=1025), dict(width=0), dict(inner=0), dict(width=(1 << 20) + 1), dict(inner=(1 << 20) + 1)]:
        refused(P.opevo_expert_layer_i8, *{**head, **change}.values(), *in8.values(), *tail.values())
        refused(P.opevo_expert_layer_mx4, *{**head, **change}.values(), *in4.values(), *tail.values())
    for change in [dict(y=0), dict(y=p + 1), dict(ld_y=39), dict(ws=0), dict(ws=p + 4), dict(size=tail["size"] - 1)]:
        refused(P.opevo_expert_layer_i8, *head.values(), *in8.values(), *{**tail, **change}.values())
        refused(P.opevo_expert_layer_mx4, *head.values(), *in4.values(), *{**tail, **change}.values())
    for change in [dict(w_in=0), dict(ld_in=39), dict(scale_in=0), dict(scale_in=p + 2), dict(w_out=0), dict(ld_out=32), dict(scale_out=0), dict(scale_out=p + 1)]:
        refused(P.opevo_expert_layer_i8, *head.values(), *{**in8, **change}.values(), *tail.values())
    for change in [dict(w_in=0), dict(ld_in=19), dict(scale_in=0), dict(ld_scale_in=1), dict(w_out=0), dict(ld_out=16), dict(scale_out=0), dict(ld_scale_out=1)]:
        refused(P.opevo_expert_layer_mx4, *head.values(), *{**in4, **change}.values(), *tail.values())
    for args in ((-1, 2, 1, 33), (257, 2, 1, 33), (4, 0, 1, 33), (4, 65, 1, 33), (4, 2, 5, 33), (4, 2, 1, 0), (4, 2, 1, (1 << 20) + 1)):
        refused(P.opevo_expert_layer_workspace, *args)
    assert P.opevo_expert_layer_workspace(0, 2, P.OPEVO_F32, 33) == 0
    P.opevo_expert_layer_i8(0, 0, P.OPEVO_F32, 0, 0, 0, 2, 3, 40, 33, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
