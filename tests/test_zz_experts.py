"""Expert layers on the GPU: dispatch, combine, their gradients, rows in 8 bits, and the 8-bit products, each against its definition in 64 bits on the host.

Tolerances, u = 2^-24 being half an ulp of fp32 and v that of the output type (2^-24, 2^-8, 2^-11 for 24, 8 and 11 significant bits):
  products   the sum is exact; its rounding, the product of the scales, the product with it and the output: (3u + v) |c|
  combine    k products and k sums: (k + 1) u sum |w x| + v |y|
  drows      one product: (u + v) |value|;  dw: `width` products and sums: (width + 1) u sum |dy x|
  rows in 8 bits: 16-bit inputs exactly; fp32 inputs exactly but where 127 x / a is within 127 * 3u of a tie (three roundings)
and 2^-25 for fp16 outputs, half of its smallest number.  Everything else is copied: exactly.
"""
import numpy as np
import pytest

import paper_2006_05664_amd as P

gpu = pytest.mark.gpu
CODE = {"f32": P.OPEVO_F32, "bf16": P.OPEVO_BF16, "f16": P.OPEVO_F16}
U = 2.0 ** -24
V = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}


def _torch():
    import torch
    assert torch.cuda.is_available()
    return torch, {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Matrix:
    """rows x width on the device, rows `ld` apart, `shift` elements into its buffer; what is around it is `fill` and has to stay so."""

    def __init__(self, rows, width, dtype, ld=None, shift=0, fill=float("nan"), values=None):
        torch, types = _torch()
        t = torch.int8 if dtype == "i8" else types[dtype]
        self.rows, self.width, self.ld, self.shift, self.fill = rows, width, ld or width, shift, 77 if dtype == "i8" else fill
        self.buf = torch.full((rows * self.ld + shift + 64,), self.fill, dtype=t, device="cuda")
        self.view = torch.as_strided(self.buf, (rows, width), (self.ld, 1), shift)
        if values is not None:
            self.view.copy_(torch.from_numpy(np.ascontiguousarray(values)).to("cuda").to(t))

    @property
    def ptr(self):
        return self.buf.data_ptr() + self.shift * self.buf.element_size()

    def host(self):
        """The matrix in float64, after a look at what surrounds it."""
        torch, _ = _torch()
        torch.cuda.synchronize()
        inside = torch.zeros(self.buf.shape, dtype=torch.bool, device="cuda")
        torch.as_strided(inside, (self.rows, self.width), (self.ld, 1), self.shift).fill_(True)
        around = self.buf[~inside]
        assert bool((torch.isnan(around) if self.fill != self.fill else around == self.fill).all()), "written outside the matrix"
        return self.view.double().cpu().numpy()


def _words(values, dtype):
    torch, _ = _torch()
    return torch.from_numpy(np.ascontiguousarray(values, dtype=dtype)).cuda()


def _route(ids, experts):
    """The definition: offsets and the row of each slot."""
    flat = [int(e) for e in np.asarray(ids).ravel()]
    offsets = np.array([np.count_nonzero((np.asarray(ids) >= 0) & (np.asarray(ids) < i)) for i in range(experts + 1)])
    row, at = [], list(offsets[:-1])
    for e in flat:
        if 0 <= e < experts:
            row.append(at[e])
            at[e] += 1
        else:
            row.append(-1)
    return offsets, np.array(row, dtype=np.int64)


def _ids(rng, tokens, k, experts, held, skew=True):
    p = np.exp(rng.standard_normal(experts) * (1.5 if skew else 0.0))
    ids = rng.choice(experts, size=(tokens, k), p=p / p.sum())
    away = rng.random((tokens, k)) >= held
    return np.where(away, np.where(rng.random((tokens, k)) < 0.5, -1 - ids, experts + ids), ids).astype(np.int32)


def _activations(rng, rows, width, dtype):
    torch, types = _torch()
    x = rng.standard_normal((rows, width)).astype(np.float32)
    return torch.from_numpy(x).to(types[dtype]).float().numpy()


def _workspace(tokens, k, experts):
    torch, _ = _torch()
    size = P.opevo_route_workspace(tokens, k, experts)
    return torch.full((size + 64,), 255, dtype=torch.uint8, device="cuda"), size


def _dispatch(ids, experts, x, dtype, rows, to8=None, stream=0):
    tokens, k = ids.shape
    d_ids = _words(ids, np.int32)
    offsets, row_of_slot = _words(np.full(experts + 2, -7), np.int32), _words(np.full(tokens * k + 1, -7), np.int32)
    ws, size = _workspace(tokens, k, experts)
    if to8 is None:
        P.opevo_route_dispatch(d_ids.data_ptr(), tokens, k, experts, x.ptr, x.ld, CODE[dtype], x.width, offsets.data_ptr(), row_of_slot.data_ptr(),
                               rows.ptr, rows.ld, ws.data_ptr(), size, stream)
    else:
        P.opevo_route_dispatch_i8(d_ids.data_ptr(), tokens, k, experts, x.ptr, x.ld, CODE[dtype], x.width, offsets.data_ptr(), row_of_slot.data_ptr(),
                                  rows.ptr, rows.ld, to8.data_ptr(), ws.data_ptr(), size, stream)
    import torch
    torch.cuda.synchronize()
    got_offsets, got_rows = offsets.cpu().numpy(), row_of_slot.cpu().numpy()
    assert got_offsets[-1] == -7 and got_rows[-1] == -7 and bool((ws[size:] == 255).all())
    want_offsets, want_rows = _route(ids, experts)
    assert np.array_equal(got_offsets[:-1], want_offsets)
    assert np.array_equal(got_rows[:-1], want_rows)
    return want_offsets, want_rows, offsets, row_of_slot


# tokens, k, experts, width, dtype, held, extra elements between rows, shift
ROUTES = [
    (1, 1, 1, 1, "bf16", 1.0, 0, 0),
    (1, 2, 8, 1024, "bf16", 1.0, 0, 0),
    (1, 2, 8, 64, "f32", 0.0, 0, 0),            # nothing is held here
    (3, 64, 1024, 7, "f16", 0.9, 2, 1),         # every slot a token can have, every expert there can be
    (5, 3, 4, 17, "f32", 0.8, 3, 1),
    (2, 8, 1000, 33, "bf16", 0.8, 0, 0),
    (16, 1, 65, 100, "f16", 0.7, 0, 0),
    (17, 1, 64, 100, "f32", 0.7, 0, 0),
    (33, 8, 40, 1001, "f16", 0.75, 0, 0),
    (64, 2, 64, 8200, "bf16", 1.0, 0, 0),       # rows longer than a workgroup holds in one go
    (257, 5, 9, 130, "bf16", 0.5, 1, 3),
    (1500, 3, 100, 24, "bf16", 0.9, 0, 0),      # counted chunk by chunk
    (4097, 1, 1, 8, "f32", 1.0, 0, 0),          # one expert takes all
    (4500, 7, 1000, 40, "f16", 0.95, 0, 0),
    (20011, 2, 13, 72, "bf16", 0.9, 8, 0),
    (150001, 2, 777, 8, "f16", 0.97, 0, 0),
]


@gpu
@pytest.mark.parametrize("tokens,k,experts,width,dtype,held,pad,shift", ROUTES)
def test_dispatch_and_its_gradient(tokens, k, experts, width, dtype, held, pad, shift):
    rng = np.random.default_rng(tokens * 31 + k)
    ids = _ids(rng, tokens, k, experts, held)
    xv = _activations(rng, tokens, width, dtype)
    x = Matrix(tokens, width, dtype, width + pad, shift, values=xv)
    rows = Matrix(tokens * k, width, dtype, width + pad, shift)
    offsets, row, _, d_row = _dispatch(ids, experts, x, dtype, rows)
    got, want = rows.host(), np.zeros((tokens * k, width))
    has = row >= 0
    want[row[has]] = xv[np.nonzero(has)[0] // k]
    assert np.array_equal(got, want)

    gv = _activations(rng, tokens * k, width, dtype)
    g = Matrix(tokens * k, width, dtype, width + pad, shift, values=gv)
    dx = Matrix(tokens, width, dtype, width + pad, shift)
    P.opevo_route_combine(g.ptr, g.ld, CODE[dtype], 0, d_row.data_ptr(), tokens, k, width, dx.ptr, dx.ld)
    terms = np.where(has[:, None], gv[row], 0.0).astype(np.float64).reshape(tokens, k, width)
    exact = terms.sum(1)
    assert np.all(np.abs(dx.host() - exact) <= (k + 1) * U * np.abs(terms).sum(1) + V[dtype] * np.abs(exact) * (1 + 1e-6) + TINY[dtype])


@gpu
@pytest.mark.parametrize("tokens,k,experts,width,dtype,held,pad,shift", ROUTES)
def test_combine_and_its_gradients(tokens, k, experts, width, dtype, held, pad, shift):
    rng = np.random.default_rng(tokens * 37 + k)
    offsets, row = _route(_ids(rng, tokens, k, experts, held), experts)
    has = row >= 0
    rv, gv = _activations(rng, tokens * k, width, dtype), _activations(rng, tokens, width, dtype)
    w = rng.random(tokens * k).astype(np.float32)
    clean = w.copy()
    w[~has] = np.nan                            # a slot without a row adds nothing, whatever its weight
    clean[~has] = 0
    d_w, d_row, d_off = _words(w, np.float32), _words(row, np.int32), _words(offsets, np.int32)
    rv[int(offsets[-1]):] = np.nan              # rows of no slot are never read
    rows, dy = Matrix(tokens * k, width, dtype, width + pad, shift, values=rv), Matrix(tokens, width, dtype, width + pad, shift, values=gv)
    y, drows = Matrix(tokens, width, dtype, width + pad, shift), Matrix(tokens * k, width, dtype, width + pad, shift)
    dw = _words(np.full(tokens * k + 1, np.nan), np.float32)
    P.opevo_route_combine(rows.ptr, rows.ld, CODE[dtype], d_w.data_ptr(), d_row.data_ptr(), tokens, k, width, y.ptr, y.ld)
    P.opevo_route_combine_grad(dy.ptr, dy.ld, rows.ptr, rows.ld, CODE[dtype], d_w.data_ptr(), d_row.data_ptr(), d_off.data_ptr(), experts, tokens, k, width,
                               drows.ptr, drows.ld, dw.data_ptr())
    values = np.where(has[:, None], rv[row], 0.0).astype(np.float64)
    terms = (clean[:, None].astype(np.float64) * values).reshape(tokens, k, width)
    exact = terms.sum(1)
    assert np.all(np.abs(y.host() - exact) <= (k + 1) * U * np.abs(terms).sum(1) + V[dtype] * np.abs(exact) * (1 + 1e-6) + TINY[dtype])

    g = gv.astype(np.float64)[np.arange(tokens * k) // k]
    want = np.zeros((tokens * k, width))
    want[row[has]] = (clean[:, None] * g)[has]
    assert np.all(np.abs(drows.host() - want) <= (U + V[dtype] * (1 + U)) * np.abs(want) + TINY[dtype])
    got = dw.cpu().numpy()
    assert np.isnan(got[-1])
    assert np.all(np.abs(got[:-1] - (g * values).sum(1)) <= (width + 1) * U * (np.abs(g * values)).sum(1))


@gpu
def test_gradients_against_differences():
    """The layer y = combine(w, rows = dispatch(x)) is linear in x and in w: a difference of the loss <y, dy> is its gradient times the step, whatever the step."""
    torch, _ = _torch()
    tokens, k, experts, width = 6, 3, 5, 19
    rng = np.random.default_rng(5)
    ids = _ids(rng, tokens, k, experts, 0.8)
    xv, w, gv = _activations(rng, tokens, width, "f32"), rng.random(tokens * k).astype(np.float32), _activations(rng, tokens, width, "f32")

    def forward(xv, w):
        x, rows, y = Matrix(tokens, width, "f32", values=xv), Matrix(tokens * k, width, "f32"), Matrix(tokens, width, "f32")
        _, _, d_off, d_row = _dispatch(ids, experts, x, "f32", rows)
        d_w = _words(w, np.float32)
        P.opevo_route_combine(rows.ptr, width, P.OPEVO_F32, d_w.data_ptr(), d_row.data_ptr(), tokens, k, width, y.ptr, width)
        return y.host(), rows, d_off, d_row, d_w

    y0, rows, d_off, d_row, d_w = forward(xv, w)
    dy, drows, dx = Matrix(tokens, width, "f32", values=gv), Matrix(tokens * k, width, "f32"), Matrix(tokens, width, "f32")
    dw = _words(np.zeros(tokens * k), np.float32)
    P.opevo_route_combine_grad(dy.ptr, width, rows.ptr, width, P.OPEVO_F32, d_w.data_ptr(), d_row.data_ptr(), d_off.data_ptr(), experts, tokens, k, width,
                               drows.ptr, width, dw.data_ptr())
    P.opevo_route_combine(drows.ptr, width, P.OPEVO_F32, 0, d_row.data_ptr(), tokens, k, width, dx.ptr, width)
    dxv, dwv = dx.host(), dw.cpu().numpy()
    # y and its neighbour carry (k + 1) u sum |w x| each; |w| < 1, |x| < 8, a step of 1 adds one more: the loss below 2 (k + 1) u k 9 sum |dy|
    tol = 2 * (k + 1) * U * k * 9 * np.abs(gv).sum()
    for t, c in ((0, 0), (1, 18), (3, 7), (5, 11)):
        moved = xv.copy()
        moved[t, c] += 1.0
        step = float(moved[t, c]) - float(xv[t, c])
        assert abs(((forward(moved, w)[0] - y0) * gv).sum() - step * dxv[t, c]) <= tol
    for s in (0, 4, 10, 17):
        moved = w.copy()
        moved[s] += 1.0
        step = float(moved[s]) - float(w[s])
        assert abs(((forward(xv, moved)[0] - y0) * gv).sum() - step * dwv[s]) <= tol


def _check_rows_in_8_bits(xv, dtype, q, scale):
    a = np.abs(xv).max(axis=1).astype(np.float64)
    finite = np.isfinite(xv).all(axis=1)
    want_scale = np.where(finite, (a.astype(np.float32) / np.float32(127)), np.float32(np.nan)).astype(np.float32)
    assert np.array_equal(scale, want_scale, equal_nan=True)
    on = finite & (a > 0)
    assert not q[~on].any()
    exact = 127.0 * xv[on].astype(np.float64) / a[on][:, None]
    off = q[on] != np.rint(exact)
    if dtype == "f32":
        near = np.abs(np.abs(exact - np.floor(exact)) - 0.5) <= 127 * 3 * U
        assert not (off & ~near).any() and np.abs(q[on] - exact).max(initial=0) <= 0.5 + 127 * 3 * U
    else:
        assert not off.any()


def _odd_rows(rng, rows, width, dtype):
    """Activations with the rows that quantisation can trip over: zeros, one value, the smallest and largest numbers, ties, infinities, NaN."""
    torch, types = _torch()
    x = _activations(rng, rows, width, dtype)
    small, large = torch.finfo(types[dtype]).smallest_normal, torch.finfo(types[dtype]).max
    with np.errstate(all="ignore"):
        specials = [np.zeros(width), np.where(np.arange(width) == width - 1, -3.0, 0.0), np.full(width, small) * np.where(rng.random(width) < 0.5, 1, 0.25),
                    np.where(rng.random(width) < 0.5, large, -large / 2), (np.arange(width) % 255 - 127) / 2.0, np.where(np.arange(width) == width // 2, np.inf, 1.0),
                    np.where(np.arange(width) == width - 1, np.nan, 1.0), np.where(np.arange(width) == 0, -np.inf, np.nan)]
    for i, s in enumerate(specials):
        if i < rows - 1:
            x[i + 1] = torch.from_numpy(np.asarray(s, dtype=np.float32)).to(types[dtype]).float().numpy()
    return x


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width,pad,shift", [(1, 1, 0, 0), (1, 1024, 0, 0), (9, 7, 3, 1), (12, 16, 0, 0), (65, 1000, 0, 0), (10, 1001, 2, 3), (300, 64, 0, 0),
                                                  (33, 2048, 0, 0), (11, 4096, 64, 0), (9, 8195, 0, 1), (9, 20000, 0, 0)])
def test_rows_in_8_bits(rows, width, pad, shift, dtype):
    torch, _ = _torch()
    rng = np.random.default_rng(rows + width)
    xv = _odd_rows(rng, rows, width, dtype)
    x, q = Matrix(rows, width, dtype, width + pad, shift, values=xv), Matrix(rows, width, "i8", width + pad, shift)
    scale = _words(np.full(rows + 1, -7), np.float32)
    P.opevo_quantize_rows_i8(x.ptr, x.ld, CODE[dtype], rows, width, q.ptr, q.ld, scale.data_ptr())
    got = q.host()
    assert scale[-1].item() == -7
    _check_rows_in_8_bits(xv, dtype, got, scale[:-1].cpu().numpy())


@gpu
@pytest.mark.parametrize("tokens,k,experts,width,dtype,held,pad,shift", ROUTES)
def test_dispatch_in_8_bits(tokens, k, experts, width, dtype, held, pad, shift):
    rng = np.random.default_rng(tokens * 41 + k)
    ids = _ids(rng, tokens, k, experts, held)
    xv = _odd_rows(rng, tokens, width, dtype)
    x, q = Matrix(tokens, width, dtype, width + pad, shift, values=xv), Matrix(tokens * k, width, "i8", width + pad, shift)
    scale = _words(np.full(tokens * k, -7), np.float32)
    offsets, row, _, _ = _dispatch(ids, experts, x, dtype, q, scale)
    got, s = q.host(), scale.cpu().numpy()
    held_at, has = int(offsets[-1]), row >= 0
    assert not got[held_at:].any() and not s[held_at:].any()
    token = np.empty(held_at, dtype=np.int64)
    token[row[has]] = np.nonzero(has)[0] // k
    _check_rows_in_8_bits(xv[token], dtype, got[:held_at], s[:held_at]) if held_at else None


def _check_product(got, a, b, sa, sb, dtype):
    exact = (a.astype(np.float64) @ b.astype(np.float64).T) * (sa.astype(np.float64)[:, None] * sb.astype(np.float64)[None, :])
    assert np.all(np.abs(got - exact) <= (3 * U + V[dtype] * (1 + 4 * U)) * np.abs(exact) + TINY[dtype]), np.abs(got - exact).max()


def _eight(rng, *shape):
    v = rng.integers(-127, 128, size=shape)
    v[rng.random(shape) < 0.02] = -128          # quantisers that use the whole range exist
    return v.astype(np.int8)


# M, N, K, output, extra between rows of a, b, c, shift
PRODUCTS = [
    (1, 1, 1, "f32", 0, 0, 0, 0), (1, 64, 64, "bf16", 0, 0, 0, 0), (1, 4096, 1024, "bf16", 0, 0, 0, 0), (1, 1000, 999, "f16", 0, 0, 0, 0), (2, 257, 4096, "f32", 0, 0, 0, 0),
    (3, 70, 129, "bf16", 5, 7, 3, 1), (4, 640, 16384, "f32", 0, 0, 0, 0), (5, 48, 16, "f16", 16, 32, 0, 0), (8, 1024, 512, "bf16", 0, 0, 0, 0), (13, 96, 100, "f32", 0, 0, 1, 0),
    (16, 512, 4096, "bf16", 0, 0, 0, 0), (17, 33, 65, "f16", 1, 1, 1, 1), (32, 1024, 4096, "f16", 0, 0, 0, 0), (33, 130, 272, "bf16", 0, 0, 0, 0), (48, 200, 2064, "f32", 0, 16, 0, 0),
    (64, 64, 128, "bf16", 0, 0, 0, 0), (100, 100, 100, "f32", 0, 0, 0, 0), (127, 129, 144, "bf16", 0, 0, 0, 0), (128, 256, 127, "f16", 0, 0, 0, 0), (129, 1000, 1008, "f32", 0, 0, 0, 0),
    (256, 256, 256, "bf16", 0, 0, 0, 0), (257, 300, 384, "f16", 0, 0, 4, 0), (333, 1001, 1000, "bf16", 0, 0, 0, 0), (512, 1024, 1024, "f32", 0, 0, 0, 0), (1000, 777, 640, "bf16", 16, 0, 1, 0),
    (300, 520, 16, "f32", 0, 0, 0, 0), (520, 300, 48, "bf16", 0, 0, 0, 0), (700, 900, 80, "f16", 0, 0, 0, 0), (16, 24, 131071, "f32", 0, 0, 0, 0), (260, 256, 131056, "f32", 0, 0, 0, 0),
]


@gpu
@pytest.mark.parametrize("M,N,K,dtype,pa,pb,pc,shift", PRODUCTS)
def test_products(M, N, K, dtype, pa, pb, pc, shift):
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    av, bv = _eight(rng, M, K), _eight(rng, N, K)
    sa, sb = (rng.random(M).astype(np.float32) + 0.1) * 1e-3, (rng.random(N).astype(np.float32) + 0.1) / (127 * np.sqrt(K).astype(np.float32))
    a, b, c = Matrix(M, K, "i8", K + pa, shift, values=av), Matrix(N, K, "i8", K + pb, shift, values=bv), Matrix(M, N, dtype, N + pc, shift)
    d_sa, d_sb = _words(sa, np.float32), _words(sb, np.float32)
    P.opevo_matmul_i8(a.ptr, a.ld, d_sa.data_ptr(), b.ptr, b.ld, d_sb.data_ptr(), c.ptr, c.ld, CODE[dtype], M, N, K)
    _check_product(c.host(), av, bv, sa, sb, dtype)


# M, N, K, output: sizes at which every kernel is the one chosen, with ragged tiles, K that ends inside a slab (multiples of 16 and others), one slab and many
LARGE = [
    (2700, 4300, 1040, "bf16"), (2691, 4374, 32, "f32"), (600, 3900, 1168, "f16"), (515, 2770, 144, "f32"), (1950, 2050, 1200, "bf16"), (2040, 2030, 1616, "f32"),
    (3272, 1052, 32, "bf16"), (700, 1900, 720, "f32"), (194, 3354, 32, "f16"), (900, 1000, 1040, "bf16"), (270, 523, 32, "f32"), (632, 520, 832, "bf16"),
    (1023, 325, 1808, "f32"), (453, 549, 1552, "f16"), (190, 250, 2000, "f32"), (150, 900, 1040, "bf16"), (9, 300, 1616, "f32"), (250, 100, 1616, "f16"),
    (2900, 4200, 1001, "bf16"), (1801, 2077, 1001, "f32"), (1801, 2077, 21, "f16"), (1500, 1100, 777, "bf16"), (477, 3836, 22, "f32"), (600, 900, 645, "f16"),
    (36, 4163, 20, "bf16"), (60, 450, 1111, "f32"), (70, 36, 1700, "bf16"), (95, 40, 279, "f32"), (12, 390, 1394, "f16"), (1, 52, 413, "bf16"),
    (1043, 1070, 1954, "bf16"), (637, 2395, 1019, "f32"), (41, 5798, 2903, "f16"), (960, 422, 2430, "f32"),
]


@gpu
@pytest.mark.parametrize("M,N,K,dtype", LARGE)
@pytest.mark.parametrize("pad", [0, 16, 3])
def test_large_products(M, N, K, dtype, pad):
    torch, _ = _torch()
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    a, b, c = Matrix(M, K, "i8", K + pad), Matrix(N, K, "i8", K + pad), Matrix(M, N, dtype, N + pad)
    for m in (a, b):
        m.view.copy_(torch.randint(-128, 128, (m.rows, K), generator=g, device="cuda", dtype=torch.int8))
    sa, sb = torch.rand(M, generator=g, device="cuda") * 1e-2, torch.rand(N, generator=g, device="cuda") * 1e-2
    P.opevo_matmul_i8(a.ptr, a.ld, sa.data_ptr(), b.ptr, b.ld, sb.data_ptr(), c.ptr, c.ld, CODE[dtype], M, N, K)
    exact = (torch.matmul(a.view.double(), b.view.double().t().contiguous()) * sa.double()[:, None] * sb.double()).cpu().numpy()
    assert np.all(np.abs(c.host() - exact) <= (3 * U + V[dtype] * (1 + 4 * U)) * np.abs(exact) + TINY[dtype])


@gpu
@pytest.mark.parametrize("M,N,K,ldb", [(1 << 21, 3, 16, 16), ((1 << 21) - 7, 40, 16, 16), (1100000, 2, 40, (1 << 24) + 16), (1100001, 5, 13, 13)])
def test_more_rows_than_a_grid_has_in_one_extent(M, N, K, ldb):
    torch, _ = _torch()
    g = torch.Generator(device="cuda").manual_seed(M + N)
    a, b, ones = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8), torch.randint(-128, 128, (N, ldb), generator=g, device="cuda", dtype=torch.int8), torch.ones(M, device="cuda")
    c = torch.full((M, N), float("nan"), device="cuda")
    P.opevo_matmul_i8(a.data_ptr(), K, ones.data_ptr(), b.data_ptr(), ldb, ones.data_ptr(), c.data_ptr(), N, P.OPEVO_F32, M, N, K)
    assert torch.equal(c, torch.matmul(a.float(), b[:, :K].float().t().contiguous()))


LARGE_GROUPS = [
    ([900, 0, 1411, 300, 2000, 77], 50, 2050, 400, "bf16"), ([300, 5, 0, 130], 3, 2200, 272, "f32"), ([700, 900, 0, 400], 60, 1700, 656, "f16"), ([128, 0, 260, 400], 11, 1300, 784, "f32"),
    ([100, 3, 300, 80], 9, 560, 416, "bf16"), ([40, 0, 90, 2], 4, 1980, 528, "f32"), ([200, 180, 200], 7, 560, 1104, "f16"), ([20, 0, 1, 40], 5, 300, 1040, "bf16"),
    ([300, 250], 20, 500, 784, "f32"), ([900, 0, 411, 500], 77, 1300, 501, "bf16"), ([300, 0, 900, 200], 20, 1300, 270, "f32"), ([150, 60, 200], 9, 700, 333, "f16"),
    ([410, 200, 0], 5, 573, 145, "f32"), ([20, 1, 0, 14], 2, 100, 275, "bf16"), ([100, 48], 9, 70, 900, "f32"), ([30, 1, 0, 9], 6, 60, 815, "bf16"),
    ([700, 0, 333, 41, 690], 22, 578, 1387, "f16"), ([500, 533, 0], 10, 365, 2361, "bf16"), ([121, 12], 5, 40, 543, "f32"), ([1541, 2101], 10, 1049, 305, "f16"), ([399, 203], 7, 776, 313, "f32"),
]


@gpu
@pytest.mark.parametrize("counts,none,N,K,dtype", LARGE_GROUPS)
def test_large_products_of_experts(counts, none, N, K, dtype):
    torch, _ = _torch()
    E, rows, g = len(counts), sum(counts) + none, torch.Generator(device="cuda").manual_seed(N + K)
    a, b, c = Matrix(rows, K, "i8"), Matrix(E * N, K, "i8"), Matrix(rows, N, dtype)
    for m in (a, b):
        m.view.copy_(torch.randint(-128, 128, (m.rows, K), generator=g, device="cuda", dtype=torch.int8))
    sa, sb = torch.rand(rows, generator=g, device="cuda") * 1e-2, torch.rand(E * N, generator=g, device="cuda") * 1e-2
    offsets = np.concatenate([[0], np.cumsum(counts)])
    sa[int(offsets[-1]):] = float("inf")
    d_off = _words(offsets, np.int32)
    P.opevo_matmul_i8_grouped(a.ptr, K, sa.data_ptr(), b.ptr, K, sb.data_ptr(), d_off.data_ptr(), E, c.ptr, N, CODE[dtype], rows, N, K)
    got = c.host()
    assert not got[offsets[-1]:].any()
    for e in range(E):
        part, own = slice(offsets[e], offsets[e + 1]), slice(e * N, (e + 1) * N)
        exact = (torch.matmul(a.view[part].double(), b.view[own].double().t().contiguous()) * sa[part].double()[:, None] * sb[own].double()).cpu().numpy()
        assert np.all(np.abs(got[part] - exact) <= (3 * U + V[dtype] * (1 + 4 * U)) * np.abs(exact) + TINY[dtype]), e


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(1, 500, 512), (40, 300, 200), (300, 700, 256)])
def test_16_bit_outputs_are_the_fp32_outputs_rounded(M, N, K, dtype):
    torch, types = _torch()
    rng = np.random.default_rng(M)
    a, b = Matrix(M, K, "i8", values=_eight(rng, M, K)), Matrix(N, K, "i8", values=_eight(rng, N, K))
    sa, sb = _words(rng.random(M) * 1e-3, np.float32), _words(rng.random(N) * 1e-2, np.float32)
    c, r = Matrix(M, N, "f32"), Matrix(M, N, dtype)
    P.opevo_matmul_i8(a.ptr, K, sa.data_ptr(), b.ptr, K, sb.data_ptr(), c.ptr, N, P.OPEVO_F32, M, N, K)
    P.opevo_matmul_i8(a.ptr, K, sa.data_ptr(), b.ptr, K, sb.data_ptr(), r.ptr, N, CODE[dtype], M, N, K)
    assert torch.equal(c.view.to(types[dtype]), r.view)


@gpu
def test_product_at_the_ends_of_its_range():
    """-128 * -128 * (2^17 - 1) fits; scales of zero, NaN and infinity go through."""
    torch, _ = _torch()
    for M, N, K in ((1, 3, 131071), (20, 70, 131056), (200, 300, 131056)):
        a, b = torch.full((M, K), -128, dtype=torch.int8, device="cuda"), torch.full((N, K), -128, dtype=torch.int8, device="cuda")
        sa, sb = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
        sa[0], sb[1], sb[2] = 0.0, float("nan"), float("inf")
        c = torch.empty(M, N, device="cuda")
        P.opevo_matmul_i8(a.data_ptr(), K, sa.data_ptr(), b.data_ptr(), K, sb.data_ptr(), c.data_ptr(), N, P.OPEVO_F32, M, N, K)
        want = torch.full((M, N), float(np.float32(16384.0 * K)))
        want[0] = 0.0
        want[:, 1], want[:, 2] = float("nan"), float("inf")
        want[0, 2] = float("nan")
        assert torch.equal(torch.nan_to_num(c.cpu(), nan=-1.0), torch.nan_to_num(want, nan=-1.0)), (M, N, K)


# rows of each expert, rows of none, N, K, output, extra between rows of a and b
GROUPS = [
    ([1], 0, 64, 64, "bf16", 0, 0), ([0, 0, 0], 4, 65, 64, "f32", 0, 0), ([0, 1, 0, 2], 0, 100, 48, "f16", 0, 0), ([3, 0, 5], 2, 33, 100, "bf16", 3, 1),
    ([1] * 64, 0, 256, 512, "f16", 0, 0), ([0] * 63 + [40], 24, 128, 1024, "bf16", 0, 0), ([70] + [0] * 64 + [1], 3, 96, 80, "f32", 0, 0),
    ([200, 3, 0, 333, 64], 100, 300, 256, "bf16", 0, 0), ([16] * 33, 0, 200, 2064, "f32", 0, 0), ([1000, 0, 24], 0, 520, 384, "bf16", 16, 0),
    ([128, 128, 256], 0, 256, 1024, "f16", 0, 0), ([129, 255, 257, 1], 7, 257, 144, "f32", 0, 0), ([2] * 1024, 5, 40, 32, "bf16", 0, 0),
    ([700, 1300, 50, 0, 2000], 46, 512, 272, "bf16", 0, 0), ([5, 9, 14, 0, 30], 6, 1000, 4096, "f16", 0, 0),
]


@gpu
@pytest.mark.parametrize("counts,none,N,K,dtype,pa,pb", GROUPS)
def test_products_of_experts(counts, none, N, K, dtype, pa, pb):
    rng = np.random.default_rng(sum(counts) + N + K)
    E, rows = len(counts), sum(counts) + none
    av, bv = _eight(rng, rows, K), _eight(rng, E * N, K)
    sa, sb = (rng.random(rows).astype(np.float32) + 0.1) * 1e-3, (rng.random(E * N).astype(np.float32) + 0.1) / (127 * np.sqrt(K).astype(np.float32))
    offsets = np.concatenate([[0], np.cumsum(counts)])
    sa[offsets[-1]:] = np.nan                   # rows of no expert become zeros, whatever they hold
    a, b, c = Matrix(rows, K, "i8", K + pa, values=av), Matrix(E * N, K, "i8", K + pb, values=bv), Matrix(rows, N, dtype)
    d_sa, d_sb, d_off = _words(sa, np.float32), _words(sb, np.float32), _words(offsets, np.int32)
    P.opevo_matmul_i8_grouped(a.ptr, a.ld, d_sa.data_ptr(), b.ptr, b.ld, d_sb.data_ptr(), d_off.data_ptr(), E, c.ptr, c.ld, CODE[dtype], rows, N, K)
    got = c.host()
    assert not got[offsets[-1]:].any()
    for e in range(E):
        part, own = slice(offsets[e], offsets[e + 1]), slice(e * N, (e + 1) * N)
        if counts[e]:
            _check_product(got[part], av[part], bv[own], sa[part], sb[own], dtype)


@gpu
def test_rows_more_than_32_bits_apart():
    """Every matrix with its last row beyond 2^32 bytes from its first."""
    torch, _ = _torch()
    far = (1 << 32) // 2 + 24
    tokens, k, width = 3, 1, 40
    x = torch.empty(2 * far + width, dtype=torch.int8, device="cuda")
    rows = torch.empty(2 * far + width, dtype=torch.int8, device="cuda")
    ids = _words([[1], [0], [2]], np.int32)
    ld = far // 2
    xs, rs = torch.as_strided(x.view(torch.bfloat16), (3, 20), (ld, 1)), torch.as_strided(rows.view(torch.bfloat16), (3, 20), (ld, 1))
    xs.copy_(torch.arange(60, device="cuda").reshape(3, 20))
    offsets, row = _words(np.zeros(4), np.int32), _words(np.zeros(3), np.int32)
    P.opevo_route_dispatch(ids.data_ptr(), 3, 1, 3, xs.data_ptr(), ld, P.OPEVO_BF16, 20, offsets.data_ptr(), row.data_ptr(), rs.data_ptr(), ld)
    assert torch.equal(rs[row.long()], xs)
    P.opevo_route_combine(rs.data_ptr(), ld, P.OPEVO_BF16, 0, row.data_ptr(), 3, 1, 20, xs.data_ptr(), ld)
    assert torch.equal(xs.float(), torch.arange(60, device="cuda").reshape(3, 20).float())
    sc = _words(np.zeros(3), np.float32)
    q = torch.as_strided(rows, (3, 20), (far, 1))
    P.opevo_quantize_rows_i8(xs.data_ptr(), ld, P.OPEVO_BF16, 3, 20, q.data_ptr(), far, sc.data_ptr())
    _check_rows_in_8_bits(xs.float().cpu().numpy(), "bf16", q.cpu().numpy().astype(np.float64), sc.cpu().numpy())
    a, b = torch.as_strided(x, (3, width), (far, 1)), torch.as_strided(rows, (3, width), (far, 1))
    rng = np.random.default_rng(3)
    av, bv = _eight(rng, 3, width), _eight(rng, 3, width)
    a.copy_(torch.from_numpy(av)), b.copy_(torch.from_numpy(bv))
    ones, c = torch.ones(3, device="cuda"), torch.empty(3, 3, device="cuda")
    P.opevo_matmul_i8(a.data_ptr(), far, ones.data_ptr(), b.data_ptr(), far, ones.data_ptr(), c.data_ptr(), 3, P.OPEVO_F32, 3, 3, width)
    assert torch.equal(c.cpu(), torch.from_numpy(av.astype(np.float32) @ bv.astype(np.float32).T))


@gpu
@pytest.mark.parametrize("ld", [1 << 24, (1 << 24) + 16, (1 << 24) - 1])
def test_products_of_many_rows_far_apart(ld):
    """Rows of a tile up to 2^32 bytes apart, and beyond that."""
    torch, _ = _torch()
    rng = np.random.default_rng(ld % 1000)
    M, N, K = 300, 270, 160
    av, bv = _eight(rng, M, K), _eight(rng, N, K)
    far_a, far_b = (torch.empty(n * ld + K, dtype=torch.int8, device="cuda") for n in (M - 1, N - 1))
    torch.as_strided(far_a, (M, K), (ld, 1)).copy_(torch.from_numpy(av))
    torch.as_strided(far_b, (N, K), (ld, 1)).copy_(torch.from_numpy(bv))
    near_b, ones, c = torch.from_numpy(bv).cuda(), torch.ones(M, device="cuda"), torch.empty(M, N, device="cuda")
    want = torch.from_numpy(av.astype(np.float32) @ bv.astype(np.float32).T)
    for b, ldb in ((far_b, ld), (near_b, K)):
        c.fill_(float("nan"))
        P.opevo_matmul_i8(far_a.data_ptr(), ld, ones.data_ptr(), b.data_ptr(), ldb, ones.data_ptr(), c.data_ptr(), N, P.OPEVO_F32, M, N, K)
        assert torch.equal(c.cpu(), want)


@gpu
def test_offsets_that_no_dispatch_writes_touch_nothing_outside():
    rng = np.random.default_rng(11)
    rows, N, K, E = 20, 40, 48, 3
    av, bv = _eight(rng, rows, K), _eight(rng, E * N, K)
    one, ones = _words(np.ones(rows), np.float32), _words(np.ones(E * N), np.float32)
    for offsets in ([0, -5, 30, 1000000], [2000000000, 7, -3, 12], [5, 5, 5, 5]):
        a, b, c = Matrix(rows, K, "i8", values=av), Matrix(E * N, K, "i8", values=bv), Matrix(rows, N, "f32", fill=3.0)
        d_off = _words(offsets, np.int32)
        P.opevo_matmul_i8_grouped(a.ptr, K, one.data_ptr(), b.ptr, K, ones.data_ptr(), d_off.data_ptr(), E, c.ptr, N, P.OPEVO_F32, rows, N, K)
        c.host()


@gpu
def test_an_empty_batch_writes_the_offsets_alone():
    offsets = _words(np.full(6, -7), np.int32)
    P.opevo_route_dispatch(0, 0, 2, 4, 0, 0, P.OPEVO_BF16, 0, offsets.data_ptr(), 0, 0, 0)
    assert offsets.cpu().tolist() == [0, 0, 0, 0, 0, -7]
    offsets.fill_(-7)
    P.opevo_route_dispatch_i8(0, 0, 2, 4, 0, 0, P.OPEVO_F16, 0, offsets.data_ptr(), 0, 0, 0, 0)
    assert offsets.cpu().tolist() == [0, 0, 0, 0, 0, -7]


@gpu
def test_layer_in_a_graph_and_on_another_stream():
    """The whole serving path recorded once and replayed on new inputs, eager work between the replays; the same on a stream of its own."""
    torch, _ = _torch()
    tokens, k, E, H, F = 700, 8, 6, 256, 192
    torch.manual_seed(1)
    ids, x = torch.empty(tokens, k, dtype=torch.int32, device="cuda"), torch.empty(tokens, H, dtype=torch.bfloat16, device="cuda")
    w = torch.randint(-127, 128, (E, F, H), dtype=torch.int8, device="cuda")
    sw, weight = torch.rand(E, F, device="cuda"), torch.rand(tokens, k, device="cuda")
    size = P.opevo_route_workspace(tokens, k, E)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def buffers():
        return dict(off=torch.empty(E + 1, dtype=torch.int32, device="cuda"), row=torch.empty(tokens * k, dtype=torch.int32, device="cuda"),
                    q=torch.empty(tokens * k, H, dtype=torch.int8, device="cuda"), s=torch.empty(tokens * k, device="cuda"),
                    h=torch.empty(tokens * k, F, dtype=torch.bfloat16, device="cuda"), y=torch.empty(tokens, F, dtype=torch.bfloat16, device="cuda"))

    def layer(o):
        stream = torch.cuda.current_stream().cuda_stream
        P.opevo_route_dispatch_i8(ids.data_ptr(), tokens, k, E, x.data_ptr(), H, P.OPEVO_BF16, H, o["off"].data_ptr(), o["row"].data_ptr(), o["q"].data_ptr(), H,
                                  o["s"].data_ptr(), ws.data_ptr(), size, stream)
        P.opevo_matmul_i8_grouped(o["q"].data_ptr(), H, o["s"].data_ptr(), w.data_ptr(), H, sw.data_ptr(), o["off"].data_ptr(), E, o["h"].data_ptr(), F, P.OPEVO_BF16,
                                  tokens * k, F, H, stream)
        P.opevo_route_combine(o["h"].data_ptr(), F, P.OPEVO_BF16, weight.data_ptr(), o["row"].data_ptr(), tokens, k, F, o["y"].data_ptr(), F, stream)

    def fill(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        ids.copy_(torch.randint(-1, E + 1, ids.shape, generator=g, device="cuda", dtype=torch.int32))
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))

    eager, recorded = buffers(), buffers()
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(recorded)
    torch.cuda.current_stream().wait_stream(side)
    layer(eager)
    torch.cuda.synchronize()
    for name in eager:
        assert torch.equal(eager[name], recorded[name]), name
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(recorded)
    for seed in range(1, 5):
        fill(seed)
        graph.replay()
        layer(eager)
        torch.cuda.synchronize()
        for name in eager:
            assert torch.equal(eager[name], recorded[name]), (seed, name)


@gpu
def test_example_layer():
    """The example's layer against 64 bits.  Trained: sums of at most 1024 fp32 products of either sign, far below 1e-4.  Served: tokens, hidden values and both weights are
    rounded to 127 steps of their row's largest, about 3.5 to 4.5 standard deviations of normal values (a step of 0.035, off by 0.035 / sqrt 12 = 1 % each), and the hidden rows, half of
    them zeros, alike: two factors a product and two products, sqrt 4 * 1 % = 2 %, twice that allowed."""
    _torch()
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "expert_layer.py")
    spec = importlib.util.spec_from_file_location("expert_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    for name, error in example.main(tokens=300, k=3, experts=7, width=256, inner=520).items():
        assert error <= (4e-2 if name.startswith("served") else 1e-4), (name, error)


def _refused(text, call, *args):
    with pytest.raises(P.OpevoError) as e:
        call(*args)
    assert e.value.status == P.OPEVO_E_ARG and text in e.value.message, e.value.message


def test_refusals():
    """Wrong arguments come back as errors before anything is launched (the pointers are never followed)."""
    p, odd = 0x10000, 0x10001
    ok = dict(expert=p, tokens=8, k=2, experts=4, x=p, ld_x=32, dtype=P.OPEVO_BF16, width=32, offsets=p, row_of_slot=p, rows=p, ld_rows=32)
    bad = [("tokens", dict(tokens=-1)), ("slots", dict(k=0)), ("slots", dict(k=65)), ("fewer than", dict(tokens=1 << 30)), ("experts", dict(experts=0)),
           ("experts", dict(experts=1025)), ("type", dict(dtype=9)), ("expert is NULL", dict(expert=0)), ("offsets", dict(offsets=p + 2)), ("row_of_slot", dict(row_of_slot=0)),
           ("x is NULL", dict(x=0)), ("x is not aligned", dict(x=odd)), ("rows is NULL", dict(rows=0)), ("rows of x are 31", dict(ld_x=31)),
           ("rows of rows are 5", dict(ld_rows=5)), ("0 elements", dict(width=0)), ("elements", dict(width=(1 << 24) + 1, ld_x=1 << 25, ld_rows=1 << 25)),
           ("workspace", dict(tokens=1 << 20))]
    for text, change in bad:
        _refused(text, P.opevo_route_dispatch, *{**ok, **change}.values())
    ok8 = {**{n: v for n, v in ok.items() if n not in ("rows", "ld_rows")}, "q": p, "ld_q": 32, "scale": p}
    for text, change in [("q is NULL", dict(q=0)), ("rows of q", dict(ld_q=31)), ("scale", dict(scale=2)), ("type", dict(dtype=-1)), ("workspace", dict(tokens=1 << 20))]:
        _refused(text, P.opevo_route_dispatch_i8, *{**ok8, **change}.values())
    okc = dict(rows=p, ld_rows=8, dtype=P.OPEVO_F32, weight=p, row_of_slot=p, tokens=4, k=2, width=8, y=p, ld_y=8)
    for text, change in [("rows is NULL", dict(rows=0)), ("rows is not aligned", dict(rows=p + 2)), ("weight", dict(weight=p + 1)), ("row_of_slot", dict(row_of_slot=0)),
                         ("y is NULL", dict(y=0)), ("rows of y", dict(ld_y=7)), ("type", dict(dtype=3)), ("slots", dict(k=100))]:
        _refused(text, P.opevo_route_combine, *{**okc, **change}.values())
    okg = dict(dy=p, ld_dy=8, rows=p, ld_rows=8, dtype=P.OPEVO_F32, weight=p, row_of_slot=p, offsets=p, experts=2, tokens=4, k=2, width=8, drows=p, ld_drows=8, dweight=p)
    for text, change in [("dy is NULL", dict(dy=0)), ("rows is NULL", dict(rows=0)), ("drows", dict(drows=0)), ("weight", dict(weight=0)), ("dweight", dict(dweight=0)),
                         ("offsets", dict(offsets=0)), ("experts", dict(experts=0)), ("rows of drows", dict(ld_drows=1))]:
        _refused(text, P.opevo_route_combine_grad, *{**okg, **change}.values())
    okq = dict(x=p, ld_x=8, dtype=P.OPEVO_F16, rows=3, width=8, q=p, ld_q=8, scale=p)
    for text, change in [("x is NULL", dict(x=0)), ("x is not aligned", dict(x=odd)), ("q is NULL", dict(q=0)), ("scale", dict(scale=0)), ("-1 rows", dict(rows=-1)),
                         ("rows of q", dict(ld_q=7)), ("type", dict(dtype=5))]:
        _refused(text, P.opevo_quantize_rows_i8, *{**okq, **change}.values())
    okm = dict(a=p, lda=8, scale_a=p, b=p, ldb=8, scale_b=p, c=p, ldc=4, out_dtype=P.OPEVO_F32, M=2, N=4, K=8)
    bad = [("a is NULL", dict(a=0)), ("b is NULL", dict(b=0)), ("c is NULL", dict(c=0)), ("c is NULL or not aligned", dict(c=p + 2)), ("scale_a", dict(scale_a=0)),
           ("scale_b", dict(scale_b=p + 1)), ("rows of a", dict(lda=7)), ("rows of b", dict(ldb=7)), ("rows of c", dict(ldc=3)), ("output type", dict(out_dtype=7)),
           ("K = 0", dict(K=0)), ("2^17", dict(K=1 << 17, lda=1 << 17, ldb=1 << 17)), ("-1 rows", dict(M=-1)), ("rows", dict(M=(1 << 21) + 1))]
    for text, change in bad:
        _refused(text, P.opevo_matmul_i8, *{**okm, **change}.values())
    okm = dict(a=p, lda=8, scale_a=p, b=p, ldb=8, scale_b=p, offsets=p, experts=2, c=p, ldc=4, out_dtype=P.OPEVO_F32, rows=2, N=4, K=8)
    for text, change in [("offsets", dict(offsets=0)), ("experts", dict(experts=0)), ("experts", dict(experts=1025)), ("b is NULL", dict(b=0)), ("K = 0", dict(K=0))]:
        _refused(text, P.opevo_matmul_i8_grouped, *{**okm, **change}.values())
    _refused("bytes", lambda: P.binding._check(P.binding.lib.opevo_route_workspace(1, 1, 1, None)))


def test_empty_extents_and_workspaces_need_no_gpu():
    P.opevo_matmul_i8(0, 8, 0, 0, 8, 0, 0, 4, P.OPEVO_F32, 0, 4, 8)
    P.opevo_matmul_i8(0, 8, 0, 0, 8, 0, 0, 4, P.OPEVO_F32, 3, 0, 8)
    P.opevo_matmul_i8_grouped(0, 8, 0, 0, 8, 0, 0, 2, 0, 4, P.OPEVO_F32, 0, 4, 8)
    P.opevo_quantize_rows_i8(0, 8, P.OPEVO_F32, 0, 8, 0, 8, 0)
    P.opevo_route_combine(0, 8, P.OPEVO_F32, 0, 0, 0, 2, 8, 0, 8)
    assert P.opevo_route_workspace(0, 1, 1) == 0 and P.opevo_route_workspace(16, 2, 8) == 0
    for tokens, k, experts in ((16384, 2, 64), (100000, 8, 1024), (4097, 1, 3)):
        size = P.opevo_route_workspace(tokens, k, experts)
        assert 0 < size <= 4 * experts * (tokens * k // 256 + 1) and size % (4 * experts) == 0
