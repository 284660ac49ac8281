"""What a layer of experts for few tokens keeps of its numbers: h as it is, in 32 bits, whatever the callers' type.

Two inner channels have the same gate row and up rows of 3 and 4, and an output channel takes them with 4 and -3: with h in 32 bits what comes out is the noise of a few roundings of
h, without them it would be zero.  u = 2^-24, S = |4 h0| + |3 h1|: the gate is the same number for both, each of U and h has up to three roundings and the parts' sums (of x for fp16 and fp32) two, their
difference meets in at most four sums: |y| <= 12 u S, and half an ulp of it in the output's type.  (h in two bf16 numbers, with 2^-17 of its value lost at the most, gives up to 128 u S.)"""
import numpy as np
import pytest

import paper_2006_05664_amd as P
import test_zz_expert_layer as L
from test_zz_experts import CODE, TINY, U, V, Matrix, _activations, _torch, _words, gpu
from test_zz_mx4 import VALUES, Bytes, _pack

class Rows:
    """Rows of small whole numbers as weights of either kind, as they are."""

    def __init__(self, values, kind):
        torch, _ = _torch()
        self.kind, (rows, K) = kind, values.shape
        if kind == "i8":
            self.q = Matrix(rows, K, "i8", values=values.astype(np.int8))
            self.scale = torch.ones(rows, device="cuda")
            self.args = (self.q.ptr, K, self.scale.data_ptr())
        else:
            code = np.searchsorted(VALUES[:8], np.abs(values)) | np.where(values < 0, 8, 0)
            assert np.array_equal(VALUES[code], values)
            self.q = Bytes(rows, (K + 1) // 2, values=_pack(code.astype(np.uint8)))
            self.f = Bytes(rows, -(-K // 32), values=np.full((rows, -(-K // 32)), 127, dtype=np.uint8))
            self.args = (self.q.ptr, self.q.ld, self.f.ptr, self.f.ld)

# tokens, k, experts, width, inner: each way of the second launch; rows of one expert in one unit and in several
@gpu
@pytest.mark.parametrize("kind", ["i8", "mx4"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,k,experts,width,inner", [(1, 2, 8, 1024, 1024), (40, 2, 3, 256, 512), (9, 3, 4, 130, 130), (64, 4, 5, 1500, 256), (100, 2, 2, 2064, 300), (30, 1, 2, 40, 12), (20, 2, 3, 2050, 1024)])
def test_h_is_kept_in_32_bits(tokens, k, experts, width, inner, dtype, kind):
    torch, _ = _torch()
    rng = np.random.default_rng(tokens + width + inner)
    win, wout = np.zeros((experts, 2, inner, width)), np.zeros((experts, width, inner))
    win[:, 0, :, 0] = 1
    win[:, 1, 0::2, 0], win[:, 1, 1::2, 0] = 3, 4
    pair = rng.integers(0, inner // 2, (experts, width))
    np.put_along_axis(wout, 2 * pair[:, :, None], 4, axis=2)
    np.put_along_axis(wout, 2 * pair[:, :, None] + 1, -3, axis=2)
    win, wout = Rows(win.reshape(-1, width), kind), Rows(wout.reshape(-1, inner), kind)
    xv = _activations(rng, tokens, width, dtype)
    x, y = Matrix(tokens, width, dtype, values=xv), Matrix(tokens, width, dtype)
    ids = np.argsort(rng.random((tokens, experts)), axis=1)[:, :k]
    size = P.opevo_expert_layer_workspace(tokens, k, CODE[dtype], inner)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    L._call(kind, x, dtype, _words(ids, np.int32), None, tokens, k, experts, width, inner, win, wout, y, ws, size)
    first = xv[:, :1].astype(np.float64)
    most = k * 24 * np.abs(first / (1 + np.exp(-first)) * first)
    assert np.all(np.abs(y.host()) <= 12 * U * most * (1 + V[dtype]) + TINY[dtype]), (np.abs(y.host()) / (U * most)).max()
