"""Factors of microscaled 4-bit products at every place that the kernels of long rows take them from: rows and bases that are multiples of 4 bytes and not of 16, where the codes are multiples of 16."""
import numpy as np
import pytest

import paper_2006_05664_amd as P
import test_zz_mx4 as X
import test_zz_mx4_ways as W
from test_zz_experts import CODE, Matrix, _torch, _words, gpu

# M, N, K: the three kernels
PLAIN = [(2949, 3460, 2048), (2048, 2048, 2048), (1361, 1531, 2048)]
# rows of each expert, rows of none, N, K
GROUPS = [([2300, 4000], 540, 1716, 2048), ([170, 305], 4, 3479, 1024), ([0, 185, 300], 4, 1848, 1024)]
AT = [(4, 0), (8, 4), (12, 8), (0, 12), (16, 4)]            # bytes between rows of factors, and in front of the first


def test_each_kernel_of_long_rows_is_chosen(tmp_path):
    lib, kernels = W._chooser(tmp_path)
    long = {k for _, k in kernels if k // 100000000 == 2}
    assert len(long) == 3
    for pad in sorted({pad for pad, _ in AT}):
        assert {lib.pick(M, N, K, K // 2, K // 2, K // 32 + pad, K // 32 + pad, 0) for M, N, K in PLAIN} == long
        assert {lib.pick(sum(counts) + none, N, K, K // 2, K // 2, K // 32 + pad, K // 32 + pad, len(counts)) for counts, none, N, K in GROUPS} == long


def _factors(g, rows, K, pad, shift):
    torch, _ = _torch()
    q, _, _ = X._operand(g, rows, K)
    b = X.Bytes(rows, K // 32, K // 32 + pad, shift, values=torch.randint(126, 129, (rows, K // 32), generator=g, device="cuda", dtype=torch.uint8))
    code = torch.stack([q.view & 15, q.view >> 4], dim=2).reshape(rows, -1).long()
    return q, b, torch.from_numpy(X.VALUES).cuda()[code] * torch.exp2(b.view.double() - 127).repeat_interleave(32, 1)


@gpu
@pytest.mark.parametrize("pad,shift", AT)
@pytest.mark.parametrize("M,N,K", PLAIN)
def test_products(M, N, K, pad, shift):
    torch, _ = _torch()
    g = torch.Generator(device="cuda").manual_seed(M + pad)
    (a, fa, av), (b, fb, bv) = _factors(g, M, K, pad, shift), _factors(g, N, K, pad, shift)
    c = Matrix(M, N, "bf16")
    P.opevo_matmul_mx4(a.ptr, a.ld, fa.ptr, fa.ld, b.ptr, b.ld, fb.ptr, fb.ld, c.ptr, c.ld, CODE["bf16"], M, N, K)
    X._check(c.host(), X._product(av, bv)[0], "bf16")


@gpu
@pytest.mark.parametrize("pad,shift", AT)
@pytest.mark.parametrize("counts,none,N,K", GROUPS)
def test_products_of_experts(counts, none, N, K, pad, shift):
    torch, _ = _torch()
    E, rows, g = len(counts), sum(counts) + none, torch.Generator(device="cuda").manual_seed(N + pad)
    (a, fa, av), (b, fb, bv) = _factors(g, rows, K, pad, shift), _factors(g, E * N, K, pad, shift)
    offsets = np.concatenate([[0], np.cumsum(counts)])
    c, d_off = Matrix(rows, N, "f32"), _words(offsets, np.int32)
    P.opevo_matmul_mx4_grouped(a.ptr, a.ld, fa.ptr, fa.ld, b.ptr, b.ld, fb.ptr, fb.ld, d_off.data_ptr(), E, c.ptr, N, CODE["f32"], rows, N, K)
    got = c.host()
    assert not got[offsets[-1]:].any()
    for e in range(E):
        part, own = slice(offsets[e], offsets[e + 1]), slice(e * N, (e + 1) * N)
        if counts[e]:
            X._check(got[part], X._product(av[part], bv[own])[0], "f32")
