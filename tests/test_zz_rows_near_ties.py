"""fp32 rows to 8 bits next to ties: 127 x and its quotient by the row's largest are rounded to fp32, each by at most 2^-24 of its value, so the quotient whose rounding q is
is right to 2^-23 (and 2^-48), not to 2^-24.  The kernel multiplies where that cannot change the integer and divides elsewhere: the result has to be the division's everywhere."""
import numpy as np
import pytest

import paper_2006_05664_amd as P


def _near_ties(rng, largest, width):
    """A row with this largest magnitude, whose other values lie within a few ulps of a tie."""
    tie = (rng.integers(0, 127, width) + 0.5) * np.where(rng.random(width) < 0.5, 1, -1)
    x = (tie * float(largest) / 127.0).astype(np.float32)
    x = (x.view(np.int32) + rng.integers(-3, 4, width).astype(np.int32)).view(np.float32)
    x[rng.integers(0, width)] = largest
    return x


def _two_roundings(x, largest):
    """127 x / largest in fp32 arithmetic (scaled by a power of two, so that neither overflows nor is subnormal), and the integer next to it."""
    pre = np.float32(2.0 ** -7 if largest > 1e30 else 2.0 ** 96 if largest < 1e-30 else 1.0)
    return np.rint(np.float32(127.0) * (x * pre) / (largest * pre))


def _rows(rng):
    largest = np.array([1.0, 127.0, 3.7, 0.99999994, 1.0000001, 1e-3, 54321.0, 2.9e35, 3e-36] + list(rng.random(247) * 100 + 0.01), dtype=np.float32)
    return largest, np.stack([_near_ties(rng, a, 4096) for a in largest])


def _check(largest, x, q):
    exact = 127.0 * x.astype(np.float64) / largest.astype(np.float64)[:, None]          # 64 bits: 29 more than the bound asks for
    assert np.array_equal(q, np.stack([_two_roundings(r, a) for r, a in zip(x, largest)]))
    assert np.all(np.abs(q - exact) <= 0.5 + np.abs(exact) * 2.0 ** -23 * (1 + 2.0 ** -20))
    return np.count_nonzero(np.abs(q - exact) > 0.5 + np.abs(exact) * 2.0 ** -24 * (1 + 2.0 ** -20))


def test_two_roundings_are_right_to_2_to_the_minus_23_and_no_better():
    largest, x = _rows(np.random.default_rng(3))
    assert _check(largest, x, np.stack([_two_roundings(r, a) for r, a in zip(x, largest)])) > 0


def test_the_promise_is_the_one_that_is_kept():
    """The header says how exact the quotient is."""
    import os
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "opevo.h")).read()
    text = " ".join(text.replace("*", " ").split())
    assert "for fp32 inputs that of a quotient right to 2^-23 of its value" in text


@pytest.mark.gpu
def test_rows_next_to_ties():
    import torch
    assert torch.cuda.is_available()
    largest, xv = _rows(np.random.default_rng(3))
    rows, width = xv.shape
    x, q, scale = torch.from_numpy(xv).cuda(), torch.full((rows, width), 77, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    P.opevo_quantize_rows_i8(x.data_ptr(), width, P.OPEVO_F32, rows, width, q.data_ptr(), width, scale.data_ptr())
    assert _check(largest, xv, q.cpu().numpy().astype(np.float64)) > 0
    assert np.array_equal(scale.cpu().numpy(), largest / np.float32(127.0))
