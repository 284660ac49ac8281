"""More workgroups than a launch takes along one extent of its grid (2^32 threads; beyond that it runs some of them and reports no error): 2^24 tokens of rows that a workgroup takes one by one, 2^30 slots, 2^26 short rows."""
import pytest

import paper_2006_05664_amd as P

pytestmark = pytest.mark.gpu
BF16, F32 = P.OPEVO_BF16, P.OPEVO_F32


@pytest.fixture
def torch():
    import torch
    assert torch.cuda.is_available()
    yield torch
    torch.cuda.synchronize()
    torch.cuda.empty_cache()            # tens of GB


def _same(torch, what, a, b):
    same = torch.equal(a, b)
    assert same, what                   # the tensors themselves are too large to print


def _nonzero_rows(torch, m, expected):
    """Which rows of a large matrix hold anything but zeros (NaN counts)."""
    found = torch.cat([torch.nonzero((part != 0).any(dim=1))[:, 0] + at for at, part in zip(range(0, m.shape[0], 1 << 22), m.split(1 << 22))])
    assert len(found) == len(expected) and found.tolist() == sorted(expected), (len(found), found[:20].tolist())


def test_combine_and_its_gradients(torch):
    tokens, width = (1 << 24) + 5, 1025
    held = [0, 1, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, (1 << 24) - 1, 1 << 24, tokens - 1]
    row_of_slot = torch.full((tokens,), -1, dtype=torch.int32, device="cuda")
    row_of_slot[held] = torch.arange(len(held), dtype=torch.int32, device="cuda")
    weight = torch.full((tokens,), 2.0, device="cuda")
    rows, out = (torch.empty(tokens, width, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows[:len(held)] = torch.randint(1, 8, (len(held), width), device="cuda").bfloat16()
    out.fill_(float("nan"))
    P.opevo_route_combine(rows.data_ptr(), width, BF16, weight.data_ptr(), row_of_slot.data_ptr(), tokens, 1, width, out.data_ptr(), width)
    _nonzero_rows(torch, out, held)
    _same(torch, "y", out[held], 2 * rows[:len(held)])

    dy = torch.empty(tokens, width, dtype=torch.bfloat16, device="cuda")
    dy[held] = torch.randint(1, 8, (len(held), width), device="cuda").bfloat16()
    offsets = torch.tensor([0, len(held)], dtype=torch.int32, device="cuda")
    dweight = torch.full((tokens,), float("nan"), device="cuda")
    out.fill_(float("nan"))
    P.opevo_route_combine_grad(dy.data_ptr(), width, rows.data_ptr(), width, BF16, weight.data_ptr(), row_of_slot.data_ptr(), offsets.data_ptr(), 1, tokens, 1, width,
                               out.data_ptr(), width, dweight.data_ptr())
    _nonzero_rows(torch, out, range(len(held)))
    _same(torch, "drows", out[:len(held)], 2 * dy[held])
    want = torch.zeros(tokens, device="cuda")
    want[held] = (dy[held].float() * rows[:len(held)].float()).sum(1)       # sums of whole numbers below 2^24: exact
    _same(torch, "dweight", dweight, want)


def test_rows_in_8_bits(torch):
    rows, width = (1 << 26) + 3, 129
    some = [0, 5, (1 << 25) - 1, 1 << 25, (1 << 26) - 1, 1 << 26, rows - 1]
    x, q, scale = torch.zeros(rows, width, device="cuda"), torch.full((rows, width), 77, dtype=torch.int8, device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    values = torch.randint(-126, 127, (len(some), width), device="cuda")
    values[:, 0] = 127
    x[some] = values.float()
    P.opevo_quantize_rows_i8(x.data_ptr(), width, F32, rows, width, q.data_ptr(), width, scale.data_ptr())
    _same(torch, "q", q[some].long(), values)
    q[some] = 1
    _nonzero_rows(torch, q, some)
    want = torch.zeros(rows, device="cuda")
    want[some] = 1.0
    _same(torch, "scale", scale, want)


@pytest.mark.parametrize("in_8_bits", [False, True])
def test_dispatch(torch, in_8_bits):
    tokens, k, experts, width = (1 << 24) + 3, 64, 3, 1
    slots, part = tokens * k, 1 << 26
    g = torch.Generator(device="cuda").manual_seed(7)
    ids = torch.randint(-1, experts + 1, (slots,), generator=g, device="cuda", dtype=torch.int32)
    x = torch.randint(1, 100, (tokens, width), generator=g, device="cuda").bfloat16()
    offsets, row = torch.full((experts + 2,), -7, dtype=torch.int32, device="cuda"), torch.full((slots + 1,), -7, dtype=torch.int32, device="cuda")
    size = P.opevo_route_workspace(tokens, k, experts)
    ws = torch.full((size + 64,), 255, dtype=torch.uint8, device="cuda")
    common = (ids.data_ptr(), tokens, k, experts, x.data_ptr(), width, BF16, width, offsets.data_ptr(), row.data_ptr())
    if in_8_bits:
        rows, scale = torch.full((slots, width), 77, dtype=torch.int8, device="cuda"), torch.full((slots,), -7.0, device="cuda")
        P.opevo_route_dispatch_i8(*common, rows.data_ptr(), width, scale.data_ptr(), ws.data_ptr(), size)
    else:
        rows = torch.full((slots, width), -7.0, dtype=torch.bfloat16, device="cuda")
        P.opevo_route_dispatch(*common, rows.data_ptr(), width, ws.data_ptr(), size)
    want = [0]
    for e in range(experts):
        want.append(want[-1] + sum(int((p == e).sum()) for p in ids.split(part)))
    assert offsets.tolist() == want + [-7] and row[-1].item() == -7 and bool((ws[size:] == 255).all())
    run = want[:experts]
    scales = torch.arange(100, dtype=torch.float32).div(torch.tensor(127.0)).cuda()      # divided on the host, where a quotient is rounded once
    for at in range(0, slots, part):                        # the definition, a part of the slots at a time
        p, r = ids[at:at + part], row[:-1][at:at + part]
        expected = torch.full_like(p, -1)
        for e in range(experts):
            mine = p == e
            upto = torch.cumsum(mine, 0, dtype=torch.int32)
            expected = torch.where(mine, run[e] + upto - 1, expected)
            run[e] += int(upto[-1])
        _same(torch, "row_of_slot from %d" % at, r, expected)
        has = torch.nonzero(r >= 0)[:, 0]
        to, token = r[has].long(), (has + at) // k
        if in_8_bits:
            _same(torch, "q", rows[to, 0], torch.full_like(rows[to, 0], 127))
            _same(torch, "scale", scale[to], scales[x[token, 0].long()])
        else:
            _same(torch, "rows", rows[to, 0], x[token, 0])
    left = bool(rows[want[-1]:].any()) or (in_8_bits and bool(scale[want[-1]:].any()))
    assert not left, "rows of no slot"
