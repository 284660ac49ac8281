"""A call answers for its own launches: an error that another call of the thread has left with the runtime is neither reported as its own nor taken away."""
import numpy as np
import pytest

import paper_2006_05664_amd as P

HIP_SUCCESS, HIP_ERROR_INVALID_DEVICE = 0, 101


@pytest.mark.gpu
def test_an_error_of_another_call_is_not_this_one_s():
    import torch
    assert torch.cuda.is_available()
    hip = P.binding.lib                         # the runtime that the library is bound to
    tokens, k, experts, width = 2100, 2, 3, 16  # more slots than are counted in one launch
    ids = torch.arange(tokens * k, device="cuda", dtype=torch.int32) % experts
    x = torch.randn(tokens, width, device="cuda")
    offsets, row = torch.empty(experts + 1, dtype=torch.int32, device="cuda"), torch.empty(tokens * k, dtype=torch.int32, device="cuda")
    size = P.opevo_route_workspace(tokens, k, experts)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    rows, y = torch.empty(tokens * k, width, device="cuda"), torch.empty(tokens, width, device="cuda")
    q, scale = torch.empty(tokens * k, width, dtype=torch.int8, device="cuda"), torch.empty(tokens * k, device="cuda")
    w, sw, c = torch.ones(experts, 8, width, dtype=torch.int8, device="cuda"), torch.ones(experts, 8, device="cuda"), torch.empty(tokens * k, 8, device="cuda")
    weight, dweight, drows = torch.ones(tokens * k, device="cuda"), torch.empty(tokens * k, device="cuda"), torch.empty(tokens * k, width, device="cuda")
    torch.cuda.synchronize()
    f32 = P.OPEVO_F32
    route = (ids.data_ptr(), tokens, k, experts, x.data_ptr(), width, f32, width, offsets.data_ptr(), row.data_ptr())
    calls = [
        (P.opevo_route_dispatch, *route, rows.data_ptr(), width, ws.data_ptr(), size),
        (P.opevo_route_dispatch_i8, *route, q.data_ptr(), width, scale.data_ptr(), ws.data_ptr(), size),
        (P.opevo_route_combine, rows.data_ptr(), width, f32, 0, row.data_ptr(), tokens, k, width, y.data_ptr(), width),
        (P.opevo_route_combine_grad, x.data_ptr(), width, rows.data_ptr(), width, f32, weight.data_ptr(), row.data_ptr(), offsets.data_ptr(), experts, tokens, k, width,
         drows.data_ptr(), width, dweight.data_ptr()),
        (P.opevo_quantize_rows_i8, x.data_ptr(), width, f32, tokens, width, q.data_ptr(), width, scale.data_ptr()),
        (P.opevo_matmul_i8, q.data_ptr(), width, scale.data_ptr(), w.data_ptr(), width, sw.data_ptr(), c.data_ptr(), 8, f32, 1, 8, width),
        (P.opevo_matmul_i8, q.data_ptr(), width, scale.data_ptr(), w.data_ptr(), width, sw.data_ptr(), c.data_ptr(), 8, f32, tokens, 8, width),
        (P.opevo_matmul_i8_grouped, q.data_ptr(), width, scale.data_ptr(), w.data_ptr(), width, sw.data_ptr(), offsets.data_ptr(), experts, c.data_ptr(), 8, f32, tokens * k, 8, width),
    ]
    failed = []
    for call, *args in calls:
        assert hip.hipSetDevice(1 << 20) == HIP_ERROR_INVALID_DEVICE          # refused by the runtime, which keeps the error for who asks next
        try:
            call(*args)
        except P.OpevoError as e:
            failed.append((call.__name__, str(e)))
        finally:
            left = hip.hipGetLastError()
        if left != HIP_ERROR_INVALID_DEVICE:
            failed.append((call.__name__, "took the error away", left))
    assert hip.hipGetLastError() == HIP_SUCCESS
    torch.cuda.synchronize()
    assert failed == []
    assert np.array_equal(offsets.cpu().numpy(), [0, 1400, 2800, 4200])       # the calls ran
    assert torch.equal(y, x * k)
