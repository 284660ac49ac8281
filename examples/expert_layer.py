"""A layer of experts: two projections with a ReLU between them, every token through k of E experts.

`ExpertLayer.serve` runs in 8-bit integers: tokens are sorted by expert and quantised on the way (opevo_route_dispatch_i8), both projections are
products of 8-bit integers by expert (opevo_matmul_i8_grouped), and the rows come back with the router's weights (opevo_route_combine).
`ExpertLayer.train` is the same layer in the weights' own precision with its gradients: opevo_route_dispatch, the experts' products by torch,
opevo_route_combine, opevo_route_combine_grad, and opevo_route_combine without weights for the gradient of the tokens.

    python examples/expert_layer.py            # one pass of each, compared with the layer in 64 bits
"""
from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2006_05664_amd as P  # noqa: E402

_CODE = {torch.float32: P.OPEVO_F32, torch.bfloat16: P.OPEVO_BF16, torch.float16: P.OPEVO_F16}


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _expect(name: str, t: torch.Tensor, shape, dtypes, device) -> None:
    """The library is given pointers: what they point to has to be what it takes them for."""
    if tuple(t.shape) != tuple(shape) or t.dtype not in dtypes or t.device != device or not t.is_contiguous():
        raise ValueError("%s: %s of shape %s on %s%s, not contiguous %s of shape %s on %s" % (
            name, t.dtype, tuple(t.shape), t.device, "" if t.is_contiguous() else ", strided", " / ".join(str(d) for d in dtypes), tuple(shape), device))


def quantize(x: torch.Tensor):
    """Rows of a contiguous matrix in 8 bits and their scales."""
    rows, width = x.shape
    q, scale = torch.empty(rows, width, dtype=torch.int8, device=x.device), torch.empty(rows, device=x.device)
    P.opevo_quantize_rows_i8(x.data_ptr(), width, _CODE[x.dtype], rows, width, q.data_ptr(), width, scale.data_ptr(), _stream())
    return q, scale


class ExpertLayer:
    """up [E, F, H] and down [E, H, F]: an output channel a row, as torch.nn.Linear stores its weights."""

    def __init__(self, up: torch.Tensor, down: torch.Tensor):
        self.experts, self.inner, self.width = up.shape
        self.up, self.down = up.contiguous(), down.contiguous()
        _expect("up", self.up, self.up.shape, _CODE, self.up.device)
        _expect("down", self.down, (self.experts, self.width, self.inner), (up.dtype,), up.device)
        self.up8, self.up_scale = quantize(self.up.reshape(-1, self.width))          # laid out once
        self.down8, self.down_scale = quantize(self.down.reshape(-1, self.inner))

    def _routing(self, x: torch.Tensor, ids: torch.Tensor, weight: torch.Tensor):
        tokens, k = ids.shape
        _expect("x", x, (tokens, self.width), _CODE, self.up.device)
        _expect("ids", ids, (tokens, k), (torch.int32,), self.up.device)
        _expect("weight", weight, (tokens, k), (torch.float32,), self.up.device)
        size = P.opevo_route_workspace(tokens, k, self.experts)
        return (tokens, k, torch.empty(self.experts + 1, dtype=torch.int32, device=ids.device), torch.empty(tokens * k, dtype=torch.int32, device=ids.device),
                torch.empty(max(size, 4), dtype=torch.uint8, device=ids.device), size)

    def _product(self, a, a_scale, w, w_scale, offsets, out):
        rows, k = a.shape
        P.opevo_matmul_i8_grouped(a.data_ptr(), k, a_scale.data_ptr(), w.data_ptr(), k, w_scale.data_ptr(), offsets.data_ptr(), self.experts, out.data_ptr(),
                                  out.shape[1], _CODE[out.dtype], rows, out.shape[1], k, _stream())
        return out

    def _combine(self, rows, weight, row_of_slot, tokens, k):
        y = torch.empty(tokens, rows.shape[1], dtype=rows.dtype, device=rows.device)
        P.opevo_route_combine(rows.data_ptr(), rows.shape[1], _CODE[rows.dtype], 0 if weight is None else weight.data_ptr(), row_of_slot.data_ptr(), tokens, k,
                              rows.shape[1], y.data_ptr(), y.shape[1], _stream())
        return y

    def serve(self, x: torch.Tensor, ids: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
        """x [tokens, H], ids int32 [tokens, k] (an id outside [0, E): a slot held elsewhere), weight fp32 [tokens, k] -> [tokens, H]."""
        tokens, k, offsets, row_of_slot, workspace, size = self._routing(x, ids, weight)
        rows = tokens * k
        q, scale = torch.empty(rows, self.width, dtype=torch.int8, device=x.device), torch.empty(rows, device=x.device)
        P.opevo_route_dispatch_i8(ids.data_ptr(), tokens, k, self.experts, x.data_ptr(), self.width, _CODE[x.dtype], self.width, offsets.data_ptr(),
                                  row_of_slot.data_ptr(), q.data_ptr(), self.width, scale.data_ptr(), workspace.data_ptr(), size, _stream())
        hidden = self._product(q, scale, self.up8, self.up_scale, offsets, torch.empty(rows, self.inner, dtype=x.dtype, device=x.device))
        hidden8, hidden_scale = quantize(torch.relu_(hidden))
        out = self._product(hidden8, hidden_scale, self.down8, self.down_scale, offsets, torch.empty(rows, self.width, dtype=x.dtype, device=x.device))
        return self._combine(out, weight, row_of_slot, tokens, k)

    def train(self, x: torch.Tensor, ids: torch.Tensor, weight: torch.Tensor, dy: torch.Tensor):
        """(y, gradients of x, weight, up and down) for the gradient dy of y."""
        _expect("x", x, x.shape, (self.up.dtype,), self.up.device)
        _expect("dy", dy, x.shape, (x.dtype,), x.device)
        tokens, k, offsets, row_of_slot, workspace, size = self._routing(x, ids, weight)
        rows = torch.empty(tokens * k, self.width, dtype=x.dtype, device=x.device)
        P.opevo_route_dispatch(ids.data_ptr(), tokens, k, self.experts, x.data_ptr(), self.width, _CODE[x.dtype], self.width, offsets.data_ptr(),
                               row_of_slot.data_ptr(), rows.data_ptr(), self.width, workspace.data_ptr(), size, _stream())
        parts = [slice(lo, hi) for lo, hi in zip(offsets.tolist(), offsets.tolist()[1:])]
        hidden, out = torch.zeros(tokens * k, self.inner, dtype=x.dtype, device=x.device), torch.zeros_like(rows)
        for e, part in enumerate(parts):
            hidden[part] = rows[part] @ self.up[e].t()
            out[part] = torch.relu(hidden[part]) @ self.down[e].t()
        y = self._combine(out, weight, row_of_slot, tokens, k)
        dout, dweight = torch.empty_like(out), torch.empty_like(weight)
        P.opevo_route_combine_grad(dy.data_ptr(), self.width, out.data_ptr(), self.width, _CODE[x.dtype], weight.data_ptr(), row_of_slot.data_ptr(),
                                   offsets.data_ptr(), self.experts, tokens, k, self.width, dout.data_ptr(), self.width, dweight.data_ptr(), _stream())
        drows, dup, ddown = torch.zeros_like(rows), torch.zeros_like(self.up), torch.zeros_like(self.down)
        for e, part in enumerate(parts):
            active = torch.relu(hidden[part])
            ddown[e] = dout[part].t() @ active
            dhidden = (dout[part] @ self.down[e]) * (hidden[part] > 0)
            dup[e] = dhidden.t() @ rows[part]
            drows[part] = dhidden @ self.up[e]
        return y, self._combine(drows, None, row_of_slot, tokens, k), dweight, dup, ddown


def in_64_bits(layer: ExpertLayer, x, ids, weight):
    """The layer's definition, token by token and expert by expert."""
    y = torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    for e in range(layer.experts):
        token, slot = torch.nonzero(ids == e, as_tuple=True)
        out = torch.relu(x[token].double() @ layer.up[e].double().t()) @ layer.down[e].double().t()
        y.index_add_(0, token, weight[token, slot].double()[:, None] * out)
    return y


def main(tokens: int = 512, k: int = 2, experts: int = 8, width: int = 1024, inner: int = 4096):
    g = torch.Generator(device="cuda").manual_seed(0)
    up = torch.randn(experts, inner, width, generator=g, device="cuda") / width ** 0.5
    down = torch.randn(experts, width, inner, generator=g, device="cuda") / inner ** 0.5
    layer = ExpertLayer(up, down)
    x = torch.randn(tokens, width, generator=g, device="cuda")
    top, ids = torch.topk(torch.randn(tokens, experts, generator=g, device="cuda"), k, dim=1)
    ids, weight = ids.to(torch.int32), torch.softmax(top, dim=1)
    want = in_64_bits(layer, x, ids, weight)
    error = {}
    for dtype in (torch.float32, torch.bfloat16):
        y = layer.serve(x.to(dtype), ids, weight).double()
        error["served, tokens in %s" % str(dtype).split(".")[1]] = float((y - want).norm() / want.norm())
    xr, wr, upr, downr = (t.double().requires_grad_() for t in (x, weight, up, down))
    ref = ExpertLayer.__new__(ExpertLayer)
    ref.experts, ref.up, ref.down = experts, upr, downr
    dy = torch.randn(tokens, width, generator=g, device="cuda")
    (in_64_bits(ref, xr, ids, wr) * dy.double()).sum().backward()
    for name, got, exact in zip(("y", "dx", "dweight", "dup", "ddown"), layer.train(x, ids, weight, dy), (want, xr.grad, wr.grad, upr.grad, downr.grad)):
        error["trained, " + name] = float((got.double() - exact).norm() / exact.norm())
    return error


if __name__ == "__main__":
    for name, value in main().items():
        print("%-28s relative error %.2e" % (name, value))
