"""The work around an expert layer, as cases that can be measured one by one.

The norm that stands before every projection, microscaled 4-bit numbers (E2M1, a power of two for every 32 of them) with their products, and a
whole layer of experts for few tokens.  A case is one pass that a program makes, over and over:

  norm          rows and their residual -> the sum, its RMS norm                               (serving)
  norm_linear   the same with the norm's rows in 8 bits -> product with 8-bit weights          (serving)
  norm_train    the norm, and its gradients                                                    (training)
  mx4_values    rows to microscaled 4 bits and back: the values a layer will compute with      (training with them)
  mx4_linear    rows to microscaled 4 bits -> product with weights that are in them
  mx4_matmul    a product of operands that are in 4 bits already
  mx4_experts   rows sorted by expert to microscaled 4 bits -> every expert's product
  layer         tokens and their experts -> gate, up, down, and the sum with the router's weights

With `own` false `run` is the plain form, in elementary torch operations and 32 bits (64 next to the border between two 8-bit integers); with `own` true it makes the
library's calls.
"""
from __future__ import annotations

import math
import random
from typing import Dict, List

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_CODE = {"f32": 0, "bf16": 1, "f16": 2}
_EPS = 1e-5


def listed() -> List[Dict]:
    return [
        # one token of a decoding sequence: launch and latency
        dict(name="norm_one_token", kind="norm", rows=1, width=4096, dtype="bf16", residual=True),
        # a whole batch of prompts: two rows read and two written for each
        dict(name="norm_16384", kind="norm", rows=16384, width=4096, dtype="bf16", residual=True),
        # a decoding batch on its way into a projection in 8 bits
        dict(name="norm_linear_32_f16", kind="norm_linear", rows=32, width=4096, n=1024, dtype="f16", out="f16", residual=True),
        # a training step of ordinary size
        dict(name="norm_train_8192", kind="norm_train", rows=8192, width=4096, dtype="bf16", residual=True),
        # a small training step in full precision, no multiples of anything, no residual
        dict(name="norm_train_1001_f32", kind="norm_train", rows=1001, width=1000, dtype="f32", residual=False),
        # activations of a training step as the 4-bit products will see them
        dict(name="mx4_values_8192", kind="mx4_values", rows=8192, width=4096, dtype="bf16"),
        # one token through a projection: the weights are read once
        dict(name="mx4_linear_one_token", kind="mx4_linear", m=1, n=4096, kk=4096, dtype="bf16", out="bf16"),
        # the largest product, the one the matrix pipes bound
        dict(name="mx4_matmul_8192", kind="mx4_matmul", m=8192, n=8192, kk=8192, dtype="mx4", out="bf16"),
        # prompts over a few experts of very different load
        dict(name="mx4_experts_prompt", kind="mx4_experts", rows=8192, experts=8, n=4096, kk=1024, dtype="bf16", out="bf16", held=1.0),
        # a decoding batch over many experts, extents that are no multiples of any tile, a tenth of the rows belongs to experts held elsewhere
        dict(name="mx4_experts_333_f32", kind="mx4_experts", rows=333, experts=24, n=1000, kk=1001, dtype="f32", out="f32", held=0.9),
        # one token through its two experts, weights in 8 bits: latency, and 25 MB of weights
        dict(name="layer_one_token", kind="layer", tokens=1, k=2, experts=8, width=1024, inner=4096, dtype="bf16", weights="i8", held=1.0),
        # a decoding batch over many experts, weights in 4 bits: nearly all of them are read
        dict(name="layer_32_mx4", kind="layer", tokens=32, k=4, experts=64, width=4096, inner=1024, dtype="bf16", weights="mx4", held=1.0),
    ]


def _log(rng: random.Random, lo: float, hi: float) -> int:
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_WIDTHS = (64, 128, 256, 320, 512, 640, 768, 1024, 1280, 1536, 1792, 2048, 2560, 3584, 4096, 5120, 7168, 8192)


def _width(rng: random.Random, lo: int, hi: int) -> int:
    """Half of them multiples of 64, as layers mostly have, the others any number."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.5 else min(_WIDTHS, key=lambda w: abs(math.log(w / n)))


def draw(rng: random.Random) -> Dict:
    kind = rng.choice(("norm", "norm_linear", "norm_train", "mx4_values", "mx4_linear", "mx4_matmul", "mx4_experts", "layer", "layer"))
    dtype, out = rng.choice(("bf16", "bf16", "f16", "f32")), rng.choice(("bf16", "bf16", "f16", "f32"))
    held, residual = rng.choice((1.0, 1.0, 0.9, 0.5)), rng.random() < 0.7
    while True:
        if kind in ("mx4_linear", "mx4_matmul"):
            case = dict(kind=kind, m=_log(rng, 1, 8192), n=_width(rng, 64, 8192), kk=_width(rng, 64, 8192),
                        dtype="mx4" if kind == "mx4_matmul" else dtype, out=out)
            if work(case)["flops"] <= 1.1e12:
                return case
        elif kind == "mx4_experts":
            case = dict(kind=kind, rows=_log(rng, 1, 32768), experts=_log(rng, 4, 128), n=_width(rng, 64, 4096), kk=_width(rng, 64, 4096),
                        dtype=dtype, out=out, held=held)
            if work(case)["flops"] <= 3e11 and case["experts"] * case["n"] * case["kk"] <= 5e8 and case["rows"] * (case["n"] + case["kk"]) <= 4e8:
                return case
        elif kind == "layer":
            experts = _log(rng, 4, 128)
            case = dict(kind=kind, tokens=_log(rng, 1, 256), k=rng.randint(1, min(8, experts)), experts=experts, width=_width(rng, 64, 4096),
                        inner=_width(rng, 64, 4096), dtype=dtype, weights=rng.choice(("i8", "mx4")), held=held)
            if case["tokens"] * case["k"] <= 512 and experts * case["width"] * case["inner"] <= 2.7e8:
                return case
        elif kind == "norm_linear":
            case = dict(kind=kind, rows=_log(rng, 1, 8192), width=_width(rng, 64, 8192), n=_width(rng, 64, 8192), dtype=dtype, out=out, residual=residual)
            if work(case)["flops"] <= 1.1e12:
                return case
        else:
            case = dict(kind=kind, rows=_log(rng, 1, 16384), width=_width(rng, 64, 8192), dtype=dtype)
            if kind != "mx4_values":
                case["residual"] = residual
            if case["rows"] * case["width"] <= 6.7e7:
                return case


def _bytes(dtype: str) -> float:
    return {"mx4": 0.5 + 1 / 32, "i8": 1, "bf16": 2, "f16": 2, "f32": 4}[dtype]


def _used(experts: int, rows: float) -> float:
    """Experts that get a row, were the load even."""
    return experts * (1.0 - (1.0 - 1.0 / experts) ** rows)


def work(case: Dict) -> Dict:
    kind, size = case["kind"], _bytes(case["dtype"])
    if kind in ("mx4_linear", "mx4_matmul"):
        m, n, k = case["m"], case["n"], case["kk"]
        return {"bytes": int(m * k * size + n * k * _bytes("mx4") + m * n * _bytes(case["out"])), "flops": 2 * m * n * k}
    if kind == "mx4_experts":
        rows, n, k = case["rows"], case["n"], case["kk"]
        held = rows * case["held"]
        return {"bytes": int(rows * k * size + _used(case["experts"], held) * n * k * _bytes("mx4") + rows * n * _bytes(case["out"])), "flops": int(2 * held * n * k)}
    if kind == "layer":
        slots = case["tokens"] * case["k"] * case["held"]
        each = 3 * case["width"] * case["inner"]
        return {"bytes": int(2 * case["tokens"] * case["width"] * size + 8 * case["tokens"] * case["k"] + _used(case["experts"], slots) * each * _bytes(case["weights"])),
                "flops": int(2 * slots * each)}
    rows, width = case["rows"], case["width"]
    if kind == "mx4_values":
        return {"bytes": int(2 * rows * width * size), "flops": 0}
    read = (2 if case["residual"] else 1) * rows * width * size + width * size           # x, the residual, the weight
    if kind == "norm_linear":
        n = case["n"]
        return {"bytes": int(read + rows * width * size * case["residual"] + n * width + 4 * n + rows * n * _bytes(case["out"])), "flops": 2 * rows * n * width}
    read += (2 if case["residual"] else 1) * rows * width * size                         # the sum and the norm are written
    if kind == "norm":
        return {"bytes": int(read), "flops": 5 * rows * width}
    # dy and the sum's gradient are read, dx written; the sum serves both directions
    return {"bytes": int(read + (3 if case["residual"] else 2) * rows * width * size + 4 * width), "flops": 15 * rows * width}


# ------------------------------------------------------------------ inputs
def _tokens(g, rows: int, width: int, dtype: str) -> torch.Tensor:
    """Activations: normal, a hundredth of the channels ten times the others."""
    wide = 1.0 + 9.0 * (torch.rand(width, generator=g, device="cuda") < 0.01)
    return (torch.randn(rows, width, generator=g, device="cuda") * wide).to(_DTYPE[dtype])


def _eight_bits(g, *shape) -> torch.Tensor:
    """Quantised normal values: the largest of a row is about 127."""
    return (torch.randn(*shape, generator=g, device="cuda") * 32.0).round_().clamp_(-127, 127).to(torch.int8)


def _four_bits(g, rows: int, width: int):
    """Normal weights of a layer, in microscaled 4 bits: two codes a byte (the earlier one in the low half), one scale for 32 values."""
    codes = torch.empty(rows, (width + 1) // 2, dtype=torch.uint8, device="cuda")
    scale = torch.empty(rows, (width + 31) // 32, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // width)
    for r in range(0, rows, step):
        x = torch.randn(min(step, rows - r), width, generator=g, device="cuda") / math.sqrt(width)
        code, exponent = _plain_mx4(x)
        code = torch.nn.functional.pad(code, (0, width % 2))
        codes[r:r + step] = (code[:, 0::2] | code[:, 1::2] << 4).to(torch.uint8)
        scale[r:r + step] = (exponent + 127).to(torch.uint8)
    return codes, scale


def prepare(case: Dict, seed: int) -> Dict:
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, state = case["kind"], {"case": case}
    new = lambda *shape, dtype=torch.uint8: torch.empty(*shape, dtype=dtype, device="cuda")     # noqa: E731
    if kind in ("mx4_linear", "mx4_matmul"):
        m, n, k = case["m"], case["n"], case["kk"]
        state["w"], state["sw"] = _four_bits(g, n, k)
        if kind == "mx4_matmul":
            state["a"], state["sa"] = _four_bits(g, m, k)
        else:
            state["x"] = _tokens(g, m, k, case["dtype"])
        if own:
            state["y"] = new(m, n, dtype=_DTYPE[case["out"]])
            if kind == "mx4_linear":
                state.update(a=new(m, (k + 1) // 2), sa=new(m, (k + 31) // 32))
        return state
    if kind == "mx4_experts":
        rows, n, k, experts = case["rows"], case["n"], case["kk"], case["experts"]
        state["x"] = _tokens(g, rows, k, case["dtype"])
        state["w"], state["sw"] = _four_bits(g, experts * n, k)
        # rows as a dispatch leaves them: some experts are wanted more than others, behind the last one's come the rows of no expert here
        share = torch.softmax(torch.randn(experts, generator=g, device="cuda"), 0)
        counts = torch.bincount(torch.multinomial(share, max(1, int(rows * case["held"])), replacement=True, generator=g), minlength=experts)
        state["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        if own:
            state.update(y=new(rows, n, dtype=_DTYPE[case["out"]]), a=new(rows, (k + 1) // 2), sa=new(rows, (k + 31) // 32))
        return state
    if kind == "layer":
        tokens, k, experts, width, inner = case["tokens"], case["k"], case["experts"], case["width"], case["inner"]
        # a router's choice: k different experts a token, some wanted more than others; slots of experts held elsewhere carry ids outside [0, experts)
        logits = torch.randn(tokens, experts, generator=g, device="cuda") + torch.randn(experts, generator=g, device="cuda")
        top, ids = torch.topk(logits, k, dim=1)
        away = torch.rand(tokens, k, generator=g, device="cuda") >= case["held"]
        state.update(ids=torch.where(away, experts + ids, ids).to(torch.int32), weight=torch.softmax(top, dim=1).contiguous(), x=_tokens(g, tokens, width, case["dtype"]))
        if case["weights"] == "i8":
            scale = lambda n, of: (torch.rand(experts, n, generator=g, device="cuda") + 0.5) / (32.0 * math.sqrt(of))   # noqa: E731
            state.update(win=_eight_bits(g, experts * 2 * inner, width), sin=scale(2 * inner, width), wout=_eight_bits(g, experts * width, inner), sout=scale(width, inner))
        else:
            state["win"], state["sin"] = _four_bits(g, experts * 2 * inner, width)
            state["wout"], state["sout"] = _four_bits(g, experts * width, inner)
        if own:
            import paper_2006_05664_amd as P
            size = P.opevo_expert_layer_workspace(tokens, k, _CODE[case["dtype"]], inner)
            state.update(y=torch.empty_like(state["x"]), workspace=new(max(size, 1)), workspace_bytes=size)
        return state
    rows, width, dtype = case["rows"], case["width"], case["dtype"]
    state["x"] = _tokens(g, rows, width, dtype)
    if kind == "mx4_values":
        if own:
            state.update(q=new(rows, (width + 1) // 2), scale=new(rows, (width + 31) // 32), y=torch.empty_like(state["x"]))
        return state
    state["weight"] = (1.0 + 0.2 * torch.randn(width, generator=g, device="cuda")).to(_DTYPE[dtype])
    if case["residual"]:
        state["residual"] = _tokens(g, rows, width, dtype)
    if kind == "norm_linear":
        state.update(w=_eight_bits(g, case["n"], width), sw=(torch.rand(case["n"], generator=g, device="cuda") + 0.5) * 1e-3)
    if kind == "norm_train":
        state["dy"] = _tokens(g, rows, width, dtype)
        if case["residual"]:
            state["dsum"] = _tokens(g, rows, width, dtype)
    if own:
        if case["residual"]:
            state["sum"] = torch.empty_like(state["x"])
        if kind == "norm_linear":
            state.update(q=new(rows, width, dtype=torch.int8), scale=new(rows, dtype=torch.float32), y=new(rows, case["n"], dtype=_DTYPE[case["out"]]))
        else:
            state["y"] = torch.empty_like(state["x"])
        if kind == "norm_train":
            import paper_2006_05664_amd as P
            size = P.opevo_norm_rows_grad_workspace(rows, width)
            state.update(inv_rms=new(rows, dtype=torch.float32), dx=torch.empty_like(state["x"]), dweight=new(width, dtype=torch.float32),
                         workspace=new(max(size, 1)), workspace_bytes=size)
    return state


# ------------------------------------------------------------------ the plain form
def _power(exponent: torch.Tensor) -> torch.Tensor:
    """2^exponent in fp32, -126 to 127."""
    return ((exponent.to(torch.int32) + 127) << 23).view(torch.float32)


def _plain_mx4(x: torch.Tensor):
    """(codes, exponents): E2M1 codes of the values over the power of two of their 32, whose largest magnitude lands in [4, 8)."""
    x = x.float()
    rows, width = x.shape
    blocks = torch.nn.functional.pad(x, (0, -width % 32)).reshape(rows, -1, 32)
    exponent = ((blocks.abs().amax(dim=2).view(torch.int32) >> 23) - 129).clamp(min=-126)
    v = blocks * _power(-exponent)[:, :, None]
    m = v.abs()
    # between two neighbours; a value in the middle goes to the one whose last bit is 0
    code = ((m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0)) | (v < 0).int() << 3
    return code.reshape(rows, -1)[:, :width], exponent


def _plain_values(code: torch.Tensor, exponent: torch.Tensor) -> torch.Tensor:
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=code.device)
    return values[code.long()] * _power(exponent).repeat_interleave(32, 1)[:, :code.shape[1]]


def _plain_unpack(q: torch.Tensor, scale: torch.Tensor, width: int) -> torch.Tensor:
    code = torch.stack([q & 15, q >> 4], dim=2).reshape(q.shape[0], -1)[:, :width]
    return _plain_values(code, scale.int() - 127)


def _plain_layer(state: Dict) -> torch.Tensor:
    case = state["case"]
    tokens, experts, width, inner = case["tokens"], case["experts"], case["width"], case["inner"]
    if case["weights"] == "i8":
        win, wout = state["win"].float() * state["sin"].reshape(-1, 1), state["wout"].float() * state["sout"].reshape(-1, 1)
    else:
        win, wout = _plain_unpack(state["win"], state["sin"], width), _plain_unpack(state["wout"], state["sout"], inner)
    held = state["ids"] < experts
    ids, token = torch.where(held, state["ids"], 0).long(), torch.arange(tokens, device=held.device)[:, None]
    # every token through every expert's first product, of which its own are taken
    up = (state["x"].float() @ win.t()).reshape(tokens, experts, 2 * inner)[token, ids]
    h = up[:, :, :inner] / (1.0 + torch.exp(-up[:, :, :inner])) * up[:, :, inner:]
    h = torch.where(held, state["weight"], 0.0)[:, :, None] * h
    dense = torch.zeros(tokens, experts, inner, device=h.device)
    dense.index_put_((token, ids), h, accumulate=True)
    y = dense.reshape(tokens, -1) @ wout.reshape(experts, width, inner).transpose(1, 2).reshape(-1, width)
    return y.to(_DTYPE[case["dtype"]])


def _plain(state: Dict):
    case = state["case"]
    kind = case["kind"]
    if kind in ("mx4_linear", "mx4_matmul"):
        a = _plain_values(*_plain_mx4(state["x"])) if kind == "mx4_linear" else _plain_unpack(state["a"], state["sa"], case["kk"])
        return (a @ _plain_unpack(state["w"], state["sw"], case["kk"]).t()).to(_DTYPE[case["out"]])
    if kind == "mx4_experts":
        rows, n, k, experts, offsets = case["rows"], case["n"], case["kk"], case["experts"], state["offsets"].long()
        a = _plain_values(*_plain_mx4(state["x"]))
        at = torch.arange(rows, device=a.device)
        expert = (at[:, None] >= offsets[None, 1:]).sum(1)
        held, expert = expert < experts, expert.clamp(max=experts - 1)
        most = int((offsets[1:] - offsets[:-1]).max())
        place = expert * most + torch.where(held, at - offsets[expert], 0)
        padded = torch.zeros(experts * most, k, device=a.device)
        padded.index_put_((place,), torch.where(held[:, None], a, 0.0), accumulate=True)
        w = _plain_unpack(state["w"], state["sw"], k).reshape(experts, n, k).transpose(1, 2).contiguous()
        y = torch.bmm(padded.reshape(experts, most, k), w).reshape(experts * most, n)[place]
        return torch.where(held[:, None], y, 0.0).to(_DTYPE[case["out"]])
    if kind == "layer":
        return _plain_layer(state)
    if kind == "mx4_values":
        return _plain_values(*_plain_mx4(state["x"])).to(_DTYPE[case["dtype"]])
    dtype, x, w = _DTYPE[case["dtype"]], state["x"].float(), state["weight"].float()
    total = (x + state["residual"].float()).to(dtype) if case["residual"] else state["x"]
    s = total.float()
    inv = 1.0 / torch.sqrt((s * s).mean(dim=1, keepdim=True) + _EPS)
    outs = {"sum": total} if case["residual"] else {}
    if kind == "norm_linear":
        v = total.double() * state["weight"].double()
        a = v.abs().amax(dim=1, keepdim=True)
        q = torch.round(127.0 * v / a).float()
        outs["y"] = ((q @ state["w"].float().t()) * ((a.float() * inv / 127.0) * state["sw"][None, :])).to(_DTYPE[case["out"]])
        return outs
    outs["y"] = (s * inv * w).to(dtype)
    if kind == "norm":
        return outs
    dy = state["dy"].float()
    dot = (w * dy * s).mean(dim=1, keepdim=True)
    dx = inv * (w * dy - s * (inv * inv * dot))
    outs["dx"] = (dx + state["dsum"].float() if case["residual"] else dx).to(dtype)
    outs["dweight"] = (dy * s * inv).sum(dim=0)
    return outs


# ------------------------------------------------------------------ the library's calls
def _own(state: Dict):
    import paper_2006_05664_amd as P
    case = state["case"]
    kind, stream = case["kind"], torch.cuda.current_stream().cuda_stream
    at = lambda name: state[name].data_ptr() if name in state else 0          # noqa: E731
    if kind in ("mx4_linear", "mx4_matmul", "mx4_experts"):
        n, k, y = case["n"], case["kk"], state["y"]
        m, half, blocks = y.shape[0], (k + 1) // 2, (k + 31) // 32
        if kind != "mx4_matmul":
            P.opevo_quantize_rows_mx4(at("x"), k, _CODE[case["dtype"]], m, k, at("a"), half, at("sa"), blocks, stream)
        if kind == "mx4_experts":
            P.opevo_matmul_mx4_grouped(at("a"), half, at("sa"), blocks, at("w"), half, at("sw"), blocks, at("offsets"), case["experts"], y.data_ptr(), n,
                                       _CODE[case["out"]], m, n, k, stream)
        else:
            P.opevo_matmul_mx4(at("a"), half, at("sa"), blocks, at("w"), half, at("sw"), blocks, y.data_ptr(), n, _CODE[case["out"]], m, n, k, stream)
        return y
    code, width = _CODE[case["dtype"]], case["width"]
    if kind == "layer":
        inner = case["inner"]
        args = (at("x"), width, code, at("ids"), at("weight"), case["tokens"], case["k"], case["experts"], width, inner)
        if case["weights"] == "i8":
            P.opevo_expert_layer_i8(*args, at("win"), width, at("sin"), at("wout"), inner, at("sout"), at("y"), width, at("workspace"), state["workspace_bytes"], stream)
        else:
            P.opevo_expert_layer_mx4(*args, at("win"), (width + 1) // 2, at("sin"), (width + 31) // 32, at("wout"), (inner + 1) // 2, at("sout"), (inner + 31) // 32,
                                     at("y"), width, at("workspace"), state["workspace_bytes"], stream)
        return state["y"]
    rows, y = case["rows"], state["y"]
    if kind == "mx4_values":
        half, blocks = (width + 1) // 2, (width + 31) // 32
        P.opevo_quantize_rows_mx4(at("x"), width, code, rows, width, at("q"), half, at("scale"), blocks, stream)
        P.opevo_dequantize_rows_mx4(at("q"), half, at("scale"), blocks, code, rows, width, at("y"), width, stream)
        return y
    given = (at("x"), width, at("residual"), width, at("weight"), _EPS, code, rows, width, at("sum"), width)
    outs = {"sum": state["sum"], "y": y} if case["residual"] else {"y": y}
    if kind == "norm_linear":
        n = case["n"]
        P.opevo_norm_rows_i8(*given, at("q"), width, at("scale"), stream)
        P.opevo_matmul_i8(at("q"), width, at("scale"), at("w"), width, at("sw"), at("y"), n, _CODE[case["out"]], rows, n, width, stream)
        return outs
    P.opevo_norm_rows(*given, at("y"), width, at("inv_rms"), stream)
    if kind == "norm":
        return outs
    P.opevo_norm_rows_grad(at("dy"), width, at("dsum"), width, at("sum" if case["residual"] else "x"), width, at("weight"), at("inv_rms"), code, rows, width,
                           at("dx"), width, at("dweight"), at("workspace"), state["workspace_bytes"], stream)
    return dict(outs, dx=state["dx"], dweight=state["dweight"])


def run(state: Dict):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ the definition, in 64 bits
def _exact_mx4(x: torch.Tensor) -> torch.Tensor:
    """The values that rows stand for in microscaled 4 bits."""
    x = x.double()
    out = torch.empty_like(x)
    for b in range(0, x.shape[1], 32):
        part = x[:, b:b + 32]
        _, e = torch.frexp(part.abs().max(dim=1).values)            # a magnitude in [1/2, 1), so the floor of the logarithm is e - 1
        unit = torch.ldexp(torch.ones_like(e, dtype=torch.float64), (e - 3).clamp(min=-127))[:, None]
        m = part.abs() / unit
        step = torch.where(m < 2.0, 0.5, torch.where(m < 4.0, 1.0, 2.0)).double()   # the distance of neighbours; rounding is to even
        out[:, b:b + 32] = torch.copysign((torch.round(m / step) * step).clamp(max=6.0), part) * unit
    return out


def _exact_unpack(q: torch.Tensor, scale: torch.Tensor, width: int) -> torch.Tensor:
    out = torch.empty(q.shape[0], 2 * q.shape[1], dtype=torch.float64, device=q.device)
    for half in range(2):
        code = (q >> 4 * half & 15).int()
        e, m = (code >> 1 & 3).double(), (code & 1).double()
        v = torch.where(e > 0, torch.exp2(e - 1.0) * (1.0 + m / 2.0), m / 2.0)
        out[:, half::2] = torch.where(code > 7, -v, v)
    unit = torch.ldexp(torch.ones_like(scale, dtype=torch.float64), scale.int() - 127)
    return out[:, :width] * unit.repeat_interleave(32, dim=1)[:, :width]


def exact(case: Dict, seed: int):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind in ("mx4_linear", "mx4_matmul"):
        a = _exact_mx4(state["x"]) if kind == "mx4_linear" else _exact_unpack(state["a"], state["sa"], case["kk"])
        return torch.matmul(a, _exact_unpack(state["w"], state["sw"], case["kk"]).t().contiguous())
    if kind == "mx4_experts":
        n, at = case["n"], state["offsets"].tolist()
        a = _exact_mx4(state["x"])
        y = torch.zeros(case["rows"], n, dtype=torch.float64, device="cuda")
        for e in range(case["experts"]):
            if at[e + 1] > at[e]:
                w = _exact_unpack(state["w"][e * n:(e + 1) * n], state["sw"][e * n:(e + 1) * n], case["kk"])
                y[at[e]:at[e + 1]] = torch.matmul(a[at[e]:at[e + 1]], w.t().contiguous())
        return y
    if kind == "layer":
        width, inner, ids = case["width"], case["inner"], state["ids"].cpu()
        y = torch.zeros(case["tokens"], width, dtype=torch.float64, device="cuda")
        for e in range(case["experts"]):
            t, j = torch.nonzero(ids == e, as_tuple=True)
            if not len(t):
                continue
            first, second = slice(e * 2 * inner, (e + 1) * 2 * inner), slice(e * width, (e + 1) * width)
            if case["weights"] == "i8":
                win, wout = state["win"][first].double() * state["sin"][e].double()[:, None], state["wout"][second].double() * state["sout"][e].double()[:, None]
            else:
                win, wout = _exact_unpack(state["win"][first], state["sin"][first], width), _exact_unpack(state["wout"][second], state["sout"][second], inner)
            t, j = t.cuda(), j.cuda()
            up = torch.matmul(state["x"][t].double(), win.t().contiguous())
            h = up[:, :inner] * torch.sigmoid(up[:, :inner]) * up[:, inner:]
            y.index_add_(0, t, torch.matmul(h, wout.t().contiguous()) * state["weight"][t, j].double()[:, None])
        return y
    if kind == "mx4_values":
        return _exact_mx4(state["x"])
    s = state["x"].double()
    outs = {}
    if case["residual"]:
        outs["sum"] = s + state["residual"].double()
        s = outs["sum"].to(_DTYPE[case["dtype"]]).double()          # the norm is that of the sum as it is stored
    w = state["weight"].double()
    inv = (s.square().mean(dim=1, keepdim=True) + _EPS).rsqrt()
    if kind == "norm_linear":
        a = (s * w).abs().max(dim=1, keepdim=True).values
        outs["y"] = torch.matmul(torch.round(127.0 * (s * w) / a), state["w"].double().t().contiguous()) * (a * inv / 127.0) * state["sw"].double()
        return outs
    outs["y"] = s * inv * w
    if kind == "norm":
        return outs
    dy = state["dy"].double()
    n = s * inv                                                     # normalised: d y / d s = inv (1 - n n^T / width) diag(w)
    dn = dy * w
    outs["dx"] = inv * (dn - n * (dn * n).mean(dim=1, keepdim=True))
    if case["residual"]:
        outs["dx"] = outs["dx"] + state["dsum"].double()
    outs["dweight"] = (dy * n).sum(dim=0)
    return outs
