"""The work the 4-bit operators are measured on: matrices quantised to microscaled 4-bit floating point (elements of two
significant bits, a shared power of two for every 32 columns of a row) and back, and matrix products with such weights.

A case is a dict of plain values.  ``op`` says which calls it stands for:

  quantize  a matrix to its 4-bit form and back to the values it stands for (weights before they are shipped, and the check of what
            they lost; activations on their way into a product)
  linear44  a GEMM with 4-bit weights whose 16-bit input is quantised on its way in, with bias, residual and ReLU
  linear16  the same with the 16-bit input as it is

Inputs are those of the other workloads: rectified normal activations, normal weights of deviation 0.02.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32                    # columns that share a scale
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _quantize(name=None, **kw):
    c = dict(op="quantize", rows=1, cols=2048, dtype="bf16", out="bf16", kind="activations")
    c.update(kw)
    return c if name is None else dict(c, name=name)


def _linear(name=None, **kw):
    c = dict(op="linear44", M=1, I=512, O=512, out="bf16", bias=True, residual=False, relu=True)
    c.update(kw)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one row of features on its way into a classifier: a call's latency
        _quantize("quantize_row"),
        # the activations of a 1x1 layer for an ordinary batch: 64 images of 7x7 pixels
        _quantize("quantize_3136", rows=3136, cols=512),
        # fp32 weights of odd sizes: the last block of a row is short
        _quantize("quantize_ragged", rows=1021, cols=1003, dtype="f32", out="f32", kind="weights"),
        # the largest activations of the network, 64 images of 56x56 pixels
        _quantize("quantize_200704", rows=200704, cols=256),
        # the classifier for one image, fp32 logits
        _linear("one_row_44", M=1, I=2048, O=1000, out="f32", relu=False),
        # a 1x1 layer for an ordinary batch
        _linear("gemm_3136_44", M=3136, I=512, O=2048),
        # the widening layer of an early block with its shortcut: few inputs, much output
        _linear("widen_200704_44", M=200704, I=64, O=256, residual=True),
        # odd sizes in every direction
        _linear("ragged_44", M=777, I=1003, O=1001, residual=True),
        # a product that is bound by arithmetic: the largest case
        _linear("large_44", M=8192, I=8192, O=8192, bias=False, relu=False),
        # few rows against wide layers: the weights' bytes are the work
        _linear("few_rows_16", M=16, I=4096, O=8192, relu=False),
        # the 1x1 layer with its input in 16 bits
        _linear("gemm_3136_16", op="linear16", M=3136, I=512, O=2048),
        # a long input against a wide layer, 16-bit input: bound by arithmetic
        _linear("large_16", op="linear16", M=8192, I=4096, O=4096, bias=False, relu=False),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, evenly over its logarithm; one in two is made a multiple of 32 where there is one."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v // 32 * 32 if v >= 32 and rng.random() < 0.5 else v


def draw(rng):
    if rng.random() < 1 / 3:
        cols = _spread(rng, 16, 8192)
        rows = _spread(rng, 1, min(262144, 200704 * 256 // cols))
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return _quantize(rows=rows, cols=cols, dtype=dtype, out=rng.choice(["bf16", "f32"]), kind=rng.choice(["activations", "weights"]))
    op = rng.choice(["linear44", "linear16"])
    I, O = _spread(rng, 32, 8192), _spread(rng, 8, 8192)
    most = min(200704, 2 ** 38 // (I * O), 200704 * 320 // (I + 2 * O))
    M = rng.choice([1, rng.randint(2, 16), _spread(rng, 17, max(18, most))])
    residual = rng.random() < 0.4
    # (fp32 results of a 16-bit input are the tests' subject: the sums are the tensor cores')
    out = rng.choice(["bf16", "bf16", "f32"]) if op == "linear44" else "bf16"
    return _linear(op=op, M=M, I=I, O=O, out=out, bias=rng.random() < 0.7, residual=residual, relu=rng.random() < 0.6)


def _inputs(case, seed):
    """The case's inputs as a program holds them, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    def normal(*size):
        return torch.randn(*size, generator=g, device="cuda")
    if case["op"] == "quantize":
        v = normal(case["rows"], case["cols"])
        v = v.relu_() if case["kind"] == "activations" else v.mul_(0.02)
        return {"x": v.to(_TYPES[case["dtype"]])}
    M, I, O = case["M"], case["I"], case["O"]
    t = {"x": normal(M, I).relu_().to(torch.bfloat16), "w": normal(O, I).mul_(0.02).to(torch.bfloat16)}
    t["bias"] = normal(O).mul_(0.1) if case["bias"] else None
    t["residual"] = normal(M, O).to(_TYPES[case["out"]]) if case["residual"] else None
    return t


def _rounded(x):
    """The values of x's 4-bit form, in fp32, blocks along the last dimension.  A block's scale is the power of two that puts its largest
    magnitude into [4, 8); elements go to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times the scale, ties to the even one, what is past 6 to 6."""
    rows, cols = x.shape
    n = (cols + BLOCK - 1) // BLOCK
    v = x.float()
    if n * BLOCK != cols:
        v = torch.cat([v, v.new_zeros(rows, n * BLOCK - cols)], 1)
    v = v.view(rows, n, BLOCK)
    top = v.abs().amax(2, keepdim=True)
    exponent = (torch.frexp(top).exponent - 3).clamp(min=-127)
    exponent = torch.where(top == 0, torch.full_like(exponent, -127), exponent)
    v = torch.ldexp(v, -exponent)
    m = v.abs()
    q = 0.5 * (m > 0.25) + 0.5 * (m >= 0.75) + 0.5 * (m > 1.25) + 0.5 * (m >= 1.75) + 1.0 * (m > 2.5) + 1.0 * (m >= 3.5) + 2.0 * (m > 5)
    return torch.ldexp(torch.copysign(q, v), exponent).view(rows, n * BLOCK)[:, :cols]


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    if case["op"] == "quantize":
        return state
    # the program keeps its weights in four bits
    w = state.pop("w")
    if own:
        import paper_2012_00596_b200 as npas
        state["w"] = npas.quantize_mx(w)
        state["ws"] = npas.linear_mx_workspace(case["M"], state["w"], quantize_x=case["op"] == "linear44")
    else:
        state["w"] = _rounded(w)
    return state


def run(state):
    case, x = state["case"], state["x"]
    if own:
        import paper_2012_00596_b200 as npas
        if case["op"] == "quantize":
            return npas.dequantize_mx(npas.quantize_mx(x), dtype=_TYPES[case["out"]])
        return npas.linear_mx(x, state["w"], state["bias"], state["residual"], relu=case["relu"], out_dtype=_TYPES[case["out"]],
                              quantize_x=case["op"] == "linear44", ws=state["ws"])
    if case["op"] == "quantize":
        return _rounded(x).to(_TYPES[case["out"]])
    y = (_rounded(x) if case["op"] == "linear44" else x.float()) @ state["w"].t()
    if state["bias"] is not None:
        y += state["bias"]
    if state["residual"] is not None:
        y += state["residual"].float()
    if case["relu"]:
        y = y.clamp_(min=0)
    return y.to(_TYPES[case["out"]])


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["dtype"]] + size[case["out"]]), "flops": 2 * n}
    M, I, O = case["M"], case["I"], case["O"]
    weights = O * I / 2 + O * ((I + BLOCK - 1) // BLOCK)
    out = M * O * size[case["out"]] * (2 if case["residual"] else 1)
    return {"bytes": int(2 * M * I + weights + out + (4 * O if case["bias"] else 0)), "flops": 2 * M * I * O}


def _nearest(x):
    """The 4-bit values of x in 64 bits: a magnitude v times 2^-scale is rounded to whole steps of 2^(e - 1), e its own exponent and
    at least 0, halves to even."""
    x = x.double()
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], BLOCK):
        b = x[:, c:c + BLOCK]
        top = b.abs().max(1, keepdim=True).values
        scale = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -125))) - 2)
        scale = scale.clamp(min=2.0 ** -127)
        v = b / scale
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=1.0)))) / 2
        out[:, c:c + BLOCK] = (torch.round(v / step) * step).clamp(-6, 6) * scale
    return out


def exact(case, seed):
    t = _inputs(case, seed)
    if case["op"] == "quantize":
        return _nearest(t["x"])
    x = _nearest(t["x"]) if case["op"] == "linear44" else t["x"].double()
    y = x @ _nearest(t["w"]).T
    if t["bias"] is not None:
        y = y + t["bias"].double()
    if t["residual"] is not None:
        y = y + t["residual"].double()
    return torch.relu(y) if case["relu"] else y
