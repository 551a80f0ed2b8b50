"""Products with microscaled 4-bit weights where the other tests do not reach: exact sums over many columns, every forced split and
tile, ragged rows quantised inside the kernel for few rows, the ends of the scale range, ReLU of NaN, buffers on 16-byte boundaries only.

Nearly all comparisons are exact: inputs are small multiples of powers of two, every partial sum in any order is a multiple of the least
product and below 2^24 of it (checked), so fp32 sums have no rounding at all and every kernel has to give the 64-bit result's bits."""
import numpy as np
import pytest
import torch

import paper_2012_00596_b200 as npas
from oracle import mx

pytestmark = pytest.mark.gpu
KINDS = ["44", "blob", "16"]
SPLITS = [(3, 1), (3, 2), (3, 4), (3, 8)]
TILES = [(4, 128), (4, 256), (4, 128 + (1 << 16)), (4, 256 + (1 << 16))]
EVERY = [(0, 0), (1, 0), (2, 0)] + SPLITS + TILES + [(5, 0), (6, 0)]


def _members(rows, I, seed, lo=-1, hi=1):
    """Members of the 4-bit type times 2^lo .. 2^hi, another power for every block, each block with a member that fixes its scale."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ints = lambda a, b, *size: torch.randint(a, b, size, generator=g, device="cuda")
    v = torch.tensor(mx.MEMBERS, device="cuda")[ints(0, 8, rows, I)] * (ints(0, 2, rows, I) * 2 - 1)
    v[:, ::32] = 4.0 + 2.0 * ints(0, 2, rows, -(-I // 32))
    return v * torch.exp2(ints(lo, hi + 1, rows, -(-I // 32)).double()).repeat_interleave(32, 1)[:, :I]


def _takes(M, w, path, variant, **kw):
    try:
        npas.linear_mx_kernel(M, w, path=path, variant=variant, **kw)
        return True
    except npas.NpasError as e:
        assert e.code == 8
        return False


def _calls(M, w, kind, combos, out_dtype=torch.bfloat16):
    """The combinations of path and variant that take the call; which of them do not is known."""
    kw = dict(dtype="mx" if kind == "blob" else torch.bfloat16, quantize_x=kind == "44", out_dtype=out_dtype)
    taken = [c for c in combos if _takes(M, w, *c, **kw)]
    tiles = -(-M // 128) * -(-w.desc.rows // 128)
    for path, variant in set(combos) - set(taken):
        # CTA pairs take 4-bit inputs, kernel 6 up to 16 rows of 16 bits; a split of more CTAs than SMs has half an SM each for its sums
        assert (path == 5 and kind == "16") or (path == 6 and (kind != "16" or M > 16)) or (path == 3 and variant > 1 and kind != "16" and tiles * variant > 148), \
            (path, variant)
    return taken


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,I,O", [(1, 16384, 130), (5, 8191, 300), (16, 16384, 700), (64, 16384, 257), (700, 4096, 1000), (4000, 4096, 2500),
                                   (1500, 8191, 1300), (2300, 16384, 264)])
def test_sums_over_many_columns_are_exact(M, I, O, kind):
    """A column, a block or a group of stages left out, or a scale from another block, changes bits.  Products are multiples of 2^-4."""
    x, w = _members(M, I, 1), _members(O, I, 2)
    size = x.abs() @ w.abs().T
    assert float(size.max()) * 16 < 2 ** 24
    want = (x @ w.T).float()
    xb, wq = x.to(torch.bfloat16), npas.quantize_mx(w.to(torch.bfloat16))
    xin = npas.quantize_mx(xb) if kind == "blob" else xb
    for path, variant in _calls(M, wq, kind, EVERY, torch.float32):
        y = npas.linear_mx(xin, wq, out_dtype=torch.float32, quantize_x=kind == "44", path=path, variant=variant)
        assert torch.equal(y, want), (path, variant)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,I,O", [(1, 33, 1), (3, 520, 40), (9, 768, 129), (16, 2049, 256), (33, 1300, 77), (127, 264, 130), (129, 1003, 128), (300, 2304, 264)])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
def test_every_split_of_the_columns(M, I, O, kind, out_dtype):
    """A cluster of two, four or eight, also where some of it have no columns or the last has a part of a stage."""
    x, w = _members(M, I, 3), _members(O, I, 4)
    res = torch.randint(-8, 9, (M, O), device="cuda").to(out_dtype)
    bias = torch.randint(-8, 9, (O,), device="cuda").float()
    want = (x @ w.T + bias + res.double()).relu().to(out_dtype)
    xb, wq = x.to(torch.bfloat16), npas.quantize_mx(w.to(torch.bfloat16))
    xin = npas.quantize_mx(xb) if kind == "blob" else xb
    for path, variant in _calls(M, wq, kind, SPLITS, out_dtype):
        ws = npas.linear_mx_workspace(M, wq, dtype="mx" if kind == "blob" else torch.bfloat16, quantize_x=kind == "44", out_dtype=out_dtype, path=path, variant=variant)
        f = lambda: npas.linear_mx(xin, wq, bias, res, relu=True, out_dtype=out_dtype, quantize_x=kind == "44", ws=ws, path=path, variant=variant)
        for _ in range(3):
            assert torch.equal(f(), want), variant
        npas.check_device_status(ws)


@pytest.mark.parametrize("kind", ["blob", "16"])
@pytest.mark.parametrize("M,I,O,res", [(20000, 256, 256, False), (20000, 64, 256, True), (19001, 500, 136, True), (3136, 512, 2048, False), (9000, 64, 333, True),
                                       (9000, 72, 131, False)])
def test_weights_loaded_for_every_tile(M, I, O, res, kind):
    """The same tiles with weights that stay and with weights that are loaded again."""
    x, w = _members(M, I, 5), _members(O, I, 6)
    r = torch.randint(-8, 9, (M, O), device="cuda").to(torch.bfloat16) if res else None
    want = x @ w.T + (r.double() if res else 0)
    want = want.to(torch.bfloat16)
    xb, wq = x.to(torch.bfloat16), npas.quantize_mx(w.to(torch.bfloat16))
    xin = npas.quantize_mx(xb) if kind == "blob" else xb
    for path, variant in _calls(M, wq, kind, TILES):
        for _ in range(5):
            assert torch.equal(npas.linear_mx(xin, wq, None, r, path=path, variant=variant), want), variant


@pytest.mark.parametrize("I", [33, 1003, 1273, 2049, 4099])
@pytest.mark.parametrize("M", [2, 3, 7, 16])
def test_ragged_rows_quantised_inside_the_kernel_for_few_rows(M, I):
    """Rows that start anywhere, a short last block, a last stage of a split with a part: bit by bit the product of the blob.  What lies
    behind the last row is NaN."""
    g = torch.Generator().manual_seed(7)
    buf = torch.full((M * I + 64,), float("nan"), dtype=torch.bfloat16, device="cuda")
    x = buf[:M * I].view(M, I)
    x.copy_(torch.randn(M, I, generator=g) * torch.exp2(torch.randint(-3, 4, (M, 1), generator=g).float()))
    w = torch.randn(200, I, generator=g).to(torch.bfloat16)
    wq, xq = npas.quantize_mx(w.cuda()), npas.quantize_mx(x)
    xv, wv = mx.values(x.double().cpu().numpy()), mx.values(w.double().numpy())
    ref, size = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    for path, variant in [(0, 0)] + SPLITS:
        y = npas.linear_mx(x, wq, out_dtype=torch.float32, quantize_x=True, path=path, variant=variant)
        # (products exact, each of the I additions off by a step of the sum of magnitudes at most)
        assert (np.abs(y.double().cpu().numpy() - ref) <= I * 2.0 ** -23 * size).all(), (path, variant)
        if path:
            assert torch.equal(y, npas.linear_mx(xq, wq, out_dtype=torch.float32, path=path, variant=variant)), variant
        z = npas.linear_mx(x, wq, quantize_x=True, path=path, variant=variant)
        assert torch.equal(z, y.to(torch.bfloat16)), (path, variant)


# powers of two of a row's blocks: codes 0, 1, 2, 126 to 129, 251, 252 (bf16's largest numbers)
ENDS = [-127, -126, -125, -1, 0, 1, 2, 124, 125]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,I,O", [(9, 96, 18), (9, 520, 36), (45, 520, 136), (153, 264, 264), (603, 96, 45)])
def test_ends_of_the_scale_range(M, I, O, kind):
    """Rows of weights and of inputs at the ends of the range against one another: wherever the sum's parts are numbers that fp32 holds
    exactly, the result is the exact one.  (The smallest elements of code 0 are 2^-128, subnormal as bf16.)"""
    powers = lambda rows: torch.tensor(ENDS, dtype=torch.float64, device="cuda")[torch.arange(rows, device="cuda") % len(ENDS)][:, None]
    x, w = _members(M, I, 8, 0, 0) * torch.exp2(powers(M)), _members(O, I, 9, 0, 0) * torch.exp2(powers(O))
    xb, wb = x.to(torch.bfloat16), w.to(torch.bfloat16)
    assert torch.equal(xb.double(), x) and torch.equal(wb.double(), w)
    wq = npas.quantize_mx(wb)
    assert torch.equal(npas.dequantize_mx(wq), wb)
    want, size = x @ w.T, x.abs() @ w.abs().T
    # least product 2^(s + t - 2), all of them together below 2^24 of it and below 2^127; fp32 holds multiples of 2^-126 as normal numbers
    power = powers(M) + powers(O).T
    exact = (power - 2 >= -126) & (size < 2.0 ** 127) & (size < torch.exp2(power + 22))
    assert int(exact.sum()) * 3 > exact.numel()
    xin = npas.quantize_mx(xb) if kind == "blob" else xb
    for path, variant in _calls(M, wq, kind, EVERY, torch.float32):
        y = npas.linear_mx(xin, wq, out_dtype=torch.float32, quantize_x=kind == "44", path=path, variant=variant)
        assert torch.equal(y.double()[exact], want[exact]), (path, variant)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,I,O", [(5, 320, 200), (16, 1003, 131), (140, 320, 200), (300, 96, 333)])
def test_relu_turns_a_nan_sum_into_zero(M, I, O, kind, out_dtype):
    x, w = _members(M, I, 10), _members(O, I, 11)
    res = torch.randint(-8, 9, (M, O), device="cuda").to(out_dtype)
    want = (x @ w.T + res.double()).relu().to(out_dtype)
    xb = x.to(torch.bfloat16)
    xb[1, 3] = float("nan")
    want[1] = 0
    wb = w.to(torch.bfloat16)
    wb[7, I - 1] = float("nan")
    want[:, 7] = 0
    res[2, 9] = float("nan")
    want[2, 9] = 0
    res[3, 9], res[3, 10] = float("inf"), float("-inf")
    want[3, 9], want[3, 10] = float("inf"), 0
    wq = npas.quantize_mx(wb)
    xin = npas.quantize_mx(xb) if kind == "blob" else xb
    for path, variant in _calls(M, wq, kind, EVERY, out_dtype):
        y = npas.linear_mx(xin, wq, None, res, relu=True, out_dtype=out_dtype, quantize_x=kind == "44", path=path, variant=variant)
        assert torch.equal(y, want), (path, variant)


def _at(t, odd):
    """A copy of t that starts `odd` times 16 bytes behind a boundary of 512."""
    n = 16 * odd // t.element_size()
    buf = torch.empty(t.numel() + n, dtype=t.dtype, device="cuda")
    v = buf[n:].view(t.shape)
    v.copy_(t)
    assert v.data_ptr() % 512 == 16 * odd
    return v


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,I,O", [(3, 264, 136), (16, 8192, 72), (130, 264, 136), (300, 1003, 131), (4000, 64, 256)])
def test_buffers_on_16_byte_boundaries(M, I, O, kind, out_dtype):
    x, w = _members(M, I, 12), _members(O, I, 13)
    res, bias = torch.randint(-8, 9, (M, O), device="cuda").to(out_dtype), torch.randint(-8, 9, (O,), device="cuda").float()
    want = (x @ w.T + bias + res.double()).to(out_dtype)
    xb, wq = _at(x.to(torch.bfloat16), 1), npas.quantize_mx(_at(w.float(), 1))
    wq = npas.MxBlob(_at(wq.data, 3), wq.desc)
    xin = npas.quantize_mx(xb) if kind == "blob" else xb
    if kind == "blob":
        xin = npas.MxBlob(_at(xin.data, 5), xin.desc)
    for path, variant in _calls(M, wq, kind, EVERY, out_dtype):
        ws = _at(npas.linear_mx_workspace(M, wq, dtype="mx" if kind == "blob" else torch.bfloat16, quantize_x=kind == "44", out_dtype=out_dtype, path=path,
                                          variant=variant), 7)
        out = _at(torch.zeros(M, O, dtype=out_dtype, device="cuda"), 1)
        y = npas.linear_mx(xin, wq, _at(bias, 1), _at(res, 3), out=out, out_dtype=out_dtype, quantize_x=kind == "44", ws=ws, path=path, variant=variant)
        assert y is out and torch.equal(out, want), (path, variant)
        npas.check_device_status(ws)


def test_one_workspace_serves_smaller_calls():
    """A workspace for many rows takes every call of fewer."""
    w = npas.quantize_mx(_members(200, 1003, 14).to(torch.bfloat16))
    x = _members(500, 1003, 15).to(torch.bfloat16)
    for q in (False, True):
        ws = npas.linear_mx_workspace(500, w, quantize_x=q)
        want = npas.linear_mx(x, w, quantize_x=q, out_dtype=torch.float32)
        for M in (500, 300, 129, 128, 17, 16, 2, 1):
            y = npas.linear_mx(x[:M].contiguous(), w, quantize_x=q, out_dtype=torch.float32, ws=ws)
            assert torch.equal(y, want[:M]), (M, q)


def test_two_streams_of_split_calls_at_once():
    """Clusters of two calls share the SMs: each has its own workspace and its own results."""
    shapes = [(16, 4096, 900), (16, 2049, 500)]
    jobs = []
    for i, (M, I, O) in enumerate(shapes):
        x, w = _members(M, I, 16 + i), _members(O, I, 18 + i)
        xb, wq = x.to(torch.bfloat16), npas.quantize_mx(w.to(torch.bfloat16))
        jobs.append((xb, npas.quantize_mx(xb), wq, (x @ w.T).float(), npas.linear_mx_workspace(M, wq, quantize_x=True, path=3), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(30):
        for xb, xq, wq, want, ws, st in jobs:
            with torch.cuda.stream(st):
                for v in (2, 4, 8):
                    got.append((npas.linear_mx(xb, wq, out_dtype=torch.float32, quantize_x=True, ws=ws, path=3, variant=v), want))
                    got.append((npas.linear_mx(xq, wq, out_dtype=torch.float32, ws=ws, path=3, variant=v), want))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y, want in got)
    for job in jobs:
        npas.check_device_status(job[4])
