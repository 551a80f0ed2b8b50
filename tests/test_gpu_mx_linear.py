"""Products with microscaled 4-bit weights on the GPU, every kernel, against the 64-bit oracle: sizes from one row to many, odd in every
direction, both kinds of input, epilogues, special values, streams, capture, shared workspaces, refusals.

Tolerance, derived: the products of elements are exact in fp32 (8 + 2 or 2 + 2 significant bits), each of the I + 3 additions (columns, bias,
residual) is off by at most one fp32 step of a partial sum, whose magnitude S = sum |x w| + |bias| + |residual| bounds:
(I + 3) 2^-23 S; then one rounding to the output type, half a step: 2^-8 of the value for bf16 (of a value that far off)."""
import numpy as np
import pytest
import torch

import paper_2012_00596_b200 as npas
from oracle import mx

pytestmark = pytest.mark.gpu


def _case(M, I, O, seed=1, bias=True, res=True, res_dtype=torch.bfloat16, spread=2):
    g = torch.Generator().manual_seed(seed)
    def scaled(rows, sigma):
        x = torch.randn(rows, I, generator=g) * sigma
        n = -(-I // 32)
        e = torch.randint(-spread, spread + 1, (rows, n), generator=g).float()
        return (x * torch.exp2(e).repeat_interleave(32, 1)[:, :I]).to(torch.bfloat16)
    c = dict(x=scaled(M, 1.0), w=scaled(O, 0.05))
    c["bias"] = torch.randn(O, generator=g) * 0.2 if bias else None
    c["res"] = torch.randn(M, O, generator=g).to(res_dtype) if res else None
    return c


def _paths(M, w, **kw):
    """Every kernel that takes the call, the automatic choice first."""
    out = [0]
    for path in npas.LINEAR_MX_KERNELS:
        try:
            npas.linear_mx_kernel(M, w, path=path, **kw)
            out.append(path)
        except npas.NpasError as e:
            assert e.code == 8
    return out


def _reference(c, kind, relu):
    x = c["x"].double().numpy()
    x = x if kind == "16" else mx.values(x)
    w = mx.values(c["w"].double().numpy())
    b = None if c["bias"] is None else c["bias"].double().numpy()
    r = None if c["res"] is None else c["res"].double().numpy()
    size = np.abs(x) @ np.abs(w).T + (0 if b is None else np.abs(b)) + (0 if r is None else np.abs(r))
    return mx.linear(x, w, b, r, relu), size


def _close(y, ref, size, I, what=""):
    eps = 2.0 ** -8 if y.dtype == torch.bfloat16 else 0.0
    got = y.double().cpu().numpy()
    off = (I + 3) * 2.0 ** -23 * size
    assert np.isfinite(got).all(), what
    over = np.abs(got - ref) - (off + eps * (np.abs(ref) + off) + 2.0 ** -133)
    assert over.max() <= 0, (what, float(over.max()), np.unravel_index(over.argmax(), over.shape))


def _run(M, I, O, kind, out_dtype=torch.bfloat16, relu=False, bias=True, res=True, seed=1, paths=None, spread=2):
    c = _case(M, I, O, seed, bias, res, out_dtype, spread)
    dev = {k: None if v is None else v.cuda() for k, v in c.items()}
    w = npas.quantize_mx(dev["w"])
    ref, size = _reference(c, kind, relu)
    x = npas.quantize_mx(dev["x"]) if kind == "blob" else dev["x"]
    q = kind == "44"
    kw = dict(dtype="mx" if kind == "blob" else torch.bfloat16, quantize_x=q, out_dtype=out_dtype, bias=bias, residual=res, relu=relu)
    for path in paths or _paths(M, w, **kw):
        ws = npas.linear_mx_workspace(M, w, path=path, **kw)
        ws[256:] = 0xFF                                        # what lies in the scratch does not matter
        call = lambda: npas.linear_mx(x, w, dev["bias"], dev["res"], relu=relu, out_dtype=out_dtype, quantize_x=q, ws=ws, path=path)
        y = call()
        npas.check_device_status(ws)
        _close(y, ref, size, I, f"path {path}")
        assert torch.equal(y, call()), path
    return c


KINDS = ["44", "blob", "16"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,I,O", [(1, 32, 8), (1, 1, 1), (1, 2048, 1000), (2, 64, 128), (7, 96, 40), (16, 512, 256), (33, 1000, 77), (64, 2048, 130),
                                   (127, 40, 129), (128, 256, 128), (129, 264, 200), (200, 72, 512), (300, 1003, 301), (1000, 128, 64)])
def test_sizes(M, I, O, kind):
    _run(M, I, O, kind, relu=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bias,res,relu", [(False, False, False), (True, False, True), (False, True, False), (True, True, True)])
def test_epilogues(bias, res, relu, out_dtype, kind):
    _run(70, 200, 264, kind, out_dtype, relu, bias, res)
    _run(300, 128, 512, kind, out_dtype, relu, bias, res)
    _run(9, 1024, 96, kind, out_dtype, relu, bias, res)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,I,O", [(3136, 512, 2048), (5000, 64, 256), (2500, 1536, 300), (1, 8192, 4096), (700, 4096, 1000)])
def test_larger_sizes(M, I, O, kind):
    _run(M, I, O, kind, relu=True, seed=3)


@pytest.mark.parametrize("M,I,O", [(1, 8192, 1024), (9, 8000, 300), (3, 16384, 130), (16, 4999, 500), (8, 4096, 1), (2, 8200, 2048)])
def test_few_rows_of_few_outputs_and_many_columns(M, I, O):
    """A cluster splits the columns; the last part may be shorter, or have no tile for some warps."""
    _run(M, I, O, "16", relu=True, seed=8, spread=1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M", list(range(1, 18)) + [24, 31, 32, 40, 63, 65, 96, 120, 136, 192, 255, 257])
def test_every_count_of_rows(M, kind):
    _run(M, 160, 144, kind, res=False)


@pytest.mark.parametrize("kind", KINDS)
def test_scales_far_apart(kind):
    """Neighbouring blocks of a row up to 2^24 apart; sums of one block only stay exact."""
    _run(40, 512, 96, kind, torch.float32, spread=12)


@pytest.mark.parametrize("kind", ["44", "blob"])
@pytest.mark.parametrize("M,I,O", [(3, 2048, 1000), (200, 256, 136)])
def test_sums_of_equal_scales_are_exact(M, I, O, kind):
    """Members of one scale: products are whole quarters, sums below 2^24 quarters, so fp32 results have no error at all."""
    g = torch.Generator().manual_seed(2)
    pick = lambda rows: torch.from_numpy(mx.MEMBERS)[torch.randint(0, 8, (rows, I), generator=g)] * (torch.randint(0, 2, (rows, I), generator=g) * 2 - 1)
    x, w = pick(M), pick(O)
    x[:, ::32], w[:, ::32] = 6.0, 4.0
    wq = npas.quantize_mx(w.to(torch.bfloat16).cuda())
    xb = x.to(torch.bfloat16).cuda()
    ref = (x @ w.T).float()
    for path in _paths(M, wq, quantize_x=True, out_dtype=torch.float32):
        y = npas.linear_mx(npas.quantize_mx(xb) if kind == "blob" else xb, wq, out_dtype=torch.float32, quantize_x=kind == "44", path=path)
        assert torch.equal(y.cpu(), ref), path


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,I,O", [(5, 320, 200), (140, 320, 200)])
def test_infinities_and_nan_stay_in_their_rows(M, I, O, kind):
    c = _case(M, I, O, seed=5, res=False)
    dev = {k: None if v is None else v.cuda() for k, v in c.items()}
    wbad = dev["w"].clone()
    wbad[7, 100] = float("nan")
    xbad = dev["x"].clone()
    xbad[3, 40], xbad[1, 319] = float("inf"), float("nan")
    w, wb = npas.quantize_mx(dev["w"]), npas.quantize_mx(wbad)
    for path in _paths(M, w, quantize_x=kind == "44", dtype="mx" if kind == "blob" else torch.bfloat16):
        f = lambda x, w: npas.linear_mx(npas.quantize_mx(x) if kind == "blob" else x, w, dev["bias"], quantize_x=kind == "44", path=path)
        clean, got = f(dev["x"], w), f(xbad, wb)
        rows = torch.ones(M, dtype=torch.bool, device="cuda")
        cols = torch.ones(O, dtype=torch.bool, device="cuda")
        rows[[1, 3]], cols[7] = False, False
        assert torch.equal(got[rows][:, cols], clean[rows][:, cols]), path
        assert bool(got[1].isnan().all()) and bool(got[:, 7].isnan().all()) and not bool(got[3].isfinite().any()), path


def test_single_row_equals_the_row_of_a_batch_in_exact_arithmetic():
    """Small whole numbers: every order of the sums gives the same result, so kernels for one row and for many agree bit by bit."""
    g = torch.Generator().manual_seed(9)
    x = torch.randint(-3, 4, (600, 512), generator=g).to(torch.bfloat16).cuda()
    w = npas.quantize_mx(torch.randint(-4, 5, (256, 512), generator=g).to(torch.bfloat16).cuda())
    for q in (False, True):
        full = npas.linear_mx(x, w, quantize_x=q, out_dtype=torch.float32)
        for n in (1, 5, 17, 64, 130):
            assert torch.equal(npas.linear_mx(x[:n].contiguous(), w, quantize_x=q, out_dtype=torch.float32), full[:n])


@pytest.mark.parametrize("kind,M,I,O,out_dtype,res", [("blob", 264000, 32, 8200, torch.bfloat16, True), ("16", 264000, 32, 8200, torch.bfloat16, False),
                                                     ("44", 264000, 32, 8195, torch.bfloat16, True), ("16", 264000, 32, 8195, torch.float32, False),
                                                     ("16", 264000, 8195, 40, torch.bfloat16, False), ("44", 264000, 8200, 40, torch.bfloat16, False)])
def test_offsets_past_32_bits(kind, M, I, O, out_dtype, res):
    """Whole numbers: the last rows of inputs and outputs of more than 2^31 elements are those of a call of them alone."""
    g = torch.Generator(device="cuda").manual_seed(4)
    few = lambda lo, hi, *size: torch.randint(lo, hi, size, generator=g, device="cuda", dtype=torch.int8)
    x, w = few(-2, 3, M, I).to(torch.bfloat16), npas.quantize_mx(few(-2, 3, O, I).to(torch.bfloat16))
    r = few(-2, 3, M, O).to(out_dtype) if res else None
    f = lambda x, r: npas.linear_mx(npas.quantize_mx(x) if kind == "blob" else x, w, None, r, out_dtype=out_dtype, quantize_x=kind == "44")
    y = f(x, r)
    assert y.numel() > 2 ** 31 or x.numel() > 2 ** 31
    for lo, n in ((M - 300, 300), (M - 1, 1), (2 ** 31 // max(I, O), 200), (0, 100)):
        assert torch.equal(y[lo:lo + n], f(x[lo:lo + n].clone(), None if r is None else r[lo:lo + n].clone())), lo


def test_rows_behind_the_last_are_left_alone():
    for M, O in ((1, 40), (33, 129), (200, 264), (5, 1001)):
        c = _case(M, 96, O, res=False)
        w = npas.quantize_mx(c["w"].cuda())
        for q in (False, True):
            for path in _paths(M, w, quantize_x=q):
                buf = torch.full(((M + 3) * O + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
                npas.linear_mx(c["x"].cuda(), w, out=buf[:M * O].view(M, O), quantize_x=q, path=path)
                assert bool((buf[M * O:] == 7.0).all()), (M, O, q, path)


def test_a_run_of_them_prune_pack_quantise_and_two_layers():
    """Weights pruned by magnitude, packed, unpacked and quantised; two layers with a shortcut; against the oracle layer by layer."""
    g = torch.Generator().manual_seed(12)
    M, I, H = 196, 256, 512
    ws, vals = [], []
    for rows, cols in ((H, I), (I, H)):
        w = (torch.randn(rows, cols, generator=g) * 0.05).to(torch.bfloat16).cuda()
        rk, ck = npas.prune_bb_magnitude(w, 64, 64, 48, 48)
        kept, _, _ = npas.unpack_bb(npas.pack_bb(w, rk, ck, 64, 64))
        ws.append(npas.quantize_mx(kept))
        vals.append(mx.values(kept.double().cpu().numpy()))
    x = torch.randn(M, I, generator=g).relu().to(torch.bfloat16)
    b = torch.randn(H, generator=g) * 0.1
    scratch = npas.linear_mx_workspace(M, ws[1], quantize_x=True)
    h = npas.linear_mx(x.cuda(), ws[0], b.cuda(), relu=True, quantize_x=True, ws=scratch)
    y = npas.linear_mx(h, ws[1], None, x.cuda(), relu=True, quantize_x=True, ws=scratch)
    npas.check_device_status(scratch)
    xv, hv = mx.values(x.double().numpy()), mx.values(h.double().cpu().numpy())
    _close(h, mx.linear(xv, vals[0], b.double().numpy(), relu=True), np.abs(xv) @ np.abs(vals[0]).T + b.abs().numpy(), I)
    r = x.double().numpy()
    _close(y, mx.linear(hv, vals[1], None, r, relu=True), np.abs(hv) @ np.abs(vals[1]).T + np.abs(r), H)
    # the same weights with 16-bit inputs behind a pruned bf16 layer of the library
    z = npas.linear_mx(h, ws[1], None, x.cuda(), relu=True)
    h64 = h.double().cpu().numpy()
    _close(z, mx.linear(h64, vals[1], None, r, relu=True), np.abs(h64) @ np.abs(vals[1]).T + np.abs(r), H)


@pytest.mark.parametrize("M", [3, 300])
@pytest.mark.parametrize("q", [False, True])
def test_streams_capture_and_workspaces(M, q):
    c = _case(M, 520, 264, res=False)
    x, w, bias = c["x"].cuda(), npas.quantize_mx(c["w"].cuda()), c["bias"].cuda()
    f = lambda ws=None: npas.linear_mx(x, w, bias, quantize_x=q, ws=ws)
    want = f()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [f() for _ in range(3)]
    mine = [f() for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(t, want) for t in got + mine)
    ws = npas.linear_mx_workspace(M, w, quantize_x=q)
    graphs = []
    for own in (None, ws, ws):                     # (two graphs on one workspace: replayed on one stream)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = f(own)
        graphs.append((g, y))
    for seed in (21, 22):
        x.copy_(_case(M, 520, 264, seed, res=False)["x"])
        for g, y in graphs:
            y.zero_()
        for g, y in graphs:
            g.replay()
        want = f()
        assert all(torch.equal(y, want) for _, y in graphs)
    npas.check_device_status(ws)


def test_blob_and_input_written_just_ahead_of_the_call():
    """What the call reads is written by a kernel of the library right ahead of it on the stream."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for M in (1, 24, 400):
        for _ in range(5):
            x = torch.randn(M, 256, device="cuda", generator=g).to(torch.bfloat16)
            w = torch.randn(192, 256, device="cuda", generator=g).to(torch.bfloat16)
            torch.cuda.synchronize()
            for q in (False, True):
                once = npas.linear_mx(x, npas.quantize_mx(w), quantize_x=q)
                wq = npas.quantize_mx(w)
                torch.cuda.synchronize()
                assert torch.equal(once, npas.linear_mx(x, wq, quantize_x=q))
                twice = npas.linear_mx(npas.quantize_mx(x), npas.quantize_mx(w))
                torch.cuda.synchronize()
                assert torch.equal(twice, npas.linear_mx(x, wq, quantize_x=True))


def test_refusals():
    c = _case(4, 64, 32)
    x, w, bias, res = c["x"].cuda(), npas.quantize_mx(c["w"].cuda()), c["bias"].cuda(), c["res"].cuda()
    for bad in (dict(x=x.t()), dict(x=x[0]), dict(bias=bias.to(torch.bfloat16)), dict(bias=bias[:16]), dict(residual=res.float()), dict(residual=res[:2]),
                dict(out=torch.empty(4, 31, device="cuda", dtype=torch.bfloat16)), dict(out=torch.empty(4, 32, device="cuda"), out_dtype=torch.bfloat16),
                dict(bias=bias.cpu()), dict(ws=torch.zeros(256, dtype=torch.uint8))):
        kw = dict(x=x, bias=None, residual=None)
        kw.update(bad)
        with pytest.raises(AssertionError):
            npas.linear_mx(kw.pop("x"), w, kw.pop("bias"), kw.pop("residual"), **kw)
    for bad, code in ((dict(x=x.float()), 3), (dict(x=c["x"].cuda()[:, :32].contiguous()), 2), (dict(x=x[:0]), 2), (dict(path=77), 8),
                      (dict(x=torch.zeros(400, 64, dtype=torch.bfloat16, device="cuda"), ws=npas.workspace(), quantize_x=True), 7), (dict(x=npas.quantize_mx(x), quantize_x=True), 3), (dict(out=x.view(-1)[:128].view(4, 32)), 8)):
        kw = dict(x=x)
        kw.update(bad)
        with pytest.raises(npas.NpasError) as e:
            npas.linear_mx(kw.pop("x"), w, **kw)
        assert e.value.code == code, bad
    with pytest.raises(TypeError):
        npas.linear_mx(x, w, out_dtype=torch.float16)


@pytest.mark.parametrize("kind,path,variant", [("blob", 4, 128), ("blob", 4, 256), ("blob", 5, 0), ("16", 4, 128), ("16", 4, 256)])
@pytest.mark.parametrize("M,I,O,res", [(1939, 585, 3768, False), (2500, 2112, 128, True), (4867, 640, 560, True), (1300, 2304, 3128, True), (9000, 64, 328, False),
                                       (20000, 40, 72, True), (1939, 96, 333, True), (3000, 640, 131, False), (30000, 64, 257, True), (700, 64, 1, True),
                                       (9000, 40, 7, False), (2500, 2304, 1130, True)])
def test_outputs_that_end_inside_a_tile_many_times(M, I, O, res, kind, path, variant):
    """Tiles with one half of 64 outputs between tiles with two, blocks of rows that end inside a tile: the order of the slabs shifts
    between the warps that fill them.  Every run has to give the same bits."""
    c = _case(M, I, O, seed=31, res=res)
    x, w = c["x"].cuda(), npas.quantize_mx(c["w"].cuda())
    x = npas.quantize_mx(x) if kind == "blob" else x
    bias, r = c["bias"].cuda(), c["res"].cuda() if res else None
    ws = npas.linear_mx_workspace(M, w, dtype="mx" if kind == "blob" else torch.bfloat16, path=path, variant=variant)
    f = lambda: npas.linear_mx(x, w, bias, r, relu=True, ws=ws, path=path, variant=variant)
    y = f()
    npas.check_device_status(ws)
    xv = npas.dequantize_mx(x, torch.float32) if kind == "blob" else x.float()
    wv = npas.dequantize_mx(w, torch.float32)
    ref = xv.double() @ wv.double().T + bias.double() + (r.double() if res else 0)
    size = xv.abs().double() @ wv.abs().double().T + bias.abs().double() + (r.abs().double() if res else 0)
    off = (I + 3) * 2.0 ** -23 * size
    over = (y.double() - ref.relu()).abs() - (off + 2.0 ** -8 * (ref.abs() + off))
    assert float(over.max()) <= 0
    for _ in range(20):
        assert torch.equal(f(), y)
    npas.check_device_status(ws)
