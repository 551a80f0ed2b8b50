"""Quantisation to microscaled 4-bit floating point and back on the GPU, bit by bit against the oracle: sizes that end inside a block or a tile,
the ends of the range, zeros and their signs, infinities and NaN, other streams, capture, repeated calls."""
import numpy as np
import pytest
import torch

import paper_2012_00596_b200 as npas
from oracle import mx

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _matrix(rows, cols, dtype, seed=1, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * sigma
    x *= torch.exp2(torch.randint(-6, 7, (rows, 1), generator=g).float())
    return x.to(DTYPES[dtype])


def _check(x, out_dtype=torch.float32):
    b = npas.quantize_mx(x.cuda())
    npas.blob_check(b)
    codes, scales = mx.encode(x.double().numpy())
    assert np.array_equal(b.data.cpu().numpy(), mx.blob(codes, scales))
    v = npas.dequantize_mx(b, dtype=out_dtype)
    assert v.dtype == out_dtype and tuple(v.shape) == tuple(x.shape)
    want = mx.decode(codes, scales)
    got = v.double().cpu().numpy()
    assert np.array_equal(got, want, equal_nan=True)
    assert np.array_equal(np.signbit(got)[~np.isnan(want)], np.signbit(want)[~np.isnan(want)])
    return b


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (1, 32), (3, 33), (127, 64), (128, 128), (129, 129), (257, 40), (33, 1003), (1, 2048), (200, 520),
                                       (64, 8191)])
def test_every_bit_matches_the_oracle(rows, cols, dtype):
    _check(_matrix(rows, cols, dtype, seed=rows + cols))
    _check(_matrix(rows, cols, dtype, seed=rows, sigma=0.02), torch.bfloat16)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_borders_and_signs(dtype):
    m = np.array([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0])
    rows = []
    for s in (-126, -100, -20, -1, 0, 3, 40, 124):
        for nudge in (1.0, 1.0 + 2.0 ** -7, 1.0 - 2.0 ** -8):
            row = np.concatenate([m * nudge, -m * nudge])
            row[12] = 4.0                                           # the block's scale stays 2^s
            rows.append(row * 2.0 ** s)
    _check(torch.from_numpy(np.array(rows)).to(DTYPES[dtype]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ends_of_the_range(dtype):
    top = torch.finfo(DTYPES[dtype]).max
    tiny = 2.0 ** -149 if dtype == "f32" else 2.0 ** -133
    x = torch.zeros(8, 96, dtype=torch.float64)
    x[0, 0], x[0, 40], x[1, 5], x[2, 33] = top, -top, tiny, -tiny
    x[3, :32] = 2.0 ** -126 * torch.linspace(-1, 1, 32)
    x[4, 0], x[4, 1] = top, tiny
    x[5, 0], x[5, 1] = 2.0 ** -124, 2.0 ** -127
    x[6] = -0.0
    _check(x.to(DTYPES[dtype]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_block_with_an_infinity_or_nan_is_nan_alone(dtype):
    x = _matrix(130, 100, "f32", seed=8)
    x[0, 3], x[64, 40], x[129, 99], x[5, 31] = float("inf"), float("nan"), -float("inf"), float("nan")
    _check(x.to(DTYPES[dtype]))
    _check(x.to(DTYPES[dtype]), torch.bfloat16)


def test_values_are_their_own_values():
    x = _matrix(300, 260, "bf16", seed=4).cuda()
    v = npas.dequantize_mx(npas.quantize_mx(x))
    assert torch.equal(npas.dequantize_mx(npas.quantize_mx(v)), v)
    assert torch.equal(npas.quantize_mx(v).data, npas.quantize_mx(npas.dequantize_mx(npas.quantize_mx(x), torch.float32)).data)


def test_pruned_weights_stay_zero():
    w = _matrix(128, 128, "bf16", seed=5, sigma=0.02).cuda()
    rk, ck = npas.prune_bb_magnitude(w, 64, 64, 32, 32)
    kept = npas.unpack_bb(npas.pack_bb(w, rk, ck, 64, 64))[0]
    v = npas.dequantize_mx(npas.quantize_mx(kept))
    assert (kept == 0).sum() >= 128 * 128 * 3 // 4 and bool((v[kept == 0] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 150, 5000])
def test_rows_that_start_anywhere(rows, dtype):
    """Every remainder of the columns: rows begin and end at every place of a 16-byte piece, inside a tile of columns and past one."""
    for cols in list(range(1, 18)) + [57, 62, 63, 64, 65] + list(range(121, 138)) + [257, 259, 262]:
        _check(_matrix(rows, cols, dtype, seed=cols), DTYPES[dtype])


def test_large_matrix_in_pieces():
    """70 000 rows: row tiles past 2^9, values past 16 MB; every 128-row piece equals the quantised piece."""
    x = torch.randn(70001, 512, device="cuda").to(torch.bfloat16)
    v = npas.dequantize_mx(npas.quantize_mx(x))
    for lo in (0, 128 * 300, 69888):
        piece = x[lo:lo + 128].contiguous()
        assert torch.equal(v[lo:lo + 128], npas.dequantize_mx(npas.quantize_mx(piece)))


def test_offsets_past_32_bits():
    """2^32 + elements: source, values and result lie past 4 GB."""
    rows = (2 ** 32 + 2 ** 20) // 4096
    x = torch.zeros(rows, 4096, dtype=torch.bfloat16, device="cuda")
    last = torch.randn(200, 4096, device="cuda").to(torch.bfloat16)
    x[-200:] = last
    v = npas.dequantize_mx(npas.quantize_mx(x))
    assert torch.equal(v[-200:], npas.dequantize_mx(npas.quantize_mx(last)))
    assert not bool(v[:128].any()) and not bool(v[2 ** 31 // 4096 - 64:2 ** 31 // 4096 + 64].any())


def test_streams_capture_and_repeats():
    x = _matrix(500, 300, "bf16", seed=6).cuda()
    want = npas.dequantize_mx(npas.quantize_mx(x))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = npas.dequantize_mx(npas.quantize_mx(x))
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = npas.dequantize_mx(npas.quantize_mx(x))
    for seed in (7, 8):
        x.copy_(_matrix(500, 300, "bf16", seed=seed))
        g.replay()
        assert torch.equal(out, npas.dequantize_mx(npas.quantize_mx(x)))


def test_refusals():
    x = _matrix(64, 64, "f32").cuda()
    for bad in (x.t()[:, ::2], x[:, :32], x[0], x.view(4, 16, 64)):
        with pytest.raises(AssertionError):
            npas.quantize_mx(bad)
    with pytest.raises(TypeError):
        npas.quantize_mx(x.half())
    with pytest.raises(npas.NpasError) as e:
        npas.quantize_mx(x[:0])
    assert e.value.code == 2
    with pytest.raises(npas.NpasError) as e:
        npas.quantize_mx(x.view(-1)[1:4033].view(63, 64))
    assert e.value.code == 4
    b = npas.quantize_mx(x)
    with pytest.raises(TypeError):
        npas.dequantize_mx(b, torch.float16)
    with pytest.raises(npas.NpasError) as e:
        npas.dequantize_mx(npas.MxBlob(b.data[:-128], b.desc))
    assert e.value.code == 7
    spoilt = npas.MxBlob(b.data.clone(), b.desc)
    spoilt.data[8] = 3
    with pytest.raises(npas.NpasError) as e:
        npas.blob_check(spoilt)
    assert e.value.code == 6


@pytest.mark.parametrize("rows,cols,dtype", [(262400, 16400, torch.bfloat16), (262400, 16397, torch.bfloat16), (140000, 16397, torch.float32)])
def test_many_elements_both_ways(rows, cols, dtype):
    """More than 2^31 elements (of bf16 2^32): the last rows, and those around 2^31 and 2^32 elements, come back as they do alone."""
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randint(-100, 101, (rows, cols), generator=g, device="cuda", dtype=torch.int8).to(dtype)
    y = npas.dequantize_mx(npas.quantize_mx(x), dtype)
    for lo in (0, 2 ** 31 // cols - 50, min(2 ** 32 // cols - 50, rows - 300), rows - 100):
        part = x[lo:lo + 100].clone()
        assert torch.equal(y[lo:lo + 100], npas.dequantize_mx(npas.quantize_mx(part), dtype)), lo
