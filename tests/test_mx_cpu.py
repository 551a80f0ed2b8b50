"""Host side of the 4-bit entry points (CPU): sizes, refusals, the choice of a kernel; no kernel is launched here."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2012_00596_b200 as npas
from oracle import mx
from paper_2012_00596_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def _p(v):
    return ctypes.c_void_p(v)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (127, 33), (128, 128), (129, 129), (1000, 2048), (5, 1003)])
def test_size_is_that_of_the_oracles_blob(lib, rows, cols):
    n = ctypes.c_size_t(0)
    d = binding.MxDesc(rows, cols, 1)
    assert lib.npas_quantize_mx_size(ctypes.byref(d), ctypes.byref(n)) == 0
    assert n.value == mx.blob(np.zeros((rows, cols), np.uint8), np.zeros((rows, -(-cols // 32)), np.uint8)).size


def test_size_passes_32_bits(lib):
    n = ctypes.c_size_t(0)
    d = binding.MxDesc(2 ** 31 - 1, 32, 1)
    assert lib.npas_quantize_mx_size(ctypes.byref(d), ctypes.byref(n)) == 0
    assert n.value == 128 + 2 ** 24 * 512 + -(-(2 ** 31 - 1) * 16 // 128) * 128


@pytest.mark.parametrize("desc,code", [((0, 32, 1), 2), ((4, 0, 1), 2), ((-1, 32, 0), 2), ((4, 2 ** 20 + 1, 0), 2), ((2 ** 31 - 1, 2 ** 20, 1), 2),
                                       ((4, 32, 2), 3), ((4, 32, 7), 3)])
def test_descriptors_that_are_refused(lib, desc, code):
    n = ctypes.c_size_t(0)
    assert lib.npas_quantize_mx_size(ctypes.byref(binding.MxDesc(*desc)), ctypes.byref(n)) == code


def test_quantising_calls_refuse_bad_arguments(lib):
    d = binding.MxDesc(4, 64, 0)
    r, null, n = ctypes.byref(d), _p(0), ctypes.c_size_t
    assert lib.npas_quantize_mx_size(None, ctypes.byref(n(0))) == 1 and lib.npas_quantize_mx_size(r, None) == 1
    assert lib.npas_quantize_mx(r, null, _p(4096), n(1 << 20), null) == 1
    assert lib.npas_quantize_mx(r, _p(4096), null, n(1 << 20), null) == 1
    assert lib.npas_quantize_mx(r, _p(4104), _p(8192), n(1 << 20), null) == 4
    assert lib.npas_quantize_mx(r, _p(4096), _p(8200), n(1 << 20), null) == 4
    assert lib.npas_quantize_mx(r, _p(4096), _p(8192), n(767), null) == 7
    assert lib.npas_quantize_mx(r, _p(4096), _p(4096), n(1 << 20), null) == 8
    assert lib.npas_dequantize_mx(r, _p(4096), n(768), 2, _p(8192), null) == 3
    assert lib.npas_dequantize_mx(r, _p(4096), n(767), 0, _p(8192), null) == 7
    assert lib.npas_dequantize_mx(r, null, n(768), 0, _p(8192), null) == 1
    assert lib.npas_dequantize_mx(r, _p(4096), n(768), 0, _p(8196), null) == 4
    assert lib.npas_mx_blob_check(r, null, n(768), null) == 1
    assert lib.npas_mx_blob_check(r, _p(4096), n(100), null) == 7


def _linear(lib, ws=256, x=4096, w=8192, bias=0, res=0, y=16384, wsp=32768, **kw):
    f = dict(M=4, I=64, O=16, x_dtype=1, quantize_x=0, y_dtype=1, relu=0, has_bias=0, has_residual=0, path=0, variant=0)
    f.update(kw)
    d = binding.MxLinearDesc(*(f[n] for n, _ in binding.MxLinearDesc._fields_))
    return lib.npas_linear_mx(ctypes.byref(d), _p(x), _p(w), _p(bias), _p(res), _p(y), _p(wsp), ctypes.c_size_t(ws), _p(0))


@pytest.mark.parametrize("kw,code", [
    (dict(x=0), 1), (dict(w=0), 1), (dict(y=0), 1), (dict(wsp=0), 1), (dict(has_bias=1), 1), (dict(has_residual=1), 1),
    (dict(M=0), 2), (dict(M=2 ** 31 - 255), 2), (dict(O=2 ** 31 - 1), 2), (dict(I=0), 2), (dict(O=-4), 2), (dict(I=2 ** 20 + 1), 2),
    (dict(x_dtype=0), 3), (dict(x_dtype=2, quantize_x=1), 3), (dict(y_dtype=2), 3),
    (dict(x=4104), 4), (dict(w=8200), 4), (dict(y=16392), 4), (dict(has_bias=1, bias=20), 4), (dict(has_residual=1, res=24), 4),
    (dict(ws=255), 7), (dict(quantize_x=1, M=400), 7), (dict(y=4096), 8), (dict(y=8192), 8), (dict(has_residual=1, res=16384), 8), (dict(path=99), 8)])
def test_products_refuse_bad_arguments(lib, kw, code):
    assert _linear(lib, **kw) == code


def test_workspace_holds_the_quantised_input(lib):
    w = npas.MxBlob(torch.empty(1, dtype=torch.uint8), binding.MxDesc(1000, 2048, 1))
    n = npas.linear_mx_workspace(64, w, quantize_x=True).numel()
    size = ctypes.c_size_t(0)
    assert lib.npas_quantize_mx_size(ctypes.byref(binding.MxDesc(64, 2048, 1)), ctypes.byref(size)) == 0
    assert n >= 256 + size.value


def test_binding_refuses_tensors_off_the_gpu(lib):
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    blob = npas.MxBlob(torch.zeros(4096, dtype=torch.uint8), binding.MxDesc(16, 64, 1))
    for call in (lambda: npas.quantize_mx(x), lambda: npas.dequantize_mx(blob), lambda: npas.linear_mx(x, blob)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(TypeError):
        npas.quantize_mx(np.zeros((4, 64), np.float32))
    with pytest.raises(npas.NpasError) as e:
        npas.dequantize_mx(npas.MxBlob(torch.zeros(10, dtype=torch.uint8), binding.MxDesc(0, 64, 1)))
    assert e.value.code == 2
    with pytest.raises(TypeError):
        npas.linear_mx(x, npas.MxBlob(blob.data, binding.BbDesc()))
