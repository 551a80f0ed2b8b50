"""The choice of a kernel for products of 4-bit weights under a forced path, and the device that the queries ask about (CPU)."""
import pytest
import torch

import paper_2012_00596_b200 as npas
from paper_2012_00596_b200 import binding, build

TENSOR_CORE = {3, 4, 5}                       # the kernels that issue tcgen05 MMAs


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.load()


def _weights(O, I):
    return npas.MxBlob(torch.empty(1, dtype=torch.uint8), binding.MxDesc(O, I, 1))


@pytest.mark.parametrize("dtype,quantize", [(torch.bfloat16, False), (torch.bfloat16, True), ("mx", False)])
@pytest.mark.parametrize("I,O", [(64, 32), (129, 1000), (2048, 1000), (8192, 1024), (1003, 77)])
@pytest.mark.parametrize("M", [1, 8, 9, 16, 17, 300, 5000])
def test_path_2_names_tcgen05_kernels_only(M, I, O, dtype, quantize):
    kid = npas.linear_mx_kernel(M, _weights(O, I), dtype=dtype, quantize_x=quantize, path=2)
    assert kid in TENSOR_CORE
    free = npas.linear_mx_kernel(M, _weights(O, I), dtype=dtype, quantize_x=quantize)
    assert free == kid or free not in TENSOR_CORE            # the same choice where it is among them already


def test_queries_ask_about_the_blobs_device(monkeypatch):
    """The choice counts a device's SMs and a header is read in a stream's order: both of the device that holds the blob."""
    seen, inside = [], []

    class Device:
        def __init__(self, t):
            seen.append(t)

        def __enter__(self):
            inside.append(True)

        def __exit__(self, *a):
            inside.pop()

    class Library:
        def __getattr__(self, name):
            def call(*a):
                assert inside, name
                return 0
            return call

    monkeypatch.setattr(torch.cuda, "device_of", Device)
    monkeypatch.setattr(binding, "load", lambda: Library())
    monkeypatch.setattr(binding, "_stream", lambda: inside[0] and None)
    w = _weights(1000, 2048)
    npas.linear_mx_kernel(4, w)
    npas.linear_mx_workspace(4, w)
    npas.blob_check(w)
    assert len(seen) == 3 and all(t is w.data for t in seen)
