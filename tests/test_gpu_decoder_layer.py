"""The example decoder layer (matmuls, paged cache, attention, norms) against the layer in
32-bit torch on the same dequantised weights.

Tolerance: along the path about ten results are rounded to bf16 (2^-8 at most, 2^-9 in the
mean square at most), each feeding the next: 10 x 2^-9 = 2e-2 of the outputs' norm.  A cache
of 8 bits adds a step of 1/255 of a row's range of about 6 deviations, 0.7 % in the mean
square, of 4 bits 12 %; they reach the residual stream through attention, whose output is
a smaller part of it than the input, averaged over the keys."""

import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(ROOT, "examples", "decoder_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("window,sinks", [(0, 0), (48, 4)])
@pytest.mark.parametrize("kind,most", [("bf16", 2e-2), ("int8", 2.7e-2), ("int4", 0.14)])
def test_decoder_layer(gpu_lib, example, kind, most, window, sinks):
    print(f"decoder layer {kind} window {window} sinks {sinks}", flush=True)
    got, want = example.run(kind=kind, window=window, sinks=sinks)
    torch.cuda.synchronize()
    for (x, h), (px, ph) in zip(got, want):
        assert x.shape == px.shape and h.shape == ph.shape
        for u, v in ((x, px), (h, ph)):
            off = ((u.float() - v).norm() / v.norm()).item()
            assert off <= most, (kind, off)
