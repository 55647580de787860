"""CPU checks of the calls that surround a layer's products: what they refuse, before any GPU work."""
import ctypes

import pytest
import torch

from paper_2503_13565_amd import binding

P, Q, P2, P8 = (ctypes.c_void_p(v) for v in (4096, 1 << 20, 4098, 4104))    # fake pointers: 16-, 2- and 8-byte aligned, never followed
NONE, NULL, SHAPE, ALIGN, WORKSPACE, ARG = 0, 1, 2, 3, 4, 6


def norm(x=P, m=4, k=64, ldx=64, r=None, ldr=64, w=None, eps=1e-6, total=None, lds=64, y=P, ldy=64, q8=None, s=None):
    return binding.load().mxfp4_rms_norm(x, m, k, ldx, r, ldr, w, eps, total, lds, y, ldy, q8, s, None)


@pytest.mark.parametrize("what,code", [
    (dict(m=0, x=None, y=None), NONE), (dict(m=-1), SHAPE), (dict(k=0), SHAPE), (dict(k=60), SHAPE), (dict(k=131072, ldx=131072, ldy=131072), SHAPE),
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(y=None, q8=P), NULL), (dict(s=P), NULL), (dict(total=P), ARG),
    (dict(eps=-1.0), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG),
    (dict(ldx=56), SHAPE), (dict(ldx=68), ALIGN), (dict(x=P8), ALIGN), (dict(r=P8), ALIGN), (dict(r=P, ldr=56), SHAPE), (dict(r=P, ldr=65), ALIGN),
    (dict(r=P, total=P8), ALIGN), (dict(r=P, total=P, lds=8), SHAPE), (dict(y=P2), ALIGN), (dict(ldy=63), SHAPE), (dict(ldy=65), ALIGN),
    (dict(ldy=72), ARG), (dict(r=Q, ldr=72, y=Q), ARG), (dict(r=Q, total=P, lds=72, y=Q), ARG), (dict(r=Q, total=Q, lds=80), ARG), (dict(r=Q, total=P), ARG),
    (dict(w=P2), ALIGN), (dict(q8=P2, s=P), ALIGN), (dict(k=40, ldx=40, ldy=40, q8=P, s=P), SHAPE),
])
def test_norm_refusals(what, code):
    assert norm(**what) == code
    assert code == NONE or binding.load().mxfp4_last_error()


def product(x=P, xs=P, m=4, q=P, s=P, n=8, k=64, bias=None, act=0, r=None, ldr=8, y=P, ldy=8):
    return binding.load().mxfp4_w4a8_gemm(x, xs, m, q, s, n, k, bias, act, r, ldr, y, ldy, None)


@pytest.mark.parametrize("what,code", [
    (dict(m=0), SHAPE), (dict(n=0), SHAPE), (dict(k=0), SHAPE), (dict(k=48), SHAPE), (dict(k=131072), SHAPE), (dict(act=2), ARG), (dict(act=1, n=7), SHAPE),
    (dict(x=None), NULL), (dict(xs=None), NULL), (dict(q=None), NULL), (dict(s=None), NULL), (dict(y=None), NULL),
    (dict(ldy=7), SHAPE), (dict(r=P, ldr=7), SHAPE), (dict(r=P, ldr=9), ARG), (dict(act=1, ldy=3), SHAPE), (dict(x=P8), ALIGN), (dict(q=P8), ALIGN), (dict(xs=P2), ALIGN),
    (dict(s=P2), ALIGN), (dict(y=ctypes.c_void_p(4097)), ALIGN), (dict(bias=ctypes.c_void_p(4097)), ALIGN), (dict(r=ctypes.c_void_p(4097)), ALIGN),
])
def test_product_refusals(what, code):
    assert product(**what) == code and binding.load().mxfp4_last_error()


def lora(x=P, m=4, ldx=64, a=P, b=P, adapters=3, r=16, n=32, k=64, ids=P, scales=None, base=None, ldb=32, y=P, ldy=32, ws=P, size=1 << 30):
    return binding.load().mxfp4_lora(x, m, ldx, a, b, adapters, r, n, k, ids, scales, base, ldb, y, ldy, ws, size, None)


@pytest.mark.parametrize("what,code", [
    (dict(m=0, x=None), NONE), (dict(m=-1), SHAPE), (dict(r=12), SHAPE), (dict(r=0), SHAPE), (dict(r=136), SHAPE), (dict(n=20), SHAPE), (dict(n=0), SHAPE),
    (dict(k=60), SHAPE), (dict(k=0), SHAPE), (dict(adapters=0), SHAPE), (dict(adapters=8193), SHAPE), (dict(x=None), NULL), (dict(a=None), NULL), (dict(b=None), NULL),
    (dict(ids=None), NULL), (dict(y=None), NULL), (dict(ldx=56), SHAPE), (dict(ldx=1 << 24), SHAPE), (dict(ldy=1 << 24), SHAPE), (dict(base=P, ldb=1 << 24), SHAPE), (dict(ldx=66), ALIGN), (dict(ldy=24), SHAPE), (dict(base=P, ldb=24), SHAPE),
    (dict(base=P, ldb=40), ARG), (dict(x=P8), ALIGN), (dict(a=P8), ALIGN), (dict(b=P8), ALIGN), (dict(y=P8), ALIGN), (dict(base=P8), ALIGN),
    (dict(ids=P2), ALIGN), (dict(scales=P2), ALIGN), (dict(ws=P8), ALIGN), (dict(ws=None), WORKSPACE), (dict(size=4), WORKSPACE),
])
def test_adapter_refusals(what, code):
    assert lora(**what) == code
    assert code == NONE or binding.load().mxfp4_last_error()


def test_adapter_workspace_size():
    size = binding.mxfp4_lora_workspace_bytes
    assert size(0, 64, 8) == 0 and size(4, 63, 8) == 0 and size(4, 64, 256) == 0
    for m, k, r in ((1, 8, 8), (17, 4096, 16), (5000, 8192, 64)):
        assert size(m, k, r) >= m * r * 4
    assert size(1 << 30, 64, 8) == size(1 << 20, 64, 8)         # (very many rows go through it in turn)


def test_binding_refusals_without_a_device():
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        binding.mxfp4_rms_norm(x)
    with pytest.raises(ValueError, match="out must be"):
        binding.mxfp4_rms_norm(x, out="int8")
    with pytest.raises(ValueError, match="GPU"):
        binding.mxfp4_w4a8_gemm(x.to(torch.uint8), x, x, x)
    with pytest.raises(ValueError, match="GPU"):
        binding.mxfp4_lora(x, x[None], x[None], torch.zeros(4, dtype=torch.int32))
