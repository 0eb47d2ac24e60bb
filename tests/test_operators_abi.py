"""Host checks of the vocabulary losses and of microscaled 4-bit floating point: sizes, and every
refusal, before any device work (the pointers here are never touched)."""
import ctypes
import os

import pytest

import paper_2403_06082_gb300 as fq

INVALID, ALIGNMENT, WORKSPACE = 1, 2, 4


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fq.lib_path()):
        import __graft_entry__
        __graft_entry__.build()
    return fq.lib()


def test_head_workspace_sizes(L):
    assert fq.fq_head_workspace_bytes(0, 64, 100, 1) == 0
    assert fq.fq_head_workspace_bytes(4, 0, 100, 1) == 0
    assert fq.fq_head_workspace_bytes(4, 64, 0, 1) == 0
    assert fq.fq_head_workspace_bytes(4, 64, 100, 0) == 0
    assert fq.fq_head_workspace_bytes(4, 64, 100, fq.FQ_DISTILL_MAX_K + 1) == 0
    assert fq.fq_head_grad_workspace_bytes(4, -1, 100, 1) == 0
    # the logits are not kept: far less than M x V for the loss, one piece of ds for the gradient
    M, d, V = 4096, 4096, 128000
    assert 0 < fq.fq_head_workspace_bytes(M, d, V, 1) < M * V * 2 // 4
    g = fq.fq_head_grad_workspace_bytes(M, d, V, 1)
    assert M * d * 2 < g < (128 << 20) + M * (d * 2 + d * 4 + 1024) + (1 << 20)
    # offsets beyond 32 bits
    assert fq.fq_head_grad_workspace_bytes(2_000_000, 4096, 2048, 1) > 2_000_000 * 4096 * 2


def _ce(L, x=0x1000, M=4, d=64, W=0x2000, V=100, target=0x3000, loss=0x4000, lse=0x5000,
        ws=0x10000, n=1 << 30):
    return L.fq_cross_entropy(x, M, d, W, V, target, loss, lse, ws, n, None)


def _ceg(L, x=0x1000, M=4, d=64, W=0x2000, V=100, target=0x3000, lse=0x4000, dloss=0x5000,
         dx=0x6000, dW=0x7000, ws=0x10000, n=1 << 30):
    return L.fq_cross_entropy_grad(x, M, d, W, V, target, lse, dloss, dx, dW, ws, n, None)


def _ds(L, index=0x3000, logit=0x8000, K=4, tau=1.0, loss=0x4000, lse=0x5000, n=1 << 30):
    return L.fq_distill(0x1000, 4, 64, 0x2000, 100, index, logit, K, tau, loss, lse, 0x10000, n,
                        None)


def _dsg(L, logit=0x8000, K=4, tau=1.0, dx=0x6000, dW=None, dloss=0x7000):
    return L.fq_distill_grad(0x1000, 4, 64, 0x2000, 100, 0x3000, logit, K, tau, 0x4000, dloss, dx,
                             dW, 0x10000, 1 << 30, None)


def test_cross_entropy_refusals(L):
    for f in (_ce, _ceg):
        for name in ("x", "W", "target", "lse"):
            assert f(L, **{name: None}) == INVALID
            assert f(L, **{name: 0x9004}) == ALIGNMENT
        for name in ("M", "d", "V"):
            assert f(L, **{name: 0}) == INVALID
            assert f(L, **{name: -8}) == INVALID
        assert f(L, d=60) == ALIGNMENT
        assert f(L, ws=None) == WORKSPACE
        assert f(L, ws=0x10010) == ALIGNMENT
        assert f(L, n=1024) == WORKSPACE
    assert _ce(L, loss=None) == INVALID
    assert _ce(L, loss=0x4008) == ALIGNMENT
    assert _ceg(L, dloss=None) == INVALID
    assert _ceg(L, dx=None, dW=None) == INVALID
    assert _ceg(L, dx=0x6002, dW=None) == ALIGNMENT
    assert _ceg(L, dx=None, dW=0x7002) == ALIGNMENT


def test_distill_refusals(L):
    for f in (_ds, _dsg):
        assert f(L, logit=None) == INVALID
        assert f(L, logit=0x8004) == ALIGNMENT
        for K in (0, -1, fq.FQ_DISTILL_MAX_K + 1):
            assert f(L, K=K) == INVALID
        for tau in (0.0, -1.0, float("inf"), float("nan")):
            assert f(L, tau=tau) == INVALID
    assert _ds(L, index=None) == INVALID
    assert _ds(L, n=4096) == WORKSPACE
    assert _dsg(L, dx=None) == INVALID


def _q(codes=0x1000, scales=0x2000, rows=128, cols=256):
    return fq._Mxfp(codes, scales, rows, cols)


def test_mxfp_sizes(L):
    assert fq.fq_mxfp_codes_bytes(3, 64) == 3 * 32
    assert fq.fq_mxfp_codes_bytes(3, 48) == 0 and fq.fq_mxfp_codes_bytes(0, 64) == 0
    assert fq.fq_mxfp_scales_bytes(128, 256) == 1024
    assert fq.fq_mxfp_scales_bytes(129, 257 + 31) == 4 * 1024
    assert fq.fq_mxfp_codes_bytes(3_000_000, 8192) == 3_000_000 * 4096      # beyond 32 bits
    assert fq.fq_mxfp_workspace_bytes(4, 256, 0) == 0
    assert fq.fq_mxfp_workspace_bytes(4, 250, 8) == 0
    assert fq.fq_mxfp_workspace_bytes(4, 256, 8) >= 256 + 4 * 128 + 1024


def test_mxfp_refusals(L):
    ref = ctypes.byref

    def quant(x=0x4000, rows=128, cols=256, q=None):
        return L.fq_mxfp_quantize(x, rows, cols, ref(q or _q()), None)

    assert quant(x=None) == INVALID
    assert quant(rows=0) == INVALID
    assert quant(cols=250) == INVALID
    assert quant(rows=127) == INVALID                       # not q's sizes
    assert quant(q=_q(codes=None)) == INVALID
    assert quant(q=_q(scales=None)) == INVALID
    assert quant(q=_q(codes=0x1008)) == ALIGNMENT
    assert quant(x=0x4002) == ALIGNMENT
    assert L.fq_mxfp_dequantize(ref(_q()), None, None) == INVALID
    assert L.fq_mxfp_dequantize(ref(_q(rows=-1)), 0x4000, None) == INVALID
    assert L.fq_mxfp_dequantize(ref(_q()), 0x4008, None) == ALIGNMENT
    assert L.fq_mxfp_product(ref(_q()), ref(_q(cols=288)), 0x4000, None, None) == INVALID
    assert L.fq_mxfp_product(ref(_q()), ref(_q()), None, None, None) == INVALID
    assert L.fq_mxfp_product(ref(_q()), ref(_q()), 0x4002, None, None) == ALIGNMENT
    assert L.fq_mxfp_product(ref(_q()), ref(_q()), 0x4000, 0x5002, None) == ALIGNMENT

    def linear(x=0x4000, M=8, d=256, q=None, y=0x5000, ws=0x10000, n=1 << 20):
        return L.fq_mxfp_linear(x, M, d, ref(q or _q()), y, ws, n, None)

    assert linear(x=None) == INVALID and linear(y=None) == INVALID
    assert linear(M=0) == INVALID and linear(d=0) == INVALID and linear(d=288) == INVALID
    assert linear(x=0x4004) == ALIGNMENT and linear(y=0x5002) == ALIGNMENT
    assert linear(ws=None) == WORKSPACE and linear(n=256) == WORKSPACE
    assert linear(ws=0x10010) == ALIGNMENT
    assert linear(q=_q(codes=None)) == INVALID


def test_binding_checks_types_and_sizes(L):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        fq._arr(x, "float32", 4, "x")
    with pytest.raises(ValueError):
        fq._arr(x, "bfloat16", 257, "x")
    with pytest.raises(ValueError):
        fq._arr(x.t(), "bfloat16", 256, "x")               # not contiguous
    assert fq._arr(None, "bfloat16", 1, "x") is None
    q = fq.Mxfp(torch.zeros(10, dtype=torch.uint8), torch.zeros(1024, dtype=torch.uint8), 4, 64)
    with pytest.raises(ValueError):
        q._c()
