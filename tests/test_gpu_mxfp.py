"""Microscaled 4-bit quantisation and product (include/framequant_mxfp.h) on the GPU against the
64-bit form.  Quantisation is exact.  A result is a sum of exact products of quantised values
kept in fp32, which loses at most 2^-22 of the sum of magnitudes per step of 64 k (and per
part of a split), and is rounded to bf16 once (2^-8)."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2403_06082_gb300 as fq  # noqa: E402
from mxref import dequantised, quantise  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
GUARD = 64


def _matrix(rows, cols, seed, loud=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device=DEV)
    if loud:
        x = torch.where(torch.rand(cols, generator=g, device=DEV) < 0.02, 30 * x, x)
        x = x * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g, device=DEV).float())
    return x.to(BF16)


def _quantised(x):
    rows, cols = x.shape
    q = fq.fq_mxfp_alloc(rows, cols)
    q.codes.fill_(255)
    q.scales.fill_(255)
    fq.fq_mxfp_quantize(x, rows, cols, q)
    return q


def _same(a, b):
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 4096), (3, 96), (127, 256), (128, 288),
                                       (129, 1024), (333, 4128), (1000, 64)])
def test_quantise_is_exact(rows, cols):
    x = _matrix(rows, cols, rows + cols)
    q = _quantised(x)
    code, exps = quantise(x)
    packed = (code[:, 0::2] | (code[:, 1::2] << 4)).to(torch.uint8)
    assert torch.equal(q.codes.cpu().view(rows, cols // 2), packed)
    # the documented place of every scale; 0 beyond the matrix
    kb = -(-cols // 256)
    want = torch.zeros(-(-rows // 128) * kb * 1024, dtype=torch.uint8)
    r = torch.arange(rows)[:, None]
    b = torch.arange(cols // 32)[None, :]
    at = ((r // 128) * kb + b // 8) * 1024 + (b // 4 % 2) * 512 + 16 * (r % 32) \
        + 4 * (r // 32 % 4) + b % 4
    want[at.flatten()] = exps.to(torch.uint8).flatten()
    assert torch.equal(q.scales.cpu(), want)
    y = torch.empty_like(x)
    fq.fq_mxfp_dequantize(q, y)
    assert torch.equal(y.double().cpu(), dequantised(x))


def test_quantise_extremes():
    """Every bf16 bit pattern in some block: largest, subnormal, zero, infinite and NaN."""
    x = torch.arange(65536, dtype=torch.int32, device=DEV).to(torch.int16).view(BF16).view(-1, 32)
    g = torch.Generator(device=DEV).manual_seed(0)
    x = torch.cat([x, x.flatten()[torch.randperm(65536, generator=g, device=DEV)].view(-1, 32),
                   torch.zeros(1, 32, dtype=BF16, device=DEV)])
    y = torch.empty_like(x)
    fq.fq_mxfp_dequantize(_quantised(x), y)
    assert _same(y.double().cpu(), dequantised(x))


def _bound(X, W, ref):
    steps = X.shape[1] / 64 + 9
    return steps * 2.0 ** -22 * (X.abs() @ W.abs().T) + 2.0 ** -8 * ref.abs()


def _linear(x, w, q=None):
    (M, d), V = x.shape, w.shape[0]
    q = q or _quantised(w)
    buf = torch.full((M * V + GUARD,), float("nan"), dtype=BF16, device=DEV)
    buf[M * V:] = 7.0
    n = fq.fq_mxfp_workspace_bytes(M, d, V)
    ws = torch.full((n + GUARD,), 255, dtype=torch.uint8, device=DEV)
    y = buf[:M * V].view(M, V)
    fq.fq_mxfp_linear(x, M, d, q, y, ws, n)
    assert fq.fq_check(ws) == 0
    assert (buf[M * V:] == 7.0).all() and (ws[n:] == 255).all()
    return y


@pytest.mark.parametrize("M,d,V", [
    (1, 32, 1), (1, 256, 128), (1, 4096, 4096), (2, 64, 130), (5, 96, 33), (16, 4096, 1000),
    (17, 1024, 257), (48, 2048, 129), (64, 288, 300), (65, 512, 513), (128, 4096, 260),
    (192, 256, 20000), (193, 320, 400), (200, 8192, 128), (333, 1056, 1031), (1000, 512, 1500)])
def test_linear(M, d, V):
    x, w = _matrix(M, d, 1), _matrix(V, d, 2, loud=False)
    X, W = dequantised(x).to(DEV), dequantised(w).to(DEV)
    ref = X @ W.T
    y = _linear(x, w).double()
    assert torch.isfinite(y).all()
    over = (y - ref).abs() - _bound(X, W, ref)
    assert (over <= 0).all(), (float(over.max()), int(over.argmax()))


@pytest.mark.parametrize("M,d,V", [
    (1, 8192, 300), (1, 8224, 300), (2, 8192, 28672), (8, 2048, 40000), (16, 1024, 130),
    (16, 1056, 130), (3, 5472, 200), (4, 4096, 4096), (5, 4096, 4096), (1, 32, 20000)])
def test_linear_of_few_tokens(M, d, V):
    """Sizes about the bounds between quantising x on the way and ahead of the product: the same
    bits as the product of the quantised x, whichever way it goes."""
    x, w = _matrix(M, d, 11), _matrix(V, d, 12, loud=False)
    q = _quantised(w)
    y = _linear(x, w, q)
    two = torch.empty_like(y)
    fq.fq_mxfp_product(_quantised(x), q, two)
    assert torch.equal(y, two)
    if V * d <= 1 << 22:
        X, W = dequantised(x).to(DEV), dequantised(w).to(DEV)
        ref = X @ W.T
        assert ((y.double() - ref).abs() <= _bound(X, W, ref)).all()


@pytest.mark.parametrize("M,d,V", [
    (256, 4096, 1031), (129, 4096, 520), (100, 11008, 1024), (192, 1024, 4096), (64, 4096, 4093),
    (97, 5472, 300), (40, 8192, 1000), (320, 288, 8805), (1275, 288, 2221), (700, 2048, 5504)])
def test_linear_of_every_kind_of_tile(M, d, V):
    """Tiles of 64, 128 and 192 tokens, one tile of all of them; one CTA, pairs, 2 to 8 CTAs that
    split k, with a last part that is shorter; rows of y that are not a multiple of 4."""
    x, w = _matrix(M, d, 13), _matrix(V, d, 14, loud=False)
    X, W = dequantised(x).to(DEV), dequantised(w).to(DEV)
    ref = X @ W.T
    y = _linear(x, w).double()
    over = (y - ref).abs() - _bound(X, W, ref)
    assert (over <= 0).all(), (float(over.max()), int(over.argmax()))


@pytest.mark.parametrize("M", [3, 300])
def test_product_of_two_quantised_is_the_linear(M):
    x, w = _matrix(M, 1024, 3), _matrix(500, 1024, 4, loud=False)
    y = torch.empty(M, 500, dtype=BF16, device=DEV)
    status = torch.full((1,), -1, dtype=torch.int32, device=DEV)
    fq.fq_mxfp_product(_quantised(x), _quantised(w), y, status)
    assert fq.fq_check(status) == 0
    assert torch.equal(y, _linear(x, w))


@pytest.mark.parametrize("M", [4, 20, 260])
def test_a_nan_block_shows_where_it_takes_part_and_nowhere_else(M):
    x, w = _matrix(M, 512, 5), _matrix(300, 512, 6, loud=False)
    clean = _linear(x, w)
    x[2, 100] = float("inf")
    w[7, 3] = float("nan")
    y = _linear(x, w)
    assert torch.isnan(y[2]).all() and torch.isnan(y[:, 7]).all()
    keep = torch.ones(M, 300, dtype=torch.bool, device=DEV)
    keep[2], keep[:, 7] = False, False
    assert torch.equal(y[keep], clean[keep])


def test_zero_rows_and_a_wide_range_of_scales():
    x, w = _matrix(20, 512, 7), _matrix(140, 512, 8)
    x[3], w[5] = 0, 0
    x[4] = (x[4].float() * 2.0 ** 60).to(BF16)
    w[6] = (w[6].float() * 2.0 ** -60).to(BF16)
    X, W = dequantised(x).to(DEV), dequantised(w).to(DEV)
    ref = X @ W.T
    y = _linear(x, w).double()
    assert (y[3] == 0).all() and (y[:, 5] == 0).all()
    assert ((y - ref).abs() <= _bound(X, W, ref)).all()


def test_same_bits_again_and_on_another_stream():
    x, w = _matrix(9, 4096, 9), _matrix(4096, 4096, 10, loud=False)
    q = _quantised(w)
    first = _linear(x, w, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = _linear(x, w, q)
    torch.cuda.synchronize()
    assert torch.equal(first, second)


def test_quantise_then_multiply_without_waiting():
    """A weight quantised right before the product that reads it, over and over."""
    w = [_matrix(512, 2048, 20 + i, loud=False) for i in range(2)]
    x = _matrix(3, 2048, 30)
    want = [_linear(x, v) for v in w]
    q = fq.fq_mxfp_alloc(512, 2048)
    n = fq.fq_mxfp_workspace_bytes(3, 2048, 512)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    got = []
    for i in range(40):
        y = torch.empty(3, 512, dtype=BF16, device=DEV)
        fq.fq_mxfp_quantize(w[i % 2], 512, 2048, q)
        fq.fq_mxfp_linear(x, 3, 2048, q, y, ws, n)
        got.append(y)
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 2])


def test_errors_launch_nothing():
    x, w = _matrix(8, 256, 1), _matrix(130, 256, 2)
    q = _quantised(w)
    y = torch.full((8, 130), 3.0, dtype=BF16, device=DEV)
    n = fq.fq_mxfp_workspace_bytes(8, 256, 130)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)

    def refused(status, f, *a):
        with pytest.raises(fq.FrameQuantError) as e:
            f(*a)
        assert e.value.status == status

    refused(1, fq.fq_mxfp_linear, x, 0, 256, q, y, ws, n)
    refused(1, fq.fq_mxfp_linear, x, 8, 224, q, y, ws, n)
    refused(4, fq.fq_mxfp_linear, x, 8, 256, q, y, ws, n - 1)
    refused(4, fq.fq_mxfp_linear, x, 8, 256, q, y, None, n)
    refused(2, fq.fq_mxfp_linear, x, 8, 256, q, y, ws[16:], n)
    refused(2, fq.fq_mxfp_linear, x.view(-1)[1:], 7, 256, q, y, ws, n)
    refused(1, fq.fq_mxfp_quantize, x, 8, 250, q)
    refused(1, fq.fq_mxfp_quantize, x, 8, 256, q)
    refused(1, fq.fq_mxfp_alloc, 8, 100)
    with pytest.raises(TypeError):
        fq.fq_mxfp_linear(x.float(), 8, 256, q, y, ws, n)
    with pytest.raises(ValueError):
        fq.fq_mxfp_linear(x, 9, 256, q, y, ws, n)
    torch.cuda.synchronize()
    assert (y == 3.0).all()
    assert fq.fq_mxfp_codes_bytes(3, 33) == 0 and fq.fq_mxfp_scales_bytes(0, 32) == 0
    assert fq.fq_mxfp_codes_bytes(129, 288) == 129 * 144
    assert fq.fq_mxfp_scales_bytes(129, 288) == 2 * 2 * 1024
