"""Matrices of more than 2^32 values (and results and offsets beyond it), at sampled rows about
the places where 31 and 32 bits end."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2403_06082_gb300 as fq  # noqa: E402
from headref import ACC, BF, reference  # noqa: E402
from mxref import dequantised  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
ROWS, COLS = 530000, 8192                            # rows 2^18 and 2^19 begin at 2^31 and 2^32
SAMPLE = [0, 1, 2 ** 18 - 1, 2 ** 18, 2 ** 19 - 1, 2 ** 19, 2 ** 19 + 1, ROWS - 2, ROWS - 1]


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV)


def test_vocabulary_losses_with_a_large_weight():
    """The output weight's rows are zero but for the sampled ones: the others' logits are 0, and
    together they count as one logit of log(their number)."""
    M, V, d = 5, ROWS, COLS
    g = torch.Generator(device=DEV).manual_seed(1)
    at = torch.tensor(SAMPLE, device=DEV)
    W = torch.zeros(V, d, dtype=BF16, device=DEV)
    W[at] = (torch.randn(len(SAMPLE), d, generator=g, device=DEV) / math.sqrt(d)).to(BF16)
    x = (4 * torch.randn(M, d, generator=g, device=DEV)).to(BF16)
    target = torch.tensor([SAMPLE[1], SAMPLE[3], SAMPLE[5], SAMPLE[-1], 777], dtype=torch.int32,
                          device=DEV)
    dloss = torch.randn(M, generator=g, device=DEV)
    loss, lse = (torch.full((M,), float("nan"), device=DEV) for _ in range(2))
    n = fq.fq_head_workspace_bytes(M, d, V)
    ws = _bytes(n)
    fq.fq_cross_entropy(x, M, d, W, V, target, loss, lse, ws, n)
    assert fq.fq_check(ws) == 0
    dx = torch.full((M, d), float("nan"), dtype=BF16, device=DEV)
    dW = torch.full((V, d), float("nan"), dtype=BF16, device=DEV)
    n = fq.fq_head_grad_workspace_bytes(M, d, V)
    ws = _bytes(n)
    fq.fq_cross_entropy_grad(x, M, d, W, V, target, lse, dloss, dx, dW, ws, n)
    assert fq.fq_check(ws) == 0

    # the bounds of headref.reference, for a vocabulary whose other rows are zero
    Wd, xd, gd = W[at].double(), x.double(), dloss.double()[:, None]
    z = xd @ Wd.T
    rest = torch.full((M, 1), math.log(V - len(SAMPLE)), dtype=torch.float64, device=DEV)
    ref = torch.logsumexp(torch.cat([z, rest], 1), 1)
    own = (target.long()[:, None] == at[None, :]).double()
    zt = (own * z).sum(1)
    e = ACC * (xd.abs() @ Wd.abs().T).amax(1) + 8 * 2.0 ** -22 * (ref.abs() + zt.abs() + 1.0)
    assert ((lse.double() - ref).abs() <= e).all()
    assert ((loss.double() - (ref - zt)).abs() <= 2 * e).all()
    q = torch.exp(z - ref[:, None])
    ds = gd * (q - own)
    eds = BF * ds.abs() + gd.abs() * (q + own) * (4 * e[:, None] + 2.0 ** -20)
    acc = 64 * ACC
    want = ds @ Wd
    bound = eds @ Wd.abs() + acc * (ds.abs() @ Wd.abs()) + 1.01 * BF * want.abs()
    assert ((dx.double() - want).abs() <= bound).all()
    want = ds.T @ xd
    bound = eds.T @ xd.abs() + acc * (ds.abs().T @ xd.abs()) + 1.01 * BF * want.abs()
    assert ((dW[at].double() - want).abs() <= bound).all()
    # a row of zeros, and the one that is a target
    q0 = torch.exp(-ref)
    for row in (2, 2 ** 18 + 5, 2 ** 19 + 5, ROWS - 3, 777):
        y0 = (target == row).double()
        d0 = gd[:, 0] * (q0 - y0)
        e0 = BF * d0.abs() + gd[:, 0].abs() * (q0 + y0) * (4 * e + 2.0 ** -20)
        want = d0 @ xd
        bound = e0 @ xd.abs() + acc * (d0.abs() @ xd.abs()) + 1.01 * BF * want.abs()
        assert ((dW[row].double() - want).abs() <= bound).all(), row


def test_vocabulary_losses_with_many_tokens():
    """Only the sampled tokens have a weight, so dW is theirs; a token whose row holds NaN has no
    target."""
    M, V, d = ROWS, 40, COLS
    g = torch.Generator(device=DEV).manual_seed(2)
    at = torch.tensor(SAMPLE, device=DEV)
    x = torch.empty(M, d, dtype=BF16, device=DEV).normal_(generator=g)
    W = (torch.randn(V, d, generator=g, device=DEV) / math.sqrt(d)).to(BF16)
    target = torch.randint(0, V, (M,), generator=g, device=DEV).to(torch.int32)
    dloss = torch.zeros(M, device=DEV)
    dloss[at] = torch.randn(len(SAMPLE), generator=g, device=DEV)
    off = 2 ** 19 + 7
    target[off], x[off] = -1, float("nan")
    loss, lse = (torch.full((M,), float("nan"), device=DEV) for _ in range(2))
    n = fq.fq_head_workspace_bytes(M, d, V)
    ws = _bytes(n)
    fq.fq_cross_entropy(x, M, d, W, V, target, loss, lse, ws, n)
    assert fq.fq_check(ws) == 0
    dx = torch.full((M, d), float("nan"), dtype=BF16, device=DEV)
    dW = torch.full((V, d), float("nan"), dtype=BF16, device=DEV)
    n = fq.fq_head_grad_workspace_bytes(M, d, V)
    ws = _bytes(n)
    fq.fq_cross_entropy_grad(x, M, d, W, V, target, lse, dloss, dx, dW, ws, n)
    assert fq.fq_check(ws) == 0
    ref, bound = reference(x[at], W, dloss[at], target[at])
    got = {"loss": loss[at], "lse": lse[at], "dx": dx[at], "dW": dW}
    for k, v in got.items():
        assert ((v.double() - ref[k]).abs() <= bound[k]).all(), k
    assert torch.isfinite(loss).all() and torch.isfinite(lse).all() and loss[off] == 0
    for row in (3, 2 ** 18 + 3, 2 ** 19 + 3, off, ROWS - 3):
        assert (dx[row] == 0).all(), row


def test_microscaled_weight():
    g = torch.Generator(device=DEV).manual_seed(3)
    at = torch.tensor(SAMPLE, device=DEV)
    w = torch.empty(ROWS, COLS, dtype=BF16, device=DEV).normal_(generator=g)
    q = fq.fq_mxfp_alloc(ROWS, COLS)
    fq.fq_mxfp_quantize(w, ROWS, COLS, q)
    rows = w[at]
    w.fill_(float("nan"))
    fq.fq_mxfp_dequantize(q, w)
    assert torch.equal(w[at].double().cpu(), dequantised(rows).cpu())
    x = torch.randn(3, COLS, generator=g, device=DEV).to(BF16)
    y = torch.full((3, ROWS), float("nan"), dtype=BF16, device=DEV)
    n = fq.fq_mxfp_workspace_bytes(3, COLS, ROWS)
    ws = _bytes(n)
    fq.fq_mxfp_linear(x, 3, COLS, q, y, ws, n)
    assert fq.fq_check(ws) == 0
    X, Wd = dequantised(x).to(DEV), dequantised(rows).to(DEV)
    _hold(y[:, at], X, Wd)


def test_microscaled_results():
    """4.3e9 results of products of 64."""
    M, V, d = 9000, 480000, 64
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(M, d, generator=g, device=DEV).to(BF16)
    w = torch.randn(V, d, generator=g, device=DEV).to(BF16)
    q = fq.fq_mxfp_alloc(V, d)
    fq.fq_mxfp_quantize(w, V, d, q)
    y = torch.full((M, V), float("nan"), dtype=BF16, device=DEV)
    n = fq.fq_mxfp_workspace_bytes(M, d, V)
    ws = _bytes(n)
    fq.fq_mxfp_linear(x, M, d, q, y, ws, n)
    assert fq.fq_check(ws) == 0
    t = torch.tensor([0, 4473, 4474, 8947, 8948, M - 1], device=DEV)      # 2^31, 2^32 in there
    c = torch.cat([torch.arange(300), torch.arange(V // 2, V // 2 + 300),
                   torch.arange(V - 300, V)]).to(DEV)
    _hold(y[t][:, c], dequantised(x[t]).to(DEV), dequantised(w[c]).to(DEV))


def _hold(y, X, W):
    """Sums of exact products in fp32, losing at most 2^-22 of the magnitudes a step of 64 k (and a
    part of a split), rounded to bf16 once."""
    ref = X @ W.T
    bound = (X.shape[1] / 64 + 9) * 2.0 ** -22 * (X.abs() @ W.abs().T) + BF * ref.abs()
    assert ((y.double() - ref).abs() <= bound).all()
