"""Losses over the vocabulary (include/framequant_head.h) and their gradients on the GPU against
the 64-bit form, elementwise within the bounds of headref.py."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2403_06082_gb300 as fq  # noqa: E402
from headref import reference  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16
GUARD = 64


def _guarded(shape, dtype):
    """A NaN-filled output with a strip of sevens behind it."""
    n = math.prod(shape)
    buf = torch.full((n + GUARD,), float("nan"), dtype=dtype, device=DEV)
    buf[n:] = 7.0
    return buf, buf[:n].view(shape)


def _inputs(M, d, V, K=0, seed=0, masked=0.1, tau=1.0, lean=6.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    sd = 1.28 / math.sqrt(d)
    W = (torch.randn(V, d, generator=g, device=DEV) * sd).to(BF16)
    y = torch.randint(0, V, (M,), generator=g, device=DEV)
    a = torch.rand(M, 1, generator=g, device=DEV) * lean / (sd * sd * d)
    x = (torch.randn(M, d, generator=g, device=DEV) + a * W[y].float()).to(BF16)
    off = torch.rand(M, generator=g, device=DEV) < masked
    s = {"x": x, "W": W, "dloss": torch.randn(M, generator=g, device=DEV) / M}
    if K == 0:
        s["target"] = torch.where(off, -100, y).to(torch.int32)
    else:
        index = torch.randint(0, V, (M, K), generator=g, device=DEV)   # some of them equal
        index[:, 0] = y
        index[torch.rand(M, K, generator=g, device=DEV) < 0.1] = -1
        index[off] = -5
        s["index"] = index.to(torch.int32)
        s["logit"] = 3 * torch.randn(M, K, generator=g, device=DEV)
        s["logit"][torch.rand(M, K, generator=g, device=DEV) < 0.05] = -math.inf
        s["tau"] = tau
    return s


def _call(s, dx=True, dW=True, stream=None, check=0):
    """Loss and gradients through the library, from a workspace full of ones bits."""
    (M, d), V = s["x"].shape, s["W"].shape[0]
    K = s["index"].shape[1] if "index" in s else 1
    lbuf, loss = _guarded((M,), torch.float32)
    ebuf, lse = _guarded((M,), torch.float32)
    n = fq.fq_head_workspace_bytes(M, d, V, K)
    ws = torch.full((n + GUARD,), 255, dtype=torch.uint8, device=DEV)
    head = (s["x"], M, d, s["W"], V)
    if K == 1 and "target" in s:
        fq.fq_cross_entropy(*head, s["target"], loss, lse, ws, n, stream)
    else:
        fq.fq_distill(*head, s["index"], s["logit"], K, s["tau"], loss, lse, ws, n, stream)
    assert fq.fq_check(ws, stream) == check
    assert (ws[n:] == 255).all()
    out, bufs = {"loss": loss, "lse": lse}, [lbuf, ebuf]
    if dx or dW:
        xbuf, gx = _guarded((M, d), BF16)
        wbuf, gW = _guarded((V, d), BF16)
        n = fq.fq_head_grad_workspace_bytes(M, d, V, K)
        ws = torch.full((n + GUARD,), 255, dtype=torch.uint8, device=DEV)
        to = (gx if dx else None, gW if dW else None)
        if K == 1 and "target" in s:
            fq.fq_cross_entropy_grad(*head, s["target"], lse, s["dloss"], *to, ws, n, stream)
        else:
            fq.fq_distill_grad(*head, s["index"], s["logit"], K, s["tau"], lse, s["dloss"], *to,
                               ws, n, stream)
        assert fq.fq_check(ws, stream) == 0
        assert (ws[n:] == 255).all()
        if dx:
            out["dx"] = gx
        if dW:
            out["dW"] = gW
        bufs += [xbuf, wbuf]
    for b in bufs:
        assert (b[-GUARD:] == 7.0).all(), "written beyond an output"
    return out


def _hold(got, s):
    ref, bound = reference(**s)
    for k, v in got.items():
        v = v.double()
        assert torch.isfinite(v).all(), k
        over = (v - ref[k]).abs() - bound[k]
        assert (over <= 0).all(), (k, float(over.max()), int(over.argmax()))


SIZES = [(1, 8, 1), (1, 64, 1000), (3, 72, 17), (128, 64, 256), (129, 264, 515),
         (200, 256, 1031), (257, 768, 2049), (64, 4096, 4099), (1, 4096, 32000)]


@pytest.mark.parametrize("M,d,V", SIZES)
def test_cross_entropy_and_gradients(M, d, V):
    s = _inputs(M, d, V, seed=M + V)
    _hold(_call(s), s)


@pytest.mark.parametrize("M,d,V", [(257, 1032, 130), (384, 1032, 2049), (300, 4096, 4099),
                                   (385, 520, 4099), (300, 4096, 24577)])
def test_three_row_tiles_by_single_ctas_and_by_pairs(M, d, V):
    s = _inputs(M, d, V, seed=M + V)
    _hold(_call(s), s)


@pytest.mark.parametrize("K,tau", [(1, 1.0), (5, 2.0), (64, 1.5), (300, 4.0), (1024, 0.5)])
@pytest.mark.parametrize("M,d,V", [(3, 72, 17), (130, 256, 1031), (300, 520, 4099)])
def test_distillation_and_gradients(M, d, V, K, tau):
    s = _inputs(M, d, V, K, seed=K + V, tau=tau)
    _hold(_call(s), s)


@pytest.mark.parametrize("K", [0, 5])
@pytest.mark.parametrize("dloss", ["mean", "zero_first", "tiny", "huge", "masked_nan"])
def test_kinds_of_dloss(K, dloss):
    """The usual 1 / tokens; a first token of no weight; sizes at the ends of fp32; and what
    tokens without a target hold, from the first one on."""
    s = _inputs(300, 128, 700, K, seed=21, tau=2.0)
    off = (s["target"] < 0) if K == 0 else (s["index"] < 0).all(1)
    if dloss == "mean":
        s["dloss"] = torch.full_like(s["dloss"], 1.0 / 271)
    elif dloss == "zero_first":
        s["dloss"][:5] = 0.0
    elif dloss == "tiny":
        s["dloss"] *= 1e-25
    elif dloss == "huge":
        s["dloss"] *= 1e25
    else:
        for k in ("target", "index"):
            if k in s:
                s[k][:40] = -1
        off[:40] = True
        s["dloss"][off] = float("nan")
    _hold(_call(s), s)


def test_the_mean_loss_gradient_is_as_exact_as_its_rounding():
    """With dloss = 1 / tokens for every token the error of the gradients' norm stays near that of
    rounding them to bf16 (1.7e-3: 2^-7 / sqrt(12) of a value's power of two, the value anywhere
    between two of them) and of rounding ds as well (sqrt(2) times that), wherever 1 / tokens lies
    between two bf16 values."""
    for count in (256, 271, 288, 300, 333, 383):
        s = _inputs(512, 256, 2000, seed=22)
        s["dloss"] = torch.full_like(s["dloss"], 1.0 / count)
        got = _call(s)
        ref, _ = reference(**s)
        for k in ("dx", "dW"):
            err = float((got[k].double() - ref[k]).norm() / ref[k].norm())
            assert err < 2.0 ** -8 * 0.625, (count, k, err)


@pytest.mark.parametrize("K", [0, 7])
def test_several_pieces_of_the_vocabulary(K):
    """33000 tokens: 2048 vocabulary entries per piece at most, so three pieces of 4099."""
    s = _inputs(33000, 64, 4099, K, seed=5, tau=2.0)
    _hold(_call(s), s)


def test_pieces_with_a_split_contraction():
    """16384 tokens of 8 values: two pieces of the vocabulary, dx in one column of tiles."""
    s = _inputs(16384, 8, 6000, seed=6)
    _hold(_call(s), s)


@pytest.mark.parametrize("dx,dW", [(True, False), (False, True)])
@pytest.mark.parametrize("K", [0, 6])
def test_one_gradient_alone_is_the_same(dx, dW, K):
    s = _inputs(200, 256, 1031, K, seed=3, tau=2.0)
    both, one = _call(s), _call(s, dx, dW)
    assert torch.equal(one["dx"], both["dx"]) if dx else torch.equal(one["dW"], both["dW"])


@pytest.mark.parametrize("K", [0, 6])
def test_every_token_masked(K):
    s = _inputs(150, 64, 700, K, seed=4, masked=1.1, tau=2.0)
    s["x"][:] = float("nan")
    s["dloss"][:] = float("inf")
    for k, v in _call(s).items():
        assert (v == 0).all(), k


@pytest.mark.parametrize("K", [0, 6])
def test_what_masked_tokens_hold_does_not_show(K):
    s = _inputs(300, 64, 700, K, seed=8, masked=0.3, tau=2.0)
    clean = _call(s)
    off = (s["target"] < 0) if K == 0 else (s["index"] < 0).all(1)
    assert 0 < int(off.sum()) < 300
    s["x"][off] = torch.tensor([float("nan"), float("inf")] * 32, dtype=BF16, device=DEV)
    s["dloss"][off] = float("nan")
    for k, v in _call(s).items():
        assert torch.equal(v, clean[k]), k


def test_nan_in_a_token_shows_in_that_token():
    s = _inputs(40, 64, 700, seed=9, masked=0.0)
    s["x"][7, 3] = float("nan")
    got = _call(s)
    for k in ("loss", "lse"):
        assert torch.isnan(got[k]).nonzero().flatten().tolist() == [7]
    assert torch.isnan(got["dx"][7]).all() and torch.isfinite(got["dx"][8:]).all()


@pytest.mark.parametrize("K", [0, 4])
def test_targets_beyond_the_vocabulary_are_reported_and_count_as_none(K):
    s = _inputs(40, 64, 700, K, seed=10, tau=2.0)
    if K == 0:
        s["target"][3] = 700
    else:
        s["index"][3, :] = 700
    got = _call(s, check=7)
    assert got["loss"][3] == 0 and (got["dx"][3] == 0).all()
    _hold(got, s)


def test_confident_and_hopeless_tokens():
    """Logits up to about 80: probabilities that are 1 and 0 in fp32."""
    s = _inputs(64, 64, 500, seed=11, lean=80.0)
    s["target"][::2] = (s["target"][::2] + 1) % 500
    _hold(_call(s), s)


@pytest.mark.parametrize("K", [0, 9])
def test_repeated_calls_give_the_same_bits_on_any_stream(K):
    s = _inputs(333, 264, 3001, K, seed=12, tau=2.0)
    first = _call(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = _call(s, stream=side)
    torch.cuda.synchronize()
    for k in first:
        assert torch.equal(first[k], second[k]), k


def test_gradient_is_the_difference_of_the_loss():
    """Steps of W along its gradient's signs that bf16 holds exactly: the loss falls by what the
    gradient says, up to the second order."""
    s = _inputs(96, 128, 600, seed=13)
    w = s["dloss"].double()
    W0 = (s["W"].double() / 2.0 ** -9).round() * 2.0 ** -9         # a grid that bf16 holds
    W0 = W0.clamp(-250 * 2.0 ** -9, 250 * 2.0 ** -9)
    s["W"] = W0.to(BF16)
    g = _call(s)["dW"].double()
    step = 2.0 ** -9 * torch.sign(g)
    ends = []
    for sign in (1, -1):
        t = dict(s)
        t["W"] = (W0 + sign * step).to(BF16)
        assert torch.equal(t["W"].double(), W0 + sign * step)
        ends.append(float((_call(t, False, False)["loss"].double() * w).sum()))
    slope = (ends[0] - ends[1]) / 2
    told = float((g * step).sum())
    assert abs(slope - told) <= 0.02 * abs(told)


def test_errors_launch_nothing():
    M, d, V, K = 16, 64, 300, 4
    s = _inputs(M, d, V, K, seed=1, tau=2.0)
    n = fq.fq_head_workspace_bytes(M, d, V, K)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
    loss = torch.full((M,), 3.0, device=DEV)
    lse = torch.full((M,), 3.0, device=DEV)

    def call(**kw):
        a = dict(x=s["x"], M=M, d=d, W=s["W"], V=V, index=s["index"], logit=s["logit"], K=K,
                 tau=2.0, loss=loss, lse=lse, ws=ws, ws_bytes=n)
        a.update(kw)
        fq.fq_distill(**a)

    for kw, status in ((dict(M=0), 1), (dict(tau=0.0), 1), (dict(tau=float("nan")), 1),
                       (dict(K=0), 1), (dict(logit=None), 1), (dict(ws=None), 4),
                       (dict(ws_bytes=n - 1), 4), (dict(d=60), 2),
                       (dict(x=s["x"].view(-1)[1:], M=M - 1), 2), (dict(loss=None), 1)):
        with pytest.raises(fq.FrameQuantError) as e:
            call(**kw)
        assert e.value.status == status, kw
    with pytest.raises(TypeError):
        call(index=s["index"].long())
    with pytest.raises(ValueError):
        call(V=V + 1)
    torch.cuda.synchronize()
    assert (loss == 3.0).all() and (lse == 3.0).all()
