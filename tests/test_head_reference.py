"""The 64-bit form of the vocabulary losses that the GPU tests compare with: its gradients
against central differences of its losses, and against autograd of the textbook form."""
import math

import pytest

torch = pytest.importorskip("torch")

from headref import reference  # noqa: E402


def _case(kind, seed=0):
    g = torch.Generator().manual_seed(seed)
    M, d, V, K = 6, 8, 13, 4
    a = {"x": torch.randn(M, d, generator=g, dtype=torch.float64),
         "W": torch.randn(V, d, generator=g, dtype=torch.float64),
         "dloss": torch.randn(M, generator=g, dtype=torch.float64)}
    if kind == "ce":
        a["target"] = torch.randint(0, V, (M,), generator=g)
        a["target"][2] = -100
    else:
        a["index"] = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(M)])
        a["logit"] = torch.randn(M, K, generator=g)
        a["index"][1, 2] = -1
        a["index"][3, :] = -1
        a["index"][4, 1] = a["index"][4, 0]
        a["logit"][5, 3] = -math.inf
        a["tau"] = 2.0
    return a


@pytest.mark.parametrize("kind", ["ce", "distill"])
@pytest.mark.parametrize("name", ["x", "W"])
def test_gradients_are_the_differences_of_the_loss(kind, name):
    a = _case(kind)
    out, _ = reference(**a)
    grad = out["d" + name]
    h = 1e-6
    for i in range(a[name].shape[0]):
        for j in range(a[name].shape[1]):
            up, down = dict(a), dict(a)
            up[name], down[name] = a[name].clone(), a[name].clone()
            up[name][i, j] += h
            down[name][i, j] -= h
            lu, ld = reference(**up)[0]["loss"], reference(**down)[0]["loss"]
            diff = float(((lu - ld) * a["dloss"]).sum() / (2 * h))
            assert abs(diff - float(grad[i, j])) < 1e-7 * (1 + abs(diff))


def test_cross_entropy_is_torchs():
    a = _case("ce")
    x, W = a["x"].requires_grad_(), a["W"].requires_grad_()
    loss = torch.nn.functional.cross_entropy(x @ W.T, a["target"], ignore_index=-100,
                                             reduction="none")
    gx, gW = torch.autograd.grad((loss * a["dloss"]).sum(), (x, W))
    out, _ = reference(x.detach(), W.detach(), a["dloss"], a["target"])
    assert torch.allclose(out["loss"], loss.detach())
    assert torch.allclose(out["dx"], gx) and torch.allclose(out["dW"], gW)


def test_tokens_without_a_target_are_nothing():
    for kind, row in (("ce", 2), ("distill", 3)):
        a = _case(kind)
        clean, _ = reference(**a)
        a["x"][row, :] = math.nan
        a["dloss"][row] = math.inf
        out, _ = reference(**a)
        assert out["loss"][row] == 0 and out["lse"][row] == 0 and (out["dx"][row] == 0).all()
        assert torch.equal(out["dW"], clean["dW"])
