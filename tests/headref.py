"""Plain 64-bit form of the losses over the vocabulary and of their gradients, with the error
bounds that the library's arithmetic allows."""
import math

import torch

# bf16 has 8 significant bits: rounding to it is at most 2^-8 of a value.  A logit is a sum of
# exact products kept in fp32: an accumulation that truncates loses at most 2^-22 of the sum of
# magnitudes per step, and the steps' partial sums are far below that sum, so four times it
# bounds a logit.
BF = 2.0 ** -8
ACC = 4 * 2.0 ** -22


def sparse_targets(M, V, target=None, index=None, logit=None, tau=1.0):
    """(has, at, p, entropy term): the entries of each token as a gather index, with their
    probabilities (0 where an entry does not count), and sum p log p."""
    if target is not None:
        at, valid = target.long()[:, None], (target[:, None] >= 0) & (target[:, None] < V)
        t = torch.zeros_like(at, dtype=torch.float64)
    else:
        at = index.long()
        valid = (at >= 0) & (at < V) & (logit != -math.inf)
        t = logit.double() / tau
    has = valid.any(1)
    t = torch.where(valid, t, -math.inf)
    p = torch.softmax(torch.where(has[:, None], t, torch.zeros_like(t)), 1)
    p = torch.where(valid, p, torch.zeros_like(p))
    h = torch.where(p > 0, p * torch.log(p), torch.zeros_like(p)).sum(1)
    return has, at.clamp(0, V - 1), p, h


def reference(x, W, dloss=None, target=None, index=None, logit=None, tau=1.0):
    """loss, lse, dx, dW in 64 bits and their elementwise bounds, as two dicts."""
    M, V = x.shape[0], W.shape[0]
    has, at, p, h = sparse_targets(M, V, target, index, logit, tau)
    x = torch.where(has[:, None], x.double(), torch.zeros((), dtype=torch.float64,
                                                           device=x.device))
    W = W.double()
    z = (x @ W.T) / tau
    mag = (x.abs() @ W.abs().T) / tau                # sum of magnitudes behind each logit
    es = ACC * mag.amax(1)                           # bound on each logit of the token
    lse = torch.logsumexp(z, 1)
    kl = (p * (lse[:, None] - z.gather(1, at))).sum(1) + h
    t2 = tau * tau if target is None else 1.0
    out = {"loss": torch.where(has, t2 * kl, 0.0), "lse": torch.where(has, lse, 0.0)}
    # fp32 exponentials, logarithms and sums besides the logits: a few 2^-22 of their magnitudes
    scale = lse.abs() + z.gather(1, at).abs().amax(1) + h.abs() + 1.0
    if logit is not None:
        scale = scale + torch.where(torch.isfinite(logit), logit.double().abs() / tau,
                                    torch.zeros((), dtype=torch.float64,
                                                device=x.device)).amax(1)
    e = es + 8 * 2.0 ** -22 * scale
    bound = {"loss": 2 * t2 * e, "lse": e}
    if dloss is not None:
        g = torch.where(has, dloss.double() * (tau if target is None else 1.0), 0.0)
        y = torch.zeros_like(z).scatter_add_(1, at, p)
        q = torch.exp(z - lse[:, None])
        ds = g[:, None] * (q - y)
        # ds: rounded to bf16, after errors of the exponent and of the probabilities
        size = g.abs()[:, None] * (q + y)
        eds = BF * ds.abs() + size * (4 * e[:, None] + 2.0 ** -20)
        out["dx"], out["dW"] = ds @ W, ds.T @ x
        acc = 64 * ACC                               # fp32 accumulation over V or M products
        bound["dx"] = eds @ W.abs() + acc * (ds.abs() @ W.abs()) + 1.01 * BF * out["dx"].abs()
        bound["dW"] = eds.T @ x.abs() + acc * (ds.abs().T @ x.abs()) + 1.01 * BF * out["dW"].abs()
    return out, bound
