"""Cases of the language-model operators around a quantized layer: the loss over a large
vocabulary (cross entropy, and distillation from a teacher's top logits) computed from hidden
states and the output weight without keeping the logits, with their gradients; and microscaled
4-bit floating point (E2M1 values in blocks of 32 with one power-of-two scale), its quantisation
and the linear layer on it.

`run` computes an operator in its plain form (elementary torch operations in fp32), or, with
`own`, through the library's entry points.  `exact` is the same result from the definition in
64 bits.
"""
import math

import torch


own = False

DEV = "cuda"
BF16 = torch.bfloat16


# ------------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token scored on its own (the last position of a prompt): latency
        dict(name="ce_eval_1", op="cross_entropy", M=1, d=4096, V=32000, grad="none"),
        # perplexity of one 2048-token window, 7B-sized head
        dict(name="ce_eval_2048", op="cross_entropy", M=2048, d=4096, V=32000, grad="none"),
        # a small ragged training step: 197 tokens, an odd vocabulary
        dict(name="ce_train_197_odd", op="cross_entropy", M=197, d=768, V=10007, grad="both"),
        # two 2048-token sequences, loss and both gradients, 7B-sized head
        dict(name="ce_train_4096", op="cross_entropy", M=4096, d=4096, V=32000, grad="both"),
        # the distillation loss of a decode batch
        dict(name="distill_eval_16", op="distill", M=16, d=4096, V=32000, K=8, grad="none"),
        # a recovery step that trains the student's head too
        dict(name="distill_train_2048", op="distill", M=2048, d=4096, V=32000, K=64, grad="both"),
        # a recovery step with the head frozen, 70B width, ragged batch, odd vocabulary
        dict(name="distill_frozen_1000", op="distill", M=1000, d=8192, V=32003, K=32, grad="dx"),
        # one decoded token through an attention projection
        dict(name="mx_linear_1", op="mx_linear", M=1, d=4096, V=4096),
        # prefill of a window cut to 2047 tokens through an MLP projection
        dict(name="mx_linear_2047", op="mx_linear", M=2047, d=4096, V=11008),
        # large prefill through the widest 70B projection
        dict(name="mx_linear_4096_wide", op="mx_linear", M=4096, d=8192, V=28672),
        # activations of a ragged batch, quantised and read back
        dict(name="mx_quantize_333", op="mx_quantize", M=333, d=4096),
        # a 70B-sized weight, quantised and read back
        dict(name="mx_quantize_28672", op="mx_quantize", M=28672, d=8192),
    ]


MOST_LOSS = 4096 * 4096 * 32000 * 3      # products of the largest listed loss case
MOST_MX = 4096 * 8192 * 28672


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["cross_entropy", "distill", "mx_linear", "mx_quantize"])
    while True:
        if op in ("cross_entropy", "distill"):
            c = dict(op=op, M=_log(rng, 1, 4096), d=8 * _log(rng, 32, 1024),
                     V=_log(rng, 1000, 64000), grad=rng.choice(["none", "dx", "both"]))
            if op == "distill":
                c["K"] = _log(rng, 1, 128)
            if c["M"] * c["d"] * c["V"] * {"none": 1, "dx": 2, "both": 3}[c["grad"]] <= MOST_LOSS:
                return c
        elif op == "mx_linear":
            c = dict(op=op, M=_log(rng, 1, 4096), d=32 * _log(rng, 8, 256), V=_log(rng, 256, 28672))
            if c["M"] * c["d"] * c["V"] <= MOST_MX:
                return c
        else:
            return dict(op=op, M=_log(rng, 1, 28672), d=32 * _log(rng, 8, 256))


def work(case):
    M, d = case["M"], case["d"]
    if case["op"] == "mx_quantize":              # bf16 in, 4.25 bits out and in again, bf16 out
        return {"bytes": M * d * (2 + 2 + 2 * 4.25 / 8), "flops": 0}
    V = case["V"]
    if case["op"] == "mx_linear":
        return {"bytes": M * d * 2 + V * d * 4.25 / 8 + M * V * 2, "flops": 2 * M * V * d}
    n = {"none": 1, "dx": 2, "both": 3}[case["grad"]]
    b = M * d * 2 + V * d * 2 + M * 8
    b += M * case["K"] * 8 if case["op"] == "distill" else M * 4
    b += {"none": 0, "dx": M * d * 2 + M * 4, "both": (M + V) * d * 2 + M * 4}[case["grad"]]
    return {"bytes": b, "flops": 2 * n * M * V * d}


# ------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _loss_inputs(case, seed):
    """Hidden states, the output weight, and what each token is to learn.  A hidden state leans
    towards its token's row of the weight by a random amount, so that logits run from unsure
    (all near zero) to confident; one token in ten has no target (padding, a prompt)."""
    g = _generator(seed)
    M, d, V = case["M"], case["d"], case["V"]
    sd = 1.28 / math.sqrt(d)
    W = torch.randn(V, d, generator=g, device=DEV).mul_(sd).to(BF16)
    y = torch.randint(0, V, (M,), generator=g, device=DEV)
    lean = torch.rand(M, 1, generator=g, device=DEV) * 8.0 / (sd * sd * d)
    x = (torch.randn(M, d, generator=g, device=DEV) + lean * W[y].float()).to(BF16)
    masked = torch.rand(M, generator=g, device=DEV) < 0.1
    masked[0] = False
    out = {"x": x, "W": W}
    if case["op"] == "cross_entropy":
        out["target"] = torch.where(masked, torch.full_like(y, -100), y).to(torch.int32)
        count = (~masked).sum()
    else:
        K = case["K"]
        step = torch.randint(1, max(2, V // K), (M, K), generator=g, device=DEV)
        step[:, 0] = 0                           # the token itself, then K - 1 others, all apart
        index = (y[:, None] + step.cumsum(1)) % V
        logit = 9.0 - 2.0 * torch.log1p(torch.arange(K, device=DEV, dtype=torch.float32))
        logit = logit + 0.5 * torch.randn(M, K, generator=g, device=DEV)
        # some tokens come with fewer entries than K, the masked ones with none
        have = torch.randint(1, K + 1, (M, 1), generator=g, device=DEV)
        full = torch.rand(M, 1, generator=g, device=DEV) < 0.8
        have = torch.where(full, torch.full_like(have, K), have)
        have = torch.where(masked[:, None], torch.zeros_like(have), have)
        none = torch.arange(K, device=DEV)[None, :] >= have
        out["index"] = torch.where(none, torch.full_like(index, -1), index).to(torch.int32)
        out["logit"] = logit
        out["tau"] = 1.0 + 0.5 * (seed % 3)
        count = (~masked).sum()
    out["dloss"] = torch.ones(M, device=DEV) / count
    return out


def _mx_inputs(case, seed):
    """Activations with 1% of channels thirty times the others, weights N(0, 0.02)."""
    g = _generator(seed)
    M, d = case["M"], case["d"]
    x = torch.randn(M, d, generator=g, device=DEV)
    loud = torch.rand(d, generator=g, device=DEV) < 0.01
    x = torch.where(loud, 30.0 * x, x).to(BF16)
    if case["op"] == "mx_quantize":
        return {"x": x}
    return {"x": x, "W": torch.randn(case["V"], d, generator=g, device=DEV).mul_(0.02).to(BF16)}


def prepare(case, seed):
    s = {"case": case}
    M, d = case["M"], case["d"]
    if own:
        import paper_2403_06082_gb300 as fq

        def scratch(n):
            return torch.zeros(n, dtype=torch.uint8, device=DEV)
    if case["op"] in ("cross_entropy", "distill"):
        s.update(_loss_inputs(case, seed))
        if own:
            V, K = case["V"], case.get("K", 1)
            n = fq.fq_head_workspace_bytes(M, d, V, K)
            if case["grad"] != "none":
                n = max(n, fq.fq_head_grad_workspace_bytes(M, d, V, K))
            s["ws"], s["ws_bytes"] = scratch(n), n
            s["loss"], s["lse"] = torch.empty(M, device=DEV), torch.empty(M, device=DEV)
            s["dx"] = torch.empty_like(s["x"]) if case["grad"] != "none" else None
            s["dW"] = torch.empty_like(s["W"]) if case["grad"] == "both" else None
        return s
    s.update(_mx_inputs(case, seed))
    if own:
        if case["op"] == "mx_quantize":
            s["q"] = fq.fq_mxfp_alloc(M, d)
            s["y"] = torch.empty_like(s["x"])
        else:
            # the weight is quantised once, when the model is loaded
            s["q"] = fq.fq_mxfp_alloc(case["V"], d)
            fq.fq_mxfp_quantize(s.pop("W"), case["V"], d, s["q"])
            s["y"] = torch.empty(M, case["V"], dtype=BF16, device=DEV)
            n = fq.fq_mxfp_workspace_bytes(M, d, case["V"])
            s["ws"], s["ws_bytes"] = scratch(n), n
    elif case["op"] == "mx_linear":
        s["codes"], s["exps"] = _mx_codes(s.pop("W"))
        s["codes"] = s["codes"][:, 0::2] | (s["codes"][:, 1::2] << 4)
    return s


# ------------------------------------------------------------------------------- plain forms
def _plain_logits(s, tau):
    has = (s["target"] >= 0) if "target" in s else (s["index"] >= 0).any(1)
    x = torch.where(has[:, None], s["x"].float(), 0.0)
    logits = x @ s["W"].float().T
    if tau != 1.0:
        logits = logits / tau
    top = logits.amax(1)
    lse = top + torch.log(torch.exp(logits - top[:, None]).sum(1))
    return has, x, logits, lse


def _plain_grads(s, has, x, dlogits):
    """dx = dlogits W, dW = dlogits^T x for the rows that have a target."""
    out = {}
    dlogits = torch.where(has[:, None], dlogits, 0.0)
    out["dx"] = (dlogits @ s["W"].float()).to(BF16)
    if s["case"]["grad"] == "both":
        out["dW"] = (dlogits.T @ x).to(BF16)
    return out


def _plain_cross_entropy(s):
    has, x, logits, lse = _plain_logits(s, 1.0)
    y = s["target"].long().clamp(min=0)[:, None]
    out = {"loss": torch.where(has, lse - logits.gather(1, y)[:, 0], 0.0),
           "lse": torch.where(has, lse, 0.0)}
    if s["case"]["grad"] == "none":
        return out
    p = torch.exp(logits - lse[:, None])
    p.scatter_add_(1, y, torch.full_like(y, -1.0, dtype=torch.float32))
    out.update(_plain_grads(s, has, x, p * s["dloss"][:, None]))
    return out


def _plain_distill(s):
    tau = s["tau"]
    has, x, logits, lse = _plain_logits(s, tau)
    valid = s["index"] >= 0
    at = s["index"].long().clamp(min=0)
    t = torch.where(valid, s["logit"] / tau, -math.inf)
    top = torch.where(has, t.amax(1), 0.0)[:, None]
    e = torch.exp(t - top)
    total = torch.where(has[:, None], e.sum(1, keepdim=True), 1.0)
    p = e / total                                          # 0 where there is no entry
    logp = torch.where(p > 0, t - top - torch.log(total), 0.0)
    kl = (p * (logp - logits.gather(1, at) + lse[:, None])).sum(1)
    out = {"loss": torch.where(has, tau * tau * kl, 0.0), "lse": torch.where(has, lse, 0.0)}
    if s["case"]["grad"] == "none":
        return out
    q = torch.exp(logits - lse[:, None])
    q.scatter_add_(1, at, -p)
    out.update(_plain_grads(s, has, x, q * (tau * s["dloss"])[:, None]))
    return out


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx_codes(x):
    """E2M1 codes (uint8, sign in bit 3) and biased block exponents (uint8; 255 marks a block
    that holds an infinity or a NaN) of a bf16 matrix: exponent floor(log2(largest)) - 2, values
    to nearest with ties to even, saturating at 6."""
    a = x.float().reshape(x.shape[0], -1, 32)
    big = a.abs().amax(-1)
    e = ((big.view(torch.int32) >> 23) - 127 - 2).clamp(min=-127)
    fine = torch.isfinite(big)
    e = torch.where(fine, e, 0)
    m = a.abs() * ((127 - e) << 23).view(torch.float32)[..., None]
    code = torch.zeros(a.shape, dtype=torch.uint8, device=x.device)
    for i, edge in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (m >= edge) if i % 2 else (m > edge)
    code += torch.signbit(a).to(torch.uint8) << 3
    code = torch.where(fine[..., None], code, 0)
    return code.reshape(x.shape), torch.where(fine, e + 127, 255).to(torch.uint8)


def _mx_values(code, exps):
    """fp32 values of E2M1 codes with biased block exponents."""
    lut = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=code.device)
    e = exps.to(torch.int32)
    scale = torch.where(e > 0, e << 23, 0x00400000).view(torch.float32)     # 2^(e - 127)
    scale = torch.where(e == 255, math.nan, scale)
    v = lut[code.int()].reshape(code.shape[0], -1, 32) * scale[..., None]
    return v.reshape(code.shape)


def _plain_mx_linear(s):
    codes = torch.stack((s["codes"] & 15, s["codes"] >> 4), -1).flatten(1)
    return {"y": (_mx_values(*_mx_codes(s["x"])) @ _mx_values(codes, s["exps"]).T).to(BF16)}


def _plain_mx_quantize(s):
    return {"values": _mx_values(*_mx_codes(s["x"])).to(BF16)}


# --------------------------------------------------------------------------- the library's own
def _own(s):
    import paper_2403_06082_gb300 as fq
    c = s["case"]
    op, M, d = c["op"], c["M"], c["d"]
    if op == "mx_quantize":
        fq.fq_mxfp_quantize(s["x"], M, d, s["q"])
        fq.fq_mxfp_dequantize(s["q"], s["y"])
        return {"values": s["y"]}
    if op == "mx_linear":
        fq.fq_mxfp_linear(s["x"], M, d, s["q"], s["y"], s["ws"], s["ws_bytes"])
        return {"y": s["y"]}
    head = (s["x"], M, d, s["W"], c["V"])
    if op == "cross_entropy":
        fq.fq_cross_entropy(*head, s["target"], s["loss"], s["lse"], s["ws"], s["ws_bytes"])
    else:
        fq.fq_distill(*head, s["index"], s["logit"], c["K"], s["tau"], s["loss"], s["lse"],
                      s["ws"], s["ws_bytes"])
    out = {"loss": s["loss"], "lse": s["lse"]}
    if c["grad"] == "none":
        return out
    if op == "cross_entropy":
        fq.fq_cross_entropy_grad(*head, s["target"], s["lse"], s["dloss"], s["dx"], s["dW"],
                                 s["ws"], s["ws_bytes"])
    else:
        fq.fq_distill_grad(*head, s["index"], s["logit"], c["K"], s["tau"], s["lse"], s["dloss"],
                           s["dx"], s["dW"], s["ws"], s["ws_bytes"])
    out["dx"] = s["dx"]
    if s["dW"] is not None:
        out["dW"] = s["dW"]
    return out


def run(state):
    if own:
        return _own(state)
    return {"cross_entropy": _plain_cross_entropy, "distill": _plain_distill,
            "mx_linear": _plain_mx_linear, "mx_quantize": _plain_mx_quantize}[
                state["case"]["op"]](state)


# ---------------------------------------------------------------------------------- in 64 bits
def _exact_mx(x):
    """The microscaled values of a matrix in 64 bits: each block's scale is the power of two
    2^(floor(log2(largest)) - 2), each value the nearest of the grid times the scale, the one with
    the even code where two are as near (even codes are tried first, and only a nearer one
    replaces them)."""
    a = x.double().unflatten(1, (-1, 32))
    big = a.abs().amax(-1, keepdim=True)
    _, ex = torch.frexp(big)
    scale = torch.exp2((ex - 3).clamp(min=-127).double())
    scale = torch.where(big == 0, torch.full_like(scale, 2.0 ** -127), scale)
    u = a.abs() / scale
    best, near = torch.zeros_like(u), u.clone()
    for code in (2, 4, 6, 1, 3, 5, 7):
        off = (u - _E2M1[code]).abs()
        closer = off < near
        best = torch.where(closer, torch.full_like(best, _E2M1[code]), best)
        near = torch.where(closer, off, near)
    v = torch.where(torch.isfinite(big), torch.copysign(best, a) * scale, math.nan)
    return v.flatten(1)


def _exact_loss(case, seed):
    s = _loss_inputs(case, seed)
    M, V, tau = case["M"], case["V"], s.get("tau", 1.0)
    # the target distribution of every token over the vocabulary, and its entropy
    if case["op"] == "cross_entropy":
        has = s["target"] >= 0
        at, p = s["target"].long().clamp(min=0)[:, None], has.double()[:, None]
        entropy = torch.zeros(M, dtype=torch.float64, device=DEV)
    else:
        valid = s["index"] >= 0
        has = valid.any(1)
        w = torch.where(valid, s["logit"].double() / tau, -math.inf)
        p = torch.softmax(torch.where(has[:, None], w, 0.0), 1) * valid
        at = s["index"].long().clamp(min=0)
        entropy = -torch.special.xlogy(p, p).sum(1)
    x = torch.where(has[:, None], s["x"].double(), 0.0)
    W = s["W"].double()
    z = (x @ W.T) / tau
    lse = torch.logsumexp(z, 1)
    cross = (p * (lse[:, None] - z.gather(1, at))).sum(1)
    out = {"loss": torch.where(has, tau * tau * (cross - entropy), 0.0),
           "lse": torch.where(has, lse, 0.0)}
    if case["grad"] == "none":
        return out
    z.sub_(lse[:, None]).exp_()
    z.scatter_add_(1, at, -p)
    z.mul_(torch.where(has, s["dloss"].double() * tau, 0.0)[:, None])
    out["dx"] = z @ W
    if case["grad"] == "both":
        out["dW"] = z.T @ x
    return out


def exact(case, seed):
    if case["op"] in ("cross_entropy", "distill"):
        return _exact_loss(case, seed)
    s = _mx_inputs(case, seed)
    if case["op"] == "mx_quantize":
        return {"values": _exact_mx(s["x"])}
    return {"y": _exact_mx(s["x"]) @ _exact_mx(s["W"]).T}
