"""Two sets of operators around a pruned language model, in their plain form and through `paper_1910_04732_b200.binding`.

Kinds of case
  linear   a product with 8-bit weights: the tokens are quantised (a scale per token), multiplied with weights quantised per
           output channel, and the sums scaled back
  compact  the forward pass of one pruned matrix on its compact factors in 8 bits: both products, the intermediate
           requantised per token
  distill  the loss of a student's logits against a teacher's top logits.  `mode`: "eval" is the loss alone, "autograd" the forward
           call and, from what it saved, the backward call, "fused" loss and gradient in one call.  `rest`: the teacher's
           log-sum-exp over the whole vocabulary is known and its remaining mass is one more bucket; without it the top
           logits are normalised among themselves
"""
from __future__ import annotations

import math

import torch

own = False     # False: elementary torch operations; True: the library's calls

BF16, F32 = torch.bfloat16, torch.float32


def listed():
    return [
        # decoding one sequence through a dense 1024 -> 4096 matrix; one Transformer-XL segment through a feed-forward matrix
        # with its odd widths, fp32 activations; a training batch's worth of tokens (64 x 256) through an SRU projection
        dict(name="linear_1_token", kind="linear", T=1, d_in=1024, d_out=4096, dtype="bf16"),
        dict(name="linear_150_ragged_f32", kind="linear", T=150, d_in=410, d_out=2100, dtype="f32"),
        dict(name="linear_16384_tokens", kind="linear", T=16384, d_in=2048, d_out=6144, dtype="bf16"),
        # pruned inference, 1024 -> 4096 with about 35 % of the rank components: one token, a batch of 16, a ragged segment, a prefill
        dict(name="compact_1_token", kind="compact", T=1, d_in=1024, d_out=4096, k=358, dtype="bf16"),
        dict(name="compact_16_tokens", kind="compact", T=16, d_in=1024, d_out=4096, k=358, dtype="bf16"),
        dict(name="compact_150_ragged_f32", kind="compact", T=150, d_in=410, d_out=2100, k=143, dtype="f32"),
        dict(name="compact_4096_tokens", kind="compact", T=4096, d_in=1024, d_out=4096, k=358, dtype="bf16"),
        # a character-level model (64 x 256 tokens); the 40K-word vocabulary in fp32, evaluated; a ragged vocabulary through
        # autograd; one short sequence; a large vocabulary with a long batch
        dict(name="distill_char_fused", kind="distill", mode="fused", T=16384, V=205, K=16, dtype="bf16", tau=1.0, rest=True),
        dict(name="distill_40k_eval_f32", kind="distill", mode="eval", T=512, V=40000, K=32, dtype="f32", tau=2.0, rest=True),
        dict(name="distill_ragged_autograd", kind="distill", mode="autograd", T=1000, V=50001, K=100, dtype="bf16", tau=2.0, rest=False),
        dict(name="distill_24_fused", kind="distill", mode="fused", T=24, V=32000, K=20, dtype="bf16", tau=1.0, rest=False),
        dict(name="distill_128k_fused", kind="distill", mode="fused", T=4096, V=128000, K=64, dtype="bf16", tau=1.0, rest=True),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm; every other one a multiple of 16."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v if rng.random() < 0.5 else (v + 15) // 16 * 16))


def draw(rng):
    kind = rng.choice(["linear", "compact", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "linear":
        d_in, d_out = _log(rng, 16, 8192), _log(rng, 16, 8192)
        return dict(kind=kind, T=_log(rng, 1, min(16384, 2 * 10 ** 11 // (d_in * d_out))), d_in=d_in, d_out=d_out, dtype=dtype)
    if kind == "compact":
        d_in, d_out = _log(rng, 64, 4096), _log(rng, 64, 4096)
        return dict(kind=kind, T=_log(rng, 1, 8192), d_in=d_in, d_out=d_out, k=max(1, round(min(d_in, d_out) * rng.uniform(0.05, 0.6))), dtype=dtype)
    V = _log(rng, 100, 200000)
    return dict(kind=kind, mode=rng.choice(["eval", "autograd", "fused"]), T=_log(rng, 1, min(16384, (200 if dtype == "f32" else 400) * 10 ** 6 // V)), V=V,
                K=_log(rng, 1, min(256, V // 2)), dtype=dtype, tau=rng.choice([1.0, 2.0, 3.5]), rest=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _matrix(rows, cols, dtype):
    """Zeros, rows padded to 16 bytes as the library's operands are."""
    per = 16 // dtype.itemsize
    return torch.zeros(rows, (cols + per - 1) // per * per, dtype=dtype, device="cuda")[:, :cols]


def _randn(g, rows, cols, dtype):
    t = _matrix(rows, cols, dtype)
    t.copy_(torch.randn(rows, cols, generator=g, device="cuda"))
    return t


def _weights(g, rows, cols):
    """Weights as a deployed model keeps them: 8 bits and a scale per output channel."""
    w = torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5
    scale = w.abs().amax(1) / 127
    q = _matrix(rows, cols, torch.int8)
    q.copy_(torch.round(w / scale[:, None]).clamp_(-127, 127))
    return q, scale


def _prepare_distill(c, g, dtype):
    T, V, K, tau = c["T"], c["V"], c["K"], c["tau"]
    S = _matrix(T, V, dtype)
    t_logits, t_idx, t_lse = torch.empty(T, K, device="cuda"), torch.empty(T, K, dtype=torch.int32, device="cuda"), torch.empty(T, device="cuda")
    step = max(1, 2 ** 27 // V)
    for lo in range(0, T, step):
        n = min(step, T - lo)
        # a bulk of unlikely words and about twenty likely ones
        teacher = torch.randn(n, V, generator=g, device="cuda") + 14 * torch.rand(n, V, generator=g, device="cuda") ** (V / 20)
        t_logits[lo:lo + n], top = teacher.topk(K, dim=1)
        t_idx[lo:lo + n] = top
        t_lse[lo:lo + n] = torch.logsumexp(teacher.double() / tau, 1)
        S[lo:lo + n] = 0.8 * teacher + 0.7 * torch.randn(n, V, generator=g, device="cuda")
    # stored teachers cut their lists by mass: shorter ones end in -1
    length = 1 + (torch.rand(T, 1, generator=g, device="cuda") * 1.5 * K).long()
    t_idx[torch.arange(K, device="cuda")[None] >= length] = -1
    # padding takes no part in the mean over tokens
    real = (torch.rand(T, generator=g, device="cuda") < 0.95).float()
    real[0] = 1
    s = dict(S=S, t_logits=t_logits, t_idx=t_idx, t_lse=t_lse if c["rest"] else None, tau=tau, loss=torch.zeros(T, device="cuda"))
    if c["mode"] == "autograd":     # the mean comes after the loss: its gradient arrives with the backward call
        s |= dict(weight=real, dloss=tau * tau * real / real.sum(), stats=torch.zeros(T, 4, device="cuda"))
    else:
        s |= dict(weight=tau * tau * real / real.sum(), dloss=None)
    if c["mode"] != "eval":
        s["dS"] = _matrix(T, V, dtype)
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    c, kind, dtype = case, case["kind"], BF16 if case["dtype"] == "bf16" else F32
    if kind == "distill":
        return dict(_prepare_distill(c, g, dtype), kind=kind, mode=c["mode"])
    s = dict(kind=kind, X=_randn(g, c["T"], c["d_in"], dtype), Y=_matrix(c["T"], c["d_out"], dtype))
    if kind == "linear":
        W, w_scale = _weights(g, c["d_out"], c["d_in"])
        return dict(s, W=W, w_scale=w_scale, Xq=_matrix(c["T"], c["d_in"], torch.int8), x_scale=torch.zeros(c["T"], device="cuda"))
    Qq, q_scale = _weights(g, c["k"], c["d_in"])
    Pq, p_scale = _weights(g, c["d_out"], c["k"])
    # scratch for the quantised tokens and the intermediate, in 32 and in 8 bits
    return dict(s, Qq=Qq, q_scale=q_scale, Pq=Pq, p_scale=p_scale, ws=torch.empty(8 * c["T"] * (c["k"] + c["d_in"] + 64) + 2 ** 20, dtype=torch.uint8, device="cuda"))


# ------------------------------------------------------------------------------------------------ the plain form
def _quantize(x):
    """(8-bit values, scale) of each row; the quotient in 64 bits, because a value next to a border must fall on its side."""
    amax = x.abs().amax(1, keepdim=True)
    q = torch.round(127.0 * x.double() / amax.double())
    return torch.where(amax > 0, q, 0.0), amax[:, 0] / 127


def _plain_linear(s):
    q, scale = _quantize(s["X"].float())
    acc = q.float() @ s["W"].float().T
    return (acc * scale[:, None] * s["w_scale"]).to(s["Y"].dtype)


def _plain_compact(s):
    q, scale = _quantize(s["X"].float())
    h = (q @ s["Qq"].double().T) * s["q_scale"].double()        # 64 bits: what is next to a border is rounded below
    hq, h_scale = _quantize(h)
    acc = hq.float() @ s["Pq"].float().T
    return (acc * (scale * h_scale).float()[:, None] * s["p_scale"]).to(s["Y"].dtype)


def _plain_distill(s):
    S, tau, idx = s["S"], s["tau"], s["t_idx"].long()
    T, V = S.shape
    listed_ = (idx >= 0) & (idx < V)
    at = torch.where(listed_, idx, V)
    in_list = torch.zeros(T, V + 1, dtype=torch.bool, device=S.device).scatter_(1, at, True)[:, :V]
    at = torch.where(listed_, idx, 0)
    x = S.float() / tau
    x -= x.amax(1, keepdim=True)
    top = torch.where(listed_, x.gather(1, at), -math.inf)
    e = x.exp_()
    rest = torch.where(in_list, 0.0, e).sum(1)
    total = rest + top.exp().sum(1)
    log_p = top - total.log()[:, None]
    t = torch.where(listed_, s["t_logits"] / tau, -math.inf)
    if s["t_lse"] is None:
        log_q = t - torch.logsumexp(t, 1, keepdim=True)
    else:
        log_q = t - s["t_lse"][:, None]
    q = log_q.exp()
    kl = torch.where(q > 0, q * (log_q - log_p), 0.0).sum(1)
    pull = torch.zeros(T, device=S.device)
    if s["t_lse"] is not None:
        r = (1 - log_q.double().exp().sum(1)).clamp_min(0).float()      # 64 bits: what is left of one
        kl += torch.where(r > 0, r * (r.log() - (rest / total).log()), 0.0)
        pull = r / rest
    loss = torch.where(s["weight"] != 0, s["weight"] * kl, 0.0)
    if s["mode"] == "eval":
        return loss
    scale = s["weight"] / tau
    if s["dloss"] is not None:
        scale = scale * s["dloss"]
    p_top = top.exp() / total[:, None]
    grad = e * (1 / total - pull)[:, None]
    grad = torch.cat([grad, grad[:, :1]], 1).scatter_(1, torch.where(listed_, idx, V), p_top - q)[:, :V]
    return loss, torch.where(scale[:, None] != 0, grad * scale[:, None], 0.0).to(S.dtype)


# ------------------------------------------------------------------------------------------------ one pass
def _own(s):
    from paper_1910_04732_b200 import binding as b
    if s["kind"] == "linear":
        b.quantize_rows(s["X"], s["Xq"], s["x_scale"])
        b.gemm_i8(s["Xq"], s["W"], s["x_scale"], s["w_scale"], s["Y"])
        return s["Y"]
    if s["kind"] == "compact":
        b.compact_fwd_i8(s["X"], s["Qq"], s["q_scale"], s["Pq"], s["p_scale"], s["Y"], s["Qq"].shape[0], s["ws"])
        return s["Y"]
    teacher = (s["t_logits"], s["t_idx"], s["t_lse"], s["weight"], s["tau"])
    if s["mode"] == "eval":
        b.distill_topk_fwd(s["S"], *teacher, s["loss"])
        return s["loss"]
    if s["mode"] == "autograd":
        b.distill_topk_fwd(s["S"], *teacher, s["loss"], s["stats"])
        b.distill_topk_bwd(s["S"], *teacher, s["stats"], s["dloss"], s["dS"])
    else:
        b.distill_topk_fwd_bwd(s["S"], *teacher, s["loss"], s["dS"])
    return s["loss"], s["dS"]


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "compact": _plain_compact, "distill": _plain_distill}[state["kind"]](state)


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def _rounded(v):
    """Rows as whole multiples of a 127th of their largest magnitude (half to even): the values that 8 bits stand for."""
    unit = v.abs().max(1, keepdim=True).values / 127
    return torch.where(unit > 0, torch.round(v / unit.clamp_min(1e-300)) * unit, v)


def _exact_distill(s):
    T, V = s["S"].shape
    tau = s["tau"]
    loss, grads = torch.zeros(T, dtype=torch.float64, device="cuda"), None
    if s["mode"] != "eval":
        grads = torch.zeros(T, V, dtype=torch.float64, device="cuda")
    step = max(1, 2 ** 26 // V)
    for lo in range(0, T, step):
        rows = slice(lo, min(T, lo + step))
        z = s["S"][rows].double() / tau
        idx = s["t_idx"][rows].long()
        row, slot = torch.nonzero((idx >= 0) & (idx < V), as_tuple=True)
        col = idx[row, slot]
        n = z.shape[0]
        t = torch.full((n, V), -math.inf, dtype=torch.float64, device="cuda")
        t[row, col] = s["t_logits"][rows].double()[row, slot] / tau
        norm = torch.logsumexp(t, 1) if s["t_lse"] is None else s["t_lse"][rows].double()
        logq = t - norm[:, None]
        logp = torch.log_softmax(z, 1)
        on = torch.isfinite(t)
        each = torch.zeros_like(z)
        each[on] = logq[on].exp() * (logq[on] - logp[on])
        kl = each.sum(1)
        g = logp.exp() - logq.exp()
        if s["t_lse"] is not None:
            left = (1 - logq.exp().sum(1)).clamp_min(0)
            off = torch.where(on, -math.inf, z)
            log_rest = torch.logsumexp(off, 1) - torch.logsumexp(z, 1)
            kl = kl + torch.xlogy(left, left) - torch.where(left > 0, left * log_rest, 0.0)
            g = g - left[:, None] * torch.softmax(off, 1)
        w = s["weight"][rows].double()
        loss[rows] = torch.where(w != 0, w * kl, 0.0)
        if grads is not None:
            w = w / tau if s["dloss"] is None else w * s["dloss"][rows].double() / tau
            grads[rows] = torch.where(w[:, None] != 0, w[:, None] * g, 0.0)
    return loss if grads is None else (loss, grads)


def exact(case, seed):
    s = prepare(case, seed)
    if s["kind"] == "distill":
        return _exact_distill(s)
    x = _rounded(s["X"].double())
    if s["kind"] == "linear":
        return x @ (s["W"].double() * s["w_scale"].double()[:, None]).T
    h = _exact_intermediate(s)
    return h @ (s["Pq"].double() * s["p_scale"].double()[:, None]).T


def _exact_intermediate(s):
    """The intermediate after its rounding.  The scale of a token belongs to its whole row, so the integers do not depend on it: the
    sums are taken over integers and stay exact."""
    X = s["X"].double()
    unit = X.abs().max(1, keepdim=True).values / 127
    whole = torch.where(unit > 0, torch.round(X / unit.clamp_min(1e-300)), 0.0)
    return _rounded((whole @ s["Qq"].double().T) * s["q_scale"].double()) * unit


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    c, kind, e = case, case["kind"], 2 if case["dtype"] == "bf16" else 4
    T = c["T"]
    if kind == "linear":
        return dict(bytes=float(e * T * (c["d_in"] + c["d_out"]) + c["d_in"] * c["d_out"] + 4 * c["d_out"]), flops=2.0 * T * c["d_in"] * c["d_out"])
    if kind == "compact":
        w = c["k"] * (c["d_in"] + c["d_out"])
        return dict(bytes=float(e * T * (c["d_in"] + c["d_out"]) + w + 4 * (c["k"] + c["d_out"])), flops=2.0 * T * w)
    # eval reads the logits, fused reads them and writes their gradient, autograd reads them once more
    passes = {"eval": 1, "fused": 2, "autograd": 3}[c["mode"]]
    return dict(bytes=float(e * passes * T * c["V"] + 8 * T * c["K"] + 12 * T), flops=8.0 * T * c["V"])
