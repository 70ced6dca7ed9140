"""Operators between and in front of the factorised matrices of a model in training, in their plain form and through
`paper_1910_04732_b200.binding`.

Kinds of case
  embed    rows of a table by word, times a scale.  `mode`: "lookup" is the forward pass alone, "step" also the table's gradient, a row per
           word that occurs and zeros elsewhere.  Words outside the table are padding: a row of zeros, no gradient
  dropout  forward and backward pass, the mask drawn anew from (seed, offset) in both; `residual`: the block's input is added
  norm     layer norm.  `form`: "plain" normalises X; "post" normalises S = R + dropout(X) and returns S too; "pre" is the same with a
           gradient that arrives at S from the blocks behind.  `mode`: "infer" is the forward pass without dropout, "step" both passes
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False     # False: elementary torch operations; True: the library's calls

BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


def listed():
    return [
        # one token decoded; a short ragged batch with an fp32 table; a batch of characters (64 x 256 tokens) into a 2048-wide model, where every
        # row of the gradient is the sum over many tokens; the same batch of words with the 40K-word table, where most rows stay empty
        dict(name="embed_1_token", kind="embed", mode="lookup", T=1, V=32000, d=1024, dtype="bf16", wgrad="bf16"),
        dict(name="embed_1000_ragged_f32", kind="embed", mode="step", T=1000, V=50001, d=410, dtype="f32", wgrad="f32"),
        dict(name="embed_char_2048", kind="embed", mode="step", T=16384, V=205, d=2048, dtype="bf16", wgrad="f32"),
        dict(name="embed_40k_1024", kind="embed", mode="step", T=16384, V=40000, d=1024, dtype="bf16", wgrad="bf16"),
        # one short sequence in fp32; a Transformer-XL batch (60 x 150 tokens, 410 wide) with its residual; an SRU layer's output (64 x 256 tokens)
        dict(name="dropout_24_f32", kind="dropout", T=24, d=768, dtype="f32", p=0.1, residual=False),
        dict(name="dropout_9000_ragged", kind="dropout", T=9000, d=410, dtype="bf16", p=0.1, residual=True),
        dict(name="dropout_16384", kind="dropout", T=16384, d=2048, dtype="bf16", p=0.2, residual=False),
        # one token in front of a pruned matrix; a BERT block's end (32 x 128 tokens); a Transformer-XL batch in fp32 with a gradient that
        # arrives behind the norm; few and long odd rows; an SRU layer's input
        dict(name="norm_1_token", kind="norm", mode="infer", form="plain", T=1, d=1024, dtype="bf16", p=0.0),
        dict(name="norm_bert_4096", kind="norm", mode="step", form="post", T=4096, d=768, dtype="bf16", p=0.1),
        dict(name="norm_9000_ragged_f32", kind="norm", mode="step", form="pre", T=9000, d=410, dtype="f32", p=0.1),
        dict(name="norm_333_wide", kind="norm", mode="step", form="plain", T=333, d=5001, dtype="bf16", p=0.0),
        dict(name="norm_16384", kind="norm", mode="step", form="plain", T=16384, d=2048, dtype="bf16", p=0.0),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm; every other one a multiple of 8."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v if rng.random() < 0.5 else (v + 7) // 8 * 8))


def draw(rng):
    kind = rng.choice(["embed", "dropout", "norm"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    room = 2 ** 24 if dtype == "f32" else 2 ** 25
    if kind == "embed":
        d = _log(rng, 16, 4096)
        return dict(kind=kind, mode=rng.choice(["lookup", "step", "step"]), T=_log(rng, 1, min(131072, room // d)), V=_log(rng, 50, min(200000, room // d)), d=d, dtype=dtype,
                    wgrad=rng.choice(["f32", "bf16"]))
    d = _log(rng, 8, 16384)
    T = _log(rng, 1, min(131072, room // d))
    if kind == "dropout":
        return dict(kind=kind, T=T, d=d, dtype=dtype, p=rng.choice([0.1, 0.15, 0.5]), residual=rng.random() < 0.5)
    mode, form = rng.choice(["infer", "step", "step"]), rng.choice(["plain", "post", "pre"])
    return dict(kind=kind, mode=mode, form=form, T=T, d=d, dtype=dtype, p=0.0 if mode == "infer" or form == "plain" else rng.choice([0.0, 0.1, 0.25]))


# ------------------------------------------------------------------------------------------------ inputs
def _matrix(rows, cols, dtype):
    """Zeros, rows padded to 16 bytes as the library's operands are."""
    per = 16 // dtype.itemsize
    return torch.zeros(rows, (cols + per - 1) // per * per, dtype=dtype, device="cuda")[:, :cols]


def _randn(g, rows, cols, dtype, by=1.0):
    t = _matrix(rows, cols, dtype)
    t.copy_(by * torch.randn(rows, cols, generator=g, device="cuda"))
    return t


def _activations(g, rows, cols, dtype):
    """A residual stream: every column has an offset of its own, one in sixty-four is many times larger, and so are some rows."""
    t = _matrix(rows, cols, dtype)
    size = torch.where(torch.rand(cols, generator=g, device="cuda") < 1 / 64, 12.0, 1.0)
    offset = 0.4 * torch.randn(cols, generator=g, device="cuda")
    loud = torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    t.copy_((torch.randn(rows, cols, generator=g, device="cuda") + offset) * size * loud)
    return t


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    c, kind, T, d = case, case["kind"], case["T"], case["d"]
    dtype = BF16 if c["dtype"] == "bf16" else F32
    s = dict(kind=kind, mode=c.get("mode"), ws=None)
    if kind == "embed":
        V = c["V"]
        # a word's frequency falls with its rank; one token in fifty is padding
        ids = (torch.exp(torch.rand(T, generator=g, device="cuda") * math.log(V + 1)) - 1).to(torch.int32).clamp_(0, V - 1)
        if T > 1:
            ids[torch.rand(T, generator=g, device="cuda") < 0.02] = -1
        s |= dict(ids=ids, E=_randn(g, V, d, dtype, d ** -0.5), scale=math.sqrt(d), Y=_matrix(T, d, dtype))
        if c["mode"] == "step":
            s |= dict(dY=_randn(g, T, d, dtype), dE=_matrix(V, d, F32 if c["wgrad"] == "f32" else BF16))
            if own:
                from paper_1910_04732_b200 import binding as b
                s["ws"] = b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, T, d, 0, V, b.F32 if dtype == F32 else b.BF16))
        return s
    # (seed, offset) of the mask: a step's own key and how far the generator has come
    s |= dict(p=c["p"], key=(int(seed) * 2654435761 + 97) % 2 ** 63, offset=int(seed) % 1000 * 2 ** 24 + 5)
    if kind == "dropout":
        return s | dict(X=_activations(g, T, d, dtype), R=_activations(g, T, d, dtype) if c["residual"] else None, dY=_randn(g, T, d, dtype),
                        Y=_matrix(T, d, dtype), dX=_matrix(T, d, dtype))
    with_sum = c["form"] != "plain"
    s |= dict(X=_activations(g, T, d, dtype), R=_activations(g, T, d, dtype) if with_sum else None, S=_matrix(T, d, dtype) if with_sum else None, Y=_matrix(T, d, dtype),
              weight=1 + 0.1 * torch.randn(d, generator=g, device="cuda"), bias=0.1 * torch.randn(d, generator=g, device="cuda"))
    if c["mode"] == "step":
        s |= dict(stats=torch.zeros(T, 2, device="cuda"), dY=_randn(g, T, d, dtype), dS=_randn(g, T, d, dtype) if c["form"] == "pre" else None, dX=_matrix(T, d, dtype),
                  dR=_matrix(T, d, dtype) if with_sum else None, dweight=torch.zeros(d, device="cuda"), dbias=torch.zeros(d, device="cuda"))
        if own:
            from paper_1910_04732_b200 import binding as b
            s["ws"] = b.alloc_workspace(b.workspace_bytes(b.OP_LAYER_NORM_BWD, T, d, 0, 0, b.F32 if dtype == F32 else b.BF16))
    return s


# ------------------------------------------------------------------------------------------------ the plain form
def _wide_product(a, c):
    """(high, low) 32 bits of a * c for a constant and a tensor of 32-bit values held in 64 bits."""
    low, high = (a & 0xFFFF) * c, (a >> 16) * c
    return (high + (low >> 16)) >> 16, (low + ((high & 0xFFFF) << 16)) & 0xFFFFFFFF


def _mask(s, T, d):
    """Philox4x32-10, counter (offset + T's row * groups of a row + group, 1), eight values of 16 bits a counter; kept where the value is not below the threshold."""
    groups = (d + 7) // 8
    n = s["offset"] + torch.arange(T * groups, dtype=torch.int64, device="cuda")
    x = [n & 0xFFFFFFFF, (n >> 32) & 0xFFFFFFFF, torch.ones_like(n), torch.zeros_like(n)]
    k0, k1 = s["key"] & 0xFFFFFFFF, s["key"] >> 32
    for _ in range(10):
        h0, l0 = _wide_product(0xD2511F53, x[0])
        h1, l1 = _wide_product(0xCD9E8D57, x[2])
        x = [h1 ^ x[1] ^ k0, l1, h0 ^ x[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    values = torch.stack([v for w in x for v in (w & 0xFFFF, w >> 16)], 1).view(T, groups * 8)[:, :d]
    return values >= _threshold(s["p"])


def _threshold(p):
    return min(int(math.floor(p * 65536 + 0.5)), 65535)


def _dropped(s, x):
    """Dropout in 32 bits: 65536 / (65536 - threshold) of what is kept."""
    if s["p"] == 0:
        return x
    return torch.where(_mask(s, *x.shape), x * (65536 / (65536 - _threshold(s["p"]))), 0.0)


def _plain_embed(s):
    ids = s["ids"].long()
    V, d = s["E"].shape
    real = (ids >= 0) & (ids < V)
    Y = torch.where(real[:, None], s["E"][torch.where(real, ids, 0)].float() * s["scale"], 0.0).to(s["E"].dtype)
    if s["mode"] == "lookup":
        return Y
    rows = torch.zeros(V + 1, d, device="cuda").index_add_(0, torch.where(real, ids, V), s["dY"].float())
    return Y, (rows[:V] * s["scale"]).to(s["dE"].dtype)


def _plain_dropout(s):
    Y = _dropped(s, s["X"].float())
    if s["R"] is not None:
        Y = Y + s["R"].float()
    return Y.to(s["Y"].dtype), _dropped(s, s["dY"].float()).to(s["dX"].dtype)


def _plain_norm(s):
    dtype = s["X"].dtype
    x = s["X"].float()
    if s["R"] is not None:
        S = (s["R"].float() + _dropped(s, x)).to(dtype)         # the residual stream in its own type: what is kept is what is normalised
        x = S.float()
    x = x - x.mean(1, keepdim=True)
    rstd = (x.square().mean(1, keepdim=True) + EPS).rsqrt()
    x = x * rstd
    Y = (x * s["weight"] + s["bias"]).to(dtype)
    out = (Y,) if s["R"] is None else (S, Y)
    if s["mode"] == "infer":
        return out
    dY = s["dY"].float()
    a = dY * s["weight"]
    g = rstd * (a - a.mean(1, keepdim=True) - x * (a * x).mean(1, keepdim=True))
    if s["dS"] is not None:
        g = g + s["dS"].float()
    out += (_dropped(s, g).to(dtype),)
    if s["R"] is not None:
        out += (g.to(dtype),)
    return out + ((dY * x).sum(0), dY.sum(0))


# ------------------------------------------------------------------------------------------------ one pass
def _own(s):
    from paper_1910_04732_b200 import binding as b
    if s["kind"] == "embed":
        b.embedding_fwd(s["ids"], s["E"], s["scale"], s["Y"])
        if s["mode"] == "lookup":
            return s["Y"]
        b.embedding_bwd(s["dY"], s["ids"], s["scale"], s["dE"], s["ws"])
        return s["Y"], s["dE"]
    random = dict(p=s["p"], seed=s["key"], offset=s["offset"])
    if s["kind"] == "dropout":
        b.dropout_fwd(s["X"], s["Y"], R=s["R"], **random)
        b.dropout_bwd(s["dY"], s["dX"], **random)
        return s["Y"], s["dX"]
    plain = s["R"] is None
    random = {} if plain else random
    step = s["mode"] == "step"
    b.layer_norm_fwd(s["X"], s["weight"], s["bias"], EPS, s["Y"], s["stats"] if step else None, R=s["R"], S=s["S"], **random)
    out = (s["Y"],) if plain else (s["S"], s["Y"])
    if not step:
        return out
    b.layer_norm_bwd(s["dY"], s["X"] if plain else s["S"], s["stats"], s["weight"], s["dX"], s["dweight"], s["dbias"], s["ws"], dS=s["dS"], dR=s["dR"], **random)
    return out + ((s["dX"],) if plain else (s["dX"], s["dR"])) + (s["dweight"], s["dbias"])


def run(state):
    if own:
        return _own(state)
    return {"embed": _plain_embed, "dropout": _plain_dropout, "norm": _plain_norm}[state["kind"]](state)


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def _kept(s, T, d):
    """The mask as 0 and 1 in 64 bits, from numpy's unsigned integers."""
    per_row = -(-d // 8)
    ctr = np.arange(T * per_row, dtype=np.uint64) + np.uint64(s["offset"])
    low = np.uint64(0xFFFFFFFF)
    a, b, c, e = ctr & low, ctr >> np.uint64(32), np.full_like(ctr, 1), np.zeros_like(ctr)
    for r in range(10):
        ka, kb = ((s["key"] & 0xFFFFFFFF) + r * 0x9E3779B9) % 2 ** 32, ((s["key"] >> 32) + r * 0xBB67AE85) % 2 ** 32
        left, right = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b, c, e = (right >> np.uint64(32)) ^ b ^ np.uint64(ka), right & low, (left >> np.uint64(32)) ^ e ^ np.uint64(kb), left & low
    words = np.stack([a, b, c, e], 1).astype("<u4")
    values = words.view("<u2").reshape(T, per_row * 8)[:, :d]
    return torch.from_numpy((values >= _threshold(s["p"])).astype(np.float64)).cuda()


def _exact_embed(s):
    V, d = s["E"].shape
    padded = torch.cat([s["E"].double() * s["scale"], torch.zeros(1, d, dtype=torch.float64, device="cuda")])
    at = s["ids"].long()
    at = torch.where(at < 0, V, at).clamp_max(V)
    Y = padded[at]
    if s["mode"] == "lookup":
        return Y
    by_word = torch.sort(at, stable=True)
    runs, counts = torch.unique_consecutive(by_word.values, return_counts=True)
    total = torch.cumsum(s["dY"].double()[by_word.indices], 0)
    total = total[torch.cumsum(counts, 0) - 1]
    total[1:] -= total[:-1].clone()
    dE = torch.zeros(V + 1, d, dtype=torch.float64, device="cuda")
    dE[runs] = total * s["scale"]
    return Y, dE[:V]


def _exact_dropout(s):
    T, d = s["X"].shape
    factor = _kept(s, T, d) * 65536 / (65536 - _threshold(s["p"]))
    Y = s["X"].double() * factor
    return Y if s["R"] is None else Y + s["R"].double(), s["dY"].double() * factor


def _exact_norm(s):
    X = s["X"].double()
    T, d = X.shape
    factor = 1.0
    if s["R"] is not None:
        if s["p"] > 0:
            factor = _kept(s, T, d) * 65536 / (65536 - _threshold(s["p"]))
        total = X * factor + s["R"].double()
        X = total.to(s["X"].dtype).double()                     # S in the type that it is kept in
    var, mean = torch.var_mean(X, 1, correction=0, keepdim=True)
    unit = torch.sqrt(var + EPS)
    xhat = (X - mean) / unit
    w = s["weight"].double()
    Y = xhat * w + s["bias"].double()
    out = [Y] if s["R"] is None else [total, Y]
    if s["mode"] == "step":
        dY = s["dY"].double()
        dx = dY * w
        dx = (dx - (dx.sum(1, keepdim=True) + xhat * (dx * xhat).sum(1, keepdim=True)) / d) / unit
        if s["dS"] is not None:
            dx = dx + s["dS"].double()
        out += [dx * factor] if s["R"] is None else [dx * factor, dx]
        out += [(dY * xhat).sum(0), dY.sum(0)]
    return tuple(out)


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "dropout": _exact_dropout, "norm": _exact_norm}[s["kind"]](s)


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    c, kind, e = case, case["kind"], 2 if case["dtype"] == "bf16" else 4
    T, d = c["T"], c["d"]
    row = e * T * d
    if kind == "embed":
        # lookup: the rows that occur, at most, and what is written; gradient: what arrives, and the whole table's gradient
        out = dict(bytes=float(4 * T + e * min(T, c["V"]) * d + row), flops=float(T * d))
        if c["mode"] == "step":
            out["bytes"] += 4.0 * T + row + (2 if c["wgrad"] == "bf16" else 4) * c["V"] * d
            out["flops"] += T * d + c["V"] * d
        return out
    if kind == "dropout":
        # X and Y, dY and dX, the residual; the generator's integer operations are not counted
        return dict(bytes=float(row * (5 if c["residual"] else 4)), flops=2.0 * T * d)
    with_sum = c["form"] != "plain"
    tensors = 4 if with_sum else 2                              # X, Y; R and S
    out = dict(bytes=float(tensors * row + 8 * d), flops=8.0 * T * d)
    if c["mode"] == "step":
        # dY and X or S again, dX; dR; the gradient that arrives at S; mean and 1 / deviation written and read
        out["bytes"] += (3 + (1 if with_sum else 0) + (1 if c["form"] == "pre" else 0)) * row + 16 * T + 12 * d
        out["flops"] += 14.0 * T * d
    return out
