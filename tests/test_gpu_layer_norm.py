"""Layer norm, alone and with dropout and residual, forward and backward, against the oracle within bounds of 32-bit evaluation."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from tests.test_gpu_embedding_rows import TYPES, filled, host, matrix

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def rows(g, T, d):
    return (g.standard_normal((T, d)) + 0.5 * g.standard_normal(d)) * np.exp(0.5 * g.standard_normal((T, 1)))


def vector(g, d, at):
    return torch.from_numpy((at + 0.3 * g.standard_normal(d)).astype(np.float32)).cuda()


def workspace(b, T, d, kind):
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_LAYER_NORM_BWD, T, d, 0, 0, b.BF16 if kind == "bf16" else b.F32))
    return ws.fill_(0xFF)


def check(b, kind, T, d, form, p=0.0, affine=True, eps=EPS, accumulate=False, seed=3, offset=4, **place):
    """One forward and one backward call; the oracle starts from the S that the forward call wrote."""
    g = np.random.default_rng(T * 7 + d)
    X, dY = filled(rows(g, T, d), kind, **place), filled(g.standard_normal((T, d)), kind, **place)
    w, bias = (vector(g, d, 1.0), vector(g, d, 0.0)) if affine else (None, None)
    wh, bh = (host(w), host(bias)) if affine else (None, None)
    eps32 = float(np.float32(eps))
    Res = S = dS = dR = None
    mask = {}
    if form != "plain":
        Res, S, dR = filled(rows(g, T, d), kind, **place), matrix(T, d, kind, **place)[0], matrix(T, d, kind, **place)[0]
        dS = filled(g.standard_normal((T, d)), kind, **place) if form == "pre" else None
        mask = dict(p=p, seed=seed, offset=offset)
    Y, buf = matrix(T, d, kind, **place)
    stats = torch.full((T, 2), float("nan"), device="cuda")
    b.layer_norm_fwd(X, w, bias, eps, Y, stats, R=Res, S=S, **mask)
    keep, s = R.dropout_mask(T, d, p, seed, offset)
    if S is not None:
        total = R.dropout(host(X), p, seed, offset, host(Res))
        assert np.all(np.abs(host(S) - total) <= R.U * (2 * s * np.abs(host(X)) + np.abs(total)) + R.HALF_STEP[kind] * np.abs(total) * (1 + 2 ** -7) + 1e-38)
    N = host(X if S is None else S)
    want, mean, rstd = R.layer_norm_fwd(N, wh, bh, eps32)
    assert np.all(np.abs(host(Y) - want) <= R.layer_norm_fwd_bound(N, wh, bh, eps32, kind)), np.abs(host(Y) - want).max()
    # nothing kept: the same rows
    Y2, _ = matrix(T, d, kind, **place)
    b.layer_norm_fwd(X, w, bias, eps, Y2, R=Res, **mask)
    assert torch.equal(Y2, Y)
    dX, out = matrix(T, d, kind, **place)
    dw, db = (vector(g, d, 0.0), vector(g, d, 1.0)) if accumulate else (torch.full((d,), float("nan"), device="cuda") for _ in range(2))
    old = (host(dw), host(db)) if accumulate else (0.0, 0.0)
    b.layer_norm_bwd(dY, X if S is None else S, stats, w, dX, dw, db, workspace(b, T, d, kind), dS=dS, dR=dR, accumulate=accumulate, **mask)
    args = host(dY), N, wh, eps32
    g_want, dw_want, db_want = R.layer_norm_bwd(*args, None if dS is None else host(dS))
    g_bound, dw_bound, db_bound = R.layer_norm_bwd_bound(*args, kind, None if dS is None else host(dS))
    if dR is not None:
        assert np.all(np.abs(host(dR) - g_want) <= g_bound), np.abs(host(dR) - g_want).max()
    dx_want = np.where(keep, g_want * s, 0.0)
    assert np.all(np.abs(host(dX) - dx_want) <= np.where(keep, s * g_bound + 2 * R.U * np.abs(dx_want), 0.0)), np.abs(host(dX) - dx_want).max()
    for name, got, was, exact, bound in (("dweight", dw, old[0], dw_want, dw_bound), ("dbias", db, old[1], db_want, db_bound)):
        assert np.all(np.abs(host(got) - (was + exact)) <= bound + R.U * np.abs(was + exact)), name
    for m, whole in ((Y, buf), (dX, out)):
        m.fill_(float("nan"))
        assert torch.isnan(whole).all()


SIZES = [(1, 1), (1, 8), (2, 3), (5, 9), (3, 64), (17, 72), (33, 136), (9, 264), (40, 410), (65, 512), (130, 768), (7, 1000), (70, 1024), (11, 1032), (20, 2048), (5, 2056),
         (6, 4096), (3, 5001), (4, 8192), (2, 8200), (3, 16384), (2, 16392), (2, 40001), (1100, 40), (3000, 16)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SIZES)
def test_plain(b, kind, T, d):
    check(b, kind, T, d, "plain")


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("form,p", [("post", 0.1), ("post", 0.0), ("pre", 0.25)])
@pytest.mark.parametrize("T,d", [(1, 1), (5, 9), (17, 72), (40, 410), (130, 768), (20, 2048), (3, 5001), (2, 16392), (600, 130)])
def test_with_dropout_and_residual(b, kind, form, p, T, d):
    check(b, kind, T, d, form, p)


@pytest.mark.parametrize("T,d", [(40, 410), (3, 5001), (900, 24)])
def test_gradients_are_added_and_vectors_are_optional(b, T, d):
    check(b, "bf16", T, d, "pre", 0.1, accumulate=True)
    check(b, "f32", T, d, "plain", affine=False)
    check(b, "f32", T, d, "post", 0.2, eps=0.1)


@pytest.mark.parametrize("d,ld,shift", [(13, 13, 0), (64, 67, 1), (410, 411, 3), (20, 24, 4), (2047, 2050, 2)])
def test_fp32_rows_of_any_pitch(b, d, ld, shift):
    check(b, "f32", 30, d, "pre", 0.3, ld=ld, shift=shift)
    check(b, "f32", 30, d, "plain", ld=ld, shift=shift)


def test_vectors_that_start_anywhere(b):
    g = torch.Generator(device="cuda").manual_seed(1)
    T, d = 30, 328
    X, dY, v = (torch.randn(*s, generator=g, device="cuda") for s in ((T, d), (T, d), (2 * d + 2,)))
    out = []
    for w, bias in ((v[1:d + 1], v[d + 1:2 * d + 1]), (v[1:d + 1].clone(), v[d + 1:2 * d + 1].clone())):
        Y, stats, dX, dw, db = torch.empty_like(X), torch.empty(T, 2, device="cuda"), torch.empty_like(X), torch.empty(d + 1, device="cuda")[1:], torch.empty(d, device="cuda")
        b.layer_norm_fwd(X, w, bias, EPS, Y, stats)
        b.layer_norm_bwd(dY, X, stats, w, dX, dw, db, workspace(b, T, d, "f32"))
        out.append((Y, dX, dw, db))
    for x, y in zip(*out):
        assert torch.equal(x, y)


@pytest.mark.parametrize("d", [72, 410, 1024, 2048, 5001, 16392])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_in_place(b, d, kind):
    """Every output that may take an input's place gives the same bits there."""
    g = np.random.default_rng(d)
    T, mask = 9, dict(p=0.2, seed=1, offset=2)
    new = lambda: filled(rows(g, T, d), kind)  # noqa: E731
    copy = lambda m: filled(host(m), kind)  # noqa: E731
    X, Res, dY, dS, w, bias = new(), new(), new(), new(), vector(g, d, 1.0), vector(g, d, 0.0)
    S, Y, stats = matrix(T, d, kind)[0], matrix(T, d, kind)[0], torch.empty(T, 2, device="cuda")
    b.layer_norm_fwd(X, w, bias, EPS, Y, stats, R=Res, S=S, **mask)
    for s_at, y_at in (("X", "R"), ("R", "X"), ("X", None), ("R", None), (None, "X"), (None, "R")):
        at = {"X": copy(X), "R": copy(Res), None: matrix(T, d, kind)[0]}
        y = at[y_at] if y_at else matrix(T, d, kind)[0]
        b.layer_norm_fwd(at["X"], w, bias, EPS, y, R=at["R"], S=at[s_at], **mask)
        assert torch.equal(y, Y) and torch.equal(at[s_at], S), (s_at, y_at)
        if s_at is None:                                     # and without S
            at = {"X": copy(X), "R": copy(Res)}
            b.layer_norm_fwd(at["X"], w, bias, EPS, at[y_at], R=at["R"], **mask)
            assert torch.equal(at[y_at], Y)
    dX, dR, dw, db = matrix(T, d, kind)[0], matrix(T, d, kind)[0], torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    b.layer_norm_bwd(dY, S, stats, w, dX, dw, db, workspace(b, T, d, kind), dS=dS, dR=dR, **mask)
    for x_at, r_at in (("dY", "dS"), ("dS", "dY"), ("S", "dY"), ("dY", "S")):
        at = {"dY": copy(dY), "dS": copy(dS), "S": copy(S)}
        dw2, db2 = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        b.layer_norm_bwd(at["dY"], at["S"], stats, w, at[x_at], dw2, db2, workspace(b, T, d, kind), dS=at["dS"], dR=at[r_at], **mask)
        assert torch.equal(at[x_at], dX) and torch.equal(at[r_at], dR) and torch.equal(dw2, dw) and torch.equal(db2, db), (x_at, r_at)


@pytest.mark.parametrize("d", [64, 410, 2048, 16392])
def test_outputs_that_are_not_wanted(b, d):
    g = np.random.default_rng(d)
    T, kind = 12, "bf16"
    S, dY, w = filled(rows(g, T, d), kind), filled(rows(g, T, d), kind), vector(g, d, 1.0)
    Y, stats = matrix(T, d, kind)[0], torch.empty(T, 2, device="cuda")
    b.layer_norm_fwd(S, w, None, EPS, Y, stats)
    dX, dw, db = matrix(T, d, kind)[0], torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    b.layer_norm_bwd(dY, S, stats, w, dX, dw, db, workspace(b, T, d, kind))
    for which in range(1, 8):
        x, w1, b1 = matrix(T, d, kind)[0], torch.full((d,), 7.0, device="cuda"), torch.full((d,), 7.0, device="cuda")
        b.layer_norm_bwd(dY, S, stats, w, x if which & 1 else None, w1 if which & 2 else None, b1 if which & 4 else None, workspace(b, T, d, kind) if which & 6 else None)
        assert not which & 1 or torch.equal(x, dX)
        assert torch.equal(w1, dw) if which & 2 else torch.all(w1 == 7)
        assert torch.equal(b1, db) if which & 4 else torch.all(b1 == 7)


@pytest.mark.parametrize("d", [1, 64, 410, 2048, 16392])
def test_rows_of_equal_values_and_rows_that_are_not_finite(b, d):
    T = 6
    X = torch.randn(T, d, device="cuda")
    X[1], X[3, 0], X[4, d - 1] = 2.5, float("nan"), float("inf")
    bias = torch.full((d,), 0.25, device="cuda")
    Y, stats = torch.empty_like(X), torch.empty(T, 2, device="cuda")
    b.layer_norm_fwd(X, None, bias, EPS, Y, stats)
    assert torch.all(Y[1] == 0.25) and stats[1].tolist() == pytest.approx([2.5, EPS ** -0.5], rel=1e-5)
    assert torch.isnan(Y[3]).all() and torch.isnan(Y[4]).all() and torch.isfinite(Y[[0, 1, 2, 5]]).all()
    dY, dX = torch.randn(T, d, device="cuda"), torch.empty_like(X)
    b.layer_norm_bwd(dY, X, stats, None, dX, None, None, None)
    assert torch.isnan(dX[3]).all() and torch.isnan(dX[4]).all() and torch.isfinite(dX[[0, 1, 2, 5]]).all()
    # a NaN behind a row's end reaches nothing
    wide = torch.full((T, d + 5), float("nan"), device="cuda")
    wide[:, :d] = X
    b.layer_norm_fwd(wide[:, :d], None, bias, EPS, dX)
    assert torch.equal(dX[[0, 1, 2, 5]], Y[[0, 1, 2, 5]])


def test_no_rows(b):
    d = 40
    none, dw, db = torch.zeros(0, d, device="cuda"), torch.ones(d, device="cuda"), torch.ones(d, device="cuda")
    b.layer_norm_fwd(none, None, None, EPS, none.clone())
    b.layer_norm_bwd(none, none, torch.zeros(0, 2, device="cuda"), None, None, dw, db, None, accumulate=True)
    assert torch.all(dw == 1)
    b.layer_norm_bwd(none, none, torch.zeros(0, 2, device="cuda"), None, None, dw, db, None)
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("T,d,kind", [(5000, 768, "bf16"), (3000, 410, "f32"), (2000, 2048, "bf16"), (700, 5001, "bf16"), (20000, 64, "bf16"), (400, 16392, "f32")])
def test_many_rows(b, T, d, kind):
    """The column sums over many rows, against 64 bits on the device; the same bits every time."""
    g = torch.Generator(device="cuda").manual_seed(T)
    S, dY = (torch.randn(T, d, generator=g, device="cuda").to(TYPES[kind]) for _ in range(2))
    if kind == "bf16" and d % 8:
        pad = torch.zeros(2, T, (d + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda")
        pad[0, :, :d], pad[1, :, :d] = S, dY
        S, dY = pad[0, :, :d], pad[1, :, :d]
    w = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    Y, dX, stats = matrix(T, d, kind)[0], matrix(T, d, kind)[0], torch.empty(T, 2, device="cuda")
    b.layer_norm_fwd(S, w, None, EPS, Y, stats)
    outs = []
    for _ in range(2):
        dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        b.layer_norm_bwd(dY, S, stats, w, dX, dw, db, workspace(b, T, d, kind))
        outs.append((dw, db, dX.clone()))
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    s64, dy64 = S.double(), dY.double()
    x = (s64 - s64.mean(1, keepdim=True)) * (s64.var(1, correction=0, keepdim=True) + EPS).rsqrt()
    # (T + 2) roundings of the magnitudes' sum, and the error of x: a few hundred steps
    for got, terms in ((dw, dy64 * x), (db, dy64)):
        assert torch.all((got.double() - terms.sum(0)).abs() <= (T + 300) * R.U * terms.abs().sum(0) + 300 * R.U * dy64.abs().sum(0))


def test_two_graphs_on_one_workspace_while_eager_calls_live(b):
    T, d = 500, 410
    S, dY, w = torch.randn(T, d, device="cuda"), torch.randn(T, d, device="cuda"), torch.ones(d, device="cuda")
    Y, stats, ws = torch.empty_like(S), torch.empty(T, 2, device="cuda"), workspace(b, T, d, "f32")
    outs = [[torch.empty_like(S), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")] for _ in range(3)]
    b.layer_norm_fwd(S, w, None, EPS, Y, stats)
    b.layer_norm_bwd(dY, S, stats, w, *outs[2], ws)
    graphs = []
    for out in outs[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.layer_norm_fwd(S, w, None, EPS, Y, stats)
            b.layer_norm_bwd(dY, S, stats, w, *out, ws)
        graphs.append(graph)
    for _ in range(2):
        for graph in graphs:
            graph.replay()
    for out in outs[:2]:
        assert all(torch.equal(x, y) for x, y in zip(out, outs[2]))


def test_offsets_beyond_32_bits(b):
    T, d = 2 ** 21 + 3, 2048
    X = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    X[-5:, ::2] = 2
    stats, dw = torch.empty(T, 2, device="cuda"), torch.empty(d, device="cuda")
    Y = torch.empty_like(X)
    b.layer_norm_fwd(X, None, None, 0.25, Y, stats)
    assert torch.all(stats[-5:, 0] == 1) and not stats[:-5, 0].any()
    x = float(torch.tensor(1.25 ** -0.5))
    assert torch.allclose(Y[-5:, ::2].float(), torch.tensor(x, device="cuda"), rtol=2 ** -8) and not Y[:-5].any()
    b.layer_norm_bwd(X, X, stats, None, Y, dw, None, workspace(b, T, d, "bf16"))
    assert torch.allclose(dw[::2], torch.tensor(5 * 2 * x, device="cuda"), rtol=1e-5) and not dw[1::2].any()
    assert not Y[:-5].any() and Y[-5:].any()
