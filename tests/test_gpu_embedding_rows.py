"""Embedding lookup and the table's gradient against the oracle: one token to many, every word the same, no word at all, odd widths, both
types, rows of any pitch."""
import numpy as np
import pytest
import torch

from oracle import rows as R

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def matrix(rows, cols, kind, fill=float("nan"), ld=None, shift=0):
    """[rows, cols] in a larger poisoned buffer: leading dimension ld, first element `shift` elements behind an aligned address."""
    ld = ld or (cols + 7) // 8 * 8
    buf = torch.full((rows * ld + shift + 16,), fill, dtype=TYPES[kind], device="cuda")
    return torch.as_strided(buf, (rows, cols), (ld, 1), shift), buf


def filled(a, kind, **kw):
    m, _ = matrix(*a.shape, kind, **kw)
    m.copy_(torch.from_numpy(a.astype(np.float32)))
    return m


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def words(g, how, T, V):
    if how == "same":
        ids = np.full(T, V // 2)
    elif how == "zipf":
        ids = np.minimum(np.exp(g.random(T) * np.log(V + 1)) - 1, V - 1).astype(int)
    elif how == "none":
        ids = g.choice([-1, V, 2 ** 31 - 1, -2 ** 31], T)
    elif how == "runs":                                                  # runs that end on, before and behind the borders of chunks of 8 and more
        ids = np.repeat(np.arange(T), g.choice([1, 7, 8, 9, 16, 24, 33, 129], T))[:T] % V
    else:
        ids = g.integers(0, V, T)
    if how in ("zipf", "any"):
        ids[g.random(T) < 0.05] = -1
    return torch.from_numpy(ids.astype(np.int32)).cuda()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 32000, 1024), (3, 10, 7), (33, 50, 410), (257, 1000, 64), (1000, 300, 129), (64, 9, 5001)])
def test_lookup(b, kind, T, V, d):
    g = np.random.default_rng(T + d)
    E, ids = filled(g.standard_normal((V, d)), kind), words(g, "any", T, V)
    Y, buf = matrix(T, d, kind)
    b.embedding_fwd(ids, E, 1.7, Y)
    want = R.embedding_fwd(ids.cpu().numpy(), host(E), float(np.float32(1.7)))
    assert np.all(np.abs(host(Y) - want) <= R.HALF_STEP[kind] * np.abs(want) * (1 + 2 ** -7) + R.U * np.abs(want))
    Y.fill_(float("nan"))
    assert torch.isnan(buf).all()                                        # nothing beside the rows was written


def check_gradient(b, kind, out, T, V, d, how, accumulate=False, scale=0.75, seed=0, **place):
    g = np.random.default_rng(seed + T + d)
    dY, ids = filled(g.standard_normal((T, d)), kind, **place), words(g, how, T, V)
    dE, buf = matrix(V, d, out, **place)
    old = np.zeros((V, d))
    if accumulate:
        dE.copy_(torch.from_numpy(g.standard_normal((V, d)).astype(np.float32)))
        old = host(dE)
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, T, d, 0, V, b.BF16 if kind == "bf16" else b.F32))
    ws.fill_(0xFF)
    b.embedding_bwd(dY, ids, scale, dE, ws, accumulate)
    want, size, count = R.embedding_bwd(host(dY), ids.cpu().numpy(), V, scale)
    want = want + old
    # a sum of n terms passes through at most n + 8 additions (its parts are joined by eight warps); the scale, the old value and the type round once each
    bound = (count[:, None] + 8 + 2) * R.U * (size + np.abs(old)) + R.HALF_STEP[out] * np.abs(want) * (1 + 2 ** -7)
    got = host(dE)
    assert np.all(np.abs(got - want) <= bound), np.abs(got - want).max()
    assert np.all(got[count == 0] == old[count == 0])
    first = dE.clone()
    if not accumulate:
        b.embedding_bwd(dY, ids, scale, dE, ws)
        assert torch.equal(dE, first)                                    # the order of the additions is fixed
    dE.fill_(float("nan"))
    assert torch.isnan(buf).all()


@pytest.mark.parametrize("kind,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("T,V,d,how", [
    (1, 1, 1, "any"), (1, 700, 40, "any"), (2, 3, 8, "same"), (7, 5, 9, "any"), (8, 100, 64, "same"), (9, 100, 72, "runs"), (31, 40, 128, "zipf"), (300, 511, 136, "runs"),
    (300, 512, 136, "runs"), (700, 40, 410, "zipf"), (1000, 300000, 24, "any"), (1500, 7, 257, "none"), (2500, 205, 264, "same"), (5000, 3, 16, "any"), (5000, 70000, 520, "zipf"),
    (20000, 100, 40, "runs"), (20000, 2, 8, "same")])
def test_gradient(b, kind, out, T, V, d, how):
    check_gradient(b, kind, out, T, V, d, how)


@pytest.mark.parametrize("kind,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("T,V,d,how", [(1, 5, 3, "any"), (600, 50, 100, "zipf"), (4000, 9, 264, "same"), (500, 9, 32, "none")])
def test_gradient_is_added(b, kind, out, T, V, d, how):
    check_gradient(b, kind, out, T, V, d, how, accumulate=True)


@pytest.mark.parametrize("T,V,d,ld,shift", [(40, 30, 13, 13, 0), (40, 30, 64, 67, 1), (200, 50, 257, 300, 3), (200, 50, 16, 20, 4)])
def test_fp32_rows_of_any_pitch(b, T, V, d, ld, shift):
    check_gradient(b, "f32", "f32", T, V, d, "zipf", ld=ld, shift=shift)
    check_gradient(b, "f32", "f32", T, V, d, "zipf", ld=ld, shift=shift, accumulate=True)
    g = np.random.default_rng(1)
    E, ids = filled(g.standard_normal((V, d)), "f32", ld=ld, shift=shift), words(g, "any", T, V)
    Y, _ = matrix(T, d, "f32", ld=ld, shift=shift)
    b.embedding_fwd(ids, E, 1.0, Y)
    assert torch.equal(Y, torch.where((ids >= 0)[:, None], E[ids.clamp_min(0).long()], 0.0))


def test_no_tokens_and_infinities(b):
    V, d = 40, 72
    dE, _ = matrix(V, d, "bf16")
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    b.embedding_bwd(torch.zeros(0, d, dtype=torch.bfloat16, device="cuda"), none, 1.0, dE, None)
    assert not dE.any()
    b.embedding_fwd(none, dE, 1.0, torch.zeros(0, d, dtype=torch.bfloat16, device="cuda"))
    # what arrives at padding, whatever it is, reaches no row; a NaN stays in its own word's row
    ids = torch.tensor([3, -1, 5, V, 3], dtype=torch.int32, device="cuda")
    dY = torch.ones(5, d, dtype=torch.bfloat16, device="cuda")
    dY[1], dY[3], dY[2, 7] = float("inf"), float("nan"), float("nan")
    b.embedding_bwd(dY, ids, 1.0, dE, b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, 5, d, 0, V, b.BF16)))
    assert torch.isnan(dE[5, 7]) and int(torch.isnan(dE).sum()) == 1 and torch.all(dE[3] == 2) and float(dE[5, 0]) == 1


def test_replayed_with_other_words(b):
    """A captured step reads its ids when it runs; two graphs on one workspace, one after the other."""
    g = torch.Generator(device="cuda").manual_seed(2)
    T, V, d = 3000, 500, 136
    ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    dY = torch.randn(T, d, generator=g, device="cuda")
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, T, d, 0, V, b.F32))
    outs, graphs = [torch.zeros(V, d, device="cuda") for _ in range(2)], []
    b.embedding_bwd(dY, ids, 1.0, outs[0], ws)
    for out, scale in zip(outs, (1.0, 2.0)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.embedding_bwd(dY, ids, scale, out, ws)
        graphs.append(graph)
    for _ in range(3):
        ids.copy_(torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32))
        for graph in graphs:
            graph.replay()
        want = torch.zeros(V, d, device="cuda", dtype=torch.float64).index_add_(0, ids.long(), dY.double())
        # ten or so terms to a word: far below 64 roundings of sums below 64
        assert torch.allclose(outs[0].double(), want, rtol=0, atol=64 * 64 * 2.0 ** -24) and torch.equal(outs[1], 2 * outs[0])


def test_offsets_beyond_32_bits(b):
    """A table of 4.3e9 elements: its last rows are found, cleared and written."""
    V, d = 2 ** 21 + 5, 2048
    dE = torch.full((V, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([V - 1, 0, V - 1, V], dtype=torch.int32, device="cuda")
    dY = torch.ones(4, d, dtype=torch.bfloat16, device="cuda")
    b.embedding_bwd(dY, ids, 1.5, dE, b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, 4, d, 0, V, b.BF16)))
    assert torch.all(dE[V - 1] == 3) and torch.all(dE[0] == 1.5) and not dE[1:V - 1].any()
    Y = torch.empty(4, d, dtype=torch.bfloat16, device="cuda")
    b.embedding_fwd(ids, dE, 2.0, Y)
    assert torch.all(Y[0] == 6) and torch.all(Y[1] == 3) and not Y[3].any()
