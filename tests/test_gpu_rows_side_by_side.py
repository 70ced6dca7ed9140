"""Matrices that lie side by side in the rows of one buffer do not overlap: each may be read and another written."""
import numpy as np
import pytest
import torch

from tests.test_gpu_embedding_rows import TYPES, filled, host, matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def columns(T, d, kind, count):
    """`count` matrices [T, d] next to one another in rows of one poisoned buffer; where rows need no alignment there is no gap between them."""
    each = (d + 7) // 8 * 8 if kind == "bf16" else d
    buf = torch.full((T, each * count), float("nan"), dtype=TYPES[kind], device="cuda")
    return buf, [buf[:, i * each:i * each + d] for i in range(count)]


def put(parts, *values):
    for part, value in zip(parts, values):
        part.copy_(value)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 8), (7, 64), (300, 70), (50, 410), (9, 2048), (5, 16392), (6, 16397)])
def test_norm_and_dropout(b, kind, T, d):
    g = np.random.default_rng(T + d)
    X, Res, dY, dS = (filled(g.standard_normal((T, d)), kind) for _ in range(4))
    w, mask = torch.ones(d, device="cuda"), dict(p=0.2, seed=1, offset=2)
    S, Y, dX, dR, Z, stats = *(matrix(T, d, kind)[0] for _ in range(5)), torch.empty(T, 2, device="cuda")
    dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_LAYER_NORM_BWD, T, d, 0, 0, b.BF16 if kind == "bf16" else b.F32))
    b.layer_norm_fwd(X, w, None, 1e-5, Y, stats, R=Res, S=S, **mask)
    b.layer_norm_bwd(dY, S, stats, w, dX, dw, db, ws, dS=dS, dR=dR, **mask)
    b.dropout_fwd(X, Z, R=Res, **mask)
    buf, at = columns(T, d, kind, 4)
    put(at, X, Res)
    b.layer_norm_fwd(at[0], w, None, 1e-5, at[3], stats, R=at[1], S=at[2], **mask)
    assert torch.equal(at[2], S) and torch.equal(at[3], Y) and torch.equal(at[0], X) and torch.equal(at[1], Res)
    at[2].fill_(float("nan"))
    b.dropout_fwd(at[0], at[2], R=at[1], **mask)
    assert torch.equal(at[2], Z) and torch.equal(at[3], Y)
    buf, at = columns(T, d, kind, 5)
    put(at, dY, S, dS)
    dw2, db2 = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    b.layer_norm_bwd(at[0], at[1], stats, w, at[3], dw2, db2, ws, dS=at[2], dR=at[4], **mask)
    assert torch.equal(at[3], dX) and torch.equal(at[4], dR) and torch.equal(dw, dw2) and torch.equal(db, db2)
    assert torch.equal(at[0], dY) and torch.equal(at[1], S) and torch.equal(at[2], dS)
    for part in at:
        part.fill_(float("nan"))
    assert torch.isnan(buf).all()                           # nothing between the matrices was written


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", [(40, 40, 72), (40, 300, 13), (3000, 200, 70)])
def test_lookup_and_table(b, kind, T, V, d):
    g = np.random.default_rng(T + d)
    rows = max(T, V)
    ids = torch.from_numpy(g.integers(-1, V, T).astype(np.int32)).cuda()
    E, dY = filled(g.standard_normal((V, d)), kind), filled(g.standard_normal((T, d)), kind)
    Y, dE = matrix(T, d, kind)[0], matrix(V, d, kind)[0]
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, T, d, 0, V, b.BF16 if kind == "bf16" else b.F32))
    b.embedding_fwd(ids, E, 2.0, Y)
    b.embedding_bwd(dY, ids, 2.0, dE, ws)
    buf, at = columns(rows, d, kind, 4)
    put([at[0][:V], at[1][:T]], E, dY)
    b.embedding_fwd(ids, at[0][:V], 2.0, at[2][:T])
    b.embedding_bwd(at[1][:T], ids, 2.0, at[3][:V], ws)
    assert torch.equal(at[2][:T], Y) and torch.equal(at[3][:V], dE) and torch.equal(at[0][:V], E) and torch.equal(at[1][:T], dY)
    for part, n in zip(at, (V, T, T, V)):
        part[:n].fill_(float("nan"))
    assert torch.isnan(buf).all()


def test_halves_that_overlap_are_refused(b):
    buf = torch.zeros(6, 40, device="cuda")
    w = torch.ones(16, device="cuda")
    for first, second in ((0, 15), (15, 0), (0, 1), (24, 9)):
        with pytest.raises(b.FlopError):
            b.dropout_fwd(buf[:, first:first + 16], buf[:, second:second + 16], 0.1, 1, 0)
    with pytest.raises(b.FlopError):                        # through the end of a row into the next one
        b.dropout_fwd(buf[:5, 30:].as_strided((5, 16), (40, 1), 30), buf[:5, :16].as_strided((5, 16), (40, 1), 40), 0.1, 1, 0)
    with pytest.raises(b.FlopError):
        b.layer_norm_fwd(buf[:, :16], w, None, 1e-5, buf[:, 8:24])
    assert not host(buf).any()
