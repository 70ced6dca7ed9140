"""What embedding lookup, dropout and layer norm refuse on the host, before anything is launched (no GPU needed: every call here returns from
its argument checks)."""
import ctypes

import pytest
import torch

from paper_1910_04732_b200 import binding as b
from paper_1910_04732_b200 import build

P = 1 << 24            # an aligned address that nothing is read from
BAD, NO, WS = b.ERR_INVALID_ARG, b.ERR_UNSUPPORTED, b.ERR_WORKSPACE
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return b.load_library()


def lookup(lib, ids=P, T=4, E=2 * P, lde=64, V=10, scale=1.0, Y=3 * P, ldy=64, d=64, dt=b.BF16):
    return lib.flop_embedding_fwd(ids, T, E, lde, V, scale, Y, ldy, d, dt, None)


@pytest.mark.parametrize("change,code", [
    (dict(T=-1), BAD), (dict(V=-1), BAD), (dict(d=-1), BAD), (dict(dt=2), BAD), (dict(T=0), b.OK), (dict(d=0), b.OK), (dict(ids=None), BAD), (dict(E=None), BAD),
    (dict(Y=None), BAD), (dict(lde=56), BAD), (dict(ldy=56), BAD), (dict(E=2 * P + 8), NO), (dict(Y=3 * P + 2), NO), (dict(lde=65), NO), (dict(ldy=66), NO),
    (dict(Y=2 * P), BAD), (dict(Y=2 * P + 256), BAD), (dict(Y=P), BAD), (dict(T=1 << 31), NO), (dict(V=1 << 31), NO), (dict(d=(1 << 30) + 1, lde=1 << 31, ldy=1 << 31), NO)])
def test_lookup(lib, change, code):
    assert lookup(lib, **change) == code


def table_gradient(lib, dY=P, lddy=64, ids=2 * P, T=4, V=10, scale=1.0, dE=3 * P, ldde=64, accumulate=0, d=64, dt=b.BF16, wdt=b.F32, ws=4 * P, wb=1 << 20):
    return lib.flop_embedding_bwd(dY, lddy, ids, T, V, scale, dE, ldde, accumulate, d, dt, wdt, ws, wb, None)


@pytest.mark.parametrize("change,code", [
    (dict(T=-1), BAD), (dict(V=-1), BAD), (dict(d=-1), BAD), (dict(dt=-1), BAD), (dict(wdt=3), BAD), (dict(V=0), b.OK), (dict(d=0), b.OK), (dict(T=0, accumulate=1), b.OK),
    (dict(dY=None), BAD), (dict(ids=None), BAD), (dict(dE=None), BAD), (dict(lddy=56), BAD), (dict(ldde=63), BAD), (dict(dY=P + 8), NO), (dict(lddy=68), NO),
    (dict(wdt=b.BF16, ldde=68), NO), (dict(wdt=b.BF16, dE=3 * P + 4), NO), (dict(dE=P), BAD), (dict(dE=P + 128), BAD), (dict(dE=2 * P), BAD),
    (dict(ws=None), WS), (dict(ws=4 * P + 16), WS), (dict(wb=64), WS), (dict(T=1 << 31), NO), (dict(V=1 << 31), NO), (dict(d=(1 << 30) + 1, lddy=1 << 31, ldde=1 << 31), NO)])
def test_table_gradient(lib, change, code):
    assert table_gradient(lib, **change) == code


def drop(lib, form, X=P, ldx=64, R=None, ldr=64, p=0.1, Y=3 * P, ldy=64, T=4, d=64, dt=b.BF16):
    if form == "bwd":
        return lib.flop_dropout_bwd(X, ldx, p, 1, 2, None, Y, ldy, T, d, dt, None)
    return lib.flop_dropout_fwd(X, ldx, R, ldr, p, 1, 2, None, Y, ldy, T, d, dt, None)


@pytest.mark.parametrize("form", ["fwd", "bwd"])
@pytest.mark.parametrize("change,code", [
    (dict(T=-1), BAD), (dict(d=-1), BAD), (dict(dt=2), BAD), (dict(T=0), b.OK), (dict(d=0), b.OK), (dict(p=1.0), BAD), (dict(p=-0.1), BAD), (dict(p=NAN), BAD),
    (dict(X=None), BAD), (dict(Y=None), BAD), (dict(ldx=56), BAD), (dict(ldy=56), BAD), (dict(X=P + 8), NO), (dict(Y=3 * P + 2), NO), (dict(ldx=65), NO), (dict(ldy=68), NO),
    (dict(Y=P + 128), BAD), (dict(Y=P, ldy=72), BAD), (dict(T=1 << 31), NO), (dict(d=(1 << 30) + 1, ldx=1 << 31, ldy=1 << 31), NO)])
def test_dropout(lib, form, change, code):
    assert drop(lib, form, **change) == code


@pytest.mark.parametrize("change,code", [(dict(R=2 * P, ldr=56), BAD), (dict(R=2 * P, ldr=65), NO), (dict(R=2 * P + 8), NO), (dict(R=3 * P + 128), BAD)])
def test_dropout_residual(lib, change, code):
    assert drop(lib, "fwd", **change) == code


def norm_fwd(lib, X=P, ldx=64, R=None, ldr=64, p=0.0, w=5 * P, bias=6 * P, eps=1e-5, S=None, lds=64, Y=3 * P, ldy=64, stats=4 * P, T=4, d=64, dt=b.BF16):
    return lib.flop_layer_norm_fwd(X, ldx, R, ldr, p, 1, 2, None, w, bias, eps, S, lds, Y, ldy, stats, T, d, dt, None)


@pytest.mark.parametrize("change,code", [
    (dict(T=-1), BAD), (dict(d=-1), BAD), (dict(dt=2), BAD), (dict(T=0), b.OK), (dict(d=0), b.OK), (dict(p=1.0), BAD), (dict(eps=-1e-5), BAD), (dict(eps=NAN), BAD),
    (dict(eps=float("inf")), BAD), (dict(X=None), BAD), (dict(Y=None), BAD), (dict(ldx=56), BAD), (dict(ldy=56), BAD), (dict(R=2 * P, ldr=56), BAD), (dict(S=2 * P, lds=56), BAD),
    (dict(X=P + 8), NO), (dict(Y=3 * P + 2), NO), (dict(R=2 * P, ldr=65), NO), (dict(S=2 * P + 8), NO), (dict(stats=4 * P + 4), NO),
    (dict(Y=P + 128), BAD), (dict(S=P + 128), BAD), (dict(S=3 * P), BAD), (dict(S=2 * P, R=2 * P, lds=72), BAD), (dict(R=2 * P, Y=2 * P + 16), BAD),
    (dict(T=1 << 31), NO), (dict(d=(1 << 30) + 1, ldx=1 << 31, ldy=1 << 31), NO)])
def test_norm_forward(lib, change, code):
    assert norm_fwd(lib, **change) == code


def norm_bwd(lib, dY=P, lddy=64, S=2 * P, lds=64, stats=4 * P, w=5 * P, dS=None, ldds=64, p=0.0, dX=3 * P, lddx=64, dR=None, lddr=64, dw=6 * P, db=7 * P, accumulate=0, T=4, d=64,
             dt=b.BF16, ws=8 * P, wb=1 << 20):
    return lib.flop_layer_norm_bwd(dY, lddy, S, lds, stats, w, dS, ldds, p, 1, 2, None, dX, lddx, dR, lddr, dw, db, accumulate, T, d, dt, ws, wb, None)


@pytest.mark.parametrize("change,code", [
    (dict(T=-1), BAD), (dict(d=-1), BAD), (dict(dt=2), BAD), (dict(d=0), b.OK), (dict(T=0, accumulate=1), b.OK), (dict(T=0, dw=None, db=None), b.OK), (dict(p=1.5), BAD),
    (dict(dY=None), BAD), (dict(S=None), BAD), (dict(stats=None), BAD), (dict(lddy=56), BAD), (dict(lds=56), BAD), (dict(dS=9 * P, ldds=56), BAD), (dict(lddx=56), BAD),
    (dict(dR=9 * P, lddr=56), BAD), (dict(dY=P + 8), NO), (dict(S=2 * P + 8), NO), (dict(dX=3 * P + 8), NO), (dict(dS=9 * P, ldds=68), NO), (dict(dR=9 * P, lddr=68), NO),
    (dict(stats=4 * P + 4), NO), (dict(dX=P + 128), BAD), (dict(dX=2 * P + 128), BAD), (dict(dR=3 * P), BAD), (dict(dS=9 * P, dR=9 * P + 16), BAD),
    (dict(ws=None), WS), (dict(ws=8 * P + 8), WS), (dict(wb=128), WS), (dict(T=1 << 31), NO), (dict(d=(1 << 30) + 1), NO)])
def test_norm_backward(lib, change, code):
    assert norm_bwd(lib, **change) == code


@pytest.mark.parametrize("change", [dict(stats=3 * P), dict(stats=P + 64), dict(w=3 * P + 128), dict(bias=3 * P), dict(stats=5 * P), dict(S=2 * P, stats=2 * P + 8), dict(R=2 * P, stats=2 * P)])
def test_norm_forward_vectors_that_overlap(lib, change):
    assert norm_fwd(lib, **change) == BAD


@pytest.mark.parametrize("change", [dict(dw=7 * P), dict(db=6 * P + 8), dict(dw=3 * P), dict(db=P), dict(dw=2 * P), dict(dw=5 * P), dict(db=4 * P), dict(dX=4 * P), dict(dX=5 * P), dict(dR=6 * P)])
def test_norm_backward_vectors_that_overlap(lib, change):
    assert norm_bwd(lib, **change) == BAD


def test_workspaces(lib):
    assert b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, 1000, 64, 0, 50, b.BF16) >= 2 * 8 * 1000
    assert b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, 0, 64, 0, 50, b.BF16) == 0
    assert b.workspace_bytes(b.OP_LAYER_NORM_BWD, 1000, 64, 0, 0, b.F32) >= 2 * 4 * 64
    assert b.workspace_bytes(b.OP_LAYER_NORM_BWD, 0, 64, 0, 0, b.F32) == 0
    out = ctypes.c_size_t(0)
    assert lib.flop_workspace_bytes(7, 1, 1, 1, 1, 0, ctypes.byref(out)) == BAD


X, V = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8)
IDS = torch.zeros(4, dtype=torch.int32)


@pytest.mark.parametrize("call,exc", [
    (lambda: b.embedding_fwd(IDS, X, 1.0, X.clone()), TypeError),                       # tensors of the host
    (lambda: b.embedding_fwd(IDS.long(), X, 1.0, X.clone()), TypeError),
    (lambda: b.embedding_fwd(IDS[:3], X, 1.0, X.clone()), AssertionError),
    (lambda: b.embedding_fwd(IDS, X, 1.0, X.float()), AssertionError),
    (lambda: b.embedding_fwd(IDS, X[:, :4], 1.0, X.clone()), AssertionError),
    (lambda: b.embedding_bwd(X, IDS, 1.0, X.float()[:, :4], None), AssertionError),
    (lambda: b.embedding_bwd(X, IDS, 1.0, X.float(), torch.zeros(64)), TypeError),
    (lambda: b.embedding_bwd(X, IDS, 1.0, X.float(), torch.zeros(64, dtype=torch.uint8)), TypeError),
    (lambda: b.embedding_bwd(X, IDS, 1.0, X.half(), None), TypeError),
    (lambda: b.dropout_fwd(X, X.clone(), 0.1, 1, 0), TypeError),
    (lambda: b.dropout_fwd(X, None, 0.1, 1, 0), AttributeError),
    (lambda: b.dropout_fwd(X, X.float(), 0.1, 1, 0), AssertionError),
    (lambda: b.dropout_fwd(X, X[:3], 0.1, 1, 0), AssertionError),
    (lambda: b.dropout_fwd(X, X.clone(), 0.1, 1, 0, R=X[:, :4]), AssertionError),
    (lambda: b.dropout_fwd(X, X.clone(), "p", 1, 0), ValueError),
    (lambda: b.dropout_fwd(X, X.clone(), 0.1, 1, 0, offset_dev=torch.zeros(1)), TypeError),
    (lambda: b.dropout_bwd(X, None, 0.1, 1, 0), AttributeError),
    (lambda: b.dropout_bwd(X, X.clone(), 0.1, 1, 0), TypeError),
    (lambda: b.layer_norm_fwd(X, V, V, 1e-5, X.clone()), TypeError),
    (lambda: b.layer_norm_fwd(X, V.bfloat16(), V, 1e-5, X.clone()), TypeError),
    (lambda: b.layer_norm_fwd(X, V[:4], V, 1e-5, X.clone()), AssertionError),
    (lambda: b.layer_norm_fwd(X, V, V, 1e-5, X.clone(), torch.zeros(4)), AssertionError),
    (lambda: b.layer_norm_fwd(X, V, V, 1e-5, X.t()), AssertionError),
    (lambda: b.layer_norm_bwd(X, X, torch.zeros(4, 2), V, X.clone(), V, V, None), TypeError),
    (lambda: b.layer_norm_bwd(X, X[:2], torch.zeros(4, 2), V, X.clone(), V, V, None), AssertionError),
    (lambda: b.layer_norm_bwd(X, X, torch.zeros(4), V, X.clone(), V, V, None), AssertionError),
    (lambda: b.layer_norm_bwd(X, X, torch.zeros(4, 2), V, X.float(), V, V, None), AssertionError)])
def test_tensors_of_another_form_are_refused(lib, call, exc):
    with pytest.raises(exc):
        call()


def test_counters():
    assert b.dropout_counters(3, 8) == 3 and b.dropout_counters(3, 9) == 6 and b.dropout_counters(0, 9) == 0
