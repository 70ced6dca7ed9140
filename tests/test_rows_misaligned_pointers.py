"""Addresses that are no multiple of their values' size are refused on the host: a kernel would fault on them (no GPU needed: every call here returns from its
argument checks)."""
import pytest

from paper_1910_04732_b200 import binding as b
from tests.test_rows_refusals import P, lib, lookup, norm_bwd, norm_fwd, table_gradient  # noqa: F401

NO = b.ERR_UNSUPPORTED
F = dict(dt=b.F32)


@pytest.mark.parametrize("change", [dict(ids=P + 2), dict(ids=P + 1), dict(E=2 * P + 2, **F), dict(Y=3 * P + 1, **F)])
def test_lookup(lib, change):  # noqa: F811
    assert lookup(lib, **change) == NO


@pytest.mark.parametrize("change", [dict(ids=2 * P + 2), dict(dE=3 * P + 2), dict(dY=P + 3, **F), dict(dE=3 * P + 1, accumulate=1), dict(dE=3 * P + 2, T=0)])
def test_table_gradient(lib, change):  # noqa: F811
    assert table_gradient(lib, **change) == NO


def drop(lib, form, X=P, R=None, at=None, Y=3 * P, dt=b.F32):  # noqa: F811
    if form == "bwd":
        return lib.flop_dropout_bwd(X, 64, 0.1, 1, 2, at, Y, 64, 4, 64, dt, None)
    return lib.flop_dropout_fwd(X, 64, R, 64, 0.1, 1, 2, at, Y, 64, 4, 64, dt, None)


@pytest.mark.parametrize("form", ["fwd", "bwd"])
@pytest.mark.parametrize("change", [dict(X=P + 2), dict(Y=3 * P + 2), dict(at=5 * P + 4), dict(at=5 * P + 4, dt=b.BF16)])
def test_dropout(lib, form, change):  # noqa: F811
    assert drop(lib, form, **change) == NO


def test_dropout_residual(lib):  # noqa: F811
    assert drop(lib, "fwd", R=2 * P + 2) == NO


def norm_with_counter(lib, form, at):  # noqa: F811
    if form == "fwd":
        return lib.flop_layer_norm_fwd(P, 64, None, 64, 0.1, 1, 2, at, 5 * P, 6 * P, 1e-5, None, 64, 3 * P, 64, 4 * P, 4, 64, b.BF16, None)
    return lib.flop_layer_norm_bwd(P, 64, 2 * P, 64, 4 * P, 5 * P, None, 64, 0.1, 1, 2, at, 3 * P, 64, None, 64, 6 * P, 7 * P, 0, 4, 64, b.BF16, 8 * P, 1 << 20, None)


@pytest.mark.parametrize("form", ["fwd", "bwd"])
def test_norm_counter(lib, form):  # noqa: F811
    assert norm_with_counter(lib, form, 9 * P + 4) == NO


@pytest.mark.parametrize("change", [dict(X=P + 2, **F), dict(Y=3 * P + 2, **F), dict(R=2 * P + 2, **F), dict(S=2 * P + 2, **F), dict(w=5 * P + 2), dict(bias=6 * P + 1), dict(stats=4 * P + 2)])
def test_norm_forward(lib, change):  # noqa: F811
    assert norm_fwd(lib, **change) == NO


@pytest.mark.parametrize("change", [
    dict(dY=P + 2, **F), dict(S=2 * P + 2, **F), dict(dX=3 * P + 2, **F), dict(dS=9 * P + 2, **F), dict(dR=9 * P + 2, **F), dict(w=5 * P + 2), dict(dw=6 * P + 2), dict(db=7 * P + 3),
    dict(T=0, dw=6 * P + 2), dict(T=0, db=7 * P + 2)])
def test_norm_backward(lib, change):  # noqa: F811
    assert norm_bwd(lib, **change) == NO
