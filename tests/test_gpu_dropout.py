"""Dropout against the oracle's mask, bit for bit, and its values, in both directions."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from tests.test_gpu_embedding_rows import filled, host, matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def check(b, kind, T, d, p, residual, seed=5, offset=9, **place):
    g = np.random.default_rng(T + d)
    X, Res = filled(g.standard_normal((T, d)), kind, **place), filled(g.standard_normal((T, d)), kind, **place) if residual else None
    Y, buf = matrix(T, d, kind, **place)
    b.dropout_fwd(X, Y, p, seed, offset, R=Res)
    keep, s = R.dropout_mask(T, d, p, seed, offset)
    x, r = host(X), host(Res) if residual else 0.0
    want = np.where(keep, x * s, 0.0) + r
    got = host(Y)
    # the factor, the product and the sum round to fp32, the result to its type
    bound = R.U * (2 * np.abs(x) * s + np.abs(want)) + R.HALF_STEP[kind] * np.abs(want) * (1 + 2 ** -7)
    assert np.all(np.abs(got - want) <= bound)
    assert np.array_equal(got == r, ~keep | (x == 0) | (got == r)) and (residual or np.array_equal(got != 0, keep & (x != 0)))
    dX, _ = matrix(T, d, kind, **place)
    b.dropout_bwd(X, dX, p, seed, offset)
    back = np.where(keep, x * s, 0.0)
    assert np.all(np.abs(host(dX) - back) <= R.U * 3 * np.abs(back) + R.HALF_STEP[kind] * np.abs(back) * (1 + 2 ** -7))
    Y.fill_(float("nan"))
    assert torch.isnan(buf).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,d,p", [(1, 1, 0.5), (1, 8, 0.1), (5, 7, 0.9), (3, 4096, 0.2), (33, 410, 0.1), (257, 65, 0.5), (1, 20000, 0.3), (2000, 8, 0.25), (700, 1001, 0.1)])
def test_both_directions(b, kind, residual, T, d, p):
    check(b, kind, T, d, p, residual)


@pytest.mark.parametrize("seed,offset", [(0, 0), (2 ** 63 + 12345, 2 ** 32 - 3), (2 ** 40, 2 ** 64 - 5)])
def test_keys_and_counters_of_64_bits(b, seed, offset):
    check(b, "f32", 6, 20, 0.5, False, seed, offset)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 2.0 ** -16, 0.999995])
def test_probabilities_at_the_ends(b, p):
    check(b, "f32", 40, 1000, p, True)


@pytest.mark.parametrize("d,ld,shift", [(13, 13, 0), (64, 67, 1), (20, 24, 4), (9, 12, 2)])
def test_fp32_rows_of_any_pitch(b, d, ld, shift):
    check(b, "f32", 50, d, 0.3, True, ld=ld, shift=shift)


def test_in_place(b):
    X = torch.randn(100, 328, device="cuda").bfloat16()
    Res, Y = torch.randn(100, 328, device="cuda").bfloat16(), torch.empty(100, 328, device="cuda", dtype=torch.bfloat16)
    b.dropout_fwd(X, Y, 0.3, 1, 2, R=Res)
    for place in (X.clone(), Res.clone()):
        x, r = (place, Res) if torch.equal(place, X) else (X, place)
        b.dropout_fwd(x, place, 0.3, 1, 2, R=r)
        assert torch.equal(place, Y)


def test_what_is_dropped_counts_as_nothing(b):
    T, d = 4, 64
    keep, _ = R.dropout_mask(T, d, 0.5, 3, 0)
    keep = torch.from_numpy(keep).cuda()
    X = torch.where(keep, 1.0, torch.tensor([float("nan"), float("inf")], device="cuda").repeat(T, d // 2))
    Y = torch.empty_like(X)
    b.dropout_fwd(X, Y, 0.5, 3, 0)
    assert torch.equal(Y, torch.where(keep, 2.0, 0.0))
    X = torch.where(keep, float("nan"), 1.0)
    b.dropout_fwd(X, Y, 0.5, 3, 0)
    assert torch.equal(torch.isnan(Y), keep)


def test_a_captured_launch_draws_anew(b):
    X, Y, dX = torch.ones(64, 96, device="cuda"), torch.empty(64, 96, device="cuda"), torch.empty(64, 96, device="cuda")
    step = b.dropout_counters(64, 96)
    at = torch.zeros(1, dtype=torch.int64, device="cuda")
    b.dropout_fwd(X, Y, 0.5, 7, 100, offset_dev=at)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.dropout_fwd(X, Y, 0.5, 7, 100, offset_dev=at)
        b.dropout_bwd(X, dX, 0.5, 7, 100, offset_dev=at)
        at.add_(step)
    for i in range(3):
        graph.replay()
        keep, _ = R.dropout_mask(64, 96, 0.5, 7, 100 + i * step)
        assert np.array_equal(host(Y) != 0, keep) and torch.equal(Y, dX)


def test_another_stream(b):
    side = torch.cuda.Stream()
    X = torch.randn(3000, 2048, device="cuda")
    Y, Z = torch.empty_like(X), torch.empty_like(X)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.dropout_fwd(X, Y, 0.5, 1, 0)
        b.dropout_bwd(Y, Z, 0.5, 1, 0)
    side.synchronize()
    assert torch.equal(Z, 2 * Y)


def test_offsets_beyond_32_bits(b):
    T, d = 2 ** 20 + 3, 4096
    X = torch.ones(T, d, dtype=torch.bfloat16, device="cuda")
    b.dropout_fwd(X, X, 0.25, 4, 0)
    groups = d // 8
    keep, _ = R.dropout_mask(3, d, 0.25, 4, (T - 3) * groups)
    assert np.array_equal(host(X[-3:]) != 0, keep)
    assert abs(float((X[::1024] != 0).float().mean()) - 0.75) < 2e-3
