"""Rows of equal values: their mean is the value itself, whatever the width, so the norm is the bias, and NaN where nothing is added to the variance."""
import numpy as np
import pytest
import torch

from tests.test_gpu_embedding_rows import TYPES, filled, matrix

pytestmark = pytest.mark.gpu
# 1 and 100 have few bits; 0.1, 100.1 and -3.3e5 / 7 fill fp32's, so that sums of them round
VALUES = [1.0, 100.0, 0.1, 100.1, -3.3e5 / 7, 2.5e-30]


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


# widths whose reciprocal in fp32 times the width is not one (41, 47, 328, 376, 440, 1000), and every way of holding a row
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1, 3, 7, 41, 47, 130, 328, 376, 440, 509, 1000, 1023, 2047, 2600, 4093, 5001, 8191, 11003, 12289, 16381, 16384, 16393, 40001])
def test_equal_values(b, kind, d):
    g = torch.Generator(device="cuda").manual_seed(d)
    T = len(VALUES)
    column = torch.tensor(VALUES, device="cuda").to(TYPES[kind])
    X, Y, S = matrix(T, d, kind)[0], matrix(T, d, kind)[0], matrix(T, d, kind)[0]
    X.copy_(column[:, None].expand(T, d))
    none = filled(np.zeros((T, d)), kind)
    weight, bias = torch.randn(d, generator=g, device="cuda"), torch.randn(d, generator=g, device="cuda")
    for form in (dict(), dict(R=none, S=S)):
        stats = torch.full((T, 2), float("nan"), device="cuda")
        b.layer_norm_fwd(X, weight, bias, 1e-5, Y, stats, **form)
        assert torch.equal(stats[:, 0], column.float())
        assert torch.equal(Y, bias.to(TYPES[kind]).expand(T, d))
        b.layer_norm_fwd(X, weight, bias, 0.0, Y, stats, **form)
        assert torch.equal(stats[:, 0], column.float()) and torch.isinf(stats[:, 1]).all()
        assert torch.isnan(Y).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("d", [2 ** 20 + 3, 2 ** 23])
def test_equal_values_of_the_widest_rows(b, kind, d):
    X = torch.full((2, (d + 7) // 8 * 8), 100.1, device="cuda").to(TYPES[kind])[:, :d]
    Y, stats = torch.empty_like(X.as_strided((2, (d + 7) // 8 * 8), ((d + 7) // 8 * 8, 1)))[:, :d], torch.empty(2, 2, device="cuda")
    b.layer_norm_fwd(X, None, None, 1e-5, Y, stats)
    assert torch.all(stats[:, 0] == X[0, 0].float()) and not Y.any()


@pytest.mark.parametrize("d", [40, 130, 410, 1000, 4093, 11003, 16384])
def test_values_that_are_nearly_equal(b, d):
    """A few steps of fp32 around a value: differences are exact, and what is left of the mean's error is that of adding up differences of at most 9 + 45 steps
    (45: additions that a sum of the values passes through), with as many roundings again, and that of dividing."""
    g = torch.Generator(device="cuda").manual_seed(d)
    T, step = 12, 2.0 ** -17                                 # of fp32 between 64 and 128
    X = (100.1 + torch.randint(-9, 10, (T, d), generator=g, device="cuda") * step).float()
    Y, stats = torch.empty_like(X), torch.empty(T, 2, device="cuda")
    b.layer_norm_fwd(X, None, None, 0.0, Y, stats)
    x = X.double()
    mean, var = x.mean(1, keepdim=True), x.var(1, correction=0, keepdim=True)
    want = (x - mean) * var.rsqrt()
    off = 48 * 2.0 ** -24 * 54 * step * var.rsqrt()
    # the variance's relative error: 45 additions and three roundings; the root halves it and is off by two steps; three products
    assert torch.all((Y - want).abs() <= off + want.abs() * ((48 / 2 + 2 + 3) * 2.0 ** -24 + off))
    assert torch.all((stats[:, :1] - mean).abs() <= step / 2 * (1 + 2.0 ** -10))


@pytest.mark.parametrize("d", [3, 20, 60, 120, 300, 410, 2047, 16000])
def test_rows_beside_equal_ones(b, d):
    """A row's result is the same whatever rows are worked on together with it."""
    g = torch.Generator(device="cuda").manual_seed(d)
    T = 50
    X = torch.randn(T, d, generator=g, device="cuda")
    alone, beside, stats, other = torch.empty_like(X), torch.empty_like(X), torch.empty(T, 2, device="cuda"), torch.empty(T, 2, device="cuda")
    b.layer_norm_fwd(X, None, None, 1e-5, alone, stats)
    mixed = X.clone()
    mixed[::3] = 100.1
    b.layer_norm_fwd(mixed, None, None, 1e-5, beside, other)
    rest = torch.arange(T, device="cuda") % 3 != 0
    assert torch.equal(beside[rest], alone[rest]) and torch.equal(other[rest], stats[rest]) and not beside[::3].any()
