"""Sizes on both sides of every rule of the operators on token rows: widths at which a row is shared by other numbers of threads, cut into segments or
walked; batches that are looked through, sorted by one cluster or by many blocks; words with few and with many tokens; columns of the last piece."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from tests.test_gpu_dropout import check as check_dropout
from tests.test_gpu_embedding_rows import check_gradient, words
from tests.test_gpu_layer_norm import check as check_norm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


# units of 16 bytes at which the plan changes: 8, 16, 32, 64, 96, 128, 256, 384, 512, 768, 1024, 1536, 2048
@pytest.mark.parametrize("units", [8, 16, 32, 64, 96, 128, 256, 384, 512, 768, 1024, 1536, 2048])
@pytest.mark.parametrize("kind,per", [("bf16", 8), ("f32", 4)])
def test_norm_widths(b, kind, per, units):
    for d in (units * per - 1, units * per, units * per + 1):
        check_norm(b, kind, 5, d, "pre", 0.2)
    check_norm(b, kind, 3, units * per, "plain")


@pytest.mark.parametrize("width", [12288, 16384])
def test_norm_widths_of_wide_fp32_rows(b, width):
    for d in (width - 1, width, width + 1):
        check_norm(b, "f32", 3, d, "pre", 0.2)
    check_norm(b, "f32", 300, width - 6, "plain")


@pytest.mark.parametrize("T", [1, 2, 147, 148, 149, 1184, 2368, 2369, 4737])
@pytest.mark.parametrize("d", [24, 264, 1032])
def test_norm_batches(b, T, d):
    check_norm(b, "bf16", T, d, "post", 0.1)


@pytest.mark.parametrize("units", [8, 16, 32, 64, 96, 128, 256, 512, 4096])
@pytest.mark.parametrize("kind,per", [("bf16", 8), ("f32", 4)])
def test_dropout_widths(b, kind, per, units):
    for d in (units * per - 1, units * per, units * per + 1):
        check_dropout(b, kind, 7, d, 0.3, d % 2 == 0)
    check_dropout(b, kind, 1, units * per + 3, 0.3, True)


@pytest.mark.parametrize("T,V,d,how", [
    (1023, 60, 72, "zipf"), (1024, 60, 72, "same"), (1024, 90000, 300, "any"), (1000, 5, 264, "runs"), (1025, 60, 72, "zipf"), (1025, 300000, 16, "any"), (2048, 511, 130, "runs"),
    (2049, 512, 130, "zipf"), (16384, 300, 40, "zipf"), (16385, 300, 40, "zipf"), (16385, 300000, 24, "any"), (40000, 262143, 8, "any"), (40000, 262144, 8, "zipf"), (70000, 3, 16, "same"),
    (300000, 100, 8, "zipf"), (1500, 40, 4104, "zipf"), (2048, 7, 256, "same"), (2048, 900, 768, "zipf"), (2048, 900, 769, "zipf"), (2047, 90000, 24, "any"), (1254, 60, 2048, "runs"),
    (1255, 60, 2048, "runs")])
def test_embedding_batches(b, T, V, d, how):
    check_gradient(b, "bf16", "f32", T, V, d, how)
    check_gradient(b, "f32", "bf16", T, V, d, how)


@pytest.mark.parametrize("T,V,d,how", [(1025, 60, 72, "zipf"), (3000, 9, 264, "runs"), (20000, 50000, 24, "any"), (1000, 7, 40, "same")])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_embedding_adds(b, T, V, d, how, out):
    check_gradient(b, "bf16", out, T, V, d, how, accumulate=True)
    check_gradient(b, "f32", out, T, V, d, how, accumulate=True)


def test_gradient_of_rows_without_a_gap(b):
    """The table's gradient as one run of bytes that does not end on 16 of them."""
    for V, d, T, shift in ((77, 13, 2000, 0), (1001, 3, 1500, 1), (5, 1, 1100, 2), (33, 2, 40, 3), (300, 410, 1100, 3), (300, 411, 900, 1), (1, 3, 1200, 1), (2, 1, 1030, 3)):
        ids = words(np.random.default_rng(V), "any", T, V)
        dY = torch.randn(T, d, device="cuda")
        whole = torch.full((V * d + 9 + shift,), 7.0, device="cuda")
        buf = whole[shift:]
        dE = buf[:V * d].view(V, d)
        b.embedding_bwd(dY, ids, 1.0, dE, b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, T, d, 0, V, b.F32)))
        want, size, count = R.embedding_bwd(dY.double().cpu().numpy(), ids.cpu().numpy(), V, 1.0)
        assert np.all(np.abs(dE.double().cpu().numpy() - want) <= (count[:, None] + 10) * R.U * size)
        assert torch.all(buf[V * d:] == 7) and torch.all(whole[:shift] == 7)
