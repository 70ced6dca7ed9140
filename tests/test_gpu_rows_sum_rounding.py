"""The sum in front of a norm, and of a dropout with a residual: what is kept is scaled and rounded to fp32, the sum is rounded to fp32 and then to the rows' type, as by a
dropout and a sum one after the other in fp32."""
import numpy as np
import pytest
import torch

from oracle import rows as R
from tests.test_gpu_embedding_rows import TYPES, matrix

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("p", [0.1, 0.15])
@pytest.mark.parametrize("T,d", [(4000, 40), (3000, 130), (3000, 410), (1500, 768), (1000, 1030), (500, 2048), (200, 5001), (120, 9000), (60, 16384), (50, 20000)])
def test_bits_of_the_sum(b, kind, p, T, d):
    g = torch.Generator(device="cuda").manual_seed(T)
    X, Res, S, Y, Z = (matrix(T, d, kind)[0] for _ in range(5))
    X.copy_(3 * torch.randn(T, d, generator=g, device="cuda"))
    Res.copy_(torch.randn(T, d, generator=g, device="cuda"))
    keep, s = R.dropout_mask(T, d, p, 7, 9)
    kept = torch.where(torch.from_numpy(keep).cuda(), X.float() * torch.tensor(np.float32(s), device="cuda"), 0.0)
    want = (kept + Res.float()).to(TYPES[kind])
    b.layer_norm_fwd(X, None, None, 1e-5, Y, R=Res, S=S, p=p, seed=7, offset=9)
    assert torch.equal(S, want), int((S != want).sum())
    b.dropout_fwd(X, Z, p, 7, 9, R=Res)
    assert torch.equal(Z, want)
