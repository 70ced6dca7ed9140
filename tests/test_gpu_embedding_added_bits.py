"""A gradient that is added to an fp32 table: the same bits wherever the table's rows start and end."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def workspace(b, T, d, V, kind):
    return b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, T, d, 0, V, b.BF16 if kind == "bf16" else b.F32))


# looked through; sorted; one word for all tokens (added up by whole blocks)
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,d", [(200, 60, 72), (5000, 400, 136), (5000, 1, 264), (5000, 1, 16)])
def test_the_same_bits_wherever_rows_start(b, kind, T, V, d):
    g = torch.Generator(device="cuda").manual_seed(T + d)
    dY, ids = torch.randn(T, d, generator=g, device="cuda").to(TYPES[kind]), torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    old, scale = torch.randn(V, d, generator=g, device="cuda"), 0.7
    sums = torch.empty(V, d, device="cuda")
    b.embedding_bwd(dY, ids, 1.0, sums, workspace(b, T, d, V, kind))
    want = sums * scale + old                                # the product is rounded, then the sum
    for shift in range(4):
        dE = torch.zeros(V * d + 8, device="cuda")[shift:shift + V * d].view(V, d)
        dE.copy_(old)
        b.embedding_bwd(dY, ids, scale, dE, workspace(b, T, d, V, kind), accumulate=True)
        assert torch.equal(dE, want), (shift, (dE - want).abs().max())


@pytest.mark.parametrize("T,V,d", [(200, 60, 72), (200, 60, 71), (5000, 400, 136), (5000, 400, 137), (5000, 1, 264)])
def test_small_values(b, T, V, d):
    """What is below the smallest normal value may count as zero where it is added, and all else is exact: values are multiples of 2^-129, of 2^21 of them at most."""
    g = torch.Generator(device="cuda").manual_seed(T)
    step, normal = 2.0 ** -129, 2.0 ** -126
    whole = torch.randint(-50, 50, (T, d), generator=g, device="cuda")
    ids, old = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32), torch.randint(-999, 999, (V, d), generator=g, device="cuda")
    dE = (old.double() * step).float()
    b.embedding_bwd((whole.double() * step).float(), ids, 1.0, dE, workspace(b, T, d, V, "f32"), accumulate=True)
    added = torch.zeros_like(old).index_add_(0, ids.long(), whole)
    zero = lambda m: torch.where(m.abs() * step < normal, 0, m)  # noqa: E731
    got = dE.double() / step
    assert torch.all((got == old + added) | (got == zero(old) + zero(added)) | (got == zero(zero(old) + zero(added))) | (got == zero(old + added)))
