"""The table's gradient by sorted tokens with values that are not finite, and words with very many tokens."""
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


def gradient(b, dY, ids, V, accumulate=False):
    T, d = dY.shape
    dE = torch.zeros(V, d, device="cuda")
    b.embedding_bwd(dY, ids, 1.0, dE, b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, T, d, 0, V, b.BF16 if dY.dtype == torch.bfloat16 else b.F32)), accumulate)
    return dE


# looked through; sorted by one cluster; by many blocks; runs that cross the borders of chunks
@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,V,d", [(300, 40, 72), (3000, 40, 72), (3000, 2900, 264), (20000, 300, 24), (20000, 3, 136)])
def test_padding_reaches_no_row_and_a_nan_stays_in_its_words(b, kind, accumulate, T, V, d):
    g = torch.Generator(device="cuda").manual_seed(T + d)
    ids = torch.randint(-1, V + 1, (T,), generator=g, device="cuda", dtype=torch.int32)
    padding = (ids < 0) | (ids >= V)
    dY = torch.ones(T, d, device="cuda", dtype=TYPES[kind])
    dY[padding] = float("nan")
    dY[padding.nonzero()[::2, 0]] = float("inf")
    at = int((~padding).nonzero()[T // 3, 0])
    word = int(ids[at])
    dY[at, 7] = float("nan")
    count = torch.bincount(ids[~padding].long(), minlength=V)[:, None].float().expand(V, d).clone()
    count[word, 7] = float("nan")
    assert torch.equal(torch.nan_to_num(gradient(b, dY, ids, V, accumulate), nan=-1.0), torch.nan_to_num(count, nan=-1.0))


@pytest.mark.parametrize("T,d", [(2 ** 20 + 5000, 16), (135000, 16), (2 ** 22 + 1, 8)])
def test_one_word_for_all_tokens_of_a_long_batch(b, T, d):
    """Thousands of parts of one run; sums of ones are exact below 2^24."""
    ids = torch.full((T,), 1, device="cuda", dtype=torch.int32)
    dE = gradient(b, torch.ones(T, d, device="cuda", dtype=torch.bfloat16), ids, 3)
    assert torch.all(dE[1] == T) and not dE[0].any() and not dE[2].any()
