"""What the operators on token rows need of a workspace does not fall as batches grow (no GPU needed)."""
import pytest

from paper_1910_04732_b200 import binding as b
from paper_1910_04732_b200 import build


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return b.load_library()


@pytest.mark.parametrize("dt", [b.BF16, b.F32])
@pytest.mark.parametrize("op", [b.OP_EMBEDDING_SORTED_BWD, b.OP_LAYER_NORM_BWD])
@pytest.mark.parametrize("d", [1, 16, 40, 64, 65, 129, 257, 410, 768, 1024, 2048, 5001, 16384, 16392, 100000])
def test_a_larger_batch_needs_no_less(op, dt, d):
    most = 0
    for T in [*range(0, 6000), *range(6000, 200000, 997), *(4096 * 256 * k + j for k in (1, 2, 5, 40) for j in (-1, 0, 1)), 2 ** 31 - 1]:
        need = b.workspace_bytes(op, T, d, 0, 1000, dt)
        assert need >= most, T
        most = need
