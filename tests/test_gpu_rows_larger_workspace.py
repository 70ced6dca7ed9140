"""A workspace that was sized for a batch serves every smaller one: the last batch of an epoch, ragged batches."""
import pytest
import torch

from oracle import rows as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


@pytest.mark.parametrize("most,d,batches", [(149, 5001, (148, 149, 111, 1)), (2369, 2048, (2368, 2369, 1185, 1184, 593, 592, 7)), (4737, 40, (4736, 2368, 300))])
def test_norm(b, most, d, batches):
    g = torch.Generator(device="cuda").manual_seed(d)
    S, dY = (torch.randn(most, (d + 7) // 8 * 8, generator=g, device="cuda").bfloat16()[:, :d] for _ in range(2))
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_LAYER_NORM_BWD, most, d, 0, 0, b.BF16))
    stats, Y = torch.empty(most, 2, device="cuda"), torch.empty_like(S.as_strided((most, (d + 7) // 8 * 8), ((d + 7) // 8 * 8, 1)))[:, :d]
    b.layer_norm_fwd(S, None, None, 1e-5, Y, stats)
    for T in batches:
        outs = []
        for w in (ws.fill_(0xFF), b.alloc_workspace(b.workspace_bytes(b.OP_LAYER_NORM_BWD, T, d, 0, 0, b.BF16))):
            dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
            b.layer_norm_bwd(dY[:T], S[:T], stats[:T], None, None, dw, db, w)
            outs.append((dw, db))
        assert all(torch.equal(x, y) for x, y in zip(*outs))
        want = dY[:T].double().sum(0)
        assert torch.all((outs[0][1] - want).abs() <= (T + 1) * R.U * dY[:T].double().abs().sum(0))


@pytest.mark.parametrize("most,d,batches", [(4737, 2048, (4736, 4737, 3000, 100)), (20000, 768, (19000, 17964, 14973, 11982, 11000, 1))])
def test_table_gradient(b, most, d, batches):
    g = torch.Generator(device="cuda").manual_seed(d)
    V = 300
    dY, ids = torch.randn(most, d, generator=g, device="cuda"), torch.randint(0, V, (most,), generator=g, device="cuda", dtype=torch.int32)
    ws = b.alloc_workspace(b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, most, d, 0, V, b.F32))
    for T in batches:
        dE = torch.empty(V, d, device="cuda")
        b.embedding_bwd(dY[:T], ids[:T], 1.0, dE, ws.fill_(0xFF))
        want, size = (torch.zeros(V, d, device="cuda", dtype=torch.float64).index_add_(0, ids[:T].long(), t.double()) for t in (dY[:T], dY[:T].abs()))
        count = torch.bincount(ids[:T].long(), minlength=V)[:, None]
        assert torch.all((dE - want).abs() <= (count + 10) * R.U * size)


def test_nothing_behind_the_workspace_is_written(b):
    """The sizes at which chunks, or rows of a block, come out shortest for their number."""
    for T, d in ((151552, 40), (151553, 40), (151555, 40), (151556, 40), (75779, 100), (37891, 256), (4736, 2048), (4737, 2048), (2368 * 4 + 1, 1024), (16, 5000), (17, 5000)):
        V = 50
        dY, ids = torch.ones(T, (d + 7) // 8 * 8, dtype=torch.bfloat16, device="cuda")[:, :d], torch.arange(T, device="cuda", dtype=torch.int32) % V
        need = b.workspace_bytes(b.OP_EMBEDDING_SORTED_BWD, T, d, 0, V, b.BF16)
        ws, dE = b.alloc_workspace(need + (1 << 20)).fill_(0xA5), torch.empty(V, d, device="cuda")
        b.embedding_bwd(dY, ids, 1.0, dE, ws[:need])
        assert torch.all(ws[need:] == 0xA5) and torch.equal(dE, torch.bincount(ids.long(), minlength=V)[:, None].float().expand(V, d))
        need = b.workspace_bytes(b.OP_LAYER_NORM_BWD, T, d, 0, 0, b.BF16)
        ws, db = b.alloc_workspace(need + (1 << 20)).fill_(0xA5), torch.empty(d, device="cuda")
        b.layer_norm_bwd(dY, dY, torch.zeros(T, 2, device="cuda"), None, None, None, db, ws[:need])
        assert torch.all(ws[need:] == 0xA5) and torch.all(db == T)
