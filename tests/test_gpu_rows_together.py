"""The first block of a pruned model in training, as a program strings the calls together: words -> scaled rows -> dropout -> gated matrix ->
dropout, residual and norm -> (a loss) -> back through all of it to the table, in fp32 against the oracle's chain in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import flop_oracle as O
from oracle import rows as R
from tests._util import HC, host, rel_fro

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


T, V, d, r, EPS, SEED, P = 190, 70, 136, 96, 1e-5, 21, 0.1


class Block:
    """The block's tensors and its calls; `step` is what a program runs for every batch."""

    def __init__(self, b):
        g = np.random.default_rng(6)
        dev = lambda *s, by=1.0: torch.from_numpy((by * g.standard_normal(s)).astype(np.float32)).cuda()  # noqa: E731
        self.b, self.scale = b, float(np.float32(np.sqrt(d)))
        ids = np.minimum(np.exp(g.random(T) * np.log(V + 1)) - 1, V - 1).astype(np.int32)
        ids[-7:] = -1
        self.ids = torch.from_numpy(ids).cuda()
        self.E, self.Q, self.Pm, self.la = dev(V, d, by=d ** -0.5), dev(r, d, by=d ** -0.5), dev(d, r, by=r ** -0.5), dev(r, by=2.0)
        self.w, self.bias, self.dY = 1 + dev(d, by=0.1), dev(d, by=0.1), dev(T, d)
        new = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
        self.z, self.dz, self.mask = new(r), new(r), torch.zeros(r, dtype=torch.uint8, device="cuda")
        self.X, self.H, self.M, self.S, self.Y, self.stats = new(T, d), new(T, r), new(T, d), new(T, d), new(T, d), new(T, 2)
        self.dM, self.dS, self.dX, self.dQ, self.dP, self.dla = new(T, d), new(T, d), new(T, d), new(r, d), new(d, r), new(r)
        self.dw, self.dbias, self.dE = new(d), new(d), new(V, d)
        size = lambda op, *a: b.alloc_workspace(b.workspace_bytes(op, *a, b.F32))  # noqa: E731
        self.ws_norm, self.ws_rows, self.ws_gate = size(b.OP_LAYER_NORM_BWD, T, d, 0, 0), size(b.OP_EMBEDDING_SORTED_BWD, T, d, 0, V), size(b.OP_BWD, T, d, d, r)
        self.at = torch.zeros(1, dtype=torch.int64, device="cuda")       # how far the generator has come
        self.first, self.second = 0, b.dropout_counters(T, d)

    def step(self):
        b = self.b
        mask1, mask2 = (dict(p=P, seed=SEED, offset=o, offset_dev=self.at) for o in (self.first, self.second))
        b.gate_sample(self.la, HC, SEED, 0, self.z, self.mask, self.dz)
        b.embedding_fwd(self.ids, self.E, self.scale, self.X)
        b.dropout_fwd(self.X, self.X, **mask1)
        b.gated_lowrank_fwd(self.X, self.Q, self.Pm, self.z, self.M, self.H)
        b.layer_norm_fwd(self.M, self.w, self.bias, EPS, self.Y, self.stats, R=self.X, S=self.S, **mask2)
        b.layer_norm_bwd(self.dY, self.S, self.stats, self.w, self.dM, self.dw, self.dbias, self.ws_norm, dR=self.dS, **mask2)
        b.gated_lowrank_bwd(self.dM, self.X, self.Q, self.Pm, self.z, self.dz, self.H, self.dX, self.dP, self.dQ, self.dla, self.ws_gate)
        self.dX += self.dS
        b.dropout_bwd(self.dX, self.dX, **mask1)
        b.embedding_bwd(self.dX, self.ids, self.scale, self.dE, self.ws_rows)

    def results(self):
        return {n: getattr(self, n) for n in ("Y", "dE", "dQ", "dP", "dla", "dw", "dbias")}

    def exact(self, at):
        z, _, dz = O.gate_sample(self.la.cpu().numpy(), *HC, seed=SEED, offset=0)
        E, Q, Pm, w, bias, dY, ids = host(self.E), host(self.Q), host(self.Pm), host(self.w), host(self.bias), host(self.dY), self.ids.cpu().numpy()
        keep1, s = R.dropout_mask(T, d, P, SEED, self.first + at)
        keep2, _ = R.dropout_mask(T, d, P, SEED, self.second + at)
        X = R.embedding_fwd(ids, E, self.scale) * keep1 * s
        M = O.gated_lowrank_fwd(X, Q, Pm, z)[2]
        S = X + M * keep2 * s
        g, dw, dbias = R.layer_norm_bwd(dY, S, w, EPS)
        G = O.gated_lowrank_bwd(g * keep2 * s, X, Q, Pm, z, dz)
        dE, _, _ = R.embedding_bwd((G["dX"] + g) * keep1 * s, ids, V, self.scale)
        return dict(Y=R.layer_norm_fwd(S, w, bias, EPS)[0], dE=dE, dQ=G["dQ"], dP=G["dP"], dla=G["dlog_alpha"], dw=dw, dbias=dbias)


def check(block, at):
    want = block.exact(at)
    for name, got in block.results().items():
        # eight stages, each within 1e-5 of its sums (the bound the fp32 products are held to), rows of moderate condition
        assert rel_fro(host(got), want[name]) <= 1e-4, name


def test_a_step_and_its_replay_with_other_masks(b):
    block = Block(b)
    block.step()
    check(block, 0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.step()
        block.at.add_(2 * b.dropout_counters(T, d))
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        check(block, i * 2 * b.dropout_counters(T, d))
    assert b.device_status() == b.OK


def test_gradient_of_the_table_by_differences(b):
    """The oracle's chain itself: a step along a direction of the table moves the loss as its gradient says."""
    block = Block(b)
    block.step()
    g = np.random.default_rng(9)
    dE, direction, dY = host(block.dE), g.standard_normal((V, d)), host(block.dY)
    h = 1e-4
    losses = [(_exact_forward(block, host(block.E) + sign * h * direction) * dY).sum() for sign in (1, -1)]
    slope = (losses[0] - losses[1]) / (2 * h)
    along = (dE * direction).sum()
    # the difference quotient is off by h^2 times a third derivative; the gradient by 1e-4 of its norm times the direction's
    assert abs(slope - along) <= 1e-4 * np.linalg.norm(dE) * np.linalg.norm(direction) + 1e-5 * abs(slope)


def _exact_forward(block, E):
    z, _, _ = O.gate_sample(block.la.cpu().numpy(), *HC, seed=SEED, offset=0)
    keep1, s = R.dropout_mask(T, d, P, SEED, block.first)
    keep2, _ = R.dropout_mask(T, d, P, SEED, block.second)
    X = R.embedding_fwd(block.ids.cpu().numpy(), E, block.scale) * keep1 * s
    S = X + O.gated_lowrank_fwd(X, host(block.Q), host(block.Pm), z)[2] * keep2 * s
    return R.layer_norm_fwd(S, host(block.w), host(block.bias), EPS)[0]
