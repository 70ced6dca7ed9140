"""One training step of a pruned output layer against a dense teacher, then its export in 8 bits, as a program strings the calls together:
gates -> gated forward (the logits) -> distillation loss and gradient -> gated backward -> penalty; compact factors -> 8-bit rows -> 8-bit
forward -> loss of the exported model."""
import numpy as np
import pytest
import torch

from oracle import flop_oracle as O
from oracle import operators as OO
from paper_1910_04732_b200 import inputs as I
from tests._util import HC, assert_close, host

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def test_step_and_export(b):
    g = np.random.default_rng(4)
    T, d, V, r, K, tau = 96, 264, 1000, 200, 16, 2.0
    dev = lambda a: b_copy(b, a)  # noqa: E731
    X, Q, P = dev(g.standard_normal((T, d))), dev(g.standard_normal((r, d)) * d ** -0.5), dev(g.standard_normal((V, r)) * 3 * r ** -0.5)
    dense = host(X) @ (host(P) @ host(Q)).T / tau                    # the teacher: every component open
    top = np.argsort(-dense, axis=1)[:, :K]
    t_logits = torch.from_numpy((np.take_along_axis(dense, top, 1) * tau).astype(np.float32)).cuda()
    t_idx = torch.from_numpy(top.astype(np.int32)).cuda()
    t_lse = torch.from_numpy(np.log(np.exp(dense).sum(1)).astype(np.float32)).cuda()
    weight = torch.full((T,), tau * tau / (T - 6), device="cuda")
    weight[-6:] = 0
    la = torch.from_numpy(I.log_alpha(("bimodal", 3.0, 0.5), r, 1).astype(np.float32)).cuda()
    z, dz, mask = torch.zeros(r, device="cuda"), torch.zeros(r, device="cuda"), torch.zeros(r, dtype=torch.uint8, device="cuda")
    b.gate_sample(la, HC, 5, 0, z, mask, dz)
    S, H = b.padded(T, V, BF), b.padded(T, r, BF)
    b.gated_lowrank_fwd(X, Q, P, z, S, H, None)
    logits = host(S)
    loss = torch.zeros(T, device="cuda")
    b.distill_topk_fwd_bwd(S, t_logits, t_idx, t_lse, weight, tau, loss, S)        # the gradient takes the logits' place
    dX, dP, dQ, dla = b.padded(T, d, BF), b.padded(V, r, BF), b.padded(r, d, BF), torch.zeros(r, device="cuda")
    b.gated_lowrank_bwd(S, X, Q, P, z, dz, H, dX, dP, dQ, dla, b.alloc_workspace(b.workspace_bytes(b.OP_BWD, T, d, V, r, b.BF16)))
    want_loss, grad, _ = OO.distill_topk(logits, t_logits.cpu().numpy(), t_idx.cpu().numpy(), t_lse.cpu().numpy(), weight.cpu().numpy(), tau)
    np.testing.assert_allclose(loss.cpu().numpy(), want_loss, rtol=1e-4, atol=1e-7)
    assert_close(S, grad, "bf16", "dS")
    G = O.gated_lowrank_bwd(host(S), host(X), host(Q), host(P), host(z), host(dz))
    for name, got in (("dX", dX), ("dP", dP), ("dQ", dQ)):
        assert_close(got, G[name], "bf16", name)
    assert not torch.any(dX[-6:]) and torch.isfinite(dla).all()
    # export
    idx, kd = torch.zeros(r, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    Pc, Qc = b.padded(V, r, BF), b.padded(r, d, BF)
    b.compact_ranks(la, 0, HC, idx, kd, torch.zeros(r, device="cuda"), P, Q, Pc, Qc)
    k = int(kd.item())
    Qq, Pq, qs, ps = b.padded(k, d, torch.int8, multiple=16), b.padded(V, k, torch.int8, multiple=16), torch.zeros(k, device="cuda"), torch.zeros(V, device="cuda")
    b.quantize_rows(Qc[:k], Qq, qs)
    b.quantize_rows(Pc[:, :k], Pq, ps)
    Y = b.padded(T, V, BF)
    b.compact_fwd_i8(X, Qq, qs, Pq, ps, Y, k, b.alloc_workspace(b.workspace_bytes(b.OP_COMPACT_FWD_I8, T, d, V, k, b.BF16)))
    want, _ = OO.compact_fwd_i8(host(X), Qq.cpu().numpy(), host(qs), Pq.cpu().numpy(), host(ps))
    assert_close(Y, want, "bf16", "8-bit logits")
    served = torch.zeros(T, device="cuda")
    b.distill_topk_fwd(Y, t_logits, t_idx, t_lse, weight, tau, served)
    want_loss, _, _ = OO.distill_topk(host(Y), t_logits.cpu().numpy(), t_idx.cpu().numpy(), t_lse.cpu().numpy(), weight.cpu().numpy(), tau)
    np.testing.assert_allclose(served.cpu().numpy(), want_loss, rtol=1e-4, atol=1e-7)
    assert b.device_status() == b.OK


def b_copy(b, a):
    t = b.padded(a.shape[0], a.shape[1], BF)
    t.copy_(torch.from_numpy(a.astype(np.float32)))
    return t


class Distill(torch.autograd.Function):
    """The calls as a caller wraps them."""

    @staticmethod
    def forward(ctx, S, t, idx, lse, tau):
        from paper_1910_04732_b200 import binding as b
        loss, stats = torch.empty(S.shape[0], device=S.device), torch.empty(S.shape[0], 4, device=S.device)
        b.distill_topk_fwd(S, t, idx, lse, None, tau, loss, stats)
        ctx.save_for_backward(S, t, idx, lse, stats)
        ctx.tau = tau
        return loss

    @staticmethod
    def backward(ctx, dloss):
        from paper_1910_04732_b200 import binding as b
        S, t, idx, lse, stats = ctx.saved_tensors
        dS = torch.empty_like(S)
        b.distill_topk_bwd(S, t, idx, lse, None, ctx.tau, stats, dloss.contiguous(), dS)
        return dS, None, None, None, None


def test_through_autograd_and_into_a_graph(b):
    g = np.random.default_rng(8)
    T, V, K = 12, 640, 10
    leaf = torch.from_numpy(g.standard_normal((T, V)).astype(np.float32)).cuda().requires_grad_()
    teacher = torch.from_numpy(g.standard_normal((T, V)).astype(np.float32)).cuda()
    t, idx = teacher.topk(K, 1)
    idx, lse = idx.int(), torch.logsumexp(teacher, 1)
    want, = torch.autograd.grad(Distill.apply(leaf, t, idx, lse, 1.0).mean(), leaf)
    _, grad, _ = OO.distill_topk(host(leaf), t.cpu().numpy(), idx.cpu().numpy(), lse.cpu().numpy(), None, 1.0)
    np.testing.assert_allclose(host(want), grad / T, rtol=1e-4, atol=1e-8)
    # the two calls of a step in a graph
    loss, stats, dS, dloss = torch.zeros(T, device="cuda"), torch.zeros(T, 4, device="cuda"), torch.zeros(T, V, device="cuda"), torch.full((T,), 1.0 / T, device="cuda")
    S, graph = leaf.detach(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.distill_topk_fwd(S, t, idx, lse, None, 1.0, loss, stats)
        b.distill_topk_bwd(S, t, idx, lse, None, 1.0, stats, dloss, dS)
    for _ in range(3):
        dS.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dS, want)
