"""What the 8-bit products and the distillation loss refuse on the host, before anything is launched (no GPU needed: every call here
returns from its argument checks)."""
import ctypes

import pytest
import torch

from paper_1910_04732_b200 import binding as b
from paper_1910_04732_b200 import build

P = 1 << 20            # an aligned address that nothing is read from


@pytest.fixture(scope="module")
def lib():
    build.build()
    return b.load_library()


def quantize(lib, X=P, ldx=64, rows=4, cols=64, dt=b.BF16, Xq=4 * P, ldxq=64, scale=8 * P):
    return lib.flop_quantize_rows(X, ldx, rows, cols, dt, Xq, ldxq, scale, None)


@pytest.mark.parametrize("change,code", [
    (dict(rows=-1), b.ERR_INVALID_ARG), (dict(cols=-1), b.ERR_INVALID_ARG), (dict(dt=2), b.ERR_INVALID_ARG), (dict(rows=0), b.OK),
    (dict(X=None), b.ERR_INVALID_ARG), (dict(Xq=None), b.ERR_INVALID_ARG), (dict(scale=None), b.ERR_INVALID_ARG),
    (dict(ldx=56), b.ERR_INVALID_ARG), (dict(ldxq=48), b.ERR_INVALID_ARG), (dict(X=P + 8), b.ERR_UNSUPPORTED), (dict(ldx=65), b.ERR_UNSUPPORTED),
    (dict(Xq=4 * P + 8), b.ERR_UNSUPPORTED), (dict(ldxq=72), b.ERR_UNSUPPORTED), (dict(Xq=P), b.ERR_INVALID_ARG), (dict(Xq=P + 256), b.ERR_INVALID_ARG),
    (dict(rows=1 << 31), b.ERR_UNSUPPORTED), (dict(cols=(1 << 30) + 1, ldx=1 << 31, ldxq=1 << 31), b.ERR_UNSUPPORTED)])
def test_quantize_rows(lib, change, code):
    assert quantize(lib, **change) == code


def gemm(lib, A=P, lda=64, sa=2 * P, B=3 * P, ldb=64, sb=4 * P, Y=5 * P, ldy=32, M=8, N=32, K=64, dt=b.BF16):
    return lib.flop_gemm_i8(A, lda, sa, B, ldb, sb, Y, ldy, M, N, K, dt, None)


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), b.ERR_INVALID_ARG), (dict(N=-1), b.ERR_INVALID_ARG), (dict(K=-1), b.ERR_INVALID_ARG), (dict(dt=5), b.ERR_INVALID_ARG),
    (dict(M=0), b.OK), (dict(N=0), b.OK), (dict(A=None), b.ERR_INVALID_ARG), (dict(B=None), b.ERR_INVALID_ARG), (dict(Y=None), b.ERR_INVALID_ARG),
    (dict(sa=None), b.ERR_INVALID_ARG), (dict(sb=None), b.ERR_INVALID_ARG), (dict(lda=48), b.ERR_INVALID_ARG), (dict(ldy=24), b.ERR_INVALID_ARG),
    (dict(lda=72), b.ERR_UNSUPPORTED), (dict(ldb=72), b.ERR_UNSUPPORTED), (dict(A=P + 1), b.ERR_UNSUPPORTED), (dict(B=P + 8), b.ERR_UNSUPPORTED),
    (dict(Y=P + 2), b.ERR_UNSUPPORTED), (dict(ldy=33), b.ERR_UNSUPPORTED), (dict(K=131072, lda=131072, ldb=131072), b.ERR_UNSUPPORTED),
    (dict(M=4000001), b.ERR_UNSUPPORTED), (dict(N=4000001, ldy=4000008), b.ERR_UNSUPPORTED)])
def test_gemm_i8(lib, change, code):
    assert gemm(lib, **change) == code


def compact(lib, X=P, ldx=64, Q=2 * P, ldq=64, qs=3 * P, Pq=4 * P, ldp=32, ps=5 * P, Y=6 * P, ldy=128, T=8, d_in=64, d_out=128, k=20, dt=b.BF16, ws=16 * P, wb=1 << 20):
    return lib.flop_compact_fwd_i8(X, ldx, Q, ldq, qs, Pq, ldp, ps, Y, ldy, T, d_in, d_out, k, dt, ws, wb, None)


@pytest.mark.parametrize("change,code", [
    (dict(T=-1), b.ERR_INVALID_ARG), (dict(k=-1), b.ERR_INVALID_ARG), (dict(dt=-1), b.ERR_INVALID_ARG), (dict(T=0), b.OK), (dict(d_out=0), b.OK),
    (dict(X=None), b.ERR_INVALID_ARG), (dict(Q=None), b.ERR_INVALID_ARG), (dict(Pq=None), b.ERR_INVALID_ARG), (dict(qs=None), b.ERR_INVALID_ARG),
    (dict(ps=None), b.ERR_INVALID_ARG), (dict(Y=None), b.ERR_INVALID_ARG), (dict(ldq=48), b.ERR_INVALID_ARG), (dict(ldp=16), b.ERR_INVALID_ARG),
    (dict(ldp=40), b.ERR_UNSUPPORTED), (dict(Q=P + 4), b.ERR_UNSUPPORTED), (dict(X=P + 2), b.ERR_UNSUPPORTED), (dict(ldy=130), b.ERR_UNSUPPORTED),
    (dict(ws=None), b.ERR_WORKSPACE), (dict(ws=16 * P + 16), b.ERR_WORKSPACE), (dict(wb=256), b.ERR_WORKSPACE),
    (dict(d_in=131072, ldx=131072, ldq=131072, wb=1 << 40), b.ERR_UNSUPPORTED)])
def test_compact_fwd_i8(lib, change, code):
    assert compact(lib, **change) == code


def test_workspace_of_the_8_bit_forward(lib):
    # quantised tokens, 32-bit sums or 8-bit intermediate, two scales per token
    assert b.workspace_bytes(b.OP_COMPACT_FWD_I8, 100, 70, 64, 30, b.BF16) >= 100 * (80 + 32 + 8)
    assert b.workspace_bytes(b.OP_COMPACT_FWD_I8, 0, 0, 0, 0, b.F32) == 0
    out = ctypes.c_size_t(0)
    assert lib.flop_workspace_bytes(7, 1, 1, 1, 1, 0, ctypes.byref(out)) == b.ERR_INVALID_ARG


STUDENT = dict(S=P, lds=64, T=4, V=64, dt=b.BF16, t=2 * P, ldt=8, idx=3 * P, ldi=8, K=8, lse=None, weight=None, tau=1.0)


def distill(lib, form, stats=5 * P, dloss=None, dS=6 * P, ldds=64, loss=4 * P, **change):
    a = list({**STUDENT, **change}.values())
    if form == "fwd":
        return lib.flop_distill_topk_fwd(*a, loss, stats, None)
    if form == "bwd":
        return lib.flop_distill_topk_bwd(*a, stats, dloss, dS, ldds, None)
    return lib.flop_distill_topk_fwd_bwd(*a, loss, dS, ldds, None)


@pytest.mark.parametrize("form", ["fwd", "bwd", "both"])
@pytest.mark.parametrize("change,code", [
    (dict(T=-1), b.ERR_INVALID_ARG), (dict(V=-1), b.ERR_INVALID_ARG), (dict(K=-1), b.ERR_INVALID_ARG), (dict(dt=9), b.ERR_INVALID_ARG), (dict(T=0), b.OK),
    (dict(tau=0.0), b.ERR_INVALID_ARG), (dict(tau=-1.0), b.ERR_INVALID_ARG), (dict(tau=float("inf")), b.ERR_INVALID_ARG), (dict(tau=float("nan")), b.ERR_INVALID_ARG),
    (dict(S=None), b.ERR_INVALID_ARG), (dict(t=None), b.ERR_INVALID_ARG), (dict(idx=None), b.ERR_INVALID_ARG), (dict(lds=56), b.ERR_INVALID_ARG),
    (dict(ldt=7), b.ERR_INVALID_ARG), (dict(ldi=7), b.ERR_INVALID_ARG), (dict(lds=65), b.ERR_UNSUPPORTED), (dict(S=P + 2), b.ERR_UNSUPPORTED),
    (dict(K=1025, ldt=1025, ldi=1025), b.ERR_UNSUPPORTED), (dict(V=524289, lds=524296, ldds=524296), b.ERR_UNSUPPORTED)])
def test_distill(lib, form, change, code):
    assert distill(lib, form, **change) == code


def test_distill_outputs(lib):
    for form in ("fwd", "both"):
        assert distill(lib, form, loss=None) == b.ERR_INVALID_ARG
    assert distill(lib, "bwd", stats=None) == b.ERR_INVALID_ARG
    for form in ("bwd", "both"):
        assert distill(lib, form, dS=None) == b.ERR_INVALID_ARG
        assert distill(lib, form, ldds=56) == b.ERR_INVALID_ARG
        assert distill(lib, form, ldds=66) == b.ERR_UNSUPPORTED
        assert distill(lib, form, dS=P + 128) == b.ERR_INVALID_ARG                      # part of the logits
        assert distill(lib, form, dS=P, ldds=72) == b.ERR_INVALID_ARG                   # the logits, in other rows


# ---- the binding: shapes and types that the library, which sees addresses, cannot check
def z(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


I8, BF = torch.int8, torch.bfloat16


@pytest.mark.parametrize("args,exc", [
    ((z(2, 16), z(2, 16), z(2)), TypeError), ((z(2, 16).half(), z(2, 16, dtype=I8), z(2)), TypeError), ((z(2, 16), z(2, 16, dtype=I8), z(1)), AssertionError),
    ((z(2, 16), z(3, 16, dtype=I8), z(2)), AssertionError), ((z(2, 16), z(2, 32, dtype=I8), z(2)), AssertionError), ((z(2, 16), z(2, 16, dtype=I8), z(2).double()), TypeError),
    ((z(16, 2).t(), z(2, 16, dtype=I8), z(2)), AssertionError), ((None, z(2, 16, dtype=I8), z(2)), AttributeError)])
def test_binding_quantize_rows(args, exc):
    with pytest.raises(exc):
        b.quantize_rows(*args)


@pytest.mark.parametrize("i,bad,exc", [(0, z(2, 16), TypeError), (1, z(4, 32, dtype=I8), AssertionError), (2, z(1), AssertionError), (3, z(8)[::2], AssertionError),
                                       (4, z(2, 4, dtype=I8), TypeError), (4, z(3, 4), AssertionError), (4, z(2, 5), AssertionError)])
def test_binding_gemm_i8(i, bad, exc):
    args = [z(2, 16, dtype=I8), z(4, 16, dtype=I8), z(2), z(4), z(2, 4)]
    args[i] = bad
    with pytest.raises(exc):
        b.gemm_i8(*args)


@pytest.mark.parametrize("i,bad,exc", [(1, z(3, 16), TypeError), (1, z(2, 16, dtype=I8), AssertionError), (1, z(3, 32, dtype=I8), AssertionError), (2, z(2), AssertionError),
                                       (3, z(8, 2, dtype=I8), AssertionError), (4, z(7), AssertionError), (5, z(2, 8, dtype=BF), AssertionError), (5, z(2, 7), AssertionError),
                                       (6, 4, AssertionError)])
def test_binding_compact_fwd_i8(i, bad, exc):
    args = [z(2, 16), z(3, 16, dtype=I8), z(3), z(8, 3, dtype=I8), z(8), z(2, 8), 3, None]
    args[i] = bad
    with pytest.raises(exc):
        b.compact_fwd_i8(*args)


@pytest.mark.parametrize("i,bad,exc", [(0, z(2, 8).half(), TypeError), (1, z(2, 3).double(), TypeError), (1, z(3, 3), AssertionError), (2, z(2, 3, dtype=torch.int64), TypeError),
                                       (2, z(2, 4, dtype=torch.int32), AssertionError), (3, z(1), AssertionError), (4, z(2, dtype=BF), TypeError), (5, "warm", ValueError),
                                       (6, z(1), AssertionError), (7, z(2, 8, dtype=BF), AssertionError), (7, z(2, 9), AssertionError)])
def test_binding_distill(i, bad, exc):
    args = [z(2, 8), z(2, 3), z(2, 3, dtype=torch.int32), z(2), z(2), 1.0, z(2), z(2, 8)]
    args[i] = bad
    with pytest.raises(exc):
        b.distill_topk_fwd_bwd(*args)
    if i < 6:
        with pytest.raises(exc):
            b.distill_topk_fwd(*args[:7])
        with pytest.raises(exc):
            b.distill_topk_bwd(*args[:6], z(2, 4), None, args[7])
