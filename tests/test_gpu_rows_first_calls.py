"""Calls that nothing prepared: the first call of a process inside a graph capture, calls on threads of their own at the same time, tensors used on a stream that is
not the one they were made on."""
import subprocess
import sys
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


FIRST = """
import torch
from paper_1910_04732_b200 import binding as b
T, V, d = 3000, 400, 264
ids = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
X, dY, E, dE = (torch.randn(n, d, device="cuda") for n in (T, T, V, V))
Y, S, dX, dR = (torch.empty(T, d, device="cuda") for _ in range(4))
w, dw, db, stats = torch.ones(d, device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda"), torch.empty(T, 2, device="cuda")
ws = [b.alloc_workspace(b.workspace_bytes(op, T, d, 0, V, b.F32)) for op in (b.OP_EMBEDDING_SORTED_BWD, b.OP_LAYER_NORM_BWD)]
b.load_library(); b._native()
torch.cuda.synchronize()

def step():
    b.embedding_fwd(ids, E, 2.0, Y)
    b.dropout_fwd(Y, X, 0.1, 1, 0)
    b.layer_norm_fwd(X, w, None, 1e-5, Y, stats, R=dY, S=S, p=0.2, seed=1, offset=9)
    b.layer_norm_bwd(dY, S, stats, w, dX, dw, db, ws[1], dR=dR, p=0.2, seed=1, offset=9)
    b.dropout_bwd(dX, dX, 0.1, 1, 0)
    b.embedding_bwd(dX, ids, 2.0, dE, ws[0])

graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (Y, S, dX, dR, dw, db, dE)]
step()
for x, y in zip(got, (Y, S, dX, dR, dw, db, dE)):
    assert torch.equal(x, y)
print("same")
"""


def test_first_calls_inside_a_capture():
    r = subprocess.run([sys.executable, "-c", FIRST], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


def test_two_threads_at_once(b):
    """Each with its own stream, workspace and sizes: the results are those of the same calls one after the other."""
    g = torch.Generator(device="cuda").manual_seed(7)
    works = []
    for T, V, d in ((5000, 300, 264), (700, 900, 1032)):
        ids = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        X, dY = (torch.randn(T, d, generator=g, device="cuda").bfloat16() for _ in range(2))
        w = torch.ones(d, device="cuda")
        works.append((ids, X, dY, w, T, V, d))

    def run(ids, X, dY, w, T, V, d):
        Y, S, dX, stats = torch.empty_like(X), torch.empty_like(X), torch.empty_like(X), torch.empty(T, 2, device="cuda")
        dw, db, dE = torch.empty(d, device="cuda"), torch.empty(d, device="cuda"), torch.empty(V, d, device="cuda")
        ws = [b.alloc_workspace(b.workspace_bytes(op, T, d, 0, V, b.BF16)) for op in (b.OP_EMBEDDING_SORTED_BWD, b.OP_LAYER_NORM_BWD)]
        for _ in range(200):
            b.layer_norm_fwd(X, w, None, 1e-5, Y, stats, R=dY, S=S, p=0.2, seed=1, offset=9)
            b.layer_norm_bwd(dY, S, stats, w, dX, dw, db, ws[1], p=0.2, seed=1, offset=9)
            b.embedding_bwd(dX, ids, 2.0, dE, ws[0])
        return Y, S, dX, dw, db, dE

    want = [run(*w) for w in works]
    torch.cuda.synchronize()
    got, errors, start = [None, None], [], threading.Barrier(2)

    def body(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                start.wait()
                got[i] = run(*works[i])
            stream.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=body, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors[0]
    for x, y in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(x, y))


def test_a_stream_of_the_callers_choice(b):
    """The calls wait for what their stream waits for, and for nothing else."""
    T, d = 4000, 2048
    X, Y, Z = torch.zeros(T, d, device="cuda"), torch.empty(T, d, device="cuda"), torch.empty(T, d, device="cuda")
    side = torch.cuda.Stream()
    for i in range(5):
        X.fill_(float(i + 1))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b.dropout_fwd(X, Y, 0.5, 3, i)
            b.dropout_bwd(Y, Z, 0.5, 3, i)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(Z, 2 * Y) and set(Y.unique().tolist()) == {0.0, 2.0 * (i + 1)}
