"""8-bit rows, their products and the compact forward in 8 bits against the fp64 oracle.

Integers are equal: the rounding is decided as in exact arithmetic.  What is left are the roundings of the scaled results: a sum to fp32, the
two scales (2^-24 each), a scale of the intermediate that is itself two products and a quotient, and the rounding to the stored type (2^-24 or 2^-8).
Every output sits in rows with padding; padding of the inputs holds 99 (or NaN), of the outputs a mark that must survive."""
import numpy as np
import pytest
import torch

from oracle import operators as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
DTYPES = [torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def b():
    from paper_1910_04732_b200 import build, binding
    build.build()
    binding.load_library()
    return binding


def padded(rows, cols, dtype, fill, extra=0):
    per = 16 // torch.empty((), dtype=dtype).element_size()
    ld = (cols + per - 1) // per * per + extra * per
    return torch.full((rows, max(ld, per)), fill, dtype=dtype, device="cuda")[:, :cols]


def behind(t):
    """The columns between a matrix's rows' ends and its leading dimension."""
    return t.as_strided((t.shape[0], t.stride(0) - t.shape[1]), (t.stride(0), 1), t.storage_offset() + t.shape[1])


def tokens(g, rows, cols, dtype, extra=0):
    x = padded(rows, cols, dtype, float("nan"), extra)
    x.copy_(torch.from_numpy((g.standard_normal((rows, cols)) * np.exp(g.uniform(-3, 3, (rows, 1)))).astype(np.float32)))
    return x


def whole(g, rows, cols, extra=0, lo=-127):
    q = padded(rows, cols, torch.int8, 99, extra)
    q.copy_(torch.from_numpy(g.integers(lo, 128, (rows, cols)).astype(np.int8)))
    return q


def host(t):
    return t.detach().cpu().double().numpy() if t.dtype != torch.int8 else t.cpu().numpy().astype(np.int64)


def check_scaled(got, want, dtype, roundings):
    got = host(got)
    assert np.all(np.isfinite(got))
    bound = np.abs(want) * (roundings * U * 1.0001 + STORE[dtype]) + 1e-38
    assert np.all(np.abs(got - want) <= bound), float(np.max(np.abs(got - want) / bound))


# ------------------------------------------------------------------------------------------------ rows
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,extra", [(1, 1, 0), (1, 1024, 0), (3, 7, 1), (5, 8, 0), (4, 410, 2), (130, 33, 0), (2, 1025, 1), (33, 4096, 0), (3, 8200, 0), (2, 20011, 1), (300, 256, 0)])
def test_rows(b, dtype, rows, cols, extra):
    x = tokens(np.random.default_rng(rows + cols), rows, cols, dtype, extra)
    q, scale = padded(rows, cols, torch.int8, 55, extra), torch.full((rows,), -1.0, device="cuda")
    b.quantize_rows(x, q, scale)
    want, ws = O.quantize_rows(host(x))
    assert np.array_equal(host(q), want) and np.array_equal(scale.cpu().numpy(), ws)
    assert torch.all(behind(q) == 55)


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_on_the_border(b, dtype):
    # 127 x / 127 = n + 1/2 exactly, and the neighbours of such x; every exponent; subnormal rows
    n = np.arange(-127, 127) + 0.5
    rows = [np.r_[n, 127.0], np.r_[np.nextafter(n.astype(np.float32), np.float32(np.inf)), np.float32(127)], np.r_[np.nextafter(n.astype(np.float32), np.float32(-np.inf)), np.float32(127)]]
    rows = np.stack(rows + [r * 2.0 ** e for r in rows[:1] for e in (-130, -100, 3, 100)] + [np.r_[n * 0, 1e-45], np.r_[np.sign(n) * 1e-40, 3e-39], np.r_[n, 1e3]])
    x = padded(rows.shape[0], rows.shape[1], dtype, float("nan"))
    x.copy_(torch.from_numpy(rows.astype(np.float32)))
    q, scale = padded(*rows.shape, torch.int8, 55), torch.zeros(rows.shape[0], device="cuda")
    b.quantize_rows(x, q, scale)
    want, ws = O.quantize_rows(host(x))
    assert np.array_equal(host(q), want) and np.array_equal(scale.cpu().numpy(), ws)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [5, 1024, 9000])
def test_rows_without_a_scale(b, dtype, cols):
    x = tokens(np.random.default_rng(cols), 6, cols, dtype)
    x[0] = 0
    x[1, cols - 1], x[2, 0], x[3, cols // 2] = float("inf"), float("nan"), float("-inf")
    x[4] = -0.0
    q, scale = padded(6, cols, torch.int8, 55), torch.zeros(6, device="cuda")
    b.quantize_rows(x, q, scale)
    want, ws = O.quantize_rows(host(x))
    assert np.array_equal(host(q), want) and np.array_equal(scale.cpu().numpy(), ws, equal_nan=True)


def test_rows_of_fp32_from_any_address(b):
    g = np.random.default_rng(9)
    base = torch.from_numpy(g.standard_normal(20000).astype(np.float32)).cuda()
    for off, ld, cols in ((1, 101, 101), (3, 1027, 1001), (2, 54, 50)):
        x = base.as_strided((9, cols), (ld, 1), off)
        q, scale = padded(9, cols, torch.int8, 55), torch.zeros(9, device="cuda")
        b.quantize_rows(x, q, scale)
        want, ws = O.quantize_rows(host(x))
        assert np.array_equal(host(q), want) and np.array_equal(scale.cpu().numpy(), ws)


def test_rows_behind_32_bit_offsets(b):
    rows, cols = 70000, 32768                        # 4.6 GB of bf16: the last rows lie beyond 2^31 elements
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-2:] = torch.randn(2, cols, device="cuda")
    q, scale = torch.full((rows, cols), 55, dtype=torch.int8, device="cuda"), torch.full((rows,), -1.0, device="cuda")
    b.quantize_rows(x, q, scale)
    want, ws = O.quantize_rows(host(x[-2:]))
    assert np.array_equal(host(q[-2:]), want) and np.array_equal(scale[-2:].cpu().numpy(), ws)
    assert not torch.any(q[:-2]) and not torch.any(scale[:-2])


# ------------------------------------------------------------------------------------------------ products
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K,extra", [(1, 1, 1, 0), (1, 4096, 1024, 0), (2, 33, 17, 1), (7, 100, 64, 0), (8, 16, 128, 0), (9, 250, 410, 2), (16, 1000, 358, 0), (17, 130, 1000, 0),
                                         (31, 65, 95, 1), (33, 2100, 410, 0), (64, 64, 512, 0), (65, 300, 4097, 0), (127, 129, 130, 0), (128, 256, 128, 0), (150, 2100, 410, 1),
                                         (256, 256, 256, 0), (257, 511, 385, 0), (300, 70, 2048, 0), (1000, 1000, 1000, 0), (600, 2600, 144, 0), (4096, 358, 200, 0), (2000, 4096, 64, 1),
                                         (5, 5001, 2100, 0), (16, 5003, 2047, 1), (32, 5000, 1100, 0), (24, 4801, 1001, 2)])
def test_products(b, dtype, M, N, K, extra):
    g = np.random.default_rng(M + N + K)
    A, B = whole(g, M, K, extra, -128), whole(g, N, K, 0, -128)
    sa, sb = (torch.from_numpy(np.exp(g.uniform(-4, 4, n)).astype(np.float32)).cuda() for n in (M, N))
    Y = padded(M, N, dtype, -7.0, extra)
    for _ in range(2):                                # twice: the second call starts while the first one drains
        b.gemm_i8(A, B, sa, sb, Y)
    check_scaled(Y, O.gemm_i8(host(A), host(B), host(sa), host(sb)), dtype, 3)
    assert torch.all(behind(Y) == -7.0) and b.device_status() == b.OK


@pytest.mark.parametrize("M,N", [(1, 40), (40, 300), (300, 300)])
def test_largest_sums(b, M, N):
    """The longest contraction, every product 128 * 128 (and -128 * 127): 2^31 - 2^14 in the 32-bit sum."""
    K = 131071
    A, B = padded(M, K, torch.int8, 99), padded(N, K, torch.int8, 99)
    A.fill_(-128), B.fill_(-128)
    B[N // 2:] = 127
    Y, one = padded(M, N, torch.float32, 0.0), torch.ones(M, device="cuda")
    b.gemm_i8(A, B, one, torch.ones(N, device="cuda"), Y)
    want = np.where(np.arange(N) < N // 2, 128 * 128 * K, -128 * 127 * K)[None].repeat(M, 0)
    check_scaled(Y, want, torch.float32, 1)
    assert b.device_status() == b.OK


@pytest.mark.parametrize("dtype", DTYPES)
def test_scales_of_zero_and_nan(b, dtype):
    g = np.random.default_rng(5)
    for M in (4, 200):
        A, B = whole(g, M, 100), whole(g, 70, 100)
        sa, sb = torch.ones(M, device="cuda"), torch.ones(70, device="cuda")
        sa[1], sa[2], sb[3] = 0.0, float("nan"), float("nan")
        Y = padded(M, 70, dtype, -7.0)
        b.gemm_i8(A, B, sa, sb, Y)
        nan = torch.isnan(Y)
        assert nan[2].all() and nan[:, 3].all() and nan.sum() == 70 + M - 1 and not torch.any(Y[1][~nan[1]])


def test_products_of_nothing(b):
    Y = padded(5, 9, torch.bfloat16, -7.0)
    b.gemm_i8(padded(5, 0, torch.int8, 0), padded(9, 0, torch.int8, 0), torch.ones(5, device="cuda"), torch.ones(9, device="cuda"), Y)
    assert not torch.any(Y) and torch.all(behind(Y) == -7.0)


@pytest.mark.parametrize("M,N,K", [(3, 50, 100), (100, 150, 100), (300, 301, 300)])
def test_fp32_results_at_any_address(b, M, N, K):
    g = np.random.default_rng(M)
    A, B = whole(g, M, K), whole(g, N, K)
    sa, sb = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    for off, ld in ((1, N), (2, N + 3), (0, N + 1)):
        base = torch.full((off + M * ld + 8,), -7.0, device="cuda")
        Y = base.as_strided((M, N), (ld, 1), off)
        b.gemm_i8(A, B, sa, sb, Y)
        check_scaled(Y, O.gemm_i8(host(A), host(B), host(sa), host(sb)), torch.float32, 3)
        assert torch.all(base[:off] == -7) and torch.all(base[off + (M - 1) * ld + N:] == -7)


# ------------------------------------------------------------------------------------------------ the compact forward
def factors(g, k, d_in, d_out, extra=0):
    Qq, Pq = whole(g, k, d_in, extra), whole(g, d_out, k, extra)
    return Qq, torch.from_numpy(np.exp(g.uniform(-2, 2, k)).astype(np.float32) * 1e-3).cuda(), Pq, torch.from_numpy(np.exp(g.uniform(-2, 2, d_out)).astype(np.float32) * 1e-3).cuda()


def run_compact(b, x, Qq, qs, Pq, ps, extra=0):
    T, k, d_out = x.shape[0], Qq.shape[0], Pq.shape[0]
    dt = b.BF16 if x.dtype == torch.bfloat16 else b.F32
    n = b.workspace_bytes(b.OP_COMPACT_FWD_I8, T, x.shape[1], d_out, k, dt)
    ws = b.alloc_workspace(n + 256).fill_(0xFF)
    Y = padded(T, d_out, x.dtype, -7.0, extra)
    for _ in range(2):
        b.compact_fwd_i8(x, Qq, qs, Pq, ps, Y, k, ws[:n])
    assert torch.all(behind(Y) == -7.0) and torch.all(ws[n:] == 0xFF) and b.device_status() == b.OK
    return Y


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1, 2, 8, 9, 16, 17, 33, 64, 100, 128, 129, 300, 1000])
@pytest.mark.parametrize("d_in,k,d_out,extra", [(1, 1, 1, 0), (30, 17, 33, 1), (1024, 358, 4096, 0), (410, 143, 2100, 0), (264, 512, 96, 0), (200, 513, 130, 0), (4096, 100, 64, 0), (77, 256, 300, 2)])
def test_compact_forward(b, dtype, T, d_in, k, d_out, extra):
    if T > 300 and d_in * d_out > 10 ** 6:
        T = 200
    g = np.random.default_rng(T + d_in)
    x, f = tokens(g, T, d_in, dtype, extra), factors(g, k, d_in, d_out, extra)
    want, _ = O.compact_fwd_i8(host(x), *(host(t) for t in f))
    check_scaled(run_compact(b, x, *f, extra), want, dtype, 6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d_in,k,d_out", [(5000, 600, 901, 70), (9000, 300, 300, 64), (19001, 150, 60, 33)])
def test_compact_forward_of_many_tokens(b, dtype, T, d_in, k, d_out):
    """More blocks of the first product than SMs; the rows looked at are the first, the last and some between."""
    g = np.random.default_rng(T)
    x, f = tokens(g, T, d_in, dtype), factors(g, k, d_in, d_out)
    Y = run_compact(b, x, *f)
    pick = np.unique(np.r_[:130, T - 130:T, g.integers(0, T, 300)])
    want, _ = O.compact_fwd_i8(host(x)[pick], *(host(t) for t in f))
    check_scaled(Y[torch.from_numpy(pick).cuda()], want, dtype, 6)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_token_does_not_depend_on_the_others(b, dtype):
    """Bit for bit the same in calls of every length: the integers and the order of the scalings do not depend on the kernels."""
    g = np.random.default_rng(2)
    x, f = tokens(g, 700, 410, dtype), factors(g, 143, 410, 600)
    all_ = run_compact(b, x, *f)
    for lo, n in ((0, 1), (5, 8), (40, 16), (3, 33), (100, 64), (200, 150), (10, 400)):
        assert torch.equal(run_compact(b, x[lo:lo + n], *f), all_[lo:lo + n]), n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [4, 40, 300])
def test_tokens_without_a_scale(b, dtype, T):
    g = np.random.default_rng(T)
    x, f = tokens(g, T, 200, dtype), factors(g, 60, 200, 90)
    x[0] = 0
    x[1, 199], x[2, 3] = float("inf"), float("nan")
    Y = run_compact(b, x, *f)
    assert not torch.any(Y[0]) and torch.isnan(Y[1:3]).all()
    want, _ = O.compact_fwd_i8(host(x[3:]), *(host(t) for t in f))
    check_scaled(Y[3:], want, dtype, 6)


@pytest.mark.parametrize("T", [3, 40, 300])
def test_intermediate_on_the_border(b, T):
    """Sums that are n + 1/2 parts of the largest one: the intermediate goes to the even neighbour, in every kernel."""
    k = 200
    x = torch.full((T, 16), 127.0, device="cuda")
    Qq, Pq = padded(k, 16, torch.int8, 99), padded(k, k, torch.int8, 99)
    Qq.zero_(), Pq.zero_()
    n = torch.arange(k, device="cuda") % 127
    Qq[:, 0], Qq[:, 1] = n, n                        # 127 * (2 n + 1): halves of 254
    Qq[:, 2] = 1
    Qq[0, :3] = torch.tensor([127, 127, 0])          # the largest: 127 * 254
    Pq.fill_diagonal_(1)
    one = torch.ones(k, device="cuda")
    Y = run_compact(b, x, Qq, one, Pq, one)
    want, hq = O.compact_fwd_i8(host(x), host(Qq), host(one), host(Pq), host(one))
    assert sorted(set(hq[0, 1:120] % 2)) == [0]      # they are ties, decided to even
    check_scaled(Y, want, torch.float32, 6)


def test_factors_of_compact_ranks(b):
    """The path of a deployed model: gates -> compact factors -> 8 bits, with the views that a kept capacity leaves."""
    from tests._util import HC, rel_fro
    g = np.random.default_rng(0)
    r, d_in, d_out, T = 200, 264, 520, 50
    la = torch.from_numpy(np.where(g.random(r) < 0.4, 4.0, -4.0).astype(np.float32)).cuda()
    P, Q = (b.padded(*s, torch.bfloat16) for s in ((d_out, r), (r, d_in)))
    P.copy_(torch.randn(d_out, r) * r ** -0.5), Q.copy_(torch.randn(r, d_in) * d_in ** -0.5)
    Pc, Qc = b.padded(d_out, r, torch.bfloat16), b.padded(r, d_in, torch.bfloat16)
    idx, kd = torch.zeros(r, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    b.compact_ranks(la, 0, HC, idx, kd, torch.zeros(r, device="cuda"), P, Q, Pc, Qc)
    k = int(kd.item())
    Qq, Pq = b.padded(k, d_in, torch.int8, multiple=16), b.padded(d_out, k, torch.int8, multiple=16)
    qs, ps = torch.zeros(k, device="cuda"), torch.zeros(d_out, device="cuda")
    b.quantize_rows(Qc[:k], Qq, qs)
    b.quantize_rows(Pc[:, :k], Pq, ps)
    X = b.padded(T, d_in, torch.bfloat16)
    X.copy_(torch.randn(T, d_in))
    Y8, Y16 = b.padded(T, d_out, torch.bfloat16), b.padded(T, d_out, torch.bfloat16)
    b.compact_fwd_i8(X, Qq, qs, Pq, ps, Y8, k, b.alloc_workspace(b.workspace_bytes(b.OP_COMPACT_FWD_I8, T, d_in, d_out, k, b.BF16)))
    b.compact_fwd(X, Qc[:k], Pc[:, :k], Y16, k, b.alloc_workspace(b.workspace_bytes(b.OP_COMPACT_FWD, T, d_in, d_out, k, b.BF16)))
    # four quantised operands, each off by at most half of 1/127 of its row's largest value: uniform in that step is
    # max / (127 sqrt 12), and the largest of a few hundred normal values is below 4 times their size: 0.0091 each
    assert rel_fro(host(Y8), host(Y16)) < 4 * 0.0091


# ------------------------------------------------------------------------------------------------ streams and graphs
def test_two_streams_and_replays(b):
    g = np.random.default_rng(3)
    f = factors(g, 143, 410, 600)
    xs = [tokens(g, n, 410, torch.bfloat16) for n in (5, 150)]
    want = [run_compact(b, x, *f) for x in xs]
    outs, graphs, streams = [], [], [torch.cuda.Stream() for _ in xs]
    for x, s in zip(xs, streams):
        ws = b.alloc_workspace(b.workspace_bytes(b.OP_COMPACT_FWD_I8, x.shape[0], 410, 600, 143, b.BF16))
        Y = padded(x.shape[0], 600, torch.bfloat16, 0.0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            b.compact_fwd_i8(x, *f, Y, 143, ws)
        outs.append((Y, ws)), graphs.append(graph)
    for _ in range(20):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for (Y, _), w in zip(outs, want):
        assert torch.equal(Y, w)
