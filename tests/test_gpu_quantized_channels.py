"""Weight channels without a scale in the compact forward in 8 bits: `flop_quantize_rows` gives a factor row that holds an infinity or a
NaN the scale NaN, so that what is computed from it is NaN.  Such a channel enters every token's intermediate, wherever in a row its
column lies and whichever kernel takes the row's maximum."""
import numpy as np
import pytest
import torch

from oracle import operators as O
from tests.test_gpu_quantized import DTYPES, b, check_scaled, factors, host, run_compact, tokens, whole  # noqa: F401

pytestmark = pytest.mark.gpu


def poisoned(b, dtype, T, d_in, k, d_out):  # noqa: F811
    g = np.random.default_rng(T + d_in + k)
    x, (Qq, qs, Pq, ps) = tokens(g, T, d_in, dtype), factors(g, k, d_in, d_out)
    if T > 1:
        x[T - 1] = 0                                 # a token of zeros: its sums are 0, and 0 times such a scale is NaN
    clean = run_compact(b, x, Qq, qs, Pq, ps)
    for at in sorted({0, 3 % k, 7 % k, 8 % k, k // 2, k - 1}):
        for n, scale in enumerate((float("nan"), float("inf"))):
            Q, s = whole(g, k, d_in), qs.clone()
            Q.copy_(Qq)
            s[at] = scale
            if n == 0:
                Q[at] = 0                            # what quantise_rows makes of such a row
            Y = run_compact(b, x, Q, s, Pq, ps)
            assert torch.isnan(Y).all(), (at, scale, int(torch.isnan(Y).all(1).sum()))
    # the calls before leave nothing behind
    assert torch.equal(run_compact(b, x, Qq, qs, Pq, ps), clean)
    rows = np.unique(np.r_[:min(T, 5), T - 1])
    want, _ = O.compact_fwd_i8(host(x)[rows], *(host(t) for t in (Qq, qs, Pq, ps)))
    check_scaled(clean[torch.from_numpy(rows).cuda()], want, dtype, 6)


# up to 16 tokens whose sums the second product's blocks scale (one to eight warps to a row); more than 1024 components
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d_in,k,d_out", [(1, 96, 17, 40), (1, 96, 358, 40), (1, 200, 1500, 100), (2, 96, 600, 64), (3, 96, 143, 90), (4, 410, 1500, 64), (5, 96, 8, 33), (8, 96, 358, 96),
                                            (8, 4096, 143, 40), (12, 96, 143, 50), (16, 96, 358, 64), (16, 64, 17, 40), (40, 96, 1500, 50), (300, 64, 1030, 40)])
def test_sums_scaled_in_fp64(b, dtype, T, d_in, k, d_out):  # noqa: F811
    poisoned(b, dtype, T, d_in, k, d_out)


# the first product's epilogue: one to four blocks to a row, whole and ragged slices
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,d_in,k,d_out", [(9, 1024, 358, 64), (12, 96, 600, 50), (16, 600, 900, 40), (17, 64, 17, 40), (40, 96, 143, 50), (40, 200, 358, 64), (130, 96, 600, 64),
                                            (300, 96, 16, 33), (300, 96, 143, 50), (300, 128, 1024, 40), (2500, 64, 300, 33)])
def test_sums_scaled_in_the_epilogue(b, dtype, T, d_in, k, d_out):  # noqa: F811
    poisoned(b, dtype, T, d_in, k, d_out)


@pytest.mark.parametrize("T,d_in,k,d_out", [(150, 410, 143, 60), (300, 264, 300, 96), (300, 96, 16, 33)])
def test_slices_that_end_inside_32_columns(b, T, d_in, k, d_out):  # noqa: F811
    """The maximum of a row is taken over what this product put into tensor memory, not over the fp32 sums that another one left behind it."""
    g = np.random.default_rng(k)
    x, f = tokens(g, T, d_in, torch.bfloat16), factors(g, k, d_in, d_out)
    want = run_compact(b, x, *f)
    check_scaled(want, O.compact_fwd_i8(host(x), *(host(t) for t in f))[0], torch.bfloat16, 6)
    X, Q, P, Y = (b.padded(*s, torch.bfloat16) for s in ((18944, 256), (64, 256), (256, 64), (18944, 256)))
    for fill in (1e30, -3.0, float("nan")):
        X.fill_(fill), Q.fill_(1.0), P.fill_(1.0)
        b.compact_fwd(X, Q, P, Y, 64, b.alloc_workspace(b.workspace_bytes(b.OP_COMPACT_FWD, 18944, 256, 256, 64, b.BF16)))
        assert torch.equal(run_compact(b, x, *f), want)
