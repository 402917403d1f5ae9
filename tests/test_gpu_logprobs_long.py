"""vsr_token_logprobs where one segment holds a whole long row: the roundings of its sums.

Bounds: a term e^d is off by 2^-20 of itself where it matters (|d| <= 30 after rounding x's
product with log2(e): |d| 2^-23 of it, weighted by e^d: 2^-22, and 2^-22 of the exponential
itself); 16 of a tile are added in 6 roundings, tiles in 64 bits (one more at their end),
lanes, waves and the move to the largest value in 6 + 2 * 3 + 4: 2^-19.5 of S, so log1p(S)
by 2^-19.5 and its own 2^-23 (1 + lse). W, whose terms are e^d d with d up to 4 above the
reference, by 2^-19.5 of sum e^d (|d| + 8): the entropy by that over 1 + S."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _rows(torch, V):
    """Rows whose sums a chain of roundings would show in."""
    i = torch.arange(V, device="cuda", dtype=torch.float32)
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.randn(V, generator=g, device="cuda")
    yield torch.where(i == V // 3, 3.0, 0.0)      # all alike below one
    yield torch.where(i == V - 1, 1.7, 0.0)
    yield torch.where(i == 0, 0.3, 0.0)
    yield i / V                                   # the largest value rises from tile to tile
    yield 30 * i / V
    yield -3 * i / V
    yield z * 0.01 + 4 * i / V
    yield z
    yield torch.where(i % 5000 == 77, 20.0, z)


@pytest.mark.parametrize("V,rows,dtype", [(152064, 1030, "float32"), (152064, 1030, "bfloat16"),
                                          (152064, 1030, "float16"), (152064, 3, "float32"),
                                          (1 << 20, 1030, "bfloat16"), (1 << 22, 1030, "bfloat16")])
def test_sums_of_long_segments(V, rows, dtype):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_01513_amd import binding as B
    given = list(_rows(torch, V))
    x = torch.zeros((rows, V), dtype=getattr(torch, dtype), device="cuda")
    for at in range(0, min(rows, len(given))):
        x[at] = given[at].to(x.dtype)
    n = min(rows, len(given))
    t = torch.arange(rows, dtype=torch.int32, device="cuda") * 11
    for top in (0, 5):
        got = B.token_logprobs(x, t, top)
        torch.cuda.synchronize()
        for r in range(n):
            y = x[r].double()
            d = y - y.max()
            e = d.exp()
            e[int(y.argmax())] = 0
            S, W, size = float(e.sum()), float((e * d).sum()), float((e * (d.abs() + 8)).sum())
            lse = np.log1p(S)
            off = 2.0 ** -19.5 * min(1.0, S)
            lp, H = float(d[int(t[r])]) - lse, lse - W / (1 + S)
            assert abs(float(got.logprob[r]) - lp) <= off + 2.0 ** -23 * (1 + abs(lp)), (r, lp)
            assert abs(float(got.entropy[r]) - H) <= off + 2.0 ** -19.5 * size / (1 + S) + \
                2.0 ** -23 * (1 + H), (r, H)
            if top:
                best = y.topk(top).values - y.max() - lse
                assert float((got.top_logprob[r].double() - best).abs().max()) <= \
                    off + 2.0 ** -23 * (1 + float(best.abs().max())), r
