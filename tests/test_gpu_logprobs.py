"""vsr_token_logprobs against a plain implementation in 64 bits.

Bounds, S the sum of exp(l - max) over the other tokens: its terms are off by 2^-20 of
themselves where they matter (the fast exponential: |x| 2^-23 of exp(x), weighted by it),
sums of up to 40 roundings in a row a lane and tree by 40 2^-24 more: log1p(S) by 2^-18
min(1, S). A log-probability adds the rounding of x - max and of itself, 2^-22 of it; an
entropy log1p(S) - W / (1 + S) has W's terms e^d d, off by 2^-18 of sum |d| e^d, over
1 + S: 2^-17 of the entropy's two parts. Ids, ranks: exact."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _check(logits, tokens, top, got):
    x = logits.double().cpu().numpy()
    got = [None if g is None else g.cpu().numpy() for g in got]
    logprob, rank, entropy, top_id, top_lp = got
    V = x.shape[1]
    for r in range(x.shape[0]):
        m = x[r].max()
        if m == -np.inf:
            assert logprob[r] == -np.inf and entropy[r] == 0
            assert (top_id[r] == -1).all() and (top_lp[r] == -np.inf).all()
            continue
        best = int(np.argmax(x[r]))
        d = x[r] - m
        e = np.exp(d)
        e[best] = 0
        S, W = e.sum(), (e * np.where(e > 0, d, 0)).sum()
        lse = np.log1p(S)
        off = 2.0 ** -18 * min(1.0, S)
        if tokens is not None:
            t = int(tokens[r])
            if 0 <= t < V:
                want = d[t] - lse
                if want == -np.inf:
                    assert logprob[r] == -np.inf
                else:
                    assert abs(logprob[r] - want) <= off + 2.0 ** -22 * abs(want), (r, logprob[r], want)
                assert rank[r] == (x[r] > x[r, t]).sum() + (x[r, :t] == x[r, t]).sum(), r
            else:
                assert logprob[r] == -np.inf and rank[r] == -1
        want = lse - W / (1 + S)
        assert abs(entropy[r] - want) <= off + 2.0 ** -17 * (lse - W / (1 + S)) + 2.0 ** -22, \
            (r, entropy[r], want)
        if top:
            order = np.argsort(-x[r], kind="stable")[:top]
            order = order[x[r, order] > -np.inf]
            n = len(order)
            assert np.array_equal(top_id[r, :n], order), (r, top_id[r], order)
            assert (top_id[r, n:] == -1).all() and (top_lp[r, n:] == -np.inf).all()
            want = d[order] - lse
            assert (np.abs(top_lp[r, :n] - want) <= off + 2.0 ** -22 * np.abs(want)).all(), r


def _run(torch, logits, tokens, top, **kw):
    from paper_2601_01513_amd import binding as B
    got = B.token_logprobs(logits, tokens, top, **kw)
    torch.cuda.synchronize()
    return got


def _inputs(torch, rows, vocab, dtype, seed, spread=4.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn((rows, vocab), generator=g, device="cuda") * spread).to(_dt(dtype))
    t = torch.randint(-2, vocab + 2, (rows,), generator=g, device="cuda", dtype=torch.int32)
    likely = torch.rand(rows, generator=g, device="cuda") < 0.5
    return x, torch.where(likely, x.float().argmax(1).int(), t)


@pytest.mark.parametrize("rows,vocab,top,dtype", [
    (1, 1, 1, "f32"), (2, 1, 0, "bf16"), (3, 7, 64, "f16"), (3, 31, 5, "bf16"), (2, 500, 64, "f32"),
    (5, 1023, 20, "f16"), (4, 1024, 20, "f32"), (4, 1025, 1, "bf16"), (3, 4095, 64, "bf16"),
    (3, 4096, 33, "f32"), (3, 4097, 3, "f16"), (40, 12347, 20, "f16"), (300, 777, 8, "bf16"),
    (2, 151936, 5, "f32"), (3, 152064, 64, "bf16"), (1500, 9001, 10, "f32"), (1100, 20011, 20, "bf16"),
    (1, 300001, 40, "f16"),
])
def test_against_plain_rows(rows, vocab, top, dtype):
    torch = _torch()
    x, t = _inputs(torch, rows, vocab, dtype, rows + vocab)
    got = _run(torch, x, t, top)
    assert (got.top_id is None) == (top == 0)
    _check(x, t, top, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_orders_that_rise_fall_and_tie(dtype):
    torch = _torch()
    V = 30011
    i = torch.arange(V, device="cuda", dtype=torch.float32)
    g = torch.Generator(device="cuda").manual_seed(3)
    few = torch.randint(0, 3, (V,), generator=g, device="cuda").float()
    rows = [i / 3000, -i / 3000, torch.zeros_like(i), -(i - 15000).abs() / 1000, i % 17, few,
            torch.where(i < V - 70, 0.0, 1.0), torch.where(i % 1024 == 5, 2.0, -1.0), -0.0 * (i % 2) + 0.0]
    x = torch.stack(rows * 130)[:1100].to(_dt(dtype))      # one segment a row
    x[8, ::3] = -0.0
    t = torch.randint(0, V, (x.shape[0],), generator=g, device="cuda", dtype=torch.int32)
    for top in (1, 20, 64):
        _check(x[:9], t[:9], top, _run(torch, x[:9].contiguous(), t[:9], top))
        got = _run(torch, x, t, top)
        _check(x[:27], t[:27], top, [o[:27] for o in got])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_segments(dtype):
    """Whole rows of 18 tiles in one segment: spans of two tiles."""
    torch = _torch()
    V = 70001
    x, t = _inputs(torch, 1030, V, dtype, 5)
    i = torch.arange(V, device="cuda", dtype=torch.float32)
    g = torch.Generator(device="cuda").manual_seed(6)
    few = torch.randint(0, 4, (V,), generator=g, device="cuda").float()
    odd = [i / 7000, -i / 7000, 0 * i, few, (i % 8192 < 40).float(), (i % 4096 == 4095).float() - 1,
           torch.where(i > V - 50, 3.0, few), torch.where(i % 2 == 0, -float("inf"), few)]
    x[:len(odd)] = torch.stack(odd).to(x.dtype)
    for top in (1, 20, 64):
        got = _run(torch, x, t, top)
        _check(x[:20], t[:20], top, [o[:20] for o in got])


def test_nothing_nan_and_infinity():
    torch = _torch()
    inf, nan = float("inf"), float("nan")
    for rows, V in ((8, 5000), (1200, 700)):
        x, t = _inputs(torch, rows, V, "f32", 4)
        t[:8] = torch.tensor([3, 3, 3, 3, 3, 3, 3, 3])
        x[0] = -inf
        x[1] = torch.finfo(torch.float32).min
        x[2, 4:] = -inf
        x[3, 699] = nan
        x[4, 7] = inf
        x[5] = nan
        x[6, 3] = -inf
        x[7, 3] = nan
        got = _run(torch, x, t, 20)
        _check(x[:3], t[:3], 20, [o[:3] for o in got])
        _check(x[6:7], t[6:7], 20, [o[6:7] for o in got])
        for r in (3, 4, 5, 7):
            assert np.isnan(float(got.logprob[r])) and np.isnan(float(got.entropy[r]))
            assert bool(torch.isnan(got.top_logprob[r]).all())
        assert got.top_id[4, 0] == 7 and got.rank[4] >= 1 and got.rank[7] == -1 and got.rank[5] == -1
        clean = torch.where(torch.isnan(x), -inf, x)
        for r in (3, 7):
            assert got.top_id[r].tolist() == clean[r].topk(20).indices.tolist()
        assert bool((got.top_id[5] == -1).all())
        _check(x[8:40], t[8:40], 20, [o[8:40] for o in got])


def test_a_near_certain_token_keeps_its_digits():
    torch = _torch()
    x = torch.full((2, 9000), -30.0, device="cuda")
    x[0, 123] = 5.0
    x[1, 8999] = 3.0
    got = _run(torch, x, torch.tensor([123, 8999], dtype=torch.int32, device="cuda"), 2)
    for r, m in ((0, 5.0), (1, 3.0)):
        want = -np.log1p(8999 * np.exp(-30.0 - m))
        assert abs(float(got.logprob[r]) - want) <= 2.0 ** -17 * abs(want)
        assert float(got.top_logprob[r, 0]) == float(got.logprob[r])
        S = 8999 * np.exp(-30.0 - m)
        want = np.log1p(S) + S * (30 + m) / (1 + S)
        assert abs(float(got.entropy[r]) - want) <= 2.0 ** -16 * want


def test_strides_and_outputs_not_asked_for():
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    x, t = _inputs(torch, 6, 4099, "bf16", 8)
    want = _run(torch, x, t, 12)
    for pad, shift in ((1, 0), (5, 3), (13, 1)):
        wide = torch.full((6 * (4099 + pad) + shift,), 99.0, device="cuda").to(x.dtype)
        view = wide[shift:].view(6, 4099 + pad)[:, :4099]
        view.copy_(x)
        got = _run(torch, view, t, 12)
        _check(x, t, 12, got)
    for drop in range(5):
        out = [None if i == drop else torch.full_like(o, 7) for i, o in enumerate(want)]
        B.token_logprobs(x, t, 12, out=out)
        torch.cuda.synchronize()
        assert all(o is None or torch.equal(o, w) for o, w in zip(out, want))
    got = _run(torch, x, None, 12)
    assert got.logprob is None and got.rank is None and torch.equal(got.top_id, want.top_id)
    assert torch.equal(got.entropy, want.entropy)
    assert B.token_logprobs(x[:0], t[:0], 3).top_id.shape == (0, 3)


def test_rows_far_apart():
    """Offsets that pass 2^31 elements."""
    torch = _torch()
    rows, V, stride = 3, 5001, 1_100_000_003
    x, t = _inputs(torch, rows, V, "f16", 41)
    far = torch.empty((rows - 1) * stride + V, dtype=x.dtype,
                      device="cuda").as_strided((rows, V), (stride, 1))
    far.copy_(x)
    _check(x, t, 9, _run(torch, far, t, 9))


def test_picks_agree():
    """The token vsr_pick_tokens picks is the likeliest here, with the same log-prob."""
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    x, _ = _inputs(torch, 5, 152064, "bf16", 12)
    x[3] = -float("inf")
    token, logprob = B.pick_tokens(x)
    got = _run(torch, x, token, 1)
    assert torch.equal(got.top_id[:, 0], token) and got.rank.tolist() == [0, 0, 0, -1, 0]
    assert torch.allclose(got.logprob, logprob, rtol=2 ** -17, atol=0)


def test_captured_streams_and_two_calls():
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    x, t = _inputs(torch, 6, 20001, "bf16", 8)
    want = _run(torch, x, t, 15)
    out = [torch.empty_like(o) for o in want]
    ws = torch.empty(B.load_library().vsr_token_logprobs_workspace_size(6, 20001, 15),
                     dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.token_logprobs(x, t, 15, out=out, workspace=ws)
    for seed in (1, 2, 3):
        y, u = _inputs(torch, 6, 20001, "bf16", seed)
        x.copy_(y)
        t.copy_(u)
        graph.replay()
        torch.cuda.synchronize()
        assert all(map(torch.equal, out, _run(torch, y, u, 15)))
    cases = [_inputs(torch, 24, 60001, "f32", s) for s in (31, 32)]
    want = [_run(torch, *c, 30) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[B.token_logprobs(*c, 30, stream=s) for c, s in zip(cases, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    for pair in got:
        for g, w in zip(pair, want):
            assert all(map(torch.equal, g, w))
