"""vsr_pick_tokens against a plain row-by-row implementation: the rules bit for
bit in fp32, the token exactly, the log-probability within the bound below.

Bound of a log-probability -log1p(S), S the sum of exp(l - max) over the other
tokens: S's terms are off by at most 2^-20 of themselves where they matter (the
fast exponential: |x| 2^-24 for exp(x), weighted by exp(x)), its sums by 40
roundings of 2^-24, so log1p(S) by 2^-18 min(1, S), and the result's own rounding
and log1p's by 2^-22 of it."""
import numpy as np
import pytest

from plain_decoder import apply_rules

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _inputs(torch, rows, vocab, dtype, seed, n_prompt=0, n_output=0, penalties=True, bias="none",
            mask="none"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    logits = (torch.randn((rows, vocab), generator=g, device="cuda") * 4).to(_dt(dtype))
    kw = {}
    for key, n in (("prompt", n_prompt), ("output", n_output)):
        if n:
            ids = (rand(rows, n) ** 3 * vocab).to(torch.int32)
            ids[rand(rows, n) < 0.1] = -1
            ids[rand(rows, n) < 0.05] = vocab + 3
            kw[key] = ids
            kw[key + "_len"] = torch.randint(-1, n + 3, (rows,), generator=g, device="cuda",
                                             dtype=torch.int32)
    if penalties:
        kw.update(repetition=0.8 + rand(rows), presence=rand(rows), frequency=0.3 * rand(rows))
    if bias != "none":
        kw["bias"] = torch.randn((1 if bias == "one" else rows, vocab), generator=g, device="cuda")
    if mask != "none":
        kw["mask"] = torch.randint(-2 ** 31, 2 ** 31 - 1, (1 if mask == "one" else rows,
                                                           (vocab + 31) // 32), generator=g,
                                   device="cuda", dtype=torch.int32)
    return logits, kw


def _row(kw, r):
    """Row r's rules and lists on the host."""
    host = {k: v.cpu().numpy() for k, v in kw.items() if v is not None}
    lists = {}
    for key in ("prompt", "output"):
        ids = host[key][r] if key in host else np.zeros(0, np.int32)
        n = int(np.clip(host[key + "_len"][r], 0, len(ids))) if key + "_len" in host else len(ids)
        lists[key] = ids[:n]
    if "repetition" not in host:
        lists["prompt"] = lists["prompt"][:0]
    rules = {k: float(host[k][r]) for k in ("repetition", "presence", "frequency") if k in host}
    for k in ("bias", "mask"):
        if k in host:
            rules[k] = host[k][r % host[k].shape[0]]
            if k == "mask":
                rules[k] = rules[k].view(np.uint32)
    return lists["prompt"], lists["output"], rules


def _check(torch, logits, kw, token, logprob, processed=None):
    torch.cuda.synchronize()
    token, logprob = token.cpu().numpy(), logprob.cpu().numpy()
    x = logits.float().cpu().numpy()
    for r in range(x.shape[0]):
        prompt, output, rules = _row(kw, r)
        y = apply_rules(x[r], prompt, output, **rules)
        if processed is not None:
            got = processed[r].cpu().numpy()
            assert np.array_equal(got, y), (r, np.flatnonzero(got != y)[:5])
        if y.max() == -np.inf:
            assert token[r] == -1 and logprob[r] == -np.inf, (r, token[r], logprob[r])
            continue
        assert token[r] == np.argmax(y), (r, token[r], np.argmax(y))
        z = y.astype(np.float64) - y.max()
        z[token[r]] = -np.inf
        S = np.exp(z).sum()
        want = -np.log1p(S)
        bound = 2.0 ** -18 * min(1.0, S) + 2.0 ** -22 * abs(want)
        assert abs(logprob[r] - want) <= bound, (r, logprob[r], want, bound)


CASES = [  # rows, vocab, dtype, prompt, output, penalties, bias, mask
    (1, 1, "f32", 0, 0, False, "none", "none"),
    (2, 1, "bf16", 3, 2, True, "one", "rows"),
    (3, 31, "f16", 5, 1, True, "rows", "one"),
    (4, 33, "f32", 1, 9, True, "none", "rows"),
    (2, 2047, "f32", 40, 40, True, "one", "one"),
    (2, 2048, "bf16", 300, 0, True, "none", "none"),
    (2, 2049, "bf16", 0, 300, True, "rows", "none"),
    (3, 4096, "f16", 100, 100, False, "one", "none"),
    (3, 4100, "f32", 1000, 900, True, "rows", "rows"),
    (5, 12347, "f16", 700, 50, True, "rows", "rows"),
    (40, 1000, "f32", 64, 64, True, "rows", "rows"),
    (2, 151936, "bf16", 512, 64, True, "one", "one"),
    (3, 152064, "f32", 5000, 1100, True, "rows", "rows"),
    (300, 777, "bf16", 20, 20, True, "none", "one"),
]


@pytest.mark.parametrize("keep", [False, True], ids=["pick", "kept"])
@pytest.mark.parametrize("rows,vocab,dtype,n_prompt,n_output,penalties,bias,mask", CASES)
def test_against_plain_rows(rows, vocab, dtype, n_prompt, n_output, penalties, bias, mask, keep):
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    logits, kw = _inputs(torch, rows, vocab, dtype, rows + vocab, n_prompt, n_output, penalties,
                         bias, mask)
    processed = torch.full((rows, vocab), 7.0, device="cuda") if keep else None
    token, logprob = B.pick_tokens(logits, processed=processed, **kw)
    _check(torch, logits, kw, token, logprob, processed)
    only = torch.empty_like(token)
    B.pick_tokens(logits, out=(only, None), **kw)
    torch.cuda.synchronize()
    assert torch.equal(only, token)


@pytest.mark.parametrize("which", ["repetition", "presence", "frequency", "none"])
def test_single_penalties(which):
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    logits, kw = _inputs(torch, 4, 3000, "f32", 11, 200, 100, True)
    for k in ("repetition", "presence", "frequency"):
        if k != which:
            kw.pop(k)
    processed = torch.empty((4, 3000), device="cuda")
    token, logprob = B.pick_tokens(logits, processed=processed, **kw)
    _check(torch, logits, kw, token, logprob, processed)


def test_ties_go_to_the_lowest_index():
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    for dtype in ("f32", "bf16"):
        x = torch.zeros((6, 20000), device="cuda").to(_dt(dtype))
        for r, at in enumerate([(0, 19999), (5, 6), (4095, 4096), (8191, 12288), (300, 700), (1, 17000)]):
            x[r, list(at)] = 3.0
        token, logprob = B.pick_tokens(x)
        torch.cuda.synchronize()
        assert token.tolist() == [0, 5, 4095, 8191, 300, 1]
        same, _ = B.pick_tokens(torch.full((1, 20000), -2.5, device="cuda").to(_dt(dtype)))
        assert same.tolist() == [0]


def test_rows_left_with_nothing_and_masked_garbage():
    """A mask of zeros; logits of -inf and of the lowest value; infinities and
    NaNs where the mask forbids them, and where it does not."""
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    inf, nan, low = float("inf"), float("nan"), torch.finfo(torch.float32).min
    V = 5000
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((8, V), generator=g, device="cuda")
    mask = torch.full((8, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
    mask[0] = 0
    x[1] = -inf
    x[2] = low
    clean = x[3].clone()
    x[3, 64:96] = torch.tensor([inf, -inf, nan, low] * 8, device="cuda")
    mask[3, 2] = 0           # forbids 64..95
    x[4, 4999] = nan         # allowed
    x[5, 7] = inf            # allowed
    x[6] = nan
    mask[7] = 0
    mask[7, 156] = 1 << 7    # only token 4999
    x[7, 4999] = -80.0
    processed = torch.empty_like(x)
    token, logprob = B.pick_tokens(x, mask=mask, processed=processed)
    torch.cuda.synchronize()
    t, p = token.tolist(), logprob.tolist()
    assert t[0] == -1 and p[0] == -inf and bool((processed[0] == -inf).all())
    assert t[1] == -1 and p[1] == -inf
    assert t[2] == 0 and abs(p[2] + np.log(V)) < 1e-5
    clean[64:96] = -inf
    assert t[3] == int(clean.argmax()) and abs(p[3] - float(clean.log_softmax(0).max())) < 1e-5
    assert t[4] == int(x[4, :4999].argmax()) and np.isnan(p[4])
    assert t[5] == 7 and np.isnan(p[5])
    assert t[6] == -1 and np.isnan(p[6])
    assert t[7] == 4999 and p[7] == 0.0
    # Mask bits past the vocabulary are not looked at.
    tail, _ = B.pick_tokens(torch.full((1, 33), -inf, device="cuda"),
                            mask=torch.full((1, 2), -1, dtype=torch.int32, device="cuda"))
    assert tail.tolist() == [-1]


def test_a_near_certain_token_keeps_its_digits():
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    x = torch.full((1, 9000), -30.0, device="cuda")
    x[0, 123] = 5.0
    _, logprob = B.pick_tokens(x)
    want = -np.log1p(8999 * np.exp(-35.0))
    assert abs(float(logprob[0]) - want) <= 2.0 ** -17 * abs(want)


def test_strides_and_in_place():
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    rows, V = 5, 4099
    logits, kw = _inputs(torch, rows, V, "f32", 4, 30, 30, True, "rows", "rows")
    want = torch.empty((rows, V), device="cuda")
    ref = B.pick_tokens(logits, processed=want, **kw)
    for pad, shift in ((1, 0), (5, 3), (13, 4)):
        wide = torch.full((rows * (V + pad) + shift,), 9.0, device="cuda")
        view = wide[shift:].view(rows, V + pad)[:, :V]
        view.copy_(logits)
        lists = {k: torch.cat([kw[k], kw[k]], 1)[:, :30] for k in ("prompt", "output")}
        got = B.pick_tokens(view, processed=view, **dict(kw, **lists))
        torch.cuda.synchronize()
        assert torch.equal(got[0], ref[0]) and torch.equal(view, want)
        # (Another alignment sums the same terms in another order.)
        assert torch.allclose(got[1], ref[1], rtol=1e-5, atol=2.0 ** -17)
        assert bool((wide[:shift] == 9).all())
        assert bool((wide[shift:].view(rows, V + pad)[:, V:] == 9).all())


def test_no_rows_another_stream_and_a_captured_call():
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    token, logprob = B.pick_tokens(torch.empty((0, 100), device="cuda"))
    assert token.shape == (0,) and logprob.shape == (0,)
    logits, kw = _inputs(torch, 6, 20001, "bf16", 8, 100, 100, True, "one", "rows")
    want = B.pick_tokens(logits, **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = B.pick_tokens(logits, stream=side, **kw)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out = torch.empty_like(want[0]), torch.empty_like(want[1])
    ws = torch.empty(B.load_library().vsr_pick_workspace_size(6, 20001), dtype=torch.uint8,
                     device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pick_tokens(logits, out=out, workspace=ws, **kw)
    for seed in (1, 2, 3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        logits.copy_(torch.randn(logits.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = B.pick_tokens(logits, **kw)
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_many_chunks_and_outputs_larger_than_the_caches():
    """More chunks than lanes of a wave; processed logits above 64 MB."""
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    logits, kw = _inputs(torch, 2, 300001, "bf16", 21, 900, 90, True, "one", "rows")
    processed = torch.empty((2, 300001), device="cuda")
    token, logprob = B.pick_tokens(logits, processed=processed, **kw)
    _check(torch, logits, kw, token, logprob, processed)
    logits, kw = _inputs(torch, 130, 130003, "f16", 22, 40, 40, True, "none", "one")
    processed = torch.empty((130, 130003), device="cuda")
    assert processed.numel() * 4 > 64 << 20
    token, logprob = B.pick_tokens(logits, processed=processed, **kw)
    for r in (0, 64, 129):
        one = {k: v if k == "mask" else v[r:r + 1] for k, v in kw.items()}
        _check(torch, logits[r:r + 1], one, token[r:r + 1], logprob[r:r + 1], processed[r:r + 1])
    assert torch.equal(processed.argmax(1).int().cpu(), token.cpu())


def test_two_calls_at_once():
    """Calls on two streams, each with its own workspace."""
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    cases = [_inputs(torch, 24, 60001, "f32", s, 500, 200, True, "one", "rows") for s in (31, 32)]
    want = [B.pick_tokens(x, **kw) for x, kw in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[B.pick_tokens(x, stream=s, **kw) for (x, kw), s in zip(cases, streams)]
           for _ in range(5)]
    torch.cuda.synchronize()
    for pair in got:
        for (t, p), (wt, wp) in zip(pair, want):
            assert torch.equal(t, wt) and torch.equal(p, wp)


def test_rows_far_apart():
    """Offsets that pass 2^31 elements, of the logits and of the kept ones."""
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    rows, V, stride = 3, 5001, 1_100_000_003
    assert (rows - 1) * stride > 2 ** 31
    x, kw = _inputs(torch, rows, V, "bf16", 41, 30, 30, True, "rows", "rows")
    far = torch.empty((rows - 1) * stride + V, dtype=torch.bfloat16,
                      device="cuda").as_strided((rows, V), (stride, 1))
    far.copy_(x)
    kept = torch.empty((rows - 1) * stride + V, device="cuda").as_strided((rows, V), (stride, 1))
    token, logprob = B.pick_tokens(far, processed=kept, **kw)
    _check(torch, x, kw, token, logprob, kept)


def test_inputs_dropped_behind_another_streams_work():
    """Picks on a busy stream; their lists, rules and logits dropped after the call
    and their memory given to others."""
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    make = lambda: _inputs(torch, 8, 30001, "f32", 51, 300, 100, True, "rows", "rows")  # noqa: E731
    logits, kw = make()
    want = B.pick_tokens(logits, **kw)
    side = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    logits, kw = make()
    shapes = [(t.shape, t.dtype) for t in (logits, *kw.values())]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            torch.mm(busy, busy)
    got = B.pick_tokens(logits, stream=side, **kw)
    del logits, kw
    others = [torch.ones(shape, dtype=dtype, device="cuda") for shape, dtype in shapes]
    torch.cuda.synchronize()
    assert all(map(torch.equal, got, want)) and len(others) == len(shapes)
