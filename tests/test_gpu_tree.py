"""vsr_tree_rows and vsr_tree_attention against plain implementations (plain_tree.py).

Bound of an output, u half a step of its type (2^-24 fp32, 2^-8 bf16,
2^-11 fp16), K keys, A = sum p |v|, X the largest sum of
|scale q k| of the row:
  - a score is a chain of at most head_dim + 2 fp32 operations: off by (hd + 2) 2^-23 X
    (matrix units may cut where they would round), so each probability by that of
    itself, its exponential by 2^-22, its product with log2(e) by 2^-23 X more;
  - a 16-bit probability is rounded: u of itself;
  - sums over keys, in pieces joined at the end: K 2^-23 of A at most, and of the
    probabilities' sum;
  - the result is rounded: u of itself.
Together |out - want| <= u |want| + (u16 + 2 ((hd + 4) 2^-23 X + K 2^-23 + 2^-20)) A; a
lse is off by (hd + 4) 2^-23 X + K 2^-23 + 2^-21 (1 + |lse|)."""
import numpy as np
import pytest

import plain_tree as PT

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


class Case:
    """Sequences with `lens` positions and `rows` drafted rows in pages of `page`."""

    def __init__(self, torch, lens, rows, hq, hk, hd, page, dtype, tree, seed=0, spare=0, lead=0,
                 trail=0, words=None):
        from paper_2601_01513_amd import binding as B
        self.torch, self.B, self.page, self.dtype = torch, B, page, _dt(dtype)
        rng = np.random.default_rng(seed)
        seqs, rows = len(lens), np.asarray(rows)
        self.lens = np.asarray(lens, np.int32)
        self.held = np.asarray([-(-(l + n) // page) for l, n in zip(lens, rows)], np.int32)
        most = int(max(self.held.max(), 1)) + spare
        self.n_pages = int(self.held.sum()) + 3
        order = rng.permutation(self.n_pages).astype(np.int32)
        self.table = rng.integers(0, self.n_pages, (seqs, most)).astype(np.int32)
        at = 0
        for s, h in enumerate(self.held):
            self.table[s, :h] = order[at:at + h]
            at += h
        self.start = np.concatenate([[0], rows.cumsum()]).astype(np.int32) + lead
        self.T = int(self.start[-1]) + trail
        self.parent = np.full(self.T, -1, np.int32)
        for s in range(seqs):
            for j in range(1, rows[s]):
                self.parent[self.start[s] + j] = rng.integers(max(-1, j - 6), j)
        self.words = words or max(1, -(-int(rows.max()) // 32))
        self.mask = None
        if tree:
            _, _, self.mask = PT.tree_rows(self.table, self.lens, self.held, page, self.start,
                                           self.parent, self.T, self.words)
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=g, device="cuda").to(self.dtype)  # noqa: E731
        self.q = normal(self.T, hq, hd) * 1.5
        self.k, self.v = normal(self.n_pages * page, hk, hd), normal(self.n_pages * page, hk, hd)
        self.scale = hd ** -0.5

    def dev(self, x):
        if x is None:
            return None
        x = x.view(np.int32) if x.dtype == np.uint32 else x
        return self.torch.tensor(x, device="cuda")

    def pages(self):
        refs = self.torch.zeros(self.n_pages, dtype=self.torch.int32, device="cuda")
        return self.B.pages(self.dev(self.table), self.dev(self.lens), self.dev(self.held), refs,
                            self.page)

    def run(self, pages=None, **kw):
        torch = self.torch
        kw.setdefault("start", self.dev(self.start))
        kw.setdefault("mask", self.dev(self.mask))
        kw.setdefault("lse", torch.full(self.q.shape[:2], 7.0, device="cuda"))
        kw.setdefault("out", torch.full_like(self.q, 7.0))
        out = self.B.tree_attention(pages or self.pages(), self.q, kw.pop("k", self.k),
                                    kw.pop("v", self.v), self.scale, **kw)
        torch.cuda.synchronize()
        return out, kw["lse"]

    def want(self, start="own"):
        f = lambda t: t.float().cpu().numpy()  # noqa: E731
        return PT.attention(f(self.q), f(self.k), f(self.v), self.table, self.lens, self.held,
                            self.page, self.start if isinstance(start, str) else start, self.mask,
                            self.scale)

    def check(self, out, lse, want=None):
        torch, hd = self.torch, self.q.shape[2]
        y, wl, mass, size = want or self.want()
        got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
        K = int((self.lens + np.diff(self.start)).max())
        u = torch.finfo(self.dtype).eps / 2
        u16 = 0 if self.dtype is torch.float32 else u
        d = (hd + 4) * 2.0 ** -23 * size + K * 2.0 ** -23
        bound = u * np.abs(y) + (u16 + 2 * (d + 2.0 ** -20))[..., None] * mass + 1e-30
        none = np.isnan(wl).all(1)  # rows of no sequence
        live = ~none
        assert (got[none] == 7).all() and (gl[none] == 7).all()
        err = np.abs(got - y)[live]
        assert (err <= bound[live]).all(), (float(err.max()), float((err / bound[live]).max()))
        with np.errstate(invalid="ignore"):
            le = np.abs(gl - wl)[live]
        same = (gl[live] == wl[live])
        lb = (d + 2.0 ** -21 * (1 + np.abs(wl)))[live]
        assert (same | (le <= lb)).all(), float(np.nanmax(le))


CASES = [  # lens, rows, hq, hk, hd, page, dtype, tree
    ([5], [1], 1, 1, 8, 1, "f32", False),
    ([0], [1], 2, 1, 64, 16, "bf16", False),
    ([1, 0, 70], [1, 3, 1], 4, 2, 64, 8, "f16", True),
    ([200, 3], [5, 7], 4, 4, 64, 16, "f32", True),
    ([63, 64, 65, 127], [1, 1, 1, 1], 16, 2, 128, 16, "bf16", False),
    ([63, 64, 65, 1], [2, 1, 64, 130], 7, 1, 128, 32, "bf16", True),
    ([300, 0, 513], [33, 0, 40], 8, 2, 128, 64, "f16", True),
    ([300, 20], [100, 70], 4, 2, 80, 16, "bf16", False),
    ([129, 40], [9, 31], 10, 5, 36, 16, "f32", True),
    ([90], [17], 3, 1, 100, 4, "f16", True),
    ([90, 10], [3, 3], 3, 3, 7, 2, "bf16", True),
    ([150, 60], [20, 4], 4, 1, 256, 16, "bf16", True),
    ([150, 60], [20, 4], 4, 2, 256, 16, "f32", True),
    ([150, 60], [2, 1], 4, 2, 256, 16, "f32", False),
    ([33, 5], [70, 90], 2, 1, 200, 8, "f32", False),
    ([150], [40], 4, 1, 128, 16, "f32", True),
    ([1000] * 5, [64, 1, 20, 64, 33], 28, 4, 128, 16, "bf16", True),
    ([7, 300], [300, 290], 4, 2, 64, 16, "f16", True),
    ([2500], [6], 28, 4, 128, 16, "f16", True),
    ([9000, 10], [1, 1], 16, 2, 128, 256, "bf16", False),
]


@pytest.mark.parametrize("lens,rows,hq,hk,hd,page,dtype,tree", CASES)
def test_attention_against_plain_rows(lens, rows, hq, hk, hd, page, dtype, tree):
    c = Case(_torch(), lens, rows, hq, hk, hd, page, dtype, tree, seed=len(lens) + hd)
    c.check(*c.run())


@pytest.mark.parametrize("parents", [True, False])
@pytest.mark.parametrize("lens,rows,page,words", [
    ([5], [1], 1, 1), ([0, 9, 100], [3, 0, 40], 8, 2), ([64, 1], [70, 33], 16, 2),
    ([1000] * 300, [4] * 300, 16, 1), ([20], [700], 64, 30), ([3, 3], [9000, 5], 64, 3)])
def test_rows_of_trees(lens, rows, page, words, parents):
    torch = _torch()
    c = Case(torch, lens, rows, 1, 1, 8, page, "f32", False, seed=3, lead=2, trail=3, words=words)
    shift = np.arange(len(lens), dtype=np.int32) * 3 - 4
    parent = c.parent if parents else None
    if parents and c.T > 6:
        c.parent[c.start[0] + rows[0] - 1] = rows[0] - 1   # itself: a root
        c.parent[c.start[0]] = 5
    want = PT.tree_rows(c.table, c.lens, c.held, page, c.start, parent, c.T, words, shift)
    out = [torch.full((c.T,), 9, dtype=torch.int32, device="cuda") for _ in range(2)]
    wide = torch.full((c.T, words + 2), 9, dtype=torch.int32, device="cuda")
    pages = c.pages()
    c.B.tree_rows(pages, c.dev(c.start), c.dev(parent), c.dev(shift),
                  out=(*out, wide[:, 1:1 + words]))
    torch.cuda.synchronize()
    for got, w in zip((*out, wide[:, 1:1 + words]), want):
        assert np.array_equal(got.cpu().numpy(), w.view(np.int32))
    assert bool((wide[:, 0] == 9).all()) and bool((wide[:, -1] == 9).all())
    pos, slot, none = c.B.tree_rows(pages, c.dev(c.start), c.dev(parent), c.dev(shift),
                                    out=(*[torch.empty_like(o) for o in out], None))
    torch.cuda.synchronize()
    assert none is None and torch.equal(pos, out[0]) and torch.equal(slot, out[1])


@pytest.mark.parametrize("n,words,step", [(70001, 2, 1), (3000, 94, 1), (2500, 80, 300), (1100, 33, 7)])
def test_long_paths_in_time(n, words, step):
    """Paths of thousands of rows, through every group of rows or past most of them."""
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    table, start = np.zeros((2, 1), np.int32), np.array([0, 3, n + 3], np.int32)
    parent = np.concatenate([[-1, 0, 1], np.arange(n) - step]).astype(np.int32)
    p = B.pages(i32(table), i32([4, 5]), i32([1, 1]), i32([1]), 64)
    pos, slot, mask = B.tree_rows(p, i32(start), i32(parent), words=words)
    torch.cuda.synchronize()
    want = PT.tree_rows(table, [4, 5], [1, 1], 64, start, parent, n + 3, words, n_pages=1)
    for got, w in zip((pos, slot, mask), want):
        assert np.array_equal(got.cpu().numpy(), w.view(np.int32))


def test_rows_without_room_or_on_bad_pages():
    torch = _torch()
    c = Case(torch, [20, 30, 40], [10, 10, 10], 1, 1, 8, 8, "f32", False, seed=5)
    c.held[0] = 3            # room for 24 positions
    c.held[1] = 99           # more than the table has
    c.lens[1] = 1000         # more than its pages have
    c.table[2, 5] = -3       # positions 40 .. 47
    c.table[2, 6] = c.n_pages
    want = PT.tree_rows(c.table, c.lens, c.held, 8, c.start, c.parent, c.T, 1, n_pages=c.n_pages)
    pos, slot, mask = c.B.tree_rows(c.pages(), c.dev(c.start), c.dev(c.parent), words=1)
    torch.cuda.synchronize()
    assert np.array_equal(slot.cpu().numpy(), want[1])
    assert np.array_equal(pos.cpu().numpy(), want[0])
    assert (want[1][:4] >= 0).all() and (want[1][4:] == -1).all()


def test_one_row_a_sequence_without_start():
    torch = _torch()
    c = Case(torch, [70, 0, 5, 129], [1] * 4, 8, 2, 128, 16, "bf16", False, seed=6)
    c.check(*c.run(start=None), want=c.want(None))
    pos, slot, mask = c.B.tree_rows(c.pages(), None, words=1)
    torch.cuda.synchronize()
    assert pos.tolist() == [70, 0, 5, 129] and mask.flatten().tolist() == [1] * 4


def test_rows_that_see_nothing_and_rows_of_no_sequence():
    torch = _torch()
    for dtype in ("f32", "bf16"):
        c = Case(torch, [0, 90, 0], [8, 4, 70], 4, 2, 64, 16, dtype, True, seed=8, lead=3, trail=5)
        c.mask[c.start[0] + 2] = 0
        c.mask[c.start[2] + 69] = 0
        c.mask[c.start[1]] = 0           # sees its context alone
        out, lse = c.run()
        c.check(out, lse)
        assert bool((out[c.start[0] + 2] == 0).all()) and bool((lse[c.start[0] + 2] == -np.inf).all())


def test_mask_bits_beyond_the_rows_and_rows_beyond_the_words():
    torch = _torch()
    c = Case(torch, [37, 10], [40, 6], 4, 2, 64, 16, "f16", True, seed=9)
    c.mask[c.start[1]:, :] = 0xffffffff           # bits past 6 rows mean nothing
    c.check(*c.run())
    c.mask = c.mask[:, :1].copy()                  # rows 32 .. 39 have no bit
    c.check(*c.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("hd", [64, 128])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, hd):
    """NaN and infinities in the room, in unused pages, in rows that others do not see;
    those that do see one have it."""
    torch = _torch()
    inf, nan = float("inf"), float("nan")
    for rows in ([12, 3], [40, 50]):
        c = Case(torch, [70, 61], rows, 8, 2, hd, 16, dtype, True, seed=10, spare=2)
        clean = c.want()
        used = np.zeros(c.n_pages * 16, bool)
        slots = []
        for s in range(2):
            at = np.arange(c.lens[s] + rows[s])
            slots.append(c.table[s, at // 16] * 16 + at % 16)
            used[slots[-1]] = True
        c.k[torch.tensor(~used, device="cuda")] = nan
        c.v[torch.tensor(~used, device="cuda")] = inf
        # Row 2 of the first draft is nobody's but its own.
        b = c.start[0]
        c.mask[b:b + rows[0]] &= ~np.uint32(4)
        c.mask[b + 2, 0] |= 4
        clean = c.want()
        at = int(slots[0][70 + 2])
        c.v[at, 0, 3], c.v[at, 0, 4], c.v[at, 1, 5] = nan, inf, -inf
        out, lse = c.run()
        got = out.clone()
        row = int(b) + 2
        assert bool(torch.isnan(got[row, :4, 3]).all())
        assert bool((got[row, :4, 4] == inf).all()) and bool((got[row, 4:, 5] == -inf).all())
        ref = torch.tensor(clean[0], device="cuda")
        for h, d in [(slice(0, 4), 3), (slice(0, 4), 4), (slice(4, 8), 5)]:
            got[row, h, d] = ref[row, h, d].to(got.dtype)
        c.check(got, lse, want=clean)
        # A key that is no number: its own row's results are none either.
        c.k[at, 1, 0] = nan
        out, lse = c.run()
        assert bool(torch.isnan(out[row, 4:]).all()) and bool(torch.isnan(lse[row, 4:]).all())
        others = [r for r in range(c.T) if r != row]
        assert bool(torch.isfinite(out[others]).all()) and bool(torch.isfinite(lse[others]).all())
        # One in the context reaches every row.
        c.v[int(slots[1][5]), 0, 1] = nan
        out, _ = c.run()
        assert bool(torch.isnan(out[int(c.start[1]):, :4, 1]).all())
        assert bool(torch.isfinite(out[int(c.start[1]):, :, 2:]).all())


def test_large_scores_and_far_maxima():
    """Maxima that rise from tile to tile, scores of hundreds, the lowest values."""
    torch = _torch()
    for dtype in ("f32", "bf16"):
        c = Case(torch, [500], [3], 4, 2, 64, 16, dtype, False, seed=11)
        at = np.arange(503)
        slots = torch.tensor(c.table[0, at // 16] * 16 + at % 16, device="cuda")
        c.k[slots] = (c.k[slots].float() * torch.linspace(0.01, 12, 503, device="cuda")[:, None, None]).to(c.dtype)
        c.check(*c.run())
        c.k[slots[:250]] = torch.finfo(c.dtype).min / 1e3
        c.q.abs_()
        want = c.want()
        out, lse = c.run()
        assert bool(torch.isfinite(out).all())
        c.check(out, lse, want)


def test_rows_without_room_and_bad_pages():
    torch = _torch()
    c = Case(torch, [20, 30, 40], [10, 10, 10], 4, 2, 64, 8, "bf16", True, seed=12)
    c.held[0] = 3
    c.table[2, 1] = -1
    c.table[2, 2] = c.n_pages + 5
    c.table[2, 3] = 2 ** 31 - 1
    c.table[2, 4] = -2 ** 31
    c.check(*c.run())
    c.held[1], c.held[0] = -2, 0
    c.check(*c.run())


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 64), ("f16", 72)])
def test_layouts(dtype, hd):
    """Slices of stacked rows, head-major caches, bases and strides off 16 bytes."""
    torch = _torch()
    c = Case(torch, [100, 45], [20, 9], 6, 2, hd, 16, dtype, True, seed=13)
    want = c.want()
    q, k, v = c.q.clone(), c.k.clone(), c.v.clone()
    stacked = torch.zeros((c.T, 10, hd), dtype=c.dtype, device="cuda")
    stacked[:, :6] = q
    c.q = stacked[:, :6]
    out = torch.full((6, c.T, hd), 7.0, dtype=c.dtype, device="cuda").transpose(0, 1)
    kh = k.transpose(0, 1).contiguous().transpose(0, 1)
    vh = v.transpose(0, 1).contiguous().transpose(0, 1)
    c.check(*c.run(k=kh, v=vh, out=out), want=want)
    S = k.shape[0]
    for pad, shift in ((1, 1), (3, 0), (8, 3)):
        wide = torch.full((2, S * 2 * (hd + pad) + shift,), float("nan"), device="cuda").to(c.dtype)
        ks, vs = (w[shift:].view(S, 2, hd + pad)[:, :, :hd] for w in wide)
        ks.copy_(k)
        vs.copy_(v)
        mine = torch.full((c.T * 6 * (hd + 1),), 7.0, dtype=c.dtype, device="cuda")
        out = mine.view(c.T, 6, hd + 1)[:, :, :hd]
        c.check(*c.run(k=ks, v=vs, out=out), want=want)
        assert bool((mine.view(c.T, 6, hd + 1)[:, :, hd] == 7).all())
    # Pages of keys and values side by side.
    both = torch.stack([k, v], 1).contiguous()
    c.check(*c.run(k=both[:, 0], v=both[:, 1]), want=want)


def test_slots_far_apart():
    """Offsets that pass 2^31 elements."""
    torch = _torch()
    c = Case(torch, [30, 17], [5, 2], 4, 2, 64, 16, "bf16", True, seed=14)
    want = c.want()
    S, stride = c.k.shape[0], 40_000_000
    assert (S - 1) * stride > 2 ** 31
    far = torch.empty((S - 1) * stride + 512, dtype=c.dtype, device="cuda")
    k = far.as_strided((S, 2, 64), (stride, 64, 1))
    v = far.as_strided((S, 2, 64), (stride, 64, 1), 256)
    k.copy_(c.k)
    v.copy_(c.v)
    c.check(*c.run(k=k, v=v), want=want)


def test_many_sequences_and_long_ones():
    torch = _torch()
    rng = np.random.default_rng(15)
    for seqs, most in ((300, 200), (4096, 3)):
        c = Case(torch, rng.integers(0, most, seqs), rng.integers(0, 4, seqs), 4, 2, 64, 8, "bf16",
                 True, seed=16)
        c.check(*c.run())
    c = Case(torch, [40001, 3], [2, 2], 4, 2, 64, 16, "f16", False, seed=17)
    c.check(*c.run())


@pytest.mark.parametrize("dtype,hd", [("f16", 128), ("bf16", 64), ("f32", 80)])
def test_many_sequences_of_many_rows(dtype, hd):
    torch = _torch()
    rng = np.random.default_rng(23)
    rows = rng.integers(0, 40, 100)
    rows[[0, 50, 99]] = 0, 140, 1
    c = Case(torch, rng.integers(0, 300, 100), rows, 8, 2, hd, 16, dtype, True, seed=24)
    c.check(*c.run())


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(scale):
    torch = _torch()
    for rows in (1, 3, 60):
        c = Case(torch, [300, 40], [rows, rows + 1], 4, 2, 64, 16, "bf16", True, seed=rows)
        c.scale = scale
        c.check(*c.run())


def test_a_captured_call_follows_its_inputs():
    """One graph over changing lengths, starts and masks, with eager work between."""
    torch = _torch()
    cases = [Case(torch, l, r, 8, 2, 128, 16, "bf16", True, seed=s, spare=20, words=2)
             for s, (l, r) in enumerate([([50, 300, 1], [10, 20, 30]), ([0, 4, 280], [60, 0, 0]),
                                         ([200, 200, 40], [1, 1, 58])])]
    most = max(c.table.shape[1] for c in cases)
    n_pages = max(c.n_pages for c in cases)
    table = torch.zeros((3, most), dtype=torch.int32, device="cuda")
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    lens, held, start, refs = i32(3), i32(3), i32(4), i32(n_pages)
    q = torch.zeros((60, 8, 128), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros((n_pages * 16, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    mask = torch.zeros((60, 2), dtype=torch.int32, device="cuda")
    B = cases[0].B
    pages = B.pages(table, lens, held, refs, 16)
    out, lse = torch.empty_like(q), torch.empty((60, 8), device="cuda")
    ws = torch.empty(B.load_library().vsr_tree_attention_workspace_size(1, 128, 60, 3, 8, 2),
                     dtype=torch.uint8, device="cuda")
    call = lambda: B.tree_attention(pages, q, k, v, 128 ** -0.5, start, mask, out, lse, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for c in cases + cases[::-1]:
        table.zero_()
        table[:, :c.table.shape[1]] = c.dev(c.table)
        for to, x in ((lens, c.lens), (held, c.held), (start, c.start)):
            to.copy_(c.dev(x))
        mask[:c.T] = c.dev(c.mask)
        q[:c.T], k[:c.k.shape[0]], v[:c.v.shape[0]] = c.q, c.k, c.v
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        c.check(out[:c.T], lse[:c.T])
        assert bool((out[c.T:] == 7).all())


def test_streams_and_two_calls_at_once():
    torch = _torch()
    cases = [Case(torch, [3000, 100], [20, 30], 8, 2, 128, 16, "f16", True, seed=s) for s in (1, 2)]
    want = [c.run() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    pages = [c.pages() for c in cases]
    args = [dict(start=c.dev(c.start), mask=c.dev(c.mask)) for c in cases]
    torch.cuda.synchronize()
    got = [[c.B.tree_attention(p, c.q, c.k, c.v, c.scale, stream=s, **a)
            for c, s, p, a in zip(cases, streams, pages, args)] for _ in range(5)]
    torch.cuda.synchronize()
    for pair in got:
        for g, (w, _) in zip(pair, want):
            assert torch.equal(g, w)


def test_no_rows():
    torch = _torch()
    c = Case(torch, [5, 9], [0, 0], 2, 1, 64, 8, "f32", False, seed=1)
    out = c.B.tree_attention(c.pages(), torch.empty((0, 2, 64), device="cuda"), c.k, c.v, 1.0,
                             start=c.dev(c.start))
    assert out.shape == (0, 2, 64)
    c = Case(torch, [5, 9], [0, 0], 2, 1, 64, 8, "f32", False, seed=1, trail=4)
    c.check(*c.run())
