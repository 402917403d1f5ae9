"""vsr_pages_update and vsr_pages_keep against plain implementations, bit for bit."""
import numpy as np
import pytest

import plain_tree as PT

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


class Cache:
    """A paged cache on the host and on the device. shape: layers, heads, head_dim."""

    def __init__(self, torch, seqs, most, n_pages, page, shape=(2, 2, 8), dtype="float16", seed=0):
        from paper_2601_01513_amd import binding as B
        self.torch, self.B, self.page, self.rng = torch, B, page, np.random.default_rng(seed)
        L, H, hd = shape
        self.table = self.rng.integers(-3, n_pages + 3, (seqs, most)).astype(np.int32)
        self.len, self.held = np.zeros(seqs, np.int32), np.zeros(seqs, np.int32)
        self.refs = np.zeros(n_pages, np.int32)
        bits = {"float16": np.uint16, "float32": np.uint32}[dtype]
        self.k, self.v = (self.rng.integers(0, np.iinfo(bits).max, (L, n_pages * page, H, hd),
                                            dtype=bits, endpoint=True) for _ in range(2))
        self.dtype = getattr(torch, dtype)

    def fill(self, lens, room=0):
        """Every sequence has its own pages, in no order."""
        order = list(self.rng.permutation(len(self.refs)))
        for s, n in enumerate(lens):
            self.len[s], self.held[s] = n, -(-(n + room) // self.page)
            for c in range(self.held[s]):
                self.table[s, c] = order.pop()
                self.refs[self.table[s, c]] = 1
        return self

    def to_device(self):
        t = lambda x: self.torch.tensor(x, device="cuda")  # noqa: E731
        signed = {2: np.int16, 4: np.int32}[self.k.itemsize]
        self.dk, self.dv = (t(x.view(signed)).view(self.dtype) for x in (self.k, self.v))
        self.pages = self.B.pages(t(self.table), t(self.len), t(self.held), t(self.refs), self.page)
        return self

    def same(self):
        self.torch.cuda.synchronize()
        p = self.pages
        for name, got, want in (("table", p.table, self.table), ("len", p.len, self.len),
                                ("held", p.held, self.held), ("refs", p.refs, self.refs)):
            assert np.array_equal(got.cpu().numpy(), want), name
        signed = {2: self.torch.int16, 4: self.torch.int32}[self.k.itemsize]
        for got, want in ((self.dk, self.k), (self.dv, self.v)):
            assert np.array_equal(got.view(signed).cpu().numpy().view(want.dtype), want)

    def update(self, source=None, room=None, **kw):
        t = lambda x: None if x is None else self.torch.tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
        ok = self.B.pages_update(self.pages, t(source), t(room), kw.pop("k", self.dk),
                                 kw.pop("v", self.dv), **kw)
        want = PT.pages_update(self.table, self.len, self.held, self.refs, self.page, source, room,
                               self.k, self.v)
        self.torch.cuda.synchronize()
        assert np.array_equal(ok.cpu().numpy(), want), (ok.tolist(), want.tolist())
        self.same()
        return want

    def keep(self, kept, n_kept=None, release=True, apart=False, **kw):
        torch = self.torch
        t = lambda x: None if x is None else torch.tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
        out = torch.full((len(self.len),), 77, dtype=torch.int32, device="cuda") if apart else None
        got = self.B.pages_keep(self.pages, t(kept), t(n_kept), kw.pop("k", self.dk),
                                kw.pop("v", self.dv), out, release, **kw)
        want = PT.pages_keep(self.table, self.len, self.held, self.refs, self.page,
                             np.asarray(kept, np.int32), n_kept, self.k, self.v, release)
        torch.cuda.synchronize()
        assert np.array_equal(got.cpu().numpy(), want), (got.tolist(), want.tolist())
        if not apart:
            self.len[:] = want
        self.same()


def test_room_alone():
    c = Cache(_torch(), 5, 8, 40, 4).fill([0, 4, 5, 31, 17]).to_device()
    assert c.update(room=[1, 1, -7, 1, 0]).all()
    assert not c.update(room=[40, 0, 27, 2, 0])[[0, 3]].any()   # more than the table has
    assert c.update().all()
    c.update(room=[2 ** 31 - 1] * 5)


def test_room_when_pages_run_out():
    c = Cache(_torch(), 6, 8, 20, 2).fill([2, 4, 6, 8, 2, 2]).to_device()   # 8 free
    assert c.update(room=[4, 8, 6, 2, 0, 2]).tolist() == [1, 1, 0, 0, 1, 0]
    assert c.update(room=[4, 8, 2, 2, 2, 0]).tolist() == [1, 1, 1, 1, 0, 1]
    assert (c.refs > 0).all()


def test_forks_moves_drops():
    torch = _torch()
    c = Cache(torch, 8, 6, 60, 4).fill([9, 8, 3, 0, 23, 1, 12, 5], room=1).to_device()
    c.update([0, 0, 0, 1, 1, 4, 4, -1])             # full and partial last pages, a drop
    c.update([1, 0, 3, 2, 5, 4, 7, 6], [1] * 8)     # everyone changes places
    c.update([2, 2, 3, 3, 3, 3, 3, 3], [5] * 8)     # the source moves and has heirs
    c.update([8, -2, 99, 3, 2 ** 31 - 1, -2 ** 31, 6, 0])   # others stay
    c.update([-1] * 8, [3, 0, 0, 9, 0, 0, 0, 0])
    assert c.refs.sum() == 4


def test_copies_without_a_page_are_cut():
    torch = _torch()
    c = Cache(torch, 6, 4, 6, 4).fill([6, 0, 0, 0, 0, 4]).to_device()   # 3 of 6 pages free
    assert c.update([0, 0, 0, 0, 0, 5], [2, 0, 4, 0, 1, 0]).tolist() == [1, 1, 1, 0, 0, 1]
    assert c.len.tolist() == [6, 6, 6, 4, 4, 4]


@pytest.mark.parametrize("seed", range(6))
def test_random_steps(seed):
    """Forks, drops, room and kept rows in turn, also when pages run short."""
    torch = _torch()
    rng = np.random.default_rng(seed)
    page, seqs = int(rng.choice([1, 2, 4, 8])), int(rng.integers(1, 12))
    c = Cache(torch, seqs, 30, int(rng.integers(20, 150)), page, seed=seed,
              dtype=["float16", "float32"][seed % 2]).to_device()
    for _ in range(15):
        source = rng.integers(-1, seqs, seqs)
        source[rng.random(seqs) < 0.6] = -7
        room = rng.integers(0, 20, seqs)
        c.update(None if rng.random() < 0.3 else source, room)
        depth = int(rng.integers(1, 7))
        kept = np.cumsum(rng.integers(1, 4, (seqs, depth)), 1) - rng.integers(0, 2)
        c.keep(kept, rng.integers(-1, depth + 2, seqs), release=bool(rng.random() < 0.7))
        assert (c.refs >= 0).all()
        count = np.bincount(np.concatenate([c.table[s, :c.held[s]] for s in range(seqs)] or [[]])
                            .astype(int), minlength=len(c.refs))
        assert np.array_equal(count, c.refs)


@pytest.mark.parametrize("seqs,n_pages", [(300, 3000), (1500, 20000), (4096, 9000)])
def test_many_sequences(seqs, n_pages):
    rng = np.random.default_rng(seqs)
    most = 4
    c = Cache(_torch(), seqs, most, n_pages, 2, shape=(1, 1, 4), seed=1)
    c.fill(rng.integers(0, 2 * min(most, n_pages // seqs // 1), seqs).clip(0, 3)).to_device()
    source = rng.integers(-1, seqs, seqs)
    c.update(source, rng.integers(0, 5, seqs))
    c.update(rng.permutation(seqs), rng.integers(0, 3, seqs))


def test_many_pages():
    """Free pages far up, and more of them than a walk's step."""
    torch = _torch()
    c = Cache(torch, 3, 40000, 100000, 1, shape=(1, 1, 2))
    c.refs[:30001] = 1
    c.refs[50000:60000] = 2
    c.to_device()
    c.refs = c.refs.copy()
    assert c.update(room=[17000, 1, 30000]).all()
    assert c.table[0, 0] == 30001
    c.update([1, 2, 0], [0, 0, 30000])


@pytest.mark.parametrize("first", [0, 16383, 16384, 16385, 40000, 99990])
def test_the_first_free_page_far_up(first):
    """None free in a walk's first steps, a few in a later one."""
    torch = _torch()
    c = Cache(torch, 3, 8, 100000, 1, shape=(1, 1, 2))
    c.refs[:first] = 1
    c.to_device()
    c.refs = c.refs.copy()
    assert c.update(room=[2, 1, 3]).all()
    assert c.table[0, 0] == first and c.table[2, 2] == first + 5
    c.update([0, 0, 1], [1, 0, 0])


def test_kept_rows():
    torch = _torch()
    for apart, release in ((False, True), (False, False), (True, False), (True, True)):
        c = Cache(torch, 7, 12, 80, 4, seed=3).fill([5, 0, 7, 8, 1, 3, 2], room=9).to_device()
        c.keep([[0, 1, 2], [2, 5, 7], [0, 3, 4], [8, 9, 10], [1, 1, 2], [3, 2, 4], [0, 0, 7]],
               [3, 3, 2, 3, 3, 3, -4], release, apart)
    c = Cache(torch, 2, 60, 130, 4, seed=4).fill([9, 10], room=200).to_device()
    c.keep(np.stack([np.arange(1, 180), np.arange(0, 179) + (np.arange(179) > 64)]))
    c = Cache(torch, 2, 60, 130, 4, seed=4).fill([9, 10], room=200).to_device()
    kept = np.stack([np.arange(0, 360, 2), np.arange(3, 183)])
    c.keep(kept)                                       # ends where the room ends
    c.keep(np.zeros((2, 0), np.int32))


@pytest.mark.parametrize("shape,dtype", [((3, 4, 128), "float16"), ((2, 3, 36), "float16"),
                                         ((2, 3, 7), "float16"), ((1, 5, 3), "float32"),
                                         ((2, 1, 256), "float32"), ((1, 16, 200), "float32")])
def test_rows_of_every_width(shape, dtype):
    torch = _torch()
    c = Cache(torch, 4, 6, 30, 8, shape, dtype, seed=5).fill([20, 9, 0, 3], room=12).to_device()
    c.update([0, 0, 1, 0], [12] * 4)
    c.keep([[0, 2, 5], [1, 2, 3], [4, 9, 11], [0, 1, 9]])


def test_layouts():
    """Head-major layers, keys and values side by side, rows apart."""
    torch = _torch()
    for how in ("heads", "pairs", "columns", "apart"):
        c = Cache(torch, 4, 6, 30, 8, (2, 3, 16), seed=6).fill([20, 9, 0, 3], room=12).to_device()
        L, S, H, hd = c.dk.shape
        if how == "heads":
            k, v = (torch.empty((L, H, S, hd), dtype=c.dtype, device="cuda").transpose(1, 2)
                    for _ in "kv")
        elif how == "pairs":
            both = torch.empty((L, 2, S, H, hd), dtype=c.dtype, device="cuda")
            k, v = both[:, 0], both[:, 1]
        elif how == "columns":
            both = torch.empty((L, S, 2, H, hd), dtype=c.dtype, device="cuda")
            k, v = both[:, :, 0], both[:, :, 1]
        else:
            k, v = (torch.empty((L, S, H, hd + 3), dtype=c.dtype, device="cuda")[..., :hd]
                    for _ in "kv")
        k.copy_(c.dk)
        v.copy_(c.dv)
        c.dk, c.dv = k, v
        c.same = lambda self=c: (setattr(self, "dk", k.contiguous()),
                                 setattr(self, "dv", v.contiguous()), Cache.same(self))
        c.update([0, 0, 1, 0], [12] * 4, k=k, v=v)
        c.keep([[0, 2, 5], [1, 2, 3], [4, 9, 11], [0, 1, 9]], k=k, v=v)


def test_slots_far_apart():
    """Offsets that pass 2^31 elements."""
    torch = _torch()
    c = Cache(torch, 3, 4, 12, 8, (1, 2, 8), seed=7).fill([20, 9, 3], room=8).to_device()
    stride = 30_000_000
    S = c.dk.shape[1]
    assert (S - 1) * stride > 2 ** 31
    far = torch.empty((S - 1) * stride + 64, dtype=c.dtype, device="cuda")
    k = far.as_strided((1, S, 2, 8), (1 << 40, stride, 8, 1))
    v = far.as_strided((1, S, 2, 8), (1 << 40, stride, 8, 1), 32)
    k.copy_(c.dk)
    v.copy_(c.dv)
    c.same = lambda: (setattr(c, "dk", k.contiguous()), setattr(c, "dv", v.contiguous()),
                      Cache.same(c))
    c.update([2, 0, 0], [8, 8, 8], k=k, v=v)
    c.keep([[0, 2], [1, 2], [4, 7]], k=k, v=v)


def test_tables_that_hold_nonsense():
    """Entries, lengths and counts out of range: nothing past the arrays is touched."""
    torch = _torch()
    c = Cache(torch, 4, 4, 10, 4, seed=8).fill([6, 3, 9, 2]).to_device()
    p = c.pages
    p.table[0, 0], p.table[0, 1], p.table[2, 2] = -5, 10, 2 ** 31 - 1
    p.len[1], p.held[3], p.len[3] = 10 ** 9, 99, -4
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    guard = p.table.clone()
    c.B.pages_update(p, i32([0, 0, 0, 1]), i32([3, 3, 3, 3]), c.dk, c.dv)
    c.B.pages_keep(p, i32([[0, 1], [0, 2], [2, 3], [0, 5]]), None, c.dk, c.dv)
    torch.cuda.synchronize()
    assert p.table.shape == guard.shape and bool((p.held >= 0).all()) and bool((p.held <= 4).all())


def test_captured_streams_and_dropped_inputs():
    torch = _torch()
    c = Cache(torch, 6, 40, 300, 4, seed=9).fill([9, 30, 2, 7, 0, 13], room=4).to_device()
    B, p = c.B, c.pages
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    source, room, kept, n_kept, ok = i32(6), i32(6), i32((6, 3)), i32(6), i32(6)
    ws = torch.empty(B.load_library().vsr_pages_update_workspace_size(6), dtype=torch.uint8,
                     device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pages_update(p, source, room, c.dk, c.dv, ok=ok, workspace=ws)
        B.pages_keep(p, kept, n_kept, c.dk, c.dv)
    rng = np.random.default_rng(1)
    for _ in range(4):
        hs, hr = rng.integers(-1, 6, 6), rng.integers(0, 9, 6)
        hk, hn = np.cumsum(rng.integers(1, 3, (6, 3)), 1) - 1, rng.integers(0, 4, 6)
        for to, x in ((source, hs), (room, hr), (kept, hk), (n_kept, hn)):
            to.copy_(torch.tensor(x.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        want = PT.pages_update(c.table, c.len, c.held, c.refs, 4, hs, hr, c.k, c.v)
        c.len[:] = PT.pages_keep(c.table, c.len, c.held, c.refs, 4, hk, hn, c.k, c.v, True)
        assert np.array_equal(ok.cpu().numpy(), want)
        c.same()
    side = torch.cuda.Stream()
    busy = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(10):
            torch.mm(busy, busy)
    src, more = torch.tensor([1, 1, 2, 2, 0, 0], dtype=torch.int32, device="cuda"), i32(6) + 5
    torch.cuda.synchronize()
    B.pages_update(p, src, more, c.dk, c.dv, stream=side)
    del src, more
    other = [torch.full((6,), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    PT.pages_update(c.table, c.len, c.held, c.refs, 4, np.array([1, 1, 2, 2, 0, 0]),
                    np.full(6, 5), c.k, c.v)
    c.same()
    assert len(other) == 2
