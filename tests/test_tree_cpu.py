"""Refusals of the paged-cache operators: every check runs before the device is touched,
so the pointers below are never dereferenced; calls that pass have nothing to do."""
import contextlib
import ctypes
import os

import numpy as np
import pytest

import plain_tree as PT
from paper_2601_01513_amd import binding as B


def _lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libvsr.so not built (python -m paper_2601_01513_amd.build)")
    return B.load_library()


MB = 1 << 20


def _pages(**kw):
    a = dict(n_seqs=4, n_pages=100, page_size=16, max_pages=10, table=MB, table_stride=10,
             len=MB + 4096, held=MB + 4160, refs=MB + 8192)
    a.update({k: v for k, v in kw.items() if k in a})
    return B.VsrPages(**a)


BAD_PAGES = [
    (dict(n_seqs=0), "n_seqs"), (dict(n_seqs=4097), "n_seqs"), (dict(page_size=0), "page_size"),
    (dict(page_size=24), "page_size"), (dict(page_size=-16), "page_size"),
    (dict(n_pages=0), "n_pages"), (dict(n_pages=1 << 27), "n_pages"),
    (dict(max_pages=0), "max_pages"), (dict(max_pages=1 << 27, table_stride=1 << 27), "max_pages"),
    (dict(table_stride=9), "table_stride"), (dict(table=None), "non-NULL"),
    (dict(len=None), "non-NULL"), (dict(held=None), "non-NULL"), (dict(table=MB + 2), "aligned"),
    (dict(held=MB + 4161), "aligned"),
]


def _message(name, rc, word):
    assert rc == B.VSR_EINVAL
    msg = _lib().vsr_last_error(None).decode()
    assert word in msg and msg.startswith(name + ": "), msg


def _rows(pages="own", **kw):
    a = dict(T=30, start=2 * MB, parent=2 * MB + 512, shift=2 * MB + 1024, pos=3 * MB,
             slot=3 * MB + 512, mask=3 * MB + 1024, stride=2, words=2)
    a.update({k: v for k, v in kw.items() if k in a})
    p = _pages(**kw) if pages == "own" else pages
    return _lib().vsr_tree_rows(ctypes.byref(p) if p else None, a["T"], a["start"], a["parent"],
                                a["shift"], a["pos"], a["slot"], a["mask"], a["stride"],
                                a["words"], None)


@pytest.mark.parametrize("kw,word", BAD_PAGES + [
    (dict(pages=None), "pages"), (dict(T=-1), "T must"), (dict(T=(1 << 24) + 1), "T must"),
    (dict(start=None), "without start"), (dict(start=2 * MB + 1), "aligned"),
    (dict(pos=None), "pos"), (dict(slot=None), "slot"), (dict(slot=3 * MB + 514), "slot"),
    (dict(words=0), "mask_words"), (dict(stride=1), "mask_stride"), (dict(mask=3 * MB + 1025), "mask"),
    (dict(pos=2 * MB + 512), "overlaps an input"), (dict(mask=MB + 32), "overlaps an input"),
    (dict(slot=3 * MB + 4), "overlap each other"), (dict(mask=3 * MB + 600), "overlap each other"),
])
def test_tree_rows_refuses(kw, word):
    _message("tree_rows", _rows(**kw), word)


def _attend(pages="own", **kw):
    lib = _lib()
    h = lambda p, n, ts, hs: B.VsrHeads(p, n, ts, hs)  # noqa: E731
    a = dict(dtype=B.VSR_BF16, hd=64, T=30, start=2 * MB, q=h(3 * MB, 8, 512, 64),
             k=h(4 * MB, 2, 128, 64), v=h(6 * MB, 2, 128, 64), mask=8 * MB, stride=2, words=2,
             scale=0.1, out=h(9 * MB, 8, 512, 64), lse=10 * MB, ws=11 * MB, wsb=1 << 40)
    a.update({k: v for k, v in kw.items() if k in a})
    p = _pages(**kw) if pages == "own" else pages
    ref = lambda s: ctypes.byref(s) if s is not None else None  # noqa: E731
    return lib.vsr_tree_attention(
        ref(p), a["dtype"], a["hd"], a["T"], a["start"], ref(a["q"]), ref(a["k"]), ref(a["v"]),
        a["mask"], a["stride"], a["words"], a["scale"], ref(a["out"]), a["lse"], a["ws"], a["wsb"],
        None)


def _h(p, n=8, ts=512, hs=64):
    return B.VsrHeads(p, n, ts, hs)


@pytest.mark.parametrize("kw,word", BAD_PAGES + [
    (dict(pages=None), "pages"), (dict(dtype=4), "dtype"), (dict(hd=0), "head_dim"),
    (dict(hd=257), "head_dim"), (dict(T=-1), "T must"), (dict(start=None), "without start"),
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(q=None), "non-NULL"), (dict(out=None), "non-NULL"), (dict(q=_h(None)), "non-NULL"),
    (dict(k=_h(4 * MB + 1, 2, 128)), "aligned"), (dict(q=_h(3 * MB, 7)), "differ"),
    (dict(v=_h(6 * MB, 1, 128)), "divides"), (dict(k=_h(4 * MB, 3, 192), v=_h(6 * MB, 3, 192)), "divides"),
    (dict(k=_h(4 * MB, 2, -1)), "strides"), (dict(k=_h(4 * MB, 2, 1 << 60)), "2^46"),
    (dict(out=_h(9 * MB, 8, 512, 63)), "themselves"), (dict(out=_h(9 * MB, 8, 511)), "themselves"),
    (dict(out=_h(3 * MB)), "overlaps q"), (dict(out=_h(4 * MB + 4096)), "overlaps k"),
    (dict(out=_h(6 * MB + 4096)), "overlaps v"), (dict(words=0), "mask_words"),
    (dict(stride=1), "mask_stride"), (dict(mask=8 * MB + 2), "mask"), (dict(lse=10 * MB + 2), "lse"),
    (dict(ws=None), "workspace"), (dict(ws=11 * MB + 128), "workspace"), (dict(wsb=4096), "smaller"),
    (dict(lse=8 * MB + 64), "lse or workspace"), (dict(lse=2 * MB), "lse or workspace"),
    (dict(ws=8 * MB), "lse or workspace"), (dict(lse=11 * MB + 512), "lse overlaps"),
])
def test_tree_attention_refuses(kw, word):
    _message("tree_attention", _attend(**kw), word)


def _cache(**kw):
    a = dict(k=16 * MB, v=32 * MB, dtype=B.VSR_F16, n_layers=2, n_heads=2, head_dim=64,
             layer_stride=1600 * 128, slot_stride=128, head_stride=64)
    a.update({x: v for x, v in kw.items() if x in a})
    return B.VsrCache(**a)


BAD_CACHES = [
    (dict(cache=None), "cache"), (dict(dtype=7), "dtype"), (dict(head_dim=0), "head_dim"),
    (dict(head_dim=300), "head_dim"), (dict(n_layers=0), "n_layers"), (dict(n_layers=4097), "n_layers"),
    (dict(k=None), "non-NULL"), (dict(v=32 * MB + 1), "aligned"), (dict(n_heads=0), "n_heads"),
    (dict(slot_stride=127), "themselves"), (dict(head_stride=63), "themselves"),
    (dict(slot_stride=-128), "strides"), (dict(layer_stride=1600 * 128 - 1), "layer_stride"),
    (dict(layer_stride=1 << 60), "2^46"), (dict(v=16 * MB), "k overlaps v"),
    (dict(v=16 * MB + 4096), "k overlaps v"),
    (dict(v=16 * MB + 2 * 1600 * 128), "k overlaps v"),            # the second layer's keys
    (dict(k=32 * MB + 2 * 1600 * 128 + 512), "k overlaps v"),
]


def _update(pages="own", cache="own", **kw):
    lib = _lib()
    a = dict(source=2 * MB, room=2 * MB + 64, ok=2 * MB + 128, ws=3 * MB,
             wsb=lib.vsr_pages_update_workspace_size(4))
    a.update({k: v for k, v in kw.items() if k in a})
    p, c = _pages(**kw) if pages == "own" else pages, _cache(**kw) if cache == "own" else cache
    ref = lambda s: ctypes.byref(s) if s is not None else None  # noqa: E731
    return lib.vsr_pages_update(ref(p), a["source"], a["room"], ref(c), a["ok"], a["ws"], a["wsb"],
                                None)


@pytest.mark.parametrize("kw,word", BAD_PAGES + BAD_CACHES + [
    (dict(pages=None), "pages"), (dict(refs=None), "non-NULL"), (dict(source=2 * MB + 1), "aligned"),
    (dict(ok=2 * MB + 130), "aligned"), (dict(room=2 * MB), "overlap"), (dict(ok=MB + 4096), "overlap"),
    (dict(source=MB + 8), "overlap"), (dict(room=MB + 8192 + 396), "overlap"), (dict(len=MB + 156), "overlap"),
    (dict(ws=None), "workspace"), (dict(ws=3 * MB + 8), "workspace"), (dict(wsb=79), "smaller"),
    (dict(ws=MB + 8192), "workspace overlaps"), (dict(ws=2 * MB), "workspace overlaps"),
])
def test_pages_update_refuses(kw, word):
    _message("pages_update", _update(**kw), word)


def _keep(pages="own", cache="own", **kw):
    a = dict(kept=2 * MB, stride=5, most=5, n_kept=2 * MB + 512, out=2 * MB + 1024, release=1)
    a.update({k: v for k, v in kw.items() if k in a})
    p, c = _pages(**kw) if pages == "own" else pages, _cache(**kw) if cache == "own" else cache
    ref = lambda s: ctypes.byref(s) if s is not None else None  # noqa: E731
    return _lib().vsr_pages_keep(ref(p), a["kept"], a["stride"], a["most"], a["n_kept"], ref(c),
                                 a["out"], a["release"], None)


@pytest.mark.parametrize("kw,word", BAD_PAGES + BAD_CACHES + [
    (dict(pages=None), "pages"), (dict(refs=None), "non-NULL"), (dict(most=-1), "max_kept"),
    (dict(most=(1 << 20) + 1, stride=1 << 21), "max_kept"), (dict(kept=None), "kept"),
    (dict(stride=4), "kept_stride"), (dict(out=None), "len_out"), (dict(kept=2 * MB + 2), "aligned"),
    (dict(n_kept=2 * MB + 76), "overlap"), (dict(out=2 * MB + 516), "overlap"),
    (dict(out=MB + 4100), "overlap"), (dict(kept=MB + 100), "overlap"),
])
def test_pages_keep_refuses(kw, word):
    _message("pages_keep", _keep(**kw), word)


def test_page_workspaces():
    lib = _lib()
    assert [lib.vsr_pages_update_workspace_size(n) for n in (0, -1, 4097)] == [0] * 3
    assert 16 < lib.vsr_pages_update_workspace_size(4096) < 1 << 18


def test_nothing_to_do_and_sizes():
    lib = _lib()
    assert _rows(T=0, pos=None, slot=None) == B.VSR_OK
    assert _attend(T=0, ws=None, wsb=0) == B.VSR_OK
    size = lib.vsr_tree_attention_workspace_size
    assert 0 < size(B.VSR_BF16, 128, 512, 8, 28, 4) < 1 << 28
    for bad in ((3, 128, 1, 1, 1, 1), (1, 0, 1, 1, 1, 1), (1, 257, 1, 1, 1, 1), (1, 64, -1, 1, 1, 1),
                (1, 64, 1, 0, 1, 1), (1, 64, 1, 4097, 1, 1), (1, 64, 1, 1, 3, 2), (1, 64, 1, 1, 0, 1)):
        assert size(*bad) == 0


def _tables(torch, seqs=3, most=5, n_pages=20):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    return dict(table=i32(seqs, most), len=i32(seqs), held=i32(seqs), refs=i32(n_pages))


def test_the_binding_refuses_what_the_library_cannot_see():
    torch = pytest.importorskip("torch")
    _lib()
    t = _tables(torch)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    p = B.pages(**t, page_size=8)
    q, k = torch.zeros(4, 2, 8), torch.zeros(160, 1, 8)
    start, kv = i32(4), torch.zeros(2, 160, 1, 8)
    att = lambda **kw: lambda: B.tree_attention(p, **dict(dict(q=q, k=k, v=k, scale=1.0, start=start), **kw))  # noqa: E731
    bad = [lambda kw=kw: B.pages(**dict(dict(t, page_size=8), **kw)) for kw in (
        dict(table=i32(3, 5).long()), dict(table=i32(5)), dict(table=i32(5, 3).t()), dict(len=i32(2)),
        dict(held=i32(3).long()), dict(len=i32(6)[::2]), dict(refs=i32(4, 5)), dict(refs=i32(20).float()))]
    bad += [lambda: B.tree_rows(p, i32(3), i32(4)), lambda: B.tree_rows(p, start, i32(4).long()),
            lambda: B.tree_rows(p, start), lambda: B.tree_rows(p, start, i32(4), i32(4)),
            lambda: B.tree_rows(p, start, i32(4), out=(i32(4), i32(5), None)),
            lambda: B.tree_rows(p, start, i32(4), out=(i32(4), i32(4), i32(3, 1))),
            lambda: B.tree_rows(p, start, i32(4)),               # host tensors
            att(), att(q=q.double()), att(q=q[0]), att(k=k.half()), att(k=k[:159]), att(v=k[:, :, :4]),
            lambda: B.pages_update(p, i32(3)), lambda: B.pages_update(p, i32(2), k=kv, v=kv),
            lambda: B.pages_update(p, room=i32(3).long()), lambda: B.pages_update(p, room=i32(3)),
            lambda: B.pages_update(p, i32(3), k=kv, v=kv[:, :, :, ::2]),
            lambda: B.pages_update(p, i32(3), k=kv[0], v=kv[0]),
            lambda: B.pages_update(p, i32(3), k=kv[:, :99], v=kv[:, :99]),
            lambda: B.pages_update(p, i32(3), k=kv, v=kv, ok=i32(4)),
            lambda: B.pages_keep(p, i32(2, 4), None, kv, kv), lambda: B.pages_keep(p, i32(3), None, kv, kv),
            lambda: B.pages_keep(p, i32(4, 3).t(), None, kv, kv),
            lambda: B.pages_keep(p, i32(3, 4), i32(4), kv, kv),
            lambda: B.pages_keep(p, i32(3, 4), None, kv, kv.half()),
            lambda: B.pages_keep(p, i32(3, 4), None, kv, kv, i32(2)),
            lambda: B.pages_keep(p, i32(3, 4), None, kv, kv),      # host tensors
            att(start=i32(5)), att(start=start.long()), att(mask=i32(3, 1)), att(mask=i32(4, 1).long()),
            att(mask=i32(2, 4).t()), att(out=q[:3]), att(out=q.half()), att(lse=torch.zeros(4, 3)),
            att(lse=torch.zeros(2, 4).t()), att(q=q.transpose(1, 2))]
    for i, f in enumerate(bad):
        with pytest.raises(B.VsrError) as e:
            f()
        assert e.value.code == B.VSR_EINVAL, i


class _Fine:
    """A library whose calls all succeed and whose sizes are 64."""

    def __getattr__(self, name):
        return lambda *a: 64 if name.endswith("size") else 0


def test_calls_on_a_given_stream_hold_their_tensors(monkeypatch):
    torch = pytest.importorskip("torch")
    seen = []
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    monkeypatch.setattr(B, "_hold", lambda stream, *ts: seen.append((stream, ts)))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    B._torch_names()
    for name, value in (("_lib", _Fine()), ("_device_now", lambda: 0), ("_raw_stream", lambda d: 0)):
        monkeypatch.setattr(B, name, value)
    stream = type("Stream", (), {"device_index": 0, "cuda_stream": 0})()
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    p = B.pages(**_tables(torch), page_size=4)
    tables = [p.table, p.len, p.held, p.refs]
    q, k, v = torch.ones(6, 4, 8), torch.ones(80, 2, 8), torch.ones(80, 2, 8)
    k4, v4 = torch.ones(2, 80, 2, 8), torch.ones(2, 80, 2, 8)
    start, parent, shift, mask = i32(4), i32(6), i32(3), i32(6, 1)
    rows, ws = (i32(6), i32(6), i32(6, 1)), torch.ones(64, dtype=torch.uint8)
    out, lse, source, room, ok = torch.ones(6, 4, 8), torch.ones(6, 4), i32(3), i32(3), i32(3)
    kept, n_kept, length = i32(3, 2), i32(3), i32(3)
    x, ids = torch.ones(3, 100), i32(3)
    lp = torch.ones(3), i32(3), torch.ones(3), i32(3, 2), torch.ones(3, 2)
    calls = [(lambda s: B.tree_rows(p, start, parent, shift, out=rows, stream=s),
              [*tables, start, parent, shift, *rows]),
             (lambda s: B.tree_attention(p, q, k, v, 1.0, start, mask, out, lse, ws, s),
              [*tables, q, k, v, start, mask, out, lse, ws]),
             (lambda s: B.pages_update(p, source, room, k4, v4, ok, ws, s),
              [*tables, source, room, k4, v4, ok, ws]),
             (lambda s: B.pages_keep(p, kept, n_kept, k4, v4, length, stream=s),
              [*tables, kept, n_kept, k4, v4, length]),
             (lambda s: B.token_logprobs(x, ids, 2, lp, ws, s), [x, ids, *lp, ws]),
             # What a call makes for itself is held too.
             (lambda s: B.tree_attention(p, q, k, v, 1.0, start, mask, stream=s),
              [*tables, q, k, v, start, mask])]
    for i, (call, tensors) in enumerate(calls):
        seen.clear()
        call(None)  # (the current stream's own order holds them)
        assert not seen, i
        call(stream)
        assert all(s is stream for s, _ in seen), i
        held = [id(t) for _, ts in seen for t in ts if t is not None]
        assert set(map(id, tensors)) <= set(held), i
        if i == len(calls) - 1:
            assert len(held) == len(tensors) + 2  # (the result and the workspace)


def test_plain_forms_by_hand():
    table = np.array([[3, 1, 0]])
    pos, slot, mask = PT.tree_rows(table, [5], [2], 4, [0, 4], np.array([-1, 0, 0, 2]), 4, 1)
    assert pos.tolist() == [5, 6, 6, 7] and slot.tolist() == [5, 6, 7, -1]
    assert mask[:, 0].tolist() == [1, 3, 5, 13]
    q, k = np.array([[[2.0]]]), np.zeros((16, 1, 1))
    k[[12, 13, 14], 0, 0] = [1, 1, 5]
    out, lse, _, _ = PT.attention(q, k, k, table, [2], [1], 4, None, np.array([[0]], np.uint32), 1.0)
    assert np.allclose(out, 1) and np.allclose(lse, 2 + np.log(2))
