"""Arrays of the paged operators that meet each other are refused: results and workspaces
inside queries, keys, values and caches, at their first bytes, in the middle and at their
last. The pointers are never dereferenced: every call here is refused."""
import ctypes
import os

import pytest

from paper_2601_01513_amd import binding as B

MB = 1 << 20


def _lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libvsr.so not built (python -m paper_2601_01513_amd.build)")
    return B.load_library()


PAGES = dict(n_seqs=4, n_pages=100, page_size=16, max_pages=10, table=MB, table_stride=10,
             len=MB + 4096, held=MB + 4160, refs=MB + 8192)
SLOTS = 1600


def _refused(name, rc, word):
    assert rc == B.VSR_EINVAL
    msg = _lib().vsr_last_error(None).decode()
    assert msg.startswith(name + ": ") and word in msg, msg


def _attend(**kw):
    h = lambda p, n, ts, hs: B.VsrHeads(p, n, ts, hs)  # noqa: E731
    a = dict(q=h(64 * MB, 8, 512, 64), k=h(128 * MB, 2, 128, 64), v=h(192 * MB, 2, 128, 64),
             out=h(256 * MB, 8, 512, 64), mask=8 * MB, lse=10 * MB, ws=320 * MB, start=2 * MB)
    a.update({k: v for k, v in kw.items() if k in a})
    p = B.VsrPages(**{**PAGES, **{k: v for k, v in kw.items() if k in PAGES}})
    ref = ctypes.byref
    return _lib().vsr_tree_attention(ref(p), B.VSR_BF16, 64, 30, a["start"], ref(a["q"]), ref(a["k"]),
                                     ref(a["v"]), a["mask"], 2, 2, 0.1, ref(a["out"]), a["lse"],
                                     a["ws"], 1 << 40, None)


Q, KV = 30 * 512 * 2, SLOTS * 128 * 2     # bytes
LSE = 30 * 8 * 4


@pytest.mark.parametrize("base,size,word", [(64 * MB, Q, "lse or workspace"), (128 * MB, KV, "lse or workspace"),
                                            (192 * MB, KV, "lse or workspace"),
                                            (256 * MB, Q, "out overlaps lse or the workspace")])
def test_results_and_workspaces_inside_heads(base, size, word):
    for at in (0, 4, size // 2 // 4 * 4, size - 4):
        _refused("tree_attention", _attend(lse=base + at), word)
    _refused("tree_attention", _attend(lse=base - LSE + 4), word)
    for at in (0, 256, size // 2 // 256 * 256, (size - 1) // 256 * 256):
        _refused("tree_attention", _attend(ws=base + at), word)
    _refused("tree_attention", _attend(ws=base - 256), word)


@pytest.mark.parametrize("kw", [dict(table=256 * MB), dict(table=256 * MB - 156), dict(len=256 * MB + 64),
                                dict(held=256 * MB + Q - 4), dict(start=256 * MB + 1000), dict(mask=256 * MB),
                                dict(mask=256 * MB - 4), dict(table=256 * MB + Q - 4)])
def test_results_over_tables_and_masks(kw):
    _refused("tree_attention", _attend(**kw), "out overlaps an input")


def test_layouts_of_heads():
    """Head-major rows, gaps too small for what lies in them, broadcast and crossed strides."""
    h = lambda p, n, ts, hs: B.VsrHeads(p, n, ts, hs)  # noqa: E731
    far = h(128 * MB, 2, 1024, 64)                       # 896 elements between slots
    for at in (128 * 2 - 4, 1024 * 2 - LSE + 4, 1024 * 2, 1024 * 2 * 7 + 100, 1024 * 2 * 1599 + 252):
        _refused("tree_attention", _attend(k=far, lse=128 * MB + at), "lse or workspace")
    heads = h(128 * MB, 2, 64, 64 * 1700)                # 100 slots' room between heads
    for at in (0, 64 * 1600 * 2 - 4, 64 * 1700 * 2 - LSE + 4, 64 * 1700 * 2 + 64 * 1600 * 2 - 4):
        _refused("tree_attention", _attend(v=heads, lse=128 * MB + at), "lse or workspace")
    for crossed in (h(128 * MB, 2, 128, 96), h(128 * MB, 2, 0, 64), h(128 * MB, 2, 128, 0)):
        _refused("tree_attention", _attend(k=crossed, lse=128 * MB + 64), "lse or workspace")


CACHE = dict(k=64 * MB, v=128 * MB, dtype=B.VSR_F16, n_layers=2, n_heads=2, head_dim=64,
             layer_stride=SLOTS * 128, slot_stride=128, head_stride=64)


def _update(cache={}, **kw):
    lib = _lib()
    a = dict(source=2 * MB, room=2 * MB + 64, ok=2 * MB + 128, ws=3 * MB)
    a.update({k: v for k, v in kw.items() if k in a})
    p = B.VsrPages(**{**PAGES, **{k: v for k, v in kw.items() if k in PAGES}})
    return lib.vsr_pages_update(ctypes.byref(p), a["source"], a["room"],
                                ctypes.byref(B.VsrCache(**{**CACHE, **cache})), a["ok"], a["ws"],
                                lib.vsr_pages_update_workspace_size(4), None)


def _keep(cache={}, **kw):
    a = dict(kept=2 * MB, n_kept=2 * MB + 512, out=2 * MB + 1024)
    a.update({k: v for k, v in kw.items() if k in a})
    p = B.VsrPages(**{**PAGES, **{k: v for k, v in kw.items() if k in PAGES}})
    return _lib().vsr_pages_keep(ctypes.byref(p), a["kept"], 5, 5, a["n_kept"],
                                 ctypes.byref(B.VsrCache(**{**CACHE, **cache})), a["out"], 1, None)


@pytest.mark.parametrize("base", [64 * MB, 128 * MB])
def test_caches(base):
    size = 2 * KV
    for at in (0, 64, KV - 16, KV, size // 2 + 4096, size - 16):
        for what in ("table", "len", "held", "refs", "source", "room", "ok"):
            _refused("pages_update", _update(**{what: base + at}), "cache overlaps another")
        _refused("pages_update", _update(ws=base + at), "cache overlaps the workspace")
        for what in ("table", "len", "held", "refs", "kept", "n_kept", "out"):
            _refused("pages_keep", _keep(**{what: base + at}), "cache overlaps another")
    for what in ("table", "len", "refs"):
        _refused("pages_update", _update(**{what: base - 4}), "cache overlaps another")
    # Rows apart: a list that does not fit between two of them.
    cache = dict(layer_stride=SLOTS * 160, slot_stride=160)
    for at in (128 * 2 - 4, 160 * 2 - 12, 160 * 2 * 1599 + 200, SLOTS * 320 + 160 * 2 * 5):
        _refused("pages_update", _update(cache, room=base + at), "cache overlaps another")
        _refused("pages_keep", _keep(cache, kept=base + at), "cache overlaps another")
