"""Refusals of vsr_rope_axes, vsr_qk_norm_rope, vsr_pick_tokens and their context
calls: every check runs before the device is touched, so the pointers below are
never dereferenced. Calls that pass every check and have nothing to do return
VSR_OK; none here would launch."""
import ctypes
import os

import numpy as np
import pytest

import plain_decoder as PD
from paper_2601_01513_amd import binding as B
from paper_2601_01513_amd import workload as W


def _lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libvsr.so not built (python -m paper_2601_01513_amd.build)")
    return B.load_library()


MB = 1 << 20


def _heads(data, n, ts, hs):
    return B.VsrHeads(data, n, ts, hs)


def _rope(norm=False, **kw):
    """A good call of T = 10 tokens, 4 query and 2 key heads of 64 in bf16; kw
    changes it."""
    lib = _lib()
    a = dict(rot=B.rotary((16, 8, 8), 1e4), dtype=B.VSR_BF16, hd=64, T=10, pos=MB, pos_stride=10,
             qi=_heads(2 * MB, 4, 512, 64), qo=_heads(3 * MB, 4, 256, 64),
             ki=_heads(2 * MB + 512, 2, 512, 64), ko=_heads(4 * MB, 2, 64, 64 * 100),
             rows=5 * MB, cap=100, gq=6 * MB, gk=6 * MB + 512, gain_dtype=B.VSR_F32, eps=1e-6)
    a.update(kw)
    ref = lambda s: ctypes.byref(s) if s is not None else None  # noqa: E731
    tail = [ref(a[k]) for k in ("qi", "qo", "ki", "ko")] + [a["rows"], a["cap"], None]
    head = [ref(a["rot"]), a["dtype"], a["hd"], a["T"], a["pos"], a["pos_stride"]]
    if norm:
        return lib.vsr_qk_norm_rope(*head, a["gq"], a["gk"], a["gain_dtype"], a["eps"], *tail)
    return lib.vsr_rope_axes(*head, *tail)


def _scheme(n_axes, sections, base=1e4, interleaved=0):
    return B.VsrRotary(n_axes, (ctypes.c_int32 * 4)(*sections), interleaved, base)


@pytest.mark.parametrize("kw,word", [
    (dict(rot=None), "scheme"), (dict(rot=_scheme(0, (32,))), "n_axes"),
    (dict(rot=_scheme(5, (8, 8, 8, 8))), "n_axes"), (dict(rot=_scheme(2, (16, -1))), "sections"),
    (dict(rot=_scheme(1, (0,))), "no pair"), (dict(rot=_scheme(3, (16, 16, 16))), "head_dim"),
    (dict(rot=_scheme(1, (2 ** 31 - 1,))), "sections"),
    (dict(rot=_scheme(1, (32,), 0.0)), "base"), (dict(rot=_scheme(1, (32,), float("nan"))), "base"),
    (dict(rot=_scheme(1, (32,), float("inf"))), "base"),
    (dict(rot=_scheme(3, (8, 8, 16), 1e4, 1)), "interleaved"),
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(hd=63), "head_dim"),
    (dict(hd=0), "head_dim"), (dict(hd=258), "head_dim"), (dict(T=-1), "T must"),
    (dict(T=(1 << 30) + 1), "T must"), (dict(pos=None), "pos"), (dict(pos=MB + 2), "pos"),
    (dict(pos_stride=-1), "pos_stride"), (dict(qi=None), "together"), (dict(ko=None), "together"),
    (dict(ki=None), "together"), (dict(qi=_heads(None, 4, 512, 64)), "non-NULL"),
    (dict(qi=_heads(2 * MB + 1, 4, 512, 64)), "aligned"),
    (dict(qi=_heads(2 * MB, 0, 512, 64)), "n_heads"),
    (dict(qi=_heads(2 * MB, 4097, 512, 64)), "n_heads"),
    (dict(qi=_heads(2 * MB, 4, -512, 64)), "strides"),
    (dict(qi=_heads(2 * MB, 4, 1 << 60, 64)), "2^46"),
    (dict(qi=_heads(2 * MB, 3, 512, 64)), "n_heads"),
    (dict(qo=_heads(3 * MB, 4, 255, 64)), "themselves"),
    (dict(qo=_heads(3 * MB, 4, 256, 63)), "themselves"),
    (dict(qo=_heads(3 * MB, 4, 0, 64)), "themselves"),
    (dict(ko=_heads(4 * MB, 2, 64, 64 * 99)), "themselves"),
    (dict(rows=None, cap=9), "k_cap"), (dict(cap=0), "k_cap"), (dict(cap=1 << 31), "k_cap"),
    (dict(rows=5 * MB + 1), "k_rows"),
    (dict(qo=_heads(2 * MB + 64, 4, 512, 64)), "q_out overlaps q_in"),
    (dict(qo=_heads(2 * MB + 256, 4, 256, 64)), "q_out overlaps"),
    (dict(qo=_heads(2 * MB + 512, 4, 512, 64)), "q_out overlaps k_in"),
    (dict(ko=_heads(2 * MB + 512, 2, 512, 64)), "k_out overlaps k_in"),  # in place, but k_rows
    (dict(ko=_heads(2 * MB, 2, 512, 64), rows=None), "k_out overlaps q_in"),
    (dict(ko=_heads(3 * MB, 2, 64, 6400)), "k_out overlaps q_out"),
])
def test_rope_axes_refuses(kw, word):
    assert _rope(**kw) == B.VSR_EINVAL
    msg = _lib().vsr_last_error(None).decode()
    assert word in msg and msg.startswith("rope_axes: "), msg


@pytest.mark.parametrize("kw,word", [
    (dict(gq=None), "gains"), (dict(gk=None), "gains"), (dict(gq=6 * MB + 2), "gains"),
    (dict(gain_dtype=5), "gain_dtype"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(eps=float("inf")), "eps"), (dict(hd=62), "head_dim"),
])
def test_qk_norm_rope_refuses(kw, word):
    assert _rope(norm=True, **kw) == B.VSR_EINVAL
    msg = _lib().vsr_last_error(None).decode()
    assert word in msg and msg.startswith("qk_norm_rope: "), msg


def test_no_tokens_is_no_work():
    assert _rope(T=0, pos=None) == B.VSR_OK
    assert _rope(norm=True, T=0, qi=_heads(None, 4, 0, 0)) == B.VSR_OK


def _pick(**kw):
    lib = _lib()
    a = dict(logits=MB, dtype=B.VSR_F32, rows=4, vocab=1000, stride=1000, processed=None,
             processed_stride=0, token=8 * MB, logprob=8 * MB + 64, ws=9 * MB,
             wsb=lib.vsr_pick_workspace_size(4, 1000))
    rules = B.VsrTokenRules(2 * MB, 2 * MB + 64, 2 * MB + 128, 3 * MB, 0, 4 * MB, 32)
    lists = B.VsrTokenLists(5 * MB, 16, 16, 5 * MB + 1024, 6 * MB, 8, 8, None)
    for k, v in kw.items():
        if k in a:
            a[k] = v
        else:
            setattr(rules if hasattr(rules, k) else lists, k, v)
    return lib.vsr_pick_tokens(a["logits"], a["dtype"], a["rows"], a["vocab"], a["stride"],
                               ctypes.byref(lists), ctypes.byref(rules), a["processed"],
                               a["processed_stride"], a["token"], a["logprob"], a["ws"], a["wsb"],
                               None)


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=9), "dtype"), (dict(rows=-1), "rows"), (dict(rows=65536), "rows"),
    (dict(vocab=0), "vocab"), (dict(vocab=(1 << 24) + 1), "vocab"), (dict(logits=None), "NULL"),
    (dict(token=None), "NULL"), (dict(ws=None), "NULL"), (dict(logits=MB + 2), "logits"),
    (dict(token=8 * MB + 1), "outputs"), (dict(logprob=8 * MB + 2), "outputs"),
    (dict(stride=999), "stride"), (dict(bias_stride=999), "bias_stride"),
    (dict(bias_stride=-4), "bias_stride"), (dict(mask_stride=31), "mask_stride"),
    (dict(repetition=2 * MB + 2), "rules"), (dict(mask=4 * MB + 1), "rules"),
    (dict(processed=7 * MB, processed_stride=999), "processed_stride"),
    (dict(processed=MB + 400, processed_stride=1000), "overlaps"),
    (dict(processed=MB, processed_stride=1004), "overlaps"),
    (dict(processed=MB, processed_stride=1000, dtype=B.VSR_F16), "overlaps"),
    (dict(n_prompt=-1), "list"), (dict(n_output=(1 << 30) + 1), "list"), (dict(output_stride=-8), "list"), (dict(prompt=5 * MB + 2), "lists"),
    (dict(prompt_len=5 * MB + 1), "lists"), (dict(ws=9 * MB + 8), "workspace"), (dict(wsb=47), "smaller"),
])
def test_pick_tokens_refuses(kw, word):
    assert _pick(**kw) == B.VSR_EINVAL
    msg = _lib().vsr_last_error(None).decode()
    assert word in msg and msg.startswith("pick_tokens: "), msg


def test_pick_sizes():
    lib = _lib()
    assert _pick(rows=0, logits=None, token=None, ws=None, wsb=0) == B.VSR_OK
    assert lib.vsr_pick_workspace_size(1, 1) > 0
    assert lib.vsr_pick_workspace_size(256, 152064) < 1 << 20
    for rows, vocab in ((0, 10), (65536, 10), (1, 0), (1, (1 << 24) + 1), (-1, 10)):
        assert lib.vsr_pick_workspace_size(rows, vocab) == 0


def test_context_calls_without_a_context():
    lib = _lib()
    rot = B.rotary((64,), 1e6)
    assert lib.vsr_set_positions(None, ctypes.byref(rot), MB, 10, 10, 10) == B.VSR_EINVAL
    assert lib.vsr_load_qk_norms(None, None, None) == B.VSR_EINVAL
    lens = (ctypes.c_int32 * 1)(1)
    assert lib.vsr_draft_ruled(None, MB, lens, 1, 1, 1, None, 0, MB, None, MB, 1) == B.VSR_EINVAL
    c = B.make_config(W.DRAFT_3B, max_new=64)
    n = lib.vsr_draft_ruled_workspace_size(ctypes.byref(c), 3)
    assert 3 * W.DRAFT_3B.vocab * 4 <= n <= 3 * W.DRAFT_3B.vocab * 4 + (1 << 16)
    for m in (0, 4):
        assert lib.vsr_draft_ruled_workspace_size(ctypes.byref(c), m) == 0
    assert lib.vsr_draft_ruled_workspace_size(None, 1) == 0


def test_the_binding_refuses_what_the_library_cannot_see():
    torch = pytest.importorskip("torch")
    _lib()
    q, k = torch.zeros(4, 2, 8), torch.zeros(4, 1, 8)
    pos, rot = torch.zeros(2, 4, dtype=torch.int32), B.rotary((2, 2), 1e4)
    bad = [
        lambda: B.rotary((), 1e4), lambda: B.rotary((1, 1, 1, 1, 1), 1e4),
        lambda: B.rope_axes(rot, pos.long(), q), lambda: B.rope_axes(rot, pos[:1], q),
        lambda: B.rope_axes(rot, pos[:, :3], q), lambda: B.rope_axes(rot, pos, q.double()),
        lambda: B.rope_axes(rot, pos, q[0]), lambda: B.rope_axes(rot, pos, q, k.half()),
        lambda: B.rope_axes(rot, pos, q, k[:3]), lambda: B.rope_axes(rot, pos, q, q_out=q[:, :1]),
        lambda: B.rope_axes(rot, pos, q.transpose(1, 2)), lambda: B.rope_axes(rot, pos, q, k_out=k),
        lambda: B.rope_axes(rot, pos, q, k, k_rows=torch.zeros(4, dtype=torch.int32)),
        lambda: B.rope_axes(rot, pos, q, k, k_out=k.clone(), k_rows=torch.zeros(3, dtype=torch.int32)),
        lambda: B.rope_axes(rot, pos, q),                       # host tensors
        lambda: B.qk_norm_rope(rot, pos, q, k, torch.ones(8), None, 1e-6),
        lambda: B.qk_norm_rope(rot, pos, q, k, torch.ones(8), torch.ones(7), 1e-6),
        lambda: B.qk_norm_rope(rot, pos, q, k, torch.ones(8), torch.ones(8).half(), 1e-6),
    ]
    x = torch.zeros(3, 100)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    bad += [lambda kw=kw: B.pick_tokens(x, **kw) for kw in (
        dict(), dict(prompt=i32(2, 5)), dict(prompt=i32(3, 5).long()), dict(output=i32(3)),
        dict(prompt=i32(3, 5), prompt_len=i32(2)), dict(repetition=torch.ones(2)),
        dict(presence=torch.ones(3).half()), dict(bias=torch.zeros(2, 100)),
        dict(bias=torch.zeros(3, 99)), dict(mask=i32(1, 3)), dict(mask=i32(3, 4).long()),
        dict(processed=torch.zeros(3, 99)), dict(processed=torch.zeros(3, 100).half()),
        dict(out=(i32(2), torch.zeros(3))), dict(out=(i32(3), torch.zeros(3).half())))]
    bad += [lambda: B.pick_tokens(x.double()), lambda: B.pick_tokens(x[0])]
    for i, f in enumerate(bad):
        with pytest.raises(B.VsrError) as e:
            f()
        assert e.value.code == B.VSR_EINVAL, i


def test_a_stream_of_another_device_is_refused():
    """Before anything is launched on it."""
    torch = pytest.importorskip("torch")
    stream, calls = type("Stream", (), {"device_index": 1, "cuda_stream": 0})(), []
    with pytest.raises(B.VsrError) as e:
        B._call(torch, 0, stream, lambda *a: calls.append(a), ())
    assert e.value.code == B.VSR_EINVAL and "stream" in str(e.value) and not calls


def test_plain_forms_by_hand():
    """The comparison's own pieces: axes of pairs, a quarter turn, the rules."""
    assert list(PD.axis_of_pair((2, 1, 1), False)) == [0, 0, 1, 2]
    assert list(PD.axis_of_pair((24, 20, 20), True)) == \
        [(0, 1, 2)[i % 3] if i < 60 else 0 for i in range(64)]
    x = np.array([[[1.0, 0.0, 7.0]]])
    y = PD.rope(x, np.array([[1]]), np.array([0]), 1e4)
    assert np.allclose(y, [[[np.cos(1), np.sin(1), 7.0]]])
    l = np.array([2.0, -2.0, 1.0, 4.0, 0.0], np.float32)
    y = PD.apply_rules(l, [0, -1, 9], [1, 1, 3], 2.0, 0.5, 0.25, np.full(5, 1.0, np.float32),
                       np.array([0b01111], np.uint32))
    assert np.array_equal(y, np.array([2.0, -4.0, 2.0, 2.25, -np.inf], np.float32))


class _Ok:
    """A library whose every call succeeds and does nothing."""
    def __getattr__(self, name):
        return lambda *a: B.VSR_OK


@pytest.fixture
def held(monkeypatch):
    """[(tensor, stream)] of the record_stream calls."""
    torch = pytest.importorskip("torch")
    _lib()
    seen = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: seen.append((t, s)))
    return seen


def _all_held(held, stream, tensors):
    ptrs = {t.data_ptr() for t, s in held if s is stream}
    return all(t.data_ptr() in ptrs for t in tensors)


def test_a_contexts_tensors_are_held_for_its_stream(held):
    """What a draft, positions and gains read or write on the context's stream is
    recorded on it, whatever stream it was made on."""
    import torch
    v = B.Verifier.__new__(B.Verifier)
    v.lib, v.h, v.stream, v.device = _Ok(), 1, object(), torch.device("cpu")
    v.cfg = W.VerifierConfig(
        name="held", n_layers=1, d_model=8, n_heads=1, n_kv_heads=1, head_dim=8, d_ff=8, vocab=40,
        rope_base=1e4, dtype=W.F32, n_prefix=4, n_visual=0, n_cands=2, cand_len=3)
    v.workspace = torch.empty(16, dtype=torch.uint8)
    v.gemm_f16, v._has_qk_norm = False, False
    i32 = lambda *s: torch.ones(s, dtype=torch.int32)  # noqa: E731
    prompts, out, ws = i32(2, 3), (i32(2, 5), torch.ones(2, 5)), torch.empty(64, dtype=torch.uint8)
    rules = dict(repetition=torch.ones(2), presence=torch.ones(2), frequency=torch.ones(2),
                 bias=torch.ones(1, 40), mask=i32(5, 2, 2))
    v.draft_ruled(prompts, [1, 2], 5, out=out, workspace=ws, **rules)
    assert _all_held(held, v.stream, [prompts, ws, *out, *rules.values()])
    pos = i32(1, 4)
    v.set_positions(B.rotary((4,), 1e4), pos, 4)
    assert _all_held(held, v.stream, [pos])
    layer = {k: torch.ones(8) for k in
             ("attn_norm", "wqkv", "wo", "ffn_norm", "wgu", "wdown", "q_norm", "k_norm")}
    v.load_weights(dict(embed=torch.ones(8), lm_head=torch.ones(8), final_norm=torch.ones(8),
                        layers=[layer]))
    assert _all_held(held, v.stream, [layer["q_norm"], layer["k_norm"]])
    v.h = None


def test_calls_on_a_given_stream_hold_their_tensors(held, monkeypatch):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    B._torch_names()
    for name, value in (("_lib", _Ok()), ("_device_now", lambda: 0), ("_raw_stream", lambda d: 0)):
        monkeypatch.setattr(B, name, value)
    stream = type("Stream", (), {"device_index": 0, "cuda_stream": 0})()
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q, k, pos, rot = torch.ones(4, 2, 8), torch.ones(4, 1, 8), i32(2, 4), B.rotary((2, 2), 1e4)
    heads = dict(q_out=q.clone(), k_out=k.clone(), k_rows=i32(4))
    gains = torch.ones(8), torch.ones(8)
    x, f32 = torch.ones(3, 100), lambda: torch.ones(3)
    pick = dict(prompt=i32(3, 5), prompt_len=i32(3), output=i32(3, 5), output_len=i32(3),
                repetition=f32(), presence=f32(), frequency=f32(), bias=torch.ones(1, 100),
                mask=i32(1, 4), processed=torch.ones(3, 100),
                workspace=torch.ones(64, dtype=torch.uint8))
    out = i32(3), f32()
    calls = [(lambda s: B.rope_axes(rot, pos, q, k, stream=s, **heads), [pos, q, k, *heads.values()]),
             (lambda s: B.qk_norm_rope(rot, pos, q, k, *gains, 1e-6, stream=s, **heads),
              [pos, q, k, *gains, *heads.values()]),
             (lambda s: B.qk_norm_rope(rot, pos, q, None, gains[0], None, 1e-6, q_out=q, stream=s),
              [pos, q, gains[0]]),
             (lambda s: B.pick_tokens(x, stream=s, out=out, **pick), [x, *out, *pick.values()])]
    for i, (call, tensors) in enumerate(calls):
        held.clear()
        call(None)  # (the current stream's own order holds them)
        assert not held, i
        call(stream)
        assert _all_held(held, stream, tensors), i
