"""Refusals of vsr_token_logprobs, before the device is touched."""
import os

import pytest

from paper_2601_01513_amd import binding as B

MB = 1 << 20


def _lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libvsr.so not built (python -m paper_2601_01513_amd.build)")
    return B.load_library()


def _call(**kw):
    a = dict(logits=MB, dtype=B.VSR_F16, rows=4, vocab=1000, stride=1000, tokens=2 * MB, top=8,
             logprob=3 * MB, rank=3 * MB + 64, entropy=3 * MB + 128, top_id=3 * MB + 256,
             top_logprob=3 * MB + 512, ws=4 * MB, wsb=1 << 20)
    a.update(kw)
    return _lib().vsr_token_logprobs(*a.values(), None)


@pytest.mark.parametrize("kw,word", [
    (dict(dtype=3), "dtype"), (dict(rows=-1), "rows"), (dict(rows=65536), "rows"),
    (dict(vocab=0), "vocab"), (dict(vocab=(1 << 24) + 1), "vocab"), (dict(top=-1), "top"),
    (dict(top=65), "top"), (dict(logits=None), "NULL"), (dict(ws=None), "NULL"),
    (dict(logits=MB + 1), "logits"), (dict(stride=999), "stride"), (dict(tokens=None), "tokens"),
    (dict(tokens=2 * MB + 2), "aligned"), (dict(top_id=3 * MB + 257), "aligned"),
    (dict(rank=3 * MB + 12), "overlaps"), (dict(top_logprob=3 * MB + 380), "overlaps"),
    (dict(entropy=2 * MB + 4), "overlaps"), (dict(logprob=MB + 7996), "overlaps"),
    (dict(ws=4 * MB + 8), "workspace"), (dict(wsb=64), "smaller"),
    (dict(ws=MB + 4096), "workspace overlaps"), (dict(ws=3 * MB + 512), "workspace overlaps"),
])
def test_refuses(kw, word):
    assert _call(**kw) == B.VSR_EINVAL
    msg = _lib().vsr_last_error(None).decode()
    assert word in msg and msg.startswith("token_logprobs: "), msg


def test_nothing_to_do_and_sizes():
    assert _call(rows=0, logits=None, ws=None, wsb=0) == B.VSR_OK
    size = _lib().vsr_token_logprobs_workspace_size
    assert 0 < size(512, 152064, 20) < 1 << 22
    for bad in ((0, 10, 1), (65536, 10, 1), (1, 0, 1), (1, (1 << 24) + 1, 1), (1, 10, -1), (1, 10, 65)):
        assert size(*bad) == 0


def test_the_binding_refuses():
    torch = pytest.importorskip("torch")
    _lib()
    x, t = torch.zeros(3, 100), torch.zeros(3, dtype=torch.int32)
    f, i = torch.zeros(3), torch.zeros(3, 4)
    bad = [lambda: B.token_logprobs(x.double(), t), lambda: B.token_logprobs(x[0], t),
           lambda: B.token_logprobs(x.t(), t), lambda: B.token_logprobs(x, t.long()),
           lambda: B.token_logprobs(x, t[:2]), lambda: B.token_logprobs(x, t),   # host tensors
           lambda: B.token_logprobs(x, t, 4, out=(f.half(), t, f, None, None)),
           lambda: B.token_logprobs(x, t, 4, out=(f, t.float(), f, None, None)),
           lambda: B.token_logprobs(x, t, 4, out=(f, t, f, i, i)),
           lambda: B.token_logprobs(x, t, 4, out=(f, t, f, i.int(), i[:, :3]))]
    for n, g in enumerate(bad):
        with pytest.raises(B.VsrError) as e:
            g()
        assert e.value.code == B.VSR_EINVAL, n
