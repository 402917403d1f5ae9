"""The call validator (vsr_set_checks) through the C ABI: bad ids give
VSR_EID, non-finite results VSR_ENONFINITE; the outputs are those of the
unchecked call (an out-of-range id is read as id 0), and valid inputs pass
unchanged. The oracle, given the same NaN visual row, also yields non-finite
scores (a NaN key reaches every later query through the softmax)."""
import sys

import numpy as np
import pytest

import oracle
from paper_2601_01513_amd import workload as W

pytestmark = pytest.mark.gpu

SMALL = W.VerifierConfig(
    name="checks bf16 L2 d256 G2 F320 V1000", n_layers=2, d_model=256, n_heads=4,
    n_kv_heads=2, head_dim=128, d_ff=320, vocab=1000, rope_base=1e6, dtype=W.BF16,
    n_prefix=300, n_visual=100, n_cands=5, cand_len=40)


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _say(msg):
    print(msg, file=sys.stderr, flush=True)


def _run(v, wl, cids, visual=None, prefix_ids=None):
    torch = _torch()
    ids = torch.tensor(wl.prefix_ids if prefix_ids is None else prefix_ids, dtype=torch.int32,
                       device="cuda")
    lp, sc, am = v.verify(wl.visual if visual is None else visual, ids,
                          torch.tensor(cids, dtype=torch.int32, device="cuda"), wl.cand_len)
    torch.cuda.synchronize()
    return lp.cpu().numpy(), sc.cpu().numpy(), int(am.cpu()[0])


def _expect(code, fn):
    from paper_2601_01513_amd.binding import VsrError
    with pytest.raises(VsrError) as e:
        fn()
    assert e.value.code == code, str(e.value)
    _say(f"  status {e.value.code}: {e.value}")


@pytest.mark.parametrize("cfg", [SMALL, W.TINY_F32], ids=["bf16", "fp32"])
def test_valid_inputs_pass_and_match_unchecked(cfg):
    torch = _torch()
    from paper_2601_01513_amd.binding import Verifier
    _say(f"case: {cfg.name} checks on, valid inputs")
    wl = W.make_workload(cfg, 0, device="cuda")
    v = Verifier(cfg, wl.weights, device="cuda")
    ref = _run(v, wl, wl.cand_ids)
    v.set_checks(ids=True, finite=True)
    got = _run(v, wl, wl.cand_ids)
    assert np.array_equal(ref[0], got[0]) and np.array_equal(ref[1], got[1])
    assert ref[2] == got[2]
    v.prefill(wl.visual, torch.tensor(wl.prefix_ids, dtype=torch.int32, device="cuda"))
    v.score(torch.tensor(wl.cand_ids, dtype=torch.int32, device="cuda"), wl.cand_len)
    torch.cuda.synchronize()


@pytest.mark.parametrize("cfg", [SMALL, W.TINY_F32], ids=["bf16", "fp32"])
def test_out_of_range_ids_report_eid(cfg):
    torch = _torch()
    from paper_2601_01513_amd.binding import VSR_EID, Verifier
    _say(f"case: {cfg.name} out-of-range ids")
    wl = W.make_workload(cfg, 1, device="cuda")
    v = Verifier(cfg, wl.weights, device="cuda")
    bad = wl.cand_ids.copy()
    bad[1, 3] = cfg.vocab + 5
    bad[2, 0] = -1
    zero = wl.cand_ids.copy()
    zero[1, 3] = 0
    zero[2, 0] = 0
    ref = _run(v, wl, zero)
    unchecked = _run(v, wl, bad)          # default: no check, id read as 0
    assert np.array_equal(ref[0], unchecked[0])
    # The two-call pass (it agrees with vsr_verify to rounding only).
    v.prefill(wl.visual, torch.tensor(wl.prefix_ids, dtype=torch.int32, device="cuda"))
    ref2 = v.score(torch.tensor(zero, dtype=torch.int32, device="cuda"), wl.cand_len)[0]
    torch.cuda.synchronize()
    ref2 = ref2.cpu().numpy()
    v.set_checks(ids=True, finite=False)
    _expect(VSR_EID, lambda: _run(v, wl, bad))
    pid = wl.prefix_ids.copy()
    pid[7] = 1 << 30
    _expect(VSR_EID, lambda: v.prefill(wl.visual, torch.tensor(pid, dtype=torch.int32,
                                                               device="cuda")))
    v.prefill(wl.visual, torch.tensor(wl.prefix_ids, dtype=torch.int32, device="cuda"))
    lens = [max(1, int(n)) for n in wl.cand_len]
    _expect(VSR_EID, lambda: v.reliability(torch.tensor(bad, dtype=torch.int32, device="cuda"),
                                           lens, 1, 2, 0.05))
    lp, sc, am = v.score(torch.tensor(zero, dtype=torch.int32, device="cuda"), wl.cand_len)
    torch.cuda.synchronize()
    assert np.array_equal(lp.cpu().numpy(), ref2)


@pytest.mark.parametrize("cfg", [SMALL, W.TINY_F32], ids=["bf16", "fp32"])
def test_nan_visual_row_reports_enonfinite(cfg):
    torch = _torch()
    from paper_2601_01513_amd.binding import VSR_ENONFINITE, Verifier
    _say(f"case: {cfg.name} NaN visual row")
    wl = W.make_workload(cfg, 2, device="cuda")
    vis = wl.visual.clone()
    vis[17, :] = float("nan")
    v = Verifier(cfg, wl.weights, device="cuda")
    v.set_checks(ids=True, finite=True)
    _expect(VSR_ENONFINITE, lambda: _run(v, wl, wl.cand_ids, visual=vis))
    _expect(VSR_ENONFINITE, lambda: v.prefill(vis, torch.tensor(
        wl.prefix_ids, dtype=torch.int32, device="cuda")))
    # The oracle on the same inputs: no finite score either.
    with np.errstate(invalid="ignore", over="ignore"):
        lp_o, sc_o, _ = oracle.score_shared_prefix(cfg, W.host_weights(wl.weights),
                                                   W.to_host_f32(vis), wl.prefix_ids,
                                                   wl.cand_ids, wl.cand_len, dtype=np.float32)
    assert not np.any(np.isfinite(sc_o))
    # Finite inputs again: the context recovers.
    _run(v, wl, wl.cand_ids)


def test_unknown_check_bits_are_rejected():
    _torch()
    from paper_2601_01513_amd.binding import VSR_EINVAL, Verifier
    wl = W.make_workload(W.TINY_F32, 0, device="cuda")
    v = Verifier(W.TINY_F32, wl.weights, device="cuda")
    assert v.lib.vsr_set_checks(v.h, 4) == VSR_EINVAL
    assert b"unknown" in v.lib.vsr_last_error(v.h)


@pytest.mark.parametrize("split", [0, 1], ids=["fast", "precise"])
@pytest.mark.parametrize("cfg", [SMALL, W.TINY_F32], ids=["bf16", "fp32"])
def test_a_nan_call_leaves_nothing_behind(cfg, split):
    """After a prefix, candidates, branches and drafts of NaN, shorter and longer
    calls give the results of a context that never saw them, bit for bit: what
    the caches hold past the rows a call writes does not reach it."""
    torch = _torch()
    from paper_2601_01513_amd.binding import Verifier
    _say(f"case: {cfg.name} split {split} calls after a NaN visual row")
    wl = W.make_workload(cfg, 6, device="cuda")
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    ids, cands, M = i32(wl.prefix_ids), i32(wl.cand_ids), cfg.n_cands
    make = lambda: Verifier(cfg, wl.weights, device="cuda", max_new=6, split_layers=split)  # noqa: E731

    def calls(v, vis, prefix, lens, m):
        out = []
        out += v.verify(vis, prefix, cands, lens)
        v.prefill(vis, prefix)
        out += v.score(cands, lens)
        out += v.reliability(cands[:m], [max(1, n) for n in lens[:m]], 1, 2, 0.05)[:2]
        out += [v.draft(cands[:m], [3] * m, 5), *v.draft_ruled(cands[:m], [2] * m, 4)]
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in out]

    nan = wl.visual.clone()
    nan[3, :] = float("nan")
    full = [int(n) for n in wl.cand_len]
    # (lengths that leave part of the last tile of the long call's rows unwritten)
    short = ids[:len(ids) - 20], [7, 1, 0, 12, 5][:M], M - 1
    long = ids, full, M
    v = make()
    bad = calls(v, nan, *long)
    assert np.isnan(bad[0]).any() and np.isnan(bad[-1]).any()
    for case in (short, long):
        got, want = calls(v, wl.visual, *case), calls(make(), wl.visual, *case)
        assert all(np.isfinite(a).all() for a in want)
        for i, (a, b) in enumerate(zip(got, want)):
            assert np.array_equal(a, b), i
        calls(v, nan, *long)
@pytest.mark.parametrize("kept", [True, False], ids=["logprobs", "tokens only"])
@pytest.mark.parametrize("cfg", [SMALL, W.TINY_F32], ids=["bf16", "fp32"])
def test_ruled_drafts(cfg, kept):
    """A ruled draft under both checks: a mask that allows nothing in a step is no
    error, a NaN prefix and an allowed infinite bias are VSR_ENONFINITE, a prompt id
    outside the vocabulary is VSR_EID."""
    torch = _torch()
    from paper_2601_01513_amd.binding import VSR_EID, VSR_ENONFINITE, Verifier
    _say(f"case: {cfg.name} ruled drafts, logprobs {kept}")
    wl = W.make_workload(cfg, 4, device="cuda")
    v = Verifier(cfg, wl.weights, device="cuda", max_new=3)
    ids = torch.tensor(wl.prefix_ids, dtype=torch.int32, device="cuda")
    prompts = torch.tensor(wl.cand_ids, dtype=torch.int32, device="cuda")
    M, words = cfg.n_cands, (cfg.vocab + 31) // 32
    mask = torch.full((3, M, words), -1, dtype=torch.int32, device="cuda")
    mask[1, M - 1] = 0

    def run(p=prompts, **kw):
        out = (torch.empty((M, 3), dtype=torch.int32, device="cuda"),
               torch.empty((M, 3), device="cuda") if kept else None)
        return v.draft_ruled(p, [2] * M, 3, mask=mask, out=out, **kw)

    v.prefill(wl.visual, ids)
    want, want_lp = run()
    v.set_checks(ids=True, finite=True)
    got, got_lp = run()
    assert torch.equal(got, want) and int(got[M - 1, 1]) == -1
    if kept:
        assert torch.equal(got_lp, want_lp) and float(got_lp[M - 1, 1]) == -np.inf
    bias = torch.zeros((1, cfg.vocab), device="cuda")
    bias[0, 5] = float("inf")
    _expect(VSR_ENONFINITE, lambda: run(bias=bias))
    bad = prompts.clone()
    bad[1, 1] = cfg.vocab
    _expect(VSR_EID, lambda: run(bad))
    v.set_checks(ids=False, finite=False)
    vis = wl.visual.clone()
    vis[0, :] = float("nan")
    v.prefill(vis, ids)
    v.set_checks(ids=False, finite=True)
    _expect(VSR_ENONFINITE, run)
    v.set_checks(ids=False, finite=False)
    assert bool((run()[0] == -1).all())  # unchecked, as a mask that allows nothing
    v.prefill(wl.visual, ids)
    v.set_checks(ids=True, finite=True)
    assert torch.equal(run()[0], want)
