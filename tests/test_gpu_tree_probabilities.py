"""What vsr_tree_attention's 16-bit probabilities hold: few strong keys before very many
weak ones, maxima that rise and fall. Against the formula in 64 bits.

Bound of an output behind many keys, fp16, u = 2^-11 half a step, K keys, V the largest
|v|: a probability is held relative to a reference that no score passes by more than 2^8,
lifted by 2^7: below 2^-21 of the likeliest key it is off by half of fp16's smallest step,
2^-25 / 2^7 = 2^-32 of it, above by u of itself. Numerator and denominator together are
off by 2 K 2^-32 V at most (the denominator is 1 at least in these units) beside the bound
of test_gpu_tree.py, u |want| + (u + 2 ((hd + 4) 2^-23 X + K 2^-23 + 2^-20)) A. Here a
sum over K equal terms passes through 64 keys of a product at a time, waves and blocks, so
K 2^-23 is that of the K / 64 tiles and 64 more."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _attend(torch, table, held, length, page, q, k, v, scale, start=None, lse=None):
    from paper_2601_01513_amd import binding as B
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    refs = torch.ones(k.shape[0] // page, dtype=torch.int32, device="cuda")
    p = B.pages(i32(table), i32(length), i32(held), refs, page)
    out = B.tree_attention(p, q, k, v, scale, start=None if start is None else i32(start), lse=lse)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("seqs,rows,group,pages,sinks", [
    (512, 1, 4, 2048, 4),     # four waves along the keys: one strong key for each
    (256, 20, 2, 1024, 1),    # eight waves along the rows
    (3, 1, 1, 2048, 4),       # every sequence in many parts
])
@pytest.mark.parametrize("below", [25.1, 28.0])
def test_many_weak_keys_behind_a_strong_one(seqs, rows, group, pages, sinks, below):
    """One page of strong keys, the others of weak ones, the same for all sequences."""
    torch = _torch()
    page, hd = 64, 64
    # (The drafted rows see the page of their own, of weak keys too.)
    table = np.ones((seqs, pages + 1), np.int32)
    table[:, 0] = 0
    k = torch.zeros((2 * page, 1, hd), dtype=torch.float16, device="cuda")
    v = torch.ones((2 * page, 1, hd), dtype=torch.float16, device="cuda")
    # The weak scores -below ln 2 in two columns, to fp16's digits twice.
    y = -below * np.log(2.0)
    hi = float(np.float16(y))
    k[:, :, 0], k[:, :, 1] = hi, float(np.float16(y - hi))
    strong = torch.arange(sinks, device="cuda") * 16
    k[strong], v[strong] = 0, 0
    q = torch.zeros((seqs * rows, group, hd), dtype=torch.float16, device="cuda")
    q[:, :, :2] = 1
    start = None if rows == 1 else np.arange(seqs + 1) * rows
    lse = torch.empty(q.shape[:2], device="cuda")
    out = _attend(torch, table, [pages + 1] * seqs, [pages * page] * seqs, page, q, k, v, 1.0, start,
                  lse)
    x = k.double().cpu().numpy()[page, 0, :2].sum()
    n = pages * page - sinks + np.arange(1, rows + 1)            # weak keys of each row
    tail = n * np.exp(x)
    want = np.tile(tail / (sinks + tail), seqs)[:, None, None]
    K, u = pages * page, 2.0 ** -11
    d = (hd + 4) * 2.0 ** -23 * 20 + (K / 64 + 64) * 2.0 ** -23
    bound = u * want + (u + 2 * (d + 2.0 ** -20)) * want + 2 * K * 2.0 ** -32
    assert (np.abs(out.double().cpu().numpy() - want) <= bound).all(), \
        (float(out.min()), float(out.max()), want.min(), bound.min())
    full = np.tile(np.log(sinks + tail), seqs)[:, None]
    assert (np.abs(lse.double().cpu().numpy() - full) <= d + 2.0 ** -20 + K * 2.0 ** -32).all()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_maxima_that_rise_and_the_lowest_values(dtype):
    """Each tile's maximum above the last; scores of tens of thousands; fp32's bound."""
    torch = _torch()
    dt, page, hd, K = getattr(torch, dtype), 16, 64, 512
    rng = np.random.default_rng(2)
    k = torch.zeros((K, 1, hd), dtype=dt, device="cuda")
    v = torch.tensor(rng.standard_normal((K, 1, hd)), device="cuda").to(dt)
    q = torch.zeros((3, 2, hd), dtype=dt, device="cuda")
    q[..., 0] = 1
    u = torch.finfo(dt).eps / 2
    for far, scale in ((np.linspace(-40, 40, K), 1.0), (np.linspace(40, -40, K), 1.0),
                       (np.linspace(-250, 250, K), 400.0), (np.linspace(9, 0, K), -3.0)):
        k[:, 0, 0] = torch.tensor(far, device="cuda").to(dt)
        lse = torch.empty((3, 2), device="cuda")
        out = _attend(torch, [np.arange(K // page)], [K // page], [K - 3], page, q, k, v, scale,
                      [0, 3], lse)
        x = k.double().cpu().numpy()[:, 0, 0] * scale
        for j in range(3):
            n = K - 2 + j
            m = x[:n].max()
            p = np.exp(x[:n] - m)
            vv = v.double().cpu().numpy()[:n, 0]
            want, A = p @ vv / p.sum(), p @ np.abs(vv) / p.sum()
            X = np.abs(x[:n]).max()
            d = (hd + 4) * 2.0 ** -23 * X + K * 2.0 ** -23
            u16 = 0 if dt is torch.float32 else u
            low = 0 if dt is not torch.float16 else 2 * K * 2.0 ** -32 * np.abs(vv).max()
            bound = u * np.abs(want) + (u16 + 2 * (d + 2.0 ** -20)) * A + low
            assert (np.abs(out[j].double().cpu().numpy() - want) <= bound).all(), (scale, j)
            full = m + np.log(p.sum())
            assert (np.abs(lse[j].double().cpu().numpy() - full)
                    <= d + 2.0 ** -21 * (1 + abs(full)) + K * 2.0 ** -32).all(), (scale, j)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("rows", [1, 20])
def test_rises_by_the_last_digit_of_scores_past_2_27(dtype, rows):
    """Scores whose fp32 neighbours lie 16 apart (in steps of log 2), one neighbour higher
    from some tile on. Whatever their roundings make of the weights, an output lies between
    the values it is a mean of, but for the roundings of test_gpu_tree.py's bound: u of itself
    and 2 (u + K 2^-23 + 2^-20) of the largest."""
    torch = _torch()
    dt, page, hd, K, n = getattr(torch, dtype), 16, 64, 256, 16
    u = torch.finfo(dt).eps / 2
    # q . k = 49152^2 + 256 i: fp32 numbers of steps of 256, times c = 16 / 256. (Four key
    # tiles a sequence: a block has its first two.)
    k = torch.zeros((K + 2 * page, 1, hd), dtype=dt, device="cuda")
    v = torch.ones_like(k)
    k[:, 0, 0] = 49152.0
    k[64:, 0, 1] = 256.0
    v[64:] = 3.0
    q = torch.zeros((n * rows, 1, hd), dtype=dt, device="cuda")
    # (Both parities of the last digit: 256 j from the third column, j a sequence's number.)
    q[:, 0, 0], q[:, 0, 1] = 49152.0, 1.0
    k[:, 0, 2] = 256.0
    q[:, 0, 2] = (torch.arange(n * rows, device="cuda") // rows).to(dt)
    start = None if rows == 1 else np.arange(n + 1) * rows
    table = np.tile(np.arange(K // page + 2), (n, 1))
    lse = torch.empty(q.shape[:2], device="cuda")
    scale = 16 / 256 / 1.4426950408889634
    out = _attend(torch, table, [K // page + 2] * n, [K - rows] * n, page, q, k, v, scale, start,
                  lse).float()
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    off = u * 3 + 2 * (u + (K + 32) * 2.0 ** -23 + 2.0 ** -20) * 3
    assert float(out.min()) >= 1 - off and float(out.max()) <= 3 + off


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_log_sums_near_nothing(dtype):
    """lse around 0 to its own digits: n equal scores of -log n, n <= 9. In steps of log 2,
    where |x| and log2 n are below 3.17: log2 is off by 2^-22 of itself, 7.6e-7, the score by
    2^-24 of itself for log2(e)'s rounding, 1.9e-7, and half a last digit, 1.2e-7, the
    probabilities by 2^-24, 0.9e-7 there; the sum of n of them is exact. Times log 2: 8.1e-7,
    with the last products' roundings below 2^-20."""
    torch = _torch()
    dt, page, hd = getattr(torch, dtype), 16, 64
    k = torch.zeros((page, 1, hd), dtype=dt, device="cuda")
    v = torch.ones_like(k)
    q = torch.zeros((9, 1, hd), dtype=dt, device="cuda")
    k[:, 0, :2] = 1
    for i in range(9):
        y = -np.log(i + 1.0)
        hi = float(torch.tensor(y).to(dt))
        q[i, 0, 0], q[i, 0, 1] = hi, float(torch.tensor(y - hi).to(dt))
    lse = torch.empty((9, 1), device="cuda")
    out = _attend(torch, [[0]], [1], [0], page, q, k, v, 1.0, [0, 9], lse)
    x = q.double()[:, 0, :2].sum(1).cpu().numpy()
    want = x + np.log(np.arange(1, 10))
    assert np.abs(lse.double().cpu().numpy()[:, 0] - want).max() <= 2.0 ** -20
    # (The sum over itself: a reciprocal and a product, 2^-24 each of it in fp32.)
    assert float((out.double() - 1).abs().max()) <= 2.0 ** -22
