"""vsr_tree_attention without masks, many rows a sequence: pieces of prompts, whose row tiles
end at key tiles of their own. Against the plain form, with the bounds of
test_gpu_tree.py."""
import numpy as np
import pytest

import test_gpu_paged_decoding as PD
from test_gpu_tree import Case, _torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,rows,hq,hk,hd,page,dtype", [
    ([0], [700], 4, 2, 128, 16, "bf16"),                  # six row tiles, no context
    ([0], [700], 4, 2, 128, 16, "f16"),
    ([100, 0, 3], [300, 257, 64], 4, 1, 64, 16, "bf16"),
    ([63, 64, 65], [129, 128, 127], 4, 2, 64, 8, "f16"),  # a row tile each, and one more row
    ([1000, 1], [150, 400], 7, 1, 128, 64, "f16"),        # groups that cross row tiles
    ([129], [333], 5, 1, 80, 16, "bf16"),
    ([70], [300], 2, 1, 256, 16, "bf16"),                 # row tiles of 128
    ([70, 20], [260, 3], 4, 2, 128, 16, "f32"),
    ([5, 0], [200, 140], 2, 1, 256, 16, "f32"),
    ([31, 90], [200, 140], 3, 1, 36, 4, "f16"),           # rows off 16 bytes: four waves, 32 rows
])
def test_chains_of_many_rows(lens, rows, hq, hk, hd, page, dtype):
    c = Case(_torch(), lens, rows, hq, hk, hd, page, dtype, False, seed=hd + len(lens), lead=1, trail=2)
    c.check(*c.run())


def test_a_chain_is_a_tree_of_one_path():
    torch = _torch()
    for dtype in ("bf16", "f16"):
        c = Case(torch, [200, 0], [300, 280], 8, 2, 128, 16, dtype, True, seed=5)
        rows = np.concatenate([np.arange(300), np.arange(280)])
        bits = np.arange(32 * c.words)[None] <= rows[:, None]
        w = (bits.reshape(580, c.words, 32) * (np.uint64(1) << np.arange(32, dtype=np.uint64))).sum(-1)
        c.mask = w.astype(np.uint32)
        want = c.want()
        c.check(*c.run(), want=want)
        c.mask = None
        c.check(*c.run(), want=want)
        # Fewer rows of the same sequences give the same rows, each within (u + u16) of what
        # they weigh together: |out| and the largest |v| at most.
        whole, lse = c.run()
        u, most = torch.finfo(c.dtype).eps / 2, float(c.v.abs().max())
        for at in (0, 17, 64, 256, 299):
            part, _ = c.run(start=c.dev(np.array([0, at + 1, at + 1], np.int32)))
            d = (part[:at + 1].float() - whole[:at + 1].float()).abs()
            assert bool((d <= 2.1 * u * (whole[:at + 1].float().abs() + most)).all())


class _Pieces(PD.Decoder):
    """A decoder whose drafts are pieces of prompts: no parents, no masks."""

    def forward(self, tokens, start):
        B, w, T = self.B, self.w, len(tokens)
        pos, slot, _ = B.tree_rows(self.pages, start, out=(self.ints([0] * T), self.ints([0] * T), None))
        x = w["embed"][self.ints(tokens).long()]
        for layer in range(PD.L):
            y = (PD._norm(x) @ w["qkv"][layer].T).view(T, PD.HQ + 2 * PD.HK, PD.HD)
            q, _ = B.rope_axes(self.rot, pos.view(1, T), y[:, :PD.HQ], y[:, PD.HQ:PD.HQ + PD.HK],
                               k_out=self.k[layer], k_rows=slot)
            self.v[layer][slot.long()] = y[:, PD.HQ + PD.HK:]
            out = B.tree_attention(self.pages, q, self.k[layer], self.v[layer], PD.HD ** -0.5,
                                   start=start)
            x = x + out.view(T, PD.HQ * PD.HD) @ w["o"][layer].T
        return PD._norm(x) @ w["head"].T


def test_prompts_in_pieces_then_tokens():
    """Room, rows of chains, attention and kept rows (all of them), piece after piece, as in
    test_gpu_paged_decoding.py and with its bound."""
    torch = _torch()
    weights, rng = PD._weights(4), np.random.default_rng(4)
    d = _Pieces(torch, 3, 130, 45, weights)
    have = [[], [], []]
    for rows in ([150, 3, 40], [1, 129, 64], [1, 1, 1], [60, 0, 1], [1, 1, 130], [1, 1, 1]):
        assert d.B.pages_update(d.pages, room=d.ints(rows)).tolist() == [1] * 3
        tokens = [rng.integers(0, PD.V, n).tolist() for n in rows]
        logits = d.forward([t for row in tokens for t in row], d.ints(np.concatenate([[0], np.cumsum(rows)])))
        want = [PD._plain(weights, h + t)[len(h):] for h, t in zip(have, tokens) if t]
        assert np.abs(logits.cpu().numpy() - np.concatenate(want)).max() <= PD.BOUND
        kept = np.tile(np.arange(max(rows), dtype=np.int32), (3, 1))
        length = d.B.pages_keep(d.pages, d.ints(kept), d.ints(rows), d.k, d.v)
        have = [h + t for h, t in zip(have, tokens)]
        assert length.tolist() == [len(h) for h in have]
