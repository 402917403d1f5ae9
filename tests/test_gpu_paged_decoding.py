"""The operators over a paged cache in a run, as a decoder with drafted trees uses them:
room and forks, rows of trees, rotary keys written to their slots, attention, log-
probabilities and picks, and the kept rows moved, over several rounds; against a decoder
in float64 that computes every row anew from its own tokens, with no cache.

Bound of a logit, u = 2^-24: a product of n terms is off by (n + 16) u of the sum of its
terms' magnitudes (the 16 for what is added after it: norms, rotations, the softmax), which
is sqrt(n) of the result's size, 5 at most for n <= 64 and weights and rows drawn from
normal laws: 80 u * 8 = 4e-5 of a stage's result. Two layers of four products and the head
make nine stages in a row; a later stage passes an earlier one's error on with the residual
and once more through its own product, so at most doubles it layer by layer: 9 * 4e-5 * 2^2
= 1.4e-3 of a logit's size, which is sqrt(d) / sqrt(d) = 1 by the head's weights. A row that
sees one other token than its own, or one at another position, is off by 1e-1."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

V, D, L, HQ, HK, HD, BASE, PAGE = 193, 64, 2, 4, 2, 32, 1e4, 8
BOUND = 1.4e-3


def _weights(seed):
    rng = np.random.default_rng(seed)
    draw = lambda *s: (rng.standard_normal(s) / np.sqrt(s[-1])).astype(np.float32)  # noqa: E731
    return {"embed": rng.standard_normal((V, D)).astype(np.float32), "head": draw(V, D),
            "qkv": draw(L, (HQ + 2 * HK) * HD, D), "o": draw(L, D, HQ * HD)}


def _norm(x):
    return x / (x * x).mean(-1, **({"keepdims": True} if isinstance(x, np.ndarray)
                                   else {"keepdim": True})) ** 0.5


def _plain(w, tokens):
    """Logits of every position of a token sequence, float64."""
    w = {k: v.astype(np.float64) for k, v in w.items()}
    n = len(tokens)
    x = w["embed"][tokens]
    angle = np.arange(n)[:, None] * BASE ** (-2.0 * np.arange(HD // 2) / HD)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]

    def turn(y):
        a, b = y[..., :HD // 2], y[..., HD // 2:]
        return np.concatenate([a * cos - b * sin, b * cos + a * sin], -1)

    for layer in range(L):
        y = (_norm(x) @ w["qkv"][layer].T).reshape(n, HQ + 2 * HK, HD)
        q, k, v = turn(y[:, :HQ]), turn(y[:, HQ:HQ + HK]), y[:, HQ + HK:]
        k, v = np.repeat(k, HQ // HK, 1), np.repeat(v, HQ // HK, 1)
        s = np.einsum("ihd,jhd->hij", q, k) / np.sqrt(HD)
        s = np.where(np.tril(np.ones((n, n), bool)), s, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        x = x + np.einsum("hij,jhd->ihd", p, v).reshape(n, HQ * HD) @ w["o"][layer].T
    return _norm(x) @ w["head"].T


class Decoder:
    def __init__(self, torch, seqs, pages, most, weights):
        from paper_2601_01513_amd import binding as B
        self.torch, self.B, self.seqs = torch, B, seqs
        self.w = {k: torch.tensor(v, device="cuda") for k, v in weights.items()}
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.pages = B.pages(i32(seqs, most), i32(seqs), i32(seqs), i32(pages), PAGE)
        self.k = torch.full((L, pages * PAGE, HK, HD), float("nan"), device="cuda")
        self.v = torch.full_like(self.k, float("nan"))
        self.rot = B.rotary((HD // 2,), BASE)

    def ints(self, x):
        return self.torch.tensor(np.asarray(x, np.int32), device="cuda")

    def forward(self, tokens, start, parent):
        """Logits of drafted rows whose keys and values go to their slots."""
        B, w, T = self.B, self.w, len(tokens)
        pos, slot, mask = B.tree_rows(self.pages, start, parent, words=2)
        assert (slot >= 0).all()
        x = w["embed"][self.ints(tokens).long()]
        for layer in range(L):
            y = (_norm(x) @ w["qkv"][layer].T).view(T, HQ + 2 * HK, HD)
            q, _ = B.rope_axes(self.rot, pos.view(1, T), y[:, :HQ], y[:, HQ:HQ + HK],
                               k_out=self.k[layer], k_rows=slot)
            self.v[layer][slot.long()] = y[:, HQ + HK:]
            out = B.tree_attention(self.pages, q, self.k[layer], self.v[layer], HD ** -0.5,
                                   start=start, mask=mask)
            x = x + out.view(T, HQ * HD) @ w["o"][layer].T
        return _norm(x) @ w["head"].T


def _tree(rng, n):
    """Parents of n rows whose first is the root."""
    return [-1][:n] + [int(rng.integers(max(0, j - 5), j)) for j in range(1, n)]


def _path(parent, j):
    path = []
    while j >= 0:
        path.append(j)
        j = parent[j]
    return path[::-1]


def test_drafted_trees_over_forked_pages():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    seqs, weights = 5, _weights(0)
    rng = np.random.default_rng(1)
    d = Decoder(torch, seqs, 60, 14, weights)
    B, p = d.B, d.pages
    held_tokens = [[] for _ in range(seqs)]
    # A round: who each sequence continues (-1: a new one), rows of each, chains or trees.
    rounds = [([-1] * 5, [9, 1, 16, 23, 0], False),
              ([0, 1, 2, 3, 3], [12, 7, 33, 1, 5], True),
              ([1, 0, 2, 2, 2], [6, 20, 0, 40, 11], True),
              ([0, 1, -1, 3, 1], [1, 1, 17, 1, 1], True),
              ([0, 0, 2, 4, 3], [8, 8, 8, 8, 8], True)]
    for source, rows, trees in rounds:
        held_tokens = [list(held_tokens[s]) if s >= 0 else [] for s in source]
        ok = B.pages_update(p, d.ints(source), d.ints(rows), d.k, d.v)
        assert ok.tolist() == [1] * seqs
        parents = [_tree(rng, n) if trees else list(range(-1, n - 1)) for n in rows]
        tokens = [rng.integers(0, V, n).tolist() for n in rows]
        start = d.ints(np.concatenate([[0], np.cumsum(rows)]))
        flat = [t for row in tokens for t in row]
        logits = d.forward(flat, start, d.ints([x for row in parents for x in row]))
        # The next token of a row with children is one of theirs, else any.
        after = []
        for n, row, up in zip(rows, tokens, parents):
            child = {up[j]: row[j] for j in range(n)}
            after += [child.get(j, int(rng.integers(0, V))) for j in range(n)]
        lp = B.token_logprobs(logits, d.ints(after), top=4)
        token, logprob = B.pick_tokens(logits)
        want = np.concatenate([
            _plain(weights, held_tokens[s] + [tokens[s][i] for i in _path(parents[s], j)])[-1:]
            for s in range(seqs) for j in range(rows[s])])
        got = logits.cpu().numpy()
        assert np.abs(got - want).max() <= BOUND, np.abs(got - want).max(1)
        x = got.astype(np.float64)
        shifted = x - x.max(1, keepdims=True)
        dist = shifted - np.log(np.exp(shifted).sum(1, keepdims=True))
        order = np.argsort(-x, 1, kind="stable")
        at = np.arange(len(after))
        # (As in the tests of the log-probabilities: 2^-17 of values of up to 10.)
        assert np.abs(lp.logprob.cpu().numpy() - dist[at, after]).max() <= 1e-4
        assert np.array_equal(lp.top_id.cpu().numpy(), order[:, :4])
        assert np.array_equal(lp.rank.cpu().numpy(), np.argsort(order, 1)[at, after])
        assert np.array_equal(token.cpu().numpy(), order[:, 0])
        assert torch.equal(lp.top_id[:, 0], token)
        assert np.abs((lp.top_logprob[:, 0] - logprob).cpu().numpy()).max() <= 1e-4
        # A path from the root stays: to any row, or nothing at all.
        ends = [int(rng.integers(-1, n)) if trees else n - 1 for n in rows]
        paths = [_path(up, j) for up, j in zip(parents, ends)]
        kept = np.zeros((seqs, max(map(len, paths)) or 1), np.int32)
        for s, path in enumerate(paths):
            kept[s, :len(path)] = path
        n_kept = [len(path) for path in paths]
        length = B.pages_keep(p, d.ints(kept), d.ints(n_kept), d.k, d.v)
        for s, path in enumerate(paths):
            held_tokens[s] += [tokens[s][i] for i in path]
        assert length.tolist() == [len(t) for t in held_tokens]
        assert p.held.tolist() == [-(-len(t) // PAGE) for t in held_tokens]
        counts = np.zeros(60, int)
        for s, n in enumerate(p.held.tolist()):
            np.add.at(counts, p.table[s, :n].cpu().numpy(), 1)
        assert p.refs.tolist() == counts.tolist()
