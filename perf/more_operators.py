"""The operators of a speculative step over a paged key/value cache: cases, plain
forms, exact values.

Each case is one call of one operator, at the sizes of this repository's own
workloads (workload.py) or generic ones:
  attend    attention of drafted trees (or single tokens) over their sequences' pages;
  rows      a tree's positions, cache slots and ancestor masks from its parents;
  update    sequences forked from others, pages copied, counted and reserved;
  keep      the accepted rows of a draft moved together, in every layer;
  logprobs  log-probabilities of given tokens with rank, entropy and alternatives.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _attend(name, seqs, ctx, n, tree, hq, hk, hd, page, dtype):
    return {"name": name, "op": "attend", "seqs": seqs, "ctx": ctx, "n": n, "tree": tree,
            "hq": hq, "hk": hk, "hd": hd, "page": page, "dtype": dtype}


def _rows(name, seqs, ctx, n, page):
    return {"name": name, "op": "rows", "seqs": seqs, "ctx": ctx, "n": n, "page": page}


def _update(name, groups, beams, ctx, room, page, layers, hk, hd, dtype):
    return {"name": name, "op": "update", "groups": groups, "beams": beams, "ctx": ctx,
            "room": room, "page": page, "layers": layers, "hk": hk, "hd": hd, "dtype": dtype}


def _keep(name, seqs, ctx, n, depth, page, layers, hk, hd, dtype):
    return {"name": name, "op": "keep", "seqs": seqs, "ctx": ctx, "n": n, "depth": depth,
            "page": page, "layers": layers, "hk": hk, "hd": hd, "dtype": dtype}


def _logprobs(name, rows, vocab, top, dtype):
    return {"name": name, "op": "logprobs", "rows": rows, "vocab": vocab, "top": top,
            "dtype": dtype}


def listed():
    return [
        # A small fp32 decoder checks a handful of drafted tokens: latency only.
        _attend("attend fp32 2 x 5, 200", 2, 200, 5, True, 4, 4, 64, 16, "f32"),
        # One decode step of many requests of the 3B-class drafter, lengths ragged.
        _attend("attend decode 3B 64 x 1, 4096", 64, 4096, 1, False, 16, 2, 128, 16, "bf16"),
        # The verifier on eight drafted trees after the headline's prefix length.
        _attend("attend trees 7B 8 x 64, 4096", 8, 4096, 64, True, 28, 4, 128, 16, "bf16"),
        # The widest model, long contexts: the largest call.
        _attend("attend trees 32B 16 x 48, 16384", 16, 16384, 48, True, 40, 8, 128, 64, "f16"),
        # Three drafts' trees before a step; then a full batch's.
        _rows("rows 3 x 21", 3, 2688, 21, 16),
        _rows("rows 256 x 100", 256, 5000, 100, 16),
        # Three drafts begin from one request; a beam step of a batch.
        _update("update 3 drafts 3B", 1, 3, 2188, 24, 16, 36, 2, 128, "bf16"),
        _update("update 16 x 4 beams 3B", 16, 4, 600, 70, 16, 36, 2, 128, "bf16"),
        # What three drafts accepted; what a batch of trees accepted, 7B-class.
        _keep("keep 3 x 21 3B", 3, 1100, 21, 5, 16, 36, 2, 128, "bf16"),
        _keep("keep 64 x 64 7B", 64, 300, 64, 9, 16, 28, 4, 128, "bf16"),
        # Three rows of a decode step; the headline's 8 candidates of 64 tokens.
        _logprobs("logprobs 3 x 151936 top 5", 3, 151936, 5, "f32"),
        _logprobs("logprobs 512 x 152064 top 20", 512, 152064, 20, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "rows", "update", "keep", "logprobs",
                     "logprobs"])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    if op == "logprobs":
        return {"op": op, "rows": _log_int(rng, 1, 512), "vocab": _log_int(rng, 500, 152064),
                "top": rng.choice([0, 1, rng.randint(2, 20), rng.randint(20, 64)]),
                "dtype": rng.choice(["f32", "bf16", "f16"])}
    if op == "rows":
        return {"op": op, "seqs": _log_int(rng, 1, 256), "ctx": _log_int(rng, 1, 16384),
                "n": _log_int(rng, 1, 250), "page": page}
    hk, hd = rng.choice([(2, 128), (4, 128), (8, 128), (4, 64), (5, 80), (1, 256), (3, 36)])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("update", "keep"):
        layers = rng.choice([2, 28, 36])
        token = 2 * layers * hk * hd * (4 if dtype == "f32" else 2)
        ctx = _log_int(rng, 1, 2048)
        if op == "update":
            room = _log_int(rng, 1, 128)
            beams = rng.randint(2, 8)
            most = max(1, (1 << 30) // (token * beams * 2 * (ctx + room + page)))
            return {"op": op, "groups": min(_log_int(rng, 1, 32), most), "beams": beams,
                    "ctx": ctx, "room": room, "page": page, "layers": layers, "hk": hk, "hd": hd,
                    "dtype": dtype}
        n = _log_int(rng, 1, 128)
        most = max(1, (1 << 30) // (token * (ctx + n + page)))
        return {"op": op, "seqs": min(_log_int(rng, 1, 64), most), "ctx": ctx, "n": n,
                "depth": rng.randint(1, 12), "page": page, "layers": layers, "hk": hk, "hd": hd,
                "dtype": dtype}
    n = rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 2, 128), _log_int(rng, 64, 512)])
    group = rng.choice([1, 2, 4, 5, 7, 8])
    seqs = _log_int(rng, 1, 64)
    # At most half the largest listed case's keys and products.
    keys = min((1 << 28) // (hk * hd * (4 if dtype == "f32" else 2)),
               (1 << 35) // (n * group * hk * hd * (8 if dtype == "f32" else 1)))
    ctx = min(_log_int(rng, 1, 16384), max(1, keys // seqs))
    return {"op": op, "seqs": seqs, "ctx": ctx, "n": n, "tree": rng.random() < 0.7,
            "hq": hk * group, "hk": hk, "hd": hd, "page": page, "dtype": dtype}


def _ceil(a, b):
    return (a + b - 1) // b


def _parents(seqs, n, ints):
    """Random trees, row by row: most nodes hang on one of the few before them."""
    j = torch.arange(n, device="cuda")
    back = ints(1, 9, (seqs, n))
    return torch.where(back > j + 1, -1, j - back).to(torch.int32)


def _ancestors(parent):
    """[seqs][n][n]: whether node i lies on node j's path, itself included."""
    seqs, n = parent.shape
    seen = torch.eye(n, dtype=torch.bool, device="cuda").repeat(seqs, 1, 1)
    s = torch.arange(seqs, device="cuda")
    for j in range(1, n):
        p = parent[:, j].long()
        seen[:, j] |= seen[s, p.clamp(min=0)] & (p >= 0)[:, None]
    return seen


def _words(bits):
    """Truth values [..., n] as int32 words, 32 a word."""
    n = bits.shape[-1]
    bits = torch.nn.functional.pad(bits.long(), (0, _ceil(n, 32) * 32 - n))
    w = (bits.unflatten(-1, (-1, 32)) << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def ints(lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=g, device=dev, dtype=torch.int32)

    def normal(dtype, *shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(dtype) \
            if math.prod(shape) < 1 << 28 else \
            torch.empty(shape, device=dev, dtype=dtype).normal_(generator=g)

    op = case["op"]
    s = {"case": case}
    if op == "logprobs":
        R, V = case["rows"], case["vocab"]
        s["logits"] = normal(torch.float32, R, V).mul_(3).to(DTYPES[case["dtype"]])
        # Half the tokens are likely ones, as drafted tokens are.
        likely = s["logits"][:, :max(1, V // 2)].argmax(1).to(torch.int32)
        s["tokens"] = torch.where(ints(0, 2, (R,)) == 1, likely, ints(0, V, (R,)))
        return s

    ps = case["page"]
    seqs = case["groups"] * case["beams"] if op == "update" else case["seqs"]
    length = ints(max(1, case["ctx"] // 2), case["ctx"] + 1, (seqs,))
    if op == "update":
        # A beam step: each group's survivors stay, the others become copies of one of
        # them. Everyone holds the pages of the step before.
        G, Bm = case["groups"], case["beams"]
        stays = ints(1, Bm, (G, 1))
        b = torch.arange(Bm, device=dev)
        pick = ints(0, 1 << 20, (G, Bm)) % stays
        source = torch.where(b < stays, b, pick) + Bm * torch.arange(G, device=dev)[:, None]
        s["source"] = source.flatten().to(torch.int32)
        s["room"] = ints(1, case["room"] + 1, (seqs,))
        held = _ceil(length, ps)
        most = _ceil(case["ctx"] + case["room"], ps) + 1
        s["most_new"] = _ceil(case["room"], ps) + 1
    else:
        # The sequences' drafts are in their pages already, behind the context.
        # (Sizes from n / 2 to n, the same ones for every seed, in another order.)
        low = max(1, case["n"] // 2)
        n = low + torch.arange(seqs, device=dev) * (case["n"] - low + 1) // seqs
        n = n[torch.randperm(seqs, generator=g, device=dev)].to(torch.int32)
        held = _ceil(length + n, ps)
        most = _ceil(case["ctx"] + case["n"], ps)
    n_pages = seqs * most + 8 + (seqs if op == "update" else 0)
    page = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    col = torch.arange(most, device=dev)
    s["table"] = page[:seqs * most].view(seqs, most).contiguous()
    s["refs"] = torch.zeros(n_pages, dtype=torch.int32, device=dev)
    s["refs"][s["table"][col < held[:, None]].long()] = 1
    s.update(len=length, held=held)
    if op in ("update", "keep"):
        shape = (case["layers"], n_pages * ps, case["hk"], case["hd"])
        s["k"], s["v"] = normal(DTYPES[case["dtype"]], *shape), normal(DTYPES[case["dtype"]], *shape)
        if op == "update":
            s["ok"] = torch.empty(seqs, dtype=torch.int32, device=dev)
            return s
        # The accepted path: a node, one a few places on, ...
        s["kept"] = (ints(1, 9, (seqs, case["depth"])).cumsum(1) - 1).to(torch.int32)
        fits = (s["kept"] < n[:, None]).sum(1).to(torch.int32)
        s["n_kept"] = torch.minimum(ints(0, case["depth"] + 1, (seqs,)), fits)
        s["len_out"] = torch.empty_like(length)
        return s

    s["start"] = torch.cat([n.new_zeros(1), n.cumsum(0)]).to(torch.int32)
    s["T"] = T = int(s["start"][-1])
    s["seq"] = torch.repeat_interleave(torch.arange(seqs, device=dev), n.long(), output_size=T)
    s["row"] = torch.arange(T, device=dev) - s["start"][s["seq"]]
    parent = _parents(seqs, case["n"], ints)
    if op == "rows":
        s["parent"] = parent[s["seq"], s["row"]].contiguous()
        words = _ceil(case["n"], 32)
        s["out"] = (torch.empty(T, dtype=torch.int32, device=dev),
                    torch.empty(T, dtype=torch.int32, device=dev),
                    torch.empty((T, words), dtype=torch.int32, device=dev))
        return s
    dt = DTYPES[case["dtype"]]
    s["k"], s["v"] = (normal(dt, n_pages * ps, case["hk"], case["hd"]) for _ in range(2))
    s["q"] = normal(dt, T, case["hq"], case["hd"])
    s["mask"] = _words(_ancestors(parent)[s["seq"], s["row"]]) if case["tree"] else None
    s["out"] = torch.empty_like(s["q"])
    s["scale"] = case["hd"] ** -0.5
    return s


# ---------------------------------------------------------------- plain forms


def _attend_plain(s):
    c = s["case"]
    ps, n, hk, hd = c["page"], c["n"], c["hk"], c["hd"]
    seqs, G = c["seqs"], c["hq"] // c["hk"]
    L = c["ctx"] + n
    p = torch.arange(L, device="cuda")
    slot = s["table"][:, p // ps].long() * ps + p % ps
    k = s["k"][slot].permute(0, 2, 3, 1).float().contiguous()    # [seqs][hk][hd][L]
    v = s["v"][slot].permute(0, 2, 1, 3).float().contiguous()    # [seqs][hk][L][hd]
    q = torch.zeros((seqs, n, hk, G, hd), device="cuda")
    q[s["seq"], s["row"]] = s["q"].float().view(-1, hk, G, hd)
    q = q.permute(0, 2, 3, 1, 4).reshape(seqs * hk, G * n, hd)
    x = torch.bmm(q, k.view(seqs * hk, hd, L)).view(seqs, hk, G, n, L) * s["scale"]
    j = p - s["len"][:, None]                                    # [seqs][L]
    i = torch.arange(n, device="cuda")
    if s["mask"] is None:
        drafted = (j[:, None] >= 0) & (j[:, None] <= i[:, None])
    else:
        words = torch.zeros((seqs, n, s["mask"].shape[1]), dtype=torch.int32, device="cuda")
        words[s["seq"], s["row"]] = s["mask"]
        at = j.clamp(0, n - 1)[:, None].expand(seqs, n, L)
        bit = torch.gather(words, 2, at // 32) >> (at % 32).to(torch.int32) & 1
        drafted = (bit == 1) & (j >= 0)[:, None] & (j < n)[:, None]
    seen = (j < 0)[:, None] | drafted                            # [seqs][n][L]
    x = torch.where(seen[:, None, None], x, -math.inf)
    x = (x - x.amax(-1, keepdim=True)).exp()
    y = torch.bmm(x.view(seqs * hk, G * n, L), v.view(seqs * hk, L, hd)).view(seqs, hk, G, n, hd)
    y = y / x.sum(-1, keepdim=True)
    y = y.permute(0, 3, 1, 2, 4)[s["seq"], s["row"]].reshape(s["q"].shape)
    return {"out": y.to(s["q"].dtype)}


def _rows_plain(s):
    c = s["case"]
    ps, n, seqs = c["page"], c["n"], c["seqs"]
    parent = torch.full((seqs, n), -1, dtype=torch.int32, device="cuda")
    parent[s["seq"], s["row"]] = s["parent"]
    # Paths by squaring: after r steps a node has 2^r nodes of its path.
    near = (parent[:, :, None] == torch.arange(n, device="cuda")).float()
    reach = torch.eye(n, device="cuda") + near
    for _ in range(max(0, (n - 1).bit_length())):
        reach = torch.bmm(reach, reach).clamp(max=1)
    reach = reach[s["seq"], s["row"]] > 0
    length = s["len"][s["seq"]]
    pos = length + reach.sum(1) - 1
    at = length + s["row"]
    slot = s["table"][s["seq"], at // ps].long() * ps + at % ps
    return {"pos": pos.to(torch.int32), "slot": slot.to(torch.int32), "mask": _words(reach)}


def _update_plain(s):
    c = s["case"]
    ps, table, refs, length, held = c["page"], s["table"], s["refs"], s["len"], s["held"]
    seqs, most = table.shape
    d = torch.arange(seqs, device="cuda")
    src = s["source"].long()
    moved = src != d
    new_len = length[src]
    full, part = new_len // ps, new_len % ps
    # Who goes on with a source's last page: itself, or the lowest of its heirs.
    heir = torch.full((seqs,), seqs, device="cuda").scatter_reduce(0, src, d, "amin")
    heir = torch.where(src == d, d, heir)
    copies = (part > 0) & (heir[src] != d)
    col = torch.arange(most, device="cuda")
    old = (col < held[:, None]) & moved[:, None]
    refs.index_add_(0, table.flatten().long(), -old.flatten().to(torch.int32))
    new = table[src]
    keeps = torch.where(moved, full + ((part > 0) & ~copies).to(full.dtype), held)
    shared = (col < keeps[:, None]) & moved[:, None]
    refs.index_add_(0, new.flatten().long(), shared.flatten().to(torch.int32))
    written = torch.where(moved, full + (part > 0).to(full.dtype), 0)
    table.copy_(torch.where(col < written[:, None], new, table))
    # Free pages in order, handed out in the order of sequences: a copy's, then the room's.
    want = _ceil(new_len + s["room"], ps)
    got = keeps + copies.to(keeps.dtype)
    extra = (want - got).clamp(min=0) * (want <= most)
    need = extra + copies.to(extra.dtype)
    upto = need.cumsum(0)
    free = refs == 0
    served = upto <= free.sum()
    ok = served & (want <= most)
    give = need * served
    order = torch.where(free, torch.arange(refs.numel(), device="cuda"), refs.numel()).sort().values
    i = torch.arange(s["most_new"] + 1, device="cuda")
    taken = i < give[:, None]
    pages = order[((upto - need)[:, None] + i).clamp(max=refs.numel() - 1)]
    refs.index_add_(0, torch.where(taken, pages, 0).flatten(), taken.flatten().to(torch.int32))
    from_page = table.gather(1, full.clamp(max=most - 1)[:, None].long())
    place = (col - keeps[:, None]).clamp(0, s["most_new"]).long()
    fresh = (col >= keeps[:, None]) & (col < (keeps + give)[:, None])
    table.copy_(torch.where(fresh, pages.gather(1, place).to(torch.int32), table))
    # The copies' rows; every other place is copied onto itself.
    r = torch.arange(ps, device="cuda")
    last = table.gather(1, ((new_len - 1).clamp(min=0) // ps)[:, None].long())
    copied = (copies & served)[:, None] & (r < part[:, None])
    to = (last * ps + r).flatten().long()
    at = (torch.where(copied, from_page, last) * ps + r).flatten().long()
    s["k"][:, to] = s["k"][:, at]
    s["v"][:, to] = s["v"][:, at]
    length.copy_(torch.where(copies & ~served, full * ps, new_len))
    held.copy_(keeps + give)
    s["ok"].copy_(ok)
    return {"ok": s["ok"], "table": table, "len": length, "held": held, "refs": refs, "k": s["k"],
            "v": s["v"]}


def _keep_plain(s):
    ps, length, kept = s["case"]["page"], s["len"], s["kept"]
    i = torch.arange(kept.shape[1], device="cuda")
    live = i < s["n_kept"][:, None]
    # (In the place of rows that are not kept, the first row is copied onto itself.)
    at, to = (torch.where(live, length[:, None] + j, 0) for j in (kept, i))

    def slot(p):
        return s["table"].gather(1, (p // ps).long()).long() * ps + p % ps

    a, t = slot(at).flatten(), slot(to).flatten()
    s["k"][:, t] = s["k"][:, a]
    s["v"][:, t] = s["v"][:, a]
    s["len_out"].copy_(length + s["n_kept"])
    return {"len": s["len_out"], "k": s["k"], "v": s["v"]}


def _logprobs_plain(s):
    x = s["logits"].float()
    top = s["case"]["top"]
    m = x.amax(1, keepdim=True)
    e = (x - m).exp()
    S = e.sum(1, keepdim=True)
    lse = S.log()
    t = torch.gather(x, 1, s["tokens"].long()[:, None])
    v = torch.arange(x.shape[1], device="cuda")
    ahead = (x > t) | ((x == t) & (v < s["tokens"][:, None]))
    got = {"logprob": (t - m - lse)[:, 0],
           "entropy": lse[:, 0] - (e * (x - m)).sum(1) / S[:, 0],
           "rank": ahead.sum(1).to(torch.int32)}
    if top:
        # One number a token that orders by logit, then by index.
        bits = (x + 0.0).view(torch.int32)
        key = (bits ^ (bits >> 31 & 0x7fffffff)).long() << 32 | (x.shape[1] - 1 - v)
        index = x.shape[1] - 1 - (key.topk(top, dim=1).values & 0xffffffff)
        got["top_id"] = index.to(torch.int32)
        got["top_logprob"] = torch.gather(x, 1, index) - m - lse
    return got


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2601_01513_amd import binding as B
        if op == "logprobs":
            r = B.token_logprobs(s["logits"], s["tokens"], top=s["case"]["top"])
            got = {"logprob": r.logprob, "entropy": r.entropy, "rank": r.rank}
            if s["case"]["top"]:
                got.update(top_id=r.top_id, top_logprob=r.top_logprob)
            return got
        pages = B.pages(s["table"], s["len"], s["held"], s["refs"], s["case"]["page"])
        if op == "attend":
            B.tree_attention(pages, s["q"], s["k"], s["v"], s["scale"], start=s["start"],
                             mask=s["mask"], out=s["out"])
            return {"out": s["out"]}
        if op == "rows":
            pos, slot, mask = B.tree_rows(pages, s["start"], s["parent"], out=s["out"])
            return {"pos": pos, "slot": slot, "mask": mask}
        if op == "update":
            B.pages_update(pages, source=s["source"], room=s["room"], k=s["k"], v=s["v"],
                           ok=s["ok"])
            return {"ok": s["ok"], "table": s["table"], "len": s["len"], "held": s["held"],
                    "refs": s["refs"], "k": s["k"], "v": s["v"]}
        B.pages_keep(pages, s["kept"], s["n_kept"], s["k"], s["v"], len_out=s["len_out"],
                     release=False)
        return {"len": s["len_out"], "k": s["k"], "v": s["v"]}
    return {"attend": _attend_plain, "rows": _rows_plain, "update": _update_plain,
            "keep": _keep_plain, "logprobs": _logprobs_plain}[op](s)


def work(case):
    e = 4 if case.get("dtype") == "f32" else 2
    op = case["op"]
    if op == "logprobs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * e + case["rows"] * (16 + 8 * case["top"]), "flops": 5 * n}
    if op == "update":  # (the copied rows of a mean step, read and written)
        seqs = case["groups"] * case["beams"]
        rows = seqs / 2 * (min(case["page"], case["ctx"]) - 1) / 2
        token = 2 * case["layers"] * case["hk"] * case["hd"] * e
        pages = seqs * (case["ctx"] * 0.75 / case["page"] + 1)
        return {"bytes": 2 * rows * token + 12 * pages + 20 * seqs, "flops": 0}
    ctx, n = 0.75 * case["ctx"], (0.75 if case["n"] > 1 else 1) * case["n"]
    T = case["seqs"] * n
    if op == "rows":
        return {"bytes": T * (12 + 4 * _ceil(case["n"], 32)) + 16 * case["seqs"], "flops": 0}
    if op == "keep":
        token = 2 * case["layers"] * case["hk"] * case["hd"] * e
        moved = case["seqs"] * min(case["depth"] / 2, n / 6)
        return {"bytes": 2 * moved * token + 4 * case["seqs"] * (3 + case["depth"]), "flops": 0}
    keys = case["seqs"] * (ctx + n)
    return {"bytes": 2 * keys * case["hk"] * case["hd"] * e + 2 * T * case["hq"] * case["hd"] * e
            + 4 * keys / case["page"],
            "flops": 4 * T * (ctx + n / 2) * case["hq"] * case["hd"]}


# ---------------------------------------------------------------- exact values


def exact(case, seed):
    if case["op"] == "rows":
        return None  # (whole numbers alone)
    s = prepare(case, seed)
    return {"attend": _attend_exact, "update": _update_exact, "keep": _keep_exact,
            "logprobs": _logprobs_exact}[case["op"]](s)


def _attend_exact(s):
    c = s["case"]
    G, ps = c["hq"] // c["hk"], c["page"]
    table, length, start = s["table"].tolist(), s["len"].tolist(), s["start"].tolist()
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for i in range(c["seqs"]):
        b, n = start[i], start[i + 1] - start[i]
        L = length[i] + n
        slots = torch.tensor([table[i][p // ps] * ps + p % ps for p in range(L)], device="cuda")
        seen = torch.ones((n, L), dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            seen = seen.tril(length[i])
        else:
            for j in range(n):
                seen[:, length[i] + j] = (s["mask"][b:b + n, j // 32] >> j % 32 & 1).bool()
        for h in range(c["hq"]):
            k = s["k"][slots, h // G].double()
            x = (s["q"][b:b + n, h].double() @ k.t()) * s["scale"]
            x = torch.softmax(x.masked_fill(~seen, -math.inf), 1)
            out[b:b + n, h] = x @ s["v"][slots, h // G].double()
    return {"out": out}


def _update_exact(s):
    """One sequence after the other, pages as lists."""
    ps = s["case"]["page"]
    refs, source, room = s["refs"].tolist(), s["source"].tolist(), s["room"].tolist()
    length, held = s["len"].tolist(), s["held"].tolist()
    was = [row[:h] for row, h in zip(s["table"].tolist(), held)]
    for d, x in enumerate(source):
        if x != d:
            for p in was[d]:
                refs[p] -= 1
            for p in was[x][:length[x] // ps]:
                refs[p] += 1
            if length[x] % ps and source[x] != x and source.index(x) == d:
                refs[was[x][length[x] // ps]] += 1
    free = [p for p, n in enumerate(refs) if n == 0]
    k, v = s["k"].double(), s["v"].double()
    for d, x in enumerate(source):
        pages, n = _ceil(length[x], ps), length[x] % ps
        if x == d:
            pages = held[d]
        elif n and (source[x] == x or source.index(x) != d):
            old, new = was[x][length[x] // ps] * ps, free.pop(0) * ps
            k[:, new:new + n], v[:, new:new + n] = k[:, old:old + n], v[:, old:old + n]
        del free[:max(0, _ceil(length[x] + room[d], ps) - pages)]
    return {"ok": None, "table": None, "len": None, "held": None, "refs": None, "k": k, "v": v}


def _keep_exact(s):
    c = s["case"]
    ps = c["page"]
    k, v = s["k"].double(), s["v"].double()
    table, length = s["table"].tolist(), s["len"].tolist()
    kept, n_kept = s["kept"].tolist(), s["n_kept"].tolist()
    for i in range(c["seqs"]):
        slot = lambda p: table[i][p // ps] * ps + p % ps  # noqa: E731
        for j in range(n_kept[i]):
            to, at = slot(length[i] + j), slot(length[i] + kept[i][j])
            k[:, to], v[:, to] = k[:, at].clone(), v[:, at].clone()
    return {"len": None, "k": k, "v": v}


def _logprobs_exact(s):
    x = s["logits"].double()
    lse = torch.logsumexp(x, 1)
    entropy = lse - torch.stack([torch.dot(r.softmax(0), r) for r in x])
    rows = torch.arange(x.shape[0], device="cuda")
    got = {"logprob": x[rows, s["tokens"].long()] - lse, "entropy": entropy, "rank": None}
    if s["case"]["top"]:
        got["top_id"] = None
        got["top_logprob"] = x.topk(s["case"]["top"], dim=1).values - lse[:, None]
    return got
