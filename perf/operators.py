"""The rotary, head-norm and token-pick operators: cases, plain forms, exact values.

Each case is one call of one operator, at the sizes of this repository's own
workloads (workload.py) or generic ones:
  rope  multi-axis rotary positions on the queries and keys of stacked QKV rows;
        the keys go to slots of a key cache [n_kv][positions][head_dim];
  norm  the same with the RMSNorm of every query and key head before it;
  pick  penalties, bias and grammar mask on logits, and the greedy pick with
        its log-probability.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _heads(name, op, T, hq, hk, hd, rot, sections, interleaved, dtype, base=1e6):
    return {"name": name, "op": op, "T": T, "hq": hq, "hk": hk, "hd": hd, "rot": rot,
            "sections": sections, "interleaved": interleaved, "dtype": dtype, "base": base}


def _pick(name, rows, vocab, dtype, prompt, output, penalties, bias, mask, processed):
    return {"name": name, "op": "pick", "rows": rows, "vocab": vocab, "dtype": dtype,
            "prompt": prompt, "output": output, "penalties": penalties, "bias": bias,
            "mask": mask, "processed": processed}


def listed():
    return [
        # One decode step of 8 branches of the 7B-class model.
        _heads("rope decode 7B x8", "rope", 8, 28, 4, 128, 128, "16,24,24", False, "bf16"),
        # The prefix of the headline workload: video rows, then text.
        _heads("rope prefix 7B x4096", "rope", 4096, 28, 4, 128, 128, "16,24,24", False, "bf16"),
        # The long prefix at the widest model: the largest call.
        _heads("rope prefix 32B x16384", "rope", 16384, 40, 8, 128, 128, "16,24,24", False,
               "bf16"),
        # The small fp32 model, an odd number of rows, axes taking turns.
        _heads("rope fp32 small x773", "rope", 773, 4, 4, 64, 64, "12,10,10", True, "f32", 1e4),
        # One decode step of three drafts of the 3B-class drafter.
        _heads("norm decode 3B x3", "norm", 3, 16, 2, 128, 128, "24,20,20", True, "f16"),
        # The candidate rows of a ragged scoring call (16 of 32 to 128 tokens).
        _heads("norm candidates 7B x1283", "norm", 1283, 28, 4, 128, 128, "24,20,20", True,
               "f16"),
        # The prefix of the 32B-class workload.
        _heads("norm prefix 32B x8192", "norm", 8192, 40, 8, 128, 128, "24,20,20", True, "bf16"),
        # Wide fp32 heads of which a quarter is rotated, two axes (images).
        _heads("norm fp32 wide x1001", "norm", 1001, 8, 2, 256, 64, "16,16", False, "f32", 1e4),
        # One answer token under a grammar, logits in bf16.
        _pick("pick 1 x 152064 masked", 1, 152064, "bf16", 0, 0, False, "none", "shared", False),
        # Three drafts in mid-answer, every rule on.
        _pick("pick 3 x 151936 ruled", 3, 151936, "f32", 512, 64, True, "shared", "rows", False),
        # Sixteen long branches, the processed logits kept.
        _pick("pick 16 x 152064 kept", 16, 152064, "f16", 3900, 700, True, "none", "none", True),
        # The most branches a call may carry, every rule on, a bias a branch.
        _pick("pick 256 x 152064 full", 256, 152064, "f32", 300, 100, True, "rows", "rows", True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "norm", "pick"])
    if op == "pick":
        vocab = _log_int(rng, 1000, 152064)
        return {"op": "pick", "rows": _log_int(rng, 1, 200), "vocab": vocab,
                "dtype": rng.choice(["f32", "bf16", "f16"]),
                "prompt": rng.choice([0, _log_int(rng, 1, 4000)]),
                "output": rng.choice([0, _log_int(rng, 1, 1000)]),
                "penalties": rng.random() < 0.7, "bias": rng.choice(["none", "shared", "rows"]),
                "mask": rng.choice(["none", "shared", "rows"]), "processed": rng.random() < 0.5}
    hq, hk = rng.choice([(4, 4), (12, 2), (16, 2), (28, 4), (40, 8), (5, 5), (14, 1)])
    hd = rng.choice([64, 128, 128, 128, 256, 80, 36])
    rot = rng.choice([hd, hd, hd, hd // 4 * 2])
    n_axes, half = rng.choice([1, 2, 3, 3]), rot // 2
    interleaved = rng.random() < 0.5
    part = half // n_axes if interleaved else rng.randint(1, max(1, half // (n_axes + 1)))
    sections = [half - part * (n_axes - 1)] + [part] * (n_axes - 1)
    dtype = rng.choice(["bf16", "f16", "bf16", "f32"])
    most = 16384 * 48 * 128 * 2 // ((hq + hk) * hd * (4 if dtype == "f32" else 2))
    return {"op": op, "T": _log_int(rng, 1, min(most, 20000)), "hq": hq, "hk": hk, "hd": hd,
            "rot": rot, "sections": ",".join(map(str, sections)), "interleaved": interleaved,
            "dtype": dtype, "base": rng.choice([1e4, 1e6])}


def _sections(case):
    return tuple(int(s) for s in case["sections"].split(","))


def _axis_of_pair(case):
    """The position axis that turns each pair, in pair order."""
    sec = _sections(case)
    n, half = len(sec), case["rot"] // 2
    if case["interleaved"]:
        return [i % n if i < n * sec[i % n] else 0 for i in range(half)]
    return [a for a in range(n) for _ in range(sec[a])]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def ints(lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=g, device=dev, dtype=torch.int32)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    if case["op"] == "pick":
        R, V = case["rows"], case["vocab"]
        s = {"case": case, "logits": (normal(R, V) * 3).to(dt), "prompt": None, "output": None,
             "prompt_len": None, "output_len": None, "repetition": None, "presence": None,
             "frequency": None, "bias": None, "mask": None, "processed": None}
        # Token ids as text has them: a few often, most never.
        skewed = lambda n: (torch.rand((R, n), generator=g, device=dev) ** 3 * V).to(torch.int32)  # noqa: E731
        for key in ("prompt", "output"):
            if case[key]:
                s[key] = skewed(case[key])
                s[key + "_len"] = ints(max(1, case[key] // 2), case[key] + 1, (R,))
        if case["penalties"]:
            s["repetition"] = 1.0 + 0.3 * torch.rand(R, generator=g, device=dev)
            s["presence"] = 0.5 * torch.rand(R, generator=g, device=dev)
            s["frequency"] = 0.2 * torch.rand(R, generator=g, device=dev)
        if case["bias"] != "none":
            n = 1 if case["bias"] == "shared" else R
            rare = torch.rand((n, V), generator=g, device=dev) < 0.01
            s["bias"] = torch.where(rare, normal(n, V) * 4, 0.0)
        if case["mask"] != "none":
            n = 1 if case["mask"] == "shared" else R
            s["mask"] = ints(-(1 << 31), (1 << 31) - 1, (n, (V + 31) // 32))
            if n > 2:
                s["mask"][n // 2] = 0  # a grammar that allows nothing here
        if case["processed"]:
            s["processed"] = torch.empty((R, V), device=dev)
        s["token"] = torch.empty(R, dtype=torch.int32, device=dev)
        s["logprob"] = torch.empty(R, device=dev)
        return s

    T, hq, hk, hd = case["T"], case["hq"], case["hk"], case["hd"]
    sec = _sections(case)
    qkv = (normal(T, hq + 2 * hk, hd) * (0.25 + 2 * torch.rand(hq + 2 * hk, 1, generator=g, device=dev))).to(dt)
    # Video rows (time, height, width) then text, where every axis counts on.
    grid = max(1, int(math.sqrt(T / 16)))
    start, t = int(ints(0, 20000, (1,)).item()), torch.arange(T, device=dev)
    video = torch.stack([t // (grid * grid), t // grid % grid, t % grid, t % 3])[:len(sec)]
    text = t.expand(len(sec), T)
    pos = (torch.where(t < T // 2, video, text) + start).to(torch.int32).contiguous()
    cap = T + 64
    first = int(ints(0, 64, (1,)).item())
    s = {"case": case, "q": qkv[:, :hq], "k": qkv[:, hq:hq + hk], "pos": pos,
         "axis": torch.tensor(_axis_of_pair(case), device=dev), "sections": sec,
         "q_out": torch.empty((T, hq, hd), dtype=dt, device=dev),
         "cache": normal(hk, cap, hd).to(dt),
         "rows": (first + t).to(torch.int32), "q_gain": None, "k_gain": None}
    if case["op"] == "norm":
        s["q_gain"], s["k_gain"] = ((1 + 0.2 * normal(hd)).to(dt) for _ in range(2))
    return s


def _norm(x, gain):
    x = x.float()
    if gain is None:
        return x
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gain.float()


def _turn(x, cos, sin):
    half = cos.shape[-1]
    a, b = x[..., :half], x[..., half:2 * half]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1)


def _heads_plain(s):
    c = s["case"]
    i = torch.arange(c["rot"] // 2, device=s["pos"].device, dtype=torch.float64)
    angle = s["pos"][s["axis"]].double().T * c["base"] ** (-2 * i / c["rot"])
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q = _turn(_norm(s["q"], s["q_gain"]), cos, sin)
    k = _turn(_norm(s["k"], s["k_gain"]), cos, sin)
    s["cache"][:, s["rows"].long()] = k.transpose(0, 1).to(s["cache"].dtype)
    return {"q": q.to(s["q"].dtype), "k": s["cache"]}


def _counts(ids, length, like):
    if ids is None:
        return torch.zeros_like(like)
    valid = torch.arange(ids.shape[1], device=ids.device) < length[:, None]
    return torch.zeros_like(like).scatter_add_(1, ids.long(), valid.float())


def _pick_plain(s):
    x = s["logits"].float()
    if s["repetition"] is not None:
        out = _counts(s["output"], s["output_len"], x)
        seen = out + _counts(s["prompt"], s["prompt_len"], x) > 0
        r = s["repetition"][:, None]
        x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
        x = x - (s["frequency"][:, None] * out + s["presence"][:, None] * (out > 0))
    if s["bias"] is not None:
        x = x + s["bias"]
    v = torch.arange(x.shape[1], device=x.device, dtype=torch.int32)
    if s["mask"] is not None:
        x = torch.where((s["mask"][:, v // 32] >> v % 32 & 1) == 1, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    none = top[:, 0] == -math.inf
    token = torch.where(x == top, v, x.shape[1]).amin(-1).to(torch.int32)
    logprob = -(x - top).exp().sum(-1).log()
    got = {"token": torch.where(none, -1, token), "logprob": torch.where(none, -math.inf, logprob)}
    if s["processed"] is not None:
        got["processed"] = x
    return got


def run(s):
    c = s["case"]
    if own:
        from paper_2601_01513_amd import binding
        if c["op"] == "pick":
            token, logprob = binding.pick_tokens(
                s["logits"], prompt=s["prompt"], prompt_len=s["prompt_len"], output=s["output"],
                output_len=s["output_len"], repetition=s["repetition"], presence=s["presence"],
                frequency=s["frequency"], bias=s["bias"], mask=s["mask"],
                processed=s["processed"], out=(s["token"], s["logprob"]))
            got = {"token": token, "logprob": logprob}
            if s["processed"] is not None:
                got["processed"] = s["processed"]
            return got
        rot = binding.rotary(s["sections"], c["base"], interleaved=c["interleaved"])
        if c["op"] == "norm":
            binding.qk_norm_rope(rot, s["pos"], s["q"], s["k"], s["q_gain"], s["k_gain"], 1e-6,
                                 q_out=s["q_out"], k_out=s["cache"].transpose(0, 1),
                                 k_rows=s["rows"])
        else:
            binding.rope_axes(rot, s["pos"], s["q"], s["k"], q_out=s["q_out"],
                              k_out=s["cache"].transpose(0, 1), k_rows=s["rows"])
        return {"q": s["q_out"], "k": s["cache"]}
    return _pick_plain(s) if c["op"] == "pick" else _heads_plain(s)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "pick":
        n = case["rows"] * case["vocab"]
        rows = {"none": 0, "shared": 1, "rows": case["rows"]}
        b = (n * e + 4 * n * case["processed"] + 4 * case["rows"] * (case["prompt"] + case["output"])
             + rows[case["bias"]] * case["vocab"] * 4 + rows[case["mask"]] * case["vocab"] / 8
             + 8 * case["rows"])
        return {"bytes": b, "flops": n * (3 + 4 * case["penalties"] + (case["bias"] != "none"))}
    n = case["T"] * (case["hq"] + case["hk"]) * case["hd"]
    norm = case["op"] == "norm"
    axes = len(_sections(case))
    return {"bytes": 2 * n * e + 4 * case["T"] * (axes + 1) + 2 * case["hd"] * e * norm,
            "flops": n * (3 + 4 * norm)}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "pick":
        return _pick_exact(case, s)
    T, half = case["T"], case["rot"] // 2
    step = [2 * math.pi * math.exp(-2 * i / case["rot"] * math.log(case["base"])) / (2 * math.pi)
            for i in range(half)]
    axis = _axis_of_pair(case)
    turn = torch.stack([s["pos"][axis[i]].to(torch.float64) * step[i] for i in range(half)], 1)
    turn = torch.polar(torch.ones_like(turn), turn).view(T, 1, half)
    got = []
    for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
        x = x.to(torch.float64)
        if gain is not None:
            x = x / ((x * x).sum(-1, keepdim=True) / case["hd"] + 1e-6).sqrt() * gain.double()
        z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * turn
        got.append(torch.cat([z.real, z.imag, x[..., 2 * half:]], -1))
    cache = s["cache"].double()
    cache.index_copy_(1, s["rows"].long(), got[1].permute(1, 0, 2).contiguous())
    return {"q": got[0], "k": cache}


def _pick_exact(case, s):
    rows = []
    for r in range(case["rows"]):
        x = s["logits"][r].double()
        if s["repetition"] is not None:
            told = [s[key][r, :int(s[key + "_len"][r])].long() for key in ("prompt", "output")
                    if s[key] is not None]
            every = torch.cat(told).unique() if told else None
            if every is not None:
                rep, old = float(s["repetition"][r]), x[every]
                x[every] = old.clamp(min=0) / rep + old.clamp(max=0) * rep
            if s["output"] is not None:
                ids, n = told[-1].unique(return_counts=True)
                x[ids] -= n * float(s["frequency"][r]) + float(s["presence"][r])
        if s["bias"] is not None:
            x = x + s["bias"][r % s["bias"].shape[0]].double()
        if s["mask"] is not None:
            words = s["mask"][r % s["mask"].shape[0]].long()
            bits = words[:, None].bitwise_right_shift(torch.arange(32, device=x.device)) & 1
            x = x.masked_fill(bits.flatten()[:case["vocab"]] == 0, -math.inf)
        rows.append(x)
    x = torch.stack(rows)
    best = x.max(-1).values
    logprob = best - torch.logsumexp(x, -1)
    got = {"token": None, "logprob": torch.where(best == -math.inf, best, logprob)}
    if s["processed"] is not None:
        got["processed"] = x
    return got
