"""Float64 decoder with positions on several axes and norms of query and key
heads, one whole sequence at a time (no cache): what contexts with
vsr_set_positions and vsr_load_qk_norms are compared with. The steps both share
with the plain decoder are the oracle's."""
import numpy as np

from oracle import decoder as D


def axis_of_pair(sections, interleaved):
    """The axis that turns each pair: runs of sections[x] pairs, or axes in turn."""
    n, half = len(sections), sum(sections)
    if interleaved:
        return np.array([i % n if i < n * sections[i % n] else 0 for i in range(half)])
    return np.repeat(np.arange(n), sections)


def rope(x, pos, axis, base):
    """x [T][H][hd], pos [axes][T], axis [rot / 2]: dims (i, i + rot/2) turned by
    pos[axis[i]] * base^(-2 i / rot), the rest as they are."""
    half = len(axis)
    i = np.arange(half, dtype=np.float64)
    ang = pos.astype(np.float64)[axis].T * base ** (-2.0 * i / (2 * half))
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:2 * half]
    return np.concatenate([a * c - b * s, b * c + a * s, x[..., 2 * half:]], -1)


def hidden(cfg, hw, x, pos, axis):
    """Final hidden rows of one causal sequence of layer-0 rows x at pos [axes][T]."""
    n = x.shape[0]
    hq, hkv, hd, f = cfg.n_heads, cfg.n_kv_heads, cfg.head_dim, cfg.d_ff
    order = np.arange(n)
    for lw in hw["layers"]:
        w = {k: np.asarray(v, np.float64) for k, v in lw.items()}
        qkv = D.rms_norm(x, w["attn_norm"], cfg.rms_eps) @ w["wqkv"].T
        q, k, v = np.split(qkv.reshape(n, hq + 2 * hkv, hd), [hq, hq + hkv], axis=1)
        if "q_norm" in w:
            q = D.rms_norm(q, w["q_norm"], cfg.rms_eps)
            k = D.rms_norm(k, w["k_norm"], cfg.rms_eps)
        q, k = (rope(t, pos, axis, cfg.rope_base) for t in (q, k))
        a = D.causal_attention(q, k, v, order, order)
        x = x + a.reshape(n, hq * hd) @ w["wo"].T
        gu = D.rms_norm(x, w["ffn_norm"], cfg.rms_eps) @ w["wgu"].T
        x = x + (D.silu(gu[:, :f]) * gu[:, f:]) @ w["wdown"].T
    return x


def logits_after(cfg, hw, visual, prefix_ids, branch, pos, next_pos, axis):
    """Logits [1 + len(branch)][vocab] at the last prefix row and after every
    branch token; branch token j sits at next_pos + j on every axis."""
    e = np.asarray(hw["embed"], np.float64)
    x = np.concatenate([np.asarray(visual, np.float64).reshape(-1, cfg.d_model),
                        e[np.asarray(prefix_ids)], e[np.asarray(branch, dtype=int)]])
    own = np.tile(next_pos + np.arange(len(branch)), (pos.shape[0], 1))
    h = hidden(cfg, hw, x, np.concatenate([pos, own], 1), axis)[pos.shape[1] - 1:]
    h = D.rms_norm(h, np.asarray(hw["final_norm"], np.float64), cfg.rms_eps)
    return h @ np.asarray(hw["lm_head"], np.float64).T


def apply_rules(x, prompt, output, repetition=None, presence=None, frequency=None, bias=None,
                mask=None):
    """One row of logits after the rules, in x's type, a rounding after every step."""
    t = x.dtype.type
    x = x.copy()
    keep = lambda ids: np.asarray([i for i in ids if 0 <= i < len(x)], dtype=int)  # noqa: E731
    count = np.bincount(keep(output), minlength=len(x))
    seen = (count + np.bincount(keep(prompt), minlength=len(x))) > 0
    with np.errstate(invalid="ignore", over="ignore"):
        if repetition is not None:
            r = t(repetition)
            x = np.where(seen, np.where(x > 0, x / r, x * r), x)
        if presence is not None or frequency is not None:
            f, p = t(frequency or 0), t(presence or 0)
            x = np.where(count > 0, x - (f * count.astype(x.dtype) + p), x)
        if bias is not None:
            x = x + bias.astype(x.dtype)
        if mask is not None:
            v = np.arange(len(x))
            x = np.where(mask.astype(np.uint32)[v // 32] >> (v % 32).astype(np.uint32) & 1 == 1,
                         x, t(-np.inf))
    return x.astype(t)
