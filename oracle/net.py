"""Plain 64-bit forms of the operators of include/kan_net.h (numpy, on the host), from their definitions.

The `scale` of a result is the sum of the magnitudes of the terms it is added up from: what a rounding error in 32 bits is
relative to, whatever cancels.
"""
import numpy as np


def _norm(v, kind, eps):
    mean = v.mean(1, keepdims=True) if kind == "layer" else np.zeros((v.shape[0], 1))
    r = 1.0 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)
    return (v - mean) * r, mean, r


def _back(q, vhat, r, kind):
    out = q - vhat * (q * vhat).mean(1, keepdims=True)
    size = np.abs(q) + np.abs(vhat) * np.abs(q * vhat).mean(1, keepdims=True)
    if kind == "layer":
        out = out - q.mean(1, keepdims=True)
        size = size + np.abs(q).mean(1, keepdims=True)
    return out * r, size * r


def _gate(p, B, n, gate_rows):
    g = p.get("gate")
    if g is None:
        return np.ones((B, n))
    return np.asarray(g, np.float64)[np.arange(B) // gate_rows if gate_rows > 0 else np.zeros(B, int)]


def _of(p, name, n, none):
    return np.full(n, none) if p.get(name) is None else np.asarray(p[name], np.float64)


def block_norm(x, f, p, kind="rms", eps=1e-5, residual_scale=1.0, gate_rows=0):
    """dict: x_out, h, their scales, and what the backward pass needs."""
    x = np.asarray(x, np.float64)
    B, n = x.shape
    s = dict(x=x, f=f)
    if f is None:
        s["x_out"], s["x_out_scale"] = x, np.abs(x)
    else:
        s["fhat"], mean, s["rf"] = _norm(np.asarray(f, np.float64), kind, eps)
        s["u"] = s["fhat"] * _of(p, "w_post", n, 1.0) + _of(p, "b_post", n, 0.0)
        s["gate"] = _gate(p, B, n, gate_rows)
        s["x_out"] = residual_scale * x + s["gate"] * s["u"]
        # what the mean takes away is part of the terms
        u_scale = (np.abs(s["fhat"]) + np.abs(mean) * s["rf"]) * np.abs(_of(p, "w_post", n, 1.0)) + np.abs(_of(p, "b_post", n, 0.0))
        s["x_out_scale"] = np.abs(residual_scale * x) + np.abs(s["gate"]) * u_scale
    s["xhat"], mean, s["rx"] = _norm(s["x_out"], kind, eps)
    w = _of(p, "w_pre", n, 1.0)
    s["h"] = s["xhat"] * w + _of(p, "b_pre", n, 0.0)
    # an error of x_out counts in its own channel and, through sigma, in all
    s["spread"] = np.sqrt((s["x_out_scale"] ** 2).mean(1, keepdims=True)) * s["rx"]
    s["h_scale"] = ((s["x_out_scale"] + np.abs(mean)) * s["rx"] + np.abs(s["xhat"]) * s["spread"]) * np.abs(w) + np.abs(_of(p, "b_pre", n, 0.0)) + np.abs(s["h"])
    return s


def block_norm_backward(s, p, gx_out, gh, kind="rms", residual_scale=1.0, gate_rows=0):
    """(gradients, scales), from what block_norm returned."""
    B, n = s["x"].shape
    d = np.zeros((B, n)) if gx_out is None else np.asarray(gx_out, np.float64)
    size = np.abs(d)
    g, scale = {}, {}
    if gh is not None:
        gh = np.asarray(gh, np.float64)
        g["gw_pre"], scale["gw_pre"] = (gh * s["xhat"]).sum(0), np.abs(gh * s["xhat"]).sum(0)
        g["gb_pre"], scale["gb_pre"] = gh.sum(0), np.abs(gh).sum(0)
        back, more = _back(gh * _of(p, "w_pre", n, 1.0), s["xhat"], s["rx"], kind)
        d, size = d + back, size + more * (1.0 + s["spread"])
    if s["f"] is None:
        g["gx"], scale["gx"] = d, size
        return g, scale
    g["gx"], scale["gx"] = residual_scale * d, abs(residual_scale) * size
    gu, gu_size = d * s["gate"], size * np.abs(s["gate"])
    g["gw_post"], scale["gw_post"] = (gu * s["fhat"]).sum(0), (gu_size * np.abs(s["fhat"])).sum(0)
    g["gb_post"], scale["gb_post"] = gu.sum(0), gu_size.sum(0)
    w = _of(p, "w_post", n, 1.0)
    g["gf"], _ = _back(gu * w, s["fhat"], s["rf"], kind)
    _, scale["gf"] = _back(gu_size * np.abs(w), np.abs(s["fhat"]), s["rf"], kind)
    groups = -(-B // gate_rows) if gate_rows > 0 else 1
    at = np.arange(B) // gate_rows if gate_rows > 0 else np.zeros(B, int)
    u_size = np.abs(s["fhat"] * w) + np.abs(_of(p, "b_post", n, 0.0))
    for out, terms in ((g, d * s["u"]), (scale, size * u_size)):
        out["ggate"] = np.zeros((groups, n))
        np.add.at(out["ggate"], at, terms)
    return g, scale


def embedding(ids, table, scale):
    ids, table = np.asarray(ids), np.asarray(table, np.float64)
    there = (ids >= 0) & (ids < len(table))
    return np.where(there[..., None], table[np.where(there, ids, 0)] * scale, 0.0)


def embedding_backward(ids, gy, V, scale):
    ids, gy = np.asarray(ids).reshape(-1), np.asarray(gy, np.float64)
    gy = gy.reshape(len(ids), -1)
    there = (ids >= 0) & (ids < V)
    out = []
    for terms in (gy, np.abs(gy)):
        g = np.zeros((V, gy.shape[1]))
        np.add.at(g, ids[there], terms[there])
        out.append(g * scale)
    return out[0], np.abs(out[1])


def token_logprob(logits, ids, temperature=1.0, top=0):
    """dict of logp, entropy, p, and top_ids / top_logp; rows of nothing but -infinity and rows with NaN or +infinity as the header says."""
    z = np.asarray(logits, np.float64)
    R, V = z.shape
    wrong = np.isnan(z).any(1) | np.isposinf(z).any(1)
    empty = np.isneginf(z).all(1)
    m = np.where(empty | wrong, 0.0, np.where(wrong[:, None], 0.0, z).max(1))
    y = (np.where(wrong[:, None], 0.0, z) - m[:, None]) / temperature
    e = np.exp(y)
    others = e.copy()
    others[np.arange(R), y.argmax(1)] = 0.0
    rest = np.where(empty, 0.0, others.sum(1))          # the sum but for the largest logit's 1, which it would be rounded against
    p = e / (1.0 + rest)[:, None]
    lp = y - np.log1p(rest)[:, None]
    other_p = np.where((np.arange(V) == y.argmax(1)[:, None]) & ~empty[:, None], (rest / (1.0 + rest))[:, None], 1.0 - p)
    with np.errstate(invalid="ignore"):
        entropy = -np.where(p > 0, p * lp, 0.0).sum(1)
    entropy = np.where(wrong, np.nan, entropy)
    lp = np.where(wrong[:, None], np.nan, lp)
    p, other_p = np.where(wrong[:, None], np.nan, p), np.where(wrong[:, None], np.nan, other_p)
    out = dict(entropy=entropy, p=p, other_p=other_p, lp=lp, empty=empty)
    if ids is not None:
        ids = np.asarray(ids)
        there = (ids >= 0) & (ids < V)
        out["there"] = there
        out["logp"] = np.where(there, lp[np.arange(R), np.where(there, ids, 0)], 0.0)
    if top:
        key = np.where(np.isnan(z), np.inf, z)
        # NaN first, then by value; a stable sort keeps the lowest index first
        order = np.lexsort((np.broadcast_to(np.arange(V), z.shape), -key, ~np.isnan(z)), axis=1)
        out["top_ids"] = order[:, :top]
        out["top_logp"] = np.take_along_axis(lp, out["top_ids"], 1)
    return out


def token_logprob_backward(fwd, ids, g_logp, g_entropy, temperature=1.0):
    p, lp = fwd["p"], fwd["lp"]
    R = len(p)
    g = np.zeros_like(p)
    scale = np.zeros_like(p)
    if g_logp is not None:
        there = fwd["there"]
        a = np.where(there, np.asarray(g_logp, np.float64), 0.0)[:, None]
        hit = np.zeros_like(p)
        hit[np.arange(R)[there], np.asarray(ids)[there]] = 1.0
        g += np.where(hit > 0, a * fwd["other_p"], -a * p)
        scale += np.abs(a * p) + np.abs(a * hit)
    if g_entropy is not None:
        b = np.asarray(g_entropy, np.float64)[:, None]
        with np.errstate(invalid="ignore"):
            inner = np.where(p == 0, 0.0, p * (lp + fwd["entropy"][:, None]))
            size = np.where(p == 0, 0.0, p * (np.abs(lp) + np.abs(fwd["entropy"][:, None])))
        g -= b * inner
        scale += np.abs(b) * size
    g = np.where(fwd["empty"][:, None], 0.0, g / temperature)
    return g, np.where(fwd["empty"][:, None], 0.0, scale / temperature)


def clip(tensors, max_norm):
    """(norm, factor)"""
    norm = np.sqrt(sum((np.asarray(t, np.float64) ** 2).sum() for t in tensors))
    return norm, (max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0)
