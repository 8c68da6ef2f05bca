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


def token_distill(logits, ids, values, temperature=1.0, teacher="logp"):
    """dict of loss, the gradient d of each row's loss, and what their errors go by: q, q_rest, P, p_rest, y (exponents of base 2 below the others' largest logit).
    Rows without a teacher, -infinity throughout, or with NaN or +infinity as the header says."""
    z, t, ids = np.asarray(logits, np.float64), np.asarray(values, np.float64), np.asarray(ids)
    R, V = z.shape
    out = dict(loss=np.zeros(R), d=np.zeros((R, V)), q=np.zeros((R, V)), q_rest=np.zeros(R), P=np.zeros(R), p_rest=np.zeros(R), y=np.zeros((R, V)),
               listed=np.zeros((R, V), bool))
    for r in range(R):
        at = [k for k in range(ids.shape[1]) if 0 <= ids[r, k] < V]
        token, v = ids[r, at], t[r, at]
        with np.errstate(all="ignore"):
            if teacher == "logits" and len(at):
                u = v / temperature
                m = u.max() if np.isfinite(u.max()) or np.isnan(u.max()) else 0.0
                log_p = u - m - np.log(np.exp(u - m).sum()) if (np.isnan(u) | (u > -np.inf)).any() else u
            else:
                log_p = v
            p = np.exp(log_p)
        if not (p != 0).any():
            continue
        p_rest = max(0.0, 1.0 - p.sum()) if teacher == "logp" else 0.0
        row = z[r]
        if np.isnan(row).any() or np.isposinf(row).any() or np.isnan(p).any():
            out["loss"][r], out["d"][r] = np.nan, np.nan
            continue
        if np.isneginf(row).all():
            out["loss"][r] = np.inf
            continue
        e = np.exp((row - row.max()) / temperature)
        others = np.ones(V, bool)
        others[token] = False
        total = e[others].sum() + e[~others].sum()
        with np.errstate(divide="ignore", invalid="ignore"):
            log_q = (row - row.max()) / temperature - np.log(total)
            off = row[others & (row > -np.inf)]
            # the others' sum behind their own largest logit: it may be below what 64 bits hold beside the listed ones
            log_rest = (off.max() - row.max()) / temperature + np.log(np.exp((off - off.max()) / temperature).sum()) - np.log(total) if len(off) else -np.inf
            q_rest = np.exp(log_rest)
            if q_rest < 1e-300:
                p_rest = 0.0
            loss = np.where(p > 0, p * (log_p - log_q[token]), 0.0).sum() + (p_rest * (np.log(p_rest) - log_rest) if p_rest > 0 else 0.0)
        P, q = p.sum() + p_rest, e / total
        d = q * P
        np.subtract.at(d, token, p)
        if len(off):
            w = np.exp((np.where(others, row, -np.inf) - off.max()) / temperature)
            w = w / w.sum()                                             # q_v / q_r
            d = np.where(others, w * (q_rest * P - p_rest), d)
            with np.errstate(invalid="ignore"):
                out["y"][r] = np.where(others & (row > -np.inf), (off.max() - row) / temperature * np.log2(np.e), 0.0)
            q = np.where(others, w * q_rest, q)
        out["loss"][r], out["d"][r], out["q"][r], out["q_rest"][r], out["P"][r], out["p_rest"][r], out["listed"][r] = loss, d / temperature, q, q_rest, P, p_rest, ~others
    return out


def beam_select(logits, scores, top, ended=None, end_id=-1, rank_scale=None, temperature=1.0):
    """dict of scores, tokens, parents, ended, and the ranks that order them (with the one behind the last)."""
    scores = np.asarray(scores, np.float64)
    N, B = scores.shape
    z = np.asarray(logits, np.float64).reshape(N, B, -1)
    out = {n: [] for n in ("scores", "tokens", "parents", "ended", "ranks")}
    for n in range(N):
        found = []
        for b in range(B):
            scale = 1.0 if rank_scale is None else float(rank_scale[n, b])
            if not np.isfinite(scores[n, b]) or not (0 < scale < np.inf):
                continue
            if ended is not None and ended[n, b]:
                found.append((-scores[n, b] * scale, b, 0.0, end_id, scores[n, b], True))
                continue
            row = z[n, b]
            if np.isnan(row).any() or np.isposinf(row).any() or np.isneginf(row).all():
                continue
            down = (row - row.max()) / temperature
            with np.errstate(invalid="ignore"):
                score = scores[n, b] + (down - np.log(np.exp(down).sum()))
            keep = np.where(score >= -np.finfo(np.float32).max)[0]
            keep = keep[np.lexsort((keep, -row[keep]))][:top + 1]
            found += [(-score[v] * scale, b, -row[v], v, score[v], v == end_id) for v in keep]
        found.sort(key=lambda f: f[:4])
        taken = found[:top] + [(np.inf, 0, 0, -1, -np.inf, False)] * (top - len(found))
        out["scores"].append([f[4] for f in taken])
        out["tokens"].append([f[3] for f in taken])
        out["parents"].append([f[1] for f in taken])
        out["ended"].append([f[5] for f in taken])
        out["ranks"].append([-f[0] for f in found[:top + 1]] + [-np.inf] * (top + 1 - len(found)))
    return {n: np.array(v) for n, v in out.items()}


def beam_reorder(parents, state, beams, before=None, dim=0):
    """The state's rows in the order of the parents; `before`: what the output holds where a parent is outside."""
    state = np.moveaxis(np.asarray(state), dim, 0)
    N, top = parents.shape
    out = np.array(state if before is None else np.moveaxis(np.asarray(before), dim, 0))
    for n in range(N):
        for j in range(top):
            if 0 <= parents[n, j] < beams:
                out[n * top + j] = state[n * beams + parents[n, j]]
    return np.moveaxis(out, 0, dim)
