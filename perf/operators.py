"""Performance cases of the operators that a residual KAN network on tokens needs around its layers.

A case is a dict of plain values; `kind` names the operator and `train` says whether a pass is a training step of it (forward
and every gradient) or the forward call of a server:

  norm     the norm before a block and the norm, gate and residual scale after it, fused over a block boundary:
             u = norm(f) * w_post + b_post,   x_out = residual_scale * x + gate * u,   h = norm(x_out) * w_pre + b_pre
  embed    rows of an embedding table by token, scaled; its dense gradient, summed over equal tokens in the order of the batch
  logprob  log probability of a given token of every row of logits, the row's entropy, and its most likely tokens
  clip     the norm over all gradients of a network, and the gradients scaled to it

`run` computes these in elementary torch operations, or through the framework's entry points where `own` is true.
`exact` is the definition in 64 bits, with gradients by automatic differentiation.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one token each of four requests between two blocks of a small network: latency is all there is
        dict(name="norm-serve-4x256", kind="norm", train=False, B=4, n=256, norm="rms", stream="f32", branch="f32", gate_rows=0, api="autograd"),
        # the 512 -> 512 layer of the benchmark as a residual block, at its batch
        dict(name="norm-train-16384x512", kind="norm", train=True, B=16384, n=512, norm="layer", stream="f32", branch="f32", gate_rows=0, api="binding"),
        # a width that is no multiple of anything; one gate for each sequence of 117 tokens; a bfloat16 stream around fp32 layers
        dict(name="norm-train-8190x771", kind="norm", train=True, B=8190, n=771, norm="layer", stream="bf16", branch="f32", gate_rows=117, api="autograd"),
        # a wide network's step, all activations in bfloat16
        dict(name="norm-train-16384x4096", kind="norm", train=True, B=16384, n=4096, norm="rms", stream="bf16", branch="bf16", gate_rows=0, api="binding"),
        # the tokens of a serving step
        dict(name="embed-serve-8", kind="embed", train=False, T=8, V=32768, n=512, table="bf16", out="f32", api="autograd"),
        # a training batch on a middling vocabulary, in fp32
        dict(name="embed-train-16384", kind="embed", train=True, T=16384, V=50001, n=512, table="f32", out="f32", api="binding"),
        # the largest table
        dict(name="embed-train-65536", kind="embed", train=True, T=65536, V=131072, n=2048, table="bf16", out="bf16", api="binding"),
        # sixteen requests' next tokens with five alternatives each
        dict(name="logprob-serve-16x32768", kind="logprob", train=False, R=16, V=32768, pad=0, type="bf16", top=5, api="autograd"),
        # the loss of a training batch: odd sizes, rows of a padded buffer
        dict(name="logprob-train-4093x50001", kind="logprob", train=True, R=4093, V=50001, pad=47, type="f32", top=0, api="autograd"),
        # the loss at the largest vocabulary, alternatives for the log
        dict(name="logprob-train-8192x131072", kind="logprob", train=True, R=8192, V=131072, pad=0, type="bf16", top=8, api="binding"),
        # the regression network of two layers (2 -> 5 -> 1)
        dict(name="clip-2-5-1", kind="clip", layers=1, n_in=2, n_out=5, G=8, type="f32", scale=3.0),
        # a stack of sixteen wide layers
        dict(name="clip-16x1024", kind="clip", layers=16, n_in=1024, n_out=1024, G=20, type="f32", scale=1e-3),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind, api = rng.choice(["norm", "norm", "embed", "logprob", "logprob", "clip"]), rng.choice(["binding", "autograd"])
    train = rng.random() < 0.6
    if kind == "norm":
        n = _log(rng, 64, 8192)
        B = _log(rng, 256, max(256, (1 << 26) // n)) if train else _log(rng, 1, 4096)
        stream = rng.choice(["f32", "bf16"])
        if stream == "f32":
            B = max(1, B // 2)
        return dict(kind=kind, train=train, B=B, n=n, norm=rng.choice(["rms", "layer"]), stream=stream,
                    branch="f32" if stream == "f32" else rng.choice(["f32", "bf16"]), gate_rows=rng.choice([0, 0, 1, _log(rng, 2, 2048)]), api=api)
    if kind == "embed":
        n, table = _log(rng, 64, 4096), rng.choice(["f32", "bf16"])
        T, V = _log(rng, 64, 65536) if train else _log(rng, 1, 4096), _log(rng, 256, 131072)
        return dict(kind=kind, train=train, T=min(T, (1 << 26) // n), V=min(V, (1 << 27) // n), n=n, table=table,
                    out="f32" if table == "f32" else rng.choice(["f32", "bf16"]), api=api)
    if kind == "logprob":
        V = _log(rng, 64, 131072)
        R = _log(rng, 64, 16384) if train else _log(rng, 1, 1024)
        return dict(kind=kind, train=train, R=max(1, min(R, (1 << 28) // V)), V=V, pad=rng.choice([0, 0, rng.randint(1, 64)]), type=rng.choice(["f32", "bf16"]),
                    top=rng.choice([0, 1, 5, 20]), api=api)
    n_in, n_out, G = _log(rng, 2, 1024), _log(rng, 1, 1024), _log(rng, 5, 64)
    layers = max(1, min(_log(rng, 1, 64), (1 << 27) // (n_in * n_out * (G + 5))))
    return dict(kind=kind, layers=layers, n_in=n_in, n_out=n_out, G=G, type=rng.choice(["f32", "f32", "bf16"]), scale=rng.choice([1e-4, 1e-2, 1.0]))


# ---- inputs ---------------------------------------------------------------------------------

def _normal(gen, std, *shape):
    return torch.randn(shape, generator=gen, device="cuda") * std


def _tokens(gen, n, V, ignored):
    """Tokens by rank-frequency: half the mass on about the square root of the vocabulary; a share has no token (-1)."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    order = torch.randperm(V, generator=gen, device="cuda")
    ids = order[ids]
    if ignored:
        ids[torch.rand(n, generator=gen, device="cuda") < ignored] = -1
    return ids


def _gate_groups(case):
    return 1 if case["gate_rows"] == 0 else -(-case["B"] // case["gate_rows"])


def _prepare_norm(case, gen):
    B, n = case["B"], case["n"]
    stream, branch = DTYPES[case["stream"]], DTYPES[case["branch"]]
    channel = torch.exp(_normal(gen, 0.5, n))                      # channels differ in size, as they do in trained networks
    s = dict(x=(_normal(gen, 1.5, B, n) * channel + 0.2).to(stream), f=(_normal(gen, 1.0, B, n) * channel.flip(0) - 0.1).to(branch))
    p = dict(w_post=1.0 + _normal(gen, 0.1, n), gate=_normal(gen, 0.5, _gate_groups(case), n), w_pre=1.0 + _normal(gen, 0.1, n))
    if case["norm"] == "layer":
        p.update(b_post=_normal(gen, 0.1, n), b_pre=_normal(gen, 0.1, n))
    s["p"] = p
    if case["train"]:
        s["gx_out"] = _normal(gen, 1.0 / math.sqrt(B), B, n).to(stream)
        s["gh"] = _normal(gen, 1.0 / math.sqrt(B), B, n).to(branch)
    return s


def _prepare_embed(case, gen):
    T, V, n = case["T"], case["V"], case["n"]
    s = dict(ids=_tokens(gen, T, V, 0.01 if case["train"] else 0.0), table=_normal(gen, 1.0 / math.sqrt(n), V, n).to(DTYPES[case["table"]]),
             scale=math.sqrt(n))
    if case["train"]:
        s["gy"] = _normal(gen, 1.0 / math.sqrt(T), T, n).to(DTYPES[case["out"]])
    return s


def _prepare_logprob(case, gen):
    R, V = case["R"], case["V"]
    logits = _normal(gen, 2.0, R, V + case["pad"])
    logits[:, :max(1, V // 64)] += 3.0                             # tokens that are common everywhere
    masked = V // 50
    if masked:
        logits[:, V - masked:V] = -math.inf                        # the end of a vocabulary that was filled up to a round size
    s = dict(logits=logits.to(DTYPES[case["type"]])[:, :V], ids=_tokens(gen, R, V - masked, 0.02 if case["train"] else 0.0))
    if case["train"]:
        s["g_logp"] = -torch.rand(R, generator=gen, device="cuda") / R
        s["g_entropy"] = torch.full((R,), -0.01 / R, device="cuda")
    return s


def _clip_shapes(case):
    i, o, rows = case["n_in"], case["n_out"], case["G"] + 3
    if case["layers"] == 1:                                        # the two layers of a regression network
        return [(i, rows, o), (i, o), (i, o), (o, 2 * case["G"] + 3, 1), (o, 1), (o, 1)]
    return [(i, rows, o), (i, o), (i, o)] * case["layers"]


def _prepare_clip(case, gen):
    dtype, shapes = DTYPES[case["type"]], _clip_shapes(case)
    grads = [_normal(gen, case["scale"], *shape).to(dtype) for shape in shapes]
    # the scaled gradients go where the optimizer reads them: one buffer, each tensor behind the other
    flat = torch.empty(sum(g.numel() for g in grads), dtype=dtype, device="cuda")
    out, at = [], 0
    for g in grads:
        out.append(flat[at:at + g.numel()].view(g.shape))
        at += g.numel()
    return dict(grads=grads, flat=flat, out=out, max_norm=1.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"norm": _prepare_norm, "embed": _prepare_embed, "logprob": _prepare_logprob, "clip": _prepare_clip}[case["kind"]](case, gen)
    s["case"] = case
    if own:
        _own_buffers(s)
    return s


# ---- plain forms ----------------------------------------------------------------------------

def _plain_norm(v, w, b, kind, eps):
    """xhat, 1/sigma and the normed rows, in 32 bits."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + eps)
    xhat = v * r
    y = xhat * w
    return xhat, r, y if b is None else y + b


def _plain_norm_back(g, xhat, r, kind):
    """The gradient of the rows a norm has read, from that of xhat."""
    back = g - xhat * (g * xhat).mean(1, keepdim=True)
    if kind == "layer":
        back = back - g.mean(1, keepdim=True)
    return back * r


def _run_norm_plain(s):
    case, p, kind = s["case"], s["p"], s["case"]["norm"]
    stream, branch, rows = DTYPES[case["stream"]], DTYPES[case["branch"]], case["gate_rows"]
    x, f, gate = s["x"].float(), s["f"].float(), p["gate"]
    if rows:
        group = torch.arange(case["B"], device="cuda") // rows
        gate = gate[group]
    fhat, rf, u = _plain_norm(f, p["w_post"], p.get("b_post"), kind, EPS)
    xo = RESIDUAL_SCALE * x + gate * u
    xhat, rx, h = _plain_norm(xo, p["w_pre"], p.get("b_pre"), kind, EPS)
    out = dict(x_out=xo.to(stream), h=h.to(branch))
    if not case["train"]:
        return out
    gh = s["gh"].float()
    d = s["gx_out"].float() + _plain_norm_back(gh * p["w_pre"], xhat, rx, kind)
    gu = d * gate
    out["gx"] = (RESIDUAL_SCALE * d).to(stream)
    out["gf"] = _plain_norm_back(gu * p["w_post"], fhat, rf, kind).to(branch)
    out["gw_post"], out["gw_pre"] = (gu * fhat).sum(0), (gh * xhat).sum(0)
    du = d * u
    out["ggate"] = torch.zeros_like(p["gate"]).index_add_(0, group, du) if rows else du.sum(0, keepdim=True)
    if kind == "layer":
        out["gb_post"], out["gb_pre"] = gu.sum(0), gh.sum(0)
    return out


def _run_embed_plain(s):
    ids, table, scale, out = s["ids"], s["table"], s["scale"], DTYPES[s["case"]["out"]]
    there = (ids >= 0) & (ids < table.shape[0])
    at = torch.where(there, ids, 0)
    r = dict(y=(table[at].float() * (there * scale).unsqueeze(1)).to(out))
    if s["case"]["train"]:
        g = torch.zeros(table.shape, dtype=torch.float32, device="cuda")
        g.index_add_(0, at, s["gy"].float() * (there * scale).unsqueeze(1))
        r["gtable"] = g.to(table.dtype)
    return r


def _plain_top(z, top):
    """Indices of the largest values of each row, the lowest index first among equal ones: unique whole-number keys."""
    bits = z.contiguous().view(torch.int32).to(torch.int64)
    key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) << 32
    key = key + (0xFFFFFFFF - torch.arange(z.shape[1], device="cuda"))
    return key.topk(top, dim=1).indices


def _run_logprob_plain(s):
    case, ids = s["case"], s["ids"]
    z = s["logits"].float() * (1.0 / TEMPERATURE)
    there = (ids >= 0) & (ids < z.shape[1])
    at = torch.where(there, ids, 0).unsqueeze(1)
    m = z.amax(1, keepdim=True)
    c = z - m
    e = torch.exp(c)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    ec = torch.where(e > 0, e * c, 0.0)
    entropy = log_total - ec.sum(1, keepdim=True) / total
    r = dict(logp=torch.where(there, (c.gather(1, at) - log_total)[:, 0], 0.0), entropy=entropy[:, 0])
    if case["top"]:
        best = _plain_top(s["logits"].float(), min(case["top"], z.shape[1]))
        r["top_ids"], r["top_logp"] = best, c.gather(1, best) - log_total
    if case["train"]:
        pr = e / total
        g_lp = torch.where(there, s["g_logp"], 0.0).unsqueeze(1)
        inner = torch.where(pr > 0, c - log_total + entropy, 0.0)
        g = -pr * (g_lp + s["g_entropy"].unsqueeze(1) * inner)
        g.scatter_add_(1, at, g_lp)
        r["glogits"] = (g * (1.0 / TEMPERATURE)).to(s["logits"].dtype)
    return r


def _run_clip_plain(s):
    total = sum((g.float() ** 2).sum() for g in s["grads"])
    norm = torch.sqrt(total)
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * factor)
    return dict(norm=norm, out=s["flat"])


EPS, RESIDUAL_SCALE, TEMPERATURE = 1e-5, 0.9, 0.8


# ---- the framework's operators --------------------------------------------------------------

def _own_buffers(s):
    """What a program keeps beside its inputs: the description of the operator, outputs and workspaces of the binding's calls."""
    from paper_2408_11200_amd import net, workloads
    case = s["case"]
    kind, train, binding = case["kind"], case.get("train"), case.get("api") == "binding"
    workspace = lambda n: torch.empty(max(int(n), 256), dtype=torch.uint8, device="cuda")
    if kind == "norm":
        spec = s["spec"] = workloads.BlockNormSpec(case["n"], case["norm"], EPS, RESIDUAL_SCALE, case["gate_rows"])
        if binding:
            s["x_out"], s["h"] = torch.empty_like(s["x"]), torch.empty_like(s["f"])
            if train:
                s["stats"] = torch.empty((case["B"], 4), device="cuda")
                s["g"] = dict(gx=torch.empty_like(s["x"]), gf=torch.empty_like(s["f"]), **{"g" + n: torch.empty_like(t) for n, t in s["p"].items()})
                s["ws"] = workspace(net.kan_block_norm_workspace_bytes(spec, case["B"]))
        elif train:
            s["x"].requires_grad_(True), s["f"].requires_grad_(True)
            for t in s["p"].values():
                t.requires_grad_(True)
    elif kind == "embed":
        if binding:
            s["y"] = torch.empty((case["T"], case["n"]), dtype=DTYPES[case["out"]], device="cuda")
            if train:
                s["gtable"] = torch.empty_like(s["table"])
                s["ws"] = workspace(net.kan_embedding_workspace_bytes(case["T"], case["V"], case["n"]))
        elif train:
            s["table"].requires_grad_(True)
    elif kind == "logprob":
        if binding:
            R, top = case["R"], min(case["top"], case["V"])
            s["o"] = dict(logp=torch.empty(R, device="cuda"), entropy=torch.empty(R, device="cuda"), stats=torch.empty((R, 2), device="cuda"))
            if top:
                s["o"].update(top_ids=torch.empty((R, top), dtype=torch.int64, device="cuda"), top_logp=torch.empty((R, top), device="cuda"))
            s["ws"] = workspace(net.kan_token_logprob_workspace_bytes(R, case["V"], top))
            if train:
                s["glogits"] = torch.empty((R, case["V"]), dtype=s["logits"].dtype, device="cuda")
        elif train:
            s["logits"].requires_grad_(True)


def _run_norm_own(s):
    from paper_2408_11200_amd import autograd, net
    case, spec, p = s["case"], s["spec"], s["p"]
    if case["api"] == "binding":
        x_out, h = net.kan_block_norm_forward(spec, s["x"], s["f"], p, x_out=s["x_out"], h=s["h"], stats=s.get("stats"))
        out = dict(x_out=x_out, h=h)
        if case["train"]:
            out.update(net.kan_block_norm_backward(spec, s["x"], s["f"], p, s["stats"], s["gx_out"], s["gh"], out=s["g"], ws=s["ws"]))
        return out
    if not case["train"]:
        with torch.no_grad():
            x_out, h = autograd.block_norm(spec, s["x"], s["f"], **p)
        return dict(x_out=x_out, h=h)
    x_out, h = autograd.block_norm(spec, s["x"], s["f"], **p)
    names = ["x", "f"] + list(p)
    g = torch.autograd.grad([x_out, h], [s["x"], s["f"]] + list(p.values()), [s["gx_out"], s["gh"]])
    return dict(x_out=x_out.detach(), h=h.detach(), **{"g" + n: t for n, t in zip(names, g)})


def _run_embed_own(s):
    from paper_2408_11200_amd import autograd, net
    case, out = s["case"], DTYPES[s["case"]["out"]]
    if case["api"] == "binding":
        r = dict(y=net.kan_embedding_forward(s["ids"], s["table"], s["scale"], y=s["y"]))
        if case["train"]:
            r["gtable"] = net.kan_embedding_backward(s["ids"], s["gy"], case["V"], s["scale"], gtable=s["gtable"], ws=s["ws"])
        return r
    if not case["train"]:
        with torch.no_grad():
            return dict(y=autograd.embedding(s["ids"], s["table"], s["scale"], out))
    y = autograd.embedding(s["ids"], s["table"], s["scale"], out)
    return dict(y=y.detach(), gtable=torch.autograd.grad(y, s["table"], s["gy"])[0])


def _run_logprob_own(s):
    from paper_2408_11200_amd import autograd, net
    case, top = s["case"], min(s["case"]["top"], s["case"]["V"])
    if case["api"] == "binding":
        o = net.kan_token_logprob_forward(s["logits"], s["ids"], TEMPERATURE, top, out=s["o"], ws=s["ws"])
        r = {n: o[n] for n in ("logp", "entropy", "top_ids", "top_logp") if n in o}
        if case["train"]:
            r["glogits"] = net.kan_token_logprob_backward(s["logits"], s["ids"], o, s["g_logp"], s["g_entropy"], TEMPERATURE, glogits=s["glogits"])
        return r
    with torch.set_grad_enabled(case["train"]):
        logp, entropy, top_ids, top_logp = autograd.token_logprob(s["logits"], s["ids"], TEMPERATURE, top)
    r = dict(logp=logp.detach(), entropy=entropy.detach())
    if top:
        r.update(top_ids=top_ids, top_logp=top_logp)
    if case["train"]:
        r["glogits"] = torch.autograd.grad([logp, entropy], s["logits"], [s["g_logp"], s["g_entropy"]])[0]
    return r


def _run_clip_own(s):
    from paper_2408_11200_amd import autograd
    return dict(norm=autograd.clip_gradients(s["grads"], s["max_norm"], out=s["out"]), out=s["flat"])


def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"norm": _run_norm_own, "embed": _run_embed_own, "logprob": _run_logprob_own, "clip": _run_clip_own}[kind](s)
    return {"norm": _run_norm_plain, "embed": _run_embed_plain, "logprob": _run_logprob_plain, "clip": _run_clip_plain}[kind](s)


# ---- the definition in 64 bits --------------------------------------------------------------

def _exact_norm(s):
    case = s["case"]
    t = {n: v.detach().double().requires_grad_(True) for n, v in dict(x=s["x"], f=s["f"], **s["p"]).items()}

    def norm(v, w, b):
        if case["norm"] == "layer":
            v = v - v.mean(-1, keepdim=True)
        y = v / torch.sqrt((v ** 2).mean(-1, keepdim=True) + EPS) * w
        return y + b if b is not None else y

    gate = t["gate"].repeat_interleave(case["gate_rows"] or case["B"], 0)[:case["B"]]
    x_out = RESIDUAL_SCALE * t["x"] + gate * norm(t["f"], t["w_post"], t.get("b_post"))
    h = norm(x_out, t["w_pre"], t.get("b_pre"))
    out = dict(x_out=x_out.detach(), h=h.detach())
    if case["train"]:
        g = torch.autograd.grad([x_out, h], list(t.values()), [s["gx_out"].double(), s["gh"].double()])
        out.update({"g" + n: v for n, v in zip(t, g)})
    return out


def _exact_embed(s):
    case, ids = s["case"], s["ids"]
    table = torch.cat([s["table"].detach().double(), torch.zeros((1, case["n"]), dtype=torch.float64, device="cuda")])     # the last row: no token
    row = torch.where(ids < 0, case["V"], ids)
    out = dict(y=table[row] * s["scale"])
    if case["train"]:
        g = torch.zeros_like(table).index_put_((row,), s["gy"].double(), accumulate=True)
        out["gtable"] = g[:case["V"]] * s["scale"]
    return out


def _exact_logprob(s):
    case, ids = s["case"], s["ids"]
    z = s["logits"].detach().double().clamp_min(-1e30).requires_grad_(True)      # masked: a probability of exactly zero
    lp = torch.log_softmax(z / TEMPERATURE, 1)
    entropy = -(lp.exp() * lp).sum(1)
    given = lp.gather(1, ids.clamp_min(0).unsqueeze(1))[:, 0]
    logp = torch.where(ids < 0, torch.zeros_like(given), given)
    out = dict(logp=logp.detach(), entropy=entropy.detach())
    if case["top"]:
        rows, cut = s["logits"].detach().float(), min(case["top"], case["V"])
        order = torch.cat([r.sort(dim=1, descending=True, stable=True).indices[:, :cut] for r in rows.split(max(1, (1 << 26) // case["V"]))])
        out["top_ids"], out["top_logp"] = order, lp.detach().gather(1, order)
    if case["train"]:
        out["glogits"] = torch.autograd.grad([logp, entropy], z, [s["g_logp"].double(), s["g_entropy"].double()])[0]
    return out


def _exact_clip(s):
    flat = torch.cat([g.reshape(-1).double() for g in s["grads"]])
    norm = torch.linalg.vector_norm(flat)
    return dict(norm=norm, out=flat * min(1.0, s["max_norm"] / float(norm)))


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "embed": _exact_embed, "logprob": _exact_logprob, "clip": _exact_clip}[case["kind"]](s)


# ---- what a pass cannot do without ----------------------------------------------------------

def work(case):
    size = lambda name: 4 if name == "f32" else 2
    kind, train = case["kind"], case.get("train")
    if kind == "norm":
        # x, f in, x_out, h out; their four gradients; about ten operations a value for each of the two norms, twice that backward
        values, row = case["B"] * case["n"], size(case["stream"]) + size(case["branch"])
        params = 4 * case["n"] * ((4 if case["norm"] == "layer" else 2) + _gate_groups(case))
        return {"bytes": values * row * (4 if train else 2) + params * (2 if train else 1), "flops": values * (48 if train else 16)}
    if kind == "embed":
        # the rows that are looked up (each once at most), what they become; gradients in, the whole table's gradient out
        T, V, n = case["T"], case["V"], case["n"]
        fwd = 8 * T + min(T, V) * n * size(case["table"]) + T * n * size(case["out"])
        return {"bytes": fwd + (T * n * size(case["out"]) + V * n * size(case["table"]) if train else 0), "flops": T * n * (3 if train else 1)}
    if kind == "logprob":
        values, top = case["R"] * case["V"], min(case["top"], case["V"])
        return {"bytes": values * size(case["type"]) * (2 if train else 1) + case["R"] * (16 + 12 * top + (8 if train else 0)),
                "flops": values * (15 if train else 6)}
    values = sum(math.prod(shape) for shape in _clip_shapes(case))
    return {"bytes": values * size(case["type"]) * 2 + 4, "flops": 3 * values}
