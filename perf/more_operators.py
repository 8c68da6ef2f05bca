"""Performance cases of the operators by which a network on tokens learns from a teacher and searches for its answers.

A case is a dict of plain values; `kind` names the operator:

  distill  the divergence of a student's probabilities from a teacher's list of likely tokens, row by row, and its gradient:
             p = exp(teacher), the probability that is left over being one outcome more ("logp"), or p = softmax(teacher / T) over the list ("logits")
             loss = sum_k p_k (log p_k - log q_k), q = softmax(logits / T)
           mode "loss": the loss alone; "train": forward, then backward with weights of the rows; "step": both at once, the weights known before
  select   the best continuations of the beams of a search: score + log softmax(logits / T) over all beams and tokens of a request;
           beams that have ended go on unchanged, those at -infinity are out of the search
  reorder  rows of the beams' states put in the order of the beams that have been chosen, in place or into other buffers

`run` computes these in elementary torch operations, or through the framework's entry points where `own` is true.
`exact` is the definition in 64 bits, with gradients by automatic differentiation.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i64": torch.int64, "u8": torch.uint8}


def listed():
    return [
        # a batch of a small network: latency counts
        dict(name="distill-train-256x1000", kind="distill", mode="train", R=256, V=1000, pad=0, type="f32", K=8, teacher="logp", list="f32", T=1.0, left=0, api="autograd"),
        # the loss of a few held-out rows on a middling vocabulary
        dict(name="distill-loss-16x32768", kind="distill", mode="loss", R=16, V=32768, pad=0, type="bf16", K=20, teacher="logp", list="f32", T=1.0, left=0, api="autograd"),
        # a training batch: odd sizes, rows of a padded buffer, a teacher's logits at a temperature, an eighth of the rows without a teacher
        dict(name="distill-train-4093x50001", kind="distill", mode="train", R=4093, V=50001, pad=47, type="f32", K=20, teacher="logits", list="f32", T=2.0, left=8, api="autograd"),
        # the same at the largest vocabulary, weights of the rows known before the call, the list kept in bfloat16
        dict(name="distill-step-8192x131072", kind="distill", mode="step", R=8192, V=131072, pad=0, type="bf16", K=64, teacher="logp", list="bf16", T=1.0, left=0, api="binding"),
        # one request with four beams
        dict(name="select-1x4x32768", kind="select", N=1, B=4, V=32768, pad=0, type="bf16", top=4, ended=0, dead=0, scale=False, T=1.0, api="autograd"),
        # the first step of a batch of requests: one beam each has a score
        dict(name="select-16x4x50001-first", kind="select", N=16, B=4, V=50001, pad=0, type="f32", top=4, ended=0, dead=3, scale=False, T=1.0, api="autograd"),
        # odd sizes, rows of a padded buffer, beams that have ended beside others, scores by length, twice as many candidates as beams
        dict(name="select-24x6x50001", kind="select", N=24, B=6, V=50001, pad=47, type="f32", top=12, ended=2, dead=0, scale=True, T=0.75, api="binding"),
        # a serving batch at the largest vocabulary
        dict(name="select-128x8x131072", kind="select", N=128, B=8, V=131072, pad=0, type="bf16", top=16, ended=0, dead=0, scale=False, T=1.0, api="binding"),
        # a wide search of few requests
        dict(name="select-4x32x131072", kind="select", N=4, B=32, V=131072, pad=0, type="bf16", top=64, ended=0, dead=0, scale=False, T=1.0, api="autograd"),
        # the windows and answers of a few requests: latency is all there is
        dict(name="reorder-4x4-windows", kind="reorder", N=4, B=4, count=2, inner=1, length=1, capacity=1, dim=17, type="i64", keep=2, place=True, api="autograd"),
        # streams of odd width, into other buffers
        dict(name="reorder-24x6x771", kind="reorder", N=24, B=6, count=8, inner=1, length=117, capacity=117, dim=771, type="bf16", keep=3, place=False, api="binding"),
        # keys and values for each head, the filled part of longer buffers, in place
        dict(name="reorder-4x8-caches", kind="reorder", N=4, B=8, count=16, inner=8, length=2000, capacity=2304, dim=128, type="bf16", keep=4, place=True, api="autograd"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind, api = rng.choice(["distill", "distill", "select", "select", "reorder"]), rng.choice(["binding", "autograd"])
    if kind == "distill":
        mode, V, type = rng.choice(["loss", "train", "train", "step"]), _log(rng, 64, 131072), rng.choice(["f32", "bf16"])
        R = _log(rng, 1, 4096) if mode == "loss" else _log(rng, 64, 16384)
        most = (1 << 30) // V if type == "bf16" else (1 << 28) // V
        return dict(kind=kind, mode=mode, R=max(1, min(R, most)), V=V, pad=rng.choice([0, 0, rng.randint(1, 64)]), type=type, K=min(_log(rng, 1, 256), V // 2),
                    teacher=rng.choice(["logp", "logp", "logits"]), list=rng.choice(["f32", "f32", "bf16"]), T=rng.choice([1.0, 1.0, 2.0, 0.75]),
                    left=rng.choice([0, 0, 4, 16]), api="binding" if mode == "step" else api)
    if kind == "select":
        V, B, N = _log(rng, 64, 131072), _log(rng, 1, 64), _log(rng, 1, 128)
        N = max(1, min(N, 1024 // B))
        ended = rng.choice([0, 0, B // 4])
        return dict(kind=kind, N=N, B=B, V=V, pad=rng.choice([0, 0, rng.randint(1, 64)]), type=rng.choice(["f32", "bf16"]), top=min(rng.choice([1, 2]) * B, 64),
                    ended=ended, dead=rng.choice([0, 0, 0, (B - ended) // 2]), scale=rng.random() < 0.3, T=rng.choice([1.0, 1.0, 0.75]), api=api)
    B, type = rng.choice([2, 3, 4, 5, 8, 16, 32]), rng.choice(["f32", "bf16", "i64", "u8"])
    N, count, inner, dim = _log(rng, 1, 64), _log(rng, 1, 48), _log(rng, 1, 16), _log(rng, 1, 1024)
    size = {"f32": 4, "bf16": 2, "i64": 8, "u8": 1}[type]
    length = _log(rng, 1, max(1, min(4096, (1 << 30) // (N * B * count * inner * dim * size))))
    return dict(kind=kind, N=N, B=B, count=count, inner=inner, length=length, capacity=length + rng.choice([0, 0, _log(rng, 1, 256)]), dim=dim, type=type,
                keep=rng.randint(1, B - 1), place=rng.random() < 0.7, api=api)


# ---- inputs ---------------------------------------------------------------------------------

def _normal(gen, std, *shape):
    return torch.randn(shape, generator=gen, device="cuda") * std


def _rows_of_logits(gen, R, V, common):
    """Rows of logits before their masks: `common` tokens are likely everywhere."""
    z = _normal(gen, 2.0, R, V)
    z[:, :common] += 3.0
    return z


def _prepare_distill(case, gen):
    R, V, K, T = case["R"], case["V"], case["K"], case["T"]
    common, masked = max(1, V // 64), V // 50
    buffer = torch.zeros((R, V + case["pad"]), dtype=DTYPES[case["type"]], device="cuda")
    ids, values = torch.empty((R, K), dtype=torch.int64, device="cuda"), torch.empty((R, K), dtype=DTYPES[case["list"]], device="cuda")
    step = max(1, (1 << 28) // V)
    for at in range(0, R, step):
        rows = slice(at, min(R, at + step))
        z = _rows_of_logits(gen, rows.stop - at, V, common)
        t = 1.1 * z + _normal(gen, 0.7, *z.shape)                    # a teacher whose opinion the student has learnt in part
        z[:, V - masked:], t[:, V - masked:] = -math.inf, -math.inf  # the end of a vocabulary that was filled up to a round size
        buffer[rows, :V] = z
        top = t.topk(K, dim=1)
        ids[rows] = top.indices
        values[rows] = (top.values / T - torch.logsumexp(t / T, 1, keepdim=True) if case["teacher"] == "logp" else top.values).to(values.dtype)
    if K > 2:
        ids[torch.rand(R, generator=gen, device="cuda") < 0.05, K - 1] = -1          # shorter lists
    if case["left"]:
        ids[torch.arange(R, device="cuda") % case["left"] == case["left"] - 1] = -1  # rows without a teacher
    return dict(logits=buffer[:, :V], ids=ids, values=values, g_loss=torch.rand(R, generator=gen, device="cuda") / R,
                loss=torch.empty(R, device="cuda"), stats=torch.empty((R, K + 2), device="cuda"),
                glogits=torch.empty((R, V), dtype=buffer.dtype, device="cuda"))


def _prepare_select(case, gen):
    N, B, V = case["N"], case["B"], case["V"]
    masked = V // 50
    logits = torch.zeros((N * B, V + case["pad"]), dtype=DTYPES[case["type"]], device="cuda")
    logits[:, :V] = _rows_of_logits(gen, N * B, V, max(1, V // 64))
    logits[:, V - masked:V] = -math.inf
    # the beams of a request lie a few nats apart, best first; which have ended goes by chance
    scores = -10.0 * torch.rand((N, 1), generator=gen, device="cuda") - (torch.rand((N, B), generator=gen, device="cuda") * 1.5).cumsum(1)
    order = torch.rand((N, B), generator=gen, device="cuda").argsort(1)
    if case["dead"]:
        scores[order >= B - case["dead"]] = -math.inf
    s = dict(logits=logits[:, :V], scores=scores, ended=None, scale=None, end_id=-1, out=dict(
        scores=torch.empty((N, case["top"]), device="cuda"), tokens=torch.empty((N, case["top"]), dtype=torch.int64, device="cuda"),
        parents=torch.empty((N, case["top"]), dtype=torch.int64, device="cuda"), ended=torch.empty((N, case["top"]), dtype=torch.bool, device="cuda")))
    if case["ended"]:
        s["ended"], s["end_id"] = order < case["ended"], 2
    if case["scale"]:
        s["scale"] = 1.0 / torch.randint(5, 40, (N, B), generator=gen, device="cuda").float() ** 0.7
    return s


def _prepare_reorder(case, gen):
    N, B, keep, dtype = case["N"], case["B"], case["keep"], DTYPES[case["type"]]
    shape = (N * B, case["inner"], case["capacity"], case["dim"])
    order = torch.rand((N, B), generator=gen, device="cuda").argsort(1)
    if case["place"]:
        # `keep` beams of each request stay where they are, the others are put on top of the rest in turn: a second pass leaves what the first has left
        parents = torch.arange(B, device="cuda").repeat(N, 1)
        moved = order[:, keep:]
        parents.scatter_(1, moved, order[:, torch.arange(B - keep, device="cuda") % keep])
    else:
        parents = order[:, torch.arange(B, device="cuda") % keep].gather(1, torch.rand((N, B), generator=gen, device="cuda").argsort(1))
    make = (lambda: torch.randint(0, 200, shape, generator=gen, device="cuda", dtype=dtype)) if case["type"] in ("i64", "u8") else \
        (lambda: torch.randn(shape, generator=gen, device="cuda", dtype=dtype))
    whole = [make() for _ in range(case["count"])]
    to = whole if case["place"] else [torch.zeros_like(t) for t in whole]
    return dict(parents=parents, whole=whole, to=to, states=[t[:, :, :case["length"]] for t in whole], out=[t[:, :, :case["length"]] for t in to])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"distill": _prepare_distill, "select": _prepare_select, "reorder": _prepare_reorder}[case["kind"]](case, gen)
    s["case"] = case
    return s


# ---- plain forms ----------------------------------------------------------------------------

def _run_distill_plain(s):
    case, T, ids = s["case"], s["case"]["T"], s["ids"]
    z, t = s["logits"].float(), s["values"].double()
    V = z.shape[1]
    there = (ids >= 0) & (ids < V)
    at = torch.where(there, ids, 0)
    # the teacher's probabilities: the rest is a difference to one, and the loss a difference of logarithms, hence 64 bits for the list
    if case["teacher"] == "logp":
        log_p = torch.where(there, t, -math.inf)
    else:
        t = torch.where(there, t / T, -math.inf)
        most = t.amax(1, keepdim=True)
        log_p = torch.where(there, t - most - torch.log(torch.exp(t - most).sum(1, keepdim=True)), -math.inf)
    p = torch.exp(log_p)
    some = p.sum(1, keepdim=True) > 0
    p_rest = (1.0 - p.sum(1, keepdim=True)).clamp_min(0.0) * some if case["teacher"] == "logp" else torch.zeros_like(p[:, :1])
    total_p = p.sum(1, keepdim=True) + p_rest
    # the student's: sums over the tokens of the list and over the others
    m = z.amax(1, keepdim=True)
    e = torch.exp((z - m) * (1.0 / T))
    listed_ = torch.zeros((z.shape[0], V + 1), dtype=torch.bool, device="cuda").scatter_(1, torch.where(there, ids, V), True)
    e = e.masked_fill_(listed_[:, :V], 0.0)
    s_rest = e.sum(1, keepdim=True).double()
    down = torch.where(there, (z.gather(1, at).double() - m.double()) / T, -math.inf)
    total = torch.exp(down).sum(1, keepdim=True) + s_rest
    log_q = down - torch.log(total)
    q_rest = s_rest / total
    terms = torch.where(p > 0, p * (log_p - log_q), 0.0)
    rest = torch.where(p_rest > 0, p_rest * (torch.log(p_rest) - torch.log(q_rest)), 0.0)
    loss = (terms.sum(1) + rest[:, 0]).float()
    if case["mode"] == "loss":
        return dict(loss=loss)
    g = s["g_loss"].double().unsqueeze(1) * some / T
    grad = e * (g * (q_rest * total_p - p_rest) / s_rest).float()
    grad.scatter_add_(1, at, torch.where(there, g * (torch.exp(log_q) * total_p - p), 0.0).float())
    return dict(loss=loss, glogits=grad.to(s["logits"].dtype))


def _plain_top(z, top):
    """Indices of the largest values of each row, the lowest index first among equal ones: unique whole-number keys."""
    bits = z.contiguous().view(torch.int32).to(torch.int64)
    key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) << 32
    key = key + (0xFFFFFFFF - torch.arange(z.shape[1], device="cuda"))
    return key.topk(top, dim=1).indices


def _run_select_plain(s):
    case = s["case"]
    N, B, top = case["N"], case["B"], case["top"]
    each = min(top, case["V"])
    # scores of two beams' tokens that lie near one another are told apart: 64 bits
    z = s["logits"].double()
    z = (z - z.amax(1, keepdim=True)) / case["T"]
    tokens = _plain_top(s["logits"].float(), each)
    score = s["scores"].double().view(-1, 1) + (z.gather(1, tokens) - torch.log(torch.exp(z).sum(1, keepdim=True)))
    if s["ended"] is not None:
        over = s["ended"].view(-1, 1)
        only = torch.full_like(score, -math.inf)
        only[:, 0] = s["scores"].double().view(-1)
        score, tokens = torch.where(over, only, score), torch.where(over, s["end_id"], tokens)
    rank = score if s["scale"] is None else score * s["scale"].double().view(-1, 1)
    best = rank.view(N, B * each).sort(dim=1, descending=True, stable=True).indices[:, :top]
    score, tokens, parents = score.view(N, -1).gather(1, best), tokens.view(N, -1).gather(1, best), best // each
    ended = tokens == s["end_id"]
    none = score == -math.inf
    return dict(scores=score.float(), tokens=torch.where(none, -1, tokens), parents=torch.where(none, 0, parents), ended=ended & ~none)


def _run_reorder_plain(s):
    B = s["case"]["B"]
    rows = (s["parents"] + B * torch.arange(s["case"]["N"], device="cuda").unsqueeze(1)).view(-1)
    moved = [o.copy_(t.index_select(0, rows)) for t, o in zip(s["states"], s["out"])]
    return dict(states=s["to"][:len(moved)])


# ---- the framework's operators --------------------------------------------------------------

def _run_distill_own(s):
    from paper_2408_11200_amd import autograd, net
    case = s["case"]
    how = dict(temperature=case["T"], teacher=case["teacher"])
    if case["mode"] == "step":
        loss, glogits = net.kan_token_distill_step(s["logits"], s["ids"], s["values"], s["g_loss"], loss=s["loss"], glogits=s["glogits"], **how)
        return dict(loss=loss, glogits=glogits)
    if case["api"] == "binding":
        fwd = net.kan_token_distill_forward(s["logits"], s["ids"], s["values"], out=dict(loss=s["loss"], stats=s["stats"]), **how)
        if case["mode"] == "loss":
            return dict(loss=fwd["loss"])
        glogits = net.kan_token_distill_backward(s["logits"], s["ids"], fwd, s["g_loss"], temperature=case["T"], glogits=s["glogits"])
        return dict(loss=fwd["loss"], glogits=glogits)
    if case["mode"] == "loss":
        return dict(loss=autograd.token_distill(s["logits"], s["ids"], s["values"], **how))
    logits = s["logits"].detach().requires_grad_(True)
    loss = autograd.token_distill(logits, s["ids"], s["values"], **how)
    return dict(loss=loss.detach(), glogits=torch.autograd.grad(loss, logits, s["g_loss"])[0])


def _run_select_own(s):
    from paper_2408_11200_amd import autograd, net
    case = s["case"]
    how = dict(ended=s["ended"], end_id=s["end_id"], rank_scale=s["scale"], temperature=case["T"])
    if case["api"] == "binding":
        o = net.kan_beam_select(s["logits"], s["scores"], case["top"], out=s["out"], **how)
        return {n: o[n] for n in ("scores", "tokens", "parents", "ended")}
    scores, tokens, parents, ended = autograd.beam_select(s["logits"], s["scores"], case["top"], **how)
    return dict(scores=scores, tokens=tokens, parents=parents, ended=ended)


def _run_reorder_own(s):
    from paper_2408_11200_amd import autograd, net
    reorder = net.kan_beam_reorder if s["case"]["api"] == "binding" else autograd.beam_reorder
    reorder(s["parents"], s["states"], s["case"]["B"], out=None if s["case"]["place"] else s["out"])
    return dict(states=s["to"])


def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"distill": _run_distill_own, "select": _run_select_own, "reorder": _run_reorder_own}[kind](s)
    return {"distill": _run_distill_plain, "select": _run_select_plain, "reorder": _run_reorder_plain}[kind](s)


# ---- the definition in 64 bits --------------------------------------------------------------

def _exact_distill(s):
    case, T, K, V = s["case"], s["case"]["T"], s["case"]["K"], s["case"]["V"]
    loss, grads = [], []
    for at in range(0, case["R"], max(1, (1 << 28) // V)):
        rows = slice(at, at + max(1, (1 << 28) // V))
        ids, t = s["ids"][rows], s["values"][rows].double()
        z = s["logits"][rows].double().clamp_min(-1e30).requires_grad_(True)      # masked: a probability of exactly zero
        lq = torch.log_softmax(z / T, 1)
        lq = torch.cat([lq, torch.full_like(lq[:, :1], -1e30)], 1)                # the last column: no token
        column = torch.where(ids < 0, V, ids)
        weight = (ids >= 0).double()
        p = weight * torch.exp(t) if case["teacher"] == "logp" else weight * torch.exp(t / T)
        if case["teacher"] == "logits":
            p = p / p.sum(1, keepdim=True).clamp_min(1e-300)
        known = (p.sum(1) > 0).double()
        kl = (torch.xlogy(p, p) - torch.where(p > 0, p * lq.gather(1, column), 0.0)).sum(1)
        if case["teacher"] == "logp":
            left = (1.0 - p.sum(1)).clamp_min(0.0)
            others = torch.ones_like(lq).scatter_(1, column, 0.0)
            others[:, V] = 0.0
            kl = kl + torch.xlogy(left, left) - left * torch.logsumexp(torch.where(others > 0, lq, -1e35), 1)
        kl = kl * known
        loss.append(kl.detach())
        if case["mode"] != "loss":
            grads.append(torch.autograd.grad(kl, z, s["g_loss"][rows].double())[0])
    out = dict(loss=torch.cat(loss))
    if case["mode"] != "loss":
        out["glogits"] = torch.cat(grads)
    return out


def _exact_select(s):
    case = s["case"]
    N, B, V, top, out = case["N"], case["B"], case["V"], case["top"], []
    for g in range(N):
        lp = torch.log_softmax(s["logits"][g * B:(g + 1) * B].double() / case["T"], 1)
        score = s["scores"][g].double().unsqueeze(1) + lp
        if s["ended"] is not None:
            score[s["ended"][g]] = -math.inf
            score[s["ended"][g], s["end_id"]] = s["scores"][g][s["ended"][g]].double()
        rank = score if s["scale"] is None else score * s["scale"][g].double().unsqueeze(1)
        at = rank.view(-1).sort(dim=0, descending=True, stable=True).indices[:top]
        out.append((score.view(-1)[at], at % V, at // V))
    scores, tokens, parents = (torch.stack(v) for v in zip(*out))
    none = torch.isinf(scores)
    return dict(scores=scores, tokens=torch.where(none, -1, tokens), parents=torch.where(none, 0, parents), ended=(tokens == s["end_id"]) & ~none)


def _exact_reorder(s):
    case, B = s["case"], s["case"]["B"]
    source = torch.cat([s["parents"][g] + g * B for g in range(case["N"])])
    states = []
    for t, to in zip(s["whole"], s["to"]):
        after = to.clone()
        after[:, :, :case["length"]] = t[source][:, :, :case["length"]]
        states.append(after.double() if after.is_floating_point() else after)
    return dict(states=states)


def exact(case, seed):
    s = prepare(case, seed)
    return {"distill": _exact_distill, "select": _exact_select, "reorder": _exact_reorder}[case["kind"]](s)


# ---- what a pass cannot do without ----------------------------------------------------------

def work(case):
    size = lambda name: {"f32": 4, "bf16": 2, "i64": 8, "u8": 1}[name]
    kind = case["kind"]
    if kind == "distill":
        # rows with a teacher are read, gradients of all rows written
        R, V, K, train = case["R"], case["V"], case["K"], case["mode"] != "loss"
        rows = R - R // case["left"] if case["left"] else R
        return {"bytes": rows * V * size(case["type"]) + (R * V * size(case["type"]) if train else 0) + R * (K * (8 + size(case["list"])) + (8 if train else 4)),
                "flops": rows * V * (8 if train else 4)}
    if kind == "select":
        N, B, V, top = case["N"], case["B"], case["V"], case["top"]
        rows = N * (B - case["ended"] - case["dead"])
        return {"bytes": rows * V * size(case["type"]) + N * B * 9 + N * top * 21, "flops": rows * V * 5}
    # in place: each moved row written, each row that takes the place of others read; into other buffers: all written
    row = case["inner"] * case["length"] * case["dim"] * size(case["type"])
    B, keep = case["B"], case["keep"]
    rows = B - keep + min(keep, B - keep) if case["place"] else B + keep
    return {"bytes": case["N"] * case["count"] * row * rows + 8 * case["N"] * B, "flops": 0}
