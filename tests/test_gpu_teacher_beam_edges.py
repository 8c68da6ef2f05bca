"""Calls of distillation, beam selection and search that the documentation allows and whose answers are easily lost: against the plain forms in 64 bits."""
import math

import numpy as np
import pytest
import torch

from oracle import net as plain
from paper_2408_11200_amd import autograd, net, tokens, workloads
import test_gpu_distill
from test_gpu_beam import case as select_case, check as select_check
from test_gpu_distill import case as distill_case, check as distill_check

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def dev(a, dtype=F32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def host(t):
    return t.detach().double().cpu().numpy()


# ---- distillation ---------------------------------------------------------------------------

@pytest.mark.parametrize("teacher", ["logp", "logits"])
@pytest.mark.parametrize("R,V,K,dtype", [(8, 24, 2, F32), (9000, 24, 2, BF16), (9000, 1000, 3, F32), (4000, 500, 40, F32), (8, 5000, 70, BF16), (8, 40000, 2, F32), (8, 140000, 3, F32), (8, 140000, 90, BF16),
                                         (300, 140000, 2, BF16)])
def test_a_nan_among_listed_logits_that_are_all_the_mask_leaves(R, V, K, dtype, teacher):
    """Every other token masked, and among the listed ones a NaN alone or beside -infinity: loss and gradients are NaN, as with any NaN in a row that has a teacher."""
    rng = np.random.default_rng(V + K)
    ids = np.stack([rng.permutation(V)[:K] for _ in range(8)])
    v = np.log(rng.dirichlet(np.ones(K + 1), 8)[:, :K]).astype(np.float32)
    z = np.full((8, V), -np.inf, np.float32)
    z[0, ids[0, 0]] = np.nan                            # the others of the list -infinity
    z[1, ids[1]] = np.nan
    z[2, ids[2, K - 1]], ids[2, :K - 1] = np.nan, -1    # the one listed token
    z[3, ids[3, 0]], v[3, 0] = np.nan, -np.inf          # the NaN's token without a probability
    z[4, ids[4]], z[4, ids[4, 0]] = 1.0, np.nan         # finite ones beside it
    ids[5] = -1                                         # no teacher: 0, whatever the row holds
    z[5] = np.nan                                       # 6: nothing left by the mask, +infinity and no gradient
    z[7] = rng.standard_normal(V)
    many = lambda a: dev(np.tile(a, (-(-R // 8), 1))[:R]) if a.dtype != np.int64 else torch.from_numpy(np.tile(a, (-(-R // 8), 1))[:R]).cuda()
    logits, di, dv, g = many(z).to(dtype), many(ids), many(v), torch.ones(R, device="cuda")
    f = plain.token_distill(host(logits[:8]), ids, host(dv[:8]), 1.0, teacher)
    assert np.isnan(f["loss"][:5]).all() and f["loss"][5] == 0 and f["loss"][6] == np.inf and np.isnan(f["d"][:5]).all()
    o = net.kan_token_distill_forward(logits, di, dv, 1.0, teacher)
    gz = net.kan_token_distill_backward(logits, di, o, g)
    loss, gs = net.kan_token_distill_step(logits, di, dv, g, 1.0, teacher)
    kind = torch.arange(R, device="cuda") % 8
    for l, d in ((o["loss"], gz), (loss, gs)):
        assert bool(torch.isnan(l[kind < 5]).all()) and bool(torch.isnan(d[kind < 5]).all())
        assert not l[kind == 5].any() and bool((l[kind == 6] == math.inf).all()) and not d[(kind == 5) | (kind == 6)].any()
        assert bool(torch.isfinite(l[kind == 7]).all()) and bool(torch.isfinite(d[kind == 7]).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [5000, 8192, 40000, 50001, 140000])
@pytest.mark.parametrize("T", [1.0, 0.75])
def test_one_token_stands_out_behind_the_first_pieces(dtype, V, T):
    """One unlisted logit 50 to 66 above all that came before it makes up the others' sum.  Its term is an exponential of an exponent near 0 (2 u), what the reference's rounding
    is off by an exponential and a product more (3 u), the other terms are below 2^-24 of it together: the sum is off by 10 u at most, so the loss by 10 u q_r (and its own rounding), and
    the gradients, q_v of either kind, by 10 u, their own factors' 10 u and half a step."""
    R = 48
    rng = np.random.default_rng(V)
    z = rng.standard_normal((R, V)).astype(np.float32)
    at = rng.integers(V // 3 * 2, V, R)
    listed = rng.integers(0, V // 2, R)
    z[np.arange(R), at] = np.linspace(50, 66, R).astype(np.float32) * T
    logits = dev(z, dtype)
    z = host(logits)
    z[np.arange(R), listed] = z[np.arange(R), at] + rng.integers(-2, 3, R)
    logits = dev(z.astype(np.float32), dtype)
    ids, v, g = torch.from_numpy(listed[:, None]).cuda(), torch.zeros((R, 1), device="cuda"), torch.ones(R, device="cuda")
    f = plain.token_distill(host(logits), listed[:, None], host(v), T)
    o = net.kan_token_distill_forward(logits, ids, v, T)
    gz = net.kan_token_distill_backward(logits, ids, o, g, T)
    loss, gs = net.kan_token_distill_step(logits, ids, v, g, T)
    assert torch.equal(loss, o["loss"]) and torch.equal(gs, gz)
    err = np.abs(host(loss) - f["loss"]) / (U * np.abs(f["loss"]) + 10 * U * f["q_rest"])
    assert err.max() <= 1, float(err.max())
    half = 2.0 ** -8 if dtype == BF16 else U
    for token in (at, listed):
        want = f["d"][np.arange(R), token]
        err = np.abs(host(gz)[np.arange(R), token] - want) / ((20 * U + half) * np.abs(want) * (1 + 2.0 ** -7))
        assert err.max() <= 1, float(err.max())


@pytest.mark.parametrize("R,V,K,dtype,T", [(4200, 33001, 20, BF16, 1.0), (4500, 16001, 12, F32, 0.75), (1100, 64007, 20, F32, 1.0), (1100, 64007, 70, F32, 1.0), (2100, 65003, 8, BF16, 1.0)])
def test_logits_that_the_caches_do_not_hold(R, V, K, dtype, T):
    """Read past the caches, by four and by eight waves a row: against the formulas, and the bits of fewer rows that are read through them."""
    few = 520
    logits, ids, values, g = distill_case(few, V, K, R, dtype=dtype, T=T)
    many = lambda t: t.repeat(-(-R // few), *[1] * (t.dim() - 1))[:R].contiguous()
    big, bi, bv, bg = many(logits), many(ids), many(values), many(g)
    assert big.numel() * big.element_size() >= 1 << 28 and few * V * big.element_size() < 1 << 28
    o = net.kan_token_distill_forward(big, bi, bv, T)
    gz = net.kan_token_distill_backward(big, bi, o, bg, T)
    f = plain.token_distill(host(logits[:6]), ids[:6].cpu().numpy(), host(values[:6]), T)
    distill_check(f, T, V, loss=o["loss"][:6], glogits=gz[:6], g=g[:6])
    loss, gs = net.kan_token_distill_step(big, bi, bv, bg, T)
    assert torch.equal(loss, o["loss"]) and torch.equal(gs, gz)
    small = net.kan_token_distill_forward(logits, ids, values, T)
    back = net.kan_token_distill_backward(logits, ids, small, g, T)
    assert torch.equal(o["loss"], many(small["loss"])) and torch.equal(gz[:few], back) and torch.equal(gz[-(R % few):], back[:R % few])


@pytest.mark.parametrize("R,V,K,dtype", [(5, 300, 70, F32), (700, 5000, 65, BF16), (9, 20000, 256, F32), (3, 140000, 100, BF16), (400, 140000, 128, F32), (2, 70001, 200, F32)])
@pytest.mark.parametrize("teacher", ["logp", "logits"])
def test_tokens_twice_in_long_lists(R, V, K, dtype, teacher):
    """Lists of more than 64 tokens, some of them two and three times and among other lanes' and entries' tokens: one wave a row, more, and rows that are cut."""
    logits, ids, values, g = distill_case(R, V, K, V, dtype=dtype, teacher=teacher, short=False)
    ids[:, K - 1] = ids[:, 0]                           # another entry of the same lane or of another one
    ids[::2, 64] = ids[::2, 0]
    ids[1::2, 64] = ids[1::2, 63]
    ids[:, K // 2] = ids[:, 3]
    rows = np.unique(np.concatenate([np.arange(min(R, 4)), [R - 1]]))
    f = plain.token_distill(host(logits)[rows] if R < 100 else host(logits[rows.tolist()]), ids.cpu().numpy()[rows], host(values)[rows], 1.0, teacher)
    o = net.kan_token_distill_forward(logits, ids, values, 1.0, teacher)
    distill_check(f, 1.0, V, loss=o["loss"][rows.tolist()])
    gz = net.kan_token_distill_backward(logits, ids, o, g)
    distill_check(f, 1.0, V, glogits=gz[rows.tolist()], g=g[rows.tolist()])
    loss, gs = net.kan_token_distill_step(logits, ids, values, g, 1.0, teacher)
    assert torch.equal(loss, o["loss"]) and torch.equal(gs, gz)


@pytest.mark.parametrize("R,V,K,options", [(4200, 257, 16, dict(dtype=F32, T=1.0)), (4111, 257, 20, dict(dtype=F32, T=1.0)), (8200, 512, 64, dict(dtype=F32, teacher="logits", T=0.75)), (8191, 512, 8, dict(dtype=F32, T=1.0)),
                                           (8011, 1001, 20, dict(dtype=BF16, pad=5, T=1.0)), (8005, 1001, 33, dict(dtype=BF16, T=2.0)), (16390, 501, 20, dict(dtype=F32, pad=1, T=1.0))])
def test_short_rows_on_both_sides_of_the_backward_line(R, V, K, options):
    """As many rows as four times a row's bytes, and fewer."""
    test_gpu_distill.test_short_rows(R, V, K, dict(dict(teacher="logp"), **options))


# ---- beam selection -------------------------------------------------------------------------

@pytest.mark.parametrize("B,top", [(8, 8), (64, 64), (64, 5), (33, 40)])
def test_ranks_of_ended_beams_are_compared_in_64_bits(B, top):
    """An ended beam's rank is the product of two floats, exact in 64 bits: products that agree to 2^-37 of themselves, and some that are equal, in the order of the products, then of the beams."""
    rng = np.random.default_rng(B)
    s = -np.float32(1.1 + rng.random(1 << 18) * 0.5)
    scale = np.float32(1.37 / -s.astype(np.float64))
    product = s.astype(np.float64) * scale
    order = np.argsort(product)
    gap = np.diff(product[order])
    near = np.where((gap > 0) & (gap < 2.0 ** -37))[0]
    N = 30
    pick = np.stack([np.concatenate([order[near[rng.integers(len(near))]] + np.zeros(1, int), order[(a := near[rng.integers(len(near))]):a + 2], rng.integers(0, len(s), B - 3)]) for _ in range(N)])
    pick[:, B // 2] = pick[:, 0]                        # one rank twice
    pick = rng.permuted(pick, axis=1)
    scores, scales = s[pick], scale[pick]
    d = torch.from_numpy
    z = torch.randn((N * B, 40), device="cuda")
    o = net.kan_beam_select(z, d(scores).cuda(), top, torch.ones((N, B), dtype=torch.bool, device="cuda"), 7, d(scales).cuda())
    want = np.argsort(-product[pick], axis=1, kind="stable")[:, :top]
    there = min(top, B)
    assert np.array_equal(o["parents"].cpu().numpy()[:, :there], want) and bool((o["tokens"][:, :there] == 7).all()) and bool((o["tokens"][:, there:] == -1).all())
    assert np.array_equal(o["scores"].cpu().numpy()[:, :there], np.take_along_axis(scores, want, 1)) and bool(o["ended"][:, :there].all())


@pytest.mark.parametrize("score,T", [(-1.0, 1e30), (-1e4, 1.0), (-1e6, 1.0), (-1e9, 1.0), (-3e4, 1e4), (0.0, 1e-3)])
@pytest.mark.parametrize("N,V,top", [(1, 262144, 64), (2, 40000, 12), (300, 40000, 12), (5, 3000, 64), (3, 33, 33)])
def test_a_beams_tokens_come_in_the_order_of_their_logits(score, T, N, V, top):
    """Scores that differ in their last bits or not at all, at a high temperature or beside a large score of the beam: one beam's candidates are its largest logits, equal ones by token, however its
    row is cut.  Where all are equal and scores of beams too, the first beam has them all."""
    rng = np.random.default_rng(V)
    z = rng.standard_normal((min(N, 3), V)).astype(np.float32)
    z[:, V // 3] = z[:, V - 1] = z.max(1)               # the largest one three times
    if V > 100:
        z[0, V // 2:V // 2 + 40] = z[0].max() - np.float32(2.0 ** -20) * np.arange(40)
    want = np.argsort(-z, axis=1, kind="stable")[:, :top]
    rows = np.arange(N) % len(z)
    logits = dev(z[rows])
    o = net.kan_beam_select(logits, torch.full((N, 1), score, device="cuda"), top, temperature=T)
    got = o["tokens"].cpu().numpy()
    there = host(o["scores"]) > -np.inf
    assert np.array_equal(got, np.where(there, want[rows], -1)) and (T == 1e-3 or there.all())
    if T == 1e30:
        both = net.kan_beam_select(logits.repeat_interleave(2, 0), torch.full((N, 2), score, device="cuda"), top, temperature=T)
        assert torch.equal(both["tokens"], o["tokens"]) and not both["parents"].any()


@pytest.mark.parametrize("N,B,V,top,dtype", [(140, 8, 62501, 16, F32), (300, 16, 16001, 64, F32), (130, 8, 131075, 8, BF16)])
def test_selection_from_logits_that_the_caches_do_not_hold(N, B, V, top, dtype):
    few = 40
    logits, scores, _, _ = select_case(few, B, V, V, dtype=dtype)
    assert N * B * V * logits.element_size() >= 1 << 28 > few * B * V * logits.element_size()
    big = logits.repeat(-(-N // few), 1)[:N * B].contiguous()
    s = torch.from_numpy(np.tile(scores, (-(-N // few), 1))[:N].copy()).cuda()
    o = net.kan_beam_select(big, s, top)
    select_check(o, plain.beam_select(host(logits[:2 * B]), scores[:2], top), V, rows=[0, 1])
    small = net.kan_beam_select(logits, s[:few], top)
    assert all(torch.equal(o[n][:few], small[n]) and torch.equal(o[n][few:2 * few], small[n]) for n in o)


# ---- reordering -----------------------------------------------------------------------------

@pytest.mark.parametrize("N,B", [(3, 4), (1, 20), (2, 64)])
def test_states_side_by_side_in_one_buffer(N, B):
    """Layers' keys and values lie between one another's rows: nothing crosses, in place, or from one half of every row into the other; and many of them in a call."""
    rng = np.random.default_rng(B)
    p = rng.integers(0, B, (N, B))
    parents = torch.from_numpy(p).cuda()
    rows = torch.from_numpy((p + B * np.arange(N)[:, None]).ravel()).cuda()
    for reorder in (net.kan_beam_reorder, autograd.beam_reorder):
        buffer = torch.randn((N * B, 3, 2, 4, 30, 5), device="cuda")
        before = buffer.clone()
        reorder(parents, [buffer[:, l, k, :, :17] for l in range(3) for k in range(2)], B)
        want = before.clone()
        want[:, :, :, :, :17] = before[rows][:, :, :, :, :17]
        assert torch.equal(buffer, want)
        buffer.copy_(before)
        reorder(parents, [buffer[:, l, 0, :, :17] for l in range(3)], B, out=[buffer[:, l, 1, :, 13:] for l in range(3)])
        want = before.clone()
        want[:, :, 1, :, 13:] = before[rows][:, :, 0, :, :17]
        assert torch.equal(buffer, want)
        wide = torch.randn((N * B, 300, 7), device="cuda", dtype=torch.float32).to(BF16)
        before = wide.clone()
        reorder(parents, [wide[:, k, :] for k in range(0, 300)], B)
        assert torch.equal(wide, before[rows])
        tall = torch.randn((6, N * B, 5), device="cuda")
        before = tall.clone()
        reorder(parents, [tall[::2], tall[1::2]], B, dim=1)
        assert torch.equal(tall, before[:, rows])


@pytest.mark.parametrize("N,B,dtype", [(3, 5, BF16), (2, 12, torch.uint8), (2, 20, F32), (1, 40, BF16), (1, 64, torch.uint8)])
def test_states_that_the_caches_do_not_hold(N, B, dtype):
    """Read past the caches, by every number of rows a thread has a piece of; in place and into other buffers."""
    rng = np.random.default_rng(B)
    p = rng.integers(0, B, (N, B))
    parents = torch.from_numpy(p).cuda()
    rows = torch.from_numpy((p + B * np.arange(N)[:, None]).ravel()).cuda()
    size = torch.empty(0, dtype=dtype).element_size()
    width = -(-(1 << 28) // (N * B * size)) | 1         # rows that start anywhere
    state = torch.randint(0, 100, (N * B, width), device="cuda", dtype=torch.uint8).to(dtype)
    assert state.numel() * size >= 1 << 28
    want = state[rows]
    out = torch.empty_like(state)
    autograd.beam_reorder(parents, [state], B, out=[out])
    assert torch.equal(out, want)
    net.kan_beam_reorder(parents, [state], B)
    assert torch.equal(state, want)


def test_states_that_cross_are_refused_and_left():
    N, B = 2, 3
    p = torch.tensor([[1, 0, 2], [2, 2, 0]], device="cuda")
    t = torch.randn((6, 9, 4), device="cuda")
    before = t.clone()
    for reorder in (net.kan_beam_reorder, autograd.beam_reorder):
        for data, out in (([t[:, 1:]], [t[:, :-1]]), ([t[:, :5]], [t[:, 4:]]), ([t[:, :3], t[:, 2:6]], None), ([before, before], [t[:, :], t.flatten(1)[:, 1:].unflatten(1, (5, 7))[:, :, :4]])):
            if out and any(d.shape != o.shape for d, o in zip(data, out)):
                data = [d[:, :o.shape[1]] for d, o in zip(data, out)]
            with pytest.raises(RuntimeError):
                reorder(p, data, B, out=out)
        assert torch.equal(t, before)
        reorder(p, [t[:, :5]], B, out=[t[:, 5:].new_empty((6, 5, 4))])


# ---- the network that is taught and asked ---------------------------------------------------

@pytest.mark.parametrize("vocab,length,beams,end_id", [(3, 2, 16, -1), (2, 3, 20, 1), (5, 1, 64, -1)])
def test_places_without_an_answer_have_no_tokens(vocab, length, beams, end_id):
    """More beams than there are answers: the places behind them are -1 throughout, not the beginning of another answer."""
    model = tokens.TokenNet(vocab=vocab, embed=8, blocks=1, seed=1)
    ids = torch.randint(0, vocab, (6, 2), device="cuda")
    answers, scores = model.search(ids, length, beams, end_id)
    none = torch.isneginf(scores)
    count = vocab ** length if end_id < 0 else length + 1         # of two tokens, one of which ends an answer
    assert bool((none.sum(1) == beams - count).all()) and not none[:, :count].any()
    assert bool((answers[none] == -1).all()) and bool((answers[~none] >= 0).all())
    assert all(len({tuple(a) for a in answers[n, :count].tolist()}) == count for n in range(6))


@pytest.mark.parametrize("teacher", ["logp", "logits"])
def test_the_mean_divergence_leaves_rows_out_whose_lists_have_no_probability(teacher):
    """Rows without a teacher: no token of the vocabulary in the list, or none whose probability is above 0 in 64 bits (the most likely tokens of a row that is masked throughout have -infinity)."""
    student = tokens.TokenNet(20, embed=8, blocks=1, seed=2)
    ids = torch.from_numpy(workloads.token_task(20, n=64)[0]).cuda()
    gen = torch.Generator(device="cuda").manual_seed(3)
    listed = torch.stack([torch.randperm(20, generator=gen, device="cuda")[:4] for _ in range(64)])
    values = torch.log_softmax(torch.randn((64, 5), generator=gen, device="cuda"), 1)[:, :4].contiguous()
    values[0::8] = -math.inf
    listed[1::8] = torch.tensor([-1, 20, 1 << 40, -7], device="cuda")
    values[2::8, 1:], listed[2::8, 0] = -math.inf, -1           # what has a probability is no token
    values[3::8] = -800.0                                       # as log probabilities nothing, as logits a quarter each
    values[4::8, 1:] = -math.inf
    with torch.no_grad():
        z = student.logits(ids)
        each = plain.token_distill(host(z), listed.cpu().numpy(), host(values), 1.0, teacher)["loss"]
    taught = np.isin(np.arange(64) % 8, [4, 5, 6, 7] + ([3] if teacher == "logits" else []))
    assert (each[~taught] == 0).all() and (each[taught] > 0).all()
    loss = student.distill_loss(ids, listed, values, teacher=teacher)
    assert abs(float(loss.detach()) - each[taught].mean()) < 1e-5 * each[taught].mean()
    values[5, 0] = math.nan                                     # a NaN is not nothing
    assert math.isnan(float(student.distill_loss(ids, listed, values, teacher=teacher).detach()))
    none = student.distill_loss(ids[:3], listed[:3], values[:3], teacher=teacher)
    none.backward()
    assert float(none.detach()) == 0 and all(not t.grad.any() for t in student.tensors())
