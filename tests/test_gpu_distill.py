"""The divergence from a teacher's likely tokens and its gradient against the plain form in 64 bits.

Tolerances, from the arithmetic: u = 2^-24 is the rounding of a 32-bit operation.  Only the sum over the tokens off the list is held in 32 bits.  Its relative
error is `delta`: a thread adds one term in 64 (rows of up to 8192 tokens) or 256, at most u of the sum each; 16 more levels join threads, waves and
parts, with a rescaling of 8 u each time the largest logit rises (at most 12 of weight) or sums are joined; an exponent y of base 2 is three roundings, 2.1 u |y| of its term, weighted by
the term itself (|y| <= 20 where terms have weight), and the exponential 2 u: delta = (V / threads + 16 + 12 * 8 + 44) u.
What follows from it: the loss has d loss / d log sum = q_r P - p_r, and half a second derivative of at most q_r P; a listed token's gradient q P q_r; the
factor of the others q_r (1 - q_r) P, whose own term adds (2.1 |y| + 6) u.  Results are rounded once: half a step.
"""
import math

import numpy as np
import pytest
import torch

from oracle import net as plain
from paper_2408_11200_amd import autograd, binding, net

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def dev(a, dtype=F32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def host(t):
    return t.detach().double().cpu().numpy()


def agree(got, ref, tol, name):
    got = host(got)
    fine = np.isfinite(ref)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)]), name
    err = np.abs(got - np.where(fine, ref, 0.0))[fine]
    over = err / (np.broadcast_to(tol, ref.shape)[fine] + 1e-37)
    assert not over.size or over.max() <= 1.0, (name, float(over.max()), float(err.max()))


def delta_of(V):
    return (V / (64 if V <= 8192 else 256) + 16 + 12 * 8 + 44) * U


def check(f, T, V, loss=None, glogits=None, g=None):
    """f: the plain form of the rows."""
    delta = delta_of(V)
    lean = np.abs(f["q_rest"] * f["P"] - f["p_rest"])
    if loss is not None:
        agree(loss, f["loss"], U * np.abs(f["loss"]) + lean * delta + f["q_rest"] * f["P"] * delta ** 2, "loss")
    if glogits is not None:
        g = host(g)[:, None]
        ref = np.where(f["d"] == 0, 0.0, g * f["d"])
        P, q_rest = f["P"][:, None], f["q_rest"][:, None]
        on = f["q"] * P * q_rest * delta / T + 3 * U * np.abs(f["d"])
        off = f["q"] * P / T * (1 - q_rest) * delta + np.abs(f["d"]) * (delta + (2.1 * f["y"] + 6) * U)
        half = 2.0 ** -8 * np.abs(ref) if glogits.dtype == BF16 else 0.0
        agree(glogits, ref, np.abs(np.nan_to_num(g)) * np.where(f["listed"], on, off) * (1 + 2.0 ** -7) + half, "glogits")


def case(R, V, K, seed, dtype=F32, teacher="logp", T=1.0, pad=0, list_dtype=F32, spread=2.0, near=0.7, masked=0, short=True):
    rng = np.random.default_rng(seed)
    buffer = torch.zeros((R, V + pad), dtype=dtype, device="cuda")
    z = rng.standard_normal((R, V)).astype(np.float32) * spread
    t = z + near * rng.standard_normal((R, V)).astype(np.float32)
    if masked:
        z[:, V - masked:] = t[:, V - masked:] = -np.inf
    buffer[:, :V] = dev(z, dtype)
    logits = buffer[:, :V]
    top = dev(t).topk(min(K, V), dim=1)
    values = top.values.double() / T - torch.logsumexp(dev(t).double() / T, 1, keepdim=True) if teacher == "logp" else top.values
    ids = torch.full((R, K), -1, dtype=torch.int64, device="cuda")
    v = torch.zeros((R, K), device="cuda")
    ids[:, :min(K, V)], v[:, :min(K, V)] = top.indices, values.float()
    if short and K > 1:
        ids[::3, K // 2] = -1
        ids[1::5, 0] = V + 3
    return logits, ids, v.to(list_dtype), dev(rng.standard_normal(R) / R)


CASES = [
    # R, V, K, options
    (3, 1, 1, dict()), (5, 2, 1, dict()), (7, 7, 3, dict(T=0.75)), (9, 9, 64, dict(dtype=BF16)), (64, 64, 8, dict(teacher="logits", T=2.0)),
    (33, 157, 5, dict(dtype=BF16, pad=3)), (300, 1000, 8, dict()), (5, 1000, 256, dict(dtype=BF16, teacher="logits")), (17, 4096, 64, dict(dtype=BF16)),
    (17, 4097, 65, dict(pad=1)), (6, 8191, 200, dict(dtype=BF16, list_dtype=BF16)), (520, 8200, 16, dict(teacher="logits", T=3.0, list_dtype=BF16)),
    (1, 32768, 20, dict()), (3, 40001, 64, dict(dtype=BF16, pad=7)), (2, 65537, 256, dict(teacher="logits")), (515, 33000, 20, dict(dtype=BF16, masked=700)),
    (4, 50001, 1, dict(masked=1000, T=0.5)), (3, 140001, 20, dict(dtype=BF16, pad=5)), (90, 131072, 64, dict(dtype=BF16, near=0.1)), (2, 300007, 100, dict(teacher="logits", T=0.75)), (8, 300, 7, dict(near=0.0)), (8, 20000, 64, dict(near=1e-3, short=False)), (8, 2000, 20, dict(spread=8.0)),
]


@pytest.mark.parametrize("R,V,K,options", CASES)
def test_loss_and_gradient(R, V, K, options):
    T, teacher = options.get("T", 1.0), options.get("teacher", "logp")
    logits, ids, values, g = case(R, V, K, R + V + K, **options)
    rows = np.unique(np.concatenate([np.arange(min(R, 8)), [R - 1, R // 2]]))
    f = plain.token_distill(host(logits)[rows], ids.cpu().numpy()[rows], host(values)[rows], T, teacher)
    o = net.kan_token_distill_forward(logits, ids, values, T, teacher)
    check(f, T, V, loss=o["loss"][rows])
    gz = net.kan_token_distill_backward(logits, ids, o, g, T)
    check(f, T, V, glogits=gz[rows], g=g[rows])
    # both at once: the same bits; and again
    for _ in range(2):
        loss, gs = net.kan_token_distill_step(logits, ids, values, g, T, teacher)
        assert torch.equal(loss, o["loss"]) and torch.equal(gs, gz)
    x = logits.detach().requires_grad_(True)
    loss = autograd.token_distill(x, ids, values, T, teacher)
    loss.backward(g)
    assert torch.equal(loss, o["loss"]) and torch.equal(x.grad, gz)
    with torch.no_grad():
        assert torch.equal(autograd.token_distill(logits, ids, values, T, teacher), o["loss"])


# many short rows, at the sizes where a lane's pieces, a row's marks and the rows of a workgroup end; lists of one entry a lane and of four, tokens twice
SHORT = [(R, V, K, dict(dtype=dtype, teacher=teacher, pad=pad, T=T))
         for R, V, K, dtype, teacher, pad, T in (
             (17, 33, 2, F32, "logp", 0, 1.0), (31, 65, 16, BF16, "logits", 1, 0.5), (16, 128, 17, F32, "logp", 0, 1.0), (15, 127, 64, F32, "logits", 3, 2.0),
             (1, 256, 20, BF16, "logp", 0, 1.0), (47, 255, 33, BF16, "logp", 2, 1.0), (4096, 257, 16, F32, "logp", 1, 1.0), (4099, 512, 64, F32, "logits", 0, 0.75),
             (4097, 1000, 20, BF16, "logp", 5, 1.0), (8193, 1021, 32, F32, "logp", 0, 1.0), (8200, 2041, 16, BF16, "logits", 7, 3.0), (8192, 1024, 33, F32, "logp", 0, 1.0))]


@pytest.mark.parametrize("R,V,K,options", SHORT)
def test_short_rows(R, V, K, options):
    """Rows of 16 lanes: against the formulas within the bound of as many additions a lane (V / 16), one call's bits and the two calls', in place, a token twice."""
    T, teacher = options["T"], options["teacher"]
    logits, ids, values, g = case(R, V, K, R + V + K, **options)
    ids[2::7, K - 1] = ids[2::7, 0]
    rows = np.unique(np.concatenate([np.arange(min(R, 20)), [R - 1, R // 2]]))
    f = plain.token_distill(host(logits)[rows], ids.cpu().numpy()[rows], host(values)[rows], T, teacher)
    o = net.kan_token_distill_forward(logits, ids, values, T, teacher)
    check(f, T, 4 * V, loss=o["loss"][rows])            # which counts V / 64 additions
    gz = net.kan_token_distill_backward(logits, ids, o, g, T)
    check(f, T, 4 * V, glogits=gz[rows], g=g[rows])
    loss, gs = net.kan_token_distill_step(logits, ids, values, g, T, teacher)
    assert torch.equal(loss, o["loss"]) and torch.equal(gs, gz)
    own = logits.contiguous().clone()
    assert torch.equal(net.kan_token_distill_backward(own, ids, o, g, T, glogits=own), gz)
    own = logits.contiguous().clone()
    loss, same = net.kan_token_distill_step(own, ids, values, g, T, teacher, glogits=own)
    assert torch.equal(loss, o["loss"]) and torch.equal(same, gz)


@pytest.mark.parametrize("R", [6, 9000])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [24, 100, 1000])
def test_short_rows_keep_to_themselves(dtype, V, R):
    """Rows without a teacher, masked throughout, with a NaN, an infinity or only listed tokens beside ordinary ones, which have the bits that they have alone; and nothing
    written behind the last row."""
    K = 8
    logits, ids, values, g = case(R, V, K, V, dtype=dtype, short=False)
    logits = logits.contiguous()
    a, b = net.kan_token_distill_step(logits, ids, values, g)
    odd = logits.clone()
    oi = ids.clone()
    odd[0::6] = -math.inf
    odd[1::6, V - 1] = math.nan
    odd[2::6, V // 2] = math.inf
    oi[3::6] = -1
    odd[3::6, 0] = math.nan
    odd[4::6] = -math.inf
    odd[4::6] = odd[4::6].scatter(1, ids[4::6], 1.0)
    buffer = torch.full((R + 3, V), 7.0, dtype=dtype, device="cuda")
    loss, gz = net.kan_token_distill_step(odd, oi, values, g, glogits=buffer[:R])
    f = plain.token_distill(host(odd)[:6], oi.cpu().numpy()[:6], host(values)[:6])
    check(f, 1.0, 4 * V, loss=loss[:6], glogits=gz[:6], g=g[:6])
    assert torch.equal(loss[5::6], a[5::6]) and torch.equal(gz[5::6], b[5::6]) and bool((buffer[R:] == 7.0).all())
    assert bool((loss[3::6] == 0).all()) and bool((gz[3::6] == 0).all()) and bool(torch.isnan(loss[1::6]).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [24, 5000, 40000, 140000])
@pytest.mark.parametrize("teacher", ["logp", "logits"])
def test_rows_out_of_the_ordinary(dtype, V, teacher):
    """One kind a row; every entry point gives what the plain form says."""
    rng = np.random.default_rng(V)
    K, R = 6, 16
    z = rng.standard_normal((R, V)).astype(np.float32) * 2
    z = host(dev(z, dtype)).astype(np.float32)
    ids = np.stack([rng.permutation(V)[:K] for _ in range(R)])
    v = np.log(rng.dirichlet(np.ones(K + 1), R)[:, :K]).astype(np.float32)
    lowest = torch.finfo(dtype).min
    z[0] = -np.inf                                      # nothing left by the mask
    z[1, 3] = np.nan
    z[2, ids[2, 0]] = np.inf
    ids[3], z[3] = -1, np.nan                           # no teacher: whatever the logits are
    z[4, ids[4, 1]] = -np.inf                           # a listed token that the student's mask leaves out
    ids[5, 1] = ids[5, 4] = ids[5, 0]                   # a token three times
    others = np.ones(V, bool)
    others[ids[6]] = False
    z[6, others] = -np.inf                              # nothing but the listed tokens
    z[7, np.setdiff1d(np.arange(V), ids[7])] = lowest          # the same, masked by the lowest value
    v[8] = -np.inf                                      # a list without a probability
    v[9, 2] = -np.inf
    v[10] = np.log(0.3)                                 # probabilities that add up to more than 1
    z[11] = lowest                                      # equal logits, all of the lowest value
    z[12] = 0.0
    z[12, ids[12, 0]] = 60.0                            # one likely token, listed
    z[13] = 0.0
    z[13, np.setdiff1d(np.arange(V), ids[13])[0]] = 60.0        # and not
    v[14, 0] = np.nan
    z[15, ids[15]] = -50.0
    g = np.float32(rng.standard_normal(R))
    g[3] = np.nan                                       # of a row without a teacher: no part of anything
    logits, di, dv, dg = dev(z, dtype), torch.from_numpy(ids).cuda(), dev(v), dev(g)
    f = plain.token_distill(host(logits), ids, host(dv), 1.0, teacher)
    assert f["loss"][0] == np.inf and np.isnan(f["loss"][[1, 2, 14]]).all() and f["loss"][3] == 0 and f["loss"][4] == np.inf and f["loss"][8] == 0
    o = net.kan_token_distill_forward(logits, di, dv, 1.0, teacher)
    gz = net.kan_token_distill_backward(logits, di, o, dg)
    loss, gs = net.kan_token_distill_step(logits, di, dv, dg, 1.0, teacher)
    assert torch.equal(loss.nan_to_num(nan=7e7), o["loss"].nan_to_num(nan=7e7)) and torch.equal(gs.nan_to_num(nan=7e7), gz.nan_to_num(nan=7e7))
    check(f, 1.0, V, loss=o["loss"])
    f["d"][3] = 0
    check(f, 1.0, V, glogits=gz, g=dg)
    assert not gz[3].any() and not gz[0].any() and not gz[8].any()
    alone = net.kan_token_distill_forward(logits, di, dv, 1.0, teacher, out=dict(stats=torch.empty((R, K + 2), device="cuda")))
    assert torch.equal(alone["loss"].nan_to_num(nan=7e7), o["loss"].nan_to_num(nan=7e7))


def test_more_tokens_than_are_marked_at_a_time():
    """Rows of more than 2^18 logits that are not cut, lists at the borders of what is marked at a time."""
    R, V, K = 513, (1 << 19) + 77, 24
    logits, ids, values, g = case(4, V, K, 3, dtype=BF16, short=False)
    border = torch.tensor([0, 1, 7, 8, 262143, 262144, 262145, 524287, 524288, V - 1], device="cuda")
    ids[1, :10] = border
    ids[2, :10] = border.flip(0)
    big = logits.repeat(-(-R // 4), 1)[:R].contiguous()
    many = lambda t: t.repeat(-(-R // 4), *[1] * (t.dim() - 1))[:R].contiguous()
    f = plain.token_distill(host(logits), ids.cpu().numpy(), host(values))
    o = net.kan_token_distill_forward(big, many(ids), many(values))
    gz = net.kan_token_distill_backward(big, many(ids), o, many(g))
    check(f, 1.0, V, loss=o["loss"][:4])
    check(f, 1.0, V, glogits=gz[508:512], g=g)
    loss, gs = net.kan_token_distill_step(big, many(ids), many(values), many(g))
    assert torch.equal(loss, o["loss"]) and torch.equal(gs, gz)
    few = net.kan_token_distill_forward(logits, ids, values)        # cut among workgroups
    check(f, 1.0, V, loss=few["loss"])


def test_rows_past_32_bit_offsets():
    R, V, K = 17000, 131072, 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn((R, V), generator=gen, device="cuda", dtype=BF16)
    ids = torch.randint(0, V, (R, K), generator=gen, device="cuda")
    values = torch.full((R, K), -3.0, device="cuda")
    g = torch.rand(R, generator=gen, device="cuda")
    rows = [0, 16383, 16384, 16999]
    f = plain.token_distill(host(logits[rows]), ids[rows].cpu().numpy(), host(values[rows]))
    want = logits[rows].clone()
    o = net.kan_token_distill_forward(logits, ids, values)
    check(f, 1.0, V, loss=o["loss"][rows])
    loss, gz = net.kan_token_distill_step(logits, ids, values, g, glogits=logits)        # in place
    assert gz.data_ptr() == logits.data_ptr() and torch.equal(loss, o["loss"])
    check(f, 1.0, V, glogits=gz[rows], g=g[rows])
    again = net.kan_token_distill_backward(want, ids[rows].contiguous(), dict(stats=o["stats"][rows].contiguous()), g[rows].contiguous())
    assert torch.equal(again, gz[rows])


@pytest.mark.parametrize("R,V", [(700, 100003 // 20), (6, 33000), (6, 140000)])
def test_in_place_and_other_layouts(R, V):
    logits, ids, values, g = case(R, V, 12, 11, dtype=BF16)
    o = net.kan_token_distill_forward(logits, ids, values)
    gz = net.kan_token_distill_backward(logits, ids, o, g)
    a, b = logits.clone(), logits.clone()
    net.kan_token_distill_backward(a, ids, o, g, glogits=a)
    net.kan_token_distill_step(b, ids, values, g, glogits=b)
    assert torch.equal(a, gz) and torch.equal(b, gz)
    # rows that start anywhere, three dimensions, lists that are slices, a broadcast gradient
    buffer = torch.full((R * V + 64 + 3,), 9.0, dtype=BF16, device="cuda")
    shifted = buffer[3:3 + R * V].view(R, V)
    shifted.copy_(logits)
    assert torch.equal(net.kan_token_distill_forward(shifted, ids, values)["loss"], o["loss"])
    x = logits.view(2, R // 2, V).detach().requires_grad_(True)
    wide = torch.stack([ids, ids], 2)[:, :, 0].view(2, R // 2, 12)
    loss = autograd.token_distill(x, wide, values.view(2, R // 2, 12))
    assert loss.shape == (2, R // 2)
    loss.mean().backward()
    even = net.kan_token_distill_backward(logits, ids, o, torch.full((R,), 1.0 / R, device="cuda"))
    assert torch.equal(x.grad.view(R, V), even)


def test_captured_steps_replay_to_the_eager_result():
    logits, ids, values, g = case(40, 140000, 20, 2)
    small, sids, svalues, sg = case(300, 777, 9, 4, dtype=BF16)
    keep = [t.clone() for t in (logits, small)]
    want = [net.kan_token_distill_step(logits, ids, values, g), net.kan_token_distill_step(small, sids, svalues, sg)]
    outs = [tuple(torch.empty_like(t) for t in w) for w in want]
    ws = torch.empty(net.kan_token_distill_workspace_bytes(40, 140000, 20), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        net.kan_token_distill_step(logits, ids, values, g, loss=outs[0][0], glogits=outs[0][1], ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.kan_token_distill_step(logits, ids, values, g, loss=outs[0][0], glogits=outs[0][1], ws=ws)
        net.kan_token_distill_step(small, sids, svalues, sg, loss=outs[1][0], glogits=outs[1][1])
    for turn in range(3):
        shift = float(turn)
        logits.copy_(keep[0] + shift)
        small.copy_(keep[1])
        for o in outs:
            for t in o:
                t.fill_(7.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = net.kan_token_distill_step(logits, ids, values, g)
        assert torch.equal(outs[0][0], eager[0]) and torch.equal(outs[0][1], eager[1])
        assert torch.equal(outs[1][0], want[1][0]) and torch.equal(outs[1][1], want[1][1])


def test_another_stream_and_no_rows():
    logits, ids, values, g = case(50, 5000, 8, 6)
    want = net.kan_token_distill_step(logits, ids, values, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = net.kan_token_distill_step(logits, ids, values, g, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    none = net.kan_token_distill_forward(logits[:0], ids[:0], values[:0])
    assert none["loss"].numel() == 0 and net.kan_token_distill_step(logits[:0], ids[:0], values[:0], g[:0])[1].shape == (0, 5000)
    x = torch.zeros((0, 9), device="cuda", requires_grad=True)
    autograd.token_distill(x, torch.zeros((0, 2), dtype=torch.int64, device="cuda"), torch.zeros((0, 2), device="cuda")).sum().backward()
    assert x.grad.shape == (0, 9)


def test_gradients_against_differences_and_refusals():
    """Along random directions; the loss is exact to half a step of 32 bits."""
    logits, ids, values, _ = case(4, 60, 5, 8)
    x = logits.clone().requires_grad_(True)
    autograd.token_distill(x, ids, values).sum().backward()
    rng = np.random.default_rng(0)
    for _ in range(4):
        way = rng.standard_normal((4, 60)).astype(np.float32)
        h = 2.0 ** -7
        ends = [host(logits) + s * h * way for s in (1, -1)]
        f = [plain.token_distill(np.float32(e), ids.cpu().numpy(), host(values)) for e in ends]
        losses = [net.kan_token_distill_forward(dev(np.float32(e)), ids, values)["loss"] for e in ends]
        for one, ref in zip(losses, f):
            check(ref, 1.0, 60, loss=one)
        slope = float((losses[0].double() - losses[1].double()).sum()) / (2 * h)
        # a third derivative of at most |way|^3 a row, and the losses' errors
        assert abs(slope - float((x.grad.double().cpu() * torch.from_numpy(way)).sum())) < h * h / 6 * (np.abs(way) ** 3).max() * 4 * 4 + 4 * 8 * U / h
    with pytest.raises(RuntimeError):
        autograd.token_distill(x, ids, values.clone().requires_grad_(True))
    y = logits.clone().requires_grad_(True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(autograd.token_distill(y, ids, values).sum(), y, create_graph=True)
    with pytest.raises(binding.KanError):
        autograd.token_distill(logits, ids, values, 0.0)
    with pytest.raises(AssertionError):
        autograd.token_distill(logits, ids, values.double())
    with pytest.raises(AssertionError):
        autograd.token_distill(logits.half(), ids, values)
