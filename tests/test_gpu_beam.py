"""Beam selection against a sort of all scores in 64 bits, and the reordering of states.

Tolerances, from the arithmetic: u = 2^-24.  A score is scores + (z - most) / T - log sum in 64 bits; the sum of exponentials is held in 32: its relative error, and so the score's
absolute one, is at most delta = (V / threads + 16 + 12 * 8 + 44) u (terms a thread adds, levels of joining, rescalings, exponents of up to 20 where terms have weight).  The result is
rounded once, u of itself.  Tokens and parents are those of the sort, but where the ranks of two neighbours lie nearer to one another than that error can tell.
"""
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


def check(got, want, V, scale=None, rows=None):
    """got: tensors of all searches; want: the plain form's of `rows`."""
    rows = slice(None) if rows is None else rows
    delta = (V / (64 if V <= 4096 else 256) + 16 + 12 * 8 + 44) * U
    most = 1.0 if scale is None else float(scale.max())
    scores, ref, ranks = host(got["scores"])[rows], want["scores"], want["ranks"]
    fine = np.isfinite(ref)
    assert np.array_equal(scores[~fine], ref[~fine])
    near = np.zeros(ref.shape, bool)
    with np.errstate(invalid="ignore"):
        gap = ranks[:, :-1] - ranks[:, 1:]
    close = np.where(np.isfinite(gap), gap, np.inf) <= 2 * delta * most
    # ties are told apart by beam and token; what is near but not equal may change places
    close &= np.where(np.isfinite(gap), gap, np.inf) > 0
    near |= close
    near[:, 1:] |= close[:, :-1]
    assert (np.abs(scores - np.where(fine, ref, 0.0))[fine] <= U * np.abs(ref[fine]) + (delta if not near.any() else 3 * delta)).all()
    for name in ("tokens", "parents", "ended"):
        value = got[name].cpu().numpy()[rows]
        assert np.array_equal(value[~near], want[name][~near]), name


def case(N, B, V, seed, dtype=F32, pad=0, step=None, ended=0, dead=0, scale=False):
    rng = np.random.default_rng(seed)
    buffer = torch.zeros((N * B, V + pad), dtype=dtype, device="cuda")
    z = rng.standard_normal((N * B, V)).astype(np.float32) * 2
    if step:
        z = np.round(z / step) * step
    buffer[:, :V] = dev(z, dtype)
    scores = -np.cumsum(rng.uniform(0, 1.5, (N, B)), 1).astype(np.float32)
    order = rng.permuted(np.tile(np.arange(B), (N, 1)), axis=1)
    scores[order >= B - dead] = -np.inf
    flags = order < ended if ended else None
    scales = rng.uniform(0.2, 1.0, (N, B)).astype(np.float32) if scale else None
    return buffer[:, :V], scores, flags, scales


CASES = [
    # N, B, V, top, options
    (1, 1, 1, 1, dict()), (2, 3, 5, 15, dict()), (3, 2, 7, 4, dict(dtype=BF16)), (4, 4, 64, 64, dict(step=0.5)), (5, 1, 200, 64, dict(ended=0)), (7, 5, 157, 10, dict(pad=3, dtype=BF16)),
    (2, 64, 33, 64, dict(step=0.25, scale=True)), (6, 6, 1000, 12, dict(ended=2, scale=True)), (3, 8, 4096, 16, dict(dead=7)), (3, 8, 4097, 16, dict(dead=3, ended=3, dtype=BF16)),
    (130, 4, 8191, 8, dict(dtype=BF16, pad=1)), (1, 4, 32768, 4, dict(dtype=BF16)), (1, 4, 50001, 64, dict()), (4, 32, 40000, 64, dict(dtype=BF16, scale=True)), (16, 4, 33333, 4, dict(dead=3)),
    (1, 64, 40001, 64, dict(ended=20)), (1, 1, 262144, 64, dict(dtype=BF16)), (9, 60, 9000, 60, dict()),
]


@pytest.mark.parametrize("N,B,V,top,options", CASES)
@pytest.mark.parametrize("T", [1.0, 0.75])
def test_selection(N, B, V, top, options, T):
    logits, scores, flags, scale = case(N, B, V, N + B + V + top, **options)
    end = V // 2 if flags is not None else -1
    want = plain.beam_select(host(logits), scores, top, flags, end, scale, T)
    d = lambda a: None if a is None else torch.from_numpy(a).cuda()
    o = net.kan_beam_select(logits, d(scores), top, d(flags), end, d(scale), T)
    check(o, want, V, scale)
    for _ in range(2):
        a = autograd.beam_select(logits, d(scores), top, d(flags), end, d(scale), T)
        assert all(torch.equal(x, o[n]) for x, n in zip(a, ("scores", "tokens", "parents", "ended")))


def test_equal_scores_go_by_beam_and_token():
    """Nothing to choose by: more candidates than there is room for, in parts and in whole rows."""
    for N, B, V, top in ((1, 4, 262144, 64), (2, 8, 30000, 64), (1, 64, 600, 64), (3, 5, 12, 60), (1, 16, 131072, 64)):
        o = net.kan_beam_select(torch.full((N * B, V), -3.0, dtype=BF16, device="cuda"), torch.zeros((N, B), device="cuda"), top)
        flat = torch.arange(top, device="cuda")
        assert torch.equal(o["tokens"], (flat % V).expand(N, top)) and torch.equal(o["parents"], (flat // V).expand(N, top)), (N, B, V)


@pytest.mark.parametrize("V,top", [(30000, 64), (30000, 5), (3000, 64), (100000, 64)])
def test_likely_tokens_at_the_end_of_a_row(V, top):
    """Rising logits: each piece of a row has larger ones than all before it, and the first round's bound keeps them all."""
    z = torch.arange(V, device="cuda").float().repeat(2, 1) * (40.0 / V)
    z[1] = z[1].flip(0)
    want = plain.beam_select(host(z), np.zeros((2, 1)), top)
    check(net.kan_beam_select(z, torch.zeros((2, 1), device="cuda"), top), want, V)
    many = net.kan_beam_select(z.repeat(300, 1), torch.zeros((600, 1), device="cuda"), top)
    check(many, want, V, rows=[0, 1])
    assert torch.equal(many["tokens"], many["tokens"][:2].repeat(300, 1))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [40, 6000, 40000])
def test_beams_out_of_the_ordinary(dtype, V):
    rng = np.random.default_rng(V)
    N, B, top, end = 9, 4, 50, 3
    z = rng.standard_normal((N, B, V)).astype(np.float32)
    scores = -rng.uniform(0, 5, (N, B)).astype(np.float32)
    ended = np.zeros((N, B), bool)
    scale = np.ones((N, B), np.float32)
    scores[0] = -np.inf                         # nothing to go on with
    ended[1] = True                             # four candidates in all
    z[2, 0, 5], z[2, 1, 7], z[2, 2] = np.nan, np.inf, -np.inf
    z[3, :, 6:] = -np.inf                       # six tokens each
    z[4, :, 4:] = torch.finfo(dtype).min        # and the others masked by the lowest value
    scores[5], scores[5, 1] = [np.nan, -1, np.inf, -np.inf], -1.0
    scale[6], ended[6, 3] = [0.0, -1.0, np.nan, 0.5], True
    z[7, 0], z[7, 0, 2] = 0.0, 80.0             # one likely token
    z[8, :, end] = 30.0                         # beams that end now
    logits = dev(z.reshape(N * B, V), dtype)
    want = plain.beam_select(host(logits), scores, top, ended, end, scale)
    assert not np.isfinite(want["scores"][0]).any() and np.isfinite(want["scores"][1]).sum() == 4 and want["ended"][8][:B].all()
    d = torch.from_numpy
    o = net.kan_beam_select(logits, d(scores).cuda(), top, d(ended).cuda(), end, d(scale).cuda())
    check(o, want, V, scale[6:7, 3:])
    assert (o["tokens"][0] == -1).all() and (o["parents"][0] == 0).all() and not o["ended"][0].any()
    assert torch.equal(o["scores"][1][:4], d(scores[1]).cuda().sort(descending=True).values)      # ended: to the bit
    # rows of beams without a candidate are not looked at: NaN there changes nothing
    out = logits.clone().view(N, B, V)
    out[0], out[1] = float("nan"), float("nan")
    again = net.kan_beam_select(out.view(N * B, V), d(scores).cuda(), top, d(ended.astype(np.uint8)).cuda(), end, d(scale).cuda())
    assert all(torch.equal(again[n], o[n]) for n in ("scores", "tokens", "parents", "ended"))


def test_selection_captured_replayed_and_on_another_stream():
    logits, scores, _, _ = case(4, 4, 40000, 3, dtype=BF16)
    s = torch.from_numpy(scores).cuda()
    ws = torch.empty(net.kan_beam_select_workspace_bytes(4, 4, 40000, 8), dtype=torch.uint8, device="cuda")
    out = net.kan_beam_select(logits, s, 8, ws=ws)
    keep = {n: t.clone() for n, t in out.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = net.kan_beam_select(logits, s, 8, stream=side)
    side.synchronize()
    assert all(torch.equal(got[n], keep[n]) for n in keep)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.kan_beam_select(logits, s, 8, out=out, ws=ws)
    for turn in range(3):
        s.copy_(torch.from_numpy(scores).cuda().roll(turn, 1))
        for t in out.values():
            t.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = net.kan_beam_select(logits, s, 8)
        assert all(torch.equal(out[n], eager[n]) for n in eager)
    none = net.kan_beam_select(logits[:0], s[:0], 8)
    assert none["tokens"].shape == (0, 8)
    three = autograd.beam_select(logits.view(4, 4, 40000), s, 8)
    assert torch.equal(three[1], eager["tokens"])
    with pytest.raises(RuntimeError):
        autograd.beam_select(logits.float().requires_grad_(True), s, 8)
    with pytest.raises(binding.KanError):
        autograd.beam_select(logits, s, 8, s > 0)           # ended beams, and no token to end with
    with pytest.raises(AssertionError):
        autograd.beam_select(logits, s.double(), 8)


def test_rows_past_32_bit_offsets():
    """More than 2^32 bytes of logits, more rows than are cut."""
    N, B, V = 545, 32, 131072
    gen = torch.Generator(device="cuda").manual_seed(5)
    logits = torch.randn((N * B, V), generator=gen, device="cuda", dtype=BF16) * 3
    scores = -torch.rand((N, B), generator=gen, device="cuda").cumsum(1)
    o = net.kan_beam_select(logits, scores, 40)
    for n in (0, 511, 512, 544):
        want = plain.beam_select(host(logits[n * B:(n + 1) * B]), host(scores[n:n + 1]), 40)
        check(o, want, V, rows=[n])


# ---- reordering -----------------------------------------------------------------------------

def values(shape, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-100 if dtype != torch.uint8 else 0, 100, shape, generator=gen, device="cuda").to(dtype)


def order(N, B, top, seed, outside=0.1):
    rng = np.random.default_rng(seed)
    p = rng.integers(0, B, (N, top))
    p[rng.random((N, top)) < outside] = rng.choice([-1, B, B + 7, -(1 << 40), 1 << 33])
    stay = rng.random((N, top)) < 0.3
    p[stay] = (np.arange(top) * np.ones((N, 1), int))[stay] % B
    return p


@pytest.mark.parametrize("N,B", [(1, 1), (1, 2), (3, 4), (2, 5), (2, 8), (5, 11), (1, 16), (2, 17), (1, 32), (2, 33), (1, 64)])
@pytest.mark.parametrize("dtype", [torch.uint8, BF16, F32, torch.int64])
def test_states_in_place(N, B, dtype):
    p = order(N, B, B, N * B)
    parents = torch.from_numpy(p).cuda()
    for seed, (shape, dim, cut) in enumerate([((N * B,), 0, None), ((N * B, 7), 0, None), ((N * B, 16), 0, None), ((N * B, 3, 50, 9), 0, 41), ((2, N * B, 5, 33), 1, None),
                                              ((2, 3, N * B, 4, 20), 2, 17), ((6, N * B), 1, None), ((N * B, 1, 1031), 0, None)]):
        for reorder in (net.kan_beam_reorder, autograd.beam_reorder):
            t = values(shape, dtype, seed)
            whole = t.clone()
            part = (lambda x: x) if cut is None else (lambda x: x[..., :cut, :] if len(shape) == 4 else x[..., :cut])
            want = whole.clone()
            part(want).copy_(torch.from_numpy(plain.beam_reorder(p, part(whole).cpu().float().numpy(), B, dim=dim)).to(dtype).cuda())
            assert reorder(parents, [part(t)], B, dim=dim)[0].data_ptr() == t.data_ptr()
            assert torch.equal(t, want), (shape, dim, cut)


@pytest.mark.parametrize("N,B,top", [(1, 1, 3), (3, 4, 8), (4, 8, 4), (2, 3, 20), (1, 40, 7), (2, 5, 40), (1, 7, 64)])
def test_states_into_other_buffers(N, B, top):
    p = order(N, B, top, N + B + top)
    parents = torch.from_numpy(p).cuda()
    for dtype in (torch.uint8, BF16, torch.float64):
        states = [values((N * B, 13), dtype, 1), values((N * B, 4, 70, 6), dtype, 2)[:, :, :61], values((N * B, 999), dtype, 3)]
        out = [values((N * top, 13), dtype, 4), values((N * top, 4, 80, 6), dtype, 5)[:, :, 3:64], values((N * top, 999), dtype, 6)]
        before = [o.clone() for o in out]
        for reorder in (net.kan_beam_reorder, autograd.beam_reorder):
            for o, b in zip(out, before):
                o.copy_(b)
            reorder(parents, states, B, out=out)
            for t, o, b in zip(states, out, before):
                want = plain.beam_reorder(p, t.cpu().float().numpy(), B, b.cpu().float().numpy())
                assert torch.equal(o.cpu().float(), torch.from_numpy(want).float())


def test_many_states_in_one_call():
    """More tensors than a launch takes, some of them empty; every one with its own size."""
    N, B = 3, 6
    p = order(N, B, B, 1)
    states = [values((N * B, k % 37 * 3), BF16, k) for k in range(90)]
    want = [plain.beam_reorder(p, t.cpu().float().numpy(), B) for t in states]
    autograd.beam_reorder(torch.from_numpy(p).cuda(), states, B)
    assert all(np.array_equal(t.cpu().float().numpy(), w) for t, w in zip(states, want))
    assert autograd.beam_reorder(torch.from_numpy(p).cuda(), [], B) == []
    autograd.beam_reorder(torch.zeros((0, 3), dtype=torch.int64, device="cuda"), [torch.zeros((0, 5), device="cuda")], 3)


def test_states_past_32_bit_offsets():
    """Rows of more than 2^30 bytes, swapped and copied in place; an odd length."""
    length = (1 << 30) + 12345
    t = torch.empty((5, length), dtype=torch.uint8, device="cuda")
    for b in range(5):
        t[b].copy_((torch.arange(length, device="cuda") % 251 + b).to(torch.uint8))
    marks = t[:, ::100003].clone()
    autograd.beam_reorder(torch.tensor([[1, 0, 2, 2, 3]], device="cuda"), [t], 5)
    assert torch.equal(t[:, ::100003], marks[[1, 0, 2, 2, 3]])
    assert torch.equal(t[0, -40:], (torch.arange(length - 40, length, device="cuda") % 251 + 1).to(torch.uint8))
    assert torch.equal(t[4, -40:], (torch.arange(length - 40, length, device="cuda") % 251 + 3).to(torch.uint8))


def test_one_state_into_several_outputs_and_two_that_would_change_places():
    """A state is read into as many outputs as are asked for; states that are one another's outputs are refused, not half exchanged."""
    N, B = 3, 4
    p = torch.from_numpy(order(N, B, B, 2, outside=0.0)).cuda()
    a, b = values((N * B, 5, 33), BF16, 1), values((N * B, 5, 33), BF16, 2)
    rows = (p + B * torch.arange(N, device="cuda")[:, None]).view(-1)
    outs = [torch.empty_like(a) for _ in range(3)]
    net.kan_beam_reorder(p, [a, b, a], B, out=outs)
    assert torch.equal(outs[0], a[rows]) and torch.equal(outs[1], b[rows]) and torch.equal(outs[2], a[rows])
    kept = a.clone(), b.clone()
    for call in (net.kan_beam_reorder, autograd.beam_reorder):
        with pytest.raises(RuntimeError):
            call(p, [a, b], B, out=[b, a])
    assert torch.equal(a, kept[0]) and torch.equal(b, kept[1])


def test_reordering_captured_replayed_and_on_another_stream():
    N, B = 4, 4
    p = torch.from_numpy(order(N, B, B, 9, outside=0.0)).cuda()
    t = values((N * B, 3, 501), BF16, 1)
    rows = (p + B * torch.arange(N, device="cuda")[:, None]).view(-1)
    side = torch.cuda.Stream()
    a = t.clone()
    side.wait_stream(torch.cuda.current_stream())
    net.kan_beam_reorder(p, [a], B, stream=side)
    side.synchronize()
    assert torch.equal(a, t[rows])
    state, graph = t.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        autograd.beam_reorder(p, [state], B)
    for _ in range(3):
        before = state.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(state, before[rows])


def test_states_that_are_refused():
    p = torch.zeros((2, 3), dtype=torch.int64, device="cuda")
    t = torch.zeros((6, 8), device="cuda")
    for bad in ([t[:5]], [t.cpu()], [t, t], [t[:1].expand(6, 8)]):
        with pytest.raises((AssertionError, binding.KanError)):
            autograd.beam_reorder(p, bad, 3)
    with pytest.raises(AssertionError):
        autograd.beam_reorder(p, [t], 3, out=[t.double()])
    with pytest.raises(AssertionError):
        autograd.beam_reorder(p, [t], 3, out=[torch.zeros((6, 9), device="cuda")])
    with pytest.raises(AssertionError):
        autograd.beam_reorder(p.int(), [t], 3)
    with pytest.raises(RuntimeError):
        autograd.beam_reorder(p, [t.clone().requires_grad_(True)], 3)
    version = t._version
    autograd.beam_reorder(p, [t], 3)
    assert t._version > version
