"""Distillation, beam selection and the reordering of states without a GPU: workspace sizes, and what the entries refuse before anything is launched."""
import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import net as plain
from paper_2408_11200_amd import binding, build, net

OK, INVALID, UNSUPPORTED, WORKSPACE = binding.KAN_OK, binding.KAN_ERR_INVALID_ARG, binding.KAN_ERR_UNSUPPORTED, binding.KAN_ERR_WORKSPACE
A = 4096          # stands for an aligned device address: nothing here gets as far as reading it


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return net.load()


def test_distill_refusals(lib):
    def forward(R=2, V=9, z=A, t=0, stride=9, K=3, ids=A, values=A, vt=0, form=0, temp=1.0, loss=A, stats=A, ws=None, size=0):
        return lib.kan_token_distill_forward(R, V, z, t, stride, K, ids, values, vt, form, temp, loss, stats, ws, size, None)

    def step(R=2, V=9, z=A, t=0, K=3, ids=A, values=A, temp=1.0, g=A, loss=A, gz=A, ws=None, size=0):
        return lib.kan_token_distill_step(R, V, z, t, V, K, ids, values, 0, 0, temp, g, loss, gz, ws, size, None)

    def backward(R=2, V=9, z=A, t=0, K=3, ids=A, temp=1.0, stats=A, g=A, gz=A):
        return lib.kan_token_distill_backward(R, V, z, t, V, K, ids, temp, stats, g, gz, None)
    for call in (forward, step, backward):
        assert call(R=0, z=None) == OK
        assert INVALID == call(R=-1) == call(V=0) == call(K=0) == call(K=-2) == call(z=None) == call(ids=None) == call(z=A + 2) == call(z=A + 1, t=1) == call(ids=A + 4)
        assert INVALID == call(temp=0.0) == call(temp=-1.0) == call(temp=float("nan")) == call(temp=float("inf")) == call(temp=1e31)
        assert UNSUPPORTED == call(t=2) == call(K=257) == call(R=1 << 31)
    assert UNSUPPORTED == forward(V=1 << 31, stride=1 << 31) == step(V=1 << 31) == backward(V=1 << 31)
    assert INVALID == forward(stride=8) == forward(values=None) == forward(values=A + 2) == forward(values=A + 1, vt=1) == forward(loss=A + 1) == forward(stats=A + 2)
    assert UNSUPPORTED == forward(vt=2) == forward(vt=-1) == forward(form=2) == forward(form=-1)
    assert INVALID == step(g=None) == step(gz=None) == step(g=A + 2) == step(gz=A + 2) == step(loss=A + 1)
    # gradients in place of a slice of wider rows
    assert INVALID == lib.kan_token_distill_backward(2, 9, A, 0, 10, 3, A, 1.0, A, A, A, None) == lib.kan_token_distill_step(2, 9, A, 0, 10, 3, A, A, 0, 0, 1.0, A, A, A, None, 0, None)
    assert INVALID == backward(stats=None) == backward(g=None) == backward(gz=None) == backward(stats=A + 1) == backward(gz=A + 2)
    need = lib.kan_token_distill_workspace_bytes(16, 65536, 20)
    assert need > 0 and need % 256 == 0
    for call in (lambda **k: forward(R=16, V=65536, stride=65536, K=20, **k), lambda **k: step(R=16, V=65536, K=20, **k)):
        assert WORKSPACE == call() == call(ws=A + 16, size=need) == call(ws=A, size=need - 1)
    assert 0 == lib.kan_token_distill_workspace_bytes(-1, 9, 3) == lib.kan_token_distill_workspace_bytes(4, 0, 3) == lib.kan_token_distill_workspace_bytes(4, 9, 0)
    assert 0 == lib.kan_token_distill_workspace_bytes(4, 65536, 257) == lib.kan_token_distill_workspace_bytes(0, 65536, 3)


def test_select_refusals(lib):
    def run(N=2, B=3, V=9, z=A, t=0, stride=9, scores=A, ended=None, scale=None, end=-1, temp=1.0, top=4, out=A, tokens=A, parents=A, flags=A, ws=A, size=1 << 20):
        return lib.kan_beam_select(N, B, V, z, t, stride, scores, ended, scale, end, temp, top, out, tokens, parents, flags, ws, size, None)
    assert run(N=0, z=None) == OK
    assert INVALID == run(N=-1) == run(B=0) == run(V=0) == run(top=0) == run(top=28) == run(stride=8) == run(temp=0.0) == run(temp=float("nan"))
    assert INVALID == run(end=9) == run(end=-2) == run(ended=A, end=-1) == run(z=None) == run(scores=None) == run(out=None) == run(tokens=None) == run(parents=None)
    assert INVALID == run(z=A + 2) == run(z=A + 1, t=1) == run(scores=A + 2) == run(scale=A + 1) == run(out=A + 3) == run(tokens=A + 4) == run(parents=A + 4)
    assert UNSUPPORTED == run(t=2) == run(B=65) == run(top=65, V=100, stride=100) == run(V=1 << 31, stride=1 << 31) == run(N=1 << 24) == run(N=(1 << 24) // 3)
    need = lib.kan_beam_select_workspace_bytes(2, 3, 9, 4)
    assert need > 0 and need % 256 == 0
    assert WORKSPACE == run(ws=None) == run(ws=A + 8, size=need) == run(size=need - 1)
    assert 0 == lib.kan_beam_select_workspace_bytes(2, 0, 9, 1) == lib.kan_beam_select_workspace_bytes(-1, 3, 9, 1) == lib.kan_beam_select_workspace_bytes(2, 65, 9, 1)


def state(data=1 << 16, out=1 << 16, outer=1, inner=1, size=24, stride=(0, 24, 0), out_stride=None):
    three = ctypes.c_int64 * 3
    return net.KanStateRef(data, out, outer, inner, size, three(*stride), three(*(out_stride or stride)))


def test_reorder_refusals(lib):
    def run(*states, N=2, B=3, top=3, parents=A, n=None):
        return lib.kan_beam_reorder(N, B, top, parents, len(states) if n is None else n, (net.KanStateRef * max(len(states), 1))(*states), None)
    s = state(data=1 << 20)
    assert run(s, N=0, parents=None) == OK and run() == OK and run(state(size=0)) == OK and run(state(data=None, out=None, outer=0)) == OK
    assert INVALID == run(s, N=-1) == run(s, B=0) == run(s, top=0) == run(s, n=-1) == run(s, parents=None) == run(s, parents=A + 4)
    assert INVALID == run(state(data=None)) == run(state(out=None)) == run(state(size=-1)) == run(state(outer=-1)) == run(state(inner=-1))
    assert INVALID == lib.kan_beam_reorder(2, 3, 3, A, 1, None, None)
    assert UNSUPPORTED == run(s, B=65) == run(s, top=65) == run(s, N=1 << 26)
    # rows, runs or blocks of an output on top of one another
    assert INVALID == run(state(data=1 << 20, stride=(0, 23, 0))) == run(state(data=1 << 20, inner=4, size=8, stride=(0, 24, 8))) == run(state(data=1 << 20, outer=2, stride=(100, 24, 0)))
    assert INVALID == run(state(data=1 << 20, stride=(0, 0, 0))) == run(state(data=1 << 20, stride=(0, -24, 0))) == run(state(data=1 << 20, outer=2, stride=(0, 24, 0)))
    # in place: as many rows as there were, where they were; and no tensor twice
    assert INVALID == run(state(), top=2) == run(state(stride=(0, 24, 0), out_stride=(0, 32, 0))) == run(s, s) == run(state(), state(data=1 << 20, out=(1 << 16) + 240), state())
    # the parents among what is written
    assert INVALID == run(state(data=1 << 20, out=A)) == run(state(data=1 << 20, out=A - 120)) == run(s, state(data=2 << 20, out=A + 40))
    # more pieces than a number of 32 bits counts
    assert UNSUPPORTED == run(state(data=1 << 20, size=1 << 36, stride=(0, 1 << 36, 0))) == run(state(data=1 << 20, outer=1 << 20, inner=1 << 12, size=1, stride=(1 << 20, 4096, 1)))


def test_reorder_refuses_a_state_that_is_written_as_another_ones_output(lib):
    """Two states that would change places, and one that is read into an output while it is reordered in place: whoever comes first would decide."""
    def run(*states, N=2, B=3, top=3):
        return lib.kan_beam_reorder(N, B, top, A, len(states), (net.KanStateRef * len(states))(*states), None)
    a, b, c = 1 << 20, 2 << 20, 3 << 20
    assert INVALID == run(state(data=a, out=b), state(data=b, out=a)) == run(state(data=a, out=a), state(data=a, out=c)) == run(state(data=b, out=c), state(data=a, out=b))
    assert INVALID == run(state(data=a, out=c), state(data=b, out=1 << 22), state(data=b, out=a))
    # one that is not looked at is in nobody's way
    assert run(state(data=a, out=b, size=0), state(data=b, out=a, outer=0)) == OK


def test_reorder_refuses_outputs_that_cross(lib):
    """A state shifted within its own buffer, outputs that begin at different bytes of one another, and one that is read behind its first row by another entry."""
    def run(*states, N=2, B=3, top=3):
        return lib.kan_beam_reorder(N, B, top, A, len(states), (net.KanStateRef * len(states))(*states), None)
    a, b, row = 1 << 20, 2 << 20, 24
    assert INVALID == run(state(data=a, out=a + 8, size=16)) == run(state(data=a + 8, out=a, size=16)) == run(state(data=a, out=a + row)) == run(state(data=a, out=a - 5 * row))
    assert INVALID == run(state(data=a, out=b), state(data=a, out=b + 5 * row + 23)) == run(state(data=b, out=b), state(data=a, out=b + 8)) == run(state(data=a, out=b), state(data=b - 23, out=3 << 20))
    # from the buffer's first half of a row into its second one, and a byte more; more rows out than in
    assert INVALID == run(state(data=a, out=a + 12, size=13)) == run(state(data=a, out=a + 6 * row), state(data=b, out=a + 12 * row - 1))
    assert INVALID == run(state(data=a, out=a + 2 * row, size=8, stride=(0, row, 0), out_stride=(0, row, 0)), top=2)
    # blocks and runs: the other's row, run or block only
    wide = dict(outer=3, inner=2, size=4)
    assert INVALID == run(state(data=a, out=b, stride=(960, 96, 24), **wide), state(data=a, out=b + 960 + 96 * 4 + 24 + 3, stride=(960, 96, 24), **wide))
    # many entries, the two that cross far from one another
    many = [state(data=a, out=b + 1024 * k) for k in range(700)]
    many[650] = state(data=a, out=b + 1024 * 7 + 143)
    assert INVALID == run(*many)
    # strides of which neither lies within the other: nothing crosses, but it takes too long to tell
    uneven = state(data=a + 8, out=1 << 40, outer=100000, size=8, stride=(16 * 999, 1 << 34, 0), out_stride=(8, 1 << 34, 0))
    assert UNSUPPORTED == run(uneven, state(data=1 << 41, out=a, outer=100000, size=8, stride=(16 * 1001, 1 << 35, 0)), N=1, B=1, top=1)
    assert INVALID == run(state(data=a, out=b, stride=(0, -(1 << 63), 0), out_stride=(0, 24, 0)))
    # no memory is like that
    assert INVALID == run(state(data=a, out=(1 << 64) - 100)) == run(state(data=a, out=b, outer=2, stride=(1 << 62, 24, 0))) == run(state(data=64, out=b, stride=(0, -24, 0), out_stride=(0, 24, 0)))


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would be launched, at addresses that are not there")
def test_reorder_refuses_what_crosses_and_nothing_else(lib):
    """Against a list of all bytes: strides that lie within one another and others, rows that are one and the same, rows backwards, entries in place and not."""
    rng = np.random.default_rng(3)
    three, base = ctypes.c_int64 * 3, 1 << 20

    def touched(at, counts, strides, size):
        where = at + sum(np.arange(n).reshape([-1 if k == d else 1 for k in range(4)]) * s for d, (n, s) in enumerate(zip((*counts, size), (*strides, 1))))
        return np.unique(where.ravel())

    refused = 0
    for _ in range(6000):
        N, B, top = int(rng.integers(1, 3)), int(rng.integers(1, 4)), int(rng.integers(1, 4))
        entries, parts, fine = [], [], True
        for _ in range(int(rng.integers(1, 4))):
            outer, inner, size = (int(v) for v in rng.integers(1, 4, 3))
            counts = (outer, N * top, inner)
            out_stride, extent = [0, 0, 0], size
            for d in rng.permutation(3):
                out_stride[d] = int(extent + rng.integers(0, 12))
                extent += out_stride[d] * (counts[d] - 1)
            out = base + int(rng.integers(0, 400))
            place = bool(rng.random() < 0.4) and top == B
            stride = out_stride if place else list(out_stride if rng.random() < 0.5 else (int(v) for v in rng.integers(-9, 40, 3)))
            data = out if place else base + int(rng.integers(0, 400))
            if data == out and not place:
                fine = False
            entries.append(net.KanStateRef(data, out, outer, inner, size, three(*stride), three(*out_stride)))
            parts.append((True, touched(out, counts, out_stride, size)))
            if not place:
                parts.append((False, touched(data, (outer, N * B, inner), stride, size)))
        if not fine:
            continue
        cross = any((p[0] or q[0]) and len(np.intersect1d(p[1], q[1])) for i, p in enumerate(parts) for q in parts[:i])
        refused += cross
        rc = lib.kan_beam_reorder(N, B, top, A, len(entries), (net.KanStateRef * len(entries))(*entries), None)
        assert rc == (INVALID if cross else binding.KAN_ERR_HIP), (N, B, top, [(e.data - base, e.out - base, e.outer, e.inner, e.bytes, list(e.stride), list(e.out_stride)) for e in entries])
    assert 1000 < refused < 5000


def test_front_ends_refuse_host_tensors_and_wrong_shapes():
    from paper_2408_11200_amd import autograd
    z, ids, v, s = torch.zeros((6, 9)), torch.zeros((6, 2), dtype=torch.int64), torch.zeros((6, 2)), torch.zeros((2, 3))
    parents = torch.zeros((2, 3), dtype=torch.int64)
    for call in (lambda: net.kan_token_distill_forward(z, ids, v), lambda: net.kan_token_distill_step(z, ids, v, torch.zeros(6)),
                 lambda: net.kan_token_distill_backward(z, ids, dict(stats=torch.zeros((6, 4))), torch.zeros(6)), lambda: net.kan_beam_select(z, s),
                 lambda: net.kan_beam_reorder(parents, [z], 3), lambda: autograd.token_distill(z, ids, v), lambda: autograd.token_distill(z, ids[:5], v[:5]),
                 lambda: autograd.token_distill(z, ids, v[:, :1]), lambda: autograd.token_distill(z, ids[:, :0], v[:, :0]), lambda: autograd.beam_select(z, s),
                 lambda: autograd.beam_select(z, s.view(-1)), lambda: autograd.beam_select(z[:5], s), lambda: autograd.beam_select(z, s, 0), lambda: autograd.beam_select(z, s, 65),
                 lambda: autograd.beam_reorder(parents, [z], 3), lambda: autograd.beam_reorder(parents.view(-1), [z], 3)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(KeyError):
        autograd.token_distill(z, ids, v, teacher="odds")


def test_states_lie_evenly_or_are_refused():
    """What a binding makes of a tensor's strides (addresses only: nothing is launched)."""
    of = lambda t, o, dim: net._state(t.shape, t.stride(), o.stride(), t.element_size(), dim)
    t = torch.zeros((2, 6, 5, 8, 3))
    cut = t[:, :, :, :4]
    assert of(cut, cut, 1) == (2, 5, 48, 6 * 480, 480, 96, 6 * 480, 480, 96)
    assert of(t, t, 0) == (1, 1, 6 * 5 * 8 * 3 * 4, 0, 6 * 480, 0, 0, 6 * 480, 0) and of(t, t, 4) == (480, 1, 4, 12, 4, 0, 12, 4, 0)
    wide = torch.zeros((2, 6, 5, 16, 3))[:, :, :, 3:11]
    assert of(t, wide, 0) == (1, 30, 96, 0, 6 * 480, 96, 0, 6 * 960, 192)
    with pytest.raises(AssertionError):
        of(t[:, :, :3, :4], t[:, :, :3, :4], 0)
    with pytest.raises(AssertionError):
        of(t[:, :4].transpose(0, 1)[:, :, :4], t[:, :4].transpose(0, 1)[:, :, :4], 3)


# ---- the plain forms themselves, against other ways to the same values ----------------------

@pytest.mark.parametrize("teacher", ["logp", "logits"])
def test_plain_distillation_is_the_gradient_of_its_loss(teacher):
    rng = np.random.default_rng(5)
    R, V, K, T = 6, 11, 4, 0.75
    z = rng.standard_normal((R, V)) * 2
    ids = np.stack([rng.permutation(V)[:K] for _ in range(R)])
    ids[1, 2], ids[2] = -1, V
    ids[3, 1] = ids[3, 0]
    v = np.log(rng.dirichlet(np.ones(K + 1), R)[:, :K]) if teacher == "logp" else rng.standard_normal((R, K))
    f = plain.token_distill(z, ids, v, T, teacher)
    assert (f["loss"][[0, 1, 4, 5]] > 0).all() and f["loss"][2] == 0 and not f["d"][2].any()
    h = 1e-5
    for r in range(R):
        for c in range(V):
            up, down = z.copy(), z.copy()
            up[r, c] += h
            down[r, c] -= h
            slope = (plain.token_distill(up, ids, v, T, teacher)["loss"][r] - plain.token_distill(down, ids, v, T, teacher)["loss"][r]) / (2 * h)
            assert abs(slope - f["d"][r, c]) < 1e-8
    if teacher == "logp":           # the whole vocabulary listed, or a teacher that is the student: the plain divergence, or none
        lp = plain.token_logprob(z, None, T)["lp"]
        same = plain.token_distill(z[[0]], ids[[0]], np.take_along_axis(lp[[0]], ids[[0]], 1), T)
        assert abs(same["loss"][0]) < 1e-14 and np.abs(same["d"]).max() < 1e-15
        p = rng.dirichlet(np.ones(V))
        whole = plain.token_distill(z[[0]], np.arange(V)[None], np.log(p)[None], T)
        assert abs(whole["loss"][0] - (p * (np.log(p) - lp[0])).sum()) < 1e-12


def test_plain_selection_is_a_sort_of_all_scores():
    rng = np.random.default_rng(7)
    N, B, V, top = 3, 4, 13, 9
    z, scores = np.round(rng.standard_normal((N * B, V)) * 2) / 2, rng.standard_normal((N, B))
    scores[0, 1] = -np.inf
    ended = np.zeros((N, B), bool)
    ended[1, 2] = True
    scale = rng.uniform(0.5, 2.0, (N, B))
    o = plain.beam_select(z, scores, top, ended, 5, scale, 0.75)
    lp = plain.token_logprob(z, None, 0.75)["lp"].reshape(N, B, V)
    for n in range(N):
        s = scores[n][:, None] + lp[n]
        for b in range(B):
            if ended[n, b]:
                s[b], s[b, 5] = -np.inf, scores[n, b]
        order = np.argsort(-(s * scale[n][:, None]).ravel(), kind="stable")[:top]
        assert np.array_equal(o["parents"][n], order // V) and np.array_equal(o["tokens"][n], order % V)
        assert np.allclose(o["scores"][n], s.ravel()[order], rtol=1e-14, atol=0)
