"""The network on tokens taught by another one and asked for whole answers: distillation, beam selection and reordering as they are used together."""
import itertools

import numpy as np
import pytest
import torch

from oracle import net as plain
from paper_2408_11200_amd import autograd, net, tokens, workloads

pytestmark = pytest.mark.gpu


def host(t):
    return t.detach().double().cpu().numpy()


def log_probabilities(model, windows, temperature=1.0):
    with torch.no_grad():
        return plain.token_logprob(host(model.logits(windows)), None, temperature)["lp"]


def test_wide_search_finds_the_most_likely_answers_of_all():
    """Three tokens of a vocabulary of five, 64 beams: nothing that leads to one of the ten best of the 125 answers is dropped (each is among the 64 best of its
    25 beginnings).  Scores are sums of three log probabilities of 32-bit logits, each rounded once."""
    model = tokens.TokenNet(vocab=5, embed=8, blocks=1, seed=2)
    ids = torch.tensor([[0, 1], [4, 4], [3, 0]], device="cuda")
    answers, scores = model.search(ids, 3, beams=64)
    every = np.array(list(itertools.product(range(5), repeat=3)))
    for n in range(3):
        lp = np.zeros(125)
        for at in range(3):
            windows = torch.from_numpy(np.concatenate([np.tile(ids[n].cpu().numpy(), (125, 1)), every], 1)[:, at:at + 2].copy()).cuda()
            lp += log_probabilities(model, windows)[np.arange(125), every[:, at]]
        order = np.argsort(-lp, kind="stable")[:10]
        got = host(scores[n])[:10]
        assert np.abs(got - lp[order]).max() <= 3 * 2.0 ** -24 * (np.abs(lp[order]).max() + 64)
        gap = np.diff(lp[np.argsort(-lp)[:11]])
        assert (np.abs(gap) > 1e-4).all() and np.array_equal(answers[n, :10].cpu().numpy(), every[order])


@pytest.mark.parametrize("end_id,length_power,temperature", [(-1, 0.0, 1.0), (2, 0.0, 1.0), (2, 0.8, 0.75), (-1, 0.5, 1.0)])
def test_search_is_the_plain_one(end_id, length_power, temperature):
    """Step by step against the plain selection on the same network's logits: answers, scores and lengths follow the parents."""
    model = tokens.TokenNet(vocab=24, embed=8, blocks=2, seed=5)
    N, B, length = 6, 5, 6
    ids = torch.from_numpy(workloads.token_task(24, n=N)[0]).cuda()
    answers, scores = model.search(ids, length, B, end_id, length_power, temperature)
    window, said = np.repeat(ids.cpu().numpy(), B, 0), np.zeros((N * B, 0), int)
    score, ended, long = np.full((N, B), -np.inf), np.zeros((N, B), bool), np.zeros((N, B))
    score[:, 0] = 0.0
    for at in range(length):
        with torch.no_grad():
            z = host(model.logits(torch.from_numpy(window).cuda()))
        grown = long + ~ended
        o = plain.beam_select(z, np.float32(score), B, ended if end_id >= 0 else None, end_id, np.maximum(grown, 1.0) ** -length_power, temperature)
        rows = (o["parents"] + B * np.arange(N)[:, None]).ravel()
        score, ended, long = o["scores"], o["ended"], grown.ravel()[rows].reshape(N, B)
        said = np.concatenate([said[rows], o["tokens"].reshape(-1, 1)], 1)
        window = np.concatenate([window[rows][:, 1:], o["tokens"].reshape(-1, 1)], 1)
    assert np.array_equal(answers.cpu().numpy(), said.reshape(N, B, length))
    assert np.abs(host(scores) - score).max() <= length * 2.0 ** -24 * (np.abs(score).max() + 64)
    if end_id >= 0:
        got = answers.cpu().numpy()
        first = np.where((got == end_id).any(-1), (got == end_id).argmax(-1), length)
        assert ((got == end_id) | (np.arange(length) < first[..., None])).all()


def test_the_step_from_a_teacher_is_the_losses_gradient():
    """The step's gradients with the loss, handed to the network, against autograd's through the mean divergence: the same bits in every parameter."""
    teacher, student = tokens.TokenNet(40, embed=12, blocks=1, seed=1), tokens.TokenNet(40, embed=8, blocks=1, seed=2)
    ids = torch.from_numpy(workloads.token_task(40, n=256)[0]).cuda()
    likely, logp = teacher.likely(ids, 8)
    assert (logp[:, :-1] >= logp[:, 1:]).all()
    loss = student.distill_loss(ids, likely, logp)
    loss.backward()
    want = [t.grad for t in student.tensors()]
    z = student.logits(ids)
    each, gz = net.kan_token_distill_step(z.detach(), likely, logp, torch.full((256,), 1.0 / 256, device="cuda"))
    got = torch.autograd.grad(z, student.tensors(), gz)
    assert abs(float(each.mean()) - float(loss.detach())) < 1e-6 and all(torch.equal(a, b) for a, b in zip(got, want))
    f = plain.token_distill(host(z), likely.cpu().numpy(), host(logp))
    assert np.abs(host(each) - f["loss"]).max() < 1e-5 and np.abs(host(gz) * 256 - f["d"]).max() < 1e-5
    # rows without a teacher count nowhere
    some = likely.clone()
    some[::2] = -1
    assert torch.equal(autograd.token_distill(z.detach(), some, logp)[::2], torch.zeros(128, device="cuda"))
    assert abs(float(student.distill_loss(ids, some, logp).detach()) - float(each[1::2].mean())) < 1e-6


def test_teaching_and_answering_run():
    teacher, student = tokens.TokenNet(16, embed=8, blocks=1), tokens.TokenNet(16, embed=4, blocks=1, seed=1)
    ids = torch.from_numpy(workloads.token_task(16, n=2048)[0]).cuda()
    losses, norms = tokens.train_from_teacher(student, teacher, ids, 12, top=5, batch=256)
    assert len(losses) == len(norms) == 12 and np.isfinite(losses).all() and min(losses) >= 0
    answers, scores = student.search(ids[:7], 5, beams=3)
    assert answers.shape == (7, 3, 5) and (answers >= 0).all() and (scores[:, :-1] >= scores[:, 1:]).all()
    one, best = student.search(ids[:7], 1, beams=3)
    likely, logp = student.likely(ids[:7], 3)
    assert torch.equal(one[:, :, 0], likely) and torch.allclose(best, logp, rtol=0, atol=1e-6)


def test_traced_operators_give_their_own_bits():
    gen = torch.Generator(device="cuda").manual_seed(0)
    z = torch.randn((12, 50), generator=gen, device="cuda")
    scores = -torch.rand((3, 4), generator=gen, device="cuda")
    ids, logp = torch.randint(0, 50, (12, 4), generator=gen, device="cuda"), torch.full((12, 4), -2.0, device="cuda")

    def both(z, scores, ids, logp):
        return autograd.token_distill(z, ids, logp), *autograd.beam_select(z, scores, 4)

    with torch.no_grad():
        traced = torch.jit.trace(both, (z, scores, ids, logp))
        other = z.flip(0).contiguous()
        for got, want in zip(traced(other, scores, ids, logp), both(other, scores, ids, logp)):
            assert torch.equal(got, want)
