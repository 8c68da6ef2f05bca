"""A residual KAN network on tokens: the operators of include/kan_net.h around KAN layers, trained and asked for its most likely tokens.

The next token from the `context` tokens before it: their rows of an embedding table side by side are the residual stream, every block is a
norm, a KAN layer as wide as the stream, and a second norm with a gate and the residual scale (fused over the boundary between two blocks);
a last KAN layer gives the logits.  The norms keep what the layers read on their grids.  A step is the log probabilities' loss with its
gradient, the gradients clipped to a norm, and Adam; every operator of it but Adam runs in the HIP library.

    python -m paper_2408_11200_amd.tokens --steps 300
"""
import argparse
import math

import numpy as np
import torch

from . import autograd, workloads

GRID = 3.0          # the layers' grids are [-3, 3]: three deviations of a normed channel


class TokenNet:
    def __init__(self, vocab=64, context=2, embed=32, blocks=2, seed=0):
        rng = np.random.default_rng(seed)
        self.vocab, self.context, self.n = vocab, context, context * embed
        n = self.n
        self.scale = math.sqrt(embed)
        self.boundary = workloads.BlockNormSpec(n, "layer", residual_scale=1.0)
        self.block = workloads.KanLayerSpec(n, n, 8, 3, -GRID, GRID)
        self.head = workloads.KanLayerSpec(n, vocab, 8, 3, -GRID, GRID)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().requires_grad_(True)
        kan = lambda spec: {k: dev(a) for k, a in workloads.kan_params(rng, spec, 0.1, w_s_std=spec.n_in ** -0.5, w_b_std=spec.n_in ** -0.5).items()}
        self.table = dev(rng.standard_normal((vocab, embed)) / self.scale)
        self.first = dict(w_pre=dev(np.ones(n)), b_pre=dev(np.zeros(n)))
        # a small gate: a block starts close to passing the stream on
        self.norms = [dict(w_post=dev(np.ones(n)), b_post=dev(np.zeros(n)), gate=dev(np.full((1, n), 0.3)), w_pre=dev(np.ones(n)),
                           b_pre=dev(np.zeros(n))) for _ in range(blocks)]
        self.layers = [kan(self.block) for _ in range(blocks)]
        self.out = kan(self.head)

    def tensors(self):
        return [self.table, *self.first.values(), *[t for p in self.norms + self.layers for t in p.values()], *self.out.values()]

    def logits(self, ids):
        """ids[B][context] -> logits[B][vocab]"""
        x = autograd.embedding(ids, self.table, self.scale).view(ids.shape[0], self.n)
        x, h = autograd.block_norm(self.boundary, x, **self.first)
        for p, norm in zip(self.layers, self.norms):
            f = autograd.kan_layer(self.block, h, p["coef"], p["w_s"], p["w_b"])
            x, h = autograd.block_norm(self.boundary, x, f, **norm)
        return autograd.kan_layer(self.head, h, self.out["coef"], self.out["w_s"], self.out["w_b"])

    def loss(self, ids, target, entropy_weight=0.0):
        """Mean negative log probability of the targets (places whose target is -1 left out), less a share of the entropy."""
        logp, entropy, _, _ = autograd.token_logprob(self.logits(ids), target)
        return -(logp.sum() + entropy_weight * entropy.sum()) / (target >= 0).sum().clamp(min=1)

    @torch.no_grad()
    def likely(self, ids, top=5, temperature=1.0):
        """(tokens, log probabilities) of the `top` most likely next tokens of every row of ids."""
        z = self.logits(ids)
        _, _, tokens, logp = autograd.token_logprob(z, torch.full((z.shape[0],), -1, device=z.device), temperature, top)
        return tokens, logp


def train(net, ids, target, steps, batch=4096, lr=3e-3, max_norm=1.0, seed=0, log_every=0):
    """Adam on clipped gradients over random batches; the loss and the gradients' norm before clipping, for each step."""
    opt = torch.optim.Adam(net.tensors(), lr=lr)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    losses, norms = [], []
    for step in range(steps):
        rows = torch.randint(0, ids.shape[0], (batch,), generator=gen, device="cuda")
        opt.zero_grad(set_to_none=True)
        loss = net.loss(ids[rows], target[rows])
        loss.backward()
        norms.append(autograd.clip_gradients([t.grad for t in net.tensors()], max_norm))
        opt.step()
        losses.append(loss.detach())
        if log_every and step % log_every == 0:
            print("step %5d  loss %.4f  gradient norm %.3f" % (step, losses[-1], norms[-1]), flush=True)
    return [float(v) for v in losses], [float(v) for v in norms]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--vocab", type=int, default=64)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--batch", type=int, default=4096)
    args = ap.parse_args()
    ids, target, floor = workloads.token_task(args.vocab)
    ids, target = torch.from_numpy(ids).cuda(), torch.from_numpy(target).cuda()
    net = TokenNet(args.vocab)
    losses, _ = train(net, ids, target, args.steps, args.batch, log_every=max(args.steps // 20, 1))
    tokens, logp = net.likely(ids[:4])
    for row in range(4):
        print("after %s: %s" % (ids[row].tolist(), "  ".join("%d (%.2f)" % (t, p) for t, p in zip(tokens[row].tolist(), logp[row].exp().tolist()))))
    print("loss %.4f -> %.4f after %d steps; %.4f is the least" % (losses[0], losses[-1], args.steps, floor))


if __name__ == "__main__":
    main()
