"""The layers as differentiable functions of torch tensors.

The autograd nodes are native (csrc_torch/kan_autograd.cpp, built into _autograd.so next to this file): `forward` calls
kan_forward / ukan_cg_forward_saved, `backward` calls kan_backward_saved / ukan_cg_backward_saved with exactly the gradients
autograd asks for (the backward passes reuse what their forward passes kept: the scale-folded table; for UKAN the
coefficient table and the CG activations).  Lets a stack of
layers be trained with a stock PyTorch optimizer (closed-form regression targets of the paper's
experiments section need nothing else).
"""
import os

import torch

from . import binding

_nodes = None


def _load():
    """The native nodes; raise if they have not been built (there is no fallback)."""
    global _nodes
    if _nodes is None:
        binding.load()
        path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_autograd.so")
        if not os.path.exists(path):
            raise RuntimeError("%s is missing: build it with `python -m paper_2408_11200_amd.build`" % path)
        from . import _autograd
        if _autograd.torch_version != torch.__version__:
            raise RuntimeError("%s was built with torch %s, this is %s: build it again with `python -m paper_2408_11200_amd.build`"
                               % (path, _autograd.torch_version, torch.__version__))
        _nodes = _autograd
    return _nodes


def kan_layer(spec, x, coef, w_s, w_b=None):
    """y = KAN layer `spec` applied to x; differentiable in x, coef, w_s, w_b."""
    return (_nodes or _load()).kan_layer(spec.n_in, spec.n_out, spec.G, spec.k, spec.grid_lo, spec.grid_hi, spec.base_act, x, coef, w_s, w_b)


def ukan_layer(spec, x, params, max_groups):
    """y = UKAN layer `spec` applied to x; `params` maps E, W1, b1, W2, b2, scale (and w_b) to tensors."""
    p = params
    return (_nodes or _load()).ukan_layer(spec.n_in, spec.n_out, spec.k, spec.h, spec.d_pe, spec.d_feat, spec.d_hidden, spec.base_act,
                                          max_groups, x, p["E"], p["W1"], p["b1"], p["W2"], p["b2"], p["scale"], p.get("w_b"))


def block_norm(spec, x, f=None, w_post=None, b_post=None, gate=None, w_pre=None, b_pre=None, want_h=True):
    """The boundary `spec` between two blocks: (x_out, h), x_out = residual_scale x + gate (norm(f) w_post + b_post) and
    h = norm(x_out) w_pre + b_pre.  Without f, the norm in front of the first block: x_out is x; with want_h=False, behind the
    last one: h is None.  Differentiable in all tensors."""
    from . import net
    out = (_nodes or _load()).block_norm(spec.n, net.NORMS[spec.norm], spec.eps, spec.residual_scale, spec.gate_rows, net.TYPE_NAMES[spec.branch], want_h,
                                         x, f, w_post, b_post, gate, w_pre, b_pre)
    return (x if f is None else out[0]), (out[-1] if want_h else None)


def embedding(ids, table, scale=1.0, dtype=None):
    """Rows of `table` by token, times `scale`, in `dtype` (default: the table's); zeros for ids outside the table.  Differentiable in table."""
    dtype = dtype or table.dtype
    assert dtype in (torch.float32, torch.bfloat16), "float32 or bfloat16 rows"
    return (_nodes or _load()).embedding(ids, table, scale, dtype == torch.float32)


def token_logprob(logits, ids, temperature=1.0, top=0):
    """(logp, entropy, top_ids, top_logp) of softmax(logits / temperature), row by row: the log probability of the given token (0 for an
    id outside the vocabulary), the entropy, and the `top` most likely tokens (None for top = 0).  logp and entropy are
    differentiable in logits."""
    out = (_nodes or _load()).token_logprob(logits, ids, temperature, top)
    return tuple(out) if top else (out[0], out[1], None, None)


def clip_gradients(tensors, max_norm, out=None):
    """The norm over all `tensors` (a device tensor; nothing waits for it), and each of them times min(1, max_norm / norm): in place, or
    into the tensors of `out`.  A norm that is not finite leaves the values as they are.  Not differentiable: tensors that require gradients are
    refused where gradients are recorded."""
    return (_nodes or _load()).clip_gradients(list(tensors), max_norm, None if out is None else list(out))
