"""The operators around the layers without a GPU: exports, workspace sizes, and what their C entries refuse before anything is launched."""
import ctypes
import os

import pytest
import torch

from paper_2408_11200_amd import binding, build, net, workloads
from test_abi import declared_functions

OK, INVALID, UNSUPPORTED, WORKSPACE = binding.KAN_OK, binding.KAN_ERR_INVALID_ARG, binding.KAN_ERR_UNSUPPORTED, binding.KAN_ERR_WORKSPACE
A = 4096          # stands for an aligned device address: nothing here gets as far as reading it


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return net.load()


def test_every_declared_symbol_is_exported(lib):
    names = declared_functions("kan_net.h")
    assert set(net.EXPORTS) == set(names) and all(hasattr(lib, n) for n in names)


def desc(n=64, norm=0, eps=1e-5, gate_rows=0, stream=0, branch=0):
    return ctypes.byref(net.KanBlockNormDesc(n, norm, eps, 1.0, gate_rows, stream, branch))


def test_block_norm_refusals(lib):
    forward = lambda d, B=4, x=A, f=A, x_out=A, h=A, stats=None, p=net.KanBlockNormParams(): lib.kan_block_norm_forward(
        d, B, x, f, ctypes.byref(p), x_out, h, stats, None)
    assert forward(desc(), B=0, x=None, f=None) == OK
    for d in (None, desc(n=0), desc(n=-3), desc(eps=0.0), desc(eps=float("nan")), desc(gate_rows=-1)):
        assert forward(d) == INVALID
    for d in (desc(n=16385), desc(norm=2), desc(stream=2), desc(branch=5), desc(stream=0, branch=1)):
        assert forward(d) == UNSUPPORTED
    assert forward(desc(), B=-1) == INVALID and forward(desc(), x=None) == INVALID and forward(desc(), x_out=None) == INVALID
    assert forward(desc(), f=None, h=None) == INVALID
    assert forward(desc(), x=A + 2) == INVALID and forward(desc(), stats=A + 1) == INVALID
    assert forward(desc(stream=1, branch=1), x=A + 1) == INVALID
    assert forward(desc(), p=net.KanBlockNormParams(A + 2)) == INVALID
    need = lib.kan_block_norm_workspace_bytes(desc(), 4)
    assert need > 0 and need % 256 == 0 and lib.kan_block_norm_workspace_bytes(desc(n=0), 4) == 0 and lib.kan_block_norm_workspace_bytes(desc(), 0) == 0
    sums = net.KanBlockNormGrads(A, A, A, A, A)
    backward = lambda d=desc(), B=4, x=A, f=A, stats=A, gx_out=A, gh=A, gx=A, gf=A, g=sums, ws=A, size=need: lib.kan_block_norm_backward(
        d, B, x, f, None, stats, gx_out, gh, gx, gf, ctypes.byref(g), ws, size, None)
    assert backward(x=None) == INVALID and backward(stats=None) == INVALID and backward(gx_out=None, gh=None) == INVALID
    assert backward(f=None) == INVALID and backward(gf=A + 2) == INVALID and backward(g=net.KanBlockNormGrads(A + 3)) == INVALID
    assert backward(f=None, gf=None, g=net.KanBlockNormGrads(None, None, A)) == INVALID
    assert backward(ws=None) == WORKSPACE and backward(ws=A + 16) == WORKSPACE and backward(size=need - 1) == WORKSPACE


def test_block_norm_workspace_is_a_share_of_the_rows():
    """Partial sums of the parameters, on the batches that training has."""
    for n, B in ((512, 16384), (4096, 16384), (64, 1 << 20), (8192, 8192)):
        for gate_rows in (0, 1, 117, 2048):
            spec = workloads.BlockNormSpec(n, gate_rows=gate_rows)
            assert 0 < net.kan_block_norm_workspace_bytes(spec, B) <= B * n * 4 * 2


def test_embedding_refusals(lib):
    forward = lambda T=4, V=10, n=8, ids=A, table=A, tt=0, y=A, yt=0: lib.kan_embedding_forward(T, V, n, ids, table, tt, 1.0, y, yt, None)
    assert forward(T=0, ids=None) == OK
    assert INVALID == forward(T=-1) == forward(V=0) == forward(n=0) == forward(ids=None) == forward(table=None) == forward(y=None) == forward(ids=A + 4)
    assert INVALID == forward(table=A + 2) == forward(tt=1, table=A + 1)
    assert UNSUPPORTED == forward(tt=0, yt=1) == forward(tt=3) == forward(T=1 << 31) == forward(V=1 << 31)
    need = lib.kan_embedding_workspace_bytes(4, 10, 8)
    assert need > 0 and lib.kan_embedding_workspace_bytes(-1, 10, 8) == 0 and lib.kan_embedding_workspace_bytes(0, 10, 8) == 0
    backward = lambda T=4, V=10, n=8, ids=A, gy=A, g=A, ws=A, size=need: lib.kan_embedding_backward(T, V, n, ids, gy, 0, 1.0, g, 0, ws, size, None)
    assert INVALID == backward(g=None) == backward(gy=None) == backward(ids=None) == backward(T=-1) == backward(gy=A + 1)
    assert WORKSPACE == backward(ws=None) == backward(ws=A + 8) == backward(size=need - 1)


def test_token_logprob_refusals(lib):
    forward = lambda R=2, V=9, z=A, t=0, stride=9, ids=A, temp=1.0, top=0, logp=A, ti=A, tl=A: lib.kan_token_logprob_forward(
        R, V, z, t, stride, ids, temp, top, logp, None, None, ti, tl, None, 0, None)
    assert forward(R=0, z=None) == OK
    assert INVALID == forward(R=-1) == forward(V=0) == forward(stride=8) == forward(temp=0.0) == forward(temp=float("nan")) == forward(temp=float("inf"))
    assert INVALID == forward(z=None) == forward(ids=None) == forward(top=10) == forward(top=-1) == forward(top=2, ti=None) == forward(top=2, tl=None)
    assert INVALID == forward(z=A + 2) == forward(z=A + 1, t=1) == forward(ids=A + 4) == forward(logp=A + 1)
    assert UNSUPPORTED == forward(t=2) == forward(V=100, stride=100, top=65) == forward(V=1 << 31, stride=1 << 31)
    backward = lambda R=2, z=A, ids=A, stats=A, h=A, a=A, b=A, g=A: lib.kan_token_logprob_backward(R, 9, z, 0, 9, ids, 1.0, stats, h, a, b, g, None)
    assert backward(R=0, z=None) == OK
    assert INVALID == backward(z=None) == backward(stats=None) == backward(g=None) == backward(a=None, b=None) == backward(ids=None) == backward(h=None)
    assert INVALID == backward(g=A + 2) == backward(a=A + 1)


def test_clip_refusals(lib):
    def run(data=A, out=A, count=4, kind=0, n=1, max_norm=1.0, norm=A, ws=A, size=lib.kan_clip_workspace_bytes(1)):
        refs = (net.KanTensorRef * 1)(net.KanTensorRef(data, out, count, kind))
        return lib.kan_clip_gradients(n, refs, max_norm, norm, ws, size, None)
    assert INVALID == run(data=None) == run(out=None) == run(count=-1) == run(n=-1) == run(norm=None) == run(norm=A + 1) == run(data=A + 2) == run(out=A + 1)
    assert INVALID == run(max_norm=-1.0) == run(max_norm=float("nan")) == run(max_norm=float("inf")) == lib.kan_clip_gradients(2, None, 1.0, A, A, 1 << 20, None)
    assert UNSUPPORTED == run(kind=7)
    assert WORKSPACE == run(ws=None) == run(ws=A + 8) == run(size=100)
    assert lib.kan_clip_workspace_bytes(-1) == 0 and lib.kan_clip_workspace_bytes(1 << 20) >= lib.kan_clip_workspace_bytes(1) > 0


def test_front_ends_refuse_host_tensors_and_wrong_shapes():
    spec, x = workloads.BlockNormSpec(8), torch.zeros((2, 8))
    with pytest.raises(AssertionError):
        net.kan_block_norm_forward(spec, x, x, {}, x_out=x, h=x)
    with pytest.raises(AssertionError):
        net.kan_block_norm_forward(spec, torch.zeros((2, 7)), None, {})
    with pytest.raises(AssertionError):
        net.kan_embedding_forward(torch.zeros(3, dtype=torch.int64), x, y=torch.zeros((3, 8)))
    with pytest.raises(AssertionError):
        net.kan_token_logprob_forward(x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(AssertionError):
        net.kan_clip_gradients([x], 1.0)
    from paper_2408_11200_amd import autograd
    for call in (lambda: autograd.block_norm(spec, x, x), lambda: autograd.block_norm(spec, x, torch.zeros((2, 7))),
                 lambda: autograd.embedding(torch.zeros(3, dtype=torch.int64), x), lambda: autograd.token_logprob(x, torch.zeros(2, dtype=torch.int64)),
                 lambda: autograd.token_logprob(x, torch.zeros(3, dtype=torch.int64)), lambda: autograd.clip_gradients([x], 1.0),
                 lambda: autograd.embedding(torch.zeros(3, dtype=torch.int64), x, 1.0, torch.float64)):
        with pytest.raises(AssertionError):
            call()
