"""The 64-bit forms of the operators around the layers: their gradients against central differences, their stated special cases."""
import numpy as np
import pytest

from oracle import net


def _numeric(f, x, eps=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        old = x[i]
        x[i] = old + eps
        hi = f()
        x[i] = old - eps
        g[i] = (hi - f()) / (2 * eps)
        x[i] = old
    return g


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("gate_rows", [0, 1, 2])
@pytest.mark.parametrize("branch", [True, False])
def test_block_norm_gradients_are_differences(kind, gate_rows, branch):
    rng = np.random.default_rng(5)
    B, n = 5, 4
    x, f = rng.standard_normal((B, n)), rng.standard_normal((B, n)) + 0.3
    p = dict(w_post=rng.standard_normal(n), b_post=rng.standard_normal(n), gate=rng.standard_normal((1 if not gate_rows else -(-B // gate_rows), n)),
             w_pre=rng.standard_normal(n), b_pre=rng.standard_normal(n))
    gx_out, gh = rng.standard_normal((B, n)), rng.standard_normal((B, n))
    args = dict(kind=kind, residual_scale=0.7, gate_rows=gate_rows)

    def loss():
        s = net.block_norm(x, f if branch else None, p, eps=1e-3, **args)
        return (s["x_out"] * gx_out).sum() + (s["h"] * gh).sum()

    g, _ = net.block_norm_backward(net.block_norm(x, f if branch else None, p, eps=1e-3, **args), p, gx_out, gh, **args)
    for name, t in dict(x=x, f=f, **p).items():
        if not branch and name in ("f", "w_post", "b_post", "gate"):
            continue
        np.testing.assert_allclose(g["g" + name], _numeric(loss, t), rtol=1e-6, atol=1e-7, err_msg=name)


def test_embedding_gradient_is_the_transpose():
    rng = np.random.default_rng(6)
    ids, table, gy = np.array([3, -1, 0, 3, 7, 5]), rng.standard_normal((5, 3)), rng.standard_normal((6, 3))
    y = net.embedding(ids, table, 0.5)
    assert not y[[1, 4, 5]].any() and np.array_equal(y[0], 0.5 * table[3])
    g, _ = net.embedding_backward(ids, gy, 5, 0.5)
    assert np.isclose((y * gy).sum(), (g * table).sum())
    np.testing.assert_allclose(g[3], 0.5 * (gy[0] + gy[3]))


@pytest.mark.parametrize("temperature", [1.0, 0.5])
def test_token_logprob_gradient_is_differences(temperature):
    rng = np.random.default_rng(7)
    z, ids = rng.standard_normal((4, 6)), np.array([2, -1, 5, 0])
    z[2, 1] = -np.inf
    a, b = rng.standard_normal(4), rng.standard_normal(4)

    def loss():
        o = net.token_logprob(z, ids, temperature)
        return (o["logp"] * a).sum() + (o["entropy"] * b).sum()

    g, _ = net.token_logprob_backward(net.token_logprob(z, ids, temperature), ids, a, b, temperature)
    assert g[2, 1] == 0.0
    z[2, 1] = -800.0
    np.testing.assert_allclose(g, _numeric(loss, z), rtol=1e-6, atol=1e-8)


def test_token_logprob_special_rows():
    z = np.array([[-np.inf] * 4, [1.0, np.nan, 2.0, 3.0], [1.0, np.inf, 2.0, 3.0], [2.0, 2.0, -0.0, 0.0]])
    o = net.token_logprob(z, np.array([1, 1, -1, 0]), top=3)
    assert o["logp"][0] == -np.inf and o["entropy"][0] == 0 and list(o["top_ids"][0]) == [0, 1, 2]
    assert np.isnan(o["logp"][1]) and list(o["top_ids"][1]) == [1, 3, 2]
    assert o["logp"][2] == 0 and np.isnan(o["entropy"][2]) and list(o["top_ids"][2]) == [1, 3, 2]
    assert list(o["top_ids"][3]) == [0, 1, 2]


def test_clip_factor():
    assert net.clip([np.array([3.0]), np.array([4.0])], 1.0) == (5.0, 0.2)
    assert net.clip([np.array([3.0, 4.0])], 6.0) == (5.0, 1.0)
    assert net.clip([np.array([3.0, np.inf])], 6.0)[1] == 1.0
