"""The operators around the layers (include/kan_net.h) against their plain forms in 64 bits.

Tolerances, from the arithmetic: u = 2^-24 is the rounding of a 32-bit operation.  The longest chain of additions in a row's sum is 8
channels a lane and piece, 6 levels in a wave and 16 waves, some 40 of them, and a handful of operations follow: 64 u of the sum of the terms'
magnitudes (what the oracle calls scale), 192 u where a gradient goes through two norms and a sum over the rows.  Sums over a vocabulary
have up to 137 terms a thread and 26 levels, and a term's exponent costs 2 u of itself: 256 u.  A bfloat16 result is rounded once more: 2^-8 of it.
"""
import numpy as np
import pytest
import torch

from oracle import net as plain
from paper_2408_11200_amd import autograd, binding, net, workloads

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def dev(a, dtype=F32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def host(t):
    return t.detach().double().cpu().numpy()


def check(got, ref, scale, ulps, name=""):
    """|got - ref| <= ulps * u * (scale + mean scale of the row), and half a unit of a bfloat16 result; NaN and infinities in the same places."""
    bf = got.dtype == BF16
    got, ref, scale = host(got), np.asarray(ref), np.broadcast_to(scale, np.shape(ref))
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    if not ref.size:
        return
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)]), name
    size = np.where(fine, scale, 0.0)
    tol = ulps * U * (size + size.mean(-1, keepdims=True)) + (2.0 ** -8 * np.abs(np.where(fine, ref, 0.0)) if bf else 0.0) + 1e-37
    err = np.where(fine, np.abs(got - np.where(fine, ref, 0.0)), 0.0)
    assert (err <= tol).all(), (name, float((err / tol).max()))


# ---- block norm -----------------------------------------------------------------------------

def norm_case(B, n, kind, gate_rows, seed, stream=F32, branch=F32, have=("w_post", "b_post", "gate", "w_pre", "b_pre"), offset=0.5):
    rng = np.random.default_rng(seed)
    spec = workloads.BlockNormSpec(n, kind, 1e-5, 0.75, gate_rows, "f32" if branch == F32 else "bf16")
    groups = 1 if not gate_rows else -(-B // gate_rows)
    a = lambda *s: rng.standard_normal(s).astype(np.float32)
    p = dict(w_post=1 + 0.2 * a(n), b_post=0.2 * a(n), gate=0.5 * a(groups, n), w_pre=1 + 0.2 * a(n), b_pre=0.2 * a(n))
    t = dict(x=dev(2.0 * a(B, n) + offset, stream), f=dev(a(B, n) - offset, branch), gx_out=dev(a(B, n), stream), gh=dev(a(B, n), branch))
    return spec, t, {k: dev(v) for k, v in p.items() if k in have}


def norm_reference(spec, t, p, branch=True, gx_out=True, gh=True):
    q = {k: host(v) for k, v in p.items()}
    s = plain.block_norm(host(t["x"]), host(t["f"]) if branch else None, q, spec.norm, spec.eps, spec.residual_scale, spec.gate_rows)
    g, scale = plain.block_norm_backward(s, q, host(t["gx_out"]) if gx_out else None, host(t["gh"]) if gh else None, spec.norm, spec.residual_scale,
                                         spec.gate_rows)
    return s, g, scale


def check_norm(spec, t, p, branch=True, gx_out=True, gh=True):
    s, g, scale = norm_reference(spec, t, p, branch, gx_out, gh)
    f = t["f"] if branch else None
    stats = torch.full((t["x"].shape[0], 4), 7.0, device="cuda")
    x_out, h = net.kan_block_norm_forward(spec, t["x"], f, p, stats=stats, want_h=gh)
    if branch:
        check(x_out, s["x_out"], s["x_out_scale"], 64, "x_out")
    else:
        assert x_out is t["x"]
    if gh:
        check(h, s["h"], s["h_scale"], 64, "h")
    got = net.kan_block_norm_backward(spec, t["x"], f, p, stats, t["gx_out"] if gx_out else None, t["gh"] if gh else None)
    assert set(got) == {"gx"} | ({"gf"} if branch else set()) | {"g" + k for k in p if branch or k in ("w_pre", "b_pre")}
    for name, v in got.items():
        if not gh and name in ("gw_pre", "gb_pre"):
            assert not v.any()
            continue
        check(v, g[name], scale[name], 192, name)
    again = net.kan_block_norm_backward(spec, t["x"], f, p, stats, t["gx_out"] if gx_out else None, t["gh"] if gh else None)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("n", [1, 5, 8, 63, 64, 65, 128, 200, 257, 512, 513, 771, 1024, 2050, 4096, 4100, 8192, 8200, 16384])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_block_norm_widths(n, kind):
    check_norm(*norm_case(37, n, kind, 0, n))


@pytest.mark.parametrize("B", [1, 2, 3, 64, 129, 1000, 2500])
@pytest.mark.parametrize("gate_rows", [0, 1, 2, 7, 64, 500, 4000])
@pytest.mark.parametrize("n", [48, 520])
def test_block_norm_rows_and_gates(B, gate_rows, n):
    check_norm(*norm_case(B, n, "layer" if gate_rows % 2 else "rms", gate_rows, B + gate_rows))


@pytest.mark.parametrize("n", [24, 515, 1030, 4097, 8199])
@pytest.mark.parametrize("types", [(BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("kind,gate_rows", [("rms", 0), ("layer", 5), ("layer", 100)])
def test_block_norm_types(n, types, kind, gate_rows):
    check_norm(*norm_case(130, n, kind, gate_rows, n, *types))


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("branch,gx_out,gh", [(False, True, True), (False, False, True), (True, True, False), (True, False, True)])
def test_block_norm_ends_of_a_network(kind, branch, gx_out, gh):
    check_norm(*norm_case(70, 100, kind, 0, 3), branch=branch, gx_out=gx_out, gh=gh)
    check_norm(*norm_case(70, 1100, kind, 30, 3), branch=branch, gx_out=gx_out, gh=gh)


@pytest.mark.parametrize("n,B,gate_rows", [(1200, 6000, 11), (1200, 6000, 12), (1200, 6000, 13), (1200, 6000, 900), (1200, 6000, 5000), (40, 40000, 5), (40, 40000, 31),
                                           (4400, 1500, 5), (4400, 1500, 6), (4400, 1500, 200), (6144, 700, 1), (6145, 700, 4)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_block_norm_groups_cut(n, B, gate_rows, kind):
    """whole groups a worker, groups in one part, in a few and in many"""
    check_norm(*norm_case(B, n, kind, gate_rows, B + gate_rows))


@pytest.mark.parametrize("have", [(), ("gate",), ("w_post",), ("w_pre", "b_pre"), ("b_post", "gate")])
@pytest.mark.parametrize("gate_rows", [0, 3, 50])
def test_block_norm_without_parameters(have, gate_rows):
    check_norm(*norm_case(200, 96, "layer", gate_rows, 4, have=have))


def test_block_norm_of_a_large_mean():
    """mean 1000, deviation 1: the mean of the squares less the squared mean would have no digit left"""
    check_norm(*norm_case(50, 300, "layer", 0, 5, offset=1000.0))


def test_block_norm_rows_of_zeros_and_in_place():
    spec, t, p = norm_case(33, 520, "layer", 0, 6)
    t["x"][3], t["f"][3], t["f"][4] = 0.0, 0.0, 2.5
    del p["b_post"], p["b_pre"]
    check_norm(spec, t, p)
    x_out, h = net.kan_block_norm_forward(spec, t["x"], t["f"], p)
    x, f = t["x"].clone(), t["f"].clone()
    net.kan_block_norm_forward(spec, x, f, p, x_out=x, h=f)
    assert torch.equal(x, x_out) and torch.equal(f, h)
    stats = torch.empty((33, 4), device="cuda")
    net.kan_block_norm_forward(spec, t["x"], t["f"], p, stats=stats)
    g = net.kan_block_norm_backward(spec, t["x"], t["f"], p, stats, t["gx_out"], t["gh"])
    gx, gf = t["gx_out"].clone(), t["gh"].clone()
    net.kan_block_norm_backward(spec, t["x"], t["f"], p, stats, gx, gf, out=dict(gx=gx, gf=gf))
    assert torch.equal(gx, g["gx"]) and torch.equal(gf, g["gf"])


def test_block_norm_keeps_what_is_wrong_in_its_row():
    spec, t, p = norm_case(40, 300, "layer", 0, 7)
    x_out, h = net.kan_block_norm_forward(spec, t["x"], t["f"], p)
    t["f"][5, 7], t["x"][9, 299], t["f"][11, 0] = float("nan"), float("inf"), -float("inf")
    x2, h2 = net.kan_block_norm_forward(spec, t["x"], t["f"], p)
    good = [r for r in range(40) if r not in (5, 9, 11)]
    assert torch.equal(x_out[good], x2[good]) and torch.equal(h[good], h2[good])
    assert h2[5].isnan().all() and h2[9].isnan().any() and h2[11].isnan().all()


def test_block_norm_of_no_rows():
    spec, t, p = norm_case(0, 64, "layer", 0, 8)
    x_out, h = net.kan_block_norm_forward(spec, t["x"], t["f"], p)
    assert x_out.shape == (0, 64) and h.shape == (0, 64)
    g = net.kan_block_norm_backward(spec, t["x"], t["f"], p, torch.empty((0, 4), device="cuda"), t["gx_out"], t["gh"])
    assert all(not v.any() for v in g.values()) and g["ggate"].shape == (1, 64)


def test_block_norm_through_autograd():
    spec, t, p = norm_case(90, 130, "layer", 30, 9, BF16, F32)
    leaves = {k: v.clone().requires_grad_(True) for k, v in dict(x=t["x"], f=t["f"], **p).items()}
    x_out, h = autograd.block_norm(spec, **leaves)
    g = torch.autograd.grad([x_out, h], list(leaves.values()), [t["gx_out"], t["gh"]])
    stats = torch.empty((90, 4), device="cuda")
    x2, h2 = net.kan_block_norm_forward(spec, t["x"], t["f"], p, stats=stats)
    ref = net.kan_block_norm_backward(spec, t["x"], t["f"], p, stats, t["gx_out"], t["gh"])
    assert torch.equal(x_out, x2) and torch.equal(h, h2)
    for name, v in zip(leaves, g):
        assert torch.equal(v, ref["g" + name]) and v.dtype == leaves[name].dtype, name
    # three dimensions, one output used, nothing recorded
    x3, f3 = t["x"].view(3, 30, 130), t["f"].view(3, 30, 130).clone().requires_grad_(True)
    x_out, h = autograd.block_norm(spec, x3, f3, **p)
    assert x_out.shape == x3.shape and torch.equal(x_out.view(90, 130), x2)
    gf, = torch.autograd.grad(h.sum(), f3)
    ref = net.kan_block_norm_backward(spec, t["x"], t["f"], p, stats, None, torch.ones_like(t["gh"]), want=["gf"])
    assert torch.equal(gf.view(90, 130), ref["gf"])
    with torch.no_grad():
        a, b = autograd.block_norm(spec, t["x"], t["f"], **p)
        assert torch.equal(a, x2) and torch.equal(b, h2) and not a.requires_grad
        a, b = autograd.block_norm(spec, t["x"], t["f"], **p, want_h=False)
        assert torch.equal(a, x2) and b is None
        a, b = autograd.block_norm(spec, t["x"], w_pre=p["w_pre"])
        assert a is t["x"] and b.dtype == F32


@pytest.mark.parametrize("have", [(), ("gate",), ("w_pre",), ("b_post", "w_pre"), ("w_post", "b_post", "gate")])
@pytest.mark.parametrize("branch", [True, False])
@pytest.mark.parametrize("frozen", [None, "x", "f", "gate"])
def test_block_norm_through_autograd_with_some_of_its_tensors(have, branch, frozen):
    """Missing and frozen tensors: each of the others gets its own gradient."""
    spec, t, p = norm_case(40, 72, "layer", 10, 13, have=have)
    leaves = dict(x=t["x"], **(dict(f=t["f"]) if branch else {}), **p)
    leaves = {k: v.clone().requires_grad_(k != frozen) for k, v in leaves.items()}
    x_out, h = autograd.block_norm(spec, **leaves)
    stats = torch.empty((40, 4), device="cuda")
    f = t["f"] if branch else None
    net.kan_block_norm_forward(spec, t["x"], f, p, stats=stats)
    ref = net.kan_block_norm_backward(spec, t["x"], f, p, stats, t["gx_out"] if branch else None, t["gh"])
    live = [k for k, v in leaves.items() if v.requires_grad and (branch or k in ("x", "w_pre", "b_pre"))]
    outs, gouts = ([x_out, h], [t["gx_out"], t["gh"]]) if branch else ([h], [t["gh"]])
    if not live:
        return
    for k, v in zip(live, torch.autograd.grad(outs, [leaves[k] for k in live], gouts)):
        assert v.shape == leaves[k].shape and torch.equal(v.view(-1), ref["g" + k].view(-1)), k


def test_block_norm_gradient_is_the_difference():
    """Along a random direction: (loss(v + e d) - loss(v - e d)) / 2 e, the loss summed in 64 bits.  32-bit outputs of size 1 are off by some 64 u
    each; over e = 2^-7 and the square root of 7000 of them that is 64 u 84 / 2^-6 = 0.02; the third derivative adds e^2 times the gradient's size."""
    spec, t, p = norm_case(70, 100, "layer", 20, 10)
    leaves = {k: v.clone().requires_grad_(True) for k, v in dict(x=t["x"], f=t["f"], **p).items()}
    x_out, h = autograd.block_norm(spec, **leaves)
    g = torch.autograd.grad([x_out, h], list(leaves.values()), [t["gx_out"], t["gh"]])
    gen, e = torch.Generator(device="cuda").manual_seed(3), 2.0 ** -7
    for (name, v), gv in zip(leaves.items(), g):
        d = torch.randn(v.shape, generator=gen, device="cuda")

        def loss(sign):
            with torch.no_grad():
                a, b = autograd.block_norm(spec, **dict(leaves, **{name: v + sign * e * d}))
            return float((a.double() * t["gx_out"]).sum() + (b.double() * t["gh"]).sum())

        want, size = float((gv.double() * d).sum()), float(gv.double().norm() * d.double().norm())
        assert abs((loss(1) - loss(-1)) / (2 * e) - want) < 0.02 + 1e-3 * size, name


# ---- embedding ------------------------------------------------------------------------------

def embed_case(T, V, n, seed, how="some", table=F32, out=F32):
    rng = np.random.default_rng(seed)
    ids = {"some": lambda: rng.integers(-1, V + 1, T), "one": lambda: np.full(T, V // 2), "few": lambda: np.minimum(rng.geometric(0.3, T) - 1, V - 1),
           "none": lambda: np.full(T, -5), "far": lambda: rng.choice([-2 ** 62, 2 ** 62, 2 ** 32, 0, V - 1], T)}[how]().astype(np.int64)
    return dev(ids, torch.int64), dev(rng.standard_normal((V, n)).astype(np.float32), table), dev(rng.standard_normal((T, n)).astype(np.float32), out)


def check_embed(ids, table, gy, scale=1.5):
    V, n = table.shape
    y = net.kan_embedding_forward(ids, table, scale, dtype=gy.dtype)
    ref = plain.embedding(ids.cpu().numpy(), host(table), np.float32(scale))
    check(y, ref, np.abs(ref), 2, "y")
    g = net.kan_embedding_backward(ids, gy, V, scale, dtype=table.dtype)
    ref, size = plain.embedding_backward(ids.cpu().numpy(), host(gy), V, np.float32(scale))
    check(g, ref, size, 192, "gtable")
    assert torch.equal(g, net.kan_embedding_backward(ids, gy, V, scale, dtype=table.dtype))


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 1000, 1024, 1025, 4095, 4096, 5000])
@pytest.mark.parametrize("V,n", [(1, 3), (2, 8), (255, 24), (256, 7), (1023, 64), (1024, 100), (70000, 9)])
def test_embedding_sizes(T, V, n):
    check_embed(*embed_case(T, V, n, T + V))


@pytest.mark.parametrize("how", ["one", "few", "none", "far"])
@pytest.mark.parametrize("T,V,n", [(70, 5, 33), (3000, 400, 520), (70001, 300, 24), (140000, 1 << 20, 8)])
def test_embedding_frequent_and_missing_tokens(how, T, V, n):
    check_embed(*embed_case(T, V, n, T, how))


@pytest.mark.parametrize("n", [1, 8, 77, 2048, 2056, 5000])
@pytest.mark.parametrize("table,out", [(F32, F32), (BF16, F32), (BF16, BF16)])
def test_embedding_types(n, table, out):
    check_embed(*embed_case(300, 50, n, n, "few", table, out))


def test_embedding_of_no_tokens():
    ids, table, gy = embed_case(0, 10, 16, 1)
    assert net.kan_embedding_forward(ids, table).shape == (0, 16)
    assert not net.kan_embedding_backward(ids, gy, 10, gtable=torch.ones((10, 16), device="cuda")).any()


def test_embedding_sums_in_the_order_of_the_batch():
    """1, 2^-24, -1 in one row's run: the order decides what is left"""
    ids = torch.zeros(3, dtype=torch.int64, device="cuda")
    gy = torch.tensor([[1.0], [2.0 ** -24], [-1.0]], device="cuda")
    assert float(net.kan_embedding_backward(ids, gy, 1)) == 0.0
    assert float(net.kan_embedding_backward(ids, gy[[0, 2, 1]].contiguous(), 1)) == 2.0 ** -24


def test_embedding_past_32_bits():
    """a table of 2^31 + elements, read and written at its end"""
    V, n = (1 << 20) + 3, 2056
    table = torch.zeros((V, n), dtype=BF16, device="cuda")
    table[-1] = 1.0
    ids = torch.tensor([V - 1, 0, V - 1], device="cuda")
    assert (net.kan_embedding_forward(ids, table, 2.0)[[0, 2]] == 2.0).all()
    g = net.kan_embedding_backward(ids, torch.ones((3, n), dtype=BF16, device="cuda"), V, gtable=table)
    assert (g[-1] == 2.0).all() and (g[0] == 1.0).all() and not g[1:-1].any()


def test_embedding_through_autograd():
    ids, table, gy = embed_case(600, 40, 36, 2, "some", BF16, F32)
    table.requires_grad_(True)
    y = autograd.embedding(ids.view(20, 30), table, 0.5, F32)
    assert y.shape == (20, 30, 36) and y.dtype == F32
    g, = torch.autograd.grad(y, table, gy.view(20, 30, 36).transpose(0, 1).contiguous().transpose(0, 1))
    assert torch.equal(g, net.kan_embedding_backward(ids, gy, 40, 0.5, dtype=BF16))
    assert autograd.embedding(ids, table).dtype == BF16


# ---- log probabilities ----------------------------------------------------------------------

def logit_case(R, V, seed, dtype=F32, pad=0, how="normal"):
    rng = np.random.default_rng(seed)
    z = 4.0 * rng.standard_normal((R, V + pad)).astype(np.float32)
    if how == "ties":
        z = np.round(z / 8.0)
    if how == "rising":
        z = np.sort(z, 1)
    if how == "falling":
        z = -np.sort(-z, 1)
    if how == "equal":
        z[:] = 3.0
    if how == "masked":
        z[rng.random(z.shape) < 0.6] = -np.inf
        z[:, V // 2] = 1.0
    if how == "lowest":
        z[rng.random(z.shape) < 0.6] = float(torch.finfo(dtype).min)
        z[:, V // 2] = 1.0
    if how == "large":
        z *= 1e4
    if how == "special":
        z[0] = -np.inf
        z[1] = float(torch.finfo(dtype).min)
        z[2, V // 2] = np.nan
        z[3, V // 3] = np.inf
        z[4] = np.where(np.arange(V + pad) == V - 1, 0.0, -np.inf)
        z[5, :] = np.nan
        z[6, V // 2:] = -np.nan
        z[7] = np.inf
    ids = rng.integers(0, V, R)
    ids[rng.random(R) < 0.2] = -1
    t = dev(z, dtype)
    return t[:, :V], dev(ids, torch.int64), dev(rng.standard_normal(R).astype(np.float32)), dev(rng.standard_normal(R).astype(np.float32))


def check_logprob(z, ids, a, b, temperature=1.0, top=0):
    n_ids = ids.cpu().numpy()
    ref = plain.token_logprob(host(z), n_ids, temperature, top)
    o = net.kan_token_logprob_forward(z, ids, temperature, top)
    check(o["logp"], ref["logp"], 1.0 + np.abs(ref["logp"]), 256, "logp")
    check(o["entropy"], ref["entropy"], 1.0 + np.abs(ref["entropy"]), 256, "entropy")
    if top:
        assert np.array_equal(o["top_ids"].cpu().numpy(), ref["top_ids"])
        check(o["top_logp"], ref["top_logp"], 1.0 + np.abs(ref["top_logp"]), 256, "top_logp")
    for ga, gb in ((a, b), (a, None), (None, b)):
        got = net.kan_token_logprob_backward(z, ids, o, ga, gb, temperature)
        g, scale = plain.token_logprob_backward(ref, n_ids, None if ga is None else host(ga), None if gb is None else host(gb), temperature)
        check(got, g, scale, 256, "glogits")


@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 64, 513, 2048, 4096, 4097, 8200, 16384, 16385, 50001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logprob_vocabularies(V, dtype):
    for top in (0, 1, min(V, 5), min(V, 64)):
        check_logprob(*logit_case(5, V, V, dtype), top=top)


@pytest.mark.parametrize("how", ["ties", "rising", "falling", "equal", "masked", "lowest", "large", "special"])
@pytest.mark.parametrize("V", [30, 700, 5000, 20011])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logprob_values(how, V, dtype):
    check_logprob(*logit_case(9, V, V, dtype, how=how), top=20)


@pytest.mark.parametrize("how", ["normal", "ties", "rising", "falling", "equal", "special"])
@pytest.mark.parametrize("top", [1, 20, 64])
@pytest.mark.parametrize("dtype,V", [(F32, 9001), (BF16, 20011)])
def test_logprob_many_rows(how, top, dtype, V):
    """enough rows that none is cut: several rounds over each, more candidates than there is room for"""
    check_logprob(*logit_case(600, V, V, dtype, how=how), top=top)


@pytest.mark.parametrize("temperature", [0.05, 0.7, 30.0])
def test_logprob_temperature(temperature):
    check_logprob(*logit_case(20, 333, 2), temperature=temperature, top=3)


@pytest.mark.parametrize("R,V,pad", [(1, 140000, 0), (2, 140000, 3), (300, 77, 1), (70000, 9, 7), (3, 300000, 1)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logprob_rows_and_strides(R, V, pad, dtype):
    check_logprob(*logit_case(R, V, R, dtype, pad), top=4)


def test_logprob_past_32_bits():
    """rows that start past 2^31 elements"""
    R, V, stride = 3, 70001, (1 << 30) + 5
    z = torch.zeros(2 * stride + V, dtype=BF16, device="cuda").as_strided((R, V), (stride, 1))
    z[2, 5] = 3.0
    o = net.kan_token_logprob_forward(z, torch.tensor([5, 5, 5], device="cuda"), top=2)
    ref = plain.token_logprob(host(z), np.array([5, 5, 5]), top=2)
    check(o["logp"], ref["logp"], 1 + np.abs(ref["logp"]), 256)
    assert np.array_equal(o["top_ids"].cpu().numpy(), ref["top_ids"])


def test_logprob_in_place_and_parts():
    z, ids, a, b = logit_case(33, 1003, 4)
    o = net.kan_token_logprob_forward(z, ids, top=2)
    g = net.kan_token_logprob_backward(z, ids, o, a, b)
    y = z.clone()
    assert net.kan_token_logprob_backward(y, ids, o, a, b, glogits=y) is y and torch.equal(y, g)
    # fewer outputs, and the same bits
    lib, logp = net.load(), torch.empty(33, device="cuda")
    assert lib.kan_token_logprob_forward(33, 1003, z.data_ptr(), 0, 1003, ids.data_ptr(), 1.0, 0, logp.data_ptr(), None, None, None, None, None, 0,
                                         torch.cuda.current_stream().cuda_stream) == binding.KAN_OK
    entropy = torch.empty(33, device="cuda")
    assert lib.kan_token_logprob_forward(33, 1003, z.data_ptr(), 0, 1003, None, 1.0, 0, None, entropy.data_ptr(), None, None, None, None, 0,
                                         torch.cuda.current_stream().cuda_stream) == binding.KAN_OK
    assert torch.equal(logp, o["logp"]) and torch.equal(entropy, o["entropy"])


def test_logprob_through_autograd():
    z, ids, a, b = logit_case(24, 500, 5, BF16, 12)
    z.requires_grad_(True)
    logp, entropy, top_ids, top_logp = autograd.token_logprob(z, ids, 0.9, 3)
    assert not top_logp.requires_grad
    o = net.kan_token_logprob_forward(z.detach(), ids, 0.9, 3)
    assert torch.equal(logp, o["logp"]) and torch.equal(entropy, o["entropy"]) and torch.equal(top_ids, o["top_ids"])
    g, = torch.autograd.grad([logp, entropy], z, [a, b])
    assert torch.equal(g, net.kan_token_logprob_backward(z.detach(), ids, o, a, b, 0.9))
    logp, entropy, top_ids, _ = autograd.token_logprob(z.view(4, 6, 500), ids.view(4, 6))
    assert logp.shape == (4, 6) and top_ids is None
    g, = torch.autograd.grad(logp.sum(), z)
    assert torch.equal(g, net.kan_token_logprob_backward(z.detach(), ids, net.kan_token_logprob_forward(z.detach(), ids), torch.ones_like(a)))
    with torch.no_grad():
        assert torch.equal(autograd.token_logprob(z, ids, 0.9)[0], o["logp"])


def test_logprob_gradient_is_the_difference():
    """Along a random direction of size one a logit; 24 rows of outputs off by 256 u of some 8 each: 24 8 256 u / 2^-6 = 0.2 at worst."""
    z, ids, a, b = logit_case(24, 50, 6)
    z = z.contiguous().requires_grad_(True)
    logp, entropy, _, _ = autograd.token_logprob(z, ids)
    g, = torch.autograd.grad([logp, entropy], z, [a, b])
    d, e = torch.randn(z.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda"), 2.0 ** -7

    def loss(sign):
        with torch.no_grad():
            lp, h, _, _ = autograd.token_logprob(z + sign * e * d, ids)
        return float((lp.double() * a).sum() + (h.double() * b).sum())

    assert abs((loss(1) - loss(-1)) / (2 * e) - float((g.double() * d).sum())) < 0.2


# ---- clipped gradients ----------------------------------------------------------------------

def clip_lists():
    rng = np.random.default_rng(8)
    t = lambda n, dtype=F32, s=1.0: dev((s * rng.standard_normal(n)).astype(np.float32), dtype)
    return {"one": [t(1)], "small": [t(n) for n in (110, 10, 10, 95, 5, 5)], "edges": [t(n) for n in (8191, 8192, 8193, 1, 7, 8, 9, 0, 16384)],
            "types": [t(1000), t(3001, BF16), t(0), t(50000, BF16), t(12345)], "many": [t(1 + 37 * i % 900) for i in range(300)],
            "large": [t(9000001), t(777)], "empty": [t(0), t(0)], "tiny values": [t(5000, s=1e-25)], "huge values": [t(5000, s=1e25)],
            "views": [t(4000)[1:2001], t(4000, BF16)[3:2000], t(4000)[7:]]}


@pytest.mark.parametrize("name", ["one", "small", "edges", "types", "many", "large", "empty", "tiny values", "huge values", "views"])
@pytest.mark.parametrize("max_norm", [0.0, 1e-2, 1e30])
def test_clip(name, max_norm):
    tensors = clip_lists()[name]
    norm, factor = plain.clip([host(t) for t in tensors], np.float64(np.float32(max_norm)))
    before = [t.clone() for t in tensors]
    out = [torch.full_like(t, 9.0) for t in tensors]
    got = net.kan_clip_gradients(tensors, max_norm, out=out)
    assert abs(float(got) - norm) <= 2 * U * norm and float(net.kan_gradient_norm(tensors)) == float(got)
    assert all(torch.equal(t, o) for t, o in zip(tensors, before))
    for t, o in zip(tensors, out):
        ref = host(t) * factor
        check(o, ref, np.abs(ref), 8)
        if factor == 1.0:
            assert torch.equal(o, t)
    assert torch.equal(net.kan_clip_gradients(tensors, max_norm), got)        # in place
    assert all(torch.equal(t, o) for t, o in zip(tensors, out))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_clip_leaves_gradients_without_a_norm(bad):
    tensors = clip_lists()["types"]
    tensors[1][17] = bad
    before = [t.clone() for t in tensors]
    norm = float(net.kan_clip_gradients(tensors, 1e-3))
    assert not np.isfinite(norm)
    for t, b in zip(tensors, before):
        assert torch.equal(t.nan_to_num(7.0), b.nan_to_num(7.0)) and torch.equal(t.isnan(), b.isnan())


def test_clip_through_autograd_module():
    tensors = clip_lists()["types"]
    tensors.append(dev(np.random.default_rng(1).standard_normal((30, 40)).astype(np.float32)).t())      # dense in another order
    norm, factor = plain.clip([host(t) for t in tensors], 0.5)
    want = [host(t) * factor for t in tensors]
    versions = [t._version for t in tensors]
    got = autograd.clip_gradients(tensors, 0.5)
    assert got.shape == () and abs(float(got) - norm) <= 2 * U * norm
    for t, w, v in zip(tensors, want, versions):
        check(t, w, np.abs(w), 8)
        assert t._version > v
    with pytest.raises(AssertionError):
        autograd.clip_gradients([tensors[0][::2]], 1.0)
    with pytest.raises(AssertionError):
        autograd.clip_gradients(tensors[:2], 1.0, out=tensors[:1])


def test_second_derivatives_are_refused():
    """not silently taken for zero"""
    z, ids, a, b = logit_case(4, 30, 1)
    z = z.clone().requires_grad_(True)
    with pytest.raises(RuntimeError, match="gradients of gradients"):
        torch.autograd.grad(autograd.token_logprob(z, ids)[0].sum(), z, create_graph=True)
    spec, t, p = norm_case(4, 30, "rms", 0, 1)
    x = t["x"].clone().requires_grad_(True)
    with pytest.raises(RuntimeError, match="gradients of gradients"):
        torch.autograd.grad(autograd.block_norm(spec, x, t["f"], **p)[1].sum(), x, create_graph=True)
    ids, table, _ = embed_case(5, 6, 7, 1)
    table.requires_grad_(True)
    with pytest.raises(RuntimeError, match="gradients of gradients"):
        torch.autograd.grad(autograd.embedding(ids, table).sum(), table, create_graph=True)


# ---- streams and graphs ---------------------------------------------------------------------

def test_operators_on_another_stream():
    spec, t, p = norm_case(200, 520, "layer", 0, 11)
    ids, table, gy = embed_case(3000, 100, 64, 3, "few")
    z, tid, a, b = logit_case(50, 3000, 7)
    grads = clip_lists()["types"]

    def everything(stream):
        stats = torch.empty((200, 4), device="cuda")
        x_out, h = net.kan_block_norm_forward(spec, t["x"], t["f"], p, stats=stats, stream=stream)
        out = [x_out, h, *net.kan_block_norm_backward(spec, t["x"], t["f"], p, stats, t["gx_out"], t["gh"], stream=stream).values()]
        out += [net.kan_embedding_forward(ids, table, stream=stream), net.kan_embedding_backward(ids, gy, 100, stream=stream)]
        o = net.kan_token_logprob_forward(z, tid, top=4, stream=stream)
        out += [*o.values(), net.kan_token_logprob_backward(z, tid, o, a, b, stream=stream)]
        clipped = [torch.empty_like(g) for g in grads]
        return out + [net.kan_clip_gradients(grads, 1.0, out=clipped, stream=stream), *clipped]

    want = everything(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = everything(side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_operators_in_a_graph_replay_to_the_eager_results():
    spec, t, p = norm_case(200, 520, "rms", 50, 12)
    ids, table, gy = embed_case(6000, 100, 64, 3, "few")
    z, tid, a, b = logit_case(50, 3000, 7)
    grads = clip_lists()["small"]
    clipped = [torch.empty_like(g) for g in grads]

    def everything():
        stats = torch.empty((200, 4), device="cuda")
        x_out, h = net.kan_block_norm_forward(spec, t["x"], t["f"], p, stats=stats)
        out = [x_out, h, *net.kan_block_norm_backward(spec, t["x"], t["f"], p, stats, t["gx_out"], t["gh"]).values()]
        out += [net.kan_embedding_forward(ids, table), net.kan_embedding_backward(ids, gy, 100)]
        o = net.kan_token_logprob_forward(z, tid, top=4)
        out += [*o.values(), net.kan_token_logprob_backward(z, tid, o, a, b)]
        return out + [net.kan_clip_gradients(grads, 1.0, out=clipped), *clipped]

    everything()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = everything()
    for k in range(4):
        for v in (t["x"], t["gh"], gy, z, *grads):
            v.mul_(-1.25)
        ids.add_(1).remainder_(100)
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in held]
        assert all(torch.equal(x, y) for x, y in zip(got, everything())), k
        torch.cuda.synchronize()
