"""GPU parity of the norms and rotations of queries and keys, and of their gradients, against the oracle.

Tolerances.  A bf16 output is rounded once: half a step, 2^-8 of the value.  Before that everything is fp32:
a value of a row is a sum of two products of normalised values (at most max|n| each), every one behind
fewer than eight roundings of 2^-24, and sines of angles that are right to 2^-22; 2^-18 max|n| covers them.
A gradient's row has the scale r (max|g w| + max|x r| mean|g w x r|) in place of max|n|, its mean adds
128 products in at most 12 sequential additions: 2^-18 of that scale again.  The weights' gradients add
at most 200 rows in a lane and 32 lanes in fp32, behind fewer than 24 roundings per term: 2^-16 of the
sum of the terms' magnitudes."""
import numpy as np
import pytest

import paper_2609_37001_amd as psa
from oracle import rope
from workloads.inputs import bf16_round

import gpu_util as gu

pytestmark = pytest.mark.gpu
AXES = {64: (24, 20, 20), 128: (44, 42, 42)}


def make(rng, b, h, n, d, dtype, layout):
    """(device rows [b, h, n, d] in the layout, the same as float64)."""
    torch = gu.torch()
    x = rng.standard_normal((b, h, n, d)).astype(np.float32) * (0.1 + np.abs(rng.standard_normal(d))).astype(np.float32)
    if dtype == "bf16":
        x = bf16_round(x)
    t = torch.from_numpy(x).to("cuda:0", torch.bfloat16 if dtype == "bf16" else torch.float32)
    if layout == "bnhd":
        t = t.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "fused":                                     # every third group of heads of a wider row
        wide = torch.full((b, n, 3, h, d), float("nan"), dtype=t.dtype, device=t.device)
        wide[:, :, 1] = t.transpose(1, 2)
        t = wide[:, :, 1].transpose(1, 2)
    if layout == "cache":                                     # the first n tokens of longer rows
        wide = torch.full((b, h, n + 3, d), float("nan"), dtype=t.dtype, device=t.device)
        wide[:, :, :n] = t
        t = wide[:, :, :n]
    return t, x.astype(np.float64)


def near(got, ref, scale, half):
    got, ref = got.double().cpu().numpy(), np.asarray(ref)
    tol = half * np.abs(ref) + 2.0 ** -18 * scale
    worst = float((np.abs(got - ref) / np.maximum(tol, 1e-300)).max())
    assert worst <= 1.0, "%.3g of the tolerance" % worst


def check(b, hq, hk, grid, d, dtype="bf16", layout="bnhd", norm=True, weight=True, pairing="adjacent", axes=None,
          origin=(0, 0, 0), eps=1e-6, theta=10000.0, seed=0):
    torch = gu.torch()
    f, h, w, text = grid
    n = f * h * w + text
    axes = axes or AXES[d]
    print("%d x %d/%d x %s x %d %s %s norm=%s %s" % (b, hq, hk, grid, d, dtype, layout, norm, pairing), flush=True)
    rng = np.random.default_rng(seed)
    x = [make(rng, b, m, n, d, dtype, layout) for m in (hq, hk)]
    wn = [(1 + 0.3 * rng.standard_normal(d)).astype(np.float32) if norm and weight else None for _ in range(2)]
    wt = [None if v is None else torch.from_numpy(v).to("cuda:0") for v in wn]
    opts = dict(q_weight=wt[0], k_weight=wt[1], norm=norm, eps=eps, theta=theta, origin=origin, pairing=pairing)
    out = psa.qk_norm_rope(x[0][0], x[1][0], grid, axes, **opts)
    dyn = [bf16_round(rng.standard_normal((b, m, n, d)).astype(np.float32)) for m in (hq, hk)]
    dy = [torch.from_numpy(v).to("cuda:0").bfloat16() for v in dyn]
    grads = psa.qk_norm_rope_bwd(dy[0], dy[1], x[0][0], x[1][0], grid, axes, **opts)
    torch.cuda.synchronize()
    ang = rope.angles(grid, axes, theta, origin, d)
    halves = pairing == "halves"
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    for i in range(2):
        xn = x[i][1]
        ref = rope.norm_rope(xn, ang, wn[i], norm, eps, halves)
        assert out[i].dtype == torch.bfloat16 and out[i].is_contiguous() and out[i].shape == x[i][0].shape
        near(out[i], ref, np.abs(ref).max(-1, keepdims=True) * 2 ** 0.5, 2.0 ** -8)
        dx, dw = rope.norm_rope_grad(dyn[i], xn, ang, wn[i], norm, eps, halves)
        gw = np.abs(rope.rotate(dyn[i].astype(np.float64), -ang, halves)) * (1 if wn[i] is None else np.abs(wn[i]))
        scale = gw.max(-1, keepdims=True)
        if norm:
            r = 1 / np.sqrt((xn * xn).mean(-1, keepdims=True) + eps)
            u = np.abs(xn * r)
            scale = r * (scale + u.max(-1, keepdims=True) * (gw * u).mean(-1, keepdims=True))
        else:
            scale = np.abs(dyn[i]).max(-1, keepdims=True) * 2
        assert grads[i].dtype == x[i][0].dtype and grads[i].shape == x[i][0].shape
        near(grads[i], dx, scale, half)
        if not norm:
            assert grads[2 + i] is None
            continue
        g = rope.rotate(dyn[i].astype(np.float64), -ang, halves)
        terms = np.abs(g * xn * r).reshape(-1, d).sum(0)
        got = grads[2 + i].double().cpu().numpy()
        assert (np.abs(got - dw) <= 2.0 ** -16 * terms + 2.0 ** -24 * np.abs(dw)).all()
    return x, dy, opts, out, grads


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["bnhd", "bhnd", "fused", "cache"])
@pytest.mark.parametrize("d,pairing,norm", [(64, "adjacent", True), (128, "adjacent", False), (64, "halves", False),
                                            (128, "halves", True), (128, "adjacent", True), (64, "halves", True)])
def test_forms(dtype, layout, d, pairing, norm):
    check(2, 5, 3, (2, 3, 7, 5), d, dtype, layout, norm, pairing=pairing, origin=(3, 0, 11))


@pytest.mark.parametrize("grid", [(1, 1, 1, 0), (1, 1, 1, 1), (2, 1, 1, 0), (1, 1, 3, 0), (1, 3, 5, 0), (1, 1, 16, 0),
                                  (1, 1, 17, 0), (3, 5, 2, 1), (1, 3, 11, 0), (7, 9, 5, 77), (1, 1, 1, 300)])
@pytest.mark.parametrize("heads,d", [((1, 1), 64), ((32, 8), 128), ((3, 40), 64), ((17, 1), 128)])
def test_sizes(grid, heads, d):
    check(1, *heads, grid, d)


def test_many_rows_per_workgroup():
    check(3, 12, 4, (9, 30, 25, 226), 128, weight=False)
    check(1, 2, 2, (5, 40, 61, 0), 64, dtype="fp32", layout="fused", pairing="halves")


@pytest.mark.parametrize("axes,pairing", [((0, 0, 0), "adjacent"), ((2, 0, 60), "adjacent"), ((0, 64, 0), "halves"),
                                          ((10, 6, 8), "adjacent"), ((62, 0, 2), "halves")])
def test_axes(axes, pairing):
    check(1, 2, 1, (3, 4, 5, 2), 64, axes=axes, pairing=pairing)


@pytest.mark.parametrize("origin", [(1 << 20, 0, 0), (2147483000, 5, 7), (-5, -100000, 1)])
def test_far_positions(origin):
    """Angles are formed in 64 bits, so far positions turn as exactly as near ones (a position of 2^31 has an
    error of 2^-22 turns or less in 64 bits)."""
    check(1, 2, 2, (2, 3, 4, 1), 128, dtype="fp32", origin=origin)


@pytest.mark.parametrize("theta,eps", [(1e6, 1e-5), (1.0, 0.0), (0.5, 1e3)])
def test_theta_and_eps(theta, eps):
    check(1, 3, 2, (2, 3, 4, 1), 64, theta=theta, eps=eps)


def test_zero_rows_stay_zero():
    torch = gu.torch()
    q = torch.zeros(1, 2, 6, 64, device="cuda:0", dtype=torch.bfloat16)
    dy = torch.ones_like(q)
    y, none = psa.qk_norm_rope(q, None, (1, 2, 3), AXES[64])
    dq, dk, dw, dkw = psa.qk_norm_rope_bwd(dy, None, q, None, (1, 2, 3), AXES[64], eps=1e-6)
    assert none is None and dk is None and dkw is None
    assert torch.equal(y, q) and torch.isfinite(dq).all() and not dw.any()


def test_repeated_rows_and_given_outputs():
    """A tensor expanded over its heads is read as it is, its gradient has a row for each head; outputs are
    written where the caller says and nowhere else."""
    torch = gu.torch()
    grid, d = (2, 3, 4, 1), 128
    one = torch.randn(1, 1, 25, d, device="cuda:0")
    k = one.expand(2, 3, 25, d)
    q = torch.randn(2, 4, 25, d, device="cuda:0")
    y, yk = psa.qk_norm_rope(q, k, grid, AXES[d])
    assert torch.equal(yk, psa.qk_norm_rope(q, k.contiguous(), grid, AXES[d])[1])
    wide = torch.full((2, 25, 3, 4, d), 7.0, device="cuda:0")
    room = torch.full((2 * 4 * 25 + 2, d), 7.0, device="cuda:0", dtype=torch.bfloat16)
    out = room[1:-1].view(2, 4, 25, d)
    assert psa.qk_norm_rope(q, k, grid, AXES[d], q_out=out)[0] is out and torch.equal(out, y)
    assert (room[0] == 7).all() and (room[-1] == 7).all()
    ref = psa.qk_norm_rope_bwd(y, yk, q, k, grid, AXES[d])
    got = psa.qk_norm_rope_bwd(y, yk, q, k, grid, AXES[d], dq=wide[:, :, 1].transpose(1, 2))
    assert torch.equal(got[0], ref[0]) and all(torch.equal(a, b) for a, b in zip(got[1:], ref[1:]))
    assert (wide[:, :, 0] == 7).all() and (wide[:, :, 2] == 7).all()


def test_refusals():
    torch = gu.torch()
    grid, d = (2, 3, 4, 1), 64
    q = torch.randn(1, 2, 25, d, device="cuda:0").bfloat16()
    call = lambda q=q, k=q, grid=grid, axes=AXES[d], **o: psa.qk_norm_rope(q, k, grid, axes, **o)
    with pytest.raises(TypeError):
        call(q=q.half(), k=None)
    with pytest.raises(TypeError):
        call(k=q.float())
    for bad in (dict(grid=(2, 3, 4, 2)), dict(k=q[:, :, :24]), dict(k=q.repeat(2, 1, 1, 1)), dict(pairing="other"),
                dict(q=q.transpose(2, 3)), dict(q=q.cpu()), dict(q_weight=torch.ones(d, device="cuda:0").bfloat16()),
                dict(q_weight=torch.ones(2 * d, device="cuda:0")), dict(q_out=torch.empty(1, 2, 25, d, device="cuda:0")),
                dict(q_out=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(axes=(24, 20))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(axes=(25, 19, 20)), dict(axes=(44, 42, 42)), dict(axes=(20, 20, 20), pairing="halves"), dict(theta=0.0),
                dict(eps=-1.0), dict(norm=False, q_weight=torch.ones(d, device="cuda:0")), dict(origin=(2 ** 31 - 1, 0, 0)),
                dict(q=torch.zeros(1, 2, 25, d + 4, device="cuda:0").bfloat16()[..., 4:], k=None)):
        with pytest.raises(psa.PsaError):
            call(**bad)
    with pytest.raises(psa.PsaError):        # rows that share memory cannot receive gradients
        psa.qk_norm_rope_bwd(q, q, q, q, grid, AXES[d], dq=q[:, :1].expand(1, 2, 25, d))
    with pytest.raises(psa.PsaError):
        psa.qk_norm_rope_bwd(q, q, q, q, grid, AXES[d], workspace=torch.empty(256, dtype=torch.uint8, device="cuda:0"))


def test_side_stream_and_graph_replays_match_eager():
    torch = gu.torch()
    x, dy, opts, out, grads = check(2, 6, 3, (3, 5, 7, 4), 128, seed=9)
    grid, axes = (3, 5, 7, 4), AXES[128]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = psa.qk_norm_rope(x[0][0], x[1][0], grid, axes, stream=side, **opts)
    gg = psa.qk_norm_rope_bwd(dy[0], dy[1], x[0][0], x[1][0], grid, axes, stream=side, **opts)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got + gg, out + grads))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = psa.qk_norm_rope(x[0][0], x[1][0], grid, axes, **opts)
        gg = psa.qk_norm_rope_bwd(dy[0], dy[1], x[0][0], x[1][0], grid, axes, **opts)
    for _ in range(3):
        for t in got + gg:
            t.zero_()
        psa.qk_norm_rope(x[1][0], x[0][0], grid, axes)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got + gg, out + grads))


def test_queries_alone_in_a_large_batch():
    """More batch elements than queries and keys together may have, in a workspace of exactly the size asked for."""
    torch = gu.torch()
    from paper_2609_37001_amd import _lib
    b, grid, d = 40000, (1, 1, 3, 0), 64
    q = torch.randn(b, 1, 3, d, device="cuda:0").bfloat16()
    dy = torch.randn_like(q)
    w = 1 + 0.2 * torch.randn(d, device="cuda:0")
    need = _lib.lib().psa_qk_norm_rope_workspace_size(b, 1, 0, d, _lib.grid_of(*grid), 1)
    room = torch.full((need + 4096,), 7, dtype=torch.uint8, device="cuda:0")
    y = psa.qk_norm_rope(q, None, grid, AXES[d], q_weight=w)[0]
    dq, _, dw, _ = psa.qk_norm_rope_bwd(dy, None, q, None, grid, AXES[d], q_weight=w, workspace=room[:need])
    own = psa.qk_norm_rope_bwd(dy, None, q, None, grid, AXES[d], q_weight=w)
    torch.cuda.synchronize()
    assert (room[need:] == 7).all() and torch.equal(own[0], dq) and torch.equal(own[2], dw)
    xn, dyn, wn = (t.double().cpu().numpy() for t in (q, dy, w))
    ang = rope.angles(grid, AXES[d], head_dim=d)
    ref = rope.norm_rope(xn, ang, wn)
    near(y, ref, np.abs(ref).max(-1, keepdims=True) * 2 ** 0.5, 2.0 ** -8)
    dx, dref = rope.norm_rope_grad(dyn, xn, ang, wn)
    r = 1 / np.sqrt((xn * xn).mean(-1, keepdims=True) + 1e-6)
    g, u = rope.rotate(dyn, -ang), np.abs(xn * r)
    gw = np.abs(g * wn)
    near(dq, dx, r * (gw.max(-1, keepdims=True) + u.max(-1, keepdims=True) * (gw * u).mean(-1, keepdims=True)), 2.0 ** -8)
    terms = np.abs(g * xn * r).reshape(-1, d).sum(0)
    assert (np.abs(dw.double().cpu().numpy() - dref) <= 2.0 ** -16 * terms + 2.0 ** -24 * np.abs(dref)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
@pytest.mark.parametrize("d", [64, 128])
def test_every_kernel(d, pairing, norm, dtype):
    """Every kernel of both directions (without a norm the backward holds twice the rows in flight and reads no x),
    on a part of a tile, and on more tiles than workgroups take at once, with fewer key heads, text and a later chunk's
    positions."""
    check(2, 3, 1, (1, 3, 7, 2), d, dtype, "fused", norm, pairing=pairing, origin=(0, -2, 3), seed=1)
    check(8, 2, 1, (3, 27, 51, 77), d, dtype, "bnhd", norm, pairing=pairing, origin=(21, 0, 0), seed=2)


def test_a_later_chunk_in_32_bits():
    """Two prompts, an odd grid, seven key heads for 28, channels paired across the halves, no norm."""
    check(2, 28, 7, (5, 23, 37, 77), 128, "fp32", norm=False, pairing="halves", origin=(21, 0, 0), seed=3)
