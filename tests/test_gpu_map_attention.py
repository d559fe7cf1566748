"""GPU parity of the attention over a block map, forward and backward, against the oracle.

Forward: the parity bar of the striped attention (gpu_util); q is not rounded here, so the normaliser of the inputs
as given is off by the weights' rounding alone, LSE_ABS_TOL, and by the fp32 sums of the scores, 2^-20 of the
magnitudes that they add.

Backward tolerances.  Both sides take the same o and lse.  A weight P is off by the fp32 score and the exponential,
2^-17 of it; dP - delta by 2^-17 of the magnitudes it adds.  P and dS are each rounded to bf16 once (2^-8 of the value
at most) before they are summed, and every output once.  So an element of dq is off by at most 2^-8 |dq| plus the
sum of (2^-8 |dS| + 2^-16 P (|do| |v| + |do| |o|)) |scale k| over the keys, dk likewise, dv with the rounding of P;
and 2^-8 of that for a rounding of the sum.  Roundings of unrelated values add as the root of their squares: the
norm of an output's error is at most 2^-8 times the root of |dq|^2 plus the sum of the squared terms (a uniform
rounding has 1 / sqrt(3) of its half step as its root mean square), beside the fp32 part.  Against the gradients
from the exact o and lse, pooled, the forward's bar holds: 1e-2 relative."""
import numpy as np
import pytest

import oracle
import paper_2609_37001_amd as psa
from oracle import selection
from workloads.inputs import bf16_round

import gpu_util as gu

pytestmark = pytest.mark.gpu
INF = 0x7FFFFFFF


def dev(x):
    return gu.torch().from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to("cuda:0").bfloat16()


def blocks(n, block):
    return -(-n // block)


def inputs(seed, b, h, hk, n_q, n_k, d):
    rng = np.random.default_rng(seed)
    return [bf16_round(rng.standard_normal((b, m, n, d)).astype(np.float32))
            for m, n in ((h, n_q), (hk, n_k), (hk, n_k), (h, n_q))]


def random_map(seed, b, h, nq, nk, density):
    """A random map with a whole and an empty row, a whole and an empty column where there is room."""
    rng = np.random.default_rng(seed)
    m = (rng.random((b, h, nq, nk)) < density).astype(np.uint8)
    if nk > 2:
        m[:, :, :, 1] = 0
        m[:, :, :, nk - 1] = 1
    if nq > 2:
        m[:, :, 1] = 1
        m[:, :, nq - 2] = 0
    return m


def bits(x):
    return x.float().cpu().numpy()


def check_forward(q, k, v, m, block, scale, o, lse, heads):
    par = gu.Parity()
    group = q.shape[1] // k.shape[1]
    for bi in range(q.shape[0]):
        for hi in heads:
            qh, kh, vh = q[bi, hi], k[bi, hi // group], v[bi, hi // group]
            ro, rl = selection.map_attention(qh, kh, vh, m[bi, hi], block, scale)
            size = abs(scale) * (np.abs(qh.astype(np.float64)) @ np.abs(kh.astype(np.float64)).T).max(1)
            par.add(o[bi, hi], ro, lse[bi, hi], rl, rl, gu.LSE_ABS_TOL + 2.0 ** -20 * size)
    par.check()


def near(got, ref, worst, fp32, squares, name):
    """got against ref, an array of bounds, its fp32 part and the squares of the rounded terms."""
    err = np.abs(got - ref)
    tol = (1 + 2.0 ** -8) * (worst + 2.0 ** -8 * np.abs(ref)) + 1e-30
    assert (err <= tol).all(), "%s: %.3g of the bound" % (name, (err / tol).max())
    norm = 2.0 ** -8 * np.sqrt((ref ** 2).sum() + squares.sum()) + np.sqrt((fp32 ** 2).sum())
    assert np.sqrt((err ** 2).sum()) <= norm + 1e-30, "%s: %.3g of the norm" % (name, np.sqrt((err ** 2).sum()) / norm)


def check_backward(q, k, v, do, m, block, scale, o, lse, got, heads, pool=True):
    dq, dk, dv = (bits(x).astype(np.float64) for x in got)
    group = q.shape[1] // k.shape[1]
    size, pooled = abs(scale), []              # the bounds are of magnitudes
    f = lambda x: np.asarray(x, dtype=np.float64)
    for bi in range(q.shape[0]):
        for hk in sorted({hi // group for hi in heads}):
            kh, vh = f(k[bi, hk]), f(v[bi, hk])
            total = [np.zeros_like(kh) for _ in range(8)]
            exact = [np.zeros_like(kh) for _ in range(2)]
            for hi in range(hk * group, hk * group + group):
                qh, gh, oh, lh = f(q[bi, hi]), f(do[bi, hi]), f(o[bi, hi]), f(lse[bi, hi])
                plain = selection.map_attention_grad(gh, qh, kh, vh, m[bi, hi], block, scale)
                rq, rk, rv = selection.map_attention_grad(gh, qh, kh, vh, m[bi, hi], block, scale, oh, lh)
                mask = selection._token_mask(m[bi, hi], block, len(qh), len(kh))
                with np.errstate(over="ignore", invalid="ignore"):
                    p = np.where(mask, np.exp(scale * (qh @ kh.T) - lh[:, None]), 0.0)
                ds = p * (gh @ vh.T - (gh * oh).sum(1)[:, None])
                fs = 2.0 ** -16 * p * (np.abs(gh) @ np.abs(vh).T + (np.abs(gh) * np.abs(oh)).sum(1)[:, None])
                es = 2.0 ** -8 * np.abs(ds) + fs
                exact[0] += plain[1]
                exact[1] += plain[2]
                if hi in heads:
                    pooled.append((dq[bi, hi], plain[0]))
                    near(dq[bi, hi], rq, size * (es @ np.abs(kh)), size * (fs @ np.abs(kh)),
                         scale ** 2 * (ds ** 2 @ kh ** 2), "dq")
                parts = (rk, size * (es.T @ np.abs(qh)), size * (fs.T @ np.abs(qh)), scale ** 2 * ((ds ** 2).T @ qh ** 2),
                         rv, (2.0 ** -8 + 2.0 ** -16) * (p.T @ np.abs(gh)), 2.0 ** -16 * (p.T @ np.abs(gh)),
                         (p ** 2).T @ gh ** 2)
                total = [t + x for t, x in zip(total, parts)]
            near(dk[bi, hk], *total[:4], "dk")
            near(dv[bi, hk], *total[4:], "dv")
            pooled += [(dk[bi, hk], exact[0]), (dv[bi, hk], exact[1])]
    num, den = sum(((a - b) ** 2).sum() for a, b in pooled), sum((b ** 2).sum() for _, b in pooled)
    assert not pool or num <= gu.REL_L2_TOL ** 2 * den


def check(b, h, hk, n_q, n_k, block, d, density=0.4, scale=None, heads=None, seed=0, m=None, data=None, pool=True, backward=True):
    torch = gu.torch()
    print(b, h, hk, n_q, n_k, block, d, density, flush=True)
    q, k, v, do = inputs(seed, b, h, hk, n_q, n_k, d) if data is None else data
    m = random_map(seed + 1, b, h, blocks(n_q, block), blocks(n_k, block), density) if m is None else m
    s = d ** -0.5 if scale is None else scale
    dm = torch.from_numpy(m).to("cuda:0")
    t = [dev(x) for x in (q, k, v, do)]
    o, lse = psa.attention_map_fwd(t[0], t[1], t[2], dm, block, scale, return_lse=True)
    torch.cuda.synchronize()
    heads = range(h) if heads is None else heads
    on, ln = bits(o), lse.cpu().numpy()
    check_forward(q, k, v, m, block, s, on, ln, heads)
    if not backward:
        return
    got = psa.attention_map_bwd(t[3], t[0], t[1], t[2], o, lse, dm, block, scale)
    torch.cuda.synchronize()
    check_backward(q, k, v, do, m, block, s, on, ln, got, heads, pool)


SHAPES = [(64, 64), (64, 128), (128, 64), (128, 128)]           # head dim, block


@pytest.mark.parametrize("d,block", SHAPES)
@pytest.mark.parametrize("n_q,n_k", [(1, 1), (1, 64), (1, 700), (3, 129), (33, 1000), (64, 64), (65, 63), (127, 300),
                                     (128, 128), (129, 257), (500, 500), (700, 90), (1030, 1030)])
def test_few_query_blocks(d, block, n_q, n_k):
    """Lists shared out over several workgroups wherever they have two blocks."""
    check(1, 2, 2, n_q, n_k, block, d)


@pytest.mark.parametrize("d,block", SHAPES)
def test_one_workgroup_per_query_block(d, block):
    check(2, 40, 40, 4 * block + 17, 5 * block + 1, block, d, heads=[0, 23, 39])


@pytest.mark.parametrize("d,block", SHAPES)
@pytest.mark.parametrize("h,hk,alike", [(140, 70, 0.0), (140, 140, 0.9), (840, 420, 0.0)])
def test_many_query_blocks(d, block, h, hk, alike):
    """More query and key blocks than run at once, in the order of their lists; neighbouring rows that keep other
    or much the same key blocks, an odd number of rows, long and empty ones."""
    nq, nk = 5, 7
    m = random_map(31, 1, h, nq, nk, 0.5)
    rng = np.random.default_rng(32)
    same = rng.random((1, h, nq, nk)) < alike
    m[:, :, 1::2] = np.where(same[:, :, 1::2], m[:, :, 0:nq - 1:2], m[:, :, 1::2])
    m[:, ::3, 2] = 1
    m[:, 1::7] = 0
    check(1, h, hk, 4 * block + 17, 6 * block + 33, block, d, m=m, heads=[0, 1, 2, h - 1])


@pytest.mark.parametrize("d,block", SHAPES)
@pytest.mark.parametrize("h,hk", [(4, 2), (6, 1), (8, 8)])
def test_shared_key_heads(d, block, h, hk):
    check(2, h, hk, 300, 450, block, d)
    check(1, 33 * h, 33 * hk, 3 * block, 200, block, d, heads=[0, h, 32 * h + 1])


@pytest.mark.parametrize("d,block", SHAPES)
@pytest.mark.parametrize("h,hk,nq,density", [(104, 26, 7, 0.1), (26, 26, 61, 0.2)])
def test_key_blocks_that_every_row_keeps(d, block, h, hk, nq, density):
    """Many key blocks, the first and the last of them on every row's list: dk and dv in pieces."""
    m = random_map(41, 1, h, nq, 20, density)
    m[:, :, :nq - 2, 0] = 1
    check(1, h, hk, nq * block - 5, 20 * block - 31, block, d, m=m, heads=[0, h - 1])


@pytest.mark.parametrize("d,block", SHAPES)
@pytest.mark.parametrize("hk,density", [(8, 0.15), (4, 0.0)])
def test_few_long_lists_of_other_lengths(d, block, hk, density):
    """As many query and key blocks as run at once and fewer: a row and a column kept whole go in pieces."""
    n = (56 if block == 64 else 31) * block
    check(1, 8, hk, n - 9, n - 1, block, d, density=density, heads=[0, 7])


@pytest.mark.parametrize("d,block", SHAPES)
@pytest.mark.parametrize("h,hk,n_k,density", [(8, 4, 6150, 0.05), (16, 8, 6150, 0.05), (4, 4, 8190, 0.1), (8, 1, 7000, 0.0), (8, 8, 6150, 0.95)])
def test_long_rows_among_short_ones(d, block, h, hk, n_k, density):
    """Rows kept whole of many and of few query blocks go in pieces, where these are longer than the others by far."""
    check(1, h, hk, 66 * 64 - 11, n_k, block, d, density=density, heads=[0, h - 1], backward=False)


@pytest.mark.parametrize("d,block", SHAPES)
@pytest.mark.parametrize("density", [0.0, 1.0])
def test_empty_and_full_maps(d, block, density):
    nq, nk = 4, 6
    m = np.full((1, 2, nq, nk), int(density), np.uint8)
    check(1, 2, 1, nq * block - 3, nk * block - 7, block, d, m=m)


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 4.0])
def test_scales(scale):
    """Scores from all equal to so far apart that a row has one key, and of the other sign."""
    check(1, 2, 2, 200, 333, 64, 64, scale=scale)
    check(1, 40, 40, 64 * 16 + 5, 333, 64, 64, scale=scale, heads=[3])
    data = inputs(5, 1, 2, 2, 200, 333, 64)
    torch = gu.torch()
    m = random_map(6, 1, 2, 4, 6, 0.5)
    t = [dev(x) for x in data]
    o, lse = psa.attention_map_fwd(*t[:3], torch.from_numpy(m).to("cuda:0"), 64, scale, return_lse=True)
    got = psa.attention_map_bwd(t[3], *t[:3], o, lse, torch.from_numpy(m).to("cuda:0"), 64, scale)
    assert all(torch.isfinite(x).all() for x in (o,) + got)


def test_whole_ranges_of_scores():
    """Rows whose scores sit far from 0, and one key that takes all the weight.  (A channel of 100 in every key
    multiplies the sum of a row's dS, which is 0 only up to the rounding of the o that the call is given: against the
    exact o, dq is off by that.)"""
    q, k, v, do = inputs(7, 1, 2, 2, 150, 400, 128)
    q, k = q * 0.25, k.copy()
    q[..., 0] = 16.0
    k[:, 0, :, 0] = 100.0
    k[:, 1, :, 0] = -100.0
    k[:, :, 77, 1:] = bf16_round(8 * q[:, :, 5, 1:])
    check(1, 2, 2, 150, 400, 64, 128, density=0.7, data=(bf16_round(q), bf16_round(k), v, do), pool=False)


def test_gradients_are_differences():
    """The oracle's loss changes by the kernel's gradients: a step in a random direction against <gradient, step>.
    The gradients' error is at most 2^-7 of their terms' magnitudes, which the tolerance takes."""
    torch = gu.torch()
    b, h, hk, n_q, n_k, d, block = 1, 2, 1, 130, 200, 64, 64
    q, k, v, do = inputs(11, b, h, hk, n_q, n_k, d)
    m = random_map(12, b, h, 3, 4, 0.6)
    t = [dev(x) for x in (q, k, v, do)]
    dm = torch.from_numpy(m).to("cuda:0")
    o, lse = psa.attention_map_fwd(*t[:3], dm, block, return_lse=True)
    grads = [bits(x).astype(np.float64) for x in psa.attention_map_bwd(t[3], *t[:3], o, lse, dm, block)]
    rng = np.random.default_rng(13)
    f = [np.asarray(x, dtype=np.float64) for x in (q, k, v)]

    def loss(x):
        return sum((do[0, i] * selection.map_attention(x[0][0, i], x[1][0, 0], x[2][0, 0], m[0, i], block, d ** -0.5)[0]).sum()
                   for i in range(h))

    for i in range(3):
        step = rng.standard_normal(f[i].shape)
        at = [[x + (s * 1e-4 * step if j == i else 0) for j, x in enumerate(f)] for s in (1, -1)]
        diff = (loss(at[0]) - loss(at[1])) / 2e-4
        want = (grads[i] * step).sum()
        assert abs(diff - want) <= 2.0 ** -7 * np.sqrt((grads[i] ** 2 * step ** 2).sum()) * 4 + 1e-3 * abs(diff)


def test_stripes_through_a_map_equal_the_striped_attention():
    torch = gu.torch()
    grid, block, heads = (4, 16, 24, 40), 128, 3
    params = [(1, 0, INF, 2, 0, INF), (2, 1, 3, 1, 0, INF), (4, 0, INF, 1, -1, 3)]
    n = 4 * 16 * 24 + 40
    q, k, v, do = inputs(21, 2, heads, heads, n, n, 128)
    t = [dev(x) for x in (q, k, v)]
    ref, rl = psa.attention_fwd(*t, grid, block, params, return_lse=True)
    m, _, _ = psa.build_blockmap(params, grid, block)
    got, gl = psa.attention_map_fwd(*t, m, block, return_lse=True)     # [heads, nb, nb]: every batch element
    again = psa.attention_map_fwd(*t, m[None].expand(2, -1, -1, -1).bool(), block)
    assert torch.equal(again, got)
    assert (got.float() - ref.float()).norm() <= 1e-2 * ref.float().norm()
    fin = torch.isfinite(rl)
    assert torch.equal(fin, torch.isfinite(gl)) and (gl[fin] - rl[fin]).abs().max() <= 2 * gu.LSE_ABS_TOL
    check_forward(q, k, v, np.broadcast_to(m.cpu().numpy(), (2,) + tuple(m.shape)), block, 128 ** -0.5, bits(got),
                  gl.cpu().numpy(), range(heads))


def test_part_of_a_cache_and_given_outputs():
    torch = gu.torch()
    q = torch.randn(2, 4, 70, 128, device="cuda:0").bfloat16()
    kc, vc = (torch.full((2, 2, 900, 128), float("nan"), device="cuda:0").bfloat16() for _ in range(2))
    kc[:, :, :333], vc[:, :, :333] = torch.randn(2, 2, 2, 333, 128, device="cuda:0").bfloat16()
    k, v = kc[:, :, :333], vc[:, :, :333]
    m = torch.from_numpy(random_map(3, 2, 4, 2, 6, 0.5)).to("cuda:0")
    ref, rl = psa.attention_map_fwd(q, k.contiguous(), v.contiguous(), m, 64, return_lse=True)
    room = torch.full((2 * 4 * 70 + 2, 128), 7.0, device="cuda:0").bfloat16()
    out = room[1:-1].view(2, 4, 70, 128)
    o, lse = psa.attention_map_fwd(q, k, v, m, 64, return_lse=True, out=out)
    assert o is out and torch.equal(o, ref) and torch.equal(lse, rl) and (room[0] == 7).all() and (room[-1] == 7).all()
    do = torch.randn_like(q)
    g1 = psa.attention_map_bwd(do, q, k, v, o, lse, m, 64)
    g2 = psa.attention_map_bwd(do, q, k.contiguous(), v.contiguous(), o.clone(), lse, m, 64)
    assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(g1, g2))


@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("n", [300, 2000])
def test_forms_of_a_map(block, n):
    """Any byte but 0 keeps a tile; a map for all batch elements, given once, repeated without a copy, or copied."""
    torch = gu.torch()
    q, k, v, do = (dev(x) for x in inputs(51, 2, 20, 10, n, n, 64))
    m = torch.from_numpy(random_map(52, 1, 20, blocks(n, block), blocks(n, block), 0.3)[0]).to("cuda:0")

    def run(bm):
        o, lse = psa.attention_map_fwd(q, k, v, bm, block, return_lse=True)
        return (o, lse) + psa.attention_map_bwd(do, q, k, v, o, lse, bm, block)

    ref = run(m)
    for other in (m * 255, m * 128, m.bool(), m[None].expand(2, -1, -1, -1), m[None].repeat(2, 1, 1, 1)):
        assert all(torch.equal(x, y) for x, y in zip(ref, run(other)))


def test_offsets_past_32_bits():
    """Key heads more than 2^32 elements apart."""
    torch = gu.torch()
    far = 2 ** 32 + 8 * 1000
    store = torch.empty(far + 200 * 64, dtype=torch.bfloat16, device="cuda:0")
    k = store.as_strided((1, 2, 200, 64), (0, far, 64, 1))
    data = torch.randn(2, 200, 64, device="cuda:0").bfloat16()
    k[0, 0], k[0, 1] = data[0], data[1]
    q, do = (torch.randn(1, 4, 90, 64, device="cuda:0").bfloat16() for _ in range(2))
    m = torch.ones(4, 2, 4, dtype=torch.uint8, device="cuda:0")
    kc = k.contiguous()
    ref, rl = psa.attention_map_fwd(q, kc, kc, m, 64, return_lse=True)
    o, lse = psa.attention_map_fwd(q, k, k, m, 64, return_lse=True)
    assert torch.equal(o, ref) and torch.equal(lse, rl)
    assert all(torch.equal(a, b) for a, b in zip(psa.attention_map_bwd(do, q, k, k, o, lse, m, 64),
                                                 psa.attention_map_bwd(do, q, kc, kc, o, lse, m, 64)))
    assert torch.equal(psa.select_blocks(q, k, 64, 2)[0], psa.select_blocks(q, kc, 64, 2)[0])


def test_longest_maps():
    """7936 blocks on either side, and one more refused."""
    torch = gu.torch()
    n = 7936 * 64
    long, short = torch.randn(1, 1, n, 64, device="cuda:0").bfloat16(), torch.randn(1, 1, 100, 64, device="cuda:0").bfloat16()
    m, kept = psa.select_blocks(short, long, 64, 33)
    assert (kept == 33).all() and (m.sum(3) == 33).all()
    o, lse = psa.attention_map_fwd(short, long, long, m, 64, return_lse=True)
    mn = m[0, 0].cpu().numpy()
    at = np.unique(np.nonzero(mn)[1])
    rows = (at[:, None] * 64 + np.arange(64)).reshape(-1)          # the kept blocks alone are the same attention
    sub = long[0, 0, torch.from_numpy(rows).to("cuda:0")].float().cpu().numpy()
    check_forward(bits(short), sub[None, None], sub[None, None], mn[None, None][..., at], 64, 0.125, bits(o), lse.cpu().numpy(), [0])
    mt = m.transpose(2, 3).contiguous()
    o, lse = psa.attention_map_fwd(long, short, short, mt, 64, return_lse=True)
    g = psa.attention_map_bwd(long, long, short, short, o, lse, mt, 64)
    rest = torch.ones(7936, dtype=torch.bool, device="cuda:0")
    rest[torch.from_numpy(at).to("cuda:0")] = False
    empty = o.view(7936, 64, 64)[rest]
    assert not empty.any() and torch.isneginf(lse.view(7936, 64)[rest]).all() and not g[0].view(7936, 64, 64)[rest].any()
    few = sub[None, None]
    check_backward(few, bits(short), bits(short), few, mt.cpu().numpy()[:, :, at], 64, 0.125,
                   bits(o).reshape(7936, 64, 64)[at].reshape(1, 1, -1, 64), lse.cpu().numpy().reshape(7936, 64)[at].reshape(1, 1, -1),
                   (g[0].view(7936, 64, 64)[torch.from_numpy(at).to("cuda:0")].view(1, 1, -1, 64), g[1], g[2]), [0])
    with pytest.raises(psa.PsaError):
        psa.attention_map_fwd(short, torch.empty(1, 1, n + 1, 64, device="cuda:0", dtype=torch.bfloat16),
                              torch.empty(1, 1, n + 1, 64, device="cuda:0", dtype=torch.bfloat16),
                              torch.zeros(1, 2, 7937, dtype=torch.uint8, device="cuda:0"), 64)


def test_refusals():
    torch = gu.torch()
    q, k = torch.randn(2, 4, 100, 64, device="cuda:0").bfloat16(), torch.randn(2, 2, 150, 64, device="cuda:0").bfloat16()
    m = torch.ones(2, 4, 2, 3, dtype=torch.uint8, device="cuda:0")
    lse = torch.zeros(2, 4, 100, device="cuda:0")
    fwd = lambda **o: psa.attention_map_fwd(**dict(dict(q=q, k=k, v=k, blockmap=m, block=64), **o))
    bwd = lambda **o: psa.attention_map_bwd(**dict(dict(do=q, q=q, k=k, v=k, o=q, lse=lse, blockmap=m, block=64), **o))
    for call in (fwd, bwd):
        for bad in (dict(v=k[:, :, :149]), dict(v=k.float()), dict(blockmap=m[..., :2]), dict(blockmap=m.int()), dict(q=q.cpu()),
                    dict(blockmap=m.transpose(2, 3).contiguous().transpose(2, 3)), dict(k=k[..., ::2], v=k[..., ::2]),
                    dict(k=k[:1], v=k[:1]), dict(block=0), dict(q=q[:, :, ::2])):
            with pytest.raises((ValueError, TypeError)):
                call(**bad)
        for bad in (dict(block=32, blockmap=torch.ones(4, 4, 5, dtype=torch.uint8, device="cuda:0")),
                    dict(k=k[:, :1].repeat(1, 3, 1, 1), v=k[:, :1].repeat(1, 3, 1, 1))):
            with pytest.raises(psa.PsaError):
                call(**bad)
    with pytest.raises(TypeError):
        fwd(out=q.float())
    for bad in (dict(lse=lse[:, :, :99]), dict(lse=lse.half()), dict(dk=q), dict(do=q[:, :2].contiguous())):
        with pytest.raises(ValueError):
            bwd(**bad)
    with pytest.raises(psa.PsaError):
        bwd(workspace=torch.empty(256, dtype=torch.uint8, device="cuda:0"))
    with pytest.raises(psa.PsaError):        # two query blocks share their lists out
        fwd(q=q[:1, :1], k=k[:1, :1].repeat(1, 1, 9, 1), v=k[:1, :1].repeat(1, 1, 9, 1),
            blockmap=torch.ones(1, 2, 22, dtype=torch.uint8, device="cuda:0"),
            workspace=torch.empty(256, dtype=torch.uint8, device="cuda:0"))


@pytest.mark.parametrize("block", [64, 128])
def test_layer_under_a_timestep_policy(block):
    """Dense steps are the dense attention; later steps the attention over the selected blocks; all blocks selected
    are the dense attention up to the rounding of another order of its sums."""
    from paper_2609_37001_amd.policy import SelectedAttention, TimestepPolicy
    torch = gu.torch()
    grid = (3, 10, 14, 33)
    n = 3 * 10 * 14 + 33
    q, k, v = (torch.randn(1, 3, n, 64, device="cuda:0").bfloat16() for _ in range(3))
    layer = SelectedAttention(2, grid, block, TimestepPolicy(5, 0.2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dense, got = layer(q, k, v, 0), [layer(q, k, v, s) for s in (1, 4)] + [layer(q, k, v, 2, stream=side)]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(dense, psa.dense_fwd(q, k, v, block))
    m, _ = psa.select_blocks(q, k, block, 2, q_text=33, k_text=33)
    ref = psa.attention_map_fwd(q, k, v, m, block)
    assert all(torch.equal(x, ref) for x in got) and not torch.equal(ref, dense)
    whole = SelectedAttention(99, grid, block, TimestepPolicy(5, 0.2))(q, k, v, 1)
    assert (whole.float() - dense.float()).norm() <= gu.REL_L2_TOL * dense.float().norm()
    with pytest.raises(ValueError):
        layer(q[:, :, 1:].contiguous(), k, v, 1)


def test_together_on_a_side_stream_and_in_a_graph():
    """A layer as it is used: norm and rotation, selection, attention over the map, and all the gradients back to
    the projections; eager, on another stream, and captured and replayed on new inputs."""
    torch = gu.torch()
    grid, axes, block = (3, 16, 20, 50), (44, 42, 42), 128
    n = 3 * 16 * 20 + 50
    xq, xk, xv = (torch.randn(2, n, h, 128, device="cuda:0").bfloat16().transpose(1, 2) for h in (6, 3, 3))
    wq, wk = (1 + 0.2 * torch.randn(128, device="cuda:0") for _ in range(2))
    do = torch.randn(2, 6, n, 128, device="cuda:0").bfloat16()

    def layer(stream=None):
        q, k = psa.qk_norm_rope(xq, xk, grid, axes, q_weight=wq, k_weight=wk, stream=stream)
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            v = xv.contiguous()
        m, kept = psa.select_blocks(q, k, block, 3, q_text=50, k_text=50, stream=stream)
        o, lse = psa.attention_map_fwd(q, k, v, m, block, return_lse=True, stream=stream)
        dq, dk, dv = psa.attention_map_bwd(do, q, k, v, o, lse, m, block, stream=stream)
        g = psa.qk_norm_rope_bwd(dq, dk, xq, xk, grid, axes, q_weight=wq, k_weight=wk, stream=stream)
        return (q, k, m, kept, o, lse, dq, dk, dv) + g

    ref = layer()
    torch.cuda.synchronize()
    qn, kn, vn = bits(ref[0]), bits(ref[1]), bits(xv)
    mn = ref[2].cpu().numpy()
    for hi in range(6):
        assert np.array_equal(mn[1, hi], selection.select_blocks(qn[1, hi], kn[1, hi // 2], block, 3, 50, 50))
    check_forward(qn, kn, vn, mn, block, 128 ** -0.5, bits(ref[4]), ref[5].cpu().numpy(), [0, 5])
    check_backward(qn, kn, vn, bits(do), mn, block, 128 ** -0.5, bits(ref[4]), ref[5].cpu().numpy(), ref[6:9], [0, 5])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = layer(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = layer()
    for replay in range(3):
        if replay == 2:
            xq.copy_(torch.randn_like(xq))
            do.copy_(torch.randn_like(do))
            ref = layer()
        for t in got:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("d,block,h,hk,n", [(128, 128, 8, 4, 6200), (64, 64, 16, 16, 6200), (128, 64, 4, 2, 8100)])
def test_replays_over_other_maps(d, block, h, hk, n):
    """A captured call orders and cuts the lists of the map that a replay finds: long rows and columns, none, all."""
    torch = gu.torch()
    q, k, v, do = (torch.randn(1, m, n, d, device="cuda:0").bfloat16() for m in (h, hk, hk, h))
    nb = blocks(n, block)
    bm = torch.zeros(1, h, nb, nb, dtype=torch.uint8, device="cuda:0")

    def layer():
        o, lse = psa.attention_map_fwd(q, k, v, bm, block, return_lse=True)
        return (o, lse) + psa.attention_map_bwd(do, q, k, v, o, lse, bm, block)

    layer()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = layer()
    for seed, density in ((61, 0.1), (62, 0.0), (63, 0.5), (64, 1.0), (61, 0.1)):
        m = np.ones((1, h, nb, nb), np.uint8) if density == 1.0 else random_map(seed, 1, h, nb, nb, density)
        bm.copy_(torch.from_numpy(m))
        ref = layer()
        for t in got:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
    check_forward(bits(q), bits(k), bits(v), m, block, d ** -0.5, bits(got[0]), got[1].cpu().numpy(), [h - 1])
    check_backward(bits(q), bits(k), bits(v), bits(do), m, block, d ** -0.5, bits(got[0]), got[1].cpu().numpy(), got[2:], [h - 1])


def test_longest_maps_of_wide_heads():
    """7936 blocks of 128 at head dim 128, where tiles and list take the most LDS: few queries over long keys and the reverse,
    against the attention over the kept blocks alone."""
    torch = gu.torch()
    d = block = 128
    nb = 7936
    long = torch.randn(1, 1, nb * block, d, device="cuda:0").bfloat16()
    short = torch.randn(1, 1, 150, d, device="cuda:0").bfloat16()
    m, kept = psa.select_blocks(short, long, block, 21)
    assert (kept == 21).all() and (m.sum(3) == 21).all()
    mn = m.cpu().numpy()
    at = np.unique(np.nonzero(mn[0, 0])[1])
    kept_rows = torch.from_numpy((at[:, None] * block + np.arange(block)).reshape(-1)).to("cuda:0")
    few = bits(long[:, :, kept_rows])
    cut = mn[..., at]
    do = torch.randn_like(short)
    o, lse = psa.attention_map_fwd(short, long, long, m, block, return_lse=True)
    g = psa.attention_map_bwd(do, short, long, long, o, lse, m, block)
    rest = torch.ones(nb, dtype=torch.bool, device="cuda:0")
    rest[torch.from_numpy(at).to("cuda:0")] = False
    assert not any(x.view(nb, block, d)[rest].any() for x in g[1:])
    check_forward(bits(short), few, few, cut, block, d ** -0.5, bits(o), lse.cpu().numpy(), [0])
    check_backward(bits(short), few, few, bits(do), cut, block, d ** -0.5, bits(o), lse.cpu().numpy(),
                   (g[0], g[1][:, :, kept_rows], g[2][:, :, kept_rows]), [0])
    mt = m.transpose(2, 3).contiguous()
    o, lse = psa.attention_map_fwd(long, short, short, mt, block, return_lse=True)
    g = psa.attention_map_bwd(long, long, short, short, o, lse, mt, block)
    assert not o.view(nb, block, d)[rest].any() and torch.isneginf(lse.view(nb, block)[rest]).all() and not g[0].view(nb, block, d)[rest].any()
    on, ln = bits(o[:, :, kept_rows]), lse[:, :, kept_rows].cpu().numpy()
    check_forward(few, bits(short), bits(short), cut.transpose(0, 1, 3, 2), block, d ** -0.5, on, ln, [0])
    check_backward(few, bits(short), bits(short), few, cut.transpose(0, 1, 3, 2), block, d ** -0.5, on, ln,
                   (g[0][:, :, kept_rows], g[1], g[2]), [0])


@pytest.mark.parametrize("d,block", SHAPES)
@pytest.mark.parametrize("h,hk,nq,nk", [(2, 1, 3, 9), (2, 2, 40, 7), (80, 40, 17, 6), (4, 2, 21, 130)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_not_finite_stay_where_they_are_kept(d, block, h, hk, nq, nk, bad):
    """A key block that the odd query blocks alone keep, one that nobody keeps, a query block that keeps nothing and one that
    keeps the second key block alone: what is not finite there changes no other row's bits."""
    torch = gu.torch()
    print(d, block, h, hk, nq, nk, flush=True)
    m = random_map(71, 1, h, nq, nk, 0.5)
    m[..., 0], m[..., 2], m[:, :, 0], m[..., 3] = 1, 0, 0, 0
    m[:, :, 1::2, 3] = 1
    m[:, :, 2] = 0
    m[:, :, 2, 4] = 1
    n_q, n_k = nq * block - 3, nk * block - 5
    clean = [dev(x) for x in inputs(72, 1, h, hk, n_q, n_k, d)]
    dm = torch.from_numpy(m).to("cuda:0")

    def run(t):
        o, lse = psa.attention_map_fwd(t[0], t[1], t[2], dm, block, return_lse=True)
        return (o, lse) + psa.attention_map_bwd(t[3], t[0], t[1], t[2], o, lse, dm, block)

    ref = run(clean)
    rows = torch.arange(n_q, device="cuda:0") // block
    keys = torch.arange(n_k, device="cuda:0") // block
    t = [x.clone() for x in clean]
    for x in t[1:3]:                                    # keys and values
        x[:, :, keys == 2] = bad
        x[:, :, 3 * block + 7] = bad
    for x in (t[0], t[3]):                              # queries and the gradient: rows that keep nothing
        x[:, :, rows == 0] = bad
    got = run(t)
    even = (rows % 2 == 0) & (rows != 0)
    for i in (0, 1, 2):
        assert torch.equal(got[i][:, :, even], ref[i][:, :, even])
    assert not got[0][:, :, rows == 0].any() and torch.isneginf(got[1][:, :, rows == 0]).all() and not got[2][:, :, rows == 0].any()
    assert not got[3][:, :, keys == 2].any() and not got[4][:, :, keys == 2].any()
    t = [x.clone() for x in clean]
    t[0][:, :, 2 * block + 9] = bad                     # a query that keeps key block 4 alone
    t[3][:, :, 2 * block + 9] = bad
    got = run(t)
    for i in (0, 1, 2):
        assert torch.equal(got[i][:, :, rows != 2], ref[i][:, :, rows != 2])
    for i in (3, 4):
        assert torch.equal(got[i][:, :, keys != 4], ref[i][:, :, keys != 4])


@pytest.mark.parametrize("d,block", SHAPES)
def test_many_short_sequences(d, block):
    """Far more query and key blocks than any other test has, in one list of each kernel's order: 256,000 of one block each."""
    torch = gu.torch()
    b, h, hk, n_q, n_k = 16000, 16, 8, 3, 2 * block + 5
    rng = np.random.default_rng(81)
    t = [torch.randn(b, m, n, d, device="cuda:0", dtype=torch.bfloat16) for m, n in ((h, n_q), (hk, n_k), (hk, n_k), (h, n_q))]
    m = torch.from_numpy((rng.random((b, h, 1, 3)) < 0.6).astype(np.uint8)).to("cuda:0")
    o, lse = psa.attention_map_fwd(*t[:3], m, block, return_lse=True)
    got = psa.attention_map_bwd(t[3], *t[:3], o, lse, m, block)
    sel, kept = psa.select_blocks(t[0], t[1], block, 2)
    assert (kept == 2).all() and (sel.sum(3) == 2).all()
    some = [0, 1, 4097, 8191, 12345, b - 2, b - 1]
    q, k, v, do = (bits(x[some]) for x in t)
    mn, on, ln = m[some].cpu().numpy(), bits(o[some]), lse[some].cpu().numpy()
    check_forward(q, k, v, mn, block, d ** -0.5, on, ln, range(h))
    check_backward(q, k, v, do, mn, block, d ** -0.5, on, ln, [x[some] for x in got], range(h))
    for i, bi in enumerate(some):
        for hi in range(h):
            assert np.array_equal(sel[bi, hi].cpu().numpy(), selection.select_blocks(q[i, hi], k[i, hi // 2], block, 2))
