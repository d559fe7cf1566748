"""Pins of the oracles of the norm and rotation, the block selection and the attention over a map:
torch's own operations, differences of the forward, invariances and hand-worked selections."""
import numpy as np
import pytest
import torch

import oracle
from oracle import rope, selection
from workloads import get_config
from workloads.inputs import _apply_rope, rope_tables


def test_rotation_equals_the_workloads_recipe():
    cfg = get_config("tiny")
    cos, sin = rope_tables(cfg)
    x = np.random.default_rng(0).standard_normal((cfg.n_tokens, 64)).astype(np.float32)
    ref = _apply_rope(x.copy(), cos, sin)
    got = rope.norm_rope(x, rope.angles((4, 16, 16, 0), cfg.rope_split), norm=False)
    np.testing.assert_allclose(got, ref, atol=1e-5)


@pytest.mark.parametrize("halves", [False, True])
def test_scores_depend_on_distances_alone(halves):
    """Turning both sides by positions leaves q.k a function of the differences of positions."""
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 64))
    grid, axes = (3, 4, 5, 0), (24, 20, 20)
    n = 60
    a = rope.angles(grid, axes)
    s = rope.rotate(np.repeat(q, n, 0), a, halves) @ rope.rotate(np.repeat(k, n, 0), a, halves).T
    t, y, x = (c.reshape(-1) for c in np.meshgrid(range(3), range(4), range(5), indexing="ij"))
    seen = {}
    for i in range(n):
        for j in range(n):
            seen.setdefault((t[j] - t[i], y[j] - y[i], x[j] - x[i]), []).append(s[i, j])
    assert all(np.ptp(v) < 1e-12 for v in seen.values())
    b = rope.angles(grid, axes, origin=(7, -3, 100))
    s2 = rope.rotate(np.repeat(q, n, 0), b, halves) @ rope.rotate(np.repeat(k, n, 0), b, halves).T
    np.testing.assert_allclose(s, s2, atol=1e-11)


def test_norm_is_torchs_rms_norm():
    x = np.random.default_rng(2).standard_normal((3, 7, 64))
    w = np.random.default_rng(3).standard_normal(64)
    ref = torch.nn.functional.rms_norm(torch.from_numpy(x), (64,), torch.from_numpy(w), 1e-3).numpy()
    np.testing.assert_allclose(rope.norm_rope(x, np.zeros((7, 32)), w, eps=1e-3), ref, rtol=1e-12)


def test_text_and_spare_channels_are_not_turned():
    a = rope.angles((2, 3, 4, 5), (8, 4, 4), head_dim=64)
    x = np.random.default_rng(4).standard_normal((29, 64))
    y = rope.norm_rope(x, a, norm=False)
    assert np.array_equal(y[24:], x[24:]) and np.array_equal(y[:, 16:], x[:, 16:])
    assert not np.allclose(y[1:24, :16], x[1:24, :16])


@pytest.mark.parametrize("norm,halves", [(True, False), (True, True), (False, False), (False, True)])
def test_norm_rope_gradients_are_differences(norm, halves):
    rng = np.random.default_rng(5)
    a = rope.angles((2, 2, 3, 1), (24, 20, 20), origin=(5, 0, 1))
    x, dy, w = rng.standard_normal((2, 13, 64)), rng.standard_normal((2, 13, 64)), rng.standard_normal(64)
    w = w if norm else None
    loss = lambda x, w: (dy * rope.norm_rope(x, a, w, norm, 1e-2, halves)).sum()
    dx, dw = rope.norm_rope_grad(dy, x, a, w, norm, 1e-2, halves)
    for _ in range(12):
        i = tuple(rng.integers(s) for s in x.shape)
        e = np.zeros_like(x)
        e[i] = 1e-5
        assert abs((loss(x + e, w) - loss(x - e, w)) / 2e-5 - dx[i]) < 1e-7 * (1 + abs(dx[i]))
        if norm:
            e = np.zeros(64)
            e[i[2]] = 1e-5
            assert abs((loss(x, w + e) - loss(x, w - e)) / 2e-5 - dw[i[2]]) < 1e-7 * (1 + abs(dw[i[2]]))


def test_selection_by_hand():
    """Blocks of two tokens with known means: order of the scores, ties, text, keep beyond the blocks."""
    k = np.repeat(np.array([[1.0], [3.0], [3.0], [-2.0], [0.5]]), 2, axis=0)
    k[0], k[1] = 0.0, 2.0                                            # mean 1
    q = np.array([[1.0], [1.0], [-1.0], [-1.0], [0.0]])              # the last block has one token
    m = selection.select_blocks(q, k, 2, 2)
    assert m.tolist() == [[0, 1, 1, 0, 0], [0, 0, 0, 1, 1], [1, 1, 0, 0, 0]]
    assert selection.select_blocks(q, k, 2, 1).tolist() == [[0, 1, 0, 0, 0], [0, 0, 0, 1, 0], [1, 0, 0, 0, 0]]
    assert selection.select_blocks(q, k, 2, 0).sum() == 0 and selection.select_blocks(q, k, 2, 9).all()
    # one token of text: the last block of both is whole; query block 2 keeps everything
    assert selection.select_blocks(q, k, 2, 1, 1, 1).tolist() == [[0, 1, 0, 0, 1], [0, 0, 0, 1, 1], [1, 1, 1, 1, 1]]
    k[2] = np.nan
    assert selection.select_blocks(q, k, 2, 4).tolist() == [[1, 0, 1, 1, 1], [1, 0, 1, 1, 1], [1, 0, 1, 1, 1]]


def test_map_attention_is_the_masked_attention():
    rng = np.random.default_rng(6)
    n, block = 75, 16
    q, k, v = rng.standard_normal((3, n, 8))
    keep = rng.random((5, 5)) < 0.5
    keep[2] = False
    o, lse = selection.map_attention(q, k, v, keep, block, 0.3)
    ro, rl = oracle.masked_attention(q, k, v, keep, block, 0.3)
    np.testing.assert_allclose(o, ro, atol=1e-14)
    np.testing.assert_array_equal(np.isneginf(lse), np.isneginf(rl))
    live = np.isfinite(rl)
    assert np.abs(lse[live] - rl[live]).max() < 1e-13


@pytest.mark.parametrize("n_q,n_k", [(45, 45), (1, 70), (33, 20)])
def test_map_attention_gradients_are_torchs_and_differences(n_q, n_k):
    rng = np.random.default_rng(7)
    block, d = 16, 8
    q, do = rng.standard_normal((2, n_q, d))
    k, v = rng.standard_normal((2, n_k, d))
    keep = rng.random((-(-n_q // block), -(-n_k // block))) < 0.6
    keep[0, 0] = True
    if len(keep) > 1:
        keep[1] = False
    dq, dk, dv = selection.map_attention_grad(do, q, k, v, keep, block, 0.4)
    tq, tk, tv = (torch.from_numpy(x).clone().requires_grad_() for x in (q, k, v))
    mask = torch.from_numpy(keep[np.arange(n_q) // block][:, np.arange(n_k) // block])
    live = mask.any(1)
    s = (0.4 * tq[live] @ tk.T).masked_fill(~mask[live], -torch.inf)
    ((torch.softmax(s, 1) @ tv) * torch.from_numpy(do)[live]).sum().backward()
    for got, ref in ((dq, tq.grad), (dk, tk.grad), (dv, tv.grad)):
        np.testing.assert_allclose(got, ref.numpy(), atol=1e-12)
    loss = lambda q, k, v: (do * selection.map_attention(q, k, v, keep, block, 0.4)[0]).sum()
    for x, g, at in ((q, dq, 0), (k, dk, 1), (v, dv, 2)):
        for _ in range(4):
            i = tuple(rng.integers(m) for m in x.shape)
            args = [[q, k, v], [q, k, v]]
            for sign, a in zip((1, -1), args):
                y = x.copy()
                y[i] += sign * 1e-5
                a[at] = y
            diff = (loss(*args[0]) - loss(*args[1])) / 2e-5
            assert abs(diff - g[i]) < 1e-6 * (1 + abs(g[i]))
