"""GPU block selection against the oracle.  The outputs are whole numbers and have to be equal: means and
scores are in 64 bits on both sides, where the sums of random bf16 values are exact and scores of random
data lie further apart than the rounding of a product; ties are made of small whole numbers, which are exact."""
import numpy as np
import pytest

import paper_2609_37001_amd as psa
from oracle import selection
from workloads.inputs import bf16_round

import gpu_util as gu

pytestmark = pytest.mark.gpu


def dev(x):
    return gu.torch().from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to("cuda:0").bfloat16()


def check(b, h, hk, n_q, n_k, d, block, keep, q_text=0, k_text=0, q=None, k=None, heads=None, seed=0):
    torch = gu.torch()
    print(b, h, hk, n_q, n_k, d, block, keep, q_text, k_text, flush=True)
    rng = np.random.default_rng(seed)
    q = bf16_round(rng.standard_normal((b, h, n_q, d)).astype(np.float32)) if q is None else q
    k = bf16_round(rng.standard_normal((b, hk, n_k, d)).astype(np.float32)) if k is None else k
    m, kept = psa.select_blocks(dev(q), dev(k), block, keep, q_text=q_text, k_text=k_text)
    torch.cuda.synchronize()
    m, kept = m.cpu().numpy(), kept.cpu().numpy()
    assert np.array_equal(kept, m.sum(3))
    for bi in range(b):
        for hi in range(h) if heads is None else heads:
            ref = selection.select_blocks(q[bi, hi], k[bi, hi // (h // hk)], block, keep, q_text, k_text)
            assert np.array_equal(m[bi, hi], ref)
    return m


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("n_q,n_k,keep", [(1, 1, 1), (1, 500, 2), (64, 64, 1), (129, 2000, 3), (2100, 2100, 5),
                                          (1000, 65, 1), (333, 1111, 100), (700, 700, 0)])
def test_sizes(d, block, n_q, n_k, keep):
    check(2, 4, 2, n_q, n_k, d, block, keep)


@pytest.mark.parametrize("q_text,k_text", [(0, 1), (1, 0), (77, 77), (64, 64), (300, 300), (999, 40), (999, 999)])
def test_text(q_text, k_text):
    check(1, 3, 3, 999, 999, 64, 64, 4, q_text, k_text)


@pytest.mark.parametrize("n_k", [624 * 64, 624 * 64 + 1, 1280 * 64 - 5, 1280 * 64 + 1, 1500 * 64 + 30])
def test_long_keys(n_k):
    """Scores in LDS, in the workspace with a lane's words in registers, and read again for every bit."""
    check(1, 2, 1, 17 * 64 + 3, n_k, 64, 64, 97, heads=[1])
    check(1, 1, 1, 40, n_k, 64, 64, 1, k_text=200)


def test_many_rows():
    check(2, 20, 4, 9000, 9000, 128, 128, 17, heads=[0, 7, 19])


@pytest.mark.parametrize("keep", [1, 2, 5, 6, 11, 29, 30])
def test_ties_go_to_the_lowest_index(keep):
    rng = np.random.default_rng(3)
    level = rng.integers(-1, 2, (30, 64))                      # block means from a few whole numbers
    level[rng.integers(0, 30, 12)] = level[0]
    k = np.repeat(level, 64, axis=0)[None, None].astype(np.float32)
    q = np.repeat(rng.integers(-1, 2, (5, 64)), 64, axis=0)[None, None].astype(np.float32)
    q[0, 0, :64] = 0                                           # every score 0, of both signs
    check(1, 1, 1, 320, 30 * 64, 64, 64, keep, q=q, k=k)
    check(1, 1, 1, 320, 30 * 64, 64, 64, keep, q=-q, k=k)


def test_values_that_are_not_finite():
    rng = np.random.default_rng(4)
    q, k = (bf16_round(rng.standard_normal((1, 1, n, 64)).astype(np.float32)) for n in (256, 1000))
    k[0, 0, 70, 3] = np.nan
    k[0, 0, 200, 5] = np.inf
    k[0, 0, 500, 6] = -np.inf
    q[0, 0, 100, 0] = np.inf
    with np.errstate(invalid="ignore"):
        for keep in (1, 3, 14, 15):
            check(1, 1, 1, 256, 1000, 64, 64, keep, q=q, k=k)


def test_small_differences_decide():
    """Scores that 32 bits cannot tell apart."""
    k = np.full((1, 1, 20 * 128, 128), 1.0, np.float32)
    for j in range(20):
        k[0, 0, 128 * j, 0] = 2.0 ** -20 * (1 + (7 * j) % 20)      # of a sum of 2^14
    q = np.full((1, 1, 128, 128), 1.0, np.float32)
    m = check(1, 1, 1, 128, 20 * 128, 128, 128, 6, q=bf16_round(q), k=bf16_round(k))
    assert m.sum() == 6


def test_strided_keys_given_outputs_and_refusals():
    torch = gu.torch()
    q = torch.randn(2, 4, 300, 64, device="cuda:0").bfloat16()
    cache = torch.randn(2, 2, 1000, 64, device="cuda:0").bfloat16()
    k = cache[:, :, :700]
    ref = psa.select_blocks(q, k.contiguous(), 64, 3)
    room = torch.full((2 * 4 * 5 * 11 + 2,), 9, dtype=torch.uint8, device="cuda:0")
    out = room[1:-1].view(2, 4, 5, 11)                          # any byte alignment
    m, kept = psa.select_blocks(q, k, 64, 3, blockmap=out)
    assert m is out and torch.equal(m, ref[0]) and torch.equal(kept, ref[1]) and room[0] == 9 and room[-1] == 9
    one = cache[:1, :1, :700].expand(2, 2, 700, 64)             # the same keys for everybody
    assert torch.equal(psa.select_blocks(q, one, 64, 3)[0], psa.select_blocks(q, one.contiguous(), 64, 3)[0])
    for bad in (dict(k=k[:, :, ::2]), dict(k=k[:1]), dict(k=k[..., :32]), dict(blockmap=m[..., :10]), dict(q=q.transpose(1, 2)),
                dict(workspace=torch.empty(4, device="cpu"))):
        with pytest.raises(ValueError):
            psa.select_blocks(**dict(dict(q=q, k=k, block=64, keep=3), **bad))
    with pytest.raises(TypeError):
        psa.select_blocks(q.float(), k, 64, 3)
    for bad in (dict(keep=-1), dict(q_text=301), dict(k_text=-1), dict(q=q[:, :3].contiguous()),
                dict(workspace=torch.empty(256, dtype=torch.uint8, device="cuda:0"))):
        with pytest.raises(psa.PsaError):
            psa.select_blocks(**dict(dict(q=q, k=k, block=64, keep=3), **bad))


def test_side_stream_and_graph_replays_match_eager():
    torch = gu.torch()
    q, k = (torch.randn(1, h, 3000, 128, device="cuda:0").bfloat16() for h in (8, 2))
    ref = psa.select_blocks(q, k, 64, 9, q_text=30, k_text=30)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = psa.select_blocks(q, k, 64, 9, q_text=30, k_text=30, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = psa.select_blocks(q, k, 64, 9, q_text=30, k_text=30)
    for _ in range(3):
        got[0].fill_(7)
        got[1].zero_()
        psa.select_blocks(k, k, 64, 2)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("blocks_k", [321, 591, 624, 625, 1280, 1281])
def test_long_keys_of_wide_heads(blocks_k, block):
    """Head dim 128 in every form of the scores: 10 words a lane from LDS, 20 from the workspace, read again."""
    n_k = blocks_k * block - 5
    check(1, 2, 1, 17 * block + 3, n_k, 128, block, 97, heads=[1])
    check(1, 1, 1, 40, n_k, 128, block, blocks_k - 20, k_text=200)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("blocks_k", [630, 1290])
def test_more_rows_than_workgroups_with_a_slab(d, blocks_k):
    """Workgroups that take several groups of 16 query blocks one after the other, their scores in the same place."""
    check(1, 700, 1, 90, blocks_k * 64 - 30, d, 64, 41, heads=[0, 1, 349, 511, 512, 520, 699])
    check(2, 15, 3, 300 * 64 - 7, blocks_k * 64, d, 64, 300, q_text=70, k_text=70, heads=[0, 14])
