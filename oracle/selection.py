"""Oracle: block selection by mean scores, and attention over any block map with its gradients (test
infrastructure only), float64, one (batch, head) at a time.

Selection: s_ij = <mean of the queries of block i, mean of the keys of block j>.  A row keeps the `keep`
highest-scoring key blocks without text (of equal scores the lowest index, NaN below everything) and every
key block that holds text; a query block that holds text keeps every key block.

Attention of L = sum(do * o) with o = softmax(scale q k^T over the kept blocks) v:

    P = exp(scale q k^T - lse),  dP = do v^T,  dS = P * (dP - rowsum(do * o))
    dq = scale dS k,  dk = scale dS^T q,  dv = P^T do
"""
import numpy as np


def block_means(x, block):
    x = np.asarray(x, dtype=np.float64)
    return np.stack([x[i:i + block].mean(0) for i in range(0, x.shape[0], block)])


def select_blocks(q, k, block, keep, q_text=0, k_text=0):
    """uint8 map [query blocks, key blocks] of one head."""
    score = block_means(q, block) @ block_means(k, block).T
    nq, nk = score.shape
    out = np.zeros((nq, nk), np.uint8)
    first = (k.shape[0] - k_text) // block if k_text else nk
    for i in range(nq):
        s = np.where(np.isnan(score[i, :first]), -np.inf, score[i, :first])
        out[i, sorted(range(first), key=lambda j: (-s[j], j))[:keep]] = 1
    out[:, first:] = 1
    if q_text:
        out[(q.shape[0] - q_text) // block:] = 1
    return out


def _token_mask(keep, block, n_q, n_k):
    keep = np.asarray(keep).astype(bool)
    return keep[np.arange(n_q) // block][:, np.arange(n_k) // block]


def map_attention(q, k, v, keep, block, scale):
    """(o [n_q, d], lse [n_q]) of queries [n_q, d] over keys [n_k, d]; rows that keep nothing give 0, -inf."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    s = np.where(_token_mask(keep, block, len(q), len(k)), scale * (q @ k.T), -np.inf)
    m = s.max(1)
    live = np.isfinite(m)
    p = np.exp(s - np.where(live, m, 0.0)[:, None])
    l = p.sum(1)
    lse = np.full(len(q), -np.inf)
    lse[live] = m[live] + np.log(l[live])
    return (p @ v) / np.where(live, l, 1.0)[:, None], lse


def map_attention_grad(do, q, k, v, keep, block, scale, o=None, lse=None):
    """(dq, dk, dv) of one head, from the o and lse given or the exact ones."""
    do, q, k, v = (np.asarray(x, dtype=np.float64) for x in (do, q, k, v))
    eo, el = map_attention(q, k, v, keep, block, scale)
    o, lse = eo if o is None else np.asarray(o, dtype=np.float64), el if lse is None else np.asarray(lse, dtype=np.float64)
    mask = _token_mask(keep, block, len(q), len(k))
    with np.errstate(over="ignore", invalid="ignore"):
        p = np.where(mask, np.exp(scale * (q @ k.T) - lse[:, None]), 0.0)
    ds = p * (do @ v.T - (do * o).sum(1)[:, None])
    return scale * (ds @ k), scale * (ds.T @ q), p.T @ do
