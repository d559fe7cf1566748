"""The operators around the attention of a layer, as cases for timing and comparing them.

A case is a dict of plain values.  Its "kind" names the operator:

* ``norm_rope``       qk_norm_rope: queries and keys from the projection to the attention's layout, each head
                      normalised (or not: the rotation alone) and rotated by its (t, h, w) position;
* ``norm_rope_grad``  qk_norm_rope_bwd: the gradients of the same, with those of the norms' weights;
* ``select``          select_blocks: for each query block the key blocks of the highest mean score;
* ``attention``       attention_map_fwd: attention over the kept blocks of a map;
* ``attention_grad``  attention_map_bwd: its gradients.

With ``own`` false, run() computes them in elementary torch operations in 32 bits (64 for the angles and
for the selection's scores); with ``own`` true it makes the library's calls.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
AXES = {64: (24, 20, 20), 128: (44, 42, 42)}          # channels of the time, height and width axes
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------
# Cases.
# ------------------------------------------------------------------------------------------------

def _rope(name, kind, batch, heads, kv_heads, grid, dim, dtype, **more):
    c = {"kind": kind, "batch": batch, "heads": heads, "kv_heads": kv_heads, "frames": grid[0], "height": grid[1],
         "width": grid[2], "text": grid[3], "dim": dim, "dtype": dtype, "norm": True, "pairing": "adjacent",
         "frame0": 0, "fused": False}
    return _named(name, dict(c, **more))


def _attn(name, kind, batch, heads, kv_heads, n_q, n_k, text, dim, block, keep):
    return _named(name, {"kind": kind, "batch": batch, "heads": heads, "kv_heads": kv_heads, "n_q": n_q, "n_k": n_k,
                         "text": text, "dim": dim, "block": block, "keep": keep})


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # The smallest call: a 16x16 latent of four frames with two heads; latency is all there is.
        _rope("tiny norm rope d64", "norm_rope", 1, 2, 2, (4, 16, 16, 0), 64, "bf16"),
        # HunyuanVideo, 720p, with text: q and k are slices of one fused projection.
        _rope("hunyuan norm rope", "norm_rope", 1, 24, 24, (33, 45, 80, 256), 128, "bf16", fused=True),
        # The rotation alone in the Wan 2.1 14B layer at 720p.
        _rope("wan14b rope", "norm_rope", 1, 40, 40, (21, 45, 80, 0), 128, "bf16", norm=False),
        # The rotation alone of a later chunk of a clip made chunk by chunk: two prompts, an odd grid, fewer key
        # heads, 32-bit projections, channels paired across the halves of a head.
        _rope("chunk rope fp32 halves", "norm_rope", 2, 28, 7, (5, 23, 37, 77), 128, "fp32", norm=False,
              pairing="halves", frame0=21),
        # The gradients in a Wan 2.1 1.3B layer at 480p.
        _rope("wan1.3b norm rope grad", "norm_rope_grad", 1, 12, 12, (21, 30, 52, 0), 128, "bf16"),
        # Block selection in the Wan 2.1 14B layer, at the density that its stripes have in the mean.
        _attn("wan14b select b128", "select", 1, 40, 40, 75600, 75600, 0, 128, 128, 141),
        # A small-model clip with text and a ragged end, two prompts, narrow heads, fine blocks.
        _attn("clip select b64 d64 text", "select", 2, 16, 16, 17776, 17776, 226, 64, 64, 56),
        # One GPU's heads of the Wan 2.1 14B layer where eight share them.
        _attn("wan14b share attention b128", "attention", 1, 5, 5, 75600, 75600, 0, 128, 128, 141),
        # The clip again: text rows keep every block.
        _attn("clip attention b64 d64 text", "attention", 2, 16, 16, 17776, 17776, 226, 64, 64, 56),
        # One new token of four sequences over a long cache with shared key heads.
        _attn("one token attention b64", "attention", 4, 32, 8, 1, 90001, 0, 128, 64, 64),
        # Gradients in the Wan 2.1 1.3B layer at a quarter of the blocks.
        _attn("wan1.3b attention grad b128", "attention_grad", 1, 12, 12, 32760, 32760, 0, 128, 128, 64),
        # Gradients of a short clip with text, narrow heads, fine blocks and shared key heads.
        _attn("preview attention grad b64", "attention_grad", 2, 8, 4, 7877, 7877, 77, 64, 64, 31),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of any kind, its sizes spread over the range of the listed ones."""
    kind = rng.choice(["norm_rope", "norm_rope", "norm_rope_grad", "select", "attention", "attention", "attention_grad"])
    dim = rng.choice([64, 128])
    batch, kv_heads, group = rng.choice([1, 1, 2, 4]), _log(rng, 1, 20), rng.choice([1, 1, 1, 2, 4])
    text = rng.choice([0, 0, 77, 226, 256])
    if kind in ("norm_rope", "norm_rope_grad"):
        grid = (rng.randint(1, 33), _log(rng, 1, 48), _log(rng, 1, 80), text)
        return _rope(None, kind, batch, kv_heads * group, kv_heads, grid, dim, rng.choice(["bf16", "bf16", "fp32"]),
                     norm=rng.random() < 0.7, pairing=rng.choice(["adjacent", "adjacent", "halves"]),
                     frame0=rng.choice([0, rng.randint(0, 2000)]), fused=rng.random() < 0.4)
    block = rng.choice([64, 128])
    if kind == "attention" and rng.random() < 0.4:                 # a few new rows over a long cache
        n_q, n_k, text = _log(rng, 1, 300), _log(rng, 1000, 100000), 0
        keep = min(-(-n_k // block), _log(rng, 4, 128))
    else:
        most = {"select": 75600, "attention": 40000, "attention_grad": 20000}[kind]
        n_k = n_q = max(text, 0) + _log(rng, 300, most)
        nb = -(-n_k // block)
        keep = max(1, int(nb * rng.uniform(0.05, 0.6)))
    c = _attn(None, kind, batch, kv_heads * group, kv_heads, n_q, n_k, text, dim, block, keep)
    budget = {"select": 6e10, "attention": 6e12, "attention_grad": 6e12}[kind]
    while _cost(c) > budget and c["kv_heads"] * c["batch"] > 1:     # no dearer than the largest listed one
        c["batch"], c["kv_heads"] = max(1, c["batch"] // 2), max(1, c["kv_heads"] // 2)
        c["heads"] = c["kv_heads"] * group
    return c


def _cost(c):
    w = work(c)
    return w["bytes"] * 30 if c["kind"] == "select" else w["flops"]


# ------------------------------------------------------------------------------------------------
# Inputs.
# ------------------------------------------------------------------------------------------------

def _blocks(n, block):
    return -(-n // block)


def _video(case):
    return case["frames"] * case["height"] * case["width"]


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(1000003 * seed + 17)
    s = dict(case)
    b, h, hk, d = case["batch"], case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] in ("norm_rope", "norm_rope_grad"):
        n = _video(case) + case["text"]
        dtype = DTYPES[case["dtype"]]
        s["grid"] = (case["frames"], case["height"], case["width"], case["text"])
        # The projection's output [batch, tokens, heads, channels]; channels of uneven size, as weights make them.
        size = 0.2 + _normal(g, d).abs()
        if case["fused"]:
            x = (_normal(g, b, n, h + 2 * hk, d) * size).to(dtype)
            q, k = x[:, :, :h], x[:, :, h:h + hk]
        else:
            q, k = (_normal(g, b, n, h, d) * size).to(dtype), (_normal(g, b, n, hk, d) * size).to(dtype)
        s["q"], s["k"] = q.transpose(1, 2), k.transpose(1, 2)
        s["q_weight"], s["k_weight"] = (1 + 0.2 * _normal(g, d) if case["norm"] else None for _ in range(2))
        if case["kind"] == "norm_rope_grad":
            s["dq_out"] = _normal(g, b, h, n, d).bfloat16()
            s["dk_out"] = _normal(g, b, hk, n, d).bfloat16()
        return s
    n_q, n_k, block = case["n_q"], case["n_k"], case["block"]
    if case["kind"] == "select":
        # Tokens share a part with their neighbours, so that the means of blocks tell them apart.
        s["q"], s["k"] = (_smooth(g, b, x, n, d, block) for x, n in ((h, n_q), (hk, n_k)))
        return s
    s["q"] = _normal(g, b, h, n_q, d).bfloat16()
    s["k"], s["v"] = (_normal(g, b, hk, n_k, d).bfloat16() for _ in range(2))
    s["blockmap"] = _map(g, case)
    # Ranges of query blocks with the most blocks that one of them keeps: those before the text, and the text's.
    nq, nk, text = _blocks(n_q, block), _blocks(n_k, block), case["text"]
    first_q, first_k = ((n_q - text) // block, (n_k - text) // block) if text else (nq, nk)
    s["ranges"] = [(0, first_q, min(case["keep"], first_k) + nk - first_k), (first_q, nq, nk)]
    if case["kind"] == "attention_grad":
        s["do"] = _normal(g, b, h, n_q, d).bfloat16()
        o, s["lse"] = _plain_attention(s)
        s["o"] = o.bfloat16()
    return s


def _smooth(g, b, h, n, d, block):
    nb = _blocks(n, block)
    part = _normal(g, b, h, nb, 1, d).expand(b, h, nb, block, d).reshape(b, h, nb * block, d)[:, :, :n]
    return (_normal(g, b, h, n, d) + 0.3 * part).bfloat16()


def _map(g, case):
    """Blocks that a score chooses: random features of both sides, nearer blocks preferred; text blocks whole."""
    b, h, block, text = case["batch"], case["heads"], case["block"], case["text"]
    nq, nk = _blocks(case["n_q"], block), _blocks(case["n_k"], block)
    score = torch.matmul(_normal(g, b, h, nq, 16), _normal(g, b, h, 16, nk)) / 4 + 0.5 * _normal(g, b, h, nq, nk)
    far = torch.arange(nq, device=DEVICE)[:, None] / nq - torch.arange(nk, device=DEVICE)[None, :] / nk
    score -= 4 * far.abs()
    first = (case["n_k"] - text) // block if text else nk
    m = torch.zeros(b, h, nq, nk, dtype=torch.uint8, device=DEVICE)
    m.scatter_(3, score[..., :first].topk(min(case["keep"], first), dim=3).indices, 1)
    if text:
        m[..., first:] = 1
        m[..., (case["n_q"] - text) // block:, :] = 1
    return m


# ------------------------------------------------------------------------------------------------
# The calls.
# ------------------------------------------------------------------------------------------------

def run(state):
    s, kind = state, state["kind"]
    if own:
        import paper_2609_37001_amd as psa
        if kind == "norm_rope":
            return psa.qk_norm_rope(s["q"], s["k"], s["grid"], AXES[s["dim"]], **_options(s))
        if kind == "norm_rope_grad":
            return psa.qk_norm_rope_bwd(s["dq_out"], s["dk_out"], s["q"], s["k"], s["grid"], AXES[s["dim"]],
                                        **_options(s))
        if kind == "select":
            return psa.select_blocks(s["q"], s["k"], s["block"], s["keep"], q_text=s["text"], k_text=s["text"])
        if kind == "attention":
            return psa.attention_map_fwd(s["q"], s["k"], s["v"], s["blockmap"], s["block"])
        return psa.attention_map_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["blockmap"], s["block"])
    if kind == "norm_rope":
        cos, sin = _angles(s, torch.float32)
        return tuple(_plain_norm_rope(s, s[x], s[x + "_weight"], cos, sin) for x in ("q", "k"))
    if kind == "norm_rope_grad":
        cos, sin = _angles(s, torch.float32)
        (dq, dqw), (dk, dkw) = (_plain_norm_rope_grad(s, s["d%s_out" % x], s[x], s[x + "_weight"], cos, sin)
                                for x in ("q", "k"))
        return dq, dk, dqw, dkw
    if kind == "select":
        return _plain_select(s)
    if kind == "attention":
        return _plain_attention(s)[0].bfloat16()
    return _plain_attention_grad(s)


def _options(s):
    return {"q_weight": s["q_weight"], "k_weight": s["k_weight"], "norm": s["norm"], "pairing": s["pairing"],
            "origin": (s["frame0"], 0, 0)}


EPS, THETA = 1e-6, 10000.0


def _angles(s, dtype):
    """cos and sin [tokens, dim / 2] of the pairs' angles; text tokens turn by nothing."""
    f, h, w, text = s["frames"], s["height"], s["width"], s["text"]
    i = torch.arange(f * h * w, device=DEVICE)
    turns = torch.cat([
        p[:, None].double() * THETA ** (-torch.arange(0, da, 2, device=DEVICE).double() / da)
        for p, da in zip((i // (h * w) + s["frame0"], i // w % h, i % w), AXES[s["dim"]])], dim=1)
    turns = torch.cat([turns, turns.new_zeros(text, turns.shape[1])])
    return turns.cos().to(dtype), turns.sin().to(dtype)


def _split(x, pairing):
    return (x[..., 0::2], x[..., 1::2]) if pairing == "adjacent" else x.chunk(2, dim=-1)


def _join(a, b, pairing):
    return torch.stack([a, b], dim=-1).flatten(-2) if pairing == "adjacent" else torch.cat([a, b], dim=-1)


def _plain_norm_rope(s, x, weight, cos, sin):
    x = x.float()
    if s["norm"]:
        x = x * (x.square().mean(dim=-1, keepdim=True) + EPS).rsqrt() * weight
    a, b = _split(x, s["pairing"])
    return _join(a * cos - b * sin, a * sin + b * cos, s["pairing"]).bfloat16()


def _plain_norm_rope_grad(s, dy, x, weight, cos, sin):
    a, b = _split(dy.float(), s["pairing"])
    g = _join(a * cos + b * sin, b * cos - a * sin, s["pairing"])
    if not s["norm"]:
        return g.to(x.dtype), None
    dtype, x = x.dtype, x.float()
    r = (x.square().mean(dim=-1, keepdim=True) + EPS).rsqrt()
    unit, t = x * r, g * weight
    dx = r * (t - unit * (t * unit).mean(dim=-1, keepdim=True))
    return dx.to(dtype), (g * unit).sum(dim=(0, 1, 2))


def _means(x, block):
    n = x.shape[2]
    nb = _blocks(n, block)
    x = torch.nn.functional.pad(x.double(), (0, 0, 0, nb * block - n)).unflatten(2, (nb, block)).sum(dim=3)
    count = (n - block * torch.arange(nb, device=DEVICE)).clamp(max=block)
    return x / count[:, None]


def _plain_select(s):
    block, text, h, hk = s["block"], s["text"], s["heads"], s["kv_heads"]
    mq, mk = _means(s["q"], block), _means(s["k"], block).repeat_interleave(h // hk, dim=1)
    score = torch.matmul(mq, mk.transpose(2, 3).contiguous())
    nq, nk = score.shape[2:]
    first = (s["n_k"] - text) // block if text else nk
    # stable: of equal scores the lowest index comes first
    order = score[..., :first].sort(dim=3, descending=True, stable=True).indices[..., :min(s["keep"], first)]
    m = torch.zeros(score.shape, dtype=torch.uint8, device=DEVICE)
    m.scatter_(3, order, 1)
    if text:
        m[..., first:] = 1
        m[..., (s["n_q"] - text) // block:, :] = 1
    return m, m.sum(dim=3, dtype=torch.int32)


def _ranges(s, arrays):
    """For each range of query blocks and as many heads at once as keep the gathered keys under `arrays` times 2^30
    elements: a slice of the heads, one of the query blocks, and of these the rows of the key head [heads, 1, 1], the
    gathered tokens [heads, query blocks, keys] and which of those do not count (blocks that fill a list up,
    places behind the last token)."""
    valid, idx = s["blockmap"].flatten(0, 1).sort(dim=2, descending=True, stable=True)
    n = idx.shape[0]
    for q0, q1, most in s["ranges"]:
        each = max(1, (q1 - q0) * most * s["block"] * max(s["dim"], min(s["block"], s["n_q"])))
        step = max(1, int(arrays * 2 ** 30) // each)
        for i in range(0, n if q1 > q0 else 0, step):
            heads, rows = slice(i, i + step), slice(q0, q1)
            kh = torch.arange(n, device=DEVICE)[heads] // (s["heads"] // s["kv_heads"])
            key = idx[heads, rows, :most, None] * s["block"] + torch.arange(s["block"], device=DEVICE)
            gone = ~valid[heads, rows, :most, None].bool() | (key >= s["n_k"])
            yield heads, rows, kh[:, None, None], key.clamp(max=s["n_k"] - 1).flatten(2), gone.flatten(2)


def _in_blocks(x, block):
    """[batch * heads, blocks, block, dim] in 32 bits, the last block filled up with zeros."""
    x = x.flatten(0, 1)
    nb = _blocks(x.shape[1], block)
    return torch.nn.functional.pad(x, (0, 0, 0, nb * block - x.shape[1])).unflatten(1, (nb, block)).float()


def _scores(s, q, kg, gone):
    score = torch.matmul(q, kg.transpose(2, 3)) * s["dim"] ** -0.5
    return score.masked_fill_(gone[:, :, None, :], -math.inf)


def _rows(s, x):
    """[batch * heads, blocks, block, dim] of queries back as they came."""
    return x.flatten(1, 2)[:, :s["n_q"]].unflatten(0, (s["batch"], s["heads"]))


def _plain_attention(s):
    # the rows of a single short block are not filled up
    q = _in_blocks(s["q"], s["block"])[:, :, :s["n_q"]]
    k, v = s["k"].flatten(0, 1), s["v"].flatten(0, 1)
    o, lse = torch.empty_like(q), torch.empty_like(q[..., :1])
    for heads, rows, kh, key, gone in _ranges(s, 2):
        p = _scores(s, q[heads, rows], k[kh, key].float(), gone)
        top = p.amax(dim=3, keepdim=True).clamp(min=-1e30)
        total = p.sub_(top).exp_().sum(dim=3, keepdim=True)
        o[heads, rows] = torch.matmul(p, v[kh, key].float()) / total.clamp(min=1e-30)
        lse[heads, rows] = top + total.log()
    return _rows(s, o), _rows(s, lse).squeeze(3).contiguous()


def _plain_attention_grad(s):
    d, scale = s["dim"], s["dim"] ** -0.5
    q, o, do, lse = (_in_blocks(x, s["block"])[:, :, :s["n_q"]] for x in (s["q"], s["o"], s["do"], s["lse"][..., None]))
    delta = (o * do).sum(dim=3, keepdim=True)
    k, v = s["k"].flatten(0, 1), s["v"].flatten(0, 1)
    dk, dv = (torch.zeros(x.shape, device=DEVICE).flatten(0, 1) for x in (k, v))
    dq = torch.empty_like(q)
    for heads, rows, kh, key, gone in _ranges(s, 1):
        kg, at = k[kh, key].float(), (kh * s["n_k"] + key).flatten()
        p = _scores(s, q[heads, rows], kg, gone).sub_(lse[heads, rows]).exp_()
        dv.index_add_(0, at, torch.matmul(p.transpose(2, 3), do[heads, rows]).flatten(0, 2))
        dp = torch.matmul(do[heads, rows], v[kh, key].float().transpose(2, 3))
        ds = p.mul_(dp.sub_(delta[heads, rows])).mul_(scale)
        dq[heads, rows] = torch.matmul(ds, kg)
        dk.index_add_(0, at, torch.matmul(ds.transpose(2, 3), q[heads, rows]).flatten(0, 2))
    dk, dv = (x.view(s["batch"], s["kv_heads"], s["n_k"], d) for x in (dk, dv))
    return tuple(x.bfloat16().contiguous() for x in (_rows(s, dq), dk, dv))


# ------------------------------------------------------------------------------------------------
# What a pass cannot do without.
# ------------------------------------------------------------------------------------------------

def _pairs(case):
    """Query-key pairs of tokens over all heads (blocks counted whole but for the sequences' ends)."""
    block, text, n_q, n_k = case["block"], case["text"], case["n_q"], case["n_k"]
    first = (n_k - text) // block if text else _blocks(n_k, block)
    kept = min(n_k, min(case["keep"], first) * block + (n_k - first * block if text else 0))
    rows = n_q - (n_q - text) // block * block if text else 0     # rows of text blocks keep everything
    return case["batch"] * case["heads"] * float((n_q - rows) * kept + rows * n_k)


def work(case):
    b, h, hk, d = case["batch"], case["heads"], case["kv_heads"], case["dim"]
    kind = case["kind"]
    if kind in ("norm_rope", "norm_rope_grad"):
        n, size = (_video(case) + case["text"]) * b * (h + hk) * d, 2 if case["dtype"] == "bf16" else 4
        if kind == "norm_rope":
            return {"bytes": n * (size + 2), "flops": n * (7 if case["norm"] else 3)}
        return {"bytes": n * (2 + size * (2 if case["norm"] else 1)), "flops": n * (14 if case["norm"] else 3)}
    block = case["block"]
    nq, nk = _blocks(case["n_q"], block), _blocks(case["n_k"], block)
    q_bytes, k_bytes = 2 * b * h * case["n_q"] * d, 2 * b * hk * case["n_k"] * d
    if kind == "select":
        return {"bytes": q_bytes + k_bytes + b * h * nq * (nk + 4), "flops": 2.0 * b * h * nq * nk * d}
    # keys and values of the blocks that some row of the key head's queries keeps
    share = 1.0 if case["text"] else 1.0 - (1.0 - min(case["keep"], nk) / nk) ** (nq * h // hk)
    if kind == "attention":
        return {"bytes": 2 * q_bytes + 2 * k_bytes * share + b * h * nq * nk, "flops": 4.0 * d * _pairs(case)}
    return {"bytes": 4 * q_bytes + 2 * k_bytes * share + 2 * k_bytes + 4 * b * h * case["n_q"] + b * h * nq * nk,
            "flops": 10.0 * d * _pairs(case)}


# ------------------------------------------------------------------------------------------------
# The same from the definitions, in 64 bits, one head at a time.
# ------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind, group = case["kind"], case["heads"] // case["kv_heads"]
    if kind in ("norm_rope", "norm_rope_grad"):
        return _exact_norm_rope(s)
    if kind == "select":
        return None                                  # whole numbers only
    res = []
    for b in range(case["batch"]):
        for hk in range(case["kv_heads"]):
            heads = range(hk * group, (hk + 1) * group)
            res.append(_exact_heads(s, b, hk, heads, kind == "attention_grad"))
    q_part = torch.cat([r[0] for r in res]).view(case["batch"], case["heads"], case["n_q"], case["dim"])
    if kind == "attention":
        return q_part
    k_parts = (torch.stack([r[i] for r in res]).view(case["batch"], case["kv_heads"], case["n_k"], case["dim"])
               for i in (1, 2))
    return (q_part, *k_parts)


def _exact_heads(s, b, hk, heads, grad):
    """One key head and its query heads, a band of query rows at a time against every key."""
    block, n_q, n_k, d = s["block"], s["n_q"], s["n_k"], s["dim"]
    k, v = s["k"][b, hk].double(), s["v"][b, hk].double()
    scale, band = 1.0 / math.sqrt(d), block * max(1, 2 ** 31 // (n_k * block))
    dk, dv, out = torch.zeros_like(k), torch.zeros_like(v), []
    for h in heads:
        for r0 in range(0, n_q, band):
            r1 = min(n_q, r0 + band)
            q = s["q"][b, h, r0:r1].double()
            keep = s["blockmap"][b, h, r0 // block:_blocks(r1, block)].bool()
            keep = keep.repeat_interleave(block, 0)[:r1 - r0].repeat_interleave(block, 1)[:, :n_k]
            x = (q @ k.T).mul_(scale).masked_fill_(~keep, -math.inf)
            if not grad:
                x = torch.softmax(x, dim=1)
                out.append(torch.nan_to_num(x) @ v)
                continue
            # from the o and lse that the call is given
            do = s["do"][b, h, r0:r1].double()
            p = x.sub_(s["lse"][b, h, r0:r1, None].double()).exp_()
            dv += p.T @ do
            ds = (do @ v.T).sub_((do * s["o"][b, h, r0:r1].double()).sum(1, keepdim=True)).mul_(p)
            dk += (ds.T @ q).mul_(scale)
            out.append((ds @ k).mul_(scale))
    return torch.stack([torch.cat(out).view(len(heads), n_q, d)]).flatten(0, 1), dk, dv


def _exact_norm_rope(s):
    """The rotation as a product of complex numbers, one head at a time."""
    cos, sin = _angles(s, torch.float64)
    turn = torch.complex(cos, sin)
    d = s["dim"]

    def pairs(x):
        return torch.view_as_complex(x.unflatten(-1, (d // 2, 2)).contiguous()) if s["pairing"] == "adjacent" \
            else torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous())

    def channels(z):
        return torch.view_as_real(z).flatten(-2) if s["pairing"] == "adjacent" else torch.cat([z.real, z.imag], -1)

    def forward(x, w):
        x = x.double()
        if s["norm"]:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.double()
        return channels(pairs(x) * turn).float()     # (held in half the space; outputs have 8 bits)

    def backward(dy, x, w):
        g = channels(pairs(dy.double()) * turn.conj())
        if not s["norm"]:
            return g, 0.0
        x = x.double()
        size = torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        gw = g * w.double()
        return (gw - x * (gw * x).mean(-1, keepdim=True) / size ** 2) / size, (g * x / size).sum(0)

    if s["kind"] == "norm_rope":
        return tuple(torch.stack([torch.stack([forward(y, s[x + "_weight"]) for y in z]) for z in s[x]])
                     for x in ("q", "k"))
    dx, dw = [], []
    for x in ("q", "k"):
        got = [[backward(dy, y, s[x + "_weight"]) for dy, y in zip(dz, z)] for dz, z in zip(s["d%s_out" % x], s[x])]
        dx.append(torch.stack([torch.stack([y[0] for y in z]) for z in got]))
        dw.append(sum(y[1] for z in got for y in z) if s["norm"] else None)
    return (*dx, *dw)
