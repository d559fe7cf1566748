"""PSA (Parameterized Stripe Attention) block-sparse attention forward for MI355X (gfx950).

Thin torch-facing wrapper around the C ABI of ``libpsa.so`` (``include/psa.h``): tensors are
only checked for dtype, device and layout, then their device pointers and the current HIP
stream are handed to the library.  Every computation runs in the library's HIP kernels; there
is no CPU or PyTorch fallback.

    params = [(T_w, T_o, T_s, S_w, S_o, S_s), ...]          # one 6-tuple per head
    o = attention_fwd(q, k, v, grid=(F, H, W, n_text), block=128, params=params)
    o_dense = dense_fwd(q, k, v, block=128)
    ws = plan(params, grid, block, batch=1)                   # plan once ...
    o = run(q, k, v, grid, block, ws)                         # ... run many times
    bmap, per_row, per_head = build_blockmap(params, (F, H, W, n_text), block=128)

3D PSABlocks with 3D padding (the paper's layout; q, k, v permuted once, e.g. for a whole DiT):

    pb = (3, 8, 16)
    qb, kb, vb = (to_blocks(x, grid, pb) for x in (q, k, v))
    ob = attention_fwd_3d(qb, kb, vb, grid, pb, params, tile=128)
    o = from_blocks(ob, grid, pb)

Norms and 3D rotary positions of queries and keys, from the projection's [batch, N, heads, d]:

    q, k = qk_norm_rope(xq.transpose(1, 2), xk.transpose(1, 2), grid, (44, 42, 42), q_weight=wq, k_weight=wk)

Attention over a map of blocks that a score of the data selects (or over any other block map):

    bmap, kept = select_blocks(q, k, block=128, keep=64)
    o, lse = attention_map_fwd(q, k, v, bmap, block=128, return_lse=True)
    dq, dk, dv = attention_map_bwd(do, q, k, v, o, lse, bmap, block=128)

No call records anything for autograd: the tensors returned have no graph, also where inputs require gradients.  The
gradients are calls of their own (`*_bwd`).
"""
import contextlib
import math

from . import _lib
from ._lib import STRIDE_INF, PsaError  # noqa: F401

__all__ = ["STRIDE_INF", "PsaError", "num_blocks", "workspace_size", "build_blockmap",
           "attention_fwd", "attention_fwd_noalloc", "plan", "run", "dense_fwd", "dense_workspace_size", "Workspace", "library_path",
           "blocked_tokens", "to_blocks", "from_blocks", "build_blockmap_3d", "plan_3d", "run_3d",
           "attention_fwd_3d", "l2_distance", "qk_norm_rope", "qk_norm_rope_bwd", "select_blocks",
           "attention_map_fwd", "attention_map_bwd"]


def library_path():
    return _lib.LIB_PATH


def _grid(grid):
    g = tuple(int(x) for x in grid)
    if len(g) == 3:
        g = g + (0,)
    if len(g) != 4:
        raise ValueError("grid is (frames, height, width[, n_text])")
    return _lib.grid_of(*g)


def num_blocks(grid, block):
    return int(_lib.lib().psa_num_blocks(_grid(grid), int(block)))


def workspace_size(batch, n_heads, grid, block):
    return int(_lib.lib().psa_workspace_size(int(batch), int(n_heads), _grid(grid), int(block)))


def _torch():
    import torch
    return torch


def _stream(stream, device):
    torch = _torch()
    if stream is None:
        stream = torch.cuda.current_stream(device)
    return ctypes_void(stream.cuda_stream)


def _on(stream):
    """Context for the allocations and the library call of one binding function: with a stream
    given, it becomes torch's current stream, so the tensors the function allocates (outputs,
    workspaces) belong to that stream's memory pool and are not handed to other work while the
    library still uses them there.  The caller orders the inputs onto that stream."""
    return contextlib.nullcontext() if stream is None else _torch().cuda.stream(stream)


def ctypes_void(x):
    """A pointer argument (the library's argument types take plain integers; 0 is NULL)."""
    return int(x) if x else None


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _check_qkv(*ts):
    torch = _torch()
    ref = ts[0]
    for t in ts:
        if t.dtype != torch.bfloat16:
            raise TypeError("q, k, v must be bfloat16")
        if not t.is_cuda:
            raise ValueError("q, k, v must be GPU tensors")
        if not t.is_contiguous():
            raise ValueError("q, k, v must be contiguous [batch, heads, N, head_dim]")
        if t.dim() != 4 or t.shape != ref.shape:
            raise ValueError("q, k, v must share the shape [batch, heads, N, head_dim]")
        if t.device != ref.device:
            raise ValueError("q, k, v must be on one device")


class Workspace:
    """Device workspace for attention_fwd / plan / run (a byte tensor on the given device).

    After plan() it also records the sizes and parameters of the plan it holds."""

    def __init__(self, batch, n_heads, grid, block, device):
        torch = _torch()
        self.nbytes = workspace_size(batch, n_heads, grid, block)
        if self.nbytes == 0:
            raise ValueError("invalid sizes for a workspace")
        self.tensor = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        self.sizes = (int(batch), int(n_heads), tuple(int(x) for x in _grid_tuple(grid)), int(block))
        self.params = None


def _grid_tuple(grid):
    g = tuple(int(x) for x in grid)
    return g + (0,) if len(g) == 3 else g


def _check_tokens(n, grid):
    """The library sees raw pointers: a tensor shorter than the grid would be read past its end."""
    f, h, w, nt = _grid_tuple(grid)
    if n != f * h * w + nt:
        raise ValueError("tensors hold %d tokens, the grid %s has %d" % (n, (f, h, w, nt), f * h * w + nt))


def build_blockmap(params, grid, block, device=None, blockmap=True, per_row=True, per_head=True,
                   stream=None):
    """Block map of the stripe parameters on the device.

    Returns (map uint8 [heads, nb, nb] | None, kept_per_row int32 [heads, nb] | None,
    kept_per_head int64 [heads] | None)."""
    torch = _torch()
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    heads = len(params)
    nb = num_blocks(grid, block)
    if nb < 0:
        raise ValueError("invalid grid or block")
    with torch.cuda.device(device), _on(stream):
        bm = torch.empty((heads, nb, nb), dtype=torch.uint8, device=device) if blockmap else None
        pr = torch.empty((heads, nb), dtype=torch.int32, device=device) if per_row else None
        ph = torch.empty((heads,), dtype=torch.int64, device=device) if per_head else None
        _lib.check(_lib.lib().psa_build_blockmap(_lib.stripes(params), heads, _grid(grid), int(block),
                                                 _ptr(bm), _ptr(pr), _ptr(ph), _stream(None, device)))
    return bm, pr, ph


def attention_fwd(q, k, v, grid, block, params, scale=None, out=None, return_lse=False,
                  workspace=None, return_kept_per_row=False, stream=None):
    """PSA block-sparse attention forward.  q, k, v: bf16 [batch, heads, N, head_dim], contiguous.

    Returns o (and lse float32 [batch, heads, N], kept_per_row int32 [heads, nb] if asked)."""
    torch = _torch()
    _check_qkv(q, k, v)
    b, h, n, d = q.shape
    if len(params) != h:
        raise ValueError("one stripe tuple per head is required")
    _check_tokens(n, grid)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    with torch.cuda.device(q.device), _on(stream):
        o = torch.empty_like(q) if out is None else out
        _check_qkv(q, o)
        lse = torch.empty((b, h, n), dtype=torch.float32, device=q.device) if return_lse else None
        kept = None
        if return_kept_per_row:
            kept = torch.empty((h, max(num_blocks(grid, block), 1)), dtype=torch.int32, device=q.device)
        ws = workspace if workspace is not None else Workspace(b, h, grid, block, q.device)
        _lib.check(_lib.lib().psa_attention_fwd(
            _ptr(q), _ptr(k), _ptr(v), _ptr(o), b, h, d, _grid(grid), int(block),
            _lib.stripes(params), scale, _ptr(ws.tensor), ws.nbytes, _ptr(lse), _ptr(kept),
            _stream(None, q.device)))
    ws.sizes = (b, h, _grid_tuple(grid), int(block))
    ws.params = [tuple(map(int, m)) for m in params]
    res = (o,)
    if return_lse:
        res += (lse,)
    if return_kept_per_row:
        res += (kept,)
    return res[0] if len(res) == 1 else res


def attention_fwd_noalloc(q, k, v, grid, block, params, out, scale=None, lse=None, kept_per_row=None,
                          stream=None):
    """attention_fwd with the plan in the library's static device scratch
    (psa_attention_fwd_noalloc): neither the library nor this wrapper allocates, so the caller
    passes the output `out` (bf16 like q) and, if wanted, `lse` (float32 [batch, heads, N]) and
    `kept_per_row` (int32 [heads, nb]).  Calls that overlap in time on one GPU must not be made."""
    torch = _torch()
    _check_qkv(q, k, v)
    _check_qkv(q, out)
    b, h, n, d = q.shape
    if len(params) != h:
        raise ValueError("one stripe tuple per head is required")
    _check_tokens(n, grid)
    nb = num_blocks(grid, block)
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (b, h, n) or not lse.is_contiguous()):
        raise ValueError("lse must be a contiguous float32 tensor [batch, heads, N]")
    if kept_per_row is not None and (kept_per_row.dtype != torch.int32 or tuple(kept_per_row.shape) != (h, nb)
                                     or not kept_per_row.is_contiguous()):
        raise ValueError("kept_per_row must be a contiguous int32 tensor [heads, nb]")
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    with torch.cuda.device(q.device):
        _lib.check(_lib.lib().psa_attention_fwd_noalloc(
            _ptr(q), _ptr(k), _ptr(v), _ptr(out), b, h, d, _grid(grid), int(block), _lib.stripes(params),
            scale, _ptr(lse), _ptr(kept_per_row), _stream(stream, q.device)))
    return out


def plan(params, grid, block, batch=1, device=None, workspace=None, return_kept_per_row=False,
         stream=None):
    """Plan of the sparse attention for these stripes and sizes (psa_attention_plan).

    Returns the Workspace holding it (and kept_per_row int32 [heads, nb] if asked)."""
    torch = _torch()
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    h = len(params)
    nb = num_blocks(grid, block)
    with torch.cuda.device(device), _on(stream):
        ws = workspace if workspace is not None else Workspace(batch, h, grid, block, device)
        kept = torch.empty((h, max(nb, 1)), dtype=torch.int32, device=device) if return_kept_per_row else None
        _lib.check(_lib.lib().psa_attention_plan(int(batch), h, _grid(grid), int(block),
                                                 _lib.stripes(params), _ptr(ws.tensor), ws.nbytes,
                                                 _ptr(kept), _stream(None, device)))
    ws.sizes = (int(batch), h, _grid_tuple(grid), int(block))
    ws.params = [tuple(map(int, m)) for m in params]
    return (ws, kept) if return_kept_per_row else ws


def run(q, k, v, grid, block, workspace, scale=None, out=None, return_lse=False, stream=None):
    """Sparse attention over a planned workspace (psa_attention_run)."""
    torch = _torch()
    _check_qkv(q, k, v)
    b, h, n, d = q.shape
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    _check_tokens(n, grid)
    ws = workspace
    if ws.params is None:
        raise ValueError("the workspace holds no plan: call plan() or attention_fwd() first")
    if ws.sizes != (b, h, _grid_tuple(grid), int(block)):
        raise ValueError("the workspace was planned for (batch, heads, grid, block) = %s, not %s"
                         % (ws.sizes, (b, h, _grid_tuple(grid), int(block))))
    with torch.cuda.device(q.device), _on(stream):
        o = torch.empty_like(q) if out is None else out
        _check_qkv(q, o)
        lse = torch.empty((b, h, n), dtype=torch.float32, device=q.device) if return_lse else None
        _lib.check(_lib.lib().psa_attention_run(
            _ptr(q), _ptr(k), _ptr(v), _ptr(o), b, h, d, _grid(grid), int(block), scale,
            _ptr(ws.tensor), ws.nbytes, _ptr(lse), _stream(None, q.device)))
    return (o, lse) if return_lse else o


def dense_workspace_size():
    return int(_lib.lib().psa_dense_workspace_size())


def dense_fwd(q, k, v, block, scale=None, out=None, return_lse=False, stream=None, workspace=None,
              balanced=True):
    """Dense attention forward with the same tile engine (the speedup baseline).

    balanced (default): a persistent grid takes the work items from per-XCD queues in a small
    workspace -- `workspace`, a uint8 device tensor of dense_workspace_size() bytes, or a fresh
    one -- so that XCDs holding different clocks finish together.  balanced=False runs the fixed
    grid (an equal share per XCD, no workspace).  Same output bits either way."""
    torch = _torch()
    _check_qkv(q, k, v)
    b, h, n, d = q.shape
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    with torch.cuda.device(q.device), _on(stream):
        o = torch.empty_like(q) if out is None else out
        _check_qkv(q, o)
        lse = torch.empty((b, h, n), dtype=torch.float32, device=q.device) if return_lse else None
        if not balanced:
            workspace = None
        elif workspace is None:
            workspace = torch.empty(dense_workspace_size(), dtype=torch.uint8, device=q.device)
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        _lib.check(_lib.lib().psa_dense_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), b, h, d, n, int(block),
                                            scale, _ptr(lse), _ptr(workspace), ws_bytes,
                                            _stream(None, q.device)))
    return (o, lse) if return_lse else o


# ---------------------------------------------------------------------------------------------
# 3D PSABlocks with 3D padding (include/psa.h, second part).
# ---------------------------------------------------------------------------------------------

def blocked_tokens(grid, pb):
    """Positions of the PSABlock-centric layout (T' H' W' bt bh bw + n_text)."""
    return int(_lib.lib().psa_blocked_tokens(_grid(grid), _lib.block3d_of(pb)))


def _layout(src, grid, pb, out, stream, to):
    torch = _torch()
    if src.dtype != torch.bfloat16 or not src.is_cuda or not src.is_contiguous() or src.dim() != 4:
        raise ValueError("expected a contiguous bf16 GPU tensor [batch, heads, tokens, head_dim]")
    b, h, n, d = src.shape
    g = _grid_tuple(grid)
    n_orig = g[0] * g[1] * g[2] + g[3]
    n_blk = blocked_tokens(grid, pb)
    if n_blk < 0:
        raise ValueError("invalid grid or PSABlock shape")
    if n != (n_orig if to else n_blk):
        raise ValueError("tensor has %d tokens, the %s layout has %d" % (n, "original" if to else "blocked",
                                                                        n_orig if to else n_blk))
    shape = (b, h, n_blk if to else n_orig, d)
    fn = _lib.lib().psa_to_blocks if to else _lib.lib().psa_from_blocks
    with torch.cuda.device(src.device), _on(stream):
        dst = torch.empty(shape, dtype=src.dtype, device=src.device) if out is None else out
        if tuple(dst.shape) != shape or not dst.is_contiguous() or dst.dtype != src.dtype:
            raise ValueError("out must be a contiguous bf16 tensor of shape %s" % (shape,))
        _lib.check(fn(_ptr(src), _ptr(dst), b * h, d, _grid(grid), _lib.block3d_of(pb),
                      _stream(None, src.device)))
    return dst


def to_blocks(x, grid, pb, out=None, stream=None):
    """[batch, heads, F*H*W + n_text, d] -> PSABlock-centric layout (psa_to_blocks)."""
    return _layout(x, grid, pb, out, stream, True)


def from_blocks(xb, grid, pb, out=None, stream=None):
    """PSABlock-centric layout -> [batch, heads, F*H*W + n_text, d] (psa_from_blocks)."""
    return _layout(xb, grid, pb, out, stream, False)


def build_blockmap_3d(params, grid, pb, device=None, blockmap=True, per_row=True, per_head=True,
                      stream=None):
    """PSABlock-level map: (uint8 [heads, G, G] | None, int32 [heads, G] | None,
    int64 [heads] | None), G = T'H'W' (+1 for the text group)."""
    torch = _torch()
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    g = _grid_tuple(grid)
    (tp, hp, wp) = (-(-g[0] // pb[0]), -(-g[1] // pb[1]), -(-g[2] // pb[2]))
    groups = tp * hp * wp + (1 if g[3] > 0 else 0)
    heads = len(params)
    with torch.cuda.device(device), _on(stream):
        bm = torch.empty((heads, groups, groups), dtype=torch.uint8, device=device) if blockmap else None
        pr = torch.empty((heads, groups), dtype=torch.int32, device=device) if per_row else None
        ph = torch.empty((heads,), dtype=torch.int64, device=device) if per_head else None
        _lib.check(_lib.lib().psa_build_blockmap_3d(_lib.stripes(params), heads, _grid(grid),
                                                    _lib.block3d_of(pb), _ptr(bm), _ptr(pr), _ptr(ph),
                                                    _stream(None, device)))
    return bm, pr, ph


class Workspace3d(Workspace):
    """Workspace of plan_3d / run_3d."""

    def __init__(self, batch, n_heads, grid, pb, tile, device):
        torch = _torch()
        self.nbytes = int(_lib.lib().psa_workspace_size_3d(int(batch), int(n_heads), _grid(grid),
                                                            _lib.block3d_of(pb), int(tile)))
        if self.nbytes == 0:
            raise ValueError("invalid sizes for a 3D workspace")
        self.tensor = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        self.sizes = (int(batch), int(n_heads), _grid_tuple(grid), tuple(int(x) for x in pb), int(tile))
        self.params = None


def plan_3d(params, grid, pb, tile=128, batch=1, device=None, workspace=None,
            return_kept_per_tile=False, stream=None):
    """Plan over the PSABlock-centric layout (psa_attention_plan_3d)."""
    torch = _torch()
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    h = len(params)
    n_tiles = -(-blocked_tokens(grid, pb) // int(tile))
    with torch.cuda.device(device), _on(stream):
        ws = workspace if workspace is not None else Workspace3d(batch, h, grid, pb, tile, device)
        kept = torch.empty((h, n_tiles), dtype=torch.int32, device=device) if return_kept_per_tile else None
        _lib.check(_lib.lib().psa_attention_plan_3d(int(batch), h, _grid(grid), _lib.block3d_of(pb),
                                                    int(tile), _lib.stripes(params), _ptr(ws.tensor),
                                                    ws.nbytes, _ptr(kept), _stream(None, device)))
    ws.sizes = (int(batch), h, _grid_tuple(grid), tuple(int(x) for x in pb), int(tile))
    ws.params = [tuple(map(int, m)) for m in params]
    return (ws, kept) if return_kept_per_tile else ws


def run_3d(q, k, v, grid, pb, tile, workspace, scale=None, out=None, return_lse=False, stream=None):
    """Sparse attention over a 3D plan; q, k, v, o in the PSABlock-centric layout."""
    torch = _torch()
    _check_qkv(q, k, v)
    b, h, n, d = q.shape
    if n != blocked_tokens(grid, pb):
        raise ValueError("q, k, v must be in the PSABlock-centric layout (%d tokens)" % blocked_tokens(grid, pb))
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    ws = workspace
    if ws.params is None:
        raise ValueError("the workspace holds no plan: call plan_3d() first")
    if ws.sizes != (b, h, _grid_tuple(grid), tuple(int(x) for x in pb), int(tile)):
        raise ValueError("the workspace was planned for %s, not %s"
                         % (ws.sizes, (b, h, _grid_tuple(grid), tuple(pb), int(tile))))
    with torch.cuda.device(q.device), _on(stream):
        o = torch.empty_like(q) if out is None else out
        _check_qkv(q, o)
        lse = torch.empty((b, h, n), dtype=torch.float32, device=q.device) if return_lse else None
        _lib.check(_lib.lib().psa_attention_run_3d(
            _ptr(q), _ptr(k), _ptr(v), _ptr(o), b, h, d, _grid(grid), _lib.block3d_of(pb), int(tile),
            scale, _ptr(ws.tensor), ws.nbytes, _ptr(lse), _stream(None, q.device)))
    return (o, lse) if return_lse else o


def attention_fwd_3d(q, k, v, grid, pb, params, tile=128, scale=None, out=None, return_lse=False,
                     workspace=None, stream=None):
    """plan_3d then run_3d (q, k, v in the PSABlock-centric layout)."""
    b = q.shape[0]
    ws = plan_3d(params, grid, pb, tile, batch=b, device=q.device, workspace=workspace, stream=stream)
    return run_3d(q, k, v, grid, pb, tile, ws, scale, out, return_lse, stream)


# ---------------------------------------------------------------------------------------------
# PSA-Search scoring (include/psa.h, third part); the search itself is in .search.
# ---------------------------------------------------------------------------------------------

def l2_distance(o, ref, sq_err=None, sq_ref=None, workspace=None, stream=None):
    """Per (batch, head) sums of (o - ref)^2 and ref^2 (float64 [batch, heads] each)."""
    torch = _torch()
    _check_qkv(o, ref)
    b, h, n, d = o.shape
    nbytes = int(_lib.lib().psa_l2_workspace_size(b * h))
    with torch.cuda.device(o.device), _on(stream):
        err = torch.empty((b, h), dtype=torch.float64, device=o.device) if sq_err is None else sq_err
        rref = torch.empty((b, h), dtype=torch.float64, device=o.device) if sq_ref is None else sq_ref
        for t in (err, rref):
            if t.dtype != torch.float64 or t.numel() != b * h or not t.is_contiguous():
                raise ValueError("sq_err and sq_ref must be contiguous float64 tensors of %d elements" % (b * h))
        ws = torch.empty(nbytes, dtype=torch.uint8, device=o.device) if workspace is None else workspace
        if ws.numel() < nbytes:
            raise ValueError("l2 workspace needs %d bytes" % nbytes)
        _lib.check(_lib.lib().psa_l2_distance(_ptr(o), _ptr(ref), b * h, n, d, _ptr(err), _ptr(rref),
                                              _ptr(ws), ws.numel(), _stream(None, o.device)))
    return err, rref


# ---------------------------------------------------------------------------------------------
# Norms and rotary positions of queries and keys (include/psa.h, fourth part).
# ---------------------------------------------------------------------------------------------

def _int32(x, name):
    """A whole number for a 32-bit argument of the library (ctypes would hand on the low bits of a larger one)."""
    x = int(x)
    if not -0x80000000 <= x <= 0x7fffffff:
        raise ValueError("%s %d is not a number of 32 bits" % (name, x))
    return x


def _on_device(device, stream):
    """Contexts of a call: the tensors' device and the stream given.  Nothing to enter where both are the current
    ones (two contexts cost as much host time as the launch of a small call)."""
    torch = _torch()
    if stream is None and device.index == torch.cuda.current_device():
        return contextlib.nullcontext()
    if stream is not None and stream.device != device:
        raise ValueError("the stream is on %s, the tensors on %s" % (stream.device, device))
    stack = contextlib.ExitStack()
    stack.enter_context(torch.cuda.device(device))
    stack.enter_context(_on(stream))
    return stack


def _like(x, dtype):
    """An uninitialised contiguous tensor of the shape of x."""
    return _torch().empty_like(x, dtype=dtype, memory_format=_torch().contiguous_format)


def _rows(x, name, dtype, tokens, like=None):
    """psa_rows_t of x, [batch, heads, N, head_dim] of any strides with the channels side by side."""
    torch = _torch()
    if dtype not in (torch.bfloat16, torch.float32) or x.dtype != dtype:
        raise TypeError("%s must be bfloat16 or float32, queries and keys alike" % name)
    if not x.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    shape, stride = x.shape, x.stride()
    if len(shape) != 4 or stride[3] != 1:
        raise ValueError("%s must be [batch, heads, N, head_dim] with contiguous channels" % name)
    if shape[2] != tokens:
        raise ValueError("%s has %d tokens, the grid %d" % (name, shape[2], tokens))
    if like is not None and (x.device != like.device or shape[0] != like.shape[0] or shape[3] != like.shape[3]):
        raise ValueError("%s must share the queries' batch, head_dim and device" % name)
    return _lib.Rows(x.data_ptr(), stride[0] if shape[0] > 1 else 0, stride[1] if shape[1] > 1 else 0,
                     stride[2] if shape[2] > 1 else 0, shape[1])


def _rope(grid, axes, theta, origin, pairing):
    if pairing not in ("adjacent", "halves"):
        raise ValueError('pairing is "adjacent" or "halves"')
    a, o = tuple(_int32(x, "axis") for x in axes), tuple(_int32(x, "origin") for x in origin)
    if len(a) != 3 or len(o) != 3:
        raise ValueError("axes and origin have three entries (time, height, width)")
    return _lib.Rope(_grid(grid), *o, *a, _lib.PAIRS_HALVES if pairing == "halves" else _lib.PAIRS_ADJACENT, theta)


def _norm_weight(w, x, name):
    if w is None:
        return
    torch = _torch()
    if (w.dtype != torch.float32 or tuple(w.shape) != (x.shape[3],) or not w.is_contiguous()
            or w.device != x.device):
        raise ValueError("%s must be a contiguous float32 tensor [head_dim] on the queries' device" % name)


def _attention_layout(x, like, name):
    """Checks a bf16 tensor in the attention's layout with the shape of `like`."""
    torch = _torch()
    if x.dtype != torch.bfloat16 or x.shape != like.shape or not x.is_contiguous() or x.device != like.device:
        raise ValueError("%s must be a contiguous bfloat16 tensor %s on the queries' device" % (name, tuple(like.shape)))


def _type_of(x):
    return _lib.TYPE_FP32 if x.dtype == _torch().float32 else _lib.TYPE_BF16


def _tokens(grid):
    f, h, w, nt = _grid_tuple(grid)
    return f * h * w + nt


def qk_norm_rope(q, k, grid, axes, q_weight=None, k_weight=None, norm=True, eps=1e-6, theta=10000.0,
                 origin=(0, 0, 0), pairing="adjacent", q_out=None, k_out=None, stream=None):
    """RMS norm of every head of the queries and keys, then the rotation by their (t, h, w) positions, into
    the attention's layout (psa_qk_norm_rope_fwd).

    q, k: bfloat16 or float32 [batch, heads, N, head_dim] of any strides with contiguous channels, such as
    ``x.view(B, N, heads, d).transpose(1, 2)`` of a projection's output or a slice of a fused one (16-byte
    aligned rows); k may have other heads than q, or be None.  Weights: float32 [head_dim], None for
    ones; norm=False rotates alone.  axes: channels of the time, height and width axes; origin: position of
    the first token (a later chunk of a clip).  Text tokens behind the video are not rotated.

    Returns (q_out, k_out): bfloat16 [batch, heads, N, head_dim], contiguous."""
    torch = _torch()
    n = _tokens(grid)
    rq = _rows(q, "q", q.dtype, n)
    rk = _rows(k, "k", q.dtype, n, like=q) if k is not None else None
    rope = _rope(grid, axes, theta, origin, pairing)
    _norm_weight(q_weight, q, "q_weight")
    _norm_weight(k_weight, q, "k_weight")
    with _on_device(q.device, stream):
        yq, yk = q_out, k_out if k is not None else None
        if yq is None:
            yq = _like(q, torch.bfloat16)
        else:
            _attention_layout(yq, q, "q_out")
        if yk is not None:
            _attention_layout(yk, k, "k_out")
        elif k is not None:
            yk = _like(k, torch.bfloat16)
        _lib.check(_lib.lib().psa_qk_norm_rope_fwd(
            rq, rk, _ptr(yq), _ptr(yk), _type_of(q), q.shape[0], q.shape[3], rope, 1 if norm else 0, _ptr(q_weight),
            _ptr(k_weight), float(eps), _stream(None, q.device.index)))
    return yq, yk


def _empty_rows(x):
    """Uninitialised rows in the order of x (a dense tensor where x is a slice or repeats rows)."""
    torch = _torch()
    if any(s == 0 and size > 1 for s, size in zip(x.stride(), x.shape)):
        return _like(x, x.dtype)
    return torch.empty_like(x)


def qk_norm_rope_bwd(dq_out, dk_out, q, k, grid, axes, q_weight=None, k_weight=None, norm=True, eps=1e-6,
                     theta=10000.0, origin=(0, 0, 0), pairing="adjacent", dq=None, dk=None, workspace=None,
                     stream=None):
    """Gradients of qk_norm_rope (psa_qk_norm_rope_bwd): dq_out and dk_out are those of its outputs (bfloat16,
    contiguous), the other arguments the forward's.

    Returns (dq, dk, dq_weight, dk_weight): dq and dk in the type and order of q and k (or in the tensors
    given, of any strides as for q and k: a fused projection's gradient), one row for each row of the outputs,
    also where an input repeats rows; the weights' float32 [head_dim], None without a norm."""
    torch = _torch()
    n = _tokens(grid)
    rq = _rows(q, "q", q.dtype, n)
    rk = _rows(k, "k", q.dtype, n, like=q) if k is not None else None
    rope = _rope(grid, axes, theta, origin, pairing)
    _norm_weight(q_weight, q, "q_weight")
    _norm_weight(k_weight, q, "k_weight")
    _attention_layout(dq_out, q, "dq_out")
    if k is not None:
        _attention_layout(dk_out, k, "dk_out")
    with _on_device(q.device, stream):
        grads, rows = [], []
        for given, x, name in ((dq, q, "dq"), (dk, k, "dk")):
            if x is None:
                grads.append(None)
                rows.append(None)
                continue
            g = _empty_rows(x) if given is None else given
            if g.shape != x.shape:
                raise ValueError("%s must have the shape %s" % (name, tuple(x.shape)))
            grads.append(g)
            rows.append(_rows(g, name, q.dtype, n, like=q))
        dw = [torch.empty(q.shape[3], dtype=torch.float32, device=q.device) if norm and x is not None else None
              for x in (q, k)]
        nbytes = int(_lib.lib().psa_qk_norm_rope_workspace_size(
            q.shape[0], q.shape[1], k.shape[1] if k is not None else 0, q.shape[3], _grid(grid), 1 if norm else 0))
        ws, ws_bytes, _keep = _workspace(workspace, nbytes, q.device)
        _lib.check(_lib.lib().psa_qk_norm_rope_bwd(
            _ptr(dq_out), _ptr(dk_out) if k is not None else None, rq, rk, rows[0], rows[1], _ptr(dw[0]), _ptr(dw[1]),
            _type_of(q), q.shape[0], q.shape[3], rope, 1 if norm else 0, _ptr(q_weight), _ptr(k_weight), float(eps),
            ws, ws_bytes, _stream(None, q.device.index)))
    return grads[0], grads[1], dw[0], dw[1]


# ---------------------------------------------------------------------------------------------
# Block selection, and attention over any block map (include/psa.h, fifth part).
# ---------------------------------------------------------------------------------------------

def _check_q(q, name="q", like=None):
    torch = _torch()
    if q.dtype != torch.bfloat16:
        raise TypeError("%s must be bfloat16" % name)
    if not q.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if q.dim() != 4 or not q.is_contiguous():
        raise ValueError("%s must be contiguous [batch, heads, N, head_dim]" % name)
    if like is not None and (q.shape != like.shape or q.device != like.device):
        raise ValueError("%s must have the shape %s, on the queries' device" % (name, tuple(like.shape)))


def _kv(q, k, v=None):
    """psa_kv_t of keys and values: [batch, kv heads, N_k, head_dim], each head's rows contiguous."""
    torch = _torch()
    for t in (k,) if v is None else (k, v):
        if t.dtype != torch.bfloat16:
            raise TypeError("k and v must be bfloat16")
        if t.device != q.device:
            raise ValueError("k and v must be on the queries' device")
        if t.dim() != 4 or t.shape[0] != q.shape[0] or t.shape[3] != q.shape[3]:
            raise ValueError("k and v must be [batch, kv heads, N_k, head_dim] with the queries' batch and head_dim")
        if t.stride(3) != 1 or (t.shape[2] > 1 and t.stride(2) != t.shape[3]):
            raise ValueError("the rows of a head of k and v must be contiguous")
    strides = [s if size > 1 else 0 for s, size in zip(k.stride()[:2], k.shape)]
    if v is not None and (v.shape != k.shape or [s if size > 1 else 0 for s, size in zip(v.stride()[:2], v.shape)] != strides):
        raise ValueError("k and v must share their shape and strides")
    return _lib.Kv(k.data_ptr(), _ptr(v), *strides, k.shape[1])


def _blocks(n, block):
    return -(-n // block) if block > 0 else 0


def _map_of(blockmap, q, n_k, block):
    """(pointer, bytes between batch elements) of a map [batch, heads, nbq, nbk] or [heads, nbq, nbk]."""
    torch = _torch()
    if blockmap.dtype not in (torch.uint8, torch.bool):
        raise TypeError("blockmap must be uint8 or bool")
    shape = (q.shape[1], _blocks(q.shape[2], block), _blocks(n_k, block))
    if blockmap.device != q.device or tuple(blockmap.shape) not in (shape, (q.shape[0],) + shape):
        raise ValueError("blockmap must be %s or %s on the queries' device" % (shape, (q.shape[0],) + shape))
    one = blockmap[0] if blockmap.dim() == 4 and q.shape[0] > 0 else blockmap
    if not one.is_contiguous():
        raise ValueError("the maps of a batch element must be contiguous")
    return blockmap.data_ptr(), blockmap.stride(0) if blockmap.dim() == 4 and q.shape[0] > 1 else 0


def _workspace(workspace, nbytes, device):
    """(pointer, bytes) of a workspace tensor, a fresh one if none is given and one is needed; and that tensor, which
    has to live until the call has been enqueued."""
    torch = _torch()
    if workspace is None and nbytes:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if workspace is None:
        return None, 0, None
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError("the workspace must be a contiguous tensor on the queries' device")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def select_blocks(q, k, block, keep, q_text=0, k_text=0, blockmap=None, workspace=None, stream=None):
    """For every query block the `keep` key blocks of the highest mean score, with the text's (psa_select_blocks).

    q: bfloat16 [batch, heads, N_q, head_dim], contiguous; k: [batch, kv heads, N_k, head_dim], each head's rows
    contiguous (kv heads divide heads); q_text, k_text: text tokens at the end of each.

    Returns (map uint8 [batch, heads, nbq, nbk], kept_per_row int32 [batch, heads, nbq])."""
    torch = _torch()
    block, keep = _int32(block, "block"), _int32(keep, "keep")
    q_text, k_text = _int32(q_text, "q_text"), _int32(k_text, "k_text")
    _check_q(q)
    kv = _kv(q, k)
    b, h, n_q, d = q.shape
    n_k = k.shape[2]
    shape = (b, h, _blocks(n_q, block), _blocks(n_k, block))
    with _on_device(q.device, stream):
        m = torch.empty(shape, dtype=torch.uint8, device=q.device) if blockmap is None else blockmap
        if tuple(m.shape) != shape or m.dtype != torch.uint8 or not m.is_contiguous() or m.device != q.device:
            raise ValueError("blockmap must be a contiguous uint8 tensor %s on the queries' device" % (shape,))
        kept = torch.empty(shape[:3], dtype=torch.int32, device=q.device)
        L = _lib.lib()
        ws, nbytes, _keep = _workspace(workspace, int(L.psa_select_workspace_size(b, h, k.shape[1], d, n_q, n_k, block)), q.device)
        _lib.check(L.psa_select_blocks(_ptr(q), kv, b, h, d, n_q, n_k, block, keep, q_text, k_text,
                                       _ptr(m), _ptr(kept), ws, nbytes, _stream(None, q.device.index)))
    return m, kept


def attention_map_fwd(q, k, v, blockmap, block, scale=None, out=None, return_lse=False, workspace=None, stream=None):
    """Attention over the kept tiles of a block map (psa_attention_map_fwd).

    q: bfloat16 [batch, heads, N_q, head_dim], contiguous; k, v: [batch, kv heads, N_k, head_dim] with the same
    strides, each head's rows contiguous (a part of a longer cache; kv heads divide heads); blockmap: uint8 or bool
    [batch, heads, nbq, nbk], or [heads, nbq, nbk] for every batch element (build_blockmap's, select_blocks').

    Returns o like q (and lse float32 [batch, heads, N_q] if asked)."""
    torch = _torch()
    block = _int32(block, "block")
    _check_q(q)
    kv = _kv(q, k, v)
    b, h, n_q, d = q.shape
    n_k = k.shape[2]
    bm, bm_stride = _map_of(blockmap, q, n_k, block)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    with _on_device(q.device, stream):
        o = torch.empty_like(q) if out is None else out
        _check_q(o, "out", q)
        lse = torch.empty((b, h, n_q), dtype=torch.float32, device=q.device) if return_lse else None
        L = _lib.lib()
        ws, nbytes, _keep = _workspace(workspace, int(L.psa_attention_map_workspace_size(b, h, d, n_q, n_k, block)), q.device)
        _lib.check(L.psa_attention_map_fwd(_ptr(q), kv, _ptr(o), b, h, d, n_q, n_k, block, bm, bm_stride, scale,
                                           _ptr(lse), ws, nbytes, _stream(None, q.device.index)))
    return (o, lse) if return_lse else o


def attention_map_bwd(do, q, k, v, o, lse, blockmap, block, scale=None, dq=None, dk=None, dv=None, workspace=None,
                      stream=None):
    """Gradients of attention_map_fwd (psa_attention_map_bwd) from do, the gradient of o, and the forward's o and
    lse; the other arguments are the forward's.  Returns (dq, dk, dv), contiguous; those of a shared key head are
    the sums over its query heads."""
    torch = _torch()
    block = _int32(block, "block")
    _check_q(q)
    _check_q(do, "do", q)
    _check_q(o, "o", q)
    kv = _kv(q, k, v)
    b, h, n_q, d = q.shape
    n_k = k.shape[2]
    if lse.dtype != torch.float32 or tuple(lse.shape) != (b, h, n_q) or not lse.is_contiguous() or lse.device != q.device:
        raise ValueError("lse must be a contiguous float32 tensor [batch, heads, N_q] on the queries' device")
    bm, bm_stride = _map_of(blockmap, q, n_k, block)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    with _on_device(q.device, stream):
        dq = torch.empty_like(q) if dq is None else dq
        dk = _like(k, k.dtype) if dk is None else dk
        dv = _like(k, k.dtype) if dv is None else dv
        _check_q(dq, "dq", q)
        _check_q(dk, "dk", k)
        _check_q(dv, "dv", k)
        L = _lib.lib()
        ws, nbytes, _keep = _workspace(workspace, int(L.psa_attention_map_bwd_workspace_size(b, h, k.shape[1], d, n_q, n_k, block)), q.device)
        _lib.check(L.psa_attention_map_bwd(_ptr(do), _ptr(q), kv, _ptr(o), _ptr(lse), b, h, d, n_q, n_k, block, bm,
                                           bm_stride, scale, _ptr(dq), _ptr(dk), _ptr(dv), ws, nbytes,
                                           _stream(None, q.device.index)))
    return dq, dk, dv
