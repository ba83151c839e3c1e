"""ctypes binding of libmts's operators (include/mts_ops.h): what one serving
instance computes in a tick on the KV blocks that the scheduler accounts for.

    rope, rope_append   rotary positions; the new tokens' keys and values to their blocks
    attend              attention of tokens, drafted trees and prompt chunks over the blocks
    weigh, evict        accumulated attention weights, eviction of the least attended slots
    sample              the next token from logits and a given random number

Tensors live on one GPU and work is enqueued on its current stream.  Every
operator runs in the HIP kernels of libmts.so; nothing falls back to PyTorch.
A pool is [blocks][kv_heads][block_tokens][head_dim] by any strides whose last
one is 1, a block table [requests][width] int32, lens [requests] int32 (slots
of each request, its new tokens' among them) and q_start [requests + 1] int32
(first new token of each request).
"""
import ctypes

import torch

from . import mts
from .mts import _check

TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}

_vp, _u32, _i64, _f32, _f64 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_int64, ctypes.c_float, ctypes.c_double
_size = ctypes.c_size_t


class mts_pool(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp),
                ("k_block", _i64), ("k_head", _i64), ("k_token", _i64),
                ("v_block", _i64), ("v_head", _i64), ("v_token", _i64),
                ("n_blocks", _u32), ("block_tokens", _u32), ("kv_heads", _u32), ("head_dim", _u32),
                ("type", _u32), ("reserved", _u32)]


class mts_batch(ctypes.Structure):
    _fields_ = [("table", _vp), ("lens", _vp), ("q_start", _vp), ("tree", _vp),
                ("n", _u32), ("table_width", _u32), ("n_tokens", _u32), ("max_q", _u32),
                ("tree_words", _u32), ("reserved", _u32)]


class mts_rope_args(ctypes.Structure):
    _fields_ = [(k, _vp) for k in ("q", "k", "v", "q_out", "k_out")] + \
               [(k, _i64) for k in ("q_token", "q_head", "k_token", "k_head", "v_token", "v_head",
                                    "qo_token", "qo_head", "ko_token", "ko_head")] + \
               [(k, _vp) for k in ("positions", "freqs", "slots", "pos")] + \
               [("pool", mts_pool), ("n_tokens", _u32), ("q_heads", _u32), ("rot", _u32), ("layout", _u32),
                ("inverse", _u32), ("mscale", _f32)]


class mts_attend_args(ctypes.Structure):
    _fields_ = [("pool", mts_pool), ("batch", mts_batch), ("q", _vp), ("out", _vp), ("lse", _vp),
                ("q_token", _i64), ("q_head", _i64), ("out_token", _i64), ("out_head", _i64),
                ("q_heads", _u32), ("scale", _f32), ("workspace", _vp), ("workspace_bytes", _size)]


class mts_weigh_args(ctypes.Structure):
    _fields_ = [("pool", mts_pool), ("batch", mts_batch), ("q", _vp), ("lse", _vp),
                ("q_token", _i64), ("q_head", _i64), ("score", _vp),
                ("q_heads", _u32), ("scale", _f32), ("decay", _f32)]


class mts_evict_args(ctypes.Structure):
    _fields_ = [("pool", mts_pool), ("batch", mts_batch), ("score", _vp), ("pos", _vp), ("next_pos", _vp),
                ("score_out", _vp), ("pos_out", _vp), ("lens_out", _vp),
                ("budget", _u32), ("recent", _u32), ("sink", _u32), ("reserved", _u32),
                ("workspace", _vp), ("workspace_bytes", _size)]


class mts_sample_args(ctypes.Structure):
    _fields_ = [("logits", _vp), ("row_stride", _i64)] + \
               [(k, _vp) for k in ("u", "temperature", "top_k", "top_p", "min_p", "token", "logprob")] + \
               [("rows", _u32), ("vocab", _u32), ("type", _u32), ("reserved", _u32)]


EXPORTED = ("mts_rope", "mts_rope_freqs", "mts_attend", "mts_attend_workspace", "mts_weigh", "mts_evict",
            "mts_evict_workspace", "mts_sample")

_lib = None


def _library():
    global _lib
    if _lib is None:
        L = mts.load_library()
        for name, args in (("mts_rope", mts_rope_args), ("mts_attend", mts_attend_args), ("mts_weigh", mts_weigh_args),
                           ("mts_evict", mts_evict_args), ("mts_sample", mts_sample_args)):
            getattr(L, name).argtypes = [ctypes.POINTER(args), _vp]
        L.mts_rope_freqs.argtypes = [_vp, _u32, _f64, _u32, _f64, _f64, _f64, _f64]
        L.mts_attend_workspace.argtypes = [_u32] * 6 + [ctypes.POINTER(_size)]
        L.mts_evict_workspace.argtypes = [_u32] * 5 + [ctypes.POINTER(_size)]
        for name in EXPORTED:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _device(t, what, device, dtype, shape=None):
    """A contiguous tensor of one type on the call's GPU."""
    _need(t.device == device and t.dtype == dtype and t.is_contiguous(), "%s: contiguous %s on %s" % (what, dtype, device))
    _need(shape is None or t.shape == shape, "%s: shape %s, got %s" % (what, shape, tuple(t.shape)))


def _rows(t, what, device, dtype):
    """[tokens][heads][dim] with the last dimension contiguous: (token, head) strides."""
    _need(t.dim() == 3 and t.device == device and t.dtype == dtype and (t.stride(2) == 1 or t.shape[2] == 1),
          "%s: [tokens][heads][dim] of %s on %s, last dimension contiguous" % (what, dtype, device))
    return t.stride(0), t.stride(1)


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


def _fill_pool(P, k_cache, v_cache):
    c = k_cache
    _need(c.dim() == 4 and c.stride(3) == 1 and c.dtype in TYPES, "a pool is [blocks][kv_heads][block_tokens][head_dim]")
    P.k = c.data_ptr()
    P.k_block, P.k_head, P.k_token = c.stride()[:3]
    if v_cache is not None:
        _need(v_cache.shape == c.shape and v_cache.dtype == c.dtype and v_cache.device == c.device and v_cache.stride(3) == 1,
              "v_cache must match k_cache")
        P.v = v_cache.data_ptr()
        P.v_block, P.v_head, P.v_token = v_cache.stride()[:3]
    P.n_blocks, P.kv_heads, P.block_tokens, P.head_dim = c.shape
    P.type = TYPES[c.dtype]


def _fill_batch(B, device, table, lens, q_start=None, n_tokens=0, max_q=0, tree=None):
    n = lens.shape[0]
    _need(table.dim() == 2 and table.shape[0] == n, "table: [requests][width]")
    _device(table, "table", device, torch.int32)
    _device(lens, "lens", device, torch.int32, (n,))
    B.table, B.lens, B.n, B.table_width = table.data_ptr(), lens.data_ptr(), n, table.shape[1]
    if q_start is not None:
        _device(q_start, "q_start", device, torch.int32, (n + 1,))
        B.q_start, B.n_tokens, B.max_q = q_start.data_ptr(), n_tokens, max_q
    if tree is not None:
        _need(tree.dim() == 2 and tree.shape[0] == n_tokens, "tree: [tokens][words] int64")
        _device(tree, "tree", device, torch.int64)
        B.tree, B.tree_words = tree.data_ptr(), tree.shape[1]


def _call(name, args, device):
    _need(device.type == "cuda", "tensors must be on a GPU")
    # the launch goes to the tensors' GPU, whatever the current one is
    if device.index == torch.cuda.current_device():
        _check(name, getattr(_library(), name)(ctypes.byref(args), _stream(device)))
    else:
        with torch.cuda.device(device):
            _check(name, getattr(_library(), name)(ctypes.byref(args), _stream(device)))


# ------------------------------------------------------------------ rotary positions


def rope_freqs(rot, base=10000.0, scaling="none", factor=1.0, trained=4096.0, fast=32.0, slow=1.0, device="cuda"):
    """Angles in radians per position of the rot / 2 pairs, float64 (mts_rope_freqs)."""
    f = torch.empty(rot // 2, dtype=torch.float64)
    _check("mts_rope_freqs", _library().mts_rope_freqs(f.data_ptr(), rot, base, SCALINGS[scaling], factor, trained, fast, slow))
    return f.to(device)


def _rope_args(q, k, positions, freqs, layout, mscale, inverse):
    a = mts_rope_args()
    any_ = q if q is not None else k
    _need(any_ is not None, "q or k")
    device, dtype = any_.device, any_.dtype
    _need(dtype in TYPES, "bfloat16, float16 or float32")
    n, D = any_.shape[0], any_.shape[2]
    for x, what in ((q, "q"), (k, "k")):
        if x is not None:
            t, h = _rows(x, what, device, dtype)
            _need(x.shape[0] == n and x.shape[2] == D, "q and k differ in tokens or head dimension")
            setattr(a, what, x.data_ptr())
            setattr(a, what + "_token", t)
            setattr(a, what + "_head", h)
    _device(positions, "positions", device, torch.int32, (n,))
    _device(freqs, "freqs", device, torch.float64)
    _need(freqs.dim() == 1, "freqs: [rot / 2]")
    a.positions, a.freqs = positions.data_ptr(), freqs.data_ptr()
    a.n_tokens, a.q_heads, a.rot = n, 0 if q is None else q.shape[1], 2 * freqs.shape[0]
    a.layout, a.inverse, a.mscale = LAYOUTS[layout], 1 if inverse else 0, mscale
    a.pool.type, a.pool.head_dim, a.pool.kv_heads = TYPES[dtype], D, 0 if k is None else k.shape[1]
    return a, device, dtype


def _out(x, out, what, a, device, dtype):
    if x is None:
        return None
    if out is None:
        out = torch.empty(x.shape, dtype=dtype, device=device)
    t, h = _rows(out, what + "_out", device, dtype)
    _need(out.shape == x.shape, "%s_out: the shape of %s" % (what, what))
    setattr(a, what + "_out", out.data_ptr())
    setattr(a, what + "o_token", t)
    setattr(a, what + "o_head", h)
    return out


def rope(q, k, positions, freqs, *, layout="half", mscale=1.0, inverse=False, q_out=None, k_out=None):
    """Queries and keys ([tokens][heads][dim], either may be None) turned by
    their positions; returns (q_out, k_out).  inverse turns back, which is
    also the gradient's rotation."""
    a, device, dtype = _rope_args(q, k, positions, freqs, layout, mscale, inverse)
    q_out = _out(q, q_out, "q", a, device, dtype)
    k_out = _out(k, k_out, "k", a, device, dtype)
    _call("mts_rope", a, device)
    return q_out, k_out


def rope_append(q, k, v, positions, slots, freqs, k_cache, v_cache, pos=None, *, layout="half", mscale=1.0, q_out=None):
    """rope() whose keys go to the pool's slots (block * block_tokens + offset,
    int64; -1: nowhere) together with the values and, to pos
    [blocks][kv_heads][block_tokens] int32, the positions; returns q_out."""
    a, device, dtype = _rope_args(q, k, positions, freqs, layout, mscale, False)
    q_out = _out(q, q_out, "q", a, device, dtype)
    _fill_pool(a.pool, k_cache, v_cache)
    _need(k is not None and k_cache.device == device and k_cache.dtype == dtype and k_cache.shape[3] == k.shape[2]
          and k_cache.shape[1] == k.shape[1], "k and the pool differ in heads, head dimension, type or device")
    if v is not None:
        _need(v.shape == k.shape and v_cache is not None, "v: the shape of k")
        a.v, (a.v_token, a.v_head) = v.data_ptr(), _rows(v, "v", device, dtype)
    _device(slots, "slots", device, torch.int64, (k.shape[0],))
    a.slots = slots.data_ptr()
    if pos is not None:
        _device(pos, "pos", device, torch.int32, k_cache.shape[:3])
        a.pos = pos.data_ptr()
    _call("mts_rope", a, device)
    return q_out


# ------------------------------------------------------------------ attention

_workspaces = {}


def _zeroed(device, nbytes):
    """The stream's zero-initialised workspace, grown as needed.  Under graph
    capture a new one from the graph's own memory."""
    _need(device.type == "cuda", "tensors must be on a GPU")
    if torch.cuda.is_current_stream_capturing():
        return torch.zeros(nbytes, dtype=torch.uint8, device=device)
    key = (device.index, _stream(device))
    w = _workspaces.get(key)
    if w is None or w.numel() < nbytes:
        w = _workspaces[key] = torch.zeros(max(nbytes, 1 << 20), dtype=torch.uint8, device=device)
    return w


def attend_workspace(n, n_tokens, max_q, q_heads, kv_heads, head_dim):
    """Bytes of a workspace for attend() calls of at most these sizes."""
    b = _size(0)
    _check("mts_attend_workspace", _library().mts_attend_workspace(n, n_tokens, max_q, q_heads, kv_heads, head_dim, ctypes.byref(b)))
    return b.value


def attend(q, k_cache, v_cache, table, lens, q_start, max_q, *, scale=None, tree=None, out=None, lse=None, workspace=None):
    """Attention of the new tokens q [tokens][q_heads][dim] over their requests'
    slots; returns (out, lse [tokens][q_heads] float32).  max_q bounds the new
    tokens of a request.  tree [tokens][words] int64: bit i of a token says
    whether it attends its request's i-th new token; without it new tokens
    attend those before them and themselves.  scale: dim ** -0.5 by default.
    workspace: a zeroed uint8 tensor of attend_workspace() bytes kept for one
    stream's calls; by default the module keeps one a stream."""
    a = mts_attend_args()
    device, dtype = q.device, q.dtype
    a.q_token, a.q_head = _rows(q, "q", device, dtype)
    N, Hq, D = q.shape
    _fill_pool(a.pool, k_cache, v_cache)
    _need(k_cache.device == device and k_cache.dtype == dtype and k_cache.shape[3] == D, "q and the pool differ in head dimension, type or device")
    _fill_batch(a.batch, device, table, lens, q_start, N, max_q, tree)
    if out is None:
        out = torch.empty((N, Hq, D), dtype=dtype, device=device)
    a.out_token, a.out_head = _rows(out, "out", device, dtype)
    _need(out.shape == q.shape, "out: the shape of q")
    if lse is None:
        lse = torch.empty((N, Hq), dtype=torch.float32, device=device)
    _device(lse, "lse", device, torch.float32, (N, Hq))
    a.q, a.out, a.lse, a.q_heads = q.data_ptr(), out.data_ptr(), lse.data_ptr(), Hq
    a.scale = D ** -0.5 if scale is None else scale
    if workspace is None:
        workspace = _zeroed(device, attend_workspace(a.batch.n, N, max_q, Hq, k_cache.shape[1], D))
    _need(workspace.device == device and workspace.dtype == torch.uint8 and workspace.is_contiguous(), "workspace: uint8 on %s" % device)
    a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
    _call("mts_attend", a, device)
    return out, lse


# ------------------------------------------------------------------ eviction


def weigh(q, lse, k_cache, table, lens, q_start, max_q, score, *, scale=None, decay=1.0, tree=None):
    """Adds to score [blocks][kv_heads][block_tokens] float32 (times decay) the
    softmax weights that every slot gets from the new tokens' queries, lse being
    attend()'s; returns score.  The new tokens' own slots start from zero."""
    a = mts_weigh_args()
    device, dtype = q.device, q.dtype
    a.q_token, a.q_head = _rows(q, "q", device, dtype)
    N, Hq, D = q.shape
    _fill_pool(a.pool, k_cache, None)
    _need(k_cache.device == device and k_cache.dtype == dtype and k_cache.shape[3] == D, "q and the pool differ in head dimension, type or device")
    _fill_batch(a.batch, device, table, lens, q_start, N, max_q, tree)
    _device(lse, "lse", device, torch.float32, (N, Hq))
    _device(score, "score", device, torch.float32, k_cache.shape[:3])
    a.q, a.lse, a.score, a.q_heads = q.data_ptr(), lse.data_ptr(), score.data_ptr(), Hq
    a.scale, a.decay = D ** -0.5 if scale is None else scale, decay
    _call("mts_weigh", a, device)
    return score


def evict(k_cache, v_cache, score, pos, table, lens, next_pos, budget, *, recent=0, sink=0, score_out=None, pos_out=None,
          lens_out=None):
    """Requests longer than budget keep, head by head, that many slots: the
    first `sink` and last `recent` positions, then the largest scores.  Kept
    rows above the budget move into the holes below it, in the pool, score_out
    and pos_out (by default score and pos themselves); returns the new lens."""
    a = mts_evict_args()
    device = k_cache.device
    _fill_pool(a.pool, k_cache, v_cache)
    _need(v_cache is not None, "v_cache")
    _fill_batch(a.batch, device, table, lens)
    n, shape = lens.shape[0], k_cache.shape[:3]
    score_out = score if score_out is None else score_out
    pos_out = pos if pos_out is None else pos_out
    for t, what, dt in ((score, "score", torch.float32), (score_out, "score_out", torch.float32), (pos, "pos", torch.int32),
                        (pos_out, "pos_out", torch.int32)):
        _device(t, what, device, dt, shape)
    _device(next_pos, "next_pos", device, torch.int32, (n,))
    if lens_out is None:
        lens_out = torch.empty(n, dtype=torch.int32, device=device)
    _device(lens_out, "lens_out", device, torch.int32, (n,))
    b = _size(0)
    _check("mts_evict_workspace", _library().mts_evict_workspace(n, shape[1], table.shape[1], shape[2], budget, ctypes.byref(b)))
    workspace = torch.empty(b.value, dtype=torch.uint8, device=device)
    a.score, a.pos, a.next_pos = score.data_ptr(), pos.data_ptr(), next_pos.data_ptr()
    a.score_out, a.pos_out, a.lens_out = score_out.data_ptr(), pos_out.data_ptr(), lens_out.data_ptr()
    a.budget, a.recent, a.sink = budget, recent, sink
    a.workspace, a.workspace_bytes = workspace.data_ptr(), b.value
    _call("mts_evict", a, device)
    return lens_out


# ------------------------------------------------------------------ sampling


def sample(logits, u, temperature, top_k, top_p, min_p, *, token=None, logprob=None):
    """The next token of every row of logits [rows][vocab] from uniform numbers
    u [rows]; returns (token int32, logprob float32).  temperature 0 is greedy;
    top_k 0, top_p 1 and min_p 0 keep everything.  A row without a logit above
    -inf gives token -1."""
    _need(logits.dim() == 2 and logits.dtype in TYPES and (logits.stride(1) == 1 or logits.shape[1] == 1),
          "logits: [rows][vocab], rows contiguous")
    device, rows = logits.device, logits.shape[0]
    a = mts_sample_args()
    for t, what, dt in ((u, "u", torch.float32), (temperature, "temperature", torch.float32), (top_k, "top_k", torch.int32),
                        (top_p, "top_p", torch.float32), (min_p, "min_p", torch.float32)):
        _device(t, what, device, dt, (rows,))
        setattr(a, what, t.data_ptr())
    if token is None:
        token = torch.empty(rows, dtype=torch.int32, device=device)
    if logprob is None:
        logprob = torch.empty(rows, dtype=torch.float32, device=device)
    _device(token, "token", device, torch.int32, (rows,))
    _device(logprob, "logprob", device, torch.float32, (rows,))
    a.logits, a.row_stride, a.rows, a.vocab, a.type = logits.data_ptr(), logits.stride(0), rows, logits.shape[1], TYPES[logits.dtype]
    a.token, a.logprob = token.data_ptr(), logprob.data_ptr()
    _call("mts_sample", a, device)
    return token, logprob
