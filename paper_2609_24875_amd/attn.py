"""Rotary positions, the paged key-value cache and its attention (include/sph.h): argument
marshalling only, as in ``sph``. ``stream``: the call runs as it would under ``torch.cuda.stream(stream)``, to which the
tensors that it returns then belong.

A decoder block runs ``gemm`` (fused q/k/v), ``kv_append`` (rotates keys and queries and writes the
cache), ``attention`` and ``gemm`` (o); ``block.AttentionBlock`` does so. The cache's pages are plain
torch tensors that the caller may hold, copy and share between layers' handles.
"""
from __future__ import annotations

import ctypes
import math

import numpy as np

from .sph import SPH_F16, SPH_F32, _check, _stream_handle, load_library

ROPE_INTERLEAVED, ROPE_INVERSE = 1, 2
KV_BITS = (16, 8, 4)
KV_HEAD_DIMS = (64, 96, 128, 192, 256)
SPH_ERR_NULL, SPH_ERR_BUFFER_TOO_SMALL = 1, 6
KV_GROUP = 32                       # channels that share an offset and a step


class CRope(ctypes.Structure):
    _fields_ = [("d_table", ctypes.c_void_p), ("max_pos", ctypes.c_int64), ("rot_dim", ctypes.c_int32),
                ("flags", ctypes.c_int32)]


class CKVCache(ctypes.Structure):
    _fields_ = [("bits", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int64), ("d_k", ctypes.c_void_p),
                ("d_v", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("d_k_par", ctypes.c_void_p), ("d_v_par", ctypes.c_void_p),
                ("par_page_stride", ctypes.c_int64), ("par_head_stride", ctypes.c_int64),
                ("par_token_stride", ctypes.c_int64)]


_declared = None


def _library():
    global _declared
    if _declared is None:
        lib = load_library()
        P, I64, SZ, I32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int32
        pr, pc = ctypes.POINTER(CRope), ctypes.POINTER(CKVCache)
        lib.sph_rope_table.argtypes = [I32, I64, ctypes.POINTER(ctypes.c_double), ctypes.c_double, P, P]
        lib.sph_rope.argtypes = [pr, I32, I64, I32, I32, P, I64, I64, P, P, I64, I64, P]
        lib.sph_kv_append.argtypes = [pc, pr, I32, I64, P, I64, I64, P, I64, I64, P, I32, P, I64, I64, P, I64, I64, P, P]
        lib.sph_kv_read.argtypes = [pc, I64, P, P, P, P]
        lib.sph_attention.argtypes = [pc, I64, I64, I32, P, I64, I64, P, I64, P, I64, P, I64, I64, ctypes.c_float,
                                      P, I64, I64, P, P, SZ, P]
        lib.sph_attention_workspace_bytes.argtypes = [pc, I64, I64, I32, I64, I64, I64, ctypes.POINTER(SZ)]
        for name in ("sph_rope_table", "sph_rope", "sph_kv_append", "sph_kv_read", "sph_attention",
                     "sph_attention_workspace_bytes"):
            getattr(lib, name).restype = ctypes.c_int
        _declared = lib
    return _declared


# ------------------------------------------------------------------ rotary positions

def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     original_max_pos: int = 4096, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(angle per position of each pair, fp64 [rot_dim/2]; common factor of cos and sin).

    base^(-2i/rot_dim), for longer contexts than a model was trained on scaled by one of
    "linear"  every frequency divided by ``factor``;
    "ntk"     the base grown by factor^(rot_dim/(rot_dim-2)), which leaves the fastest pair and divides the
              slowest by ``factor``;
    "yarn"    pairs that turn more than ``beta_fast`` times over ``original_max_pos`` tokens kept, those
              with fewer than ``beta_slow`` turns divided by ``factor``, a linear ramp over the pair index between, and cos and sin times
              0.1 ln(factor) + 1.
    """
    if rot_dim < 16 or rot_dim % 16 or not base > 1.0 or not factor >= 1.0:
        raise ValueError("rot_dim must be a positive multiple of 16, base above 1, factor at least 1")
    i = np.arange(rot_dim // 2, dtype=np.float64)
    if scaling == "ntk":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = base ** (-2.0 * i / rot_dim)
    if scaling in ("none", "ntk"):
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":
        # the pair that makes `turns` turns over the original context
        def pair(turns):
            return rot_dim * math.log(original_max_pos / (turns * 2.0 * math.pi)) / (2.0 * math.log(base))
        # (the slow end may lie behind the last pair, which then stops short of the whole factor)
        lo, hi = max(math.floor(pair(beta_fast)), 0), min(math.ceil(pair(beta_slow)), rot_dim - 1)
        keep = 1.0 - np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    raise ValueError(f"scaling must be none, linear, ntk or yarn, not {scaling!r}")


def rope_table(rot_dim: int, max_pos: int, device="cuda", stream=None, **scaling):
    """fp32 [max_pos][rot_dim/2][2] of (cos, sin) (sph_rope_table); keywords as ``rope_frequencies``."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return rope_table(rot_dim, max_pos, device, **scaling)
    f, magnitude = rope_frequencies(rot_dim, **scaling)
    out = torch.empty((max_pos, rot_dim // 2, 2), dtype=torch.float32, device=device)
    _on_gpu(out)
    arr = (ctypes.c_double * len(f))(*f)
    _check(_library().sph_rope_table(rot_dim, max_pos, arr, magnitude, out.data_ptr(), _stream_handle()), "sph_rope_table")
    return out


def _ints(t, name: str, device, count: int | None = None):
    import torch
    if isinstance(t, torch.Tensor) and t.dtype is torch.int32 and t.device == device and t.dim() == 1 and t.is_contiguous() and \
            (count is None or t.shape[0] == count):
        return t.data_ptr()
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32:
        raise TypeError(f"{name} must be a torch.int32 tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the rows on {device}")
    raise ValueError(f"{name} must be contiguous [{'n' if count is None else count}], got shape {tuple(t.shape)} and strides {tuple(t.stride())}")


def _rows(t, name: str, device, dtypes, shape=None):
    """Checks [tokens][heads][channels] rows with unit channel stride; (pointer, token stride, head stride)."""
    import torch
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and (device is None or t.device == device):
        sh = t.shape
        if len(sh) == 3 and (shape is None or sh == shape):
            s0, s1, s2 = t.stride()
            if s2 == 1 or sh[2] <= 1 or t.numel() == 0:
                # the stride of a dimension of one element is never used and may hold anything
                return t.data_ptr(), s0 if sh[0] > 1 else 0, s1 if sh[1] > 1 else 0
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise TypeError(f"{name} must be a tensor of {' or '.join(str(d) for d in dtypes)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    raise ValueError(f"{name} must be {list(shape) if shape else '[tokens][heads][channels]'} with unit channel stride, got "
                     f"shape {tuple(t.shape)} and strides {tuple(t.stride())}")


def _rope_desc(table, device, interleaved: bool, inverse: bool) -> CRope:
    import torch
    if not isinstance(table, torch.Tensor) or table.dtype is not torch.float32:
        raise TypeError("table must be a torch.float32 tensor")
    if table.device != device:
        raise ValueError(f"table is on {table.device}, the rows on {device}")
    n, pairs, two = table.shape if table.dim() == 3 else (0, 0, 0)
    if two != 2 or not table.is_contiguous():
        raise ValueError(f"table must be contiguous [positions][pairs][2], got shape {tuple(table.shape)}")
    return CRope(table.data_ptr(), n, 2 * pairs,
                 (ROPE_INTERLEAVED if interleaved else 0) | (ROPE_INVERSE if inverse else 0))


def _on_gpu(t):
    import torch
    if not t.is_cuda:
        raise ValueError(f"tensors must be on a GPU, not on {t.device}")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"tensors are on {t.device}, the current device is cuda:{torch.cuda.current_device()}")


def _new(x):
    """A contiguous tensor like x (``empty_like`` takes half of ``empty``'s time)."""
    import torch
    return torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)


def aligned_rows(t):
    """``t`` itself where its rows suit the library (unit channel stride, 16-byte aligned, no broadcast), else a copy: what
    autograd hands a backward pass may be any view."""
    per = 16 // t.element_size()
    if t.is_contiguous() and t.shape[-1] % per == 0:
        return t if t.data_ptr() % 16 == 0 else t.clone()
    ok = t.stride(-1) == 1 and t.data_ptr() % 16 == 0 and all(t.stride(d) % per == 0 for d in range(t.dim() - 1) if t.shape[d] > 1)
    return t if ok else t.contiguous()


def rope(x, positions, table, interleaved: bool = False, inverse: bool = False, out=None, stream=None):
    """Rotary positions of device rows x[tokens][heads][channels], fp16 or fp32 (sph_rope): the first
    2 * table.shape[1] channels of each row turn by the angles of its token's position, the others are
    copied. ``inverse`` turns back and is the gradient (``train.rope`` is the differentiable form).
    ``out`` may be x."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return rope(x, positions, table, interleaved, inverse, out)
    half = (torch.float16, torch.float32)
    px, xt, xh = _rows(x, "x", None, half)
    dev, n = x.device, x.shape[0]
    desc = _rope_desc(table, dev, interleaved, inverse)
    pos = _ints(positions, "positions", dev, n)
    out = _new(x) if out is None else out
    py, yt, yh = _rows(out, "out", dev, (x.dtype,), x.shape)
    _on_gpu(x)
    st = _library().sph_rope(ctypes.byref(desc), SPH_F16 if x.dtype is torch.float16 else SPH_F32, n, x.shape[1], x.shape[2],
                             px, xt, xh, pos, py, yt, yh, _stream_handle())
    _check(st, "sph_rope")
    return out


def rope_gradient(grad, positions, table, interleaved: bool, inverse: bool = False):
    """The gradient of ``rope``'s rows from that of its result, whose tensors have passed ``rope``'s checks: they are not repeated, since
    Python on autograd's thread costs several times what it does elsewhere."""
    grad = aligned_rows(grad)
    n, heads, dim = grad.shape
    gt, gh, _ = grad.stride()
    out = _new(grad)
    desc = CRope(table.data_ptr(), table.shape[0], 2 * table.shape[1],
                 (ROPE_INTERLEAVED if interleaved else 0) | (0 if inverse else ROPE_INVERSE))
    st = _library().sph_rope(ctypes.byref(desc), SPH_F16 if grad.element_size() == 2 else SPH_F32, n, heads, dim, grad.data_ptr(),
                             gt if n > 1 else 0, gh if heads > 1 else 0, positions.data_ptr(), out.data_ptr(), heads * dim, dim,
                             _stream_handle())
    _check(st, "sph_rope")
    return out


# ------------------------------------------------------------------ the cache

class KVCache:
    """A paged key-value cache over caller-owned tensors (sph_kv_cache): ``k`` and ``v``
    [pages][kv heads][tokens a page][channels], fp16 with ``bits`` 16; with 8 or 4 bits uint8 codes
    ([..][channels * bits / 8]) and ``k_par``, ``v_par`` fp16 [pages][kv heads][tokens a page][channels / 32][2]
    of (offset, step). Any strides of the first three dimensions that keep rows 16-byte aligned and are the
    same for keys and values, so both may be views of one allocation or of another order. The handle keeps the
    attention's workspaces (``attention_workspace_bytes``: a few MB for decode steps, tens for drafts behind long caches), one a stream,
    and those that larger calls have outgrown; calls that a graph captures (``torch.cuda.graph``)
    have theirs in the graph's memory pool, so that its replays need no order with other calls' or other graphs'."""

    def __init__(self, k, v, k_par=None, v_par=None, bits: int = 16):
        import torch
        if bits not in KV_BITS:
            raise ValueError(f"bits must be one of {KV_BITS}")
        want = torch.float16 if bits == 16 else torch.uint8
        for t, name in ((k, "k"), (v, "v")):
            if not isinstance(t, torch.Tensor) or t.dtype != want:
                raise TypeError(f"{name} must be a {want} tensor for {bits} bits")
            if t.dim() != 4 or t.stride(3) != 1:
                raise ValueError(f"{name} must be [pages][kv heads][tokens a page][channels] with unit channel stride")
        strides = self._strides(k, k.element_size())
        if v.shape != k.shape or v.device != k.device or self._strides(v, v.element_size()) != strides:
            raise ValueError("k and v must have the same shape, device and strides")
        pages, heads, page, width = k.shape
        dim = width * 8 // bits if bits < 16 else width
        par = (0, 0, 0)
        if bits < 16:
            for t, name in ((k_par, "k_par"), (v_par, "v_par")):
                if not isinstance(t, torch.Tensor) or t.dtype != torch.float16:
                    raise TypeError(f"{name} must be a torch.float16 tensor for {bits} bits")
                if tuple(t.shape) != (pages, heads, page, dim // KV_GROUP, 2) or t.device != k.device or t.stride(4) != 1 or \
                        (t.shape[3] > 1 and t.stride(3) != 2):
                    raise ValueError(f"{name} must be [{pages}][{heads}][{page}][{dim // KV_GROUP}][2] on {k.device} with contiguous pairs")
            par = self._strides(k_par, 2)
            if self._strides(v_par, 2) != par:
                raise ValueError("k_par and v_par must have the same strides")
        elif k_par is not None or v_par is not None:
            raise ValueError("a 16-bit cache has no offsets and steps")
        self.k, self.v, self.k_par, self.v_par = k, v, k_par, v_par
        self.bits, self.n_pages, self.kv_heads, self.page_size, self.head_dim = bits, pages, heads, page, dim
        self.device = k.device
        self.workspaces, self.outgrown = {}, []
        self.desc = CKVCache(bits, heads, dim, page, pages, k.data_ptr(), v.data_ptr(), *strides,
                             k_par.data_ptr() if bits < 16 else None, v_par.data_ptr() if bits < 16 else None, *par)
        self._ref = ctypes.byref(self.desc)

    @staticmethod
    def _strides(t, size: int):
        # a dimension of one element may carry any stride: the library is told what a contiguous one would have
        got, inner = [], t.shape[3] * size * (t.shape[4] if t.dim() == 5 else 1)
        for d in (2, 1, 0):
            st = t.stride(d) * size if t.shape[d] > 1 else inner
            got.append(st)
            inner = max(inner, st * t.shape[d])
        return tuple(reversed(got))

    @classmethod
    def empty(cls, n_pages: int, kv_heads: int, head_dim: int, page_size: int = 64, bits: int = 16, device="cuda"):
        """A cache over new tensors (uninitialised: slots are written before they are read)."""
        import torch
        if bits not in KV_BITS or head_dim not in KV_HEAD_DIMS:
            raise ValueError(f"bits must be one of {KV_BITS}, head_dim one of {KV_HEAD_DIMS}")
        shape = (n_pages, kv_heads, page_size)
        if bits == 16:
            return cls(*(torch.empty((*shape, head_dim), dtype=torch.float16, device=device) for _ in range(2)))
        codes = [torch.empty((*shape, head_dim * bits // 8), dtype=torch.uint8, device=device) for _ in range(2)]
        par = [torch.empty((*shape, head_dim // KV_GROUP, 2), dtype=torch.float16, device=device) for _ in range(2)]
        return cls(*codes, *par, bits=bits)

    @property
    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.k, self.v, self.k_par, self.v_par) if t is not None)


def kv_append(cache: KVCache, k, v, slots, positions=None, table=None, interleaved: bool = False, q=None, q_out=None, stream=None):
    """Write a key and a value row per token and head, k and v [tokens][kv heads][channels] (fp16 or fp32,
    any row strides), to the int32 ``slots`` (sph_kv_append; page * page_size + place in the page, -1 for a padding token). With
    ``table`` and ``positions`` the keys are rotated on the way, and so are the queries q [tokens][q heads][channels] in
    the same launch. Returns the rotated queries in fp16 (``q_out`` or a new tensor; None without q)."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return kv_append(cache, k, v, slots, positions, table, interleaved, q, q_out)
    dev = cache.device
    dt = (k.dtype,) if isinstance(k, torch.Tensor) and k.dtype is torch.float16 else (torch.float32,)
    n = k.shape[0] if isinstance(k, torch.Tensor) and k.dim() else 0
    shape = (n, cache.kv_heads, cache.head_dim)
    pk, kt, kh = _rows(k, "k", dev, dt, shape)
    pv, vt, vh = _rows(v, "v", dev, dt, shape)
    ps = _ints(slots, "slots", dev, n)
    desc = pos = None
    if table is not None:
        desc = ctypes.byref(_rope_desc(table, dev, interleaved, False))
        pos = _ints(positions, "positions", dev, n)
    elif positions is not None or q is not None:
        raise ValueError("positions and q need a table")
    pq = po = None
    heads = qt = qh = ot = oh = 0
    if q is not None:
        heads = q.shape[1] if q.dim() == 3 else 0
        shape = (n, heads, cache.head_dim)
        pq, qt, qh = _rows(q, "q", dev, dt, shape)
        if q_out is None:
            q_out = torch.empty(shape, dtype=torch.float16, device=dev)
        po, ot, oh = _rows(q_out, "q_out", dev, (torch.float16,), shape)
    _on_gpu(k)
    st = _library().sph_kv_append(cache._ref, desc, SPH_F16 if dt[0] is torch.float16 else SPH_F32, n, pk, kt, kh, pv, vt, vh, ps,
                                  heads, pq, qt, qh, po, ot, oh, pos, _stream_handle())
    _check(st, "sph_kv_append")
    return q_out if q is not None else None


def kv_read(cache: KVCache, slots, out=None, stream=None):
    """The keys and values of int32 ``slots`` as two fp16 tensors [tokens][kv heads][channels]
    (sph_kv_read); rows of slots outside the pool are zero. ``out``: a pair of contiguous tensors."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return kv_read(cache, slots, out)
    dev = cache.device
    ps = _ints(slots, "slots", dev)
    shape = (slots.shape[0], cache.kv_heads, cache.head_dim)
    if out is None:
        k = torch.empty(shape, dtype=torch.float16, device=dev)
        v = torch.empty_like(k)
    else:
        k, v = out
        for t in out:
            if t.dtype != torch.float16 or t.device != dev or t.shape != shape or not t.is_contiguous():
                raise ValueError(f"out must be two contiguous fp16 tensors of shape {shape} on {dev}")
    _on_gpu(slots)
    _check(_library().sph_kv_read(cache._ref, shape[0], ps, k.data_ptr(), v.data_ptr(), _stream_handle()), "sph_kv_read")
    return k, v


# ------------------------------------------------------------------ attention

def attention_workspace_bytes(cache: KVCache, batch: int, tokens: int, q_heads: int, max_q: int, max_len: int, window: int = 0) -> int:
    out = ctypes.c_size_t(0)
    _check(_library().sph_attention_workspace_bytes(cache._ref, batch, tokens, q_heads, max_q, max_len, window, ctypes.byref(out)),
           "sph_attention_workspace_bytes")
    return out.value


def _attention_workspace(cache: KVCache, need: int, handle: int):
    """A workspace of at least ``need`` bytes for calls on the current stream, ``handle``, kept with the cache; streams do not share
    one, since their calls may run together. One that a larger call outgrows is kept, and its successor is twice its size or more: all of
    them together take less than twice the last."""
    import torch
    if torch.cuda.is_current_stream_capturing():
        # memory of the graph's own pool must not serve later calls outside it
        raise RuntimeError("no workspace of this size on this stream yet: make one call on the capture stream before "
                           "capturing a graph")
    old = cache.workspaces.get(handle)
    ws = torch.empty(need if old is None else max(need, 2 * old.numel()), dtype=torch.uint8, device=cache.device)
    if old is not None:
        cache.outgrown.append(old)
    cache.workspaces[handle] = ws
    return ws


def attention(q, cache: KVCache, pages, seq_lens, q_start=None, max_q: int = 1, max_len: int | None = None, window: int = 0,
              scale: float | None = None, out=None, return_lse: bool = False, stream=None):
    """Attention of new tokens over a cache that already holds their keys and values (sph_attention).

    q: fp16 [tokens][q heads][channels] (rotated). pages: int32 [batch][columns], the pages of every sequence in
    order. seq_lens: int32 [batch], tokens in the cache with the new ones. Sequence b asks with its last
    q_start[b+1] - q_start[b] tokens (at most ``max_q``), or without q_start with its last one. A query sees the tokens up to its
    own, with ``window`` only the last ``window`` of them. max_len: bound of the lengths that the launch is planned for
    (default: what the pages' columns hold). scale: default channels^-0.5. Returns fp16 o like q, with ``return_lse`` also fp32
    [tokens][q heads], the logarithm of each softmax's sum."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return attention(q, cache, pages, seq_lens, q_start, max_q, max_len, window, scale, out, return_lse)
    dev, half = cache.device, (torch.float16,)
    pq, qt, qh = _rows(q, "q", dev, half)
    n, heads, dim = q.shape
    if dim != cache.head_dim:
        raise ValueError(f"q has {dim} channels a head, the cache {cache.head_dim}")
    if not isinstance(pages, torch.Tensor) or pages.dtype is not torch.int32:
        raise TypeError("pages must be a torch.int32 tensor")
    batch, cols = pages.shape if pages.dim() == 2 else (-1, 0)
    if batch < 0 or pages.device != dev or (cols > 1 and batch > 0 and pages.stride(1) != 1):
        raise ValueError(f"pages must be [batch][columns] on {dev} with unit stride along the columns")
    lens = _ints(seq_lens, "seq_lens", dev, batch)
    start = None if q_start is None else _ints(q_start, "q_start", dev, batch + 1)
    held = cols * cache.page_size
    if max_len is None:
        max_len = held
    elif max_len > held:
        raise ValueError(f"max_len {max_len} is more than the {cols} columns of pages hold")
    row = pages.stride(0) if batch > 1 else cols
    if row < cols:
        raise ValueError("rows of pages must not overlap")
    if out is None:
        out = _new(q)
        po, ot, oh = out.data_ptr(), heads * dim, dim
    else:
        po, ot, oh = _rows(out, "out", dev, half, (n, heads, dim))
    lse = torch.empty((n, heads), dtype=torch.float32, device=dev) if return_lse else None
    _on_gpu(q)
    handle = _stream_handle()
    ws = cache.workspaces.get(handle)

    def call(ws):
        return _library().sph_attention(cache._ref, batch, n, heads, pq, qt, qh, start, max_q, pages.data_ptr(), row, lens, max_len,
                                        window, dim ** -0.5 if scale is None else scale, po, ot, oh,
                                        None if lse is None else lse.data_ptr(), None if ws is None else ws.data_ptr(),
                                        0 if ws is None else ws.numel(), handle)

    if ws is not None and torch.cuda.is_current_stream_capturing():
        need = attention_workspace_bytes(cache, batch, n, heads, max_q, max_len, window)
        if need <= ws.numel():
            # in the pool of its graph, whose replays may run beside any call and any other graph: let go when the call is captured, it
            # serves only later calls of the graph
            ws = torch.empty(need, dtype=torch.uint8, device=dev)
    st = call(ws)
    if st in (SPH_ERR_NULL, SPH_ERR_BUFFER_TOO_SMALL):
        # the library found, before it launched anything, that it needs a workspace or a larger one
        need = attention_workspace_bytes(cache, batch, n, heads, max_q, max_len, window)
        if need > (0 if ws is None else ws.numel()):
            st = call(_attention_workspace(cache, need, handle))
    _check(st, "sph_attention")
    return (out, lse) if return_lse else out
