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
MAX_AXES = 16                       # of a rotation's positions


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
        lib.sph_rope_axes.argtypes = [pr, P, I32, I64, *lib.sph_rope.argtypes[1:]]
        lib.sph_kv_append.argtypes = [pc, pr, I32, I64, P, I64, I64, P, I64, I64, P, I32, P, I64, I64, P, I64, I64, P, P]
        lib.sph_kv_append_axes.argtypes = [pc, pr, P, I32, I64, *lib.sph_kv_append.argtypes[2:]]
        lib.sph_kv_read.argtypes = [pc, I64, P, P, P, P]
        lib.sph_attention.argtypes = [pc, I64, I64, I32, P, I64, I64, P, I64, P, I64, P, I64, I64, ctypes.c_float,
                                      P, I64, I64, P, P, SZ, P]
        lib.sph_attention_workspace_bytes.argtypes = [pc, I64, I64, I32, I64, I64, I64, ctypes.POINTER(SZ)]
        lib.sph_attention_shared.argtypes = [pc, I64, P, I64, P, I64, P, I64, I64, I64, I32, P, I64, I64, P, I64, P, I64, P, I64,
                                             ctypes.c_float, P, I64, I64, P, P, SZ, P]
        lib.sph_attention_shared_workspace_bytes.argtypes = [pc, I64, I64, I64, I64, I64, I32, I64, I64, ctypes.POINTER(SZ)]
        lib.sph_attention_weights.argtypes = [pc, I64, I64, I32, P, I64, I64, P, I64, P, I64, P, I64, I64, ctypes.c_float, P, I32,
                                              P, I64, I64, P, I64, I64, P, SZ, P]
        lib.sph_attention_weights_workspace_bytes.argtypes = [pc, I64, I64, I32, I32, I64, I64, I64, ctypes.POINTER(SZ)]
        lib.sph_kv_evict.argtypes = [pc, I64, P, I64, P, I64, P, I32, I64, I64, I64, I64, I64, P, I64, P, P, I64, I64, I64, P, P]
        for name in ("sph_rope_table", "sph_rope", "sph_rope_axes", "sph_kv_append", "sph_kv_append_axes", "sph_kv_read",
                     "sph_attention", "sph_attention_workspace_bytes", "sph_attention_shared",
                     "sph_attention_shared_workspace_bytes", "sph_attention_weights", "sph_attention_weights_workspace_bytes",
                     "sph_kv_evict"):
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


def rope_table(rot_dim: int, max_pos: int, device="cuda", stream=None, frequencies=None, **scaling):
    """fp32 [max_pos][rot_dim/2][2] of (cos, sin) (sph_rope_table); keywords as ``rope_frequencies``, or ``frequencies``: the angle
    a position of every pair, for instance of axes with a spectrum each."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return rope_table(rot_dim, max_pos, device, frequencies=frequencies, **scaling)
    if frequencies is None:
        f, magnitude = rope_frequencies(rot_dim, **scaling)
    else:
        if scaling:
            raise ValueError("frequencies are given: no scaling")
        f, magnitude = [float(x) for x in frequencies], 1.0
        if len(f) != rot_dim // 2:
            raise ValueError(f"{len(f)} frequencies for {rot_dim // 2} pairs")
    out = torch.empty((max_pos, rot_dim // 2, 2), dtype=torch.float32, device=device)
    _on_gpu(out)
    arr = (ctypes.c_double * len(f))(*f)
    _check(_library().sph_rope_table(rot_dim, max_pos, arr, magnitude, out.data_ptr(), _stream_handle()), "sph_rope_table")
    return out


def rope_axes(sections, cycled: bool = False, device="cuda", stream=None):
    """The axis of every pair, as ``rope`` takes it: uint8 [pairs]. ``sections``: how many pairs each axis turns (1 to 16 axes, a
    multiple of 8 pairs in all). Axis 0 has the first pairs, axis 1 the next ones and so on, or with ``cycled`` the axes take the pairs in
    turn, each until its share is used up. For axes with a spectrum each, give ``rope_table`` the frequencies (``frequencies=``) in this order."""
    import torch
    left = [int(n) for n in sections]
    if not 1 <= len(left) <= MAX_AXES or any(n != m or n < 0 for n, m in zip(left, sections)) or sum(left) < 8 or sum(left) % 8:
        raise ValueError(f"sections must be the pairs of 1 to {MAX_AXES} axes, a multiple of 8 in all, not {sections!r}")
    axis = []
    if cycled:
        while any(left):
            for a, n in enumerate(left):
                if n:
                    left[a] -= 1
                    axis.append(a)
    else:
        axis = [a for a, n in enumerate(left) for _ in range(n)]
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return torch.tensor(axis, dtype=torch.uint8, device=device)
    return torch.tensor(axis, dtype=torch.uint8, device=device)


def _axes(axes, positions, table, device, tokens: int):
    """(axes' pointer, number of axes, elements between their positions, positions' pointer)."""
    import torch
    if not isinstance(axes, torch.Tensor) or axes.dtype is not torch.uint8:
        raise TypeError("axes must be a torch.uint8 tensor")
    if axes.device != device:
        raise ValueError(f"axes is on {axes.device}, the rows on {device}")
    if axes.shape != table.shape[1:2] or not axes.is_contiguous() or axes.data_ptr() % 8:
        raise ValueError(f"axes must be contiguous [{table.shape[1]}], 8-byte aligned, got shape {tuple(axes.shape)}")
    if not isinstance(positions, torch.Tensor) or positions.dtype is not torch.int32:
        raise TypeError("positions must be a torch.int32 tensor")
    if positions.device != device:
        raise ValueError(f"positions is on {positions.device}, the rows on {device}")
    if positions.dim() != 2 or not 1 <= positions.shape[0] <= MAX_AXES or positions.shape[1] != tokens or (tokens > 1 and positions.stride(1) != 1):
        raise ValueError(f"positions must be [axes][{tokens}] with unit stride along the tokens, got shape {tuple(positions.shape)} and "
                         f"strides {tuple(positions.stride())}")
    count = positions.shape[0]
    return axes.data_ptr(), count, positions.stride(0) if count > 1 else 0, positions.data_ptr()


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


def rope(x, positions, table, interleaved: bool = False, inverse: bool = False, out=None, stream=None, axes=None):
    """Rotary positions of device rows x[tokens][heads][channels], fp16 or fp32 (sph_rope): the first
    2 * table.shape[1] channels of each row turn by the angles of its token's position, the others are
    copied. ``inverse`` turns back and is the gradient (``train.rope`` is the differentiable form).
    ``out`` may be x. With ``axes`` (``rope_axes``: uint8, the axis of every pair) positions is int32 [axes][tokens], and each pair turns by
    its own axis's position, as in images and videos (sph_rope_axes)."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return rope(x, positions, table, interleaved, inverse, out, axes=axes)
    half = (torch.float16, torch.float32)
    px, xt, xh = _rows(x, "x", None, half)
    dev, n = x.device, x.shape[0]
    desc = _rope_desc(table, dev, interleaved, inverse)
    if axes is None:
        pos = _ints(positions, "positions", dev, n)
    else:
        *more, pos = _axes(axes, positions, table, dev, n)
    out = _new(x) if out is None else out
    py, yt, yh = _rows(out, "out", dev, (x.dtype,), x.shape)
    _on_gpu(x)
    args = (SPH_F16 if x.dtype is torch.float16 else SPH_F32, n, x.shape[1], x.shape[2], px, xt, xh, pos, py, yt, yh, _stream_handle())
    if axes is None:
        _check(_library().sph_rope(ctypes.byref(desc), *args), "sph_rope")
    else:
        _check(_library().sph_rope_axes(ctypes.byref(desc), *more, *args), "sph_rope_axes")
    return out


def rope_gradient(grad, positions, table, interleaved: bool, inverse: bool = False, axes=None):
    """The gradient of ``rope``'s rows from that of its result. positions, table and axes have passed ``rope``'s checks, but come back through
    whatever autograd's hooks for saved tensors make of them: what the kernel reads by is checked again."""
    import torch
    grad = aligned_rows(grad)
    n, heads, dim = grad.shape
    gt, gh, _ = grad.stride()
    gpu, lead, (rows, pairs, two) = grad.get_device(), positions.stride(), table.shape
    # (in few steps, since Python on autograd's thread costs several times what it does elsewhere: where they do not do, rope's checks say why)
    if not (table.dtype is torch.float32 and positions.dtype is torch.int32 and table.get_device() == gpu == positions.get_device() and
            table.is_contiguous() and lead[-1] == 1 and positions.shape[-1] == n and len(lead) == (1 if axes is None else 2) and
            two == 2 and (axes is None or (axes.dtype is torch.uint8 and axes.get_device() == gpu and axes.numel() == pairs and axes.is_contiguous()))):
        dev = grad.device
        _rope_desc(table, dev, interleaved, inverse)
        _ints(positions, "positions", dev, n) if axes is None else _axes(axes, positions, table, dev, n)
    out = _new(grad)
    desc = CRope(table.data_ptr(), rows, 2 * pairs, (ROPE_INTERLEAVED if interleaved else 0) | (0 if inverse else ROPE_INVERSE))
    args = (SPH_F16 if grad.element_size() == 2 else SPH_F32, n, heads, dim, grad.data_ptr(), gt if n > 1 else 0, gh if heads > 1 else 0,
            positions.data_ptr(), out.data_ptr(), heads * dim, dim, _stream_handle())
    if axes is None:
        _check(_library().sph_rope(ctypes.byref(desc), *args), "sph_rope")
    else:
        count = positions.shape[0]
        _check(_library().sph_rope_axes(ctypes.byref(desc), axes.data_ptr(), count, lead[0] if count > 1 else 0, *args), "sph_rope_axes")
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


def kv_append(cache: KVCache, k, v, slots, positions=None, table=None, interleaved: bool = False, q=None, q_out=None, stream=None,
              axes=None):
    """Write a key and a value row per token and head, k and v [tokens][kv heads][channels] (fp16 or fp32,
    any row strides), to the int32 ``slots`` (sph_kv_append; page * page_size + place in the page, -1 for a padding token). With
    ``table`` and ``positions`` the keys are rotated on the way, and so are the queries q [tokens][q heads][channels] in
    the same launch. Returns the rotated queries in fp16 (``q_out`` or a new tensor; None without q). ``axes``: as in ``rope``."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return kv_append(cache, k, v, slots, positions, table, interleaved, q, q_out, axes=axes)
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
        if axes is None:
            pos = _ints(positions, "positions", dev, n)
        else:
            *more, pos = _axes(axes, positions, table, dev, n)
    elif positions is not None or q is not None or axes is not None:
        raise ValueError("positions, axes and q need a table")
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
    args = (SPH_F16 if dt[0] is torch.float16 else SPH_F32, n, pk, kt, kh, pv, vt, vh, ps, heads, pq, qt, qh, po, ot, oh, pos,
            _stream_handle())
    if axes is None:
        _check(_library().sph_kv_append(cache._ref, desc, *args), "sph_kv_append")
    else:
        _check(_library().sph_kv_append_axes(cache._ref, desc, *more, *args), "sph_kv_append_axes")
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


def _with_workspace(cache: KVCache, handle: int, call, need):
    """``call(workspace)`` on the current stream, ``handle``, and its status. ``need()``: the bytes that the call wants, asked for only
    where the one at hand may not do."""
    import torch
    ws = cache.workspaces.get(handle)
    if ws is not None and torch.cuda.is_current_stream_capturing():
        least = need()
        if least <= ws.numel():
            # in the pool of its graph, whose replays may run beside any call and any other graph: let go when the call is captured, it
            # serves only later calls of the graph
            ws = torch.empty(least, dtype=torch.uint8, device=cache.device)
    st = call(ws)
    if st in (SPH_ERR_NULL, SPH_ERR_BUFFER_TOO_SMALL):
        # the library found, before it launched anything, that it needs a workspace or a larger one
        least = need()
        if least > (0 if ws is None else ws.numel()):
            st = call(_attention_workspace(cache, least, handle))
    return st


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

    def call(ws):
        return _library().sph_attention(cache._ref, batch, n, heads, pq, qt, qh, start, max_q, pages.data_ptr(), row, lens, max_len,
                                        window, dim ** -0.5 if scale is None else scale, po, ot, oh,
                                        None if lse is None else lse.data_ptr(), None if ws is None else ws.data_ptr(),
                                        0 if ws is None else ws.numel(), handle)

    st = _with_workspace(cache, handle, call, lambda: attention_workspace_bytes(cache, batch, n, heads, max_q, max_len, window))
    _check(st, "sph_attention")
    return (out, lse) if return_lse else out


# ------------------------------------------------------------------ shared prefixes

def _sums(t, name: str, device, batch: int, heads, width: int):
    """Checks fp32 [batch][heads][width or more] sums with unit stride along the tokens; (pointer, sequence stride, head stride)."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32:
        raise TypeError(f"{name} must be a torch.float32 tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    sh = t.shape
    if len(sh) == 3 and sh[0] == batch and sh[1] in heads and sh[2] >= width:
        s0, s1, s2 = t.stride()
        if s2 == 1 or sh[2] <= 1:
            # (the stride of a dimension of one element is never used and may hold anything)
            return t.data_ptr(), s0 if batch > 1 else 0, s1 if sh[1] > 1 else 0
    raise ValueError(f"{name} must be [{batch}][{' or '.join(str(h) for h in heads)}][{width} or more] with unit stride along the tokens, "
                     f"got shape {tuple(t.shape)} and strides {tuple(t.stride())}")


def _page_table(pages, name: str, device, batch: int):
    """Checks int32 [batch][columns]; (pointer, row stride, columns)."""
    import torch
    if not isinstance(pages, torch.Tensor) or pages.dtype is not torch.int32:
        raise TypeError(f"{name} must be a torch.int32 tensor")
    sh = pages.shape
    rows, cols = sh if len(sh) == 2 else (-1, 0)
    row, one = pages.stride() if rows >= 0 else (0, 0)
    if rows != batch or pages.device != device or (cols > 1 and rows > 0 and one != 1):
        raise ValueError(f"{name} must be [{batch}][columns] on {device} with unit stride along the columns")
    row = row if batch > 1 else cols
    if row < cols:
        raise ValueError(f"rows of {name} must not overlap")
    return pages.data_ptr(), row, cols


def attention_shared_workspace_bytes(cache: KVCache, prefixes: int, max_group: int, max_prefix: int, batch: int, tokens: int, q_heads: int,
                                     max_q: int, max_len: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_library().sph_attention_shared_workspace_bytes(cache._ref, prefixes, max_group, max_prefix, batch, tokens, q_heads, max_q, max_len,
                                                           ctypes.byref(out)), "sph_attention_shared_workspace_bytes")
    return out.value


def attention_shared(q, cache: KVCache, prefix_pages, prefix_lens, pages, seq_lens, first=None, q_start=None, max_q: int = 1,
                     max_group: int | None = None, max_prefix: int | None = None, max_len: int | None = None, scale: float | None = None,
                     out=None, return_lse: bool = False, stream=None):
    """``attention`` of sequences that share long prefixes, each of which is read once for all of them (sph_attention_shared).

    prefix_pages: int32 [prefixes][columns], prefix_lens: int32 [prefixes], the tokens that come before the own ones of sequences
    first[g] .. first[g+1]-1 (``first``: int32 [prefixes + 1], ascending; default, with one prefix: of all; sequences outside have none). pages,
    seq_lens: a sequence's own tokens, with the new ones; q, q_start, max_q, scale, out, return_lse: as in ``attention``. A query
    sees the whole prefix and its own tokens up to its position. max_group, max_prefix, max_len: bounds of the sequences behind a
    prefix (default: all), of its tokens and of the own ones (default: what the columns hold) that the launch is planned for. There is no window."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return attention_shared(q, cache, prefix_pages, prefix_lens, pages, seq_lens, first, q_start, max_q, max_group, max_prefix, max_len,
                                    scale, out, return_lse)
    dev, half = cache.device, (torch.float16,)
    pq, qt, qh = _rows(q, "q", dev, half)
    n, heads, dim = q.shape
    if dim != cache.head_dim:
        raise ValueError(f"q has {dim} channels a head, the cache {cache.head_dim}")
    batch = seq_lens.shape[0] if isinstance(seq_lens, torch.Tensor) and seq_lens.dim() else 0
    lens = _ints(seq_lens, "seq_lens", dev, batch)
    pp, row, cols = _page_table(pages, "pages", dev, batch)
    prefixes = prefix_lens.shape[0] if isinstance(prefix_lens, torch.Tensor) and prefix_lens.dim() else 0
    plens = _ints(prefix_lens, "prefix_lens", dev, prefixes)
    pf, prow, pcols = _page_table(prefix_pages, "prefix_pages", dev, prefixes)
    if prefixes < 1 or (first is None and prefixes > 1):
        raise ValueError(f"{prefixes} prefixes: at least one, and several need first")
    at = None if first is None else _ints(first, "first", dev, prefixes + 1)
    start = None if q_start is None else _ints(q_start, "q_start", dev, batch + 1)
    if max_group is None or first is None:
        max_group = max(1, batch)
    page = cache.page_size
    max_len = cols * page if max_len is None else max_len
    max_prefix = pcols * page if max_prefix is None else max_prefix
    if max_len > cols * page or max_prefix > pcols * page:
        raise ValueError(f"max_len {max_len} or max_prefix {max_prefix} is more than the {cols} and {pcols} columns of pages hold")
    if out is None:
        out = _new(q)
        po, ot, oh = out.data_ptr(), heads * dim, dim
    else:
        po, ot, oh = _rows(out, "out", dev, half, (n, heads, dim))
    lse = torch.empty((n, heads), dtype=torch.float32, device=dev) if return_lse else None
    _on_gpu(q)
    handle = _stream_handle()

    def call(ws):
        return _library().sph_attention_shared(cache._ref, prefixes, at, max_group, pf, prow, plens, max_prefix, batch, n, heads, pq, qt, qh,
                                               start, max_q, pp, row, lens, max_len, dim ** -0.5 if scale is None else scale, po, ot, oh,
                                               None if lse is None else lse.data_ptr(), None if ws is None else ws.data_ptr(),
                                               0 if ws is None else ws.numel(), handle)

    st = _with_workspace(cache, handle, call, lambda: attention_shared_workspace_bytes(cache, prefixes, max_group, max_prefix, batch, n, heads,
                                                                                       max_q, max_len))
    _check(st, "sph_attention_shared")
    return (out, lse) if return_lse else out


# ------------------------------------------------------------------ attention that tokens got

def attention_weights_workspace_bytes(cache: KVCache, batch: int, tokens: int, q_heads: int, heads: int, max_q: int, max_len: int,
                                      window: int = 0) -> int:
    out = ctypes.c_size_t(0)
    _check(_library().sph_attention_weights_workspace_bytes(cache._ref, batch, tokens, q_heads, heads, max_q, max_len, window, ctypes.byref(out)),
           "sph_attention_weights_workspace_bytes")
    return out.value


def attention_weights(q, cache: KVCache, pages, seq_lens, lse, before=None, per_head: bool = True, q_start=None, max_q: int = 1,
                      max_len: int | None = None, window: int = 0, scale: float | None = None, out=None, stream=None):
    """How much attention every cached token got from the new ones (sph_attention_weights): their softmax weights added up, over the query
    heads of each kv head (``per_head``) or over all, on top of ``before`` (fp32 [batch][kv heads or 1][tokens], the sums of
    earlier calls). q, pages, seq_lens, q_start, max_q, max_len, window, scale: as ``attention`` had them; lse: what it
    returned with ``return_lse``. Returns fp32 [batch][kv heads or 1][max_len], or ``out``, which may be ``before``; zeros from a sequence's length
    on. ``kv_evict`` goes by these sums."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return attention_weights(q, cache, pages, seq_lens, lse, before, per_head, q_start, max_q, max_len, window, scale, out)
    dev = cache.device
    pq, qt, qh = _rows(q, "q", dev, (torch.float16,))
    n, q_heads, dim = q.shape
    if dim != cache.head_dim:
        raise ValueError(f"q has {dim} channels a head, the cache {cache.head_dim}")
    batch = seq_lens.shape[0] if isinstance(seq_lens, torch.Tensor) and seq_lens.dim() else 0
    lens = _ints(seq_lens, "seq_lens", dev, batch)
    pp, row, cols = _page_table(pages, "pages", dev, batch)
    start = None if q_start is None else _ints(q_start, "q_start", dev, batch + 1)
    held = cols * cache.page_size
    if max_len is None:
        max_len = held
    elif max_len > held:
        raise ValueError(f"max_len {max_len} is more than the {cols} columns of pages hold")
    if not isinstance(lse, torch.Tensor) or lse.dtype is not torch.float32:
        raise TypeError("lse must be a torch.float32 tensor")
    if lse.device != dev or lse.shape != (n, q_heads) or not lse.is_contiguous():
        raise ValueError(f"lse must be contiguous [{n}][{q_heads}] on {dev}, got shape {tuple(lse.shape)} and strides {tuple(lse.stride())}")
    heads = cache.kv_heads if per_head else 1
    pb, bs, bh = (None, 0, 0) if before is None else _sums(before, "before", dev, batch, (heads,), max_len)
    if out is None:
        out = torch.empty((batch, heads, max_len), dtype=torch.float32, device=dev)
        po, os, oh = out.data_ptr(), heads * max_len, max_len
    else:
        po, os, oh = _sums(out, "out", dev, batch, (heads,), max_len)
    _on_gpu(q)
    handle = _stream_handle()

    def call(ws):
        return _library().sph_attention_weights(cache._ref, batch, n, q_heads, pq, qt, qh, start, max_q, pp, row, lens, max_len, window,
                                                dim ** -0.5 if scale is None else scale, lse.data_ptr(), heads, pb, bs, bh, po, os, oh,
                                                None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(), handle)

    st = _with_workspace(cache, handle, call, lambda: attention_weights_workspace_bytes(cache, batch, n, q_heads, heads, max_q, max_len, window))
    _check(st, "sph_attention_weights")
    return out


# ------------------------------------------------------------------ eviction

def kv_evict(cache: KVCache, pages, seq_lens, sums, keep: int, recent: int = 0, first: int = 0, to_pages=None, max_len: int | None = None,
             lens_out=None, sums_out=None, stream=None):
    """Shrink sequences to ``keep`` tokens (sph_kv_evict): the ``first`` ones, the last ``recent``, and of the others those with the largest
    ``sums`` (fp32 [batch][kv heads][tokens], as ``attention_weights`` gives them: each kv head chooses its own; or [batch][1][tokens]: one choice
    for all), in order. pages, seq_lens, max_len: as in ``attention`` (max_len default: what pages and sums hold). Without
    ``to_pages`` tokens move within their pages, which other sequences must not share from the first evicted token on; with int32 [batch][columns] ``to_pages``
    (pages of no sequence here) they are copied there, and pages may be shared. Returns (lens int32 [batch]: the new lengths, ``lens_out`` or a
    new tensor; sums: the kept tokens' and zeros behind them, ``sums_out``, which may be sums, or new fp32 [batch][heads][max_len]; kept int32
    [batch][heads][min(keep, max_len), at least 1]: which tokens were kept, then -1)."""
    import torch
    if stream is not None:                      # what is made for the call belongs to its stream
        with torch.cuda.stream(stream):
            return kv_evict(cache, pages, seq_lens, sums, keep, recent, first, to_pages, max_len, lens_out, sums_out)
    dev = cache.device
    batch = seq_lens.shape[0] if isinstance(seq_lens, torch.Tensor) and seq_lens.dim() else 0
    lens = _ints(seq_lens, "seq_lens", dev, batch)
    pp, row, cols = _page_table(pages, "pages", dev, batch)
    held = cols * cache.page_size
    if max_len is None:
        max_len = min(held, sums.shape[2] if isinstance(sums, torch.Tensor) and sums.dim() == 3 else held)
    elif max_len > held:
        raise ValueError(f"max_len {max_len} is more than the {cols} columns of pages hold")
    ps, ss, sh = _sums(sums, "sums", dev, batch, (cache.kv_heads, 1) if cache.kv_heads > 1 else (1,), max_len)
    if keep < 1 or recent < 0 or first < 0 or recent + first > keep:
        raise ValueError(f"keep {keep} must be positive and hold recent {recent} and first {first}")
    most = min(keep, max_len)
    if to_pages is None:
        pt, to_row = pp, row
    else:
        pt, to_row, to_cols = _page_table(to_pages, "to_pages", dev, batch)
        if to_cols * cache.page_size < most:
            raise ValueError(f"the {to_cols} columns of to_pages do not hold {most} tokens")
    heads = sums.shape[1]
    if sums_out is None:
        sums_out = torch.empty((batch, heads, max_len), dtype=torch.float32, device=dev)
        pn, ns, nh = sums_out.data_ptr(), heads * max_len, max_len
    else:
        pn, ns, nh = _sums(sums_out, "sums_out", dev, batch, (heads,), most)
    if lens_out is None:
        lens_out = torch.empty_like(seq_lens)
        pl = lens_out.data_ptr()
    else:
        pl = _ints(lens_out, "lens_out", dev, batch)
    _on_gpu(seq_lens)
    if keep > max_len:                          # nothing goes: a row of what was kept is no longer than a sequence can be
        keep, recent, first = max(max_len, 1), 0, 0
    kept = torch.empty((batch, heads, keep), dtype=torch.int32, device=dev)
    st = _library().sph_kv_evict(cache._ref, batch, pp, row, lens, max_len, ps, heads, ss, sh, keep, recent, first, pt, to_row, pl, pn,
                                 sums_out.shape[2], ns, nh, kept.data_ptr(), _stream_handle())
    _check(st, "sph_kv_evict")
    return lens_out, sums_out, kept
