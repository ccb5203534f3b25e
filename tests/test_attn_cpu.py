"""CPU checks of the rotary positions, the paged cache and its attention: refusals of the C ABI and of the
binding (before any HIP call), the rotary frequencies, and models of the launches' arithmetic: equal shares of
ragged sequences, and cache blocks spread among query blocks."""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
import random

import numpy as np
import pytest

import paper_2609_24875_amd as pkg
from paper_2609_24875_amd import attn as A

torch = pytest.importorskip("torch")

needs_lib = pytest.mark.skipif(not os.path.exists(pkg.LIB_PATH), reason="libsph.so not built")
OK, NULL, SHAPE, FORMAT, VALUE, SMALL = 0, 1, 2, 3, 5, 6
P = 1 << 20                                       # stands for a device pointer; no call here gets as far as using one


def _cache(**kw):
    bits, heads, dim, page = kw.get("bits", 8), kw.get("kv_heads", 2), kw.get("head_dim", 128), kw.get("page_size", 16)
    row = dim * bits // 8
    d = dict(bits=bits, kv_heads=heads, head_dim=dim, page_size=page, n_pages=4, d_k=P, d_v=P, page_stride=heads * page * row,
             head_stride=page * row, token_stride=row, d_k_par=P, d_v_par=P, par_page_stride=heads * page * dim // 8,
             par_head_stride=page * dim // 8, par_token_stride=dim // 8)
    d.update(kw)
    return A.CKVCache(*[d[n] for n, _ in A.CKVCache._fields_])


def _rope(**kw):
    d = dict(d_table=P, max_pos=100, rot_dim=64, flags=0)
    d.update(kw)
    return A.CRope(*[d[n] for n, _ in A.CRope._fields_])


# ------------------------------------------------------------------ refusals

CACHE_FAULTS = [(dict(bits=5), FORMAT), (dict(bits=32), FORMAT), (dict(head_dim=80, token_stride=80), FORMAT), (dict(d_k=0), NULL),
                (dict(d_v=None), NULL), (dict(d_k_par=0), NULL), (dict(d_v_par=0), NULL), (dict(page_size=0), SHAPE),
                (dict(page_size=24), SHAPE), (dict(page_size=1 << 17), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=1025), SHAPE),
                (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 28), SHAPE), (dict(d_k=P + 8), SHAPE), (dict(token_stride=64), SHAPE),
                (dict(token_stride=136), SHAPE), (dict(page_stride=0), SHAPE), (dict(head_stride=-16), SHAPE),
                (dict(page_size=65536, token_stride=1 << 16), SHAPE), (dict(d_k_par=P + 2), SHAPE), (dict(par_token_stride=8), SHAPE),
                (dict(par_page_stride=18), SHAPE)]


@needs_lib
@pytest.mark.parametrize("fault,want", CACHE_FAULTS)
def test_every_call_refuses_a_wrong_cache(fault, want):
    lib, c = A._library(), _cache(**fault)
    r = ctypes.byref(c)
    assert lib.sph_kv_read(r, 1, P, P, P, None) == want
    assert lib.sph_kv_append(r, None, 0, 1, P, 256, 128, P, 256, 128, P, 0, None, 0, 0, None, 0, 0, None, None) == want
    n = ctypes.c_size_t(0)
    assert lib.sph_attention_workspace_bytes(r, 1, 1, 8, 1, 64, 0, ctypes.byref(n)) == want
    assert lib.sph_attention(r, 1, 1, 8, P, 1024, 128, None, 1, P, 4, P, 64, 0, 1.0, P, 1024, 128, None, P, 1 << 30, None) == want


ROPE_FAULTS = [(dict(), dict(dtype=2), SHAPE), (dict(), dict(tokens=-1), SHAPE), (dict(), dict(tokens=(1 << 26) + 1), SHAPE),
               (dict(), dict(heads=0), SHAPE), (dict(), dict(dim=72), SHAPE), (dict(), dict(dim=528), SHAPE), (dict(), dict(x=None), NULL),
               (dict(), dict(y=None), NULL), (dict(), dict(pos=None), NULL), (dict(), dict(x=P + 4), SHAPE), (dict(), dict(xt=1020), SHAPE),
               (dict(), dict(xh=-128), SHAPE), (dict(), dict(yt=0), SHAPE), (dict(), dict(yh=0), SHAPE), (dict(), dict(pos=P + 2), SHAPE),
               (dict(d_table=None), {}, NULL), (dict(d_table=P + 4), {}, SHAPE), (dict(max_pos=0), {}, SHAPE), (dict(max_pos=1 << 31), {}, SHAPE),
               (dict(rot_dim=144), {}, SHAPE), (dict(rot_dim=24), {}, SHAPE), (dict(rot_dim=0), {}, SHAPE), (dict(flags=4), {}, SHAPE)]


@needs_lib
@pytest.mark.parametrize("desc,args,want", ROPE_FAULTS)
def test_rope_refusals(desc, args, want):
    a = dict(dtype=0, tokens=2, heads=8, dim=128, x=P, xt=1024, xh=128, pos=P, y=P, yt=1024, yh=128)
    a.update(args)
    st = A._library().sph_rope(ctypes.byref(_rope(**desc)), a["dtype"], a["tokens"], a["heads"], a["dim"], a["x"], a["xt"], a["xh"], a["pos"],
                               a["y"], a["yt"], a["yh"], None)
    assert st == want


@needs_lib
def test_rope_table_refusals():
    lib = A._library()
    f = (ctypes.c_double * 32)(*[0.5] * 32)
    assert lib.sph_rope_table(64, 10, None, 1.0, P, None) == NULL
    assert lib.sph_rope_table(64, 10, f, 1.0, None, None) == NULL
    for rot, n, out in ((0, 10, P), (24, 10, P), (528, 10, P), (64, 0, P), (64, 1 << 31, P), (64, 10, P + 8)):
        assert lib.sph_rope_table(rot, n, f, 1.0, out, None) == SHAPE
    assert lib.sph_rope_table(64, 10, f, math.inf, P, None) == VALUE
    f[31] = math.nan
    assert lib.sph_rope_table(64, 10, f, 1.0, P, None) == VALUE


@needs_lib
@pytest.mark.parametrize("args,want", [
    (dict(dtype=3), SHAPE), (dict(tokens=-1), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL), (dict(slots=None), NULL), (dict(pos=None), NULL),
    (dict(q=None), NULL), (dict(qo=None), NULL), (dict(heads=-1), SHAPE), (dict(rope=None), NULL), (dict(k=P + 2), SHAPE), (dict(vt=100), SHAPE),
    (dict(qt=100), SHAPE), (dict(qot=0), SHAPE), (dict(qoh=4), SHAPE), (dict(slots=P + 1), SHAPE), (dict(desc=dict(rot_dim=256)), SHAPE),
    (dict(tokens=0, k=None, v=None, slots=None), OK)])
def test_append_refusals(args, want):
    a = dict(dtype=0, tokens=2, k=P, kt=256, kh=128, v=P, vt=256, vh=128, slots=P, heads=8, q=P, qt=1024, qh=128, qo=P, qot=1024, qoh=128,
             pos=P, rope=True, desc={})
    a.update(args)
    st = A._library().sph_kv_append(ctypes.byref(_cache()), ctypes.byref(_rope(**a["desc"])) if a["rope"] else None, a["dtype"], a["tokens"],
                                    a["k"], a["kt"], a["kh"], a["v"], a["vt"], a["vh"], a["slots"], a["heads"], a["q"], a["qt"], a["qh"],
                                    a["qo"], a["qot"], a["qoh"], a["pos"], None)
    assert st == want


@needs_lib
@pytest.mark.parametrize("args,want", [
    (dict(batch=-1), SHAPE), (dict(batch=70000), SHAPE), (dict(tokens=-1), SHAPE), (dict(heads=0), SHAPE), (dict(heads=7), SHAPE),
    (dict(max_q=0), SHAPE), (dict(max_len=-1), SHAPE), (dict(max_len=(1 << 30) + 1), SHAPE), (dict(window=-1), SHAPE),
    (dict(scale=math.nan), VALUE), (dict(scale=math.inf), VALUE), (dict(start=None), SHAPE), (dict(cols=3), SHAPE), (dict(cols=1 << 31), SHAPE),
    (dict(q=None), NULL), (dict(o=None), NULL), (dict(lens=None), NULL), (dict(pages=None), NULL), (dict(q=P + 8), SHAPE), (dict(qt=1028), SHAPE),
    (dict(oh=-128), SHAPE), (dict(ot=0), SHAPE), (dict(oh=0), SHAPE), (dict(lens=P + 1), SHAPE), (dict(lse=P + 2), SHAPE), (dict(ws=P + 16), SHAPE),
    (dict(max_len=4096, cols=256, ws=None), NULL), (dict(max_len=4096, cols=256, nws=64), SMALL), (dict(batch=0, q=None), OK),
    (dict(tokens=0, lens=None), OK)])
def test_attention_refusals(args, want):
    a = dict(batch=2, tokens=4, heads=8, q=P, qt=1024, qh=128, start=P, max_q=2, pages=P, cols=4, lens=P, max_len=64, window=0, scale=0.1, o=P,
             ot=1024, oh=128, lse=None, ws=P, nws=1 << 30)
    a.update(args)
    st = A._library().sph_attention(ctypes.byref(_cache()), a["batch"], a["tokens"], a["heads"], a["q"], a["qt"], a["qh"], a["start"], a["max_q"],
                                    a["pages"], a["cols"], a["lens"], a["max_len"], a["window"], a["scale"], a["o"], a["ot"], a["oh"], a["lse"],
                                    a["ws"], a["nws"], None)
    assert st == want


@needs_lib
def test_attention_workspace():
    def need(**kw):
        a = dict(batch=1, tokens=1, heads=8, max_q=1, max_len=64, window=0)
        a.update(kw)
        n = ctypes.c_size_t(1)
        assert A._library().sph_attention_workspace_bytes(ctypes.byref(_cache()), a["batch"], a["tokens"], a["heads"], a["max_q"], a["max_len"],
                                                          a["window"], ctypes.byref(n)) == OK
        return n.value
    assert need() == 0                                          # short: one workgroup a sequence and head
    assert need(max_len=1 << 20) > 0
    assert need(max_len=1 << 20, window=64) == 0
    assert need(batch=513, tokens=513, max_len=1 << 20) == 0     # enough sequences to fill the chip
    assert need(batch=0, max_len=1 << 20) == 0 and need(tokens=0, max_len=1 << 20) == 0
    assert need(batch=64, tokens=64 * 512, max_q=512, max_len=1 << 14) == 0   # enough rows
    assert need(batch=1, tokens=64, max_q=64, max_len=1 << 14) > 0
    assert A._library().sph_attention_workspace_bytes(ctypes.byref(_cache()), 1, 1, 8, 1, 64, 0, None) == NULL


@needs_lib
@pytest.mark.parametrize("kv_heads,heads,batch,max_q", [(1, 65535, 1, 1 << 24), (1, 32768, 1, 1 << 24), (1, 49152, 3, 1 << 24), (2, 65534, 65536, 1 << 24),
                                                        (1024, 64512, 65536, 1 << 20), (8, 32, 65536, 1 << 13), (8, 32, 4096, 65536)])
def test_rows_beyond_a_launch_are_refused(kv_heads, heads, batch, max_q):
    """Tiles of rows that pass 32 bits, or a launch's 2^24 workgroups, on the way to a plan: a status from both entries."""
    lib, r, n = A._library(), ctypes.byref(_cache(kv_heads=kv_heads)), ctypes.c_size_t(7)
    for max_len in (64, 4096, 1 << 30):
        assert lib.sph_attention_workspace_bytes(r, batch, 1 << 26, heads, max_q, max_len, 0, ctypes.byref(n)) == SHAPE
        assert lib.sph_attention(r, batch, 1 << 26, heads, P, heads * 128, 128, P, max_q, P, 1 << 26, P, max_len, 0, 1.0, P, heads * 128, 128,
                                 None, P, 1 << 40, None) == SHAPE


# ------------------------------------------------------------------ the binding

def _cpu_cache(bits=8, **kw):
    a = dict(n_pages=4, kv_heads=2, head_dim=64, page_size=16, bits=bits, device="cpu")
    a.update(kw)
    return pkg.KVCache.empty(**a)


def test_cache_checks_its_tensors():
    c = _cpu_cache()
    assert (c.n_pages, c.kv_heads, c.page_size, c.head_dim, c.bits) == (4, 2, 16, 64, 8)
    assert c.nbytes == 2 * 4 * 2 * 16 * (64 + 8)
    d = c.desc
    assert (d.page_stride, d.head_stride, d.token_stride) == (2 * 16 * 64, 16 * 64, 64)
    assert (d.par_page_stride, d.par_head_stride, d.par_token_stride) == (2 * 16 * 8, 16 * 8, 8)
    assert _cpu_cache(4).head_dim == 64 and _cpu_cache(4).k.shape[3] == 32
    k16 = torch.zeros(4, 16, 2, 64, dtype=torch.float16).transpose(1, 2)      # token-major pages
    d = pkg.KVCache(k16, k16.clone(memory_format=torch.preserve_format)).desc
    assert (d.page_stride, d.head_stride, d.token_stride) == (2 * 16 * 128, 128, 256)
    one = torch.zeros(1, 1, 1, 64, dtype=torch.float16).as_strided((1, 1, 1, 64), (0, 7, 3, 1))
    d = pkg.KVCache(one, one).desc                              # strides that are never used
    assert (d.page_stride, d.head_stride, d.token_stride) == (128, 128, 128)
    for f in (lambda: pkg.KVCache(c.k, c.v, c.k_par, c.v_par, bits=7), lambda: pkg.KVCache(c.k[..., ::2], c.v, c.k_par, c.v_par, bits=8),
              lambda: pkg.KVCache(c.k, c.v[:2], c.k_par, c.v_par, bits=8), lambda: pkg.KVCache(c.k, c.v, c.k_par[:, :, :, :1], c.v_par, bits=8),
              lambda: pkg.KVCache(k16, k16.contiguous()), lambda: pkg.KVCache(k16, k16, c.k_par, None),
              lambda: pkg.KVCache.empty(2, 2, 80, device="cpu"), lambda: pkg.KVCache.empty(2, 2, 64, bits=2, device="cpu")):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: pkg.KVCache(c.k, c.v, bits=16), lambda: pkg.KVCache(c.k, c.v, bits=8), lambda: pkg.KVCache(k16, None)):
        with pytest.raises(TypeError):
            f()


@needs_lib
def test_binding_refusals():
    c = _cpu_cache(16)
    x, pos, tab = torch.zeros(3, 4, 64), torch.zeros(3, dtype=torch.int32), torch.zeros(10, 32, 2)
    h, kv = torch.zeros(3, 4, 64).half(), torch.zeros(3, 2, 64).half()
    pages, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    wrong_type = (lambda: pkg.rope(x.double(), pos, tab), lambda: pkg.rope(x, pos.long(), tab), lambda: pkg.rope(x, pos, tab.double()),
                  lambda: pkg.kv_append(c, kv.double(), kv, pos), lambda: pkg.kv_append(c, kv, kv.float(), pos),
                  lambda: pkg.kv_append(c, kv, kv, pos.long()), lambda: pkg.kv_append(c, kv, kv, pos, positions=pos, table=tab, q=h.float()),
                  lambda: pkg.kv_read(c, pos.long()), lambda: pkg.attention(x, c, pages, lens), lambda: pkg.attention(h, c, pages.long(), lens),
                  lambda: pkg.attention(h, c, pages, lens.long()))
    wrong_value = (lambda: pkg.rope(x[..., ::2], pos, tab), lambda: pkg.rope(x[0], pos, tab), lambda: pkg.rope(x, pos[:2], tab),
                   lambda: pkg.rope(x, pos, tab[..., :1]), lambda: pkg.rope(x, pos, tab, out=torch.zeros(3, 4, 32)),
                   lambda: pkg.kv_append(c, kv[:, :1], kv, pos), lambda: pkg.kv_append(c, kv, kv[:2], pos), lambda: pkg.kv_append(c, kv, kv, pos[:2]),
                   lambda: pkg.kv_append(c, kv, kv, pos, q=h), lambda: pkg.kv_append(c, kv, kv, pos, positions=pos),
                   lambda: pkg.kv_append(c, kv, kv, pos, positions=pos, table=tab, q=h[:2]),
                   lambda: pkg.kv_read(c, pos[None]), lambda: pkg.kv_read(c, pos, out=(kv[:2], kv[:2])),
                   lambda: pkg.attention(h[..., :32], c, pages, lens), lambda: pkg.attention(h, c, pages[0], lens),
                   lambda: pkg.attention(h, c, pages, lens[:2]), lambda: pkg.attention(h, c, pages, lens, q_start=lens),
                   lambda: pkg.attention(h, c, pages, lens, max_len=65), lambda: pkg.attention(h, c, pages.t(), lens),
                   lambda: pkg.attention(h, c, pages[:1].expand(3, 4), lens), lambda: pkg.attention(h, c, pages, lens, out=h[:2]))
    for f in wrong_type:
        with pytest.raises(TypeError):
            f()
    for f in wrong_value:
        with pytest.raises(ValueError):
            f()
    # what would be right on a GPU does not reach the library from the CPU
    for f in (lambda: pkg.rope(x, pos, tab), lambda: pkg.kv_append(c, kv, kv, pos, positions=pos, table=tab, q=h), lambda: pkg.kv_read(c, pos),
              lambda: pkg.attention(h, c, pages, lens)):
        with pytest.raises(ValueError, match="GPU"):
            f()


@needs_lib
def test_a_table_is_made_on_a_gpu_only():
    with pytest.raises(ValueError, match="GPU"):
        pkg.rope_table(64, 10, device="cpu")


def test_calls_on_another_gpu_than_the_current_one_are_refused(monkeypatch):
    """The launch goes to the current device, where another device's addresses mean nothing."""
    class Tensor:
        is_cuda, device = True, "cuda:1"

        def get_device(self):
            return 1
    for now in (1, 0):
        monkeypatch.setattr(torch.cuda, "current_device", lambda: now)
        if now:
            A._on_gpu(Tensor())
        else:
            with pytest.raises(ValueError, match="cuda:1"):
                A._on_gpu(Tensor())


class _Streams:
    """Stands for torch.cuda.stream: which stream is current, and on which one each tensor was made."""

    def __init__(self, monkeypatch):
        self.now, self.made = [None], []
        monkeypatch.setattr(torch.cuda, "stream", self.stream)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
        for name in ("empty", "empty_like", "zeros"):
            monkeypatch.setattr(torch, name, self.recorded(getattr(torch, name)))

    def recorded(self, f):
        def make(*a, **kw):
            self.made.append(self.now[-1])
            return f(*a, **kw)
        return make

    @contextlib.contextmanager
    def stream(self, s):
        self.now.append(self.now[-1] if s is None else s)
        yield
        self.now.pop()


class _Stream:
    cuda_stream = 77


def test_tensors_made_for_a_stream_are_made_on_it(monkeypatch):
    """A tensor belongs to the stream that it was made on: the allocator hands its memory to that stream's later work as soon as it is let go, and
    takes it from that stream's earlier work. So results of a call on another stream than the current one are made on that stream."""
    class Lib:
        def __getattr__(self, name):
            return lambda *a: 0
    c = _cpu_cache(16)
    h, kv, pos, tab = torch.zeros(3, 4, 64).half(), torch.zeros(3, 2, 64).half(), torch.zeros(3, dtype=torch.int32), torch.zeros(10, 32, 2)
    pages = torch.zeros(3, 4, dtype=torch.int32)
    monkeypatch.setattr(A, "_library", Lib)
    monkeypatch.setattr(A, "_on_gpu", lambda *t: None)
    monkeypatch.setattr(A, "_stream_handle", lambda s=None: 77)
    st, on = _Streams(monkeypatch), _Stream()
    calls = (lambda **kw: pkg.rope(h, pos, tab, **kw), lambda **kw: pkg.rope(h[:, :2], pos, tab, **kw), lambda **kw: pkg.rope_table(64, 10, device="cpu", **kw),
             lambda **kw: pkg.kv_append(c, kv, kv, pos, positions=pos, table=tab, q=h, **kw), lambda **kw: pkg.kv_read(c, pos, **kw),
             lambda **kw: pkg.attention(h, c, pages, pos, return_lse=True, **kw), lambda **kw: pkg.attention(h[:, :2], c, pages, pos, **kw))
    for f in calls:
        st.made.clear()
        f(stream=on)
        assert st.made and all(s is on for s in st.made)
    with torch.cuda.stream(on):
        st.made.clear()
        A.rope_gradient(h, pos, tab, False)
        assert st.made == [on]


def test_a_block_on_a_given_stream_runs_on_it_whole(monkeypatch):
    """The rows and the outputs between a block's four calls are let go when it returns, before the stream has read them: they have to be
    that stream's, as its result."""
    from paper_2609_24875_amd import block as K

    class Weights:
        def __init__(self, n, k):
            self.n, self.k = n, k

    st, on, seen = _Streams(monkeypatch), _Stream(), []

    def gemm(w, x, out_dtype=None, stream=None):
        seen.append((st.now[-1], stream))
        return torch.empty(x.shape[0], w.n, dtype=out_dtype)

    monkeypatch.setattr(K.B, "gemm", gemm)
    monkeypatch.setattr(K.A, "kv_append", lambda *a, q=None, stream=None, **kw: seen.append((st.now[-1], stream)) or q)
    monkeypatch.setattr(K.A, "attention", lambda *a, stream=None, **kw: seen.append((st.now[-1], stream)))
    block = K.AttentionBlock(Weights(8 * 64, 256), Weights(256, 4 * 64), _cpu_cache(16), None, 4)
    x = torch.zeros(3, 256).half()
    st.made.clear()
    assert block(x, None, None, None, None, stream=on).shape == (3, 256)
    assert len(seen) == 4 and all(now is on and s in (None, on) for now, s in seen)
    assert len(st.made) == 3 and all(s is on for s in st.made)
    seen.clear()
    block(x, None, None, None, None)
    assert all(s == (None, None) for s in seen)


# ------------------------------------------------------------------ rotary frequencies

def test_rope_frequencies():
    f, m = pkg.rope_frequencies(64, base=10000.0)
    assert m == 1.0 and f[0] == 1.0 and np.allclose(f, [10000.0 ** (-2 * i / 64) for i in range(32)], rtol=1e-14)
    lin, _ = pkg.rope_frequencies(64, scaling="linear", factor=4.0)
    assert np.allclose(lin, f / 4, rtol=1e-15)
    ntk, m = pkg.rope_frequencies(64, scaling="ntk", factor=4.0)
    assert m == 1.0 and ntk[0] == 1.0 and np.isclose(ntk[-1], f[-1] / 4, rtol=1e-12) and np.all(ntk <= f)
    yarn, m = pkg.rope_frequencies(64, scaling="yarn", factor=4.0, original_max_pos=4096)
    assert np.isclose(m, 0.1 * math.log(4.0) + 1.0)
    turns = 4096 * f / (2 * math.pi)
    assert np.allclose(yarn[turns > 40], f[turns > 40]) and np.allclose(yarn[turns < 0.7], f[turns < 0.7] / 4)
    assert np.all(yarn <= f * (1 + 1e-15)) and np.all(yarn >= f / 4 * (1 - 1e-15)) and np.all(np.diff(yarn) < 0)
    for kw in (dict(scaling="no"), dict(factor=0.5), dict(base=1.0)):
        with pytest.raises(ValueError):
            pkg.rope_frequencies(64, **kw)
    for rot in (0, 24, -16):
        with pytest.raises(ValueError):
            pkg.rope_frequencies(rot)


@pytest.mark.parametrize("base,rot,original", [(10000.0, 128, 4096), (10000.0, 128, 65536), (10000.0, 128, 131072), (10000.0, 128, 1 << 20),
                                               (10000.0, 64, 262144), (500000.0, 128, 8192), (500000.0, 128, 1 << 23), (1e6, 128, 32768)])
def test_yarn_divides_by_the_whole_factor_only_behind_the_slow_pair(base, rot, original):
    """The pair index at which a pair makes `turns` turns over the original context solves original base^(-2i/rot) = 2 pi turns; the ramp goes from
    the index of 32 turns, rounded down, to that of one, rounded up, which for long contexts lies behind the last pair. In exact steps of one
    pair, so that a pair between has its own share."""
    factor = 4.0
    f, _ = pkg.rope_frequencies(rot, base=base)
    y, m = pkg.rope_frequencies(rot, base=base, scaling="yarn", factor=factor, original_max_pos=original)
    fast, slow = (math.log(original / (2 * math.pi * turns), base) * rot / 2 for turns in (32, 1))
    lo, hi = max(math.floor(fast), 0), math.ceil(slow)
    assert lo < hi < rot
    for i in range(rot // 2):
        stretched = 0.0 if i <= lo else 1.0 if i >= hi else (i - lo) / (hi - lo)
        assert math.isclose(y[i], f[i] * (1 - stretched) + f[i] / factor * stretched, rel_tol=1e-12)
    turns = original * f / (2 * math.pi)
    assert np.all(y[turns > 1] > f[turns > 1] / factor * (1 + 1e-3)) and np.all(np.diff(y) < 0)


# ------------------------------------------------------------------ launch arithmetic

def test_cache_blocks_are_spread_evenly_and_each_runs_once():
    """Block i of total writes the cache if floor((i + 1) f / 2^32) passes floor(i f / 2^32), f = ceil(kv 2^32 / total)."""
    rng = random.Random(3)
    for _ in range(200):
        kv, q = rng.randint(1, 3000), rng.randint(1, 3000)
        total = kv + q
        f = ((kv << 32) + total - 1) // total
        assert f < 1 << 32
        at = [(i * f) >> 32 for i in range(total + 1)]
        kvs = [at[i] for i in range(total) if at[i + 1] != at[i]]
        qs = [i - at[i] for i in range(total) if at[i + 1] == at[i]]
        assert kvs == list(range(kv)) and qs == list(range(q))
    for kv, q in ((1, (1 << 24) - 2), ((1 << 24) - 2, 1), (8388607, 8388608)):
        total = kv + q
        f = ((kv << 32) + total - 1) // total
        assert (total * f) >> 32 == kv and f < 1 << 32


def test_equal_shares_cover_every_tile_once():
    """The shares of k_attn: every sequence's tiles are covered once and in order, and the parts' slots
    (share + sequence) are distinct, follow each other and stay below shares + batch."""
    rng = random.Random(4)
    for _ in range(300):
        batch, shares = rng.choice([1, 2, 7, 64, 512]), rng.choice([1, 3, 32, 96, 511])
        tiles = [rng.choice([0, 1, 1, 5, rng.randint(1, 400)]) for _ in range(batch)]
        before = np.concatenate([[0], np.cumsum(tiles)])
        total = int(before[-1])
        if total == 0:
            continue
        per = max(4, -(-total // shares))
        got, slots, where = [[] for _ in range(batch)], [], {}
        for w in range(shares):
            pos, end = w * per, min(total, (w + 1) * per)
            if pos >= total:
                continue
            b = int(np.searchsorted(before, pos, side="right")) - 1
            while pos < end:
                if before[b + 1] == before[b]:
                    b += 1
                    continue
                lo, hi = pos - before[b], min(end, before[b + 1]) - before[b]
                got[b] += list(range(lo, hi))
                s_lo, s_hi = int(before[b]) // per, (int(before[b + 1]) - 1) // per
                if lo == 0:
                    where[b] = (s_lo + b, s_hi - s_lo + 1)
                slots.append((w + b, b))
                pos = int(before[b] + hi)
                b += 1
        assert all(got[b] == list(range(tiles[b])) for b in range(batch))
        assert len({s for s, _ in slots}) == len(slots) and max(s for s, _ in slots) < shares + batch
        for b in range(batch):
            mine = [s for s, x in slots if x == b]
            assert mine == ([] if not tiles[b] else list(range(where[b][0], where[b][0] + where[b][1])))


def test_spare_shares_cut_each_sequence_evenly():
    """Where there are at least twice as many shares as sequences, each share is a stretch of one: every tile is covered once, no
    stretch is longer than the common bound, and the shares suffice."""
    rng = random.Random(5)
    for _ in range(300):
        batch = rng.choice([1, 2, 7, 64, 255])
        shares = rng.randint(2 * batch, 511) if 2 * batch <= 511 else 511
        tiles = [rng.choice([0, 1, 1, 5, rng.randint(1, 40000)]) for _ in range(batch)]
        total = sum(tiles)
        per = max(4, -(-total // (shares - batch)))
        counts = [-(-t // per) for t in tiles]
        before = np.concatenate([[0], np.cumsum(counts)])
        assert before[-1] <= shares
        got = [[] for _ in range(batch)]
        for share in range(int(before[-1])):
            b = int(np.searchsorted(before, share, side="right")) - 1
            i, n = share - int(before[b]), counts[b]
            lo, hi = i * tiles[b] // n, (i + 1) * tiles[b] // n
            assert 0 < hi - lo <= per
            got[b].append((lo, hi))
        for b in range(batch):
            edges = [0] + [hi for _, hi in got[b]]
            assert edges[-1] == tiles[b] and [lo for lo, _ in got[b]] == edges[:-1]


@pytest.mark.parametrize("kv_heads", [1, 2, 4, 8, 16, 64, 256])
def test_folded_rows_are_taken_once_and_balanced(kv_heads):
    """Where workgroups of many rows share CUs in pairs, every sequence's tiles are each some workgroup's, and a single sequence's pairs
    have equal sums (the kernel's arithmetic, in Python)."""
    fold = 256 // kv_heads
    for batch in (1, 2, 3, 4, 7, 16):
        for tiles in range(1, 2 * fold // batch + 1):
            if not fold < tiles * batch <= 2 * fold:
                continue
            at = []
            for b in range(batch):
                row = []
                for place in range(tiles):
                    tile = tiles - 1 - place
                    if batch > 1:
                        if b * tiles >= fold:
                            tile = place
                    else:
                        shared = tiles - fold
                        tile = 2 * shared - 1 - place if place < shared else tiles - 1 - (place - shared) if place < fold else place - fold
                    row.append(tile)
                assert sorted(row) == list(range(tiles))
                at += row
            if batch == 1:
                pairs = {at[i] + at[i + fold] for i in range(tiles - fold)}
                assert pairs == {2 * (tiles - fold) - 1}
