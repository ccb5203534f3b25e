"""CPU checks of the cache's eviction: refusals of the C ABI and of the binding before any HIP call."""
from __future__ import annotations

import ctypes
import os

import pytest

import paper_2609_24875_amd as pkg
from paper_2609_24875_amd import attn as A

torch = pytest.importorskip("torch")

needs_lib = pytest.mark.skipif(not os.path.exists(pkg.LIB_PATH), reason="libsph.so not built")
OK, NULL, SHAPE, FORMAT = 0, 1, 2, 3
P = 1 << 20                                       # stands for a device pointer; no call here gets as far as using one


@needs_lib
@pytest.mark.parametrize("args,want", [
    (dict(batch=-1), SHAPE), (dict(batch=65537), SHAPE), (dict(max_len=-1), SHAPE), (dict(max_len=(1 << 30) + 1), SHAPE), (dict(heads=0), SHAPE),
    (dict(heads=3), SHAPE), (dict(keep=0), SHAPE), (dict(keep=(1 << 30) + 1), SHAPE), (dict(recent=-1), SHAPE), (dict(first=-1), SHAPE),
    (dict(recent=20, first=13), SHAPE), (dict(recent=33), SHAPE), (dict(stride=3), SHAPE), (dict(stride=1 << 31), SHAPE), (dict(to_stride=1), SHAPE),
    (dict(width=31), SHAPE), (dict(width=(1 << 30) + 1), SHAPE), (dict(ss=-1), SHAPE), (dict(sh=1 << 40), SHAPE), (dict(ns=-64), SHAPE),
    (dict(nh=31), SHAPE), (dict(ns=32, nh=32), SHAPE), (dict(ns=0), SHAPE), (dict(lens=None), NULL), (dict(new_lens=None), NULL),
    (dict(kept=None), NULL), (dict(pages=None), NULL), (dict(to=None), NULL), (dict(sums=None), NULL), (dict(new=None), NULL),
    (dict(pages=P + 2), SHAPE), (dict(to=P + 1), SHAPE), (dict(sums=P + 2), SHAPE), (dict(new=P + 2), SHAPE), (dict(kept=P + 2), SHAPE),
    (dict(lens=P + 2), SHAPE), (dict(new=P, ns=256), SHAPE), (dict(new=P, sh=128, nh=200, ns=400), SHAPE), (dict(to=P, to_stride=5), SHAPE),
    (dict(bits=5), FORMAT), (dict(cache=False), NULL), (dict(batch=0, pages=None, lens=None), OK)])
def test_refusals(args, want):
    a = dict(bits=8, cache=True, batch=2, pages=P, stride=4, lens=P, max_len=64, sums=P, heads=2, ss=200, sh=100, keep=32, recent=8, first=4,
             to=P + 4096, to_stride=4, new_lens=P, new=P + 8192, width=32, ns=64, nh=32, kept=P)
    a.update(args)
    c = A.CKVCache(a["bits"], 2, 128, 16, 8, P, P, 4096, 2048, 128, P, P, 512, 256, 16)
    st = A._library().sph_kv_evict(ctypes.byref(c) if a["cache"] else None, a["batch"], a["pages"], a["stride"], a["lens"], a["max_len"], a["sums"],
                                   a["heads"], a["ss"], a["sh"], a["keep"], a["recent"], a["first"], a["to"], a["to_stride"], a["new_lens"],
                                   a["new"], a["width"], a["ns"], a["nh"], a["kept"], None)
    assert st == want


@needs_lib
def test_launches_past_their_bounds_are_refused():
    c = A.CKVCache(16, 1024, 64, 16, 8, P, P, 1 << 21, 2048, 128, None, None, 0, 0, 0)
    args = [ctypes.byref(c), 65536, P, 4, P, 64, P, 1024, 1 << 20, 64, 32, 8, 4, P + 4096, 4, P, P + 8192, 32, 1 << 20, 64, P, None]
    assert A._library().sph_kv_evict(*args) == SHAPE


@needs_lib
def test_binding_refusals():
    cache = pkg.KVCache.empty(8, 2, 64, page_size=16, device="cpu")
    i32 = dict(dtype=torch.int32)
    base = dict(pages=torch.zeros(3, 2, **i32), seq_lens=torch.zeros(3, **i32), sums=torch.zeros(3, 2, 32), keep=16)
    for kw, err in ((dict(pages=base["pages"].long()), TypeError), (dict(pages=base["pages"][:2]), ValueError), (dict(pages=base["pages"][0]), ValueError),
                    (dict(pages=torch.zeros(2, 3, **i32).t()), ValueError), (dict(pages=torch.zeros(1, 2, **i32).expand(3, 2)), ValueError),
                    (dict(seq_lens=[0, 0, 0]), TypeError), (dict(seq_lens=torch.zeros(3)), TypeError), (dict(sums=torch.zeros(3, 2, 32).double()), TypeError),
                    (dict(sums=torch.zeros(3, 3, 32)), ValueError), (dict(sums=torch.zeros(2, 2, 32)), ValueError), (dict(sums=torch.zeros(3, 32)), ValueError),
                    (dict(sums=torch.zeros(3, 32, 2).transpose(1, 2)), ValueError), (dict(max_len=33), ValueError),
                    (dict(sums=torch.zeros(3, 2, 20), max_len=24), ValueError), (dict(keep=0), ValueError), (dict(recent=10, first=7), ValueError),
                    (dict(recent=-1), ValueError), (dict(to_pages=torch.zeros(3, 0, **i32)), ValueError), (dict(to_pages=[1]), TypeError),
                    (dict(keep=20, to_pages=torch.zeros(3, 1, **i32)), ValueError), (dict(sums_out=torch.zeros(3, 1, 32)), ValueError),
                    (dict(sums_out=torch.zeros(3, 2, 15)), ValueError), (dict(lens_out=torch.zeros(2, **i32)), ValueError), (dict(), ValueError)):
        with pytest.raises(err):                  # (the last: right, but not on a GPU)
            pkg.kv_evict(cache, **{**base, **kw})
