"""CPU checks of the accumulated attention weights: refusals of the C ABI and of the binding before any HIP call."""
from __future__ import annotations

import ctypes
import math
import os

import pytest

import paper_2609_24875_amd as pkg
from paper_2609_24875_amd import attn as A

torch = pytest.importorskip("torch")

needs_lib = pytest.mark.skipif(not os.path.exists(pkg.LIB_PATH), reason="libsph.so not built")
OK, NULL, SHAPE, FORMAT, VALUE, SMALL = 0, 1, 2, 3, 5, 6
P = 1 << 20                                       # stands for a device pointer; no call here gets as far as using one


@needs_lib
@pytest.mark.parametrize("args,want", [
    (dict(batch=-1), SHAPE), (dict(batch=65537), SHAPE), (dict(tokens=-1), SHAPE), (dict(q_heads=0), SHAPE), (dict(q_heads=7), SHAPE),
    (dict(heads=0), SHAPE), (dict(heads=3), SHAPE), (dict(max_q=0), SHAPE), (dict(max_q=1 << 25), SHAPE), (dict(max_len=-1), SHAPE),
    (dict(max_len=(1 << 30) + 1), SHAPE), (dict(window=-1), SHAPE), (dict(scale=math.nan), VALUE), (dict(scale=math.inf), VALUE),
    (dict(start=None, max_q=2), SHAPE), (dict(start=None, tokens=3), SHAPE), (dict(cols=3), SHAPE), (dict(cols=1 << 31), SHAPE),
    (dict(qt=1028), SHAPE), (dict(qh=-128), SHAPE), (dict(bs=-1), SHAPE), (dict(bh=1 << 40), SHAPE), (dict(os=63), SHAPE), (dict(oh=0), SHAPE),
    (dict(os=64, oh=64), SHAPE), (dict(q=None), NULL), (dict(lse=None), NULL), (dict(pages=None), NULL), (dict(lens=None), NULL),
    (dict(out=None), NULL), (dict(q=P + 8), SHAPE), (dict(start=P + 2), SHAPE), (dict(pages=P + 1), SHAPE), (dict(lens=P + 2), SHAPE),
    (dict(lse=P + 2), SHAPE), (dict(before=P + 2), SHAPE), (dict(out=P + 2), SHAPE), (dict(ws=P + 128), SHAPE),
    (dict(before=P + 4096, bs=256), SHAPE), (dict(max_q=40, heads=1, oh=0, ws=None), NULL), (dict(max_q=40, heads=1, nws=1023), SMALL),
    (dict(bits=5), FORMAT), (dict(cache=False), NULL), (dict(batch=0, lens=None), OK), (dict(max_len=0, out=None), OK)])
def test_refusals(args, want):
    a = dict(bits=8, cache=True, batch=2, tokens=2, q_heads=8, q=P, qt=1024, qh=128, start=P, max_q=1, pages=P, cols=4, lens=P, max_len=64,
             window=0, scale=1.0, lse=P, heads=2, before=None, bs=128, bh=64, out=P + 4096, os=128, oh=64, ws=P, nws=1 << 30)
    a.update(args)
    c = A.CKVCache(a["bits"], 2, 128, 16, 8, P, P, 4096, 2048, 128, P, P, 512, 256, 16)
    st = A._library().sph_attention_weights(ctypes.byref(c) if a["cache"] else None, a["batch"], a["tokens"], a["q_heads"], a["q"], a["qt"],
                                            a["qh"], a["start"], a["max_q"], a["pages"], a["cols"], a["lens"], a["max_len"], a["window"],
                                            a["scale"], a["lse"], a["heads"], a["before"], a["bs"], a["bh"], a["out"], a["os"], a["oh"],
                                            a["ws"], a["nws"], None)
    assert st == want


@needs_lib
def test_workspace_is_the_parts():
    """One number a kv head, part of the rows and token, where more than one are added; none for few rows."""
    lib, n = A._library(), ctypes.c_size_t(7)
    c = A.CKVCache(8, 2, 128, 16, 1 << 16, P, P, 4096, 2048, 128, P, P, 512, 256, 16)
    r = ctypes.byref(c)

    def need(batch, heads, max_q, max_len):
        assert lib.sph_attention_weights_workspace_bytes(r, batch, 1 << 20, 8, heads, max_q, max_len, 0, ctypes.byref(n)) == OK
        return n.value
    assert need(4, 1, 8, 5000) == need(4, 2, 8, 5000) == 0
    assert need(4, 1, 9, 100000) == 4 * 2 * 100000 * 4               # both heads' sums; the keys alone fill the chip
    assert need(4, 2, 9, 100000) == 0
    assert need(1, 2, 2048, 1000) == 2 * 32 * 1000 * 4               # 2 heads of 4 tiles of keys: 8192 rows in 32 parts of 256
    assert need(0, 1, 40, 64) == need(1, 1, 40, 0) == 0
    assert lib.sph_attention_weights_workspace_bytes(r, 1, 1, 8, 1, 1, 64, 0, None) == NULL
    assert lib.sph_attention_weights_workspace_bytes(r, 65536, 1, 8, 2, 1, 1 << 20, 0, ctypes.byref(n)) == SHAPE


@needs_lib
def test_binding_refusals():
    cache = pkg.KVCache.empty(8, 2, 64, page_size=16, device="cpu")
    i32 = dict(dtype=torch.int32)
    base = dict(q=torch.zeros(3, 8, 64).half(), pages=torch.zeros(3, 2, **i32), seq_lens=torch.zeros(3, **i32), lse=torch.zeros(3, 8))
    for kw, err in ((dict(q=base["q"].float()), TypeError), (dict(q=base["q"][..., :32]), ValueError), (dict(pages=base["pages"].long()), TypeError),
                    (dict(pages=base["pages"][:2]), ValueError), (dict(seq_lens=torch.zeros(3)), TypeError), (dict(lse=base["lse"].half()), TypeError),
                    (dict(lse=base["lse"][:2]), ValueError), (dict(lse=torch.zeros(8, 3).t()), ValueError), (dict(lse=None), TypeError),
                    (dict(max_len=33), ValueError), (dict(before=torch.zeros(3, 1, 32)), ValueError), (dict(before=torch.zeros(3, 2, 31)), ValueError),
                    (dict(before=torch.zeros(3, 2, 32).half()), TypeError), (dict(per_head=False, out=torch.zeros(3, 2, 32)), ValueError),
                    (dict(out=torch.zeros(3, 32, 2).transpose(1, 2)), ValueError), (dict(q_start=torch.zeros(3, **i32)), ValueError), (dict(), ValueError)):
        with pytest.raises(err):                  # (the last: right, but not on a GPU)
            pkg.attention_weights(**{"cache": cache, **base, **kw})
