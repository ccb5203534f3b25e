"""CPU checks of the attention behind shared prefixes: refusals of the C ABI and of the binding before any HIP call, and the workspace."""
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
    (dict(prefixes=0), SHAPE), (dict(prefixes=65537), SHAPE), (dict(max_group=0), SHAPE), (dict(max_group=65537), SHAPE),
    (dict(max_prefix=-1), SHAPE), (dict(max_prefix=(1 << 30) + 1), SHAPE), (dict(batch=-1), SHAPE), (dict(batch=65537), SHAPE),
    (dict(tokens=-1), SHAPE), (dict(q_heads=7), SHAPE), (dict(q_heads=0), SHAPE), (dict(max_q=0), SHAPE), (dict(max_len=-1), SHAPE),
    (dict(tokens=1 << 25, max_q=1 << 24), SHAPE), (dict(scale=math.nan), VALUE), (dict(start=None, max_q=2), SHAPE),
    (dict(start=None, tokens=5), SHAPE), (dict(first=None), SHAPE), (dict(first=None, prefixes=1, max_group=3), SHAPE), (dict(pstride=7), SHAPE),
    (dict(pstride=1 << 31), SHAPE), (dict(stride=3), SHAPE), (dict(qt=1028), SHAPE), (dict(oh=-128), SHAPE), (dict(ot=0), SHAPE), (dict(oh=0), SHAPE),
    (dict(q=None), NULL), (dict(o=None), NULL), (dict(lens=None), NULL), (dict(plens=None), NULL), (dict(pages=None), NULL), (dict(ppages=None), NULL),
    (dict(q=P + 8), SHAPE), (dict(o=P + 8), SHAPE), (dict(ws=P + 64), SHAPE), (dict(first=P + 2), SHAPE), (dict(ppages=P + 2), SHAPE),
    (dict(plens=P + 1), SHAPE), (dict(start=P + 2), SHAPE), (dict(pages=P + 2), SHAPE), (dict(lens=P + 2), SHAPE), (dict(lse=P + 2), SHAPE),
    (dict(ws=None), NULL), (dict(nws=1000), SMALL), (dict(bits=5), FORMAT), (dict(cache=False), NULL), (dict(batch=0, tokens=0, q=None), OK),
    (dict(tokens=0, lens=None), OK)])
def test_refusals(args, want):
    a = dict(bits=8, cache=True, prefixes=2, first=P, max_group=4, ppages=P, pstride=8, plens=P, max_prefix=128, batch=4, tokens=4, q_heads=8,
             q=P, qt=1024, qh=128, start=P, max_q=1, pages=P, stride=4, lens=P, max_len=64, scale=1.0, o=P, ot=1024, oh=128, lse=None, ws=P,
             nws=1 << 30)
    a.update(args)
    c = A.CKVCache(a["bits"], 2, 128, 16, 8, P, P, 4096, 2048, 128, P, P, 512, 256, 16)
    st = A._library().sph_attention_shared(ctypes.byref(c) if a["cache"] else None, a["prefixes"], a["first"], a["max_group"], a["ppages"],
                                           a["pstride"], a["plens"], a["max_prefix"], a["batch"], a["tokens"], a["q_heads"], a["q"], a["qt"],
                                           a["qh"], a["start"], a["max_q"], a["pages"], a["stride"], a["lens"], a["max_len"], a["scale"], a["o"],
                                           a["ot"], a["oh"], a["lse"], a["ws"], a["nws"], None)
    assert st == want


@needs_lib
def test_workspace_holds_the_parts():
    lib, n = A._library(), ctypes.c_size_t(7)
    c = A.CKVCache(8, 2, 128, 16, 1 << 16, P, P, 4096, 2048, 128, P, P, 512, 256, 16)

    def need(prefixes, max_group, max_prefix, batch, tokens, max_q, max_len):
        st = lib.sph_attention_shared_workspace_bytes(ctypes.byref(c), prefixes, max_group, max_prefix, batch, tokens, 8, max_q, max_len,
                                                      ctypes.byref(n))
        return n.value if st == OK else -st
    row = (128 + 2) * 4                                       # a row's sums, its maximum and its weight
    # short: one part for the own tokens, one for the prefix, a pair of numbers for every sequence and prefix
    assert need(1, 4, 64, 4, 4, 1, 64) == 2 * (4 * 8) * row + 5 * 8
    assert need(1, 4, 64, 0, 0, 1, 64) == 0
    # more sequences, more rows; longer ones, more parts
    assert need(1, 4, 64, 4, 4, 1, 64) < need(1, 8, 64, 8, 8, 1, 64) < need(1, 8, 1 << 16, 8, 8, 1, 64)
    assert need(65536, 65536, 1 << 20, 65536, 1 << 20, 16, 64) == -SHAPE
    assert lib.sph_attention_shared_workspace_bytes(ctypes.byref(c), 1, 1, 1, 1, 1, 8, 1, 1, None) == NULL


@needs_lib
def test_binding_refusals():
    cache = pkg.KVCache.empty(8, 2, 64, page_size=16, device="cpu")
    i32 = dict(dtype=torch.int32)
    base = dict(q=torch.zeros(3, 8, 64).half(), prefix_pages=torch.zeros(2, 4, **i32), prefix_lens=torch.zeros(2, **i32),
                pages=torch.zeros(3, 2, **i32), seq_lens=torch.zeros(3, **i32), first=torch.zeros(3, **i32))
    for kw, err in ((dict(q=base["q"].float()), TypeError), (dict(q=base["q"][..., :32]), ValueError), (dict(prefix_pages=base["prefix_pages"][:1]), ValueError),
                    (dict(prefix_pages=base["prefix_pages"].long()), TypeError), (dict(prefix_lens=torch.zeros(2)), TypeError), (dict(prefix_lens=[1, 2]), TypeError),
                    (dict(pages=base["pages"][:2]), ValueError), (dict(seq_lens=torch.zeros(3)), TypeError), (dict(first=torch.zeros(2, **i32)), ValueError),
                    (dict(first=None), ValueError), (dict(prefix_pages=base["prefix_pages"][:0], prefix_lens=base["prefix_lens"][:0]), ValueError),
                    (dict(q_start=torch.zeros(3, **i32)), ValueError), (dict(max_len=33), ValueError), (dict(max_prefix=65), ValueError),
                    (dict(out=torch.zeros(3, 8, 64)), TypeError), (dict(), ValueError)):
        with pytest.raises(err):                  # (the last: right, but not on a GPU)
            pkg.attention_shared(**{"cache": cache, **base, **kw})
