"""CPU checks of rotary positions with several axes: the axes' shares of the pairs, and refusals of the C ABI and of the
binding before any HIP call."""
from __future__ import annotations

import ctypes
import os

import pytest

import paper_2609_24875_amd as pkg
from paper_2609_24875_amd import attn as A

torch = pytest.importorskip("torch")

needs_lib = pytest.mark.skipif(not os.path.exists(pkg.LIB_PATH), reason="libsph.so not built")
OK, NULL, SHAPE = 0, 1, 2
P = 1 << 20                                       # stands for a device pointer; no call here gets as far as using one


def test_axes_take_their_shares_of_the_pairs():
    def of(*a, **k):
        t = pkg.rope_axes(*a, device="cpu", **k)
        assert t.dtype is torch.uint8
        return t.tolist()
    assert of([2, 3, 3]) == [0, 0, 1, 1, 1, 2, 2, 2]
    assert of([2, 3, 3], cycled=True) == [0, 1, 2, 0, 1, 2, 1, 2]
    assert of([8]) == [0] * 8
    assert of([0, 8]) == [1] * 8
    assert of((16, 24, 24))[15:17] == [0, 1]
    for wrong in ([], [4, 3], [0], [-8, 16], [0.5, 7.5], [1] * 17, [4]):
        with pytest.raises(ValueError):
            pkg.rope_axes(wrong, device="cpu")


@needs_lib
def test_table_of_given_frequencies_refusals():
    with pytest.raises(ValueError):
        pkg.rope_table(32, 10, device="cpu", frequencies=[1.0] * 15)
    with pytest.raises(ValueError):
        pkg.rope_table(32, 10, device="cpu", frequencies=[1.0] * 16, base=100.0)


def _cache():
    return A.CKVCache(8, 2, 128, 16, 4, P, P, 4096, 2048, 128, P, P, 512, 256, 16)


FAULTS = [(dict(axes=None), NULL), (dict(axes=P + 4), SHAPE), (dict(n=0), SHAPE), (dict(n=17), SHAPE), (dict(n=-1), SHAPE),
          (dict(stride=-1), SHAPE), (dict(stride=1 << 40), SHAPE), (dict(pos=None), NULL), (dict(pos=P + 2), SHAPE), (dict(rope=None), NULL),
          (dict(rot=24), SHAPE), (dict(tokens=-1), SHAPE), (dict(tokens=0, pos=None), OK), (dict(tokens=0, axes=None), NULL)]


@needs_lib
@pytest.mark.parametrize("args,want", FAULTS)
def test_refusals(args, want):
    a = dict(axes=P, n=3, stride=2, pos=P, rope=True, rot=64, tokens=2)
    a.update(args)
    lib = A._library()
    r = ctypes.byref(A.CRope(P, 100, a["rot"], 0)) if a["rope"] else None
    assert lib.sph_rope_axes(r, a["axes"], a["n"], a["stride"], 0, a["tokens"], 8, 128, P, 1024, 128, a["pos"], P, 1024, 128, None) == want
    assert lib.sph_kv_append_axes(ctypes.byref(_cache()), r, a["axes"], a["n"], a["stride"], 0, a["tokens"], P, 256, 128, P, 256, 128, P,
                                  8, P, 1024, 128, P, 1024, 128, a["pos"], None) == want


@needs_lib
def test_binding_refusals():
    x, table = torch.zeros(4, 2, 64).half(), torch.zeros(10, 16, 2)
    pos, axes = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(16, dtype=torch.uint8)
    for kw, err in ((dict(axes=axes.int()), TypeError), (dict(axes=[0] * 16), TypeError), (dict(axes=axes[:8]), ValueError),
                    (dict(axes=torch.zeros(32, dtype=torch.uint8)[::2]), ValueError), (dict(axes=torch.zeros(24, dtype=torch.uint8)[1:17]), ValueError),
                    (dict(positions=pos.long()), TypeError), (dict(positions=pos[0]), ValueError), (dict(positions=pos[:, :3]), ValueError),
                    (dict(positions=torch.zeros(4, 3, dtype=torch.int32).t()), ValueError),
                    (dict(positions=torch.zeros(17, 4, dtype=torch.int32)), ValueError), (dict(positions=[0, 1]), TypeError), (dict(), ValueError)):
        a = dict(positions=pos, axes=axes)
        a.update(kw)                              # (the last: right, but not on a GPU)
        with pytest.raises(err):
            pkg.rope(x, a["positions"], table, axes=a["axes"])
    c = pkg.KVCache.empty(2, 2, 64, device="cpu")
    with pytest.raises(ValueError):
        pkg.kv_append(c, x, x, torch.zeros(4, dtype=torch.int32), axes=axes)
