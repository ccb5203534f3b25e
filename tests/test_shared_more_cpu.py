"""CPU checks of the workspace of the attention behind shared prefixes."""
from __future__ import annotations

import ctypes
import os

import pytest

import paper_2609_24875_amd as pkg
from paper_2609_24875_amd import attn as A

needs_lib = pytest.mark.skipif(not os.path.exists(pkg.LIB_PATH), reason="libsph.so not built")
P = 1 << 20                                       # stands for a device pointer; no call here gets as far as using one


def _need(prefixes, max_group, max_prefix, batch, tokens, q_heads, max_q, max_len, dim=128, kv=2, bits=8):
    c = A.CKVCache(bits, kv, dim, 16, 1 << 16, P, P, 4096 * kv, 4096, 256, P, P, 512 * kv, 512, 32)
    n = ctypes.c_size_t(7)
    st = A._library().sph_attention_shared_workspace_bytes(ctypes.byref(c), prefixes, max_group, max_prefix, batch, tokens, q_heads, max_q, max_len,
                                                           ctypes.byref(n))
    assert st == 0
    return n.value


@needs_lib
@pytest.mark.parametrize("prefixes", [2, 63, 64, 1000])
def test_room_for_what_becomes_of_many_starts(prefixes):
    """A part for every own and every prefix's row, a pair of numbers for every sequence and prefix, and where prefixes are more than a wave looks at
    at once one pair more."""
    row, batch = (128 + 2) * 4, 4
    rows = batch * 8 + prefixes * 2 * 16             # rows of all own parts; of the prefixes', two kv heads, four sequences of four heads
    assert _need(prefixes, 4, 64, batch, batch, 8, 1, 64) == rows * row + (batch + prefixes) * 8 + (8 if prefixes > 63 else 0)
