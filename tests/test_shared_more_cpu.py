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


@needs_lib
@pytest.mark.parametrize("batch,chunk", [(64, 4096), (128, 4096), (1, 300)])
def test_prompts_beside_single_tokens_have_a_part_for_every_row(batch, chunk):
    """One prompt and a token each of the other sequences: parts for the rows that there are, not for as many as the longest's of every sequence."""
    row, tokens = (128 + 2) * 4, chunk + batch - 1
    for max_prefix, max_len in ((1024, 8192), (1, 8192)):
        need = _need(1, batch, max_prefix, batch, tokens, 32, chunk, max_len, kv=8)
        parts, rest = divmod(need - (batch + 1) * 8, 32 * tokens * row)
        # one for the own tokens and one for the prefix; a single sequence's few rows are cut for the chip's sake
        assert rest == 0 and (parts == 2 or batch == 1 and 2 < parts < 64)
