"""CPU checks of the rotation's gradient: what autograd's hooks for saved tensors may hand back is refused before any pointer is used."""
from __future__ import annotations

import os

import pytest

import paper_2609_24875_amd as pkg
from paper_2609_24875_amd import attn as A

torch = pytest.importorskip("torch")

needs_lib = pytest.mark.skipif(not os.path.exists(pkg.LIB_PATH), reason="libsph.so not built")


@needs_lib
@pytest.mark.parametrize("several", [False, True])
def test_tensors_that_came_back_otherwise_are_refused(several):
    i32 = dict(dtype=torch.int32)
    base = dict(grad=torch.zeros(5, 2, 64), positions=torch.zeros((3, 5) if several else 5, **i32), table=torch.zeros(7, 32, 2),
                axes=torch.zeros(32, dtype=torch.uint8) if several else None)
    wide = torch.zeros((3, 10) if several else 10, **i32)
    cases = [(dict(table=base["table"].half()), TypeError), (dict(table=torch.zeros(32, 7, 2).transpose(0, 1)), ValueError), (dict(table=torch.zeros(7, 64)), ValueError),
             (dict(table=torch.zeros(7, 16, 4)), ValueError), (dict(positions=base["positions"].long()), TypeError),
             (dict(positions=base["positions"].float()), TypeError), (dict(positions=wide[..., ::2]), ValueError), (dict(positions=wide[..., :4]), ValueError)]
    if several:
        cases += [(dict(positions=wide[0, :5]), ValueError), (dict(axes=base["axes"].int()), TypeError), (dict(axes=base["axes"][:16]), ValueError),
                  (dict(axes=torch.zeros(64, dtype=torch.uint8)[::2]), ValueError)]
    else:
        cases += [(dict(positions=wide.view(2, 5)), ValueError)]
    for kw, err in cases:
        with pytest.raises(err):
            A.rope_gradient(**{**base, **kw}, interleaved=False)
