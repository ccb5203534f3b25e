"""The rotation's gradient on the GPU where hooks keep what the forward pass saved somewhere else."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_24875_amd as pkg  # noqa: E402
from paper_2609_24875_amd import train  # noqa: E402

DEV = torch.device("cuda:0")


def _inputs(several, tokens=37):
    g = torch.Generator(DEV).manual_seed(3)
    x, dy = (torch.randn((tokens, 3, 64), generator=g, device=DEV) for _ in range(2))
    pos = torch.randint(0, 50, (3, tokens) if several else (tokens,), generator=g, device=DEV).int()
    return x.requires_grad_(), dy, pos, pkg.rope_table(64, 50), pkg.rope_axes([8, 12, 12]) if several else None


@pytest.mark.parametrize("tokens", [1, 37])
@pytest.mark.parametrize("several", [False, True])
def test_saved_on_the_host_and_back(several, tokens):
    x, dy, pos, table, axes = _inputs(several, tokens)
    want, = torch.autograd.grad(train.rope(x, pos, table, axes=axes), x, dy)
    with torch.autograd.graph.save_on_cpu():
        y = train.rope(x, pos, table, axes=axes)
    got, = torch.autograd.grad(y, x, dy)
    assert torch.equal(got, want)
    # (strided positions, which come back without their gaps)
    wide = torch.zeros((3, tokens + 9) if several else (tokens,), dtype=torch.int32, device=DEV)
    wide[..., :tokens] = pos
    with torch.autograd.graph.save_on_cpu():
        y = train.rope(x, wide[..., :tokens], table, axes=axes)
    got, = torch.autograd.grad(y, x, dy)
    assert torch.equal(got, want)


@pytest.mark.parametrize("several", [False, True])
def test_saved_as_something_else_is_refused(several):
    x, dy, pos, table, axes = _inputs(several)
    for unpack, err in ((lambda t: t.half() if t.is_floating_point() else t, TypeError), (lambda t: t.cpu(), ValueError),
                        (lambda t: t.long() if t.dtype is torch.int32 else t, TypeError), (lambda t: t[..., :1] if t.dtype is torch.int32 else t, ValueError)):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
            y = train.rope(x, pos, table, axes=axes)
        with pytest.raises(err):
            torch.autograd.grad(y, x, dy)
