"""Eviction on the GPU, what else its arguments allow. Choices on the host, pools and sums are test_gpu_evict's."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_24875_amd as pkg  # noqa: E402

from test_gpu_evict import _chosen, _setup  # noqa: E402


def _bytes(t):
    return t.contiguous().view(torch.uint8)


@pytest.mark.parametrize("n,keep", [(60, 20), (60, 60), (1025, 512), (20001, 10000), (70001, 3)])
@pytest.mark.parametrize("within", [True, False])
@pytest.mark.parametrize("heads", [1, 2])
def test_what_is_given_stays_as_it_is(n, keep, within, heads):
    """Sums, lengths and tables are read only where results go elsewhere, byte by byte: sums with NaN of several kinds and zeros of both signs."""
    cache, pages, to, lens, sums = _setup(64, 8, 16, [n, n // 3, 0], 2, heads, keep=keep)
    sums[:, :, ::7] = -0.0
    sums[:, :, 3::11] = math.nan
    sums.view(torch.int32)[:, :, 4::13] = 0x7FC01234
    given = [sums, lens, pages, to]
    old = [t.clone() for t in given]
    new_lens, new_sums, kept = pkg.kv_evict(cache, pages, lens, sums, keep, min(5, keep // 3), min(2, keep // 3), to_pages=None if within else to)
    torch.cuda.synchronize()
    for t, w in zip(given, old):
        assert torch.equal(_bytes(t), _bytes(w))
    # (kept sums are moved, not computed: their bytes, too)
    hs = old[0].cpu()
    for b, m in enumerate(old[1].tolist()):
        for h in range(heads):
            c = _chosen(hs[b, h, :m].tolist(), m, keep, min(5, keep // 3), min(2, keep // 3))
            assert torch.equal(_bytes(new_sums[b, h, :len(c)].cpu()), _bytes(hs[b, h, c]))
