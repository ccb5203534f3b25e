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


@pytest.mark.parametrize("keep", [80, 81, 1000, 1 << 20, 1 << 30])
@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("within", [True, False])
def test_room_for_more_than_there_is(keep, heads, within):
    """A budget that no sequence can pass changes nothing, takes no more memory than the cache's length asks for, and says of each token that it was kept."""
    cache, pages, to, lens, sums = _setup(64, 16, 16, [80, 0, 33], 2, heads, keep=80)
    lens[2] = 81                                  # (a wrong one: left alone)
    pools = [cache.k.clone(), cache.v.clone()]
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    new_lens, new_sums, kept = pkg.kv_evict(cache, pages, lens, sums, keep, min(keep, 90), 4 if keep > 100 else 0, to_pages=None if within else to)
    torch.cuda.synchronize()
    assert torch.cuda.max_memory_allocated() - before < 1 << 16
    assert kept.shape == (3, heads, 80) and new_lens.tolist() == [80, 0, 81]
    assert torch.equal(kept[0], torch.arange(80, dtype=torch.int32, device=kept.device).expand(heads, -1)) and (kept[1:] == -1).all()
    assert torch.equal(_bytes(new_sums[0]), _bytes(sums[0])) and not new_sums[1].any() and new_sums[2].isnan().all()
    if within:
        assert all(torch.equal(_bytes(x), _bytes(y)) for x, y in zip((cache.k, cache.v), pools))
    else:
        for x, y in zip((cache.k, cache.v), pools):
            assert torch.equal(x[to[0].long()], y[pages[0].long()]) and torch.equal(x[pages.long()], y[pages.long()])
            assert torch.equal(x[to[1:].long()], y[to[1:].long()])


def test_room_where_there_is_no_token():
    cache, pages, to, lens, sums = _setup(64, 16, 16, [0, 0], 2, 2, keep=20)
    new_lens, new_sums, kept = pkg.kv_evict(cache, pages, lens, sums, 1 << 30, 7, 3, max_len=0)
    assert new_lens.tolist() == [0, 0] and new_sums.shape == (2, 2, 0) and kept.shape == (2, 2, 1) and (kept == -1).all()
