"""Eviction from the cache on the GPU, against choices made one sequence and head at a time on the host: everything is moved or counted, so
every result has to be equal. Every head size and number of bits, own and other pages, ties, sums that are no numbers, lengths from zero
to ones that do not fit the registers, wrong lengths and pages."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_24875_amd as pkg  # noqa: E402

DEV = torch.device("cuda:0")
NAN, INF = math.nan, math.inf


def _gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _fill(cache, seed=1):
    """Rubbish in every byte of the pool, offsets and steps being numbers."""
    for i, t in enumerate((cache.k, cache.v, cache.k_par, cache.v_par)):
        if t is not None:
            if t.dtype is torch.uint8:
                t.copy_(torch.randint(0, 256, t.shape, generator=_gen(seed + i), device=DEV).to(torch.uint8))
            else:
                t.copy_(torch.randn(t.shape, generator=_gen(seed + i), device=DEV))


def _chosen(sums, n, keep, recent, first):
    """Indices that stay, ascending, from one row of sums on the host."""
    if n <= keep:
        return list(range(n))
    key = [math.inf if math.isnan(x) else x for x in sums]
    middle = sorted(range(first, n - recent), key=lambda j: (not math.isnan(sums[j]), -key[j], j))
    return sorted([*range(first), *middle[:keep - first - recent], *range(n - recent, n)])


def _check(cache, pages, lens, sums, keep, recent=0, first=0, to_pages=None, in_place=False, max_len=None):
    """Runs the call and compares everything that it may and may not have changed."""
    pools = [t for t in (cache.k, cache.v, cache.k_par, cache.v_par) if t is not None]
    before = [t.clone() for t in pools]
    old_sums, old_lens = sums.clone(), lens.clone()
    width = max_len if max_len is not None else min(pages.shape[1] * cache.page_size, sums.shape[2])
    out = dict(sums_out=sums, lens_out=lens) if in_place else {}
    new_lens, new_sums, kept = pkg.kv_evict(cache, pages, lens, sums, keep, recent, first, to_pages=to_pages, max_len=max_len, **out)
    torch.cuda.synchronize()
    assert (new_sums is sums and new_lens is lens) if in_place else (torch.equal(sums.isnan(), old_sums.isnan()) and torch.equal(lens, old_lens))
    ps, kv, heads = cache.page_size, cache.kv_heads, sums.shape[1]
    want_pools = [t.clone() for t in before]
    want_kept = torch.full((len(lens), heads, keep), -1, dtype=torch.int32)
    want_sums = torch.zeros(len(lens), heads, new_sums.shape[2])
    hp, ht, hs = pages.tolist(), (pages if to_pages is None else to_pages).tolist(), old_sums.cpu()
    for b, n in enumerate(old_lens.tolist()):
        for h in range(heads):
            c = _chosen(hs[b, h, :n].tolist(), n, keep, recent, first)
            want_kept[b, h, :len(c)] = torch.tensor(c, dtype=torch.int32)
            want_sums[b, h, :len(c)] = hs[b, h, c]
            if not c:
                continue
            src = torch.tensor([hp[b][j // ps] * ps + j % ps for j in c], device=DEV)
            dst = torch.tensor([ht[b][i // ps] * ps + i % ps for i in range(len(c))], device=DEV)
            for kh in (range(kv) if heads == 1 else (h,)):
                for w, t in zip(want_pools, before):
                    w[dst // ps, kh, dst % ps] = t[src // ps, kh, src % ps]
    assert torch.equal(new_lens.cpu(), old_lens.clamp_max(keep).cpu())
    assert torch.equal(kept.cpu(), want_kept)
    got = new_sums.cpu()
    assert torch.equal(got.isnan(), want_sums.isnan()) and torch.equal(got.nan_to_num(7.0), want_sums.nan_to_num(7.0))
    assert new_sums.shape[2] == (sums.shape[2] if in_place else width)
    for t, w in zip(pools, want_pools):
        assert torch.equal(t.view(torch.uint8), w.view(torch.uint8))
    return new_lens, new_sums, kept


def _setup(dim, bits, page, lens, kv=2, heads=2, keep=20, seed=1, ties=False):
    cols = max(1, -(-max(max(lens), 1) // page))
    b, new = len(lens), -(-keep // page)
    cache = pkg.KVCache.empty(b * (cols + new) + 1, kv, dim, page_size=page, bits=bits)
    _fill(cache, seed)
    order = torch.randperm(b * (cols + new), generator=_gen(seed), device=DEV).int()
    pages, to = order[:b * cols].view(b, cols), order[b * cols:].view(b, new)
    sums = torch.rand((b, heads, cols * page), generator=_gen(seed + 9), device=DEV)
    if ties:
        sums = (sums * 4).floor()
    return cache, pages, to, _i32(lens), sums


@pytest.mark.parametrize("within", [True, False])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim,page,kv,heads", [(64, 16, 2, 2), (96, 8, 3, 1), (128, 64, 2, 2), (192, 1, 2, 2), (256, 32, 1, 1)])
def test_every_head_size(dim, page, kv, heads, bits, within):
    cache, pages, to, lens, sums = _setup(dim, bits, page, [70, 0, 21, 20, 1, 53], kv, heads)
    _check(cache, pages, lens, sums, 20, 5, 2, None if within else to, in_place=within)


@pytest.mark.parametrize("within", [True, False])
@pytest.mark.parametrize("keep,recent,first", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (40, 40, 0), (40, 20, 20), (40, 0, 40), (99, 3, 3), (100, 50, 4), (130, 7, 7)])
def test_shares_of_the_kept(keep, recent, first, within):
    """Only the ends kept, only one token, all but one, all."""
    cache, pages, to, lens, sums = _setup(64, 8, 16, [100, 41, 40, 129], keep=keep, ties=True)
    _check(cache, pages, lens, sums, keep, recent, first, None if within else to, in_place=within)


@pytest.mark.parametrize("n,keep", [(1024, 1000), (1025, 512), (5000, 1), (5000, 4999), (16384, 7000), (16399, 5), (20001, 10000), (66000, 33000), (70001, 69990)])
@pytest.mark.parametrize("ties", [False, True])
def test_long_rows(n, keep, ties):
    """Sums in registers and read again, few and nearly all kept, in place; with ties at the last kept one."""
    cache, pages, to, lens, sums = _setup(64, 4, 64, [n, n // 3], 1, 1, keep=keep, ties=ties)
    _check(cache, pages, lens, sums, keep, min(keep // 3, 40), min(keep // 3, 4), in_place=True)


@pytest.mark.parametrize("values", [[0.0], [-0.0, 0.0], [NAN], [INF, -INF], [NAN, INF, 1.0, 0.0, -0.0, -1.0, -INF, 1e-45, -1e-45, 3.4e38, -3.4e38],
                                    [-INF], [-3.4e38, -INF], [1.0, 1.0000001, 0.99999994]])
def test_sums_of_any_kind(values):
    cache, pages, to, lens, sums = _setup(64, 16, 16, [200, 57, 33], keep=32)
    pick = torch.randint(0, len(values), sums.shape, generator=_gen(3), device=DEV)
    sums = torch.tensor(values, device=DEV)[pick]
    _check(cache, pages, lens, sums, 32, 4, 2, to)
    for m in (1, 5, 31):
        _check(cache, pages, lens, sums.clone(), m, 0, 0)


def test_sums_and_tables_of_any_strides():
    cache, pages, to, lens, sums = _setup(96, 8, 16, [60, 33, 9], kv=3, heads=3)
    wide = torch.rand((3, 3, 90), generator=_gen(5), device=DEV)
    view = wide[..., 7:7 + 64].transpose(0, 1)                       # heads' rows first
    table = torch.full((3, 9), 10 ** 8, dtype=torch.int32, device=DEV)
    table[:, 2:2 + pages.shape[1]] = pages
    rows = torch.zeros(3, 5, 40, device=DEV)
    out = pkg.kv_evict(cache, table[:, 2:2 + pages.shape[1]], lens, view, 20, 3, 1, to_pages=to, sums_out=rows[:, 1:4, 5:30])
    again = pkg.kv_evict(cache, pages, lens, view.contiguous(), 20, 3, 1, to_pages=to)
    assert torch.equal(out[1][..., :20], again[1][..., :20]) and torch.equal(out[2], again[2]) and torch.equal(out[0], again[0])
    assert not rows[:, 0].any() and not rows[:, 4].any() and not rows[..., :5].any() and not rows[..., 25:].any()
    _check(cache, pages, lens, wide[..., 7:7 + 64], 20, 3, 1, in_place=True)


def test_pools_of_other_orders():
    """Keys and values in one allocation, tokens before heads."""
    buf = torch.zeros((2, 12, 16, 2, 64), dtype=torch.float16, device=DEV)
    cache = pkg.KVCache(buf[0].transpose(1, 2), buf[1].transpose(1, 2))
    _fill(cache)
    pages = torch.randperm(12, generator=_gen(2), device=DEV).int()[:8].view(2, 4)
    sums = torch.rand((2, 2, 64), generator=_gen(4), device=DEV)
    _check(cache, pages, _i32([64, 37]), sums, 24, 6, 2, in_place=True)


def test_shared_pages_are_only_read():
    """Two sequences of the same pages go to their own ones."""
    cache, pages, to, lens, sums = _setup(64, 8, 16, [60, 60])
    pages = pages[:1].expand(2, -1).contiguous()
    _check(cache, pages, lens, sums, 20, 3, 1, to)


def test_wrong_lengths_and_pages():
    cache, pages, to, lens, sums = _setup(64, 16, 16, [60, 60, 60, 60], heads=1)
    pools = cache.k.clone(), cache.v.clone()
    bad = _i32([-1, 60, 65, 2 ** 31 - 1])
    new, ns, kept = pkg.kv_evict(cache, pages, bad, sums, 20, 3, 1)
    assert new.tolist() == [-1, 20, 65, 2 ** 31 - 1] and (kept[[0, 2, 3]] == -1).all() and ns[[0, 2, 3]].isnan().all() and ns[1].isfinite().all()
    for t, w in zip((cache.k, cache.v), pools):
        changed = (t != w).any(dim=3).any(dim=2).any(dim=1)
        assert set(changed.nonzero().flatten().tolist()) <= set(pages[1].tolist())
    # tokens of a page outside the pool are NaN in their new place; a page outside receives nothing
    for bits in (16, 8, 4):
        for within in (True, False):
            cache, pages, to, lens, sums = _setup(64, bits, 16, [60, 60], keep=20, heads=1)
            pages[0, 2], to[1, 1] = 10 ** 9, -5
            before = cache.k.clone()
            new, _, kept = pkg.kv_evict(cache, pages, lens, sums, 20, 3, 1, to_pages=None if within else to)
            table = pages if within else to
            i = torch.arange(20, device=DEV)
            k, v = pkg.kv_read(cache, (table[0].long()[i // 16] * 16 + i % 16).int())
            lost = (kept[0, 0] >= 32) & (kept[0, 0] < 48)
            assert lost.any() and k[lost].isnan().all() and v[lost].isnan().all() and k[~lost].isfinite().all()
            if not within:
                assert torch.equal(cache.k[pages[1].long()], before[pages[1].long()])


def test_no_sequences_and_no_tokens():
    cache = pkg.KVCache.empty(2, 2, 64, page_size=16)
    lens, sums, kept = pkg.kv_evict(cache, torch.zeros((0, 3), dtype=torch.int32, device=DEV), _i32([]), torch.zeros((0, 2, 48), device=DEV), 8)
    assert lens.shape == (0,) and sums.shape == (0, 2, 48) and kept.shape == (0, 2, 8)
    lens, sums, kept = pkg.kv_evict(cache, torch.zeros((2, 0), dtype=torch.int32, device=DEV), _i32([0, 0]), torch.zeros((2, 1, 0), device=DEV), 8)
    assert lens.tolist() == [0, 0] and sums.shape == (2, 1, 0) and (kept == -1).all()


def test_evicted_caches_attend_over_what_was_kept():
    """Attention over the shrunk cache is, bit for bit, that over a cache that never held the others."""
    cache, pages, to, lens, sums = _setup(128, 8, 16, [70, 45], keep=32)
    q = torch.randn((2, 8, 128), generator=_gen(6), device=DEV).half()
    _, _, kept = pkg.kv_evict(cache, pages, lens, sums, 32, 8, 2, to_pages=to)
    o = pkg.attention(q, cache, to, _i32([32, 32]))
    fresh = pkg.KVCache.empty(4, 2, 128, page_size=16, bits=8)
    for b in range(2):
        for h in range(2):
            j = kept[b, h].long()
            src, i = pages[b].long()[j // 16], torch.arange(32, device=DEV)
            for f, t in ((fresh.k, cache.k), (fresh.v, cache.v), (fresh.k_par, cache.k_par), (fresh.v_par, cache.v_par)):
                f[2 * b + i // 16, h, i % 16] = t[src, h, j % 16]
    assert torch.equal(o, pkg.attention(q, fresh, _i32([[0, 1], [2, 3]]), _i32([32, 32])))


def test_streams_and_graphs():
    """A captured eviction within the pages, replayed after tokens were added each time, against eager calls on a copy."""
    cache, pages, to, lens, sums = _setup(64, 16, 16, [60, 44], keep=20)
    twin = pkg.KVCache(cache.k.clone(), cache.v.clone())
    lens2, sums2 = lens.clone(), sums.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = pkg.kv_evict(twin, pages, lens2.clone(), sums2.clone(), 20, 3, 1, to_pages=to, stream=side)
    side.synchronize()
    b = pkg.kv_evict(twin, pages, lens2.clone(), sums2.clone(), 20, 3, 1, to_pages=to)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    twin.k.copy_(cache.k), twin.v.copy_(cache.v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, _, kept = pkg.kv_evict(cache, pages, lens, sums, 20, 3, 1, lens_out=lens, sums_out=sums)
    for step in range(4):
        graph.replay()
        _, _, want = pkg.kv_evict(twin, pages, lens2, sums2, 20, 3, 1, lens_out=lens2, sums_out=sums2)
        assert torch.equal(kept, want) and torch.equal(lens, lens2) and torch.equal(sums, sums2) and torch.equal(cache.k, twin.k)
        assert torch.equal(cache.v, twin.v)
        more = torch.rand((2, 2, 30), generator=_gen(step), device=DEV)
        for x, y in ((sums, lens), (sums2, lens2)):
            x[..., 20:50] = more
            y += 30
        torch.cuda.synchronize()
