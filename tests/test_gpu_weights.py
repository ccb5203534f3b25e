"""Accumulated attention weights on the GPU, against a plain implementation in 64 bits: every head size, number of bits and page size, single
tokens, drafts and prompts, windows, sums per head and over all, rows that see nothing, what masked places hold, wrong lengths and
pages, streams and graphs, and a run of attention, weights and eviction together.

Tolerance (derived before the first run). A weight exp(s - lse), from a score s that is an fp32 sum of dim exact products, is off by dim 2^-23 S
with S = scale sum |q||k| for the sum, by 2^-23 (|s| + |lse|) for the roundings of the scale, the logarithm and their difference, and 2^-21 for the exponential and
its argument, all relative; the logarithm given is taken as it is. The sum of n weights adds 2^-24 (n + 2) of itself, what was there before 2^-23."""
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


def _pool(pages, kv, dim, page, bits, seed=1):
    cache = pkg.KVCache.empty(pages, kv, dim, page_size=page, bits=bits)
    n = pages * page
    rows = [torch.randn((n, kv, dim), generator=_gen(seed + i), device=DEV).half() for i in range(2)]
    pkg.kv_append(cache, *rows, torch.arange(n, device=DEV).int())
    return cache


class Case:
    def __init__(self, lens, new, kv=2, group=4, dim=64, page=16, bits=16, window=0, seed=1, scale=None, size=1.5, max_len=None):
        self.lens, self.new, self.window, self.group = lens, new, window, group
        b = len(lens)
        self.max_len = max(1, max(lens)) if max_len is None else max_len
        cols = -(-self.max_len // page)
        self.cache = _pool(b * cols + 1, kv, dim, page, bits, seed)
        self.pages = torch.randperm(b * cols + 1, generator=_gen(seed), device=DEV)[:b * cols].int().view(b, cols)
        self.seq_lens = _i32(lens)
        self.start = _i32([sum(new[:i]) for i in range(b + 1)])
        self.max_q = max(1, max(new))
        self.q = (size * torch.randn((sum(new), kv * group, dim), generator=_gen(seed + 7), device=DEV)).half()
        self.scale = dim ** -0.5 if scale is None else scale
        self.kw = dict(q_start=self.start, max_q=self.max_q, max_len=self.max_len, window=window, scale=scale)

    def attend(self):
        return pkg.attention(self.q, self.cache, self.pages, self.seq_lens, return_lse=True, **self.kw)

    def weights(self, lse, before=None, per_head=True, **kw):
        return pkg.attention_weights(self.q, self.cache, self.pages, self.seq_lens, lse, before=before, per_head=per_head, **{**self.kw, **kw})

    def exact(self, lse, before, per_head):
        """(sums, bound of their error), fp64 [batch][heads][max_len]."""
        kv, g, dim, page = self.cache.kv_heads, self.group, self.cache.head_dim, self.cache.page_size
        sums = torch.zeros((len(self.lens), kv, self.max_len), dtype=torch.float64, device=DEV)
        off = sums.clone()
        for b, (n, m) in enumerate(zip(self.lens, self.new)):
            if not n or not m:
                continue
            j = torch.arange(n, device=DEV)
            keys = pkg.kv_read(self.cache, (self.pages[b].long()[j // page] * page + j % page).int())[0].double()
            at = int(self.start[b])
            q = self.q[at:at + m].double().view(m, kv, g, dim)
            pos = n - m + torch.arange(m, device=DEV)
            seen = (j[None] <= pos[:, None]) & ((j[None] > pos[:, None] - self.window) if self.window else True)
            for h in range(kv):
                x = q[:, h].reshape(m * g, dim) @ keys[:, h].t().contiguous() * self.scale
                big = q[:, h].reshape(m * g, dim).abs() @ keys[:, h].abs().t().contiguous() * abs(self.scale)
                ls = lse[at:at + m, h * g:h * g + g].double().reshape(m * g, 1)
                w = torch.where(seen.repeat_interleave(g, dim=0), (x - ls).exp(), 0.0)
                rel = dim * 2.0 ** -23 * big + 2.0 ** -23 * (x.abs() + torch.where(ls.isfinite(), ls, 0.0).abs()) + 2.0 ** -21
                sums[b, h, :n] = w.sum(dim=0)
                off[b, h, :n] = (w * rel).sum(dim=0) + 2.0 ** -24 * (m * g + 2) * w.sum(dim=0)
        if not per_head:
            off = off.sum(dim=1, keepdim=True) + 2.0 ** -24 * kv * sums.sum(dim=1, keepdim=True)
            sums = sums.sum(dim=1, keepdim=True)
        if before is not None:
            there = torch.arange(self.max_len, device=DEV) < self.seq_lens[:, None, None]
            add = torch.where(there, before[..., :self.max_len].double(), 0.0)
            sums, off = sums + add, off + 2.0 ** -23 * (add.abs() + sums)
        return sums, off

    def check(self, per_head=(True, False)):
        _, lse = self.attend()
        for each in per_head:
            for before in (None, torch.rand((len(self.lens), self.cache.kv_heads if each else 1, self.max_len + 3), generator=_gen(9), device=DEV)):
                want, off = self.exact(lse, before, each)
                got = self.weights(lse, before, each)
                assert got.shape == want.shape
                assert ((got.double() - want).abs() <= off).all(), float(((got.double() - want).abs() / off.clamp_min(1e-30)).max())
                assert torch.equal(got, self.weights(lse, before, each))
        return lse


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim,page,kv,group", [(64, 16, 2, 4), (96, 8, 3, 1), (128, 64, 2, 8), (192, 1, 1, 16), (256, 32, 5, 3)])
def test_single_tokens(dim, page, kv, group, bits):
    Case([1, 300, 0, 33, 64, 65, 517], [1] * 7, kv, group, dim, page, bits).check()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim,page,kv,group", [(64, 16, 2, 4), (96, 8, 3, 3), (128, 64, 2, 8), (192, 2, 1, 16), (256, 32, 5, 1)])
def test_prompts(dim, page, kv, group, bits):
    """Steps of rows that are whole, end inside a token's heads, begin inside a tile of keys."""
    Case([700, 333, 64, 1, 100], [257, 333, 64, 1, 0], kv, group, dim, page, bits).check()


@pytest.mark.parametrize("window", [1, 16, 63, 200, 1000])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [5, 3, 1, 2], [90, 200, 7, 1]])
def test_windows(new, window):
    Case([300, 257, 30, 400], new, 2, 4, 64, window=window).check()
    Case([300, 257, 30, 400], new, 1, 3, 128, bits=8, window=window).check(per_head=(True,))


@pytest.mark.parametrize("group,new", [(32, 1), (33, 1), (16, 2), (11, 3), (1, 32), (1, 33), (64, 1), (1, 64), (1, 65), (5, 13), (40, 8)])
def test_numbers_of_rows(group, new):
    """Around what a product, a step and the two kernels take."""
    Case([200, 77], [new, max(1, new // 2)], 1, group, 64).check()
    Case([200, 77], [new, max(1, new // 2)], 3, group, 96, bits=4).check()


def test_rows_split_between_workgroups():
    c = Case([500], [450], 2, 5, 128, seed=5)
    assert pkg.attention_weights_workspace_bytes(c.cache, 1, 450, 10, 2, 450, 500) == 2 * 8 * 500 * 4
    c.check()


def test_new_tokens_before_their_keys_and_empty_rows():
    """More new tokens than the sequence has: the first ones see nothing, and have a logarithm of -inf."""
    c = Case([3, 0, 40], [5, 2, 50], 2, 2, 64)
    lse = c.check()
    assert (lse[:2] == -INF).all() and (lse[5:7] == -INF).all()


@pytest.mark.parametrize("new", [[1, 1], [40, 30]])
@pytest.mark.parametrize("bits", [16, 8])
def test_what_no_row_sees_is_not_used(new, bits):
    """NaN and infinities behind the end, before the window, in other pages; table entries behind the last page are anything."""
    c = Case([90, 37], new, 2, 4, 64, bits=bits, window=50, max_len=128)
    _, lse = c.attend()
    want = c.weights(lse)
    lo = [max(0, n - m - 49) for n, m in zip(c.lens, c.new)]
    t = c.cache.k if bits == 16 else c.cache.k_par
    free = torch.ones(c.cache.n_pages, 16, dtype=torch.bool, device=DEV)
    for b, n in enumerate(c.lens):
        for j in range(lo[b], n):
            free[int(c.pages[b, j // 16]), j % 16] = False
    t.transpose(1, 2)[free] = NAN
    for b, n in enumerate(c.lens):
        c.pages[b, -(-n // 16):] = 2 ** 31 - 1
        c.pages[b, :lo[b] // 16] = -7
    assert torch.equal(c.weights(lse), want) and torch.isfinite(want).all()
    assert all((want[b, :, :lo[b]] == 0).all() and (want[b, :, n:] == 0).all() for b, n in enumerate(c.lens))


@pytest.mark.parametrize("new", [1, 60])
def test_pages_outside_the_pool_are_nan_where_seen(new):
    c = Case([100, 100], [new, new], 2, 4, 64)
    lse = torch.zeros(2 * new, 8, device=DEV)
    want = c.weights(lse)
    c.pages[0, 2] = c.cache.n_pages
    got = c.weights(lse)
    assert got[0, :, 32:48].isnan().all()
    got[0, :, 32:48] = want[0, :, 32:48]
    assert torch.equal(got, want)
    c.window, c.kw["window"] = 20, 20              # page 2 out of sight of all rows, and of some
    got = c.weights(lse)
    assert got[0, :, 32:48].isnan().any() == (new == 60) and got[1].isfinite().all()


@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("per_head", [True, False])
def test_wrong_lengths_and_counts_are_nan(new, per_head):
    c = Case([100] * 5, [new] * 5, 2, 4, 64)
    _, lse = c.attend()
    want = c.weights(lse, per_head=per_head)
    for lens in ([-1, 100, 101, 100, 2 ** 31 - 1],):
        got = c.weights(lse, per_head=per_head) if lens is None else pkg.attention_weights(
            c.q, c.cache, c.pages, _i32(lens), lse, per_head=per_head, **c.kw)
        assert got[[0, 2, 4]].isnan().all() and torch.equal(got[[1, 3]], want[[1, 3]])
    for start in ([0, -1, 2 * new, 3 * new, 4 * new, 5 * new], [0, new, 2 * new, 2 * new - 1, 4 * new, 5 * new],
                  [0, new, 2 * new, 3 * new, 4 * new, 5 * new + 1], [0, new, 2 * new, 3 * new, 4 * new, 2 ** 31 - 1]):
        got = pkg.attention_weights(c.q, c.cache, c.pages, c.seq_lens, lse, per_head=per_head, **{**c.kw, "q_start": _i32(start)})
        wrong = [a < 0 or b < a or b > 5 * new or b - a > new for a, b in zip(start, start[1:])]
        right = [not w and a == i * new and b == a + new for i, (a, b, w) in enumerate(zip(start, start[1:], wrong))]
        assert got[torch.tensor(wrong)].isnan().all() and torch.equal(got[torch.tensor(right)], want[torch.tensor(right)])


@pytest.mark.parametrize("new", [1, 50])
def test_logarithms_that_are_no_numbers(new):
    c = Case([80], [new], 2, 4, 64)
    _, lse = c.attend()
    lse[0, 0], lse[-1, 5] = NAN, INF
    got, first = c.weights(lse), 80 - new
    assert got[0, 0, :first + 1].isnan().all() and got[0, 0, first + 1:].isfinite().all() and got[0, 1].isfinite().all()


def test_strides_in_place_and_untouched_rest():
    c = Case([100, 37, 64], [1, 1, 1], 2, 4, 64)
    _, lse = c.attend()
    wide = torch.rand((2, 3, 140), generator=_gen(3), device=DEV)
    keep = wide.clone()
    view = wide[..., 10:130].transpose(0, 1)                          # heads' rows first
    want = c.weights(lse, before=view.contiguous())
    assert c.weights(lse, before=view, out=view) is view
    assert torch.equal(view[..., :100], want)
    wide[..., 10:110] = keep[..., 10:110]
    assert torch.equal(wide, keep)
    rows = torch.randn((3, 11, 64), generator=_gen(4), device=DEV).half()
    q = rows[:, 2:10]
    assert torch.equal(pkg.attention_weights(q, c.cache, c.pages, c.seq_lens, lse, max_len=100),
                       pkg.attention_weights(q.contiguous(), c.cache, c.pages, c.seq_lens, lse, max_len=100))


def test_scales():
    for scale in (0.0, -0.2, 1.0):
        Case([90, 40], [1, 1], 2, 4, 64, scale=scale).check()
        Case([90, 40], [50, 30], 2, 4, 64, scale=scale).check()


def test_nothing_to_do():
    c = Case([5], [1], 2, 4, 64)
    empty = torch.zeros((0, 8, 64), dtype=torch.float16, device=DEV)
    no = torch.zeros((0, 8), device=DEV)
    assert pkg.attention_weights(empty, c.cache, c.pages[:0], _i32([]), no).shape == (0, 2, 16)
    got = pkg.attention_weights(empty, c.cache, c.pages, _i32([5]), no, q_start=_i32([0, 0]), before=torch.ones(1, 2, 16, device=DEV))
    assert (got[..., :5] == 1).all() and (got[..., 5:] == 0).all()


def test_sums_of_all_weights_are_the_rows():
    """The weights of a row add up to 1, whatever the cache holds: each within 2^-20 and the scores' own error."""
    c = Case([1000, 300], [200, 1], 2, 4, 128, bits=8)
    _, lse = c.attend()
    got = c.weights(lse).double().sum(dim=2)
    want = torch.tensor([[200 * 4] * 2, [4] * 2], dtype=torch.float64, device=DEV)
    assert ((got - want).abs() <= 1e-4 * want).all()


def test_streams_and_graphs():
    c = Case([90, 60], [40, 30], 2, 4, 64)
    _, lse = c.attend()
    want = c.weights(lse, per_head=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.weights(lse, per_head=False, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    sums = torch.zeros(2, 1, 90, device=DEV)
    eager = sums.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.weights(lse, before=sums, per_head=False, out=sums)
    for _ in range(4):
        graph.replay()
        c.weights(lse, before=eager, per_head=False, out=eager)          # beside the replay, with a workspace of its own
        torch.cuda.synchronize()
        assert torch.equal(sums, eager)


def test_decoding_with_a_bounded_cache():
    """Steps of a decode loop: append, attend, add up the weights, and from time to time evict: the kept tokens are the ones that a plain program keeps,
    and the attention is over exactly them."""
    kv, group, dim, page, b = 2, 4, 64, 16, 3
    cache = _pool(b * 5, kv, dim, page, 8)
    pages = torch.randperm(b * 5, generator=_gen(2), device=DEV).int().view(b, 5)
    table, lens, sums = pkg.rope_table(dim, 400), _i32([40, 17, 64]), torch.zeros(b, kv, 80, device=DEV)
    held = [[list(range(n)) for _ in range(kv)] for n in (40, 17, 64)]      # which token every place holds
    rows = {}
    at = torch.arange(80, device=DEV)
    for i in range(b):
        slots = (pages[i].long()[at // page] * page + at % page).int()
        rows[i] = [list(x.unbind(0)) for x in pkg.kv_read(cache, slots)]
    count = [40, 17, 64]
    tokens = [[[rows[i][x][j] for j in range(count[i])] for x in (0, 1)] for i in range(b)]
    for step in range(40):
        x = torch.randn((b, kv * (group + 2), dim), generator=_gen(100 + step), device=DEV).half()
        q, k, v = x[:, :kv * group], x[:, kv * group:kv * group + kv], x[:, kv * group + kv:]
        idx = torch.arange(b, device=DEV)
        slots = (pages[idx, (lens // page).long()] * page + lens % page).int()
        q = pkg.kv_append(cache, k, v, slots, positions=_i32(count), table=table, q=q)
        lens += 1
        kr, vr = pkg.kv_read(cache, slots)
        for i in range(b):
            for h in range(kv):
                held[i][h].append(count[i])
            tokens[i][0].append(kr[i])
            tokens[i][1].append(vr[i])
            count[i] += 1
        o, lse = pkg.attention(q, cache, pages, lens, max_len=80, return_lse=True)
        pkg.attention_weights(q, cache, pages, lens, lse, before=sums, out=sums, max_len=80)
        for i in range(b):
            for h in range(kv):
                kk, vv = (torch.stack([tokens[i][x][j][h] for j in held[i][h]]).double() for x in (0, 1))
                p = torch.softmax(q[i, h * group:h * group + group].double() @ kk.t().contiguous() / 8.0, dim=1)
                ref = p @ vv
                # half an ulp, weights rounded to fp16, and fp32 scores (dim 2^-23 of sums of 64 products of size about 30)
                assert ((o[i, h * group:h * group + group].double() - ref).abs() <= 2.0 ** -10 * (ref.abs() + p @ vv.abs()) + 1e-5).all()
        if step % 8 == 7:
            old = sums.clone()
            _, _, kept = pkg.kv_evict(cache, pages, lens, sums, 48, recent=8, first=1, lens_out=lens, sums_out=sums)
            for i in range(b):
                for h in range(kv):
                    mine = [j for j in kept[i, h].tolist() if j >= 0]
                    n = len(held[i][h])
                    if n > 48:
                        middle = sorted(range(1, n - 8), key=lambda j: (-float(old[i, h, j]), j))[:39]
                        assert mine == sorted([0, *middle, *range(n - 8, n)])
                    held[i][h] = [held[i][h][j] for j in mine]
    assert lens.tolist() == [48, 48, 48]
