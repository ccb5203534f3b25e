"""Attention behind shared prefixes on the GPU, against a plain implementation in 64 bits: every head size, number of bits and page size,
one prefix and several, sequences without one, drafts and prompts behind a prefix, empty ones, what masked places hold, wrong values, streams and
graphs.

Tolerance (derived before the first run), as for the attention without prefixes: half an ulp of fp16 of the output (2^-11 |o|, 2^-25 below its
normal range); weights rounded to fp16, 2^-11 each, or 2^-25 of the largest of its part where they are below the normal range; scores from fp32 sums of dim exact
products, dim 2^-23 S with S = scale sum |q||k|, and an exponent of up to |s| with a few roundings of 2^-22 each, both of which scale a
weight, and as much again for the joins; all of it on A = sum p |v|."""
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


class Case:
    """Prefixes of `plens` tokens with `sizes` sequences each, then `loose` sequences without one; own lengths and new tokens per sequence."""

    def __init__(self, plens, sizes, lens, new=None, kv=2, group=4, dim=64, page=16, bits=16, seed=1, scale=None, before=0, size=1.5):
        self.plens, self.lens, self.new = plens, lens, [1] * len(lens) if new is None else new
        self.kv, self.group, self.dim, self.page = kv, group, dim, page
        pc, oc = (max(1, -(-max([*x, 1]) // page)) for x in (plens, lens))
        total = len(plens) * pc + len(lens) * oc + 2
        self.cache = pkg.KVCache.empty(total, kv, dim, page_size=page, bits=bits)
        rows = [torch.randn((total * page, kv, dim), generator=_gen(seed + i), device=DEV).half() for i in range(2)]
        pkg.kv_append(self.cache, *rows, torch.arange(total * page, device=DEV).int())
        order = torch.randperm(total, generator=_gen(seed + 3), device=DEV).int()
        self.ppages, self.pages = order[:len(plens) * pc].view(-1, pc), order[len(plens) * pc:len(plens) * pc + len(lens) * oc].view(-1, oc)
        at = [before + sum(sizes[:i]) for i in range(len(sizes) + 1)]
        self.of = [next((g for g in range(len(plens)) if at[g] <= b < at[g + 1]), -1) for b in range(len(lens))]
        self.first, self.start = _i32(at), _i32([sum(self.new[:i]) for i in range(len(lens) + 1)])
        self.q = (size * torch.randn((sum(self.new), kv * group, dim), generator=_gen(seed + 7), device=DEV)).half()
        self.scale = dim ** -0.5 if scale is None else scale
        self.one = len(plens) == 1 and at == [0, len(lens)]
        self.sizes, self.prefix_lens, self.seq_lens = sizes, _i32(plens), _i32(lens)

    def args(self, **kw):
        a = dict(q=self.q, cache=self.cache, prefix_pages=self.ppages, prefix_lens=self.prefix_lens, pages=self.pages, seq_lens=self.seq_lens,
                 scale=self.scale, return_lse=True, max_prefix=max([*self.plens, 1]), max_len=max([*self.lens, 1]))
        if not self.one:
            a |= dict(first=self.first, max_group=max([*self.sizes, 1]))
        if any(m != 1 for m in self.new):
            a |= dict(q_start=self.start, max_q=max(self.new))
        return {**a, **kw}

    def run(self, **kw):
        return pkg.attention_shared(**self.args(**kw))

    def tokens(self, pages, n):
        j = torch.arange(n, device=DEV)
        return [x.double() for x in pkg.kv_read(self.cache, (pages.long()[j // self.page] * self.page + j % self.page).int())]

    def exact(self):
        g, dim, kv = self.group, self.dim, self.kv
        o = torch.zeros(self.q.shape, dtype=torch.float64, device=DEV)
        lse = torch.full(self.q.shape[:2], -INF, dtype=torch.float64, device=DEV)
        ob, lb = torch.zeros_like(o) + 2.0 ** -25, torch.zeros_like(lse)
        pre = [self.tokens(self.ppages[i], n) for i, n in enumerate(self.plens)]
        t = 0
        for b, (n, m) in enumerate(zip(self.lens, self.new)):
            mine = self.tokens(self.pages[b], n)
            pn = 0
            if self.of[b] >= 0:
                pn = self.plens[self.of[b]]
                mine = [torch.cat([x, y]) for x, y in zip(pre[self.of[b]], mine)]
            j = torch.arange(pn + n, device=DEV)[None] - pn
            sees = ((j < 0) | (j <= n - m + torch.arange(m, device=DEV)[:, None])).repeat_interleave(g, dim=0)
            some = sees.any(dim=1)
            for h in range(kv):
                if not some.any():
                    continue
                k, v = (x[:, h] for x in mine)
                q = self.q[t:t + m, h * g:h * g + g].double().reshape(m * g, dim)
                x = torch.where(sees, q @ k.t().contiguous() * self.scale, -INF)
                big = (torch.where(sees, q.abs() @ k.abs().t().contiguous(), 0.0) * abs(self.scale)).amax(dim=1)
                w = torch.where(some[:, None], torch.softmax(x, dim=1), 0.0)
                r, a = w @ v, w @ v.abs()
                ls = torch.logsumexp(x, dim=1)
                ds = dim * 2.0 ** -23 * big + 2.0 ** -21 * (1 + torch.where(sees, x.abs(), 0.0).amax(dim=1))
                bound = 2.0 ** -11 * r.abs() + 2.0 ** -25 + a * (2.0 ** -11 + 4 * ds + 2.0 ** -19)[:, None] + \
                    sees.sum(dim=1)[:, None] * 2.0 ** -25 * v.abs().amax(dim=0)
                o[t:t + m, h * g:h * g + g] = r.view(m, g, dim)
                ob[t:t + m, h * g:h * g + g] = bound.view(m, g, dim)
                lse[t:t + m, h * g:h * g + g] = torch.where(some, ls, -INF).view(m, g)
                lb[t:t + m, h * g:h * g + g] = (2 * ds + 2.0 ** -19 * (1 + ls.abs())).view(m, g)
            t += m
        return o, lse, ob, lb

    def check(self, **kw):
        o, lse = self.run(**kw)
        ro, rl, ob, lb = self.exact()
        assert torch.isfinite(o).all()
        assert ((o.double() - ro).abs() <= ob).all(), float(((o.double() - ro).abs() / ob).max())
        seen = torch.isfinite(rl)
        assert torch.equal(lse == -INF, ~seen) and ((lse.double() - rl).abs()[seen] <= lb[seen]).all() and not o[~seen].any()
        again = self.run(**kw)
        assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
        return o, lse


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("page", [1, 8, 16, 64])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_single_tokens_behind_one_prefix(dim, page, bits):
    """Few rows behind the prefix, then many."""
    Case([333], [3], [1, 40, 0], dim=dim, page=page, bits=bits).check()
    Case([515], [40], [1 + 7 * i for i in range(40)], dim=dim, page=page, bits=bits).check()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("new", [[5, 1, 3], [60, 2, 33]])
def test_several_new_tokens(new, dim, bits):
    """Drafts, and prompts whose own rows go the way of many."""
    Case([257], [3], [64, 1, 50], new, dim=dim, bits=bits).check()


@pytest.mark.parametrize("group", [1, 3, 8, 16, 17, 40])
@pytest.mark.parametrize("size", [1, 2, 9])
def test_groups_of_heads_and_sequences(group, size):
    """Rows of a prefix around what one and two blocks of 16 and a workgroup of 128 take."""
    Case([150, 40], [size, max(1, size - 1)], [33] * (2 * size - (size > 1)), group=group, kv=1, dim=64).check()
    Case([150, 40], [size, max(1, size - 1)], [33] * (2 * size - (size > 1)), group=group, kv=3, dim=128, bits=8).check()


@pytest.mark.parametrize("bits", [16, 4])
def test_several_prefixes_and_none(bits):
    """Prefixes of no, one and many tokens and sequences, and sequences before and behind them without one."""
    lens = [20, 1, 0, 64, 65, 3, 100, 17, 5, 9, 33]
    for before in (0, 2):
        Case([70, 0, 1, 300, 64], [3, 1, 0, 4, 1], lens, before=before, bits=bits).check()
        Case([70, 0, 1, 300, 64], [3, 1, 0, 4, 1], lens, [1, 3, 2, 7, 1, 3, 50, 1, 5, 9, 2], before=before, bits=bits, dim=128).check()


@pytest.mark.parametrize("n", [63, 64, 65, 200, 513])
def test_many_prefixes(n):
    """Around what a wave looks up at once, and more than are shared out by their lengths."""
    plens = [(37 * i) % 90 for i in range(n)]
    sizes = [(i % 3) for i in range(n)]
    c = Case(plens, sizes, [(11 * i) % 40 for i in range(sum(sizes) + 2)], dim=64, kv=1, before=1)
    c.check()


@pytest.mark.parametrize("plen,lens,new", [(5000, [700, 2000, 3], None), (20000, [3000, 1], None), (4000, [900] * 20, None), (300, [6000, 5000], None),
                                           (7000, [600, 500], [200, 100]), (6000, [3000, 2500, 40], [5, 6, 2])])
def test_long_ones_are_shared_out(plen, lens, new):
    Case([plen], [len(lens)], lens, new, dim=128, kv=2, bits=8).check()


def test_empty_prefix_and_empty_own_tokens():
    Case([0], [3], [0, 5, 0]).check()
    o, lse = Case([0], [40], [0] * 40).check()
    assert not o.any() and (lse == -INF).all()
    Case([90], [3], [0, 0, 0]).check()
    Case([90], [40], [0] * 40, dim=128).check()


def test_agrees_with_attention_over_whole_sequences():
    """A page in the tables of all sequences: the same keys, so the same result within both bounds."""
    c = Case([128], [20], [1 + 3 * i for i in range(20)], dim=128, bits=8)
    o, lse = c.run()
    whole = torch.cat([c.ppages.expand(20, -1), c.pages], dim=1).contiguous()
    o2, lse2 = pkg.attention(c.q, c.cache, whole, _i32([128 + n for n in c.lens]), scale=c.scale, return_lse=True)
    _, _, ob, lb = c.exact()
    assert ((o.double() - o2.double()).abs() <= 2 * ob).all() and ((lse.double() - lse2.double()).abs() <= 2 * lb).all()


@pytest.mark.parametrize("size", [2, 40])
@pytest.mark.parametrize("bits", [16, 8])
def test_what_no_row_sees_is_not_used(size, bits):
    c = Case([70, 33], [size, size], [20] * (2 * size), bits=bits)
    want = c.run(max_prefix=80, max_len=32)
    free = torch.ones(c.cache.n_pages, 16, dtype=torch.bool, device=DEV)
    for pages, lens in ((c.ppages, c.plens), (c.pages, c.lens)):
        for b, n in enumerate(lens):
            for j in range(n):
                free[int(pages[b, j // 16]), j % 16] = False
    for t in (c.cache.k, c.cache.v) if bits == 16 else (c.cache.k_par, c.cache.v_par):
        t.transpose(1, 2)[free] = NAN
    c.ppages[1, 3:] = 2 ** 31 - 1
    got = c.run(max_prefix=80, max_len=32)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.isfinite(want[0]).all()


@pytest.mark.parametrize("size", [2, 40])
def test_infinite_and_nan_values_reach_the_rows_that_see_them(size):
    c = Case([70, 64], [size, size], [20] * (2 * size))
    c.cache.v[int(c.ppages[0, 4]), 0, 2, 5] = INF
    c.cache.v[int(c.pages[size, 0]), 1, 3, 9] = NAN
    o, lse = c.run()
    assert torch.isfinite(lse).all()
    bad = torch.zeros_like(o, dtype=torch.bool)
    bad[:size, :4, 5] = True
    assert (o[:size, :4, 5] == INF).all()
    bad[size, 4:, 9] = True
    assert o[size, 4:, 9].isnan().all() and torch.isfinite(o[~bad]).all()


@pytest.mark.parametrize("size", [2, 40])
@pytest.mark.parametrize("new", [1, 40])
def test_wrong_values_are_nan(size, new):
    n = 3 * size
    c = Case([70, 33, 50], [size] * 3, [60] * n, [new] * n)
    want = c.run()
    seqs = torch.arange(n, device=DEV).repeat_interleave(new)

    def check(bad, **kw):
        o, lse = c.run(**kw)
        bad = torch.tensor(bad, device=DEV)[seqs]
        assert o[bad].isnan().all() and lse[bad].isnan().all()
        assert torch.equal(o[~bad], want[0][~bad]) and torch.equal(lse[~bad], want[1][~bad])

    group = [b // size for b in range(n)]
    check([g == 1 for g in group], prefix_lens=_i32([70, -1, 50]))
    check([g == 2 for g in group], prefix_lens=_i32([70, 33, 71]))
    check([b == 1 for b in range(n)], seq_lens=_i32([61 if b == 1 else 60 for b in range(n)]))
    pages = c.ppages.clone()
    pages[0, 1] = -1
    check([g == 0 for g in group], prefix_pages=pages)
    own = c.pages.clone()
    own[size, 0] = 10 ** 9
    check([b == size for b in range(n)], pages=own)
    # more sequences behind a prefix than was said: the two that have them
    if size == 40:
        o, _ = c.run(first=_i32([0, size - 1, 3 * size - 1, 3 * size]), max_group=size)
        assert o[(size - 1) * new:(3 * size - 1) * new].isnan().all() and torch.isfinite(o[:(size - 1) * new]).all()
    # starts of prefixes that are anything: nothing outside the arrays is read, and whoever has no prefix by them has none
    for first in ([5, 3, 1, 0], [-1, size, 2 * size, n], [0, size, 2 * size, n + 1], [2 ** 31 - 1, -2 ** 31, 7, n], [n, n, n, n]):
        c.run(first=_i32(first))
    torch.cuda.synchronize()


def _many_short(dim=64, page=16, bits=16, new=1, kv=4, several=False):
    """More sequences than there are workgroups' places: each by a wave, of no token to eight steps of them."""
    n = 131
    lens = [(37 * b) % 231 for b in range(n)]
    lens[5], lens[6], lens[7], lens[n - 1] = 0, 32, 33, 1
    rows = [1 + b % new for b in range(n)]
    if several:
        return Case([(13 * g) % 90 for g in range(65)], [2] * 65, lens, rows, kv=kv, dim=dim, page=page, bits=bits)
    return Case([150], [n], lens, rows, kv=kv, dim=dim, page=page, bits=bits)


@pytest.mark.parametrize("several", [False, True])
@pytest.mark.parametrize("new", [1, 3, 8])
@pytest.mark.parametrize("dim,page,bits", [(64, 16, 16), (64, 4, 8), (96, 8, 16), (96, 32, 4), (128, 16, 16), (128, 64, 8), (128, 8, 4), (192, 32, 8),
                                           (256, 16, 16), (256, 8, 4)])
def test_many_short_sequences(dim, page, bits, new, several):
    _many_short(dim, page, bits, new, several=several).check()


@pytest.mark.parametrize("several", [False, True])
def test_many_short_sequences_with_wrong_and_odd_values(several):
    c = _many_short(several=several)
    want = c.run()
    lens, pages = c.seq_lens.clone(), c.pages.clone()
    lens[3], lens[40], pages[17, 1] = -1, 10 ** 9, 10 ** 9
    c.cache.v[int(c.pages[70, 2]), 1, 3, 9] = NAN
    c.cache.v[int(c.pages[71, 0]), 2, 3, 5] = -INF
    # behind a length, and in pages that nobody's length reaches: anything
    for b in (7, 12, 50):
        n = c.lens[b]
        c.cache.v[int(c.pages[b, n // 16]), :, n % 16] = NAN
        c.cache.k[int(c.pages[b, n // 16]), :, n % 16] = NAN
    pages[130, 1:] = -7
    o, lse = c.run(seq_lens=lens, pages=pages)
    bad = torch.zeros(131, dtype=torch.bool, device=DEV)
    bad[[3, 40, 17]] = True
    assert o[bad].isnan().all() and lse[bad].isnan().all()
    odd = torch.zeros_like(o, dtype=torch.bool)
    odd[70, 4:8, 9] = odd[71, 8:12, 5] = True
    assert o[70, 4:8, 9].isnan().all() and (o[71, 8:12, 5] == -INF).all()
    same = ~odd & ~bad[:, None, None]
    assert torch.equal(o[same], want[0][same]) and torch.equal(lse[~bad], want[1][~bad])
    again = c.run(seq_lens=lens, pages=pages)
    assert torch.equal(o[same], again[0][same])


def test_wrong_starts_of_tokens():
    c = Case([70], [4], [60] * 4, [40] * 4)
    for start in ([0, -1, 80, 120, 160], [0, 40, 39, 120, 160], [0, 40, 80, 120, 161], [0, 40, 80, 2 ** 31 - 1, -2 ** 31], [7, 7, 7, 7, 7],
                  [-2 ** 31, 40, 80, 120, 160], [-2 ** 31, 2 ** 31 - 1, -5, 2 ** 31 - 1, 160]):
        c.run(q_start=_i32(start))
    torch.cuda.synchronize()
    # one sequence claims more than max_q: all its tokens are NaN, and the others' prefix holds no more than it may
    o, lse = c.run(q_start=_i32([0, 30, 60, 110, 140]))
    assert o[60:110].isnan().all() and lse[60:110].isnan().all() and torch.isfinite(o[:60]).all() and torch.isfinite(o[110:140]).all()


def test_strides_and_scales():
    c = Case([90], [5], [20] * 5, dim=64)
    want = c.run()
    rows = torch.zeros((5, 13, 64), dtype=torch.float16, device=DEV)
    rows[:, 3:11] = c.q
    out = torch.full((5, 20, 64), 7.0, dtype=torch.float16, device=DEV)
    o, _ = c.run(q=rows[:, 3:11], out=out[:, 6:14])
    assert o.data_ptr() == out[:, 6:14].data_ptr() and torch.equal(o, want[0]) and (out[:, :6] == 7).all() and (out[:, 14:] == 7).all()
    same = rows[:, 3:11].clone()
    assert torch.equal(c.run(q=same, out=same)[0], want[0])           # in place
    wide = torch.full((1, 30), 10 ** 9, dtype=torch.int32, device=DEV)
    wide[:, 4:4 + c.ppages.shape[1]] = c.ppages
    assert torch.equal(c.run(prefix_pages=wide[:, 4:], max_prefix=90)[0], want[0])
    for scale in (0.0, -0.3, 1.0):
        Case([90], [5], [20] * 5, dim=64, scale=scale).check()
        Case([90], [50], [20] * 50, dim=128, scale=scale).check()


def test_nothing_to_do():
    c = Case([90], [3], [5] * 3)
    o, lse = pkg.attention_shared(c.q[:0], c.cache, c.ppages, _i32([90]), c.pages[:0], _i32([]), return_lse=True)
    assert o.shape == (0, 8, 64) and lse.shape == (0, 8)


@pytest.mark.parametrize("size", [3, 40])
def test_streams_and_graphs(size):
    """Captured once, replayed beside eager calls while lengths move on in place."""
    c = Case([600], [size], [40] * size, bits=8, dim=128)
    plens, lens = _i32([600]), _i32([10] * size)
    want = c.run(prefix_lens=plens, seq_lens=lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.run(prefix_lens=plens, seq_lens=lens, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        o, lse = c.run(prefix_lens=plens, seq_lens=lens)
    for _ in range(4):
        graph.replay()
        eager = c.run(prefix_lens=plens, seq_lens=lens)
        torch.cuda.synchronize()
        assert torch.equal(o, eager[0]) and torch.equal(lse, eager[1])
        lens += 9
        plens -= 100
        torch.cuda.synchronize()


def test_weights_and_eviction_beside_a_prefix():
    """The logarithms that come with shared prefixes give the own tokens' weights: with those of the prefix they add up to one."""
    c = Case([100], [6], [40] * 6, dim=64)
    _, lse = c.run()
    own = pkg.attention_weights(c.q, c.cache, c.pages, _i32([40] * 6), lse, max_len=40, scale=c.scale)
    start = _i32([0, 6])
    pre = pkg.attention_weights(c.q, c.cache, c.ppages, _i32([106]), lse, q_start=start, max_q=6, max_len=106, scale=c.scale) \
        if c.ppages.shape[1] * 16 >= 106 else None
    total = own.double().sum(dim=(0, 2))
    if pre is not None:                           # (a prefix of 100 tokens, of which the queries, put behind it, see 100 to 106)
        total = total + pre[0, :, :100].double().sum(dim=1)
        assert ((total - 24.0).abs() <= 1e-4 * 24).all()
    lens, sums, kept = pkg.kv_evict(c.cache, c.pages, _i32([40] * 6), own, 24, recent=8)
    assert lens.tolist() == [24] * 6 and (sums[..., 24:] == 0).all()
    o, lse2 = c.run(seq_lens=lens)
    assert torch.isfinite(o).all() and (lse2 <= lse + 1e-3).all()
