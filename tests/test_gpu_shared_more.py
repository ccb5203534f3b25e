"""Attention behind shared prefixes on the GPU, what else its arguments allow: starts of prefixes that descend, long prefixes with few rows each, whose tiles are
counted and shared out by their lengths, prompts beside single tokens. Cases, results in
64 bits and bounds are test_gpu_shared's."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_shared import DEV, Case, _i32  # noqa: E402


def _all_nan(c, first, **kw):
    for _ in range(2):
        o, lse = c.run(first=_i32(first), **kw)
        assert o.isnan().all() and lse.isnan().all(), first


@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("size", [2, 40])
def test_starts_of_prefixes_that_descend(size, new):
    """Two prefixes that claim the same sequences, prefixes that nobody finds, descents beside sequences of no prefix: every sequence is NaN, again and
    again, with few rows behind a prefix and many."""
    n = 3 * size
    c = Case([70, 33, 50], [size] * 3, [60] * n, [new] * n, dim=128, bits=8)
    want = c.run(max_group=n)
    for first in ([0, size + 1, 1, n], [n - 1, size, 1, 0], [0, n, 0, n], [0, 0, n, n - 1], [1, 0, 0, 0], [size, size, size, size - 1], [-1, -2, 0, n],
                  [2 ** 31 - 1, -2 ** 31, 7, n], [0, size, 2 * size, -1], [n, n, n, n - 1]):
        _all_nan(c, first, max_group=n)
    # (and the same call with starts that ascend is as before, those of no prefix among them)
    got = c.run(max_group=n)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for first in ([0, 0, 0, 0], [n, n, n, n], [1, 1, 2, 2], [0, n, n, n]):
        o, lse = c.run(first=_i32(first), max_group=n)
        assert torch.isfinite(o).all() and torch.isfinite(lse).all()


def test_one_prefix_whose_starts_descend():
    c = Case([70], [2], [20] * 4, before=1)
    c.check()
    _all_nan(c, [3, 1], max_group=4)
    _all_nan(c, [0, -1], max_group=4)


@pytest.mark.parametrize("kv,group", [(1, 4), (2, 20)])
@pytest.mark.parametrize("n", [62, 63, 64, 65, 255, 256, 257, 700])
def test_many_prefixes_whose_starts_descend(n, kv, group):
    """Around what a wave looks at at once and what a workgroup does, the descent at any place."""
    c = Case([(37 * i) % 90 for i in range(n)], [2] * n, [(11 * i) % 40 for i in range(2 * n)], kv=kv, group=group)
    want = c.run()
    right = c.first.tolist()
    for at in {0, 1, n // 2, n - 2, n - 1, min(n - 1, 63), min(n - 1, 64), min(n - 1, 255), min(n - 1, 256)}:
        _all_nan(c, right[:at] + [right[at + 1] + 1] + right[at + 1:])
    got = c.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.isfinite(want[0]).all()


@pytest.mark.parametrize("n", [3, 80])
def test_starts_that_change_under_a_graph(n):
    """Starts are read by the device: a replay after they were put right gives what a call does."""
    c = Case([50] * n, [2] * n, [20] * (2 * n))
    first, side = c.first.clone(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(first=first, stream=side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        o, lse = c.run(first=first)
    for wrong in (False, True, True, False, True, False):
        first.copy_(c.first)
        if wrong:
            first[n // 2] = 2 * n
        torch.cuda.synchronize()
        graph.replay()
        want = c.run()
        torch.cuda.synchronize()
        assert (o.isnan().all() and lse.isnan().all()) if wrong else (torch.equal(o, want[0]) and torch.equal(lse, want[1]))


def _check_but(c, bad, **kw):
    """As Case.check, but for sequences `bad`, which are NaN."""
    o, lse = c.run(**kw)
    ro, rl, ob, lb = c.exact()
    wrong = torch.tensor([b in bad for b in range(len(c.lens))], device=DEV).repeat_interleave(_i32(c.new))
    assert o[wrong].isnan().all() and lse[wrong].isnan().all()
    # (rows that see nothing have a logarithm of -inf on both sides)
    assert ((o.double() - ro).abs() <= ob)[~wrong].all() and (((lse.double() - rl).abs() <= lb) | (lse.double() == rl))[~wrong].all()
    again = c.run(**kw)
    assert torch.equal(o[~wrong], again[0][~wrong]) and torch.equal(lse[~wrong], again[1][~wrong])


def _ragged(n, kv, new=None, **kw):
    """Prefixes of 1000 to 5999 tokens, an empty one and one of one token among them, with two, one or no sequences each, and a sequence before and
    behind them without one."""
    plens = [1000 + 1237 * i % 5000 for i in range(n)]
    plens[n // 2], plens[-1] = 0, 1
    sizes = [(2, 1, 0, 2)[i % 4] for i in range(n)]
    lens = [(53 * b) % 200 for b in range(sum(sizes) + 2)]
    if new:
        lens, new = [n + 3 for n in lens], [new[b % len(new)] for b in range(len(lens))]
    return Case(plens, sizes, lens, new, kv=kv, before=1, **kw)


# Several prefixes of at most 32 rows (16 above 128 channels), bounds above 1536 tokens of 64 channels, 768 of 128, 384 of 256: counted shares. With
# five prefixes the shares are many, a stretch of one prefix each; 24 prefixes of eight heads (at 16 bits from 96 channels on, at 8 from 192 on), 40 of them at 8 bits and 300 of
# one leave fewer than two a prefix, which hold the end of one prefix and the start of the next.
@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_long_prefixes_are_shared_out(dim, bits, page):
    _ragged(5, 2, dim=dim, bits=bits, page=page).check()
    _ragged(24, 8, dim=dim, bits=bits, page=page).check()


@pytest.mark.parametrize("n", [2, 3, 40, 300])
@pytest.mark.parametrize("dim,bits", [(64, 16), (128, 8)])
def test_any_number_of_long_prefixes(n, dim, bits):
    _ragged(n, 1, dim=dim, bits=bits).check()


@pytest.mark.parametrize("n,kv", [(5, 2), (40, 8)])
def test_drafts_behind_long_prefixes(n, kv):
    """Up to 24 rows behind a prefix, in two blocks, beside own tokens of one and of two."""
    _ragged(n, kv, (3, 1, 2, 3), dim=128, bits=8).check()
    _ragged(n, kv, (3, 1, 0, 2), dim=64, page=1).check()


@pytest.mark.parametrize("n,kv,dim", [(5, 2, 128), (24, 8, 128), (24, 8, 256)])
def test_long_prefixes_with_wrong_values(n, kv, dim):
    """Wrong lengths and pages: the sequences behind them are NaN, the others right however the shares fall."""
    c = _ragged(n, kv, dim=dim)
    behind = [{b for b, g in enumerate(c.of) if g == i} for i in range(n)]
    for at, wrong in ((0, -1), (3, 6000), (1, 2 ** 31 - 1)):
        lens = c.prefix_lens.clone()
        lens[at] = wrong
        _check_but(c, behind[at], prefix_lens=lens)
    for column in (0, -1):
        pages = c.ppages.clone()
        at = max(range(n), key=lambda g: c.plens[g] if behind[g] else -1)
        pages[at, (c.plens[at] - 1) // c.page if column else 0] = 10 ** 9
        _check_but(c, behind[at], prefix_pages=pages)
    lens = c.seq_lens.clone()
    lens[2] = -5
    _check_but(c, {2}, seq_lens=lens)


@pytest.mark.parametrize("n", [512, 513])
def test_prefixes_up_to_what_is_shared_out_by_lengths(n):
    """One long prefix among short ones, with a bound that has 512 of them counted and 513 not."""
    plens = [(37 * i) % 90 for i in range(n)]
    plens[7] = 4500
    sizes = [i % 3 for i in range(n)]
    sizes[7] = 2
    Case(plens, sizes, [(11 * i) % 40 for i in range(sum(sizes) + 2)], dim=64, kv=1, before=1).check()


def test_long_prefixes_under_a_graph():
    """Captured once, replayed while the prefixes' lengths change: the shares are counted anew each time."""
    c = _ragged(5, 2, dim=128, bits=8)
    plens, side = c.prefix_lens.clone(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(prefix_lens=plens, stream=side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        o, lse = c.run(prefix_lens=plens)
    for cut in (0, 700, 5999, 1, 3000):
        plens.copy_((c.prefix_lens - cut).clamp_min(0))
        torch.cuda.synchronize()
        graph.replay()
        want = c.run(prefix_lens=plens)
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_prompts_beside_single_tokens(dim, bits):
    """Parts are in the order of the tokens: prompts, tokens and sequences without new ones in any order, of one split and of several."""
    new = [1, 300, 0, 1, 77, 1, 1, 0]
    Case([257], [8], [n + 40 * (b % 3) for b, n in enumerate(new)], new, dim=dim, bits=bits).check()
    Case([90, 0, 700], [3, 1, 2], [n + 900 * (b % 2) for b, n in enumerate(new)], new, dim=dim, bits=bits, before=1).check()


@pytest.mark.parametrize("group", [1, 3, 40])
def test_groups_of_heads_of_prompts(group):
    new = [200, 1, 3, 0, 60]
    Case([400], [5], [2000 if n == 200 else n + 5 for n in new], new, kv=2, group=group, dim=128, bits=8).check()


@pytest.mark.parametrize("new", [[1] * 6, [3, 1, 5, 0, 2, 1], [60, 1, 40, 0, 7, 1]])
def test_tokens_behind_the_last_sequence(new):
    """A padded batch, as graphs of a fixed size have: rows of no sequence stay as they are, whatever the padding holds, and the others' are the same."""
    c = Case([90, 300], [4, 1], [n + 20 for n in new], new, dim=128, bits=8)
    start = dict(q_start=c.start, max_q=max(new))
    want = c.run(**start)
    n = c.q.shape[0]
    q = torch.full((n + 9, *c.q.shape[1:]), float("nan"), dtype=torch.float16, device=DEV)
    q[:n] = c.q
    out = torch.full_like(q, 7.0)
    o, lse = c.run(q=q, out=out, **start)
    assert o is out and torch.equal(o[:n], want[0]) and torch.equal(lse[:n], want[1]) and (o[n:] == 7).all()
