"""Attention behind shared prefixes on the GPU, what else its arguments allow: starts of prefixes that descend. Cases, results in
64 bits and bounds are test_gpu_shared's."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from test_gpu_shared import DEV, Case, _i32  # noqa: E402

INF = math.inf


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
