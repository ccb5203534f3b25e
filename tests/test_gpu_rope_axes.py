"""Rotary positions with several axes on the GPU, against a plain implementation in 64 bits: axes' shares in blocks and in turn,
odd shares, both ways of pairing and types, gradients, the cache written on the way, wrong positions and axes.

Tolerance, as for one axis: three fp32 roundings of terms of at most |x_a| + |x_b| and the table's own 2^-24, then the output type's
rounding: 2^-22 (|x_a| + |x_b|) + half an ulp of the output."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_24875_amd as pkg  # noqa: E402
from paper_2609_24875_amd import train  # noqa: E402

DEV = torch.device("cuda:0")


def _gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def _randn(*shape, seed=0, dtype=torch.float16):
    return torch.randn(shape, generator=_gen(seed), device=DEV).to(dtype)


def _positions(axes, tokens, most=4096, seed=1):
    return torch.randint(0, most, (axes, tokens), generator=_gen(seed), device=DEV).int()


def _turn64(x, pos, axes, f, inter, inverse=False):
    r = 2 * len(f)
    a = (pos[axes.long()].t().double() * torch.tensor(f, dtype=torch.float64, device=DEV))[:, None]
    c, s = a.cos(), a.sin() * (-1.0 if inverse else 1.0)
    y, size = x.double().clone(), x.double().abs()
    i, j = (slice(0, r, 2), slice(1, r, 2)) if inter else (slice(0, r // 2), slice(r // 2, r))
    p, q = x[..., i].double(), x[..., j].double()
    y[..., i], y[..., j] = p * c - q * s, p * s + q * c
    size[..., i] = size[..., j] = p.abs() + q.abs()
    return y, size


def _bound(y, size, dtype):
    return 2.0 ** -22 * size + (2.0 ** -11 * y.abs() + 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -24 * y.abs())


SHAPES = [(1, 1, 16, (3, 5), False), (3, 5, 64, (8, 12, 12), False), (7, 40, 128, (16, 24, 24), False), (129, 3, 96, (7, 9, 8), False),
          (33, 8, 192, (1, 2, 13), True), (5, 2, 512, (64, 128, 32, 32), True), (65, 7, 80, (8,), False), (700, 48, 128, (24, 20, 20), True),
          (2, 3, 256, (8,) * 16, False)]


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("tokens,heads,dim,sections,cycled", SHAPES)
def test_rope(tokens, heads, dim, sections, cycled, dtype, inter, inverse):
    rot = 2 * sum(sections)
    f, _ = pkg.rope_frequencies(rot, base=500000.0)
    table = pkg.rope_table(rot, 4096, base=500000.0)
    axes = pkg.rope_axes(sections, cycled=cycled)
    pos = _positions(len(sections), tokens)
    x = _randn(tokens, heads, dim, seed=2, dtype=dtype)
    y = pkg.rope(x, pos, table, interleaved=inter, inverse=inverse, axes=axes)
    ref, size = _turn64(x, pos, axes, f, inter, inverse)
    assert ((y.double() - ref).abs() <= _bound(ref, size, dtype)).all()
    assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("inter", [False, True])
def test_axes_with_a_spectrum_each(inter):
    f = [100.0 ** (-i / n) for n in (12, 20) for i in range(n)]
    table = pkg.rope_table(64, 50, frequencies=f)
    pos = _positions(2, 9, 50)
    axes = pkg.rope_axes([12, 20])
    x = _randn(9, 4, 64, seed=3, dtype=torch.float32)
    ref, size = _turn64(x, pos, axes, f, inter)
    assert ((pkg.rope(x, pos, table, interleaved=inter, axes=axes).double() - ref).abs() <= _bound(ref, size, x.dtype)).all()


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_positions_that_agree_give_the_bits_of_one_axis(dtype, inter):
    table = pkg.rope_table(96, 4096)
    pos = _positions(1, 77)
    x = _randn(77, 9, 128, seed=4, dtype=dtype)
    want = pkg.rope(x, pos[0], table, interleaved=inter)
    for sections, cycled in (((48,), False), ((5, 20, 23), False), ((16, 16, 16), True)):
        same = pos.expand(len(sections), 77)
        axes = pkg.rope_axes(sections, cycled=cycled)
        assert torch.equal(pkg.rope(x, same.contiguous(), table, interleaved=inter, axes=axes), want)
        assert torch.equal(pkg.rope(x, same, table, interleaved=inter, axes=axes), want)      # one row read for all axes


def test_rows_of_wider_buffers_strided_positions_and_in_place():
    table, axes = pkg.rope_table(64, 100), pkg.rope_axes([8, 12, 12])
    pos = torch.full((3, 70), 10 ** 6, dtype=torch.int32, device=DEV)
    pos[:, 5:55] = _positions(3, 50, 100)
    buf = _randn(50, 9 * 64 + 32, seed=3)
    x = buf[:, 32:].unflatten(1, (9, 64))[:, 2:7]
    want = pkg.rope(x.contiguous(), pos[:, 5:55].contiguous(), table, axes=axes)
    before = buf.clone()
    out = pkg.rope(x, pos[:, 5:55], table, out=x, axes=axes)
    assert out is x and torch.equal(x, want) and torch.isfinite(want).all()
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep[:, 32:].unflatten(1, (9, 64))[:, 2:7] = False
    assert torch.equal(buf[keep], before[keep])


@pytest.mark.parametrize("inter", [False, True])
def test_wrong_positions_and_axes_give_nan_in_their_pairs(inter):
    table = pkg.rope_table(32, 10)
    axes = torch.tensor([0] * 6 + [1] * 5 + [2] * 4 + [200], dtype=torch.uint8, device=DEV)
    pos = torch.tensor([[0, 9, -1, 3], [5, 10, 2, 4], [2 ** 31 - 1, 0, 1, 9]], dtype=torch.int32, device=DEV)
    x = _randn(4, 2, 64, seed=5)
    y = pkg.rope(x, pos, table, interleaved=inter, axes=axes)
    bad = (pos < 0) | (pos >= 10)
    pair = torch.cat([bad, torch.ones(198, 4, dtype=torch.bool, device=DEV)])[axes.long()].t()
    want = torch.zeros(4, 64, dtype=torch.bool, device=DEV)
    want[:, :32] = pair.repeat_interleave(2, dim=1) if inter else pair.repeat(1, 2)
    assert torch.equal(torch.isnan(y), want[:, None].expand(4, 2, 64)) and torch.equal(y[..., 32:], x[..., 32:])
    assert pkg.rope(x[:0], pos[:, :0], table, axes=axes).shape == (0, 2, 64)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_gradient_is_the_formulas(dtype, inter):
    f, _ = pkg.rope_frequencies(48)
    table, axes = pkg.rope_table(48, 512), pkg.rope_axes([7, 9, 8], cycled=True)
    pos = _positions(3, 37, 512, seed=6)
    x = _randn(37, 6, 80, seed=7, dtype=dtype).requires_grad_(True)
    g = _randn(37, 6, 80, seed=8, dtype=dtype)
    y = train.rope(x, pos, table, interleaved=inter, axes=axes)
    assert torch.equal(y, pkg.rope(x.detach(), pos, table, interleaved=inter, axes=axes))
    (dx,) = torch.autograd.grad(y, x, g)
    ref, size = _turn64(g, pos, axes, f, inter, inverse=True)
    assert ((dx.double() - ref).abs() <= _bound(ref, size, dtype)).all()


def test_gradient_against_differences_and_of_the_gradient():
    """A rotation is linear, so central differences of <g, rope(x)> have no truncation error; what is left are fp32
    roundings of sums of 2 x 64 terms, far below 1e-4 for a step of 1."""
    table, axes = pkg.rope_table(32, 64), pkg.rope_axes([6, 10])
    pos = torch.tensor([[5, 63], [0, 17]], dtype=torch.int32, device=DEV)
    x, g = (_randn(2, 1, 64, seed=s, dtype=torch.float32) for s in (9, 10))
    xr, gr = x.clone().requires_grad_(True), g.clone().requires_grad_(True)
    (dx,) = torch.autograd.grad(train.rope(xr, pos, table, axes=axes), xr, gr, create_graph=True)
    for i in (0, 3, 17, 31, 40, 64, 90, 127):
        e = torch.zeros_like(x).view(-1)
        e[i] = 1.0
        e = e.view_as(x)
        up, down = ((g.double() * pkg.rope(x + s * e, pos, table, axes=axes).double()).sum() for s in (1.0, -1.0))
        assert abs(float((up - down) / 2 - dx.detach().view(-1)[i])) <= 1e-4
    h = _randn(2, 1, 64, seed=11, dtype=torch.float32)
    (dg,) = torch.autograd.grad(dx, gr, h)
    assert torch.equal(dg, pkg.rope(h, pos, table, axes=axes))


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim,sections,cycled", [(64, (8, 12, 12), False), (96, (5, 9, 10), True), (128, (16, 24, 24), False), (256, (64, 64), False)])
def test_cache_written_with_axes_holds_the_rotated_rows(dim, sections, cycled, bits, dtype, inter):
    """Keys and queries that kv_append rotates are the bits of rope's, in fp32 before they are rounded or quantised."""
    table, axes = pkg.rope_table(2 * sum(sections), 300), pkg.rope_axes(sections, cycled=cycled)
    n = 37
    pos = _positions(len(sections), n, 300)
    rows = _randn(n, 9, dim, seed=12, dtype=dtype)
    q, k, v = rows[:, :5], rows[:, 5:7], rows[:, 7:]
    slots = torch.randperm(64, generator=_gen(13), device=DEV)[:n].int()
    slots[3] = -1
    a, b = (pkg.KVCache.empty(4, 2, dim, page_size=16, bits=bits) for _ in range(2))
    for c in (a, b):
        for t in (c.k, c.v, c.k_par, c.v_par):
            if t is not None:
                t.zero_()
    qo = pkg.kv_append(a, k, v, slots, positions=pos, table=table, interleaved=inter, q=q, axes=axes)
    turned = pkg.rope(rows.float(), pos, table, interleaved=inter, axes=axes)
    assert torch.equal(qo, turned[:, :5].half())
    pkg.kv_append(b, turned[:, 5:7], v.float(), slots)
    assert torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
    if bits < 16:
        assert torch.equal(a.k_par, b.k_par) and torch.equal(a.v_par, b.v_par)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("tokens", [1, 2, 6, 21, 131])
@pytest.mark.parametrize("kv,dim,rot", [(1, 64, 64), (1, 96, 96), (1, 192, 192), (3, 64, 48), (5, 96, 96), (2, 192, 176), (1, 256, 256), (16, 256, 64)])
def test_cache_tokens_that_begin_anywhere_in_a_workgroup(kv, dim, rot, tokens, inter):
    """Tokens of few and many heads, also such that a workgroup ends inside one: keys as rope turns them, with wrong positions and axes and
    padding tokens among them."""
    n_axes = 3
    table = pkg.rope_table(rot, 50)
    axes = torch.randint(0, n_axes, (rot // 2,), generator=_gen(31), device=DEV).to(torch.uint8)
    axes[5] = 77
    pos = _positions(n_axes, tokens, 50, seed=32)
    pos[1, tokens // 2] = 50
    rows = _randn(tokens, 2 * kv, dim, seed=33)
    slots = torch.randperm(2 * tokens + 16, generator=_gen(34), device=DEV)[:tokens].int()
    if tokens > 5:
        slots[tokens - 2] = -1
    cache = pkg.KVCache.empty((2 * tokens + 16 + 7) // 8, kv, dim, page_size=8)
    cache.k.zero_(), cache.v.zero_()
    want_k, want_v = torch.zeros_like(cache.k), torch.zeros_like(cache.v)
    pkg.kv_append(cache, rows[:, :kv], rows[:, kv:], slots, positions=pos, table=table, interleaved=inter, axes=axes)
    turned = pkg.rope(rows[:, :kv].contiguous(), pos, table, interleaved=inter, axes=axes)
    live = slots >= 0
    at = slots[live].long()
    want_k[at // 8, :, at % 8], want_v[at // 8, :, at % 8] = turned[live], rows[:, kv:][live]
    torch.testing.assert_close(cache.k, want_k, rtol=0, atol=0, equal_nan=True)
    assert torch.equal(cache.v, want_v) and torch.isnan(cache.k).any()


def test_streams_graphs_and_the_block():
    """On a stream of its own, and captured and replayed with positions that move on in place."""
    table, axes = pkg.rope_table(64, 200), pkg.rope_axes([8, 12, 12])
    pos = _positions(3, 20, 100)
    x = _randn(20, 4, 64, seed=14)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = pkg.rope(x, pos, table, axes=axes, stream=side)
    a = pkg.rope_axes([8, 12, 12], stream=side)
    side.synchronize()
    assert torch.equal(y, pkg.rope(x, pos, table, axes=axes)) and torch.equal(a, axes)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pkg.rope(x, pos, table, axes=axes)
    for _ in range(3):
        graph.replay()
        assert torch.equal(out, pkg.rope(x, pos, table, axes=axes))
        pos += 7
        torch.cuda.synchronize()
