"""The decoder block with positions along several axes and behind shared prefixes: against the calls that it stands for, and a prompt
computed once for all against the same prompt in every sequence."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_24875_amd as pkg  # noqa: E402
from paper_2609_24875_amd.block import AttentionBlock  # noqa: E402
from test_gpu_block import DIM, HEADS, HIDDEN, KV, PAGE, _block, _call, _place  # noqa: E402

DEV = torch.device("cuda:0")


def _x(n, seed):
    return torch.randn(n, HIDDEN, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).half()


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def test_positions_along_axes():
    """The same bits as the block's calls one after the other; positions that agree along all axes, as without axes."""
    block, _, _ = _block(8)
    axes = pkg.rope_axes([8, 12, 12])
    several = AttentionBlock(block.w_qkv, block.w_o, block.cache, block.table, HEADS, axes=axes)
    lens = [50, 33]
    pages = torch.randperm(64, device=DEV)[:2 * 4].reshape(2, 4).int()
    pos, slots, start = _place(pages, lens, lens)
    x, ln = _x(sum(lens), 1), _i32(lens)
    same = pos.expand(3, -1).contiguous()
    y = several(x, same, slots, pages, ln, q_start=start, max_q=50)
    assert torch.equal(y, block(x, pos, slots, pages, ln, q_start=start, max_q=50))
    grid = torch.stack([pos, pos // 7, pos % 7]).contiguous()
    y = several(x, grid, slots, pages, ln, q_start=start, max_q=50)
    rows = pkg.gemm(block.w_qkv, x, out_dtype=torch.float16).view(-1, HEADS + 2 * KV, DIM)
    q = pkg.kv_append(block.cache, rows[:, HEADS:HEADS + KV], rows[:, HEADS + KV:], slots, positions=grid, table=block.table, q=rows[:, :HEADS], axes=axes)
    o = pkg.attention(q, block.cache, pages, ln, q_start=start, max_q=50)
    assert torch.equal(y, pkg.gemm(block.w_o, o.view(-1, HEADS * DIM), out_dtype=torch.float16))


@pytest.mark.parametrize("bits", [16, 8])
def test_a_prompt_computed_once_for_all(bits):
    """Three sequences that begin alike: whole, and behind a prefix. The same keys and values, so what differs are sums' orders before
    the roundings to fp16 (bar as for prompts in parts)."""
    block, _, _ = _block(bits)
    pre, lens = 45, [30, 7, 16]
    head, tails = _x(pre, 2), [_x(n, 3 + i) for i, n in enumerate(lens)]
    pages = torch.arange(3 * 5, device=DEV).reshape(3, 5).int()
    whole = [pre + n for n in lens]
    want = _call(block, torch.cat([torch.cat([head, t]) for t in tails]), pages, whole, whole).split(whole)
    ppages, own = torch.arange(20, 23, device=DEV).int()[None], torch.arange(30, 36, device=DEV).reshape(3, 2).int()
    first = _call(block, head, ppages, [pre], [pre])
    assert float((first.float() - want[0][:pre].float()).square().mean().sqrt()) <= 4e-3 * float(want[0].float().square().mean().sqrt())
    pos, slots, start = _place(own, lens, lens)
    prefix = dict(prefix_pages=ppages, prefix_lens=_i32([pre]))
    got = block(torch.cat(tails), pos + pre, slots, own, _i32(lens), q_start=start, max_q=30, prefix=prefix)
    for g, w in zip(got.split(lens), want):
        w = w[pre:].float()
        assert float((g.float() - w).square().mean().sqrt()) <= 4e-3 * float(w.square().mean().sqrt())
    # and one more token each, on a stream of its own, by two groups
    x = _x(3, 9)
    pos, slots, _ = _place(own, [n + 1 for n in lens], [1, 1, 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    two = dict(prefix_pages=ppages.expand(2, -1).contiguous(), prefix_lens=_i32([pre, pre]), first=_i32([0, 2, 3]), max_group=2)
    y = block(x, pos + pre, slots, own, _i32([n + 1 for n in lens]), stream=side, prefix=two)
    side.synchronize()
    z = block(x, pos + pre, slots, own, _i32([n + 1 for n in lens]), prefix=prefix)
    assert torch.isfinite(y).all() and float((y.float() - z.float()).square().mean().sqrt()) <= 4e-3 * float(z.float().square().mean().sqrt())


def test_a_window_and_a_prefix_are_refused():
    block, _, _ = _block(16, window=20)
    with pytest.raises(ValueError):
        block(_x(1, 1), _i32([5]), _i32([5]), _i32([[0]]), _i32([6]), prefix=dict(prefix_pages=_i32([[1]]), prefix_lens=_i32([4])))
