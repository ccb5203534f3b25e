"""The attention half of a decoder block (gemm, kv_append, attention, gemm) against the same in 64 bits, and prompts against
the same tokens one by one."""
from __future__ import annotations

import os
import subprocess
import sys

import numpy as np
import pytest

import synth
from oracle import sph as O

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2609_24875_amd as pkg  # noqa: E402
from paper_2609_24875_amd.block import AttentionBlock  # noqa: E402

DEV = torch.device("cuda:0")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADS, KV, DIM, HIDDEN, PAGE = 6, 2, 64, 256, 16


def _matrix(n, k, seed):
    """A packed matrix with outputs of about the inputs' size, and what it stands for in fp64."""
    D, V = synth.FORMATS["W2"]
    g = synth.rng(seed)
    codes = synth.uniform_codes(n, k, D, V, g)
    codes["gmin"], codes["gstep"] = synth.row_scale_group_params(n, k, V, g)
    for key in ("gmin", "gstep"):
        codes[key] = (codes[key].view(np.float16) / 16).view(np.uint16)
    cb = synth.random_codebook(D, g)
    dense = O.gemm(codes, cb, np.eye(k, dtype=np.float16).view(np.uint16)).T
    return pkg.pack(D, V, codes, cb, device=DEV), torch.from_numpy(np.ascontiguousarray(dense)).to(DEV)


def _block(bits=16, window=0, pages=64):
    w_qkv, d_qkv = _matrix((HEADS + 2 * KV) * DIM, HIDDEN, 1)
    w_o, d_o = _matrix(HIDDEN, HEADS * DIM, 2)
    cache = pkg.KVCache.empty(pages, KV, DIM, page_size=PAGE, bits=bits, device=DEV)
    table = pkg.rope_table(DIM, 512)
    return AttentionBlock(w_qkv, w_o, cache, table, HEADS, window=window), d_qkv, d_o


def _place(pages, lens, new):
    """positions, slots and starts of each sequence's last tokens."""
    pos = torch.cat([torch.arange(ln - m, ln, device=DEV) for ln, m in zip(lens, new)])
    b = torch.arange(len(lens), device=DEV).repeat_interleave(torch.tensor(new, device=DEV))
    slots = pages[b, pos // PAGE] * PAGE + pos % PAGE
    start = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=DEV)
    return pos.int(), slots.int(), start


def _call(block, x, pages, lens, new):
    pos, slots, start = _place(pages, lens, new)
    return block(x, pos, slots, pages, torch.tensor(lens, dtype=torch.int32, device=DEV), q_start=start, max_q=max(new))


def _dense64(x, d_qkv, d_o, window):
    """One sequence from its start, in 64 bits without any rounding."""
    n = x.shape[0]
    rows = (x.double() @ d_qkv.t().contiguous()).view(n, HEADS + 2 * KV, DIM)
    a = torch.arange(n, device=DEV).double()[:, None, None] * torch.tensor(pkg.rope_frequencies(DIM)[0], device=DEV)
    lo, hi = rows[..., :DIM // 2], rows[..., DIM // 2:]
    turned = torch.cat([lo * a.cos() - hi * a.sin(), lo * a.sin() + hi * a.cos()], -1)
    q, k, v = turned[:, :HEADS], turned[:, HEADS:HEADS + KV], rows[:, HEADS + KV:]
    k, v = (t.repeat_interleave(HEADS // KV, 1).transpose(0, 1).contiguous() for t in (k, v))
    s = q.transpose(0, 1) @ k.transpose(1, 2).contiguous() * DIM ** -0.5
    i, j = torch.arange(n, device=DEV)[:, None], torch.arange(n, device=DEV)[None]
    s = s.masked_fill((j > i) | ((j <= i - window) if window else False), -float("inf"))
    o = (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(n, -1)
    return o @ d_o.t().contiguous()


@pytest.mark.parametrize("bits,bar", [(16, 2e-3), (8, 2e-2), (4, 3e-1)])
@pytest.mark.parametrize("window", [0, 20])
def test_block_against_64_bits(window, bits, bar):
    """16 bits: four fp16 roundings (rows, queries, weights and outputs) of 2^-11 each on the way, far inside the library's bar of 2e-3
    in root mean square. A cache of 8 (4) bits moves a value by up to half a step, 1/510 (1/30) of the range of its 32 channels, which
    is about 4 times their root mean square: 2^-8 (2^-3.5) of it in root mean square at most."""
    block, d_qkv, d_o = _block(bits, window)
    lens = [150, 33]
    pages = torch.randperm(64, device=DEV)[:2 * 10].reshape(2, 10).int()
    x = torch.randn(sum(lens), HIDDEN, generator=torch.Generator(DEV).manual_seed(3), device=DEV).half()
    y = _call(block, x, pages, lens, lens)
    for got, rows in zip(y.split(lens), x.split(lens)):
        ref = _dense64(rows, d_qkv, d_o, window)
        assert float((got.double() - ref).square().mean().sqrt() / ref.square().mean().sqrt()) <= bar


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_prompts_in_parts_and_token_by_token_give_the_same(bits):
    """The same tokens in one call, in two and one by one: sums in other orders before each rounding to fp16 or to a code."""
    block, _, _ = _block(bits)
    n = 60
    pages = torch.arange(8, device=DEV).reshape(2, 4).int()
    x = torch.randn(2, n, HIDDEN, generator=torch.Generator(DEV).manual_seed(4), device=DEV).half()
    whole = _call(block, x.reshape(2 * n, HIDDEN), pages, [n, n], [n, n]).view(2, n, HIDDEN).float()
    rms = float(whole.square().mean().sqrt())
    bar = {16: 2e-3, 8: 4e-3, 4: 2e-2}[bits] * rms
    a = _call(block, x[:, :41].reshape(-1, HIDDEN), pages, [41, 41], [41, 41]).view(2, 41, HIDDEN)
    b = _call(block, x[:, 41:].reshape(-1, HIDDEN), pages, [n, n], [n - 41, n - 41]).view(2, n - 41, HIDDEN)
    parts = torch.cat([a, b], 1).float()
    assert float((parts - whole).square().mean().sqrt()) <= bar
    steps = torch.stack([_call(block, x[:, i].contiguous(), pages, [i + 1, i + 1], [1, 1]) for i in range(n)], 1).float()
    assert float((steps - whole).square().mean().sqrt()) <= bar


def test_block_on_a_stream_of_its_own():
    """Calls queued on another stream, while tensors of the current one come and go in memory that was let go."""
    block, _, _ = _block(8)
    lens = [150, 33]
    pages = torch.randperm(64, device=DEV)[:2 * 10].reshape(2, 10).int()
    pos, slots, start = _place(pages, lens, lens)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    xs = [torch.randn(sum(lens), HIDDEN, generator=torch.Generator(DEV).manual_seed(20 + i), device=DEV).half() for i in range(4)]
    want = [block(x, pos, slots, pages, ln, q_start=start, max_q=150) for x in xs]
    torch.cuda.synchronize()
    side, got = torch.cuda.Stream(), []
    for x in xs:
        got.append(block(x, pos, slots, pages, ln, q_start=start, max_q=150, stream=side))
        for n in (HEADS + 2 * KV, HEADS):
            torch.full((sum(lens), n, DIM), 1e4, dtype=torch.float16, device=DEV)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_block_checks_its_parts():
    block, _, _ = _block()
    for args in ((block.w_o, block.w_o), (block.w_qkv, block.w_qkv)):
        with pytest.raises(ValueError):
            AttentionBlock(*args, block.cache, block.table, HEADS)
    with pytest.raises(ValueError):
        AttentionBlock(block.w_qkv, block.w_o, block.cache, block.table, 5)


def test_example_runs():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "paged_decode.py"), "--batch", "3", "--prompt", "100", "--steps", "4"],
                       capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "prompts: 3 x 100" in r.stdout and "finite: True" in r.stdout
