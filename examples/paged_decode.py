"""Prompts and decode steps of an 8B-class block's attention on 2-bit weights and an 8-bit paged cache.

  python examples/paged_decode.py [--batch 16] [--prompt 1024] [--steps 32] [--bits 8]

Random codes stand for the weights. The prompts of all sequences go through in one call, then each step adds one token a sequence; the
step is captured once as a HIP graph and replayed while positions, slots and lengths move on in place."""
from __future__ import annotations

import argparse
import os
import sys
import time

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2609_24875_amd as sph  # noqa: E402
import synth  # noqa: E402
from paper_2609_24875_amd.block import AttentionBlock  # noqa: E402

HIDDEN, Q_HEADS, KV_HEADS, DIM, PAGE = 4096, 32, 8, 128, 64
DEV = torch.device("cuda:0")


def packed(n, k, seed):
    D, V = synth.FORMATS["W2"]
    g = synth.rng(seed)
    codes = synth.uniform_codes(n, k, D, V, g)
    codes["gmin"], codes["gstep"] = synth.row_scale_group_params(n, k, V, g)
    codes["gstep"] = (codes["gstep"].view("float16") / 64).view("uint16")     # outputs of about the inputs' size
    codes["gmin"] = (codes["gmin"].view("float16") / 64).view("uint16")
    return sph.pack(D, V, codes, synth.random_codebook(D, g), device=DEV)


def main():
    ap = argparse.ArgumentParser(description=__doc__)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--bits", type=int, default=8, choices=(16, 8, 4))
    a = ap.parse_args()
    most = a.prompt + a.steps
    cols = -(-most // PAGE)
    cache = sph.KVCache.empty(a.batch * cols, KV_HEADS, DIM, page_size=PAGE, bits=a.bits, device=DEV)
    table = sph.rope_table(DIM, most, base=500000.0, device=DEV)
    block = AttentionBlock(packed((Q_HEADS + 2 * KV_HEADS) * DIM, HIDDEN, 1), packed(HIDDEN, Q_HEADS * DIM, 2), cache, table, Q_HEADS)

    pages = torch.randperm(a.batch * cols, device=DEV).int().reshape(a.batch, cols)
    seq = torch.arange(a.batch, device=DEV)

    def slots_of(b, at):
        return (pages[b, at // PAGE] * PAGE + at % PAGE).int()

    # every prompt at once
    b, at = seq.repeat_interleave(a.prompt), torch.arange(a.prompt, device=DEV).repeat(a.batch)
    start = (torch.arange(a.batch + 1, device=DEV) * a.prompt).int()
    x = torch.randn(a.batch * a.prompt, HIDDEN, device=DEV).half()
    lens = torch.full((a.batch,), a.prompt, dtype=torch.int32, device=DEV)
    slots, at32 = slots_of(b, at), at.int()
    y = block(x, at32, slots, pages, lens, q_start=start, max_q=a.prompt, max_len=most)
    torch.cuda.synchronize()
    t = time.perf_counter()
    y = block(x, at32, slots, pages, lens, q_start=start, max_q=a.prompt, max_len=most)
    torch.cuda.synchronize()
    print(f"prompts: {a.batch} x {a.prompt} tokens in {1e3 * (time.perf_counter() - t):.2f} ms, output rms {float(y.float().square().mean().sqrt()):.3f}")

    # one token a sequence
    x = torch.randn(a.batch, HIDDEN, device=DEV).half()
    pos, slots = lens.clone(), slots_of(seq, lens.long())
    lens += 1
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(x, pos, slots, pages, lens, max_len=most)           # the workspaces of this stream
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = block(x, pos, slots, pages, lens, max_len=most)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for step in range(a.steps):
        graph.replay()
        if step + 1 < a.steps:
            x.copy_(y)
            pos += 1
            lens += 1
            slots.copy_(slots_of(seq, pos.long()))
    torch.cuda.synchronize()
    us = 1e6 * (time.perf_counter() - t) / a.steps
    print(f"decode: {a.steps} steps of {a.batch} sequences, {us:.1f} us a step, finite: {bool(torch.isfinite(y).all())}, cache {cache.nbytes / 2**20:.0f} MiB")


if __name__ == "__main__":
    main()
