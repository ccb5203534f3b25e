"""The attention half of a decoder block on packed weights and a paged cache: fused q/k/v product
(``gemm``), rotation and cache write (``kv_append``), attention over the pages (``attention``) and o product
(``gemm``): four calls, for one new token a sequence, for several, and for prompts."""
from __future__ import annotations

from . import attn as A
from . import sph as B


class AttentionBlock:
    """``w_qkv``: packed [(q heads + 2 kv heads) * channels][hidden], the rows of q, k and v one under the
    other; ``w_o``: packed [hidden][q heads * channels]; ``cache``: this layer's pages; ``table``: rotary positions
    (``rope_table``), shared by all layers. Graphs of a block use the products' workspaces of the stream that captured them, as graphs of
    ``gemm`` do, so their replays are ordered with each other and with the block's calls on that stream."""

    def __init__(self, w_qkv: B.SphWeights, w_o: B.SphWeights, cache: A.KVCache, table, q_heads: int, interleaved: bool = False,
                 window: int = 0, scale: float | None = None):
        dim = cache.head_dim
        if q_heads < 1 or q_heads % cache.kv_heads:
            raise ValueError(f"{q_heads} query heads over {cache.kv_heads} kv heads")
        if w_qkv.n != (q_heads + 2 * cache.kv_heads) * dim or w_o.k != q_heads * dim or w_o.n != w_qkv.k:
            raise ValueError(f"q/k/v {w_qkv.n} x {w_qkv.k} and o {w_o.n} x {w_o.k} do not fit {q_heads} + 2 * {cache.kv_heads} heads of {dim}")
        self.w_qkv, self.w_o, self.cache, self.table = w_qkv, w_o, cache, table
        self.q_heads, self.interleaved, self.window, self.scale = q_heads, interleaved, window, scale

    def __call__(self, x, positions, slots, pages, seq_lens, q_start=None, max_q: int = 1, max_len: int | None = None, stream=None):
        """y fp16 [tokens][hidden] of x fp16 [tokens][hidden], the new tokens of all sequences one after the other. positions, slots:
        int32 [tokens], where each stands and is kept; pages, seq_lens, q_start, max_q, max_len, stream: as ``attention``."""
        import torch
        if stream is not None:                  # so that the rows between the calls, let go at the end, are that stream's
            with torch.cuda.stream(stream):
                return self(x, positions, slots, pages, seq_lens, q_start, max_q, max_len)
        h, kv, n = self.q_heads, self.cache.kv_heads, x.shape[0]
        rows = B.gemm(self.w_qkv, x, out_dtype=torch.float16).view(n, h + 2 * kv, self.cache.head_dim)
        # the queries turn where they are
        q = A.kv_append(self.cache, rows[:, h:h + kv], rows[:, h + kv:], slots, positions=positions, table=self.table,
                        interleaved=self.interleaved, q=rows[:, :h], q_out=rows[:, :h])
        o = torch.empty((n, h, self.cache.head_dim), dtype=torch.float16, device=x.device)
        A.attention(q, self.cache, pages, seq_lens, q_start=q_start, max_q=max_q, max_len=max_len, window=self.window, scale=self.scale,
                    out=o)
        return B.gemm(self.w_o, o.view(n, -1), out_dtype=torch.float16)
