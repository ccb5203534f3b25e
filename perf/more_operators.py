"""What long prompts of text, images and video add to a decoder block's cache and attention.

Four operators: rotary positions with several axes, for images and video, where every pair of
channels turns by the position along its own axis (``rope``, its gradient, and ``append``: the same
on the way into the paged cache); ``shared`` (attention of sequences that share long prefixes, each
prefix read once for all of them), ``weights`` (how much attention every cached token got, added to
what it got before) and ``evict`` (sequences shrink to the tokens with the largest of these sums).
Head counts come from the library's benchmark configurations (8B- and 32B-class backbones: 32 or 40
query heads over 8 key-value heads of 128 channels) or are generic.

Where ``own`` is false, ``run`` computes the same from elementary torch operations in 32 bits;
where it is true it calls the library. ``exact`` recomputes the results in 64 bits.

Cache pages are plain tensors: fp16 ``[pages][kv heads][tokens a page][channels]``, or codes (uint8;
at 4 bits the 32-bit word of channels 8w..8w+7 holds channel 8w + 2i at bit 4i and 8w + 2i + 1 at
bit 16 + 4i) with an fp16 (offset, step) pair for every 32 channels. A code q stands for the fp16
number offset + q step.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
GROUP = 32                                        # channels that share an offset and a step
DTYPES = {"f16": torch.float16, "f32": torch.float32}
BASE = 500000.0                                   # of the rotary frequencies


def listed():
    return [
        # Queries and keys of a video prompt: time, height and width each turn a part of the pairs.
        {"name": "rope_video", "op": "rope", "tokens": 8192, "heads": 48, "dim": 128, "sections": "16,24,24", "cycled": False,
         "restart": False, "inter": False, "dtype": "f16", "grad": False, "max_pos": 32768, "pad": 8},
        # A training step over image patches: two axes with frequencies of their own, neighbouring channels as pairs,
        # fp32, an odd number of tokens.
        {"name": "rope_image_grad", "op": "rope", "tokens": 2051, "heads": 32, "dim": 128, "sections": "32,32", "cycled": False,
         "restart": True, "inter": True, "dtype": "f32", "grad": True, "max_pos": 8192, "pad": 0},
        # The patches of one image written to an 8-bit cache, axes taking the pairs in turn.
        {"name": "append_image_q8", "op": "append", "tokens": 1369, "run": 1369, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "sections": "24,20,20", "cycled": True, "restart": False, "inter": False, "bits": 8, "page": 64, "max_pos": 32768},
        # Four answers early in a conversation behind a short common prompt: the smallest attention, where latency counts.
        {"name": "shared_short", "op": "shared", "groups": 1, "size": 4, "q_len": 1, "prefix": 1031, "ctx": 37, "ragged": True,
         "q_heads": 32, "kv_heads": 8, "dim": 128, "bits": 16, "page": 64},
        # 32 conversations behind one system prompt.
        {"name": "shared_batch", "op": "shared", "groups": 1, "size": 32, "q_len": 1, "prefix": 8192, "ctx": 512, "ragged": True,
         "q_heads": 32, "kv_heads": 8, "dim": 128, "bits": 16, "page": 64},
        # Eight answers each to eight prompts of several lengths, on the 32B-class heads, 8 bits, small pages.
        {"name": "shared_samples_q8", "op": "shared", "groups": 8, "size": 8, "q_len": 1, "prefix": 4099, "ctx": 700, "ragged": True,
         "q_heads": 40, "kv_heads": 8, "dim": 128, "bits": 8, "page": 16},
        # Drafted tokens of 24 sequences checked behind one prompt, 4 bits, 96 channels.
        {"name": "shared_draft_q4", "op": "shared", "groups": 1, "size": 24, "q_len": 5, "prefix": 5003, "ctx": 403, "ragged": True,
         "q_heads": 12, "kv_heads": 4, "dim": 96, "bits": 4, "page": 32},
        # Many questions about one long document: the largest.
        {"name": "shared_document", "op": "shared", "groups": 1, "size": 128, "q_len": 1, "prefix": 32768, "ctx": 1024, "ragged": False,
         "q_heads": 32, "kv_heads": 8, "dim": 128, "bits": 16, "page": 64},
        # A decode step's weights of 64 sequences of all lengths up to 8192 from an 8-bit cache.
        {"name": "weights_batch_q8", "op": "weights", "batch": 64, "q_len": 1, "ctx": 8192, "ragged": True, "q_heads": 32,
         "kv_heads": 8, "dim": 128, "bits": 8, "page": 64, "window": 0, "per_head": True},
        # What the last 2048 tokens of a 16384-token prompt looked at, over all heads.
        {"name": "weights_prompt", "op": "weights", "batch": 1, "q_len": 2048, "ctx": 16384, "ragged": False, "q_heads": 32,
         "kv_heads": 8, "dim": 128, "bits": 16, "page": 64, "window": 0, "per_head": False},
        # One short sequence of a 4-bit cache halved, all heads alike: latency.
        {"name": "evict_short_q4", "op": "evict", "batch": 1, "ctx": 517, "ragged": False, "keep": 256, "recent": 32, "first": 4,
         "kv_heads": 8, "dim": 128, "bits": 4, "page": 16, "per_head": False},
        # 32 sequences of up to 8192 tokens shrunk to half of that, each head choosing its own.
        {"name": "evict_batch", "op": "evict", "batch": 32, "ctx": 8192, "ragged": True, "keep": 4096, "recent": 256, "first": 4,
         "kv_heads": 8, "dim": 128, "bits": 16, "page": 64, "per_head": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _sections(rng, pairs):
    """2 to 4 axes' shares of the pairs: in steps of eight, or any."""
    n = rng.choice([2, 3, 3, 4])
    step = rng.choice([8, 8, 1]) if pairs >= 8 * n else 1
    cuts = sorted(rng.sample(range(1, pairs // step), n - 1))
    return ",".join(str(step * (b - a)) for a, b in zip([0] + cuts, cuts + [pairs // step]))


def draw(rng):
    op = rng.choice(["rope", "rope", "append", "shared", "shared", "shared", "shared", "weights", "weights", "weights", "evict", "evict"])
    dim = rng.choice([64, 96, 128, 128, 128, 128, 192, 256])
    bits = rng.choice([16, 8, 4])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    kv, group = rng.choice([(8, 4), (8, 5), (8, 4), (4, 3), (1, 16), (2, 7), (16, 1), (4, 8)])
    rot = rng.choice([dim, dim, dim // 2])
    turn = {"sections": _sections(rng, rot // 2), "cycled": rng.random() < 0.3, "restart": rng.random() < 0.4, "inter": rng.random() < 0.5}
    if op == "rope":
        heads = rng.choice([1, 7, 8, 32, 40, 48])
        grad = rng.random() < 0.4
        return {"op": op, "tokens": _log(rng, 1, min(32768, 25 * 10**6 // (heads * dim) * (1 if grad else 2))), "heads": heads,
                "dim": dim, **turn, "dtype": rng.choice(["f16", "f32"]), "grad": grad, "max_pos": 32768, "pad": rng.choice([0, 0, 8])}
    if op == "append":
        tokens = _log(rng, 1, 8192 * 56 * 128 // ((group + 2) * kv * dim))
        return {"op": op, "tokens": tokens, "run": rng.randint(1 + tokens // 16, tokens), "q_heads": kv * group,
                "kv_heads": kv, "dim": dim, **turn, "bits": bits, "page": page, "max_pos": 131072}
    heads = {"kv_heads": kv, "dim": dim, "bits": bits, "page": page}
    if op == "shared":
        groups = rng.choice([1, 1, 1, _log(rng, 2, 16)])
        size = _log(rng, 2, max(2, 128 // groups))
        # rows times keys at most the largest listed case's
        ctx = _log(rng, 1, min(4096, (1 << 27) // (groups * size * kv * dim)))
        most = 128 * 32768 * 32 * 128 // (size * kv * group * dim)
        prefix = _log(rng, 64, min(32768, (1 << 25) // (groups * kv * dim), max(64, most // groups - ctx)))
        q_len = 1 if rng.random() < 0.7 else _log(rng, 1, max(1, min(ctx, 8, most // (groups * (prefix + ctx)))))
        return {"op": op, "groups": groups, "size": size, "q_len": q_len, "prefix": prefix, "ctx": ctx, "ragged": rng.random() < 0.6,
                "q_heads": kv * group, **heads}
    batch = _log(rng, 1, 96)
    ctx = _log(rng, 1, min(131072, (1 << 28) // (batch * kv * dim)))
    if op == "weights":
        kind = rng.choice(["one", "one", "one", "few", "prompt"])
        q_len = 1
        if kind != "one":
            pairs = (1 << 24) * 32 * 128 // (batch * kv * group * dim)
            q_len = _log(rng, 1, max(1, min(ctx, 8 if kind == "few" else 2048, pairs // ctx)))
        return {"op": op, "batch": batch, "q_len": q_len, "ctx": ctx, "ragged": rng.random() < 0.5, "q_heads": kv * group, **heads,
                "window": rng.choice([0, 0, 0, _log(rng, 16, 4096)]), "per_head": rng.random() < 0.7}
    ctx = max(1, ctx // 2) if batch * ctx * kv * dim > 1 << 27 else ctx
    keep = rng.randint(1, ctx)
    recent = rng.randint(0, keep // 4)
    return {"op": op, "batch": batch, "ctx": ctx, "ragged": rng.random() < 0.5, "keep": keep, "recent": recent,
            "first": min(keep - recent, rng.choice([0, 1, 4])), **heads, "per_head": rng.random() < 0.7}


# ------------------------------------------------------------------------------------ inputs

def _gen(seed, stream):
    return torch.Generator(DEVICE).manual_seed((seed * 64 + stream) % (1 << 62))


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _shares(case):
    return [int(n) for n in case["sections"].split(",")]


def _axis_of(case):
    """Axis of every pair: one axis's share behind the other's, or taken in turn while they last."""
    left = _shares(case)
    if not case["cycled"]:
        return [a for a, n in enumerate(left) for _ in range(n)]
    got = []
    while any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                got.append(a)
    return got


def _freqs(case):
    """Angle a position of every pair, fp64: one spectrum over all pairs, or one for each axis."""
    axis, share = _axis_of(case), _shares(case)
    f, seen = [], [0] * len(share)
    for i, a in enumerate(axis):
        f.append(BASE ** -(seen[a] / share[a] if case["restart"] else i / len(axis)))
        seen[a] += 1
    return torch.tensor(f, dtype=torch.float64, device=DEVICE)


def _table(case):
    """(cos, sin) of every position and pair, fp32 [max_pos][pairs][2]: kept by the program."""
    a = torch.arange(case["max_pos"], dtype=torch.float64, device=DEVICE)[:, None] * _freqs(case)
    return torch.stack([a.cos(), a.sin()], dim=-1).float()


def _positions(case, seed):
    """int32 [axes][tokens]: a run of text, whose axes agree, then frames of patches in rows."""
    n, axes = case["tokens"], len(_shares(case))
    text = n // 8
    width = max(1, math.isqrt(max(1, (n - text) // (4 if axes > 2 else 1))))
    t = torch.arange(n, device=DEVICE)
    i = (t - text).clamp_min(0)
    grid = [i // (width * width), i // width % width, i % width, i % 7] if axes > 2 else [i // width, i % width]
    start = int(torch.randint(0, max(1, case["max_pos"] - n - 8), (1,), generator=_gen(seed, 2), device=DEVICE))
    return torch.stack([torch.where(t < text, t, text + g) for g in grid[:axes]]).add_(start).int()


def _slots(case, seed, pages):
    """The cache slots of the tokens: runs of consecutive tokens over pages in no order."""
    run, page = case["run"], case["page"]
    t = torch.arange(case["tokens"], device=DEVICE)
    per = -(-run // page)                         # pages of a run
    order = torch.randperm(pages, generator=_gen(seed, 9), device=DEVICE)
    return (order[(t // run) * per + t % run // page] * page + t % run % page).int()


def _channels(n, seed, stream):
    """Channel magnitudes of a head: they differ by a factor of two or three."""
    return torch.exp(0.25 * torch.randn(n, generator=_gen(seed, stream), device=DEVICE))


def _pool(case, pages, seed, stream):
    """Cache pages with the statistics of keys or values: bell-shaped, channels of several sizes."""
    kv, page, dim, bits = case["kv_heads"], case["page"], case["dim"], case["bits"]
    g = _gen(seed, stream)
    x = torch.randn((pages, kv, page, dim), generator=g, device=DEVICE, dtype=torch.float32)
    if bits == 16:
        return x.mul_(_channels(dim, seed, stream + 1)).half(), None
    top = (1 << bits) - 1
    codes = x.mul_(top / 4.2).add_(0.5 * top).round_().clamp_(0, top).to(torch.uint8)
    size = _channels(dim // GROUP, seed, stream + 1) * (0.8 + 0.4 * torch.rand((pages, kv, page, dim // GROUP), generator=g, device=DEVICE))
    return _pack(codes, bits), torch.stack([-2.1 * size, 4.2 / top * size], dim=-1).half()


def _pools(s, case, pages, seed):
    s["k"], s["k_par"] = _pool(case, pages, seed, 10)
    s["v"], s["v_par"] = _pool(case, pages, seed, 12)


def _empty_pool(case, pages):
    kv, page, dim, bits = case["kv_heads"], case["page"], case["dim"], case["bits"]
    if bits == 16:
        return torch.zeros((pages, kv, page, dim), dtype=torch.float16, device=DEVICE), None
    return (torch.zeros((pages, kv, page, dim * bits // 8), dtype=torch.uint8, device=DEVICE),
            torch.zeros((pages, kv, page, dim // GROUP, 2), dtype=torch.float16, device=DEVICE))


def _lens(batch, m, ctx, ragged):
    """(cached tokens, new tokens among them) of every sequence. A ragged batch has an idle slot."""
    if not ragged:
        return [ctx] * batch, [m] * batch
    new = [1 + (7 * i) % m for i in range(batch)]
    return [0 if batch > 1 and i == 0 else new[i] + round((ctx - m) * (0.61803399 * i % 1.0) ** 2) for i in range(batch)], new


def _prefixes(case):
    """(tokens of every prefix, sequences behind each): several ragged ones differ in both, the number of sequences stays."""
    n, size = case["groups"], case["size"]
    if not case["ragged"] or n == 1:
        return [case["prefix"]] * n, [size] * n
    lens = [max(1, round(case["prefix"] * (1.0 - 0.61803399 * i % 1.0))) for i in range(n)]
    more = [(i % 2) * (size // 4) for i in range(n // 2 * 2)] + [0] * (n % 2)
    less = [((i + 1) % 2) * (size // 4) for i in range(n // 2 * 2)] + [0] * (n % 2)
    return lens, [size + a - b for a, b in zip(more, less)]


def _own_lens(case):
    return _lens(sum(_prefixes(case)[1]), case["q_len"], case["ctx"], case["ragged"])


def _starts(new):
    return [sum(new[:i]) for i in range(len(new) + 1)]


def _tables(s, case, rows, seed):
    """Page tables of rows = [(name, sequences, columns)] over one pool, in no order."""
    total = sum(n * c for _, n, c in rows)
    order = torch.randperm(total, generator=_gen(seed, 9), device=DEVICE).int()
    at = 0
    for name, n, c in rows:
        s[name] = order[at:at + n * c].reshape(n, c)
        at += n * c
    return total


def prepare(case, seed):
    s = dict(case)
    op = case["op"]
    if op in ("rope", "append"):
        s["table"] = _table(case)
        s["axes"] = torch.tensor(_axis_of(case), dtype=torch.uint8, device=DEVICE)
        s["pos"] = _positions(case, seed)
    if op == "rope":
        n, h, d = case["tokens"], case["heads"], case["dim"]
        dt = DTYPES[case["dtype"]]
        s["x"] = torch.randn((n, h + case["pad"], d), generator=_gen(seed, 0), device=DEVICE).to(dt)[:, :h]
        s["g"] = torch.randn((n, h, d), generator=_gen(seed, 1), device=DEVICE).to(dt) if case["grad"] else None
        return s
    page = case["page"]
    if op == "append":
        pages = -(-case["tokens"] // case["run"]) * -(-case["run"] // page) + 3
        q, kv = case["q_heads"], case["kv_heads"]
        # the output of the fused q/k/v product
        rows = torch.randn((case["tokens"], q + 2 * kv, case["dim"]), generator=_gen(seed, 0), device=DEVICE)
        rows = (rows * _channels(case["dim"], seed, 1)).half()
        s["q"], s["kn"], s["vn"] = rows[:, :q], rows[:, q:q + kv], rows[:, q + kv:]
        s["slots"] = _slots(case, seed, pages)
        s["k"], s["k_par"] = _empty_pool(case, pages)
        s["v"], s["v_par"] = _empty_pool(case, pages)
    elif op == "shared":
        plens, sizes = _prefixes(case)
        lens, new = _own_lens(case)
        total = _tables(s, case, [("prefix_pages", len(plens), -(-case["prefix"] // page)), ("pages", len(lens), -(-case["ctx"] // page))], seed)
        _pools(s, case, total, seed)
        s["prefix_lens"], s["lens"], s["sizes"] = _int(plens), _int(lens), sizes
        s["at"], s["start"] = _int(_starts(sizes)), _int(_starts(new))
        s["q"] = (1.5 * torch.randn((sum(new), case["q_heads"], case["dim"]), generator=_gen(seed, 0), device=DEVICE)).half()
    elif op == "weights":
        lens, new = _lens(case["batch"], case["q_len"], case["ctx"], case["ragged"])
        _pools(s, case, _tables(s, case, [("pages", len(lens), -(-case["ctx"] // page))], seed), seed)
        s["lens"], s["start"] = _int(lens), _int(_starts(new))
        s["q"] = (1.5 * torch.randn((sum(new), case["q_heads"], case["dim"]), generator=_gen(seed, 0), device=DEVICE)).half()
        heads = case["kv_heads"] if case["per_head"] else 1
        # what earlier tokens gave: much to a few, little to most
        before = torch.rand((case["batch"], heads, case["ctx"]), generator=_gen(seed, 3), device=DEVICE).clamp_min_(1e-3).reciprocal_().mul_(0.01)
        old = s["lens"] - (s["start"][1:] - s["start"][:-1])
        s["before"] = before * (torch.arange(case["ctx"], device=DEVICE) < old[:, None, None])
        with torch.no_grad():                     # the attention's own result
            x, which = _scores(s)
            s["lse"] = _to_tokens(s, torch.logsumexp(x, dim=-1, keepdim=True), which)[..., 0]
    else:
        lens, _ = _lens(case["batch"], 1, case["ctx"], case["ragged"])
        b, keep = case["batch"], min(case["keep"], case["ctx"])
        cols, new_cols = -(-case["ctx"] // page), -(-keep // page)
        # new pages come first in the pool; other sequences may share the old ones
        s["pages"] = (b * new_cols + torch.randperm(b * cols, generator=_gen(seed, 9), device=DEVICE)).int().reshape(b, cols)
        s["to"] = torch.randperm(b * new_cols, generator=_gen(seed, 8), device=DEVICE).int().reshape(b, new_cols)
        _pools(s, case, b * (cols + new_cols), seed)
        s["new_pages"] = b * new_cols
        for x in ("k", "v", "k_par", "v_par"):
            if s[x] is not None:
                s[x][:b * new_cols] = 0
        s["lens"] = _int(lens)
        heads = case["kv_heads"] if case["per_head"] else 1
        sums = torch.rand((b, heads, case["ctx"]), generator=_gen(seed, 3), device=DEVICE).clamp_min_(1e-3).reciprocal_()
        # tokens that got next to nothing are many and alike: ties
        s["sums"] = torch.where(sums < 1.4, 0.0, sums)
        if case["bits"] < 16:                     # where the kept tokens are, to read them back
            i = torch.arange(keep, device=DEVICE)
            s["slots"] = (s["to"].long()[:, i // page] * page + i % page).int().flatten()
    if own:                                       # the handle that a program keeps beside its pages
        import paper_2609_24875_amd as sph
        s["cache"] = sph.KVCache(s["k"], s["v"], s["k_par"], s["v_par"], bits=case["bits"])
    return s


# ------------------------------------------------------------------------------------ the operators

def run(s):
    if own:
        return _run_own(s)
    with torch.no_grad():
        return {"rope": _plain_rope, "append": _plain_append, "shared": _plain_shared, "weights": _plain_weights, "evict": _plain_evict}[s["op"]](s)


def _run_own(s):
    import paper_2609_24875_amd as sph
    from paper_2609_24875_amd import train
    if s["op"] == "rope":
        if not s["grad"]:
            return {"y": sph.rope(s["x"], s["pos"], s["table"], interleaved=s["inter"], axes=s["axes"])}
        x = s["x"].detach().requires_grad_(True)
        y = train.rope(x, s["pos"], s["table"], interleaved=s["inter"], axes=s["axes"])
        (dx,) = torch.autograd.grad(y, x, s["g"])
        return {"y": y.detach(), "dx": dx}
    if s["op"] == "append":
        q = sph.kv_append(s["cache"], s["kn"], s["vn"], s["slots"], positions=s["pos"], table=s["table"],
                          interleaved=s["inter"], q=s["q"], axes=s["axes"])
        k, v = sph.kv_read(s["cache"], s["slots"])
        return {"q": q, "k": k, "v": v}
    if s["op"] == "shared":
        more = {} if s["groups"] == 1 else {"first": s["at"], "max_group": max(s["sizes"])}
        if s["q_len"] > 1:
            more |= {"q_start": s["start"], "max_q": s["q_len"]}
        o, lse = sph.attention_shared(s["q"], s["cache"], s["prefix_pages"], s["prefix_lens"], s["pages"], s["lens"],
                                      max_prefix=s["prefix"], max_len=s["ctx"], return_lse=True, **more)
        return {"o": o, "lse": lse}
    if s["op"] == "weights":
        more = {"q_start": s["start"], "max_q": s["q_len"]} if s["q_len"] > 1 else {}
        return {"sums": sph.attention_weights(s["q"], s["cache"], s["pages"], s["lens"], s["lse"], before=s["before"],
                                              per_head=s["per_head"], max_len=s["ctx"], window=s["window"], **more)}
    lens, sums, kept = sph.kv_evict(s["cache"], s["pages"], s["lens"], s["sums"], min(s["keep"], s["ctx"]), recent=s["recent"],
                                    first=s["first"], to_pages=s["to"], max_len=s["ctx"])
    got = {"lens": lens, "sums": sums, "kept": kept}
    if s["bits"] == 16:
        return got | {"k": s["k"][:s["new_pages"]], "v": s["v"][:s["new_pages"]]}
    k, v = sph.kv_read(s["cache"], s["slots"])
    return got | {"k": k, "v": v}


def _rotate(x, s, sign=1.0):
    """Pairs of the first channels of x (fp32) turned by the table's angles at their axis's position, or back."""
    half = s["table"].shape[1]
    cs = s["table"][s["pos"].long()[s["axes"].long()].t(), torch.arange(half, device=x.device)][:, None]
    c, sn = cs[..., 0], sign * cs[..., 1]
    head, rest = x[..., :2 * half], x[..., 2 * half:]
    if s["inter"]:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([a * c - b * sn, a * sn + b * c], dim=-1).flatten(-2)
    else:
        a, b = head[..., :half], head[..., half:]
        turned = torch.cat([a * c - b * sn, a * sn + b * c], dim=-1)
    return torch.cat([turned, rest], dim=-1)


def _plain_rope(s):
    y = _rotate(s["x"].float(), s).to(s["x"].dtype)
    if not s["grad"]:
        return {"y": y}
    return {"y": y, "dx": _rotate(s["g"].float(), s, -1.0).to(s["x"].dtype)}


def _shifts(device):
    i = torch.arange(8, dtype=torch.int32, device=device)
    return 4 * (i // 2) + 16 * (i % 2)


def _pack(codes, bits):
    if bits == 8:
        return codes
    w = (codes.unflatten(-1, (-1, 8)).long() << _shifts(codes.device).long()).sum(dim=-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).int().view(torch.uint8)


def _unpack(codes, bits):
    if bits == 8:
        return codes.float()
    return ((codes.view(torch.int32)[..., None] >> _shifts(codes.device)) & 15).flatten(-2).float()


def _values(codes, par, bits):
    """What pages stand for, in fp32."""
    if bits == 16:
        return codes.float()
    q = _unpack(codes, bits).unflatten(-1, (-1, GROUP))
    p = par.float()
    return (p[..., 0:1] + q * p[..., 1:2]).flatten(-2).half().float()


def _quantise(x, bits):
    """fp32 values as fp16, or as codes and (offset, step) pairs."""
    if bits == 16:
        return x.half(), None
    g = x.unflatten(-1, (-1, GROUP))
    top = (1 << bits) - 1
    off = g.amin(dim=-1, keepdim=True).half().float()
    step = ((g.amax(dim=-1, keepdim=True) - off) / top).half().float()
    q = torch.where(step > 0, ((g - off) / torch.where(step > 0, step, 1.0)).round().clamp(0, top), 0.0)
    return _pack(q.flatten(-2).to(torch.uint8), bits), torch.cat([off, step], dim=-1).half()


def _read(s, slots):
    at, off = (slots // s["page"]).long(), (slots % s["page"]).long()
    got = [_values(s[x][at, :, off], s[x + "_par"][at, :, off] if s["bits"] < 16 else None, s["bits"]).half() for x in "kv"]
    return {"k": got[0], "v": got[1]}


def _plain_append(s):
    at, off = (s["slots"] // s["page"]).long(), (s["slots"] % s["page"]).long()
    q = _rotate(s["q"].float(), s).half()
    k, k_par = _quantise(_rotate(s["kn"].float(), s), s["bits"])
    v, v_par = _quantise(s["vn"].float(), s["bits"])
    s["k"][at, :, off], s["v"][at, :, off] = k, v
    if k_par is not None:
        s["k_par"][at, :, off], s["v_par"][at, :, off] = k_par, v_par
    return {"q": q, **_read(s, s["slots"])}


def _gathered(s, x, pages):
    """Keys or values of every sequence side by side, fp32 [sequences][kv heads][keys][channels]."""
    at = pages.long()
    got = _values(s[x][at], s[x + "_par"][at] if s["bits"] < 16 else None, s["bits"])
    return got.transpose(1, 2).flatten(2, 3)


def _padded(s):
    """Queries fp32 [sequences][new tokens][heads][channels], which of them are real, and their positions among the own tokens."""
    m, dev = s["q_len"], s["q"].device
    new = (s["start"][1:] - s["start"][:-1]).long()
    t = torch.arange(m, device=dev)
    row = (s["start"][:-1].long()[:, None] + t[None]).clamp_max(s["q"].shape[0] - 1)
    return s["q"][row].float(), t[None] < new[:, None], s["lens"].long()[:, None] - new[:, None] + t[None]


def _by_kv_head(s, q):
    """[sequences][tokens][heads][..] as [sequences][kv heads][tokens * heads of the group][..]."""
    b, m, h, kv = q.shape[0], q.shape[1], q.shape[2], s["kv_heads"]
    return q.reshape(b, m, kv, h // kv, -1).transpose(1, 2).reshape(b, kv, m * (h // kv), -1)


def _to_tokens(s, x, real):
    """[sequences][kv heads][tokens * group][..] as [tokens][heads][..] of the real tokens."""
    b, kv, m = x.shape[0], s["kv_heads"], s["q_len"]
    x = x.reshape(b, kv, m, -1, x.shape[-1]).transpose(1, 2).flatten(2, 3)
    which = torch.arange(s["q"].shape[0], device=x.device)
    at = torch.searchsorted(s["start"][1:].long(), which, right=True)
    return x[at, which - s["start"][at].long()]


def _scores(s):
    """Scores of all rows over the sequences' own tokens, -inf where a row does not see a key."""
    q, real, pos = _padded(s)
    g = s["q_heads"] // s["kv_heads"]
    k = _gathered(s, "k", s["pages"])
    key = torch.arange(k.shape[2], device=k.device)
    seen = (key <= pos[..., None]) & real[..., None]
    if s.get("window"):
        seen &= key > pos[..., None] - s["window"]
    seen = seen[:, None, :, None].expand(-1, 1, -1, g, -1).flatten(2, 3)
    x = torch.matmul(_by_kv_head(s, q), k.transpose(2, 3).contiguous()).mul_(s["dim"] ** -0.5)
    return x.masked_fill_(~seen, -math.inf), real


def _plain_shared(s):
    kv, dim, m, n = s["kv_heads"], s["dim"], s["q_len"], s["groups"]
    x_own, real = _scores(s)
    b, rows = x_own.shape[0], x_own.shape[2]
    # the sequences of a prefix beside each other: [prefixes][kv heads][sequences * rows]
    most = max(s["sizes"])
    seq = (s["at"][:-1].long()[:, None] + torch.arange(most, device=x_own.device)).clamp_max(b - 1)
    q = _by_kv_head(s, _padded(s)[0])[seq].transpose(1, 2).reshape(n, kv, most * rows, dim)
    k, v = _gathered(s, "k", s["prefix_pages"]), _gathered(s, "v", s["prefix_pages"])
    hidden = torch.arange(k.shape[2], device=k.device) >= s["prefix_lens"][:, None, None, None]
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(dim ** -0.5).masked_fill_(hidden, -math.inf)
    # each sequence's place in its group
    which = torch.searchsorted(s["at"][1:].long(), torch.arange(b, device=x.device), right=True)
    place = torch.arange(b, device=x.device) - s["at"].long()[which]

    def of_sequences(y):
        return y.reshape(n, kv, most, rows, -1).transpose(1, 2)[which, place]

    def of_groups(y):
        return y[seq].transpose(1, 2).reshape(n, kv, most * rows, -1)

    top = torch.maximum(x_own.amax(dim=-1, keepdim=True), of_sequences(x.amax(dim=-1, keepdim=True)))
    top = torch.where(torch.isfinite(top), top, 0.0)
    p_own, p = x_own.sub_(top).exp_(), x.sub_(of_groups(top)).exp_()
    total = p_own.sum(dim=-1, keepdim=True) + of_sequences(p.sum(dim=-1, keepdim=True))
    o = torch.matmul(p_own, _gathered(s, "v", s["pages"])) + of_sequences(torch.matmul(p, v))
    o = o / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + total.clamp_min(1e-38).log(), -math.inf)
    return {"o": _to_tokens(s, o, real).half(), "lse": _to_tokens(s, lse, real)[..., 0]}


def _plain_weights(s):
    x, real = _scores(s)
    b, m, h = s["lens"].shape[0], s["q_len"], s["q_heads"]
    t = torch.arange(m, device=x.device)
    row = (s["start"][:-1].long()[:, None] + t[None]).clamp_max(s["q"].shape[0] - 1)
    lse = _by_kv_head(s, s["lse"][row][..., None])
    w = x.sub_(torch.where(torch.isfinite(lse), lse, 0.0)).exp_().sum(dim=2)[..., :s["ctx"]]
    return {"sums": s["before"] + (w if s["per_head"] else w.sum(dim=1, keepdim=True))}


def _plain_evict(s):
    page, keep = s["page"], min(s["keep"], s["ctx"])
    ln = s["lens"].long()[:, None, None]
    b, heads, ctx = s["sums"].shape
    j = torch.arange(ctx, device=ln.device).expand(b, heads, ctx)
    # always kept first, then by their sums, then what is not there; a stable sort leaves ties in order
    always = (j < s["first"]) | (j >= ln - s["recent"])
    rank = torch.where(j >= ln, -math.inf, torch.where(always, math.inf, s["sums"].clamp(-3e38, 3e38)))
    best = rank.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    left = ln.clamp_max(keep)
    i = torch.arange(keep, device=ln.device)
    kept = torch.where(i < left, best, ctx).sort(dim=-1).values
    there = i < left
    kept = torch.where(there, kept, 0)
    # rows of every kv head, from their old pages to the new ones
    src = kept.expand(b, s["kv_heads"], keep)
    page_of = s["pages"].long().gather(1, (src // page).flatten(1)).view_as(src)
    to_page = s["to"].long()[:, None, i // page].expand_as(src)
    head = torch.arange(s["kv_heads"], device=ln.device)[None, :, None]
    some = there.expand_as(src)
    for x in ("k", "v", "k_par", "v_par"):
        if s[x] is not None:
            rows = s[x][page_of, head, src % page]
            to = (to_page, head, (i % page).expand_as(src))
            s[x][to] = torch.where(some.reshape(some.shape + (1,) * (rows.dim() - 3)), rows, s[x][to])
    sums = torch.zeros_like(s["sums"])
    sums[..., :keep] = torch.where(there, s["sums"].gather(2, kept), 0.0)
    got = {"lens": left.flatten().int(), "sums": sums, "kept": torch.where(there, kept, -1).int()}
    if s["bits"] == 16:
        return got | {"k": s["k"][:s["new_pages"]], "v": s["v"][:s["new_pages"]]}
    return got | _read(s, s["slots"])


# ------------------------------------------------------------------------------------ work

def _token_bytes(case):
    """Bytes of one token of one head in the cache."""
    d, b = case["dim"], case["bits"]
    return 2 * d if b == 16 else d * b // 8 + 4 * (d // GROUP)


def work(case):
    op = case["op"]
    if op in ("rope", "append"):
        axes, rot = len(_shares(case)), 2 * sum(_shares(case))
    if op == "rope":
        size = 2 if case["dtype"] == "f16" else 4
        n, h, d = case["tokens"], case["heads"], case["dim"]
        passes = 2 if case["grad"] else 1
        return {"bytes": passes * 2 * size * n * h * d + n * (4 * axes + 4 * rot), "flops": passes * 3 * n * h * rot}
    kv, d, tok = case["kv_heads"], case["dim"], _token_bytes(case)
    if op == "append":
        n, h = case["tokens"], case["q_heads"]
        # rows read, queries written, codes written and read again, fp16 values written
        return {"bytes": n * (4 + 4 * axes + 4 * rot + 2 * d * (2 * h + 2 * kv) + 2 * kv * (2 * tok + 2 * d)),
                "flops": n * (3 * (h + kv) * rot + 12 * kv * d)}
    if op == "shared":
        plens, sizes = _prefixes(case)
        lens, new = _own_lens(case)
        at, h = _starts(sizes), case["q_heads"]
        nbytes = 2 * kv * tok * (sum(plens) + sum(lens)) + sum(new) * h * (4 * d + 4)
        pairs = sum(p * sum(new[a:b]) for p, a, b in zip(plens, at, at[1:]))
        pairs += sum(max(0, ln - m + t + 1) for ln, m in zip(lens, new) for t in range(m))
        return {"bytes": nbytes, "flops": 4 * d * h * pairs}
    heads = kv if case["per_head"] else 1
    if op == "weights":
        nbytes = flops = 0
        w = case["window"]
        for ln, m in zip(*_lens(case["batch"], case["q_len"], case["ctx"], case["ragged"])):
            first = [max(0, ln - m + t + 1 - w) if w else 0 for t in range(m)]
            pairs = sum(max(0, ln - m + t + 1 - first[t]) for t in range(m))
            # keys that some row sees, queries, logarithms, earlier sums of the sequence; sums written
            nbytes += max(0, ln - first[0]) * kv * tok + m * case["q_heads"] * (2 * d + 4) + 4 * heads * (ln + case["ctx"])
            flops += 2 * d * case["q_heads"] * pairs
        return {"bytes": nbytes, "flops": flops}
    lens, _ = _lens(case["batch"], 1, case["ctx"], case["ragged"])
    keep = min(case["keep"], case["ctx"])
    left = sum(min(ln, keep) for ln in lens)
    # sums read and written, indices written, tokens read and written (and read back as fp16 where they are codes)
    nbytes = 4 * heads * (sum(lens) + case["batch"] * (case["ctx"] + keep)) + 4 * kv * left * tok
    nbytes += 0 if case["bits"] == 16 else case["batch"] * keep * (4 + 2 * kv * (tok + 2 * d))
    return {"bytes": nbytes, "flops": 0}


# ------------------------------------------------------------------------------------ 64 bits

def _turn64(x, s, case, back=False):
    """The rotation from its definition: pair i of the first channels is a complex number."""
    pos = torch.stack([s["pos"][a] for a in _axis_of(case)], dim=1).double()
    a = (pos * _freqs(case))[:, None]
    w = torch.polar(torch.ones_like(a), -a if back else a)
    y, r = x.double().clone(), 2 * a.shape[-1]
    if case["inter"]:
        z = torch.complex(y[..., 0:r:2], y[..., 1:r:2]) * w
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    else:
        z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * w
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    return y


def _through_cache64(x, case):
    """Values as a cache of this many bits gives them back."""
    if case["bits"] == 16:
        return x
    top = 2 ** case["bits"] - 1
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    lo = g.min(dim=-1, keepdim=True).values.half().double()
    st = ((g.max(dim=-1, keepdim=True).values - lo) / top).half().double()
    level = torch.round((g - lo) / st.clamp_min(1e-30)).clamp(0, top)
    return (lo + level * st * (st > 0)).reshape(x.shape)


def _stored64(s, x, page, head, off):
    """The numbers that tokens of the cache stand for, code by code."""
    c = s[x][page, head, off]
    if s["bits"] == 16:
        return c.double()
    ch = torch.arange(s["dim"], device=c.device)
    if s["bits"] == 4:
        # byte of the word and nibble of the byte that hold a channel
        bit = 4 * (ch % 8 // 2) + 16 * (ch % 2)
        c = (c[..., 4 * (ch // 8) + bit // 8] >> (bit % 8).to(torch.uint8)) & 15
    par = s[x + "_par"][page, head, off].double()
    return par[..., ch // GROUP, 0] + c.double() * par[..., ch // GROUP, 1]


def _tokens64(s, x, pages, n, head):
    """The first n tokens of a row of pages under one head."""
    j = torch.arange(n, device=pages.device)
    return _stored64(s, x, pages.long()[j // s["page"]], head, j % s["page"]).half().double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        out = {"y": _turn64(s["x"], s, case)}
        if case["grad"]:
            out["dx"] = _turn64(s["g"], s, case, back=True)
        return out
    if case["op"] == "append":
        return {"q": _turn64(s["q"], s, case), "k": _through_cache64(_turn64(s["kn"], s, case), case),
                "v": _through_cache64(s["vn"].double(), case)}
    kv, dim = case["kv_heads"], case["dim"]
    if case["op"] == "evict":
        return _exact_evict(s, case)
    g = case["q_heads"] // kv
    if case["op"] == "weights":
        sums = s["before"].double()
        at = 0
        for i, (ln, m) in enumerate(zip(*_lens(case["batch"], case["q_len"], case["ctx"], case["ragged"]))):
            j = torch.arange(ln, device=DEVICE)[None]
            p = ln - m + torch.arange(m, device=DEVICE)[:, None]
            sees = (j <= p) & ((j > p - case["window"]) if case["window"] else True)
            for h in range(kv) if ln else ():
                k = _tokens64(s, "k", s["pages"][i], ln, h).t().contiguous()
                for hq in range(h * g, h * g + g):
                    x = s["q"][at:at + m, hq].double() @ k / math.sqrt(dim) - s["lse"][at:at + m, hq].double()[:, None]
                    sums[i, h if case["per_head"] else 0, :ln] += torch.where(sees, x.exp(), 0.0).sum(dim=0)
            at += m
        return {"sums": sums}
    # attention, one sequence and one key-value head at a time: the prefix's tokens, then its own
    plens, sizes = _prefixes(case)
    lens, new = _own_lens(case)
    group = [i for i, n in enumerate(sizes) for _ in range(n)]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
    for h in range(kv):
        old = None, None, None
        at = 0
        for i, (ln, m) in enumerate(zip(lens, new)):
            if old[0] != group[i]:
                old = (group[i], *(_tokens64(s, x, s["prefix_pages"][group[i]], plens[group[i]], h) for x in "kv"))
            k, v = (torch.cat([old[1 + e], _tokens64(s, x, s["pages"][i], ln, h)]) for e, x in enumerate("kv"))
            j = torch.arange(k.shape[0], device=DEVICE)[None] - plens[group[i]]
            sees = (j <= ln - m + torch.arange(m, device=DEVICE)[:, None]) | (j < 0)
            x = s["q"][at:at + m, h * g:h * g + g].double().flatten(0, 1) @ k.t().contiguous() / math.sqrt(dim)
            x = torch.where(sees.repeat_interleave(g, dim=0), x, -math.inf)
            lse[at:at + m, h * g:h * g + g] = torch.logsumexp(x, dim=1).view(m, g)
            o[at:at + m, h * g:h * g + g] = (torch.softmax(x, dim=1) @ v).view(m, g, dim)
            at += m
    return {"o": o, "lse": lse}


def _exact_evict(s, case):
    """Choices made one sequence and head at a time on the host, values taken code by code."""
    page, keep, kv = case["page"], min(case["keep"], case["ctx"]), case["kv_heads"]
    sums, lens = s["sums"].cpu(), s["lens"].tolist()
    b, heads, ctx = sums.shape
    new_sums = torch.zeros((b, heads, ctx), dtype=torch.float64)
    kept = torch.full((b, heads, keep), -1, dtype=torch.int32)
    for i, n in enumerate(lens):
        last = max(0, n - case["recent"])
        for h in range(heads):
            if n <= keep:
                chosen = torch.arange(n)
            else:
                middle = torch.arange(case["first"], last)
                by = torch.argsort(-sums[i, h, middle].double(), stable=True)[:keep - case["first"] - (n - last)]
                chosen = torch.cat([torch.arange(case["first"]), middle[by].sort().values, torch.arange(last, n)])
            kept[i, h, :len(chosen)] = chosen.int()
            new_sums[i, h, :len(chosen)] = sums[i, h, chosen].double()
    dev = s["lens"].device
    out = {"lens": None, "sums": new_sums.to(dev), "kept": None}
    at = kept.to(dev).long().expand(b, kv, keep)
    there = at >= 0
    at = at.clamp_min(0)
    got = []
    for x in "kv":
        old = _stored64(s, x, s["pages"].long().gather(1, (at // page).flatten(1)).view_as(at), torch.arange(kv, device=dev)[None, :, None], at % page)
        got.append(torch.where(there[..., None], old, 0.0))
    if case["bits"] < 16:                         # as they are read back: [tokens][kv heads][channels]
        return out | {x: y.transpose(1, 2).flatten(0, 1) for x, y in zip("kv", got)}
    for x, y in zip("kv", got):
        pages = torch.zeros(s[x][:s["new_pages"]].shape, dtype=torch.float64, device=dev)
        cols = s["to"].shape[1]
        y = torch.cat([y, torch.zeros((b, kv, cols * page - keep, y.shape[-1]), dtype=y.dtype, device=dev)], dim=2)
        pages[s["to"].long().flatten()] = y.unflatten(2, (cols, page)).transpose(1, 2).flatten(0, 1)
        out[x] = pages
    return out
