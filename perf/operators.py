"""Operators for a prompt that goes on in a low-bit cache, as cases to be timed and compared.

Every case is a plain dict.  `kind` says what one pass is:

  attend    a chunk of new tokens per sequence attends to the sequence's cache (quantized tokens, outlier pools,
            residual ring) and, causally, to itself (KVCache.attend, RaggedKVCache.attend); with `cross` there are
            no new tokens and every query sees the whole cache (an encoder's states, say).
  extend    a shared prefix: the sequence in slot 0 is forked into every other slot, and each of those takes up a chunk
            of its own (RaggedKVCache.fork, .extend, .advance_by); the quantized tokens come back as rows.
  fork      slots take over other slots' sequences, all layers (RaggedKVCache.fork).
  compact   the free pages of a pool are listed and the live ones moved to another pool (RaggedKVCache.free_pages,
            .compact_into).
  rotate    queries and Keys of a chunk rotated by positions with several axes (KVCache.rotate), or the rows of
            cosines and sines for a decode step (KVCache.rope_rows).

With `own` the calls are the framework's, without it the same results come from elementary torch operations.
Caches are drawn as such: random codes, with the steps and zeros of Keys ~ N(0,1) with four large channels per kv head
and Values ~ N(0,1), a few tokens per unit in the pools, some fp16 rows in the ring.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

HD = 128
DEV = "cuda"


def _case(name, kind, **kw):
    c = dict(kind=kind, layers=1, batch=1, q_heads=32, kv_heads=8, bits=2, group_k=32, group_v=32, residual=128,
             budget=8, aux=32)
    if name:
        c["name"] = name
    c.update(kw)
    return c


def listed():
    return [
        # a short question behind a document of a thousand tokens: what is left is the launch and its latencies
        _case("attend_question_b1_1k", "attend", tokens=9, history=1003, ragged=False),
        # few rows over a long cache: a call to a tool in the middle of a long conversation
        _case("attend_turn_b2_32k", "attend", batch=2, tokens=45, history=32768 + 77, ragged=False, budget=32),
        # a long prompt taken in chunks: the third chunk of 512 tokens and later, four sequences
        _case("attend_chunk_b4_8k", "attend", batch=4, tokens=512, history=8192 + 130, ragged=False),
        # continuous batching on a multi-head model, 4-bit pages of 128 tokens, every length different
        _case("attend_ragged_b16_4bit_paged", "attend", batch=16, tokens=700, history=6000, ragged=True, paged=True,
              kv_heads=32, bits=4, group_k=128, group_v=128, residual=32, budget=3),
        # the first prompt of a sequence: nothing cached, causal among itself
        _case("attend_prompt_b1_8k", "attend", tokens=8192, history=0, ragged=False),
        # four requests behind one system prompt, one layer: the smallest extension
        _case("extend_b4_short", "extend", batch=5, prefix=500, chunk=75),
        # sixteen requests with retrieved documents behind one system prompt
        _case("extend_b16_2k", "extend", batch=17, prefix=2083, chunk=2000, bits=4, group_k=64),
        # beams of a stack of 32 layers: a quarter of the slots takes over the others, pages shared
        _case("fork_beams_b32", "fork", layers=32, batch=32, history=1900),
        # a small pool of one layer: latency
        _case("compact_small", "compact", batch=4, history=900, spare=70),
        # the pool of a stack of 32 layers, half of it free
        _case("compact_stack_b32_4k", "compact", layers=32, batch=32, history=4096, spare=4000, bits=4),
        # one decode step of a batch: rows of cosines and sines for positions in time, height and width
        _case("rotate_rows_b128", "rotate", tokens=128, rows=True, axes=3),
        # queries and Keys of a long prompt with images, views of one projection's output
        _case("rotate_images_16k", "rotate", tokens=16411, rows=False, axes=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend"] * 5 + ["extend", "extend", "fork", "compact", "rotate", "rotate"])
    g = rng.choice([1, 2, 4, 8])
    kvh = rng.choice([1, 2, 4, 8, 8, 16])
    gk, gv = rng.choice([(32, 32), (64, 64), (128, 128), (32, 128), (64, 32)])
    c = _case(None, kind, q_heads=g * kvh, kv_heads=kvh, bits=rng.choice([2, 4]), group_k=gk, group_v=gv,
              residual=rng.choice([0, 32, 100, 128]), budget=rng.choice([0, 3, 8, 32]), aux=rng.choice([8, 32]))
    if kind == "attend":
        c.update(batch=_log(rng, 1, 24), tokens=_log(rng, 1, 2048), history=_log(rng, 1, 20000) - 1,
                 ragged=rng.random() < 0.5, paged=rng.random() < 0.5, cross=rng.random() < 0.2)
        while c["batch"] > 1 and work(c)["flops"] > 2e11:
            c["batch"] = (c["batch"] + 1) // 2
        if work(c)["flops"] > 5e11:
            c["tokens"] = 200
    elif kind == "extend":
        c.update(batch=1 + _log(rng, 1, 12), prefix=_log(rng, 1, 3500), chunk=_log(rng, 1, 1500))
    elif kind == "fork":
        c.update(layers=_log(rng, 1, 24), batch=_log(rng, 2, 32), history=_log(rng, 1, 4000))
    elif kind == "compact":
        c.update(layers=_log(rng, 1, 16), batch=_log(rng, 1, 24), history=_log(rng, 40, 4000), spare=_log(rng, 1, 2000))
    else:
        c.update(tokens=_log(rng, 1, 12000), rows=rng.random() < 0.4, axes=rng.choice([1, 2, 3]))
    return c


# ---- sizes ---------------------------------------------------------------------------------------------------------

def _split(c, n):
    """(quantized tokens, rows in the ring) of a sequence of n tokens."""
    G, R = c["group_k"], c["residual"]
    nq = G * ((n - R) // G) if n >= R + G else 0
    return nq, n - nq


def _res_rows(c):
    G = c["group_k"]
    return G * ((c["residual"] + 2 * G - 1) // G)


def _lengths(c):
    """(cached tokens, new tokens) of every sequence."""
    B, h, n = c["batch"], c["history"], c["tokens"]
    if not c.get("ragged"):
        return [h] * B, [n] * B
    rng = random.Random(B * 7919 + h * 31 + n)
    hist = [h] + [rng.randrange(h + 1) for _ in range(B - 1)]
    new = [n] + [_log(rng, 1, n) if rng.random() < 0.9 else 0 for _ in range(B - 1)]
    return hist, new


def _chunks(c):
    """New tokens of every slot of an `extend` case (slot 0 holds the prefix and gets none)."""
    rng = random.Random(c["batch"] * 977 + c["chunk"])
    return [0, c["chunk"]] + [rng.randint(1, c["chunk"]) for _ in range(c["batch"] - 2)]


def _token_bytes(c):
    """Codes, steps and zeros, mask bit of one quantized token of one unit, Keys and Values."""
    return 2 * HD * c["bits"] / 8 + 512 / c["group_k"] + 4 * (HD // c["group_v"]) + 1 / 8


def _parents(c):
    """(from, to) of a `fork` case: three quarters of the slots stay, the last ones take over."""
    rng = random.Random(c["batch"] * 131 + c["history"])
    B = c["batch"]
    first = max(1, B - max(1, B // 4))
    return [(rng.randrange(first), b) for b in range(first, B)]


def _fork_states(c):
    rng = random.Random(c["batch"] * 17 + c["history"])
    return [_split(c, rng.randint(1, c["history"])) for _ in range(c["batch"])]


def work(case):
    c = case
    H, g = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    slots = c["budget"] + c["aux"] // 2
    if c["kind"] == "attend":
        b = f = 0
        for h, n in zip(*_lengths(c)):
            if n == 0:
                continue
            nq, nr = _split(c, h)
            m = min(slots, nq)
            seen = n * h + (0 if c.get("cross") else n * (n + 1) // 2)
            f += 4 * HD * g * H * seen
            b += n * H * HD * 2 * (2 * g + (0 if c.get("cross") else 2))
            b += H * (nq * _token_bytes(c) + (nr + m) * 4 * HD)
        return {"bytes": int(b), "flops": int(f)}
    if c["kind"] == "extend":
        nq, nr = _split(c, c["prefix"])
        b = H * (nr + slots) * 4 * HD
        for n in _chunks(c)[1:]:
            groups = max(0, (nr + n - c["residual"]) // c["group_k"])
            done = groups * c["group_k"]
            b += H * (n * 4 * HD + (nr + n - done + slots) * 4 * HD + done * (_token_bytes(c) + 4 * HD))
        return {"bytes": int(b), "flops": int(b)}
    if c["kind"] == "fork":
        st = _fork_states(c)
        b = 0
        for src, _ in _parents(c):
            b += 2 * c["layers"] * H * (st[src][1] + slots) * 4 * HD
        return {"bytes": int(b), "flops": 0}
    if c["kind"] == "compact":
        b = 2 * c["layers"] * H * _live_pages(c) * c["group_k"] * _token_bytes(c)
        return {"bytes": int(b), "flops": 0}
    n = c["tokens"]
    if c["rows"]:
        return {"bytes": n * (HD * 4 + 4 * c["axes"]), "flops": n * 64 * 40}
    heads = c["q_heads"] + H
    return {"bytes": n * (heads * HD * 4 + 4 * c["axes"]), "flops": n * heads * HD * 3}


def _compact_lengths(c):
    rng = random.Random(c["batch"] * 19 + c["history"] + c["spare"])
    return [c["history"]] + [rng.randint(0, c["history"]) for _ in range(c["batch"] - 1)]


def _live_pages(c):
    return sum(_split(c, n)[0] // c["group_k"] for n in _compact_lengths(c))


# ---- the packed layout, as documented ---------------------------------------------------------------------------------

def _word_byte(bits, lane, f):
    return 16 * lane + 4 * (f >> 1) if bits == 2 else 1024 * (f >> 2) + 16 * lane + 4 * (f & 3)


def _code_bit(bits, f, x):
    v, e = x >> 1, x & 1
    return (16 * e + 2 * (v + 1) + 8 * (f & 1)) % 32 if bits == 2 else (16 * e + 2 + 4 * (v & 1) + 8 * (v >> 1)) % 32


_places = {}


def _place(bits, which):
    """Word and bit of the code of (token in its block, channel): int64 [32 * 128] each."""
    key = bits, which
    if key not in _places:
        word, bit = np.zeros((32, HD), np.int64), np.zeros((32, HD), np.int64)
        for t in range(32):
            for ch in range(HD):
                if which == "k":
                    lane, f, x = 16 * ((ch % 32) // 8) + t % 16, 4 * (t // 16) + ch // 32, ch % 8
                else:
                    lane, f, x = 16 * (t // 8) + ch % 16, ch // 16, t % 8
                word[t, ch], bit[t, ch] = _word_byte(bits, lane, f) // 4, _code_bit(bits, f, x)
        _places[key] = tuple(torch.from_numpy(a.reshape(-1)).to(DEV) for a in (word, bit))
    return _places[key]


def _codes(words, bits, which):
    """int32 [..., blocks, 128 * bits] -> integer codes float32 [..., blocks * 32, 128]."""
    word, bit = _place(bits, which)
    w = words[..., word].long() & 0xFFFFFFFF
    code = ((w >> bit) | (w << (32 - bit))) & ((1 << bits) - 1)
    return code.float().view(*words.shape[:-2], words.shape[-2] * 32, HD)


def _dequantized(c, k_words, k_meta, v_words, v_meta):
    """Quantized tokens of [..., groups] as fp32 rows: zero + code * step.  k_words, v_words int32 [..., blocks, words];
    k_meta fp16 [..., groups, 2, 128]; v_meta fp16 [..., blocks, 2, 16, NV, 2]."""
    bits, G = c["bits"], c["group_k"]
    k = _codes(k_words, bits, "k")
    km = k_meta.float()
    k = k.view(*km.shape[:-2], G, HD) * km[..., 0, :].unsqueeze(-2) + km[..., 1, :].unsqueeze(-2)
    k = k.flatten(-3, -2)
    v = _codes(v_words, bits, "v")
    vm = v_meta.float().movedim(-1, -2)                     # [..., blocks, 2, 16, 2, NV]
    vm = vm.flatten(-3, -2)                                 # [..., blocks, 2, 32, NV]
    nv = HD // c["group_v"]
    v = v.view(*vm.shape[:-3], 32, nv, c["group_v"]) * vm[..., 0, :, :, None] + vm[..., 1, :, :, None]
    return k, v.flatten(-2, -1).flatten(-3, -2)


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed * 1009 + 17)


def _half(gen, *shape, scale=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * scale).half()


def _raw(gen, n):
    return torch.randint(0, 256, (n,), generator=gen, device=DEV, dtype=torch.uint8)


def _meta(c, gen, units, groups):
    """Steps and zeros of `units` runs of `groups` groups."""
    top = 2 ** c["bits"] - 1
    nv, blocks = HD // c["group_v"], groups * c["group_k"] // 32

    def pair(*shape):
        step = (3.2 + 1.6 * torch.rand(*shape, generator=gen, device=DEV)) / top
        zero = -1.6 - 0.8 * torch.rand(*shape, generator=gen, device=DEV)
        return step, zero
    ks, kz = pair(units, groups, HD)
    big = torch.ones(units, 1, HD, device=DEV)
    big[:, :, [5, 40, 77, 126]] = 6.0
    k_meta = torch.stack([ks * big, kz * big], 2).half()
    vs, vz = pair(units, blocks, 16, nv, 2)
    return k_meta, torch.stack([vs, vz], 2).half()


def _state(c, lengths, groups, seed, n_pages=None, spare_pages=0):
    """A cache of len(lengths) sequences with room for `groups` groups each, every layer: its arrays as tensors.
    With pages they are dealt at random, and `spare_pages` more are free."""
    gen = _gen(seed)
    B, H, Ly, G = len(lengths), c["kv_heads"], c["layers"], c["group_k"]
    nv, slots, rows = HD // c["group_v"], c["budget"] + c["aux"], _res_rows(c)
    s = {"batch": B, "groups": groups}
    rng = random.Random(seed * 3 + 1)
    split = [_split(c, n) for n in lengths]
    starts = [G * rng.randrange(rows // G) for _ in lengths]
    s["split"], s["starts_in_ring"] = split, starts
    s["seq_state"] = torch.tensor([[nq, st, nr, 1] for (nq, nr), st in zip(split, starts)], dtype=torch.int32, device=DEV)
    if c.get("paged"):
        n_pages = B * groups + spare_pages
        deal = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed + 5))[:B * groups]
        s["table"] = deal.view(B, groups).to(torch.int32).to(DEV)
        s["n_pages"] = n_pages
        units, per = Ly * H, n_pages
    else:
        units, per = Ly * B * H, groups
    blocks = per * G // 32
    s["k_codes"], s["v_codes"] = _raw(gen, units * blocks * 512 * c["bits"]), _raw(gen, units * blocks * 512 * c["bits"])
    s["k_meta"], s["v_meta"] = _meta(c, gen, units, per)
    # outlier tokens of every unit: `filled` of them, ascending, in the pool and then in the auxiliary pool
    s["pool_k"], s["pool_v"] = _half(gen, Ly * B * H, slots, HD, scale=0.05), _half(gen, Ly * B * H, slots, HD)
    s["pool_idx"] = torch.zeros(Ly * B * H, slots, dtype=torch.int32, device=DEV)
    s["pool_score"] = s["pool_k"].double().abs().sum(-1)
    counts = []
    mask = torch.zeros(Ly, B, H, groups * G // 32, 32, dtype=torch.int64, device=DEV)
    for b, (nq, _) in enumerate(split):
        inside = min(c["budget"], nq)
        behind = min(c["aux"] // 2, nq - inside) if c["budget"] else 0
        counts.append((inside, behind))
        if inside + behind == 0:
            continue
        pick = torch.rand(Ly * H, nq, generator=gen, device=DEV).topk(inside + behind, 1).indices.sort(1).values
        pick = pick[:, torch.randperm(inside + behind, generator=torch.Generator().manual_seed(seed + b))]
        own_idx = s["pool_idx"].view(Ly, B, H, slots)[:, b]
        own_idx[..., :inside] = pick.view(Ly, H, -1)[..., :inside].int()
        own_idx[..., c["budget"]:c["budget"] + behind] = pick.view(Ly, H, -1)[..., inside:].int()
        flat = torch.zeros(Ly * H, groups * G, dtype=torch.int64, device=DEV).scatter_(1, pick, 1)
        mask[:, b] = flat.view(Ly, H, -1, 32)
    words = (mask << torch.arange(32, device=DEV)).sum(-1)
    words = torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()           # [layers, batch, heads, blocks]
    if c.get("paged"):
        pool = torch.zeros(Ly, H, s["n_pages"], G // 32, dtype=torch.int32, device=DEV)
        pool[:, :, s["table"].long()] = words.permute(0, 2, 1, 3).reshape(Ly, H, B, groups, G // 32)
        words = pool
    s["mask"] = words.contiguous()
    s["counts"] = counts
    per_unit = torch.tensor(counts, dtype=torch.int32, device=DEV).view(1, B, 1, 2).expand(Ly, B, H, 2).reshape(-1, 2)
    s["pool_count"], s["aux_count"] = per_unit[:, 0].contiguous(), per_unit[:, 1].contiguous()
    s["frozen"] = torch.zeros(Ly * B * H, dtype=torch.int32, device=DEV)
    s["k_res"], s["v_res"] = _half(gen, Ly * B * H, rows, HD), _half(gen, Ly * B * H, rows, HD)
    return s


_ARRAYS = ("k_codes", "k_meta", "v_codes", "v_meta", "mask", "pool_k", "pool_v", "pool_idx", "pool_score", "pool_count",
           "aux_count", "frozen", "k_res", "v_res")


def _own_cache(c, s, ragged):
    """The framework's cache with the contents of `s`."""
    from paper_2505_10938_amd import cache as KC
    cfg = KC.make_config(c["layers"], s["batch"], c["q_heads"], c["kv_heads"], s["groups"] * c["group_k"], c["bits"],
                         c["group_k"], c["group_v"], c["residual"], c["budget"], c["aux"])
    kv = (KC.RaggedKVCache if ragged else KC.KVCache)(cfg, n_pages=s.get("n_pages"))
    for name in _ARRAYS:
        src = s[name].contiguous().view(-1).view(torch.uint8)
        getattr(kv, name)[:src.numel()].copy_(src)
    if "table" in s:
        kv.page_table.copy_(s["table"])
    if ragged:
        kv.seq_state.copy_(s["seq_state"])
        kv.longest = max(nq + nr for nq, nr in s["split"])
    else:
        kv.n_quant, kv.n_res = [s["split"][0][0]] * c["layers"], [s["split"][0][1]] * c["layers"]
        kv.res_start = [s["starts_in_ring"][0]] * c["layers"]
    return kv


def _attend_inputs(c, seed):
    hist, new = _lengths(c)
    G = c["group_k"]
    groups = max(1, max(_split(c, h)[0] for h in hist) // G)
    s = _state(c, hist, groups, seed)
    if not c.get("ragged"):                                 # a batch of one length: one place in the ring
        s["starts_in_ring"] = [s["starts_in_ring"][0]] * c["batch"]
        s["seq_state"][:, 1] = s["starts_in_ring"][0]
    gen = _gen(seed + 100003)
    total, H, Hq = sum(new), c["kv_heads"], c["q_heads"]
    # one projection's output holds queries, Keys and Values of a token
    s["qkv"] = _half(gen, total, Hq + 2 * H, HD)
    s["new"] = new
    s["starts"] = torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device=DEV)
    return s


def _extend_inputs(c, seed):
    c = dict(c, paged=True)
    nq, nr = _split(c, c["prefix"])
    new, G = _chunks(c), c["group_k"]
    more = max(0, (nr + max(new) - c["residual"]) // G)
    lengths = [c["prefix"]] + [0] * (c["batch"] - 1)
    s = _state(c, lengths, nq // G + max(1, more), seed)
    # what nobody has written is zero
    live = s["table"][0, :nq // G].long()
    for name in ("k_codes", "v_codes", "k_meta", "v_meta"):
        t = s[name].view(torch.uint8).view(c["layers"], c["kv_heads"], s["n_pages"], -1)
        kept = t[:, :, live].clone()
        t.zero_()
        t[:, :, live] = kept
    gen = _gen(seed + 200003)
    H = c["kv_heads"]
    k, v = _half(gen, sum(new), H, HD), _half(gen, sum(new), H, HD)
    k[:, :, [3, 17, 64, 101]] *= 20.0
    small = torch.rand(sum(new), H, 1, generator=gen, device=DEV) < 0.02
    k = torch.where(small, k * 0.05, k)
    s["chunk_k"], s["chunk_v"], s["new"] = k, v, new
    s["starts"] = torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device=DEV)
    s["pairs"] = torch.tensor([[0, b] for b in range(1, c["batch"])], dtype=torch.int32, device=DEV)
    s["first"], s["more"] = nq, more
    return s


def _fork_inputs(c, seed):
    c = dict(c, paged=True)
    states = _fork_states(c)
    s = _state(c, [nq + nr for nq, nr in states], max(1, max(nq for nq, _ in states) // c["group_k"]), seed)
    s["pairs"] = torch.tensor(_parents(c), dtype=torch.int32, device=DEV)
    return s


def _compact_inputs(c, seed):
    c = dict(c, paged=True)
    lengths = _compact_lengths(c)
    groups = max(1, max(_split(c, n)[0] for n in lengths) // c["group_k"])
    return _state(c, lengths, groups, seed, spare_pages=c["spare"])


def _rotate_inputs(c, seed):
    gen = _gen(seed)
    n, axes = c["tokens"], c["axes"]
    s = {}
    i = np.arange(HD // 2)
    s["freq"] = torch.from_numpy((10000.0 ** (-2.0 * i / HD)).astype(np.float32)).to(DEV)
    s["pair_axis"] = [0 if p < 16 or axes == 1 else 1 if p < 40 or axes == 2 else 2 for p in range(HD // 2)]
    far = torch.randint(0, 100000, (1,), generator=gen, device=DEV)
    s["positions"] = (far + torch.randint(0, 4 * n + 2, (axes, n), generator=gen, device=DEV)).to(torch.int32)
    if not c["rows"]:
        s["qkv"] = _half(gen, n, c["q_heads"] + 2 * c["kv_heads"], HD)
    return s


_INPUTS = {"attend": _attend_inputs, "extend": _extend_inputs, "fork": _fork_inputs, "compact": _compact_inputs,
           "rotate": _rotate_inputs}


def prepare(case, seed):
    c = dict(case)
    s = _INPUTS[c["kind"]](c, seed)
    s["case"] = c
    if not own:
        return s
    if c["kind"] == "attend":
        s["kv"] = _own_cache(c, s, bool(c.get("ragged")))
        for name in _ARRAYS:
            del s[name]
    elif c["kind"] in ("extend", "fork"):
        s["kv"] = _own_cache(c, s, True)
        for name in _ARRAYS:
            del s[name]
    elif c["kind"] == "compact":
        from paper_2505_10938_amd import cache as KC
        s["kv"] = _own_cache(c, s, True)
        s["to"] = KC.PagePool(s["kv"].cfg, _live_pages(c) + 3)
        for name in _ARRAYS:
            del s[name]
    else:
        from paper_2505_10938_amd import cache as KC
        s["kv"] = KC.KVCache(KC.make_config(1, 1, c["q_heads"], c["kv_heads"], 32))
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(state):
    return (_RUN_OWN if own else _RUN)[state["case"]["kind"]](state)


def _views(s):
    c = s["case"]
    Hq, H = c["q_heads"], c["kv_heads"]
    return s["qkv"][:, :Hq], s["qkv"][:, Hq:Hq + H], s["qkv"][:, Hq + H:]


def _own_attend(s):
    c = s["case"]
    q, k, v = _views(s)
    if c.get("cross"):
        k = v = None
    if c.get("ragged"):
        return s["kv"].attend(0, q, s["starts"], max(s["new"]), k, v)
    def batched(t):
        return None if t is None else t.unflatten(0, (c["batch"], c["tokens"]))
    return s["kv"].attend(0, batched(q), batched(k), batched(v)).flatten(0, 1)


def _sequence(c, s, b, units):
    """Codes, steps, zeros and mask words of sequence b, kv heads `units`, of a one-layer cache: [heads, groups ...]."""
    G, H = c["group_k"], c["kv_heads"]
    groups = s["split"][b][0] // G
    out = []
    for name, per in (("k_codes", G // 32), ("k_meta", 1), ("v_codes", G // 32), ("v_meta", G // 32), ("mask", G // 32)):
        t = s[name].contiguous().view(-1).view(torch.uint8)
        if "table" in s:
            t = t.view(H, s["n_pages"], -1)[units][:, s["table"][b, :groups].long()]
        else:
            t = t.view(c["batch"], H, s["groups"], -1)[b, units][:, :groups]
        t = t.contiguous()
        if name == "k_meta":
            out.append(t.view(torch.float16).view(-1, groups, 2, HD))
        elif name == "v_meta":
            out.append(t.view(torch.float16).view(-1, groups * per, 2, 16, HD // c["group_v"], 2))
        else:
            out.append(t.view(torch.int32).view(t.shape[0], groups * per, -1))
    return out


def _live(c, s, b, units, dequantize, dtype):
    """Rows a sequence's queries see in its cache, kv heads `units`, and which of them count: K, V [heads, rows, 128]."""
    H = c["kv_heads"]
    nq, nr = s["split"][b]
    at = torch.arange(H, device=DEV)[units] + b * H
    parts_k, parts_v, ok = [], [], []
    if nq:
        kc, km, vc, vm, mk = _sequence(c, s, b, units)
        k, v = dequantize(c, kc, km, vc, vm)
        parts_k.append(k.to(dtype))
        parts_v.append(v.to(dtype))
        bits = (mk.long().view(mk.shape[0], -1, 1) >> torch.arange(32, device=DEV)) & 1
        ok.append(bits.flatten(1) == 0)
        inside, behind = s["counts"][b]
        for first, count in ((0, inside), (c["budget"], behind)):
            parts_k.append(s["pool_k"][at, first:first + count].to(dtype))
            parts_v.append(s["pool_v"][at, first:first + count].to(dtype))
            ok.append(torch.ones(len(at), count, dtype=torch.bool, device=DEV))
    row = (torch.arange(nr, device=DEV) + s["starts_in_ring"][b]) % _res_rows(c)
    parts_k.append(s["k_res"][at][:, row].to(dtype))
    parts_v.append(s["v_res"][at][:, row].to(dtype))
    ok.append(torch.ones(len(at), nr, dtype=torch.bool, device=DEV))
    return torch.cat(parts_k, 1), torch.cat(parts_v, 1), torch.cat(ok, 1)


def _plain_attend(s):
    c = s["case"]
    q, k, v = _views(s)
    H, g = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    out = torch.empty(q.shape[0], c["q_heads"], HD, dtype=torch.float16, device=DEV)
    at = 0
    for b, n in enumerate(s["new"]):
        if n == 0:
            continue
        seen = sum(s["split"][b]) + (0 if c.get("cross") else n)
        step = max(1, min(H, 2 ** 28 // max(1, n * g * max(1, seen))))
        for h0 in range(0, H, step):
            heads = slice(h0, min(H, h0 + step))
            K, V, ok = _live(c, s, b, heads, _dequantized, torch.float32)
            hs = K.shape[0]
            ok = ok[:, None].expand(hs, n, -1)
            if not c.get("cross"):
                K = torch.cat([K, k[at:at + n, heads].float().transpose(0, 1)], 1)
                V = torch.cat([V, v[at:at + n, heads].float().transpose(0, 1)], 1)
                i = torch.arange(n, device=DEV)
                ok = torch.cat([ok, (i[None, :] <= i[:, None]).expand(hs, n, n)], 2)
            qs = q[at:at + n].float().view(n, H, g, HD)[:, heads].permute(1, 0, 2, 3).reshape(hs, n * g, HD)
            if K.shape[1] == 0:
                o = torch.zeros_like(qs)
            else:
                x = torch.matmul(qs, K.transpose(1, 2).contiguous()).view(hs, n, g, -1) * HD ** -0.5
                x.masked_fill_(~ok[:, :, None], -math.inf)
                x -= x.amax(-1, keepdim=True).clamp_min(-1e30)
                x.exp_()
                x /= x.sum(-1, keepdim=True).clamp_min(1e-37)
                o = torch.matmul(x.view(hs, n * g, -1), V)
            out[at:at + n].view(n, H, g, HD)[:, heads] = o.view(hs, n, g, HD).permute(1, 0, 2, 3).half()
        at += n
    return out


def _tensors(s, kv=None):
    """What an extension or a fork leaves, as a dict of the whole arrays."""
    c = s["case"]
    units, slots, rows = c["layers"] * s["batch"] * c["kv_heads"], c["budget"] + c["aux"], _res_rows(c)
    def of(name, dtype, *shape):
        t = getattr(kv, name) if kv is not None else s["now"][name]
        return t.contiguous().view(-1).view(torch.uint8)[:units * math.prod(shape) * dtype.itemsize].view(dtype).view(units, *shape)
    out = {"pool_k": of("pool_k", torch.float16, slots, HD), "pool_v": of("pool_v", torch.float16, slots, HD),
           "pool_idx": of("pool_idx", torch.int32, slots), "pool_score": of("pool_score", torch.float64, slots),
           "pool_count": of("pool_count", torch.int32), "aux_count": of("aux_count", torch.int32),
           "frozen": of("frozen", torch.int32), "k_res": of("k_res", torch.float16, rows, HD),
           "v_res": of("v_res", torch.float16, rows, HD)}
    out["seq_state"] = kv.seq_state if kv is not None else s["now"]["seq_state"]
    out["page_table"] = kv.page_table if kv is not None else s["now"]["table"]
    return out


def _own_extend(s):
    from paper_2505_10938_amd import binding as B
    c, kv = s["case"], s["kv"]
    kv.fork(s["pairs"])
    kv.extend(0, s["chunk_k"], s["chunk_v"], s["starts"], max(s["new"]))
    kv.advance_by(s["starts"], max(s["new"]))
    kv.longest = c["prefix"] + max(s["new"])                # (the same passes again: nobody got longer)
    out = _tensors(s, kv)
    n = s["more"] * c["group_k"]
    if n:
        rows = torch.empty(2, s["batch"], c["kv_heads"], n, HD, dtype=torch.float16, device=DEV)
        B.kvq_dequantize(kv.cfg, 0, kv.qcache, s["first"] + n, kv.pool, s["first"], n, rows[0], rows[1], n * HD)
        out["k_rows"], out["v_rows"] = rows[0], rows[1]
    return out


def _fork_arrays(s):
    """The plain fork: live ring rows, occupied slots, counts, state and table entries of whole groups."""
    c, now = s["case"], {}
    B, H, Ly = s["batch"], c["kv_heads"], c["layers"]
    for name in ("pool_k", "pool_v", "pool_idx", "pool_score", "pool_count", "aux_count", "frozen", "k_res", "v_res",
                 "seq_state", "table"):
        now[name] = s[name].clone()
    src, dst = s["pairs"][:, 0].long(), s["pairs"][:, 1].long()
    state = s["seq_state"][src]
    def units(name):
        return s[name].view(Ly, B, H, *s[name].shape[1:]), now[name].view(Ly, B, H, *s[name].shape[1:])
    rows = _res_rows(c)
    live = (torch.arange(rows, device=DEV)[None] - state[:, 1:2]) % rows < state[:, 2:3]
    for name in ("k_res", "v_res"):
        old, new = units(name)
        new[:, dst] = torch.where(live[None, :, None, :, None], old[:, src], old[:, dst])
    slot = torch.arange(c["budget"] + c["aux"], device=DEV)
    n_in, n_aux = (units(name)[0][:, src][..., None] for name in ("pool_count", "aux_count"))
    held = (slot < n_in) | ((slot >= c["budget"]) & (slot - c["budget"] < n_aux))
    for name in ("pool_k", "pool_v", "pool_idx", "pool_score"):
        old, new = units(name)
        keep = held[..., None] if name in ("pool_k", "pool_v") else held
        new[:, dst] = torch.where(keep, old[:, src], old[:, dst])
    for name in ("pool_count", "aux_count", "frozen"):
        old, new = units(name)
        new[:, dst] = old[:, src]
    now["seq_state"][dst] = state
    group = torch.arange(s["groups"], device=DEV)[None] * c["group_k"]
    now["table"][dst] = torch.where(group < state[:, :1], s["table"][src], s["table"][dst])
    s["now"] = now
    return now


def _plain_fork(s):
    _fork_arrays(s)
    return _tensors(s)


def _own_fork(s):
    s["kv"].fork(s["pairs"])
    return _tensors(s, s["kv"])


def _quantize(x, dim, bits):
    """Codes (fp32), step and zero (fp16) of x (fp16) along `dim`."""
    x = x.float()
    low, high = x.amin(dim, keepdim=True) + 0.0, x.amax(dim, keepdim=True)
    third = torch.tensor(1.0 / (2 ** bits - 1), dtype=torch.float32, device=DEV)
    step = ((high - low) * third).half()
    t = x - low
    code = torch.zeros_like(t)
    for k in range(2 ** bits - 1):
        code += t >= (k + 0.5) * step.float()
    return torch.where(step == 0, torch.zeros_like(code), code), step, low.half()


def _compete(c, pool, first, rows_k, rows_v):
    """One group's competition, all units at once; `pool` is updated, the selected flags come back."""
    N, A, S = c["budget"], c["aux"], c["budget"] + c["aux"]
    U, G = rows_k.shape[:2]
    if N == 0:
        return torch.zeros(U, G, dtype=torch.bool, device=DEV)
    slot, token = torch.arange(N, device=DEV), torch.arange(G, device=DEV)
    n_old = pool["pool_count"][:, None].long()
    score = torch.cat([torch.where(slot < n_old, pool["pool_score"][:, :N], math.inf), rows_k.double().abs().sum(-1)], 1)
    index = torch.cat([torch.where(slot < n_old, pool["pool_idx"][:, :N].long(), 2 ** 40 + slot),
                       (first + token).expand(U, G)], 1)
    by_index = index.argsort(1)
    order = by_index.gather(1, score.gather(1, by_index).sort(dim=1, stable=True).indices)
    rank = torch.empty_like(order).scatter_(1, order, torch.arange(N + G, device=DEV).expand(U, -1))
    keep = torch.clamp(n_old + G, max=N)
    out = (rank[:, :N] >= keep) & (slot < n_old)
    new = rank[:, N:] < keep
    n_out, n_aux = out.sum(1, keepdim=True), pool["aux_count"][:, None].long()
    stop = (pool["frozen"][:, None] != 0) | (n_aux + n_out > A)
    out, new = out & ~stop, new & ~stop
    n_out = n_out * ~stop
    turn_out, turn_new = out.cumsum(1) - 1, new.cumsum(1) - 1
    freed = torch.where(out, slot, N).sort(1).values
    to_aux = torch.where(out, N + n_aux + turn_out, S)
    to_pool = torch.where(turn_new < n_out, freed.gather(1, turn_new.clamp(0, N - 1)), n_old - n_out + turn_new)
    to_pool = torch.where(new, to_pool, S)
    moved = {"pool_k": rows_k, "pool_v": rows_v, "pool_score": score[:, N:], "pool_idx": index[:, N:].int()}
    for name, fresh in moved.items():
        t = pool[name]
        wide = torch.cat([t, t[:, :1]], 1)                  # (a slot behind the last for what does not move)
        a, p = (to_aux[..., None], to_pool[..., None]) if t.dim() == 3 else (to_aux, to_pool)
        wide.scatter_(1, a.expand(-1, -1, *t.shape[2:]), t[:, :N])
        wide.scatter_(1, p.expand(-1, -1, *t.shape[2:]), fresh)
        t.copy_(wide[:, :S])
    pool["pool_count"].copy_(torch.where(stop, n_old, keep)[:, 0])
    pool["aux_count"].add_(n_out[:, 0].int())
    pool["frozen"].copy_(stop[:, 0])
    return new


def _plain_extend(s):
    c = s["case"]
    G, R, H, rows = c["group_k"], c["residual"], c["kv_heads"], _res_rows(c)
    now = _fork_arrays(s)
    (nq, nr), start = s["split"][0], s["starts_in_ring"][0]
    ring = (torch.arange(nr, device=DEV) + start) % rows
    n = s["more"] * G
    out = torch.zeros(2, s["batch"], H, n, HD, dtype=torch.float16, device=DEV)
    at = 0
    for b, new in enumerate(s["new"]):
        if new == 0:
            continue
        u = slice(b * H, (b + 1) * H)
        k = torch.cat([now["k_res"][u][:, ring], s["chunk_k"][at:at + new].transpose(0, 1)], 1)
        v = torch.cat([now["v_res"][u][:, ring], s["chunk_v"][at:at + new].transpose(0, 1)], 1)
        at += new
        groups = (nr + new - R) // G if nr + new >= R + G else 0
        pool = {name: now[name][u] for name in ("pool_k", "pool_v", "pool_idx", "pool_score", "pool_count", "aux_count",
                                                "frozen")}
        for j in range(groups):
            gk, gv = k[:, j * G:(j + 1) * G], v[:, j * G:(j + 1) * G]
            new_ones = _compete(c, pool, nq + j * G, gk, gv)[..., None]
            fk, fv = ((torch.where(new_ones, (x.double().sum(1, keepdim=True) / G).float().half(), x)) for x in (gk, gv))
            code, step, zero = _quantize(fk, 1, c["bits"])
            out[0, b, :, j * G:(j + 1) * G] = torch.where(new_ones, gk, (zero.float() + code * step.float()).half())
            code, step, zero = _quantize(fv.view(H, G, -1, c["group_v"]), 3, c["bits"])
            x = (zero.float() + code * step.float()).half().view(H, G, HD)
            out[1, b, :, j * G:(j + 1) * G] = torch.where(new_ones, gv, x)
        left = torch.arange(max(groups * G, nr), nr + new, device=DEV)
        now["k_res"][u][:, (left + start) % rows] = k[:, left]
        now["v_res"][u][:, (left + start) % rows] = v[:, left]
        now["seq_state"][b] = torch.tensor([nq + groups * G, (start + groups * G) % rows, nr + new - groups * G, 1],
                                           dtype=torch.int32)
    result = _tensors(s)
    if n:
        result["k_rows"], result["v_rows"] = out[0], out[1]
    return result


def _plain_compact(s):
    c = s["case"]
    G, pages = c["group_k"], s["n_pages"]
    live = torch.arange(s["groups"], device=DEV)[None] * G < s["seq_state"][:, :1]
    used = torch.zeros(pages + 1, dtype=torch.int64, device=DEV)
    used[torch.where(live, s["table"].long(), pages).view(-1)] = 1
    used = used[:pages]
    new = used.cumsum(0) - 1
    count = _live_pages(c)
    to = count + 3
    gone = torch.arange(pages, device=DEV) - used.cumsum(0)
    free = torch.full((pages + 1,), -1, dtype=torch.int32, device=DEV)
    free.scatter_(0, torch.where(used == 0, gone, pages), torch.arange(pages, device=DEV, dtype=torch.int32))
    out = {"free": free[:pages], "counts": torch.stack([pages - used.sum(), used.sum()]).int(),
           "table": torch.where(live, new[s["table"].long()], -1).int()}
    source = torch.empty(count, dtype=torch.int64, device=DEV)
    source = torch.cat([source, source[:1] if count else source.new_zeros(1)])
    source.scatter_(0, torch.where(used == 1, new, count), torch.arange(pages, device=DEV))
    for name in ("k_codes", "k_meta", "v_codes", "v_meta", "mask"):
        t = s[name].view(-1).view(torch.uint8).view(c["layers"] * c["kv_heads"], pages, -1)
        moved = torch.zeros(t.shape[0], to, t.shape[2], dtype=torch.uint8, device=DEV)
        moved[:, :count] = t[:, source[:count]]
        out[name] = moved.view(torch.int32)
    return out


def _own_compact(s):
    c, kv, to = s["case"], s["kv"], s["to"]
    free, counts = kv.free_pages()
    kv.compact_into(to)
    out = {"free": free, "counts": counts, "table": to.page_table}
    for name in ("k_codes", "k_meta", "v_codes", "v_meta", "mask"):
        per = getattr(to, name).numel() // (c["layers"] * c["kv_heads"] * to.n_pages)
        out[name] = getattr(to, name)[:c["layers"] * c["kv_heads"] * to.n_pages * per].view(
            c["layers"] * c["kv_heads"], to.n_pages, per).view(torch.int32)
    return out


def _angles(s):
    axis = torch.tensor(s["pair_axis"], device=DEV)
    turned = s["positions"].double().t()[:, axis] * s["freq"].double()
    return turned.cos(), turned.sin()


def _plain_rotate(s):
    cos, sin = (t.float() for t in _angles(s))
    if s["case"]["rows"]:
        return torch.cat([cos, sin], 1)
    q, k, _ = _views(s)
    out = []
    for x in (q, k):
        a, b = x.float().split(HD // 2, -1)
        cs, sn = cos[:, None], sin[:, None]
        out.append(torch.cat([a * cs - b * sn, b * cs + a * sn], -1).half())
    return out


def _own_rotate(s):
    if s["case"]["rows"]:
        return s["kv"].rope_rows(s["positions"], s["freq"], s["pair_axis"])
    q, k, _ = _views(s)
    return list(s["kv"].rotate(q, k, s["positions"], s["freq"], s["pair_axis"]))


_RUN = {"attend": _plain_attend, "extend": _plain_extend, "fork": _plain_fork, "compact": _plain_compact,
        "rotate": _plain_rotate}
_RUN_OWN = {"attend": _own_attend, "extend": _own_extend, "fork": _own_fork, "compact": _own_compact,
            "rotate": _own_rotate}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------

def _exact_rows(c, k_words, k_meta, v_words, v_meta):
    """As _dequantized, in 64 bits: field by field of every lane's words."""
    bits, G, nv = c["bits"], c["group_k"], HD // c["group_v"]
    top = 2 ** bits - 1
    lane = torch.arange(64, device=DEV)
    r, m = lane // 16, lane % 16
    lead = k_words.shape[:-1]
    code = {"k": torch.empty(*lead, 32, HD, dtype=torch.float64, device=DEV),
            "v": torch.empty(*lead, 32, HD, dtype=torch.float64, device=DEV)}
    for f in range(8):
        word = lane * 4 + f // 2 if bits == 2 else (f // 4) * 256 + lane * 4 + f % 4
        for which, words in (("k", k_words), ("v", v_words)):
            w = words[..., word].long() & 0xFFFFFFFF
            for x in range(8):
                v, e = divmod(x, 2)
                bit = (16 * e + 2 * v + 2 + 8 * (f % 2) if bits == 2 else 16 * e + 2 + 4 * (v % 2) + 8 * (v // 2)) % 32
                value = (((w << 32) | w) >> bit) & top
                if which == "k":
                    code["k"][..., 16 * (f // 4) + m, 32 * (f % 4) + 8 * r + x] = value.double()
                else:
                    code["v"][..., 8 * r + x, 16 * f + m] = value.double()
    k = code["k"].flatten(-3, -2).unflatten(-2, (-1, G))
    k = (k * k_meta[..., :1, :].double() + k_meta[..., 1:, :].double()).flatten(-3, -2)
    v = code["v"]
    for t in range(32):
        for j in range(nv):
            part = v[..., t, j * c["group_v"]:(j + 1) * c["group_v"]]
            pair = v_meta[..., :, t // 2, j, t % 2].double()
            part.mul_(pair[..., :1]).add_(pair[..., 1:])
    return k, v.flatten(-3, -2)


def _exact_attend(c, s):
    q, k, v = _views(s)
    H, g = c["kv_heads"], c["q_heads"] // c["kv_heads"]
    out = torch.zeros(q.shape[0], c["q_heads"], HD, dtype=torch.float64, device=DEV)
    at = 0
    for b, n in enumerate(s["new"]):
        for h in range(H if n else 0):
            K, V, ok = _live(c, s, b, slice(h, h + 1), _exact_rows, torch.float64)
            K, V = K[0][ok[0]], V[0][ok[0]]
            for j in range(h * g, (h + 1) * g):
                for t0 in range(0, n, 1024):
                    t1 = min(n, t0 + 1024)
                    Kt, Vt, hidden = K, V, 0
                    if not c.get("cross"):
                        Kt, Vt = torch.cat([K, k[at:at + t1, h].double()]), torch.cat([V, v[at:at + t1, h].double()])
                    if Kt.shape[0] == 0:
                        continue
                    x = q[at + t0:at + t1, j].double() @ Kt.t() / math.sqrt(HD)
                    if not c.get("cross"):
                        hidden = torch.ones(t1 - t0, t1, dtype=torch.bool, device=DEV).triu(t0 + 1)
                        x[:, K.shape[0]:].masked_fill_(hidden, -math.inf)
                    out[at + t0:at + t1, j] = torch.softmax(x, -1) @ Vt
        at += n
    return out


def _exact_extend(c, s):
    """Rows and scores of the extension, unit by unit."""
    G, R, H, N, A, bits = c["group_k"], c["residual"], c["kv_heads"], c["budget"], c["aux"], c["bits"]
    rows, top = _res_rows(c), 2 ** c["bits"] - 1
    (nq, nr), start = s["split"][0], s["starts_in_ring"][0]
    n = s["more"] * G
    out = np.zeros((2, s["batch"], H, n, HD))
    ring = [(start + i) % rows for i in range(nr)]
    held = {name: s[name].cpu().numpy() for name in ("pool_score", "pool_idx", "pool_count", "aux_count", "k_res", "v_res")}
    ck, cv = s["chunk_k"].cpu().numpy(), s["chunk_v"].cpu().numpy()
    scores = held["pool_score"].copy().reshape(s["batch"], H, -1)
    at = 0

    def codes(x, axis):
        low, high = x.min(axis, keepdims=True), x.max(axis, keepdims=True)
        step = ((high - low) / top).astype(np.float32).astype(np.float16).astype(np.float64)
        safe = np.where(step == 0, 1.0, step)
        return low + step * np.where(step == 0, 0.0, np.clip(np.floor((x - low) / safe + 0.5), 0, top))
    for b, new in enumerate(s["new"]):
        for h in range(H if new else 0):
            k = np.concatenate([held["k_res"][h][ring], ck[at:at + new, h]]).astype(np.float64)
            v = np.concatenate([held["v_res"][h][ring], cv[at:at + new, h]]).astype(np.float64)
            n_in, n_aux = int(held["pool_count"][h]), int(held["aux_count"][h])
            score_of = scores[b, h]
            score_of[:n_in] = held["pool_score"][h, :n_in]
            score_of[N:N + n_aux] = held["pool_score"][h, N:N + n_aux]
            member = [(held["pool_score"][h, i], int(held["pool_idx"][h, i]), i) for i in range(n_in)]
            stopped = False
            for j in range((nr + new - R) // G if nr + new >= R + G else 0):
                gk, gv = k[j * G:(j + 1) * G], v[j * G:(j + 1) * G]
                chosen = []
                if N and not stopped:
                    all_of = sorted(member + [(np.abs(gk[t]).sum(), nq + j * G + t, -1 - t) for t in range(G)])
                    stay, fall = all_of[:N], sorted((m for m in all_of[N:] if m[2] >= 0), key=lambda m: m[2])
                    if n_aux + len(fall) > A:
                        stopped = True
                    else:
                        for i, m in enumerate(fall):
                            score_of[N + n_aux + i] = m[0]
                        n_aux += len(fall)
                        chosen = sorted((m for m in stay if m[2] < 0), key=lambda m: m[1])
                        places = [m[2] for m in fall] + list(range(len(member), N))
                        member = [m for m in stay if m[2] >= 0]
                        for m, place in zip(chosen, places):
                            member.append((m[0], m[1], place))
                            score_of[place] = m[0]
                taken = [-1 - m[2] for m in chosen]
                for which, x, axis in ((0, gk, 0), (1, gv, 2)):
                    y = x.copy()
                    y[taken] = x.mean(0).astype(np.float32).astype(np.float16)
                    y = codes(y, 0) if axis == 0 else codes(y.reshape(G, -1, c["group_v"]), 2).reshape(G, HD)
                    y[taken] = x[taken]
                    out[which, b, h, j * G:(j + 1) * G] = y
        at += new
    result = dict.fromkeys(["pool_k", "pool_v", "pool_idx", "pool_score", "pool_count", "aux_count", "frozen", "k_res",
                            "v_res", "seq_state", "page_table"])
    result["pool_score"] = torch.from_numpy(scores.reshape(s["batch"] * H, -1)).to(DEV)
    if n:
        result["k_rows"], result["v_rows"] = torch.from_numpy(out[0]).to(DEV), torch.from_numpy(out[1]).to(DEV)
    return result


def _exact_rotate(c, s):
    out = []
    pos, freq = s["positions"].cpu().numpy().astype(np.float64), s["freq"].cpu().numpy().astype(np.float64)
    angle = np.stack([pos[a] * f for a, f in zip(s["pair_axis"], freq)], 1)
    turn = torch.from_numpy(np.exp(1j * angle)).to(DEV)
    if c["rows"]:
        return torch.cat([turn.real, turn.imag], 1)
    for x in _views(s)[:2]:
        x = x.double()
        y = torch.complex(x[..., :HD // 2], x[..., HD // 2:]) * turn[:, None]
        out.append(torch.cat([y.real, y.imag], -1))
    return out


def exact(case, seed):
    c = dict(case)
    if c["kind"] in ("fork", "compact"):                    # (copies: nothing is computed)
        return None
    s = _INPUTS[c["kind"]](c, seed)
    s["case"] = c
    return {"attend": _exact_attend, "extend": _exact_extend, "rotate": _exact_rotate}[c["kind"]](c, s)
