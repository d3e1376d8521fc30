"""Sequences with a chunk behind them, on the CPU in 64 bits, for the tests of chunks of tokens."""
from __future__ import annotations

import numpy as np

import kvq_synth as S
from oracle import kvq_oracle as O
from paper_2505_10938_amd import cache as KC

HALF = 2.0 ** -11          # an fp16 rounding, relative


def config(layers=1, batch=2, q_heads=8, kv_heads=2, max_seq=1024, **kw):
    return KC.make_config(layers, batch, q_heads, kv_heads, max_seq, **kw)


def split(cfg, n):
    """(quantized tokens, ring rows) of a sequence of n tokens."""
    G, R = cfg.group_k, cfg.residual
    nq = G * ((n - R) // G) if n >= R + G else 0
    return nq, n - nq


def rows_of(cfg, lengths, layer=0, seed=0):
    """Keys and Values of every sequence: lists over the batch of fp16 [kv_heads, length, 128]."""
    out = ([], [])
    for b, n in enumerate(lengths):
        both = [S.unit_kv(seed, layer, b, h, n) for h in range(cfg.kv_heads)]
        for i in (0, 1):
            out[i].append(np.stack([x[i] for x in both]))
    return out


def state_of(cfg, k, v, layer=0):
    """The oracle's state of a unit after its first tokens (fp16 [n, 128]), and the rows that are left to the ring."""
    nq, _ = split(cfg, len(k))
    G = cfg.group_k
    budget = 0 if layer < cfg.untraced_layers else cfg.outlier_budget
    st = O.UnitState(128, cfg.bits, G, cfg.group_v, budget, cfg.aux_capacity)
    for i in range(0, nq, G):
        st.append_group(k[i:i + G], v[i:i + G])
    return st, k[nq:], v[nq:]


def attention(q, K, V, first_own=None, exact_rows=None):
    """Queries [n, g, 128] over rows K, V [L, 128] in 64 bits.  `first_own`: rows from there on are the queries' own
    tokens, of which query i sees the first i + 1.  Returns the outputs and the errors allowed (both [n, g, 128]):

    * the output's rounding, HALF of its magnitude;
    * the rounding of the softmax weights and of the dequantized Values to fp16, HALF each of sum(p |v|);
    * the rounding of the dequantized Keys (rows where `exact_rows` is false) shifts a score by at most
      d = HALF sum(|q| |k|) / sqrt(128), its fp32 sum by 128 * 2^-24 of the same sum, and weights by a factor of exp(+-d)
      each in numerator and denominator: (exp(2 d) - 1) sum(p |v|);
    * exp2, the running sums of up to L weights and rescalings: 2^-20 + L 2^-24 of sum(p |v|);
    * weights are taken relative to at most the largest one; those below 2^-14 of that are rounded to multiples of 2^-24:
      2^-25 max |v| each, over a sum of weights that is 1 at least.
    """
    q, K, V = (np.asarray(x, np.float64) for x in (q, K, V))
    n, g, L = q.shape[0], q.shape[1], K.shape[0]
    if L == 0:
        return np.zeros(q.shape), np.zeros(q.shape)
    x = np.einsum("ngd,ld->ngl", q, K) / np.sqrt(128.0)
    own = np.zeros(L, bool) if exact_rows is None else exact_rows
    size = np.einsum("ngd,ld->ngl", np.abs(q), np.abs(K)) / np.sqrt(128.0)
    shift = size * np.where(own, 128 * 2.0 ** -24, HALF + 128 * 2.0 ** -24)
    if first_own is not None:
        hidden = np.arange(L)[None, :] - first_own > np.arange(n)[:, None]
        x = np.where(hidden[:, None], -np.inf, x)
        shift = np.where(hidden[:, None], 0.0, shift)
    p = np.exp(x - x.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    out = p @ V
    heavy = p @ np.abs(V)
    d = shift.max(-1, keepdims=True)
    allowed = HALF * np.abs(out) + (2 * HALF + np.expm1(2 * d) + 2.0 ** -20 + L * 2.0 ** -24) * heavy
    return out, allowed + L * 2.0 ** -25 * np.abs(V).max() + 2.0 ** -25      # (and fp16 outputs below its normal numbers)


def live_state(cache, states):
    """Everything that a cache holds, without what holds no token: states = per sequence (n_quant, res_start, n_res), the same
    in every layer.  A dict of numpy arrays, for comparison."""
    c, sz = cache.cfg, cache.sizes
    out = {}
    names = ("k_codes", "k_meta", "v_codes", "v_meta", "mask")
    groups = c.max_seq // c.group_k
    for name, t in zip(names, cache.dense_quantized()):
        t = t[:t.numel() // (sz.units * groups) * sz.units * groups]
        a = t.cpu().numpy().reshape(c.layers, c.batch, c.kv_heads, groups, -1)
        for b, (nq, _, _) in enumerate(states):
            out[name, b] = a[:, b, :, :nq // c.group_k]
    shape = (c.layers, c.batch, c.kv_heads)
    ring = {"k_res": cache.res_view("k"), "v_res": cache.res_view("v")}
    for name, t in ring.items():
        a = t.cpu().numpy().view(np.uint16).reshape(*shape, sz.res_rows, 128)
        for b, (_, rs, nr) in enumerate(states):
            out[name, b] = a[:, b][:, :, (rs + np.arange(nr)) % sz.res_rows]
    count = {}
    for name in ("pool_count", "aux_count", "frozen"):
        count[name] = getattr(cache, name).cpu().numpy().view(np.int32)[:sz.units].reshape(shape)
        out[name, "all"] = count[name]
    slots, N = sz.pool_slots, c.outlier_budget
    for name, kind, width in (("pool_k", np.uint16, 128), ("pool_v", np.uint16, 128), ("pool_idx", np.int32, 1),
                              ("pool_score", np.float64, 1)):
        if slots == 0:
            continue
        a = getattr(cache, name).cpu().numpy().view(kind)[:sz.units * slots * width].reshape(*shape, slots, width)
        for where in np.ndindex(shape):
            out[name, where] = np.concatenate([a[where][:count["pool_count"][where]],
                                               a[where][N:N + count["aux_count"][where]]])
    return out


def assert_same(got, want):
    assert got.keys() == want.keys()
    for key in want:
        assert np.array_equal(got[key], want[key]), key
