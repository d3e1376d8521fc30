"""A chunk that joins a cache (kvq_extend, kvq_seq_extend) against the same tokens appended one by one, bit for bit, and
against the oracle."""
import numpy as np
import pytest

from paper_2505_10938_amd import cache as KC
from tests import chunk_helpers as H

pytestmark = pytest.mark.gpu

SETTINGS = [dict(), dict(bits=4, group_k=64, group_v=64), dict(group_k=128, group_v=128, residual=32, outlier_budget=3),
            dict(residual=0), dict(residual=37, group_v=128), dict(outlier_budget=0), dict(outlier_budget=40, aux_capacity=64),
            dict(outlier_budget=8, aux_capacity=4), dict(outlier_budget=20, aux_capacity=64, group_k=64, bits=4),
            dict(outlier_budget=64, aux_capacity=64, group_k=128, group_v=32)]


def tokens(cfg, n, seed=0, layer=0):
    """Keys and Values of n tokens of every sequence, device fp16 [batch, n, kv_heads, 128]."""
    import torch
    K, V = H.rows_of(cfg, [n] * cfg.batch, layer=layer, seed=seed)
    return tuple(torch.from_numpy(np.stack(x).transpose(0, 2, 1, 3).copy()).cuda() for x in (K, V))


def state(cache, layer=0):
    return cache.n_quant[layer], cache.res_start[layer], cache.n_res[layer]


@pytest.mark.parametrize("kw", SETTINGS)
@pytest.mark.parametrize("chunks", [[1, 500, 2, 131], [159, 1, 160], [700], [33, 32, 31, 64, 200]])
def test_equals_appending_one_by_one(kw, chunks):
    cfg = H.config(1, 2, 4, 2, 1024, **kw)
    k, v = tokens(cfg, sum(chunks))
    chunked, single = KC.KVCache(cfg), KC.KVCache(cfg)
    at = 0
    for n in chunks:
        chunked.extend(0, k[:, at:at + n].contiguous(), v[:, at:at + n].contiguous())
        for i in range(at, at + n):
            single.append(0, k[:, i].contiguous(), v[:, i].contiguous())
        at += n
        assert state(chunked) == state(single)
        states = [state(single)] * cfg.batch
        H.assert_same(H.live_state(chunked, states), H.live_state(single, states))


def test_equals_the_oracle():
    from tests import helpers as TH
    import kvq_synth as S
    w = S.Workload("extend", 1, 2, 4, 2, 900, outlier_budget=8)
    K, V = S.layer_kv(w, 0)
    import torch
    cfg = H.config(1, 2, 4, 2, 1024)
    cache = KC.KVCache(cfg)
    k, v = (torch.from_numpy(x.transpose(0, 2, 1, 3).copy()).cuda() for x in (K, V))
    for a, b in ((0, 300), (300, 301), (301, 900)):
        cache.extend(0, k[:, a:b].contiguous(), v[:, a:b].contiguous())
    TH.compare_state(cache, TH.oracle_states(w, K, V, w.n_quant), w, w.n_quant)
    assert state(cache)[0] == w.n_quant and state(cache)[2] == w.n_res


def test_behind_a_prompt_and_on_from_there():
    """A prompt by the call for prompts, a chunk, single tokens: the decode step's outputs are those of single tokens."""
    import torch
    cfg = H.config(1, 2, 8, 2, 2048)
    k, v = tokens(cfg, 1200)
    a, b = KC.KVCache(cfg), KC.KVCache(cfg)
    rows = [x[:, :500].transpose(1, 2).contiguous() for x in (k, v)]
    for c in (a, b):
        c.prefill(0, *rows)
    a.extend(0, k[:, 500:1100].contiguous(), v[:, 500:1100].contiguous())
    for i in range(500, 1100):
        b.append(0, k[:, i].contiguous(), v[:, i].contiguous())
    for i in range(1100, 1200):
        q = torch.randn(2, 8, 128, device="cuda").half()
        assert torch.equal(a.step(0, k[:, i].contiguous(), v[:, i].contiguous(), q),
                           b.step(0, k[:, i].contiguous(), v[:, i].contiguous(), q))


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kw", [dict(), dict(bits=4, group_k=128, group_v=64, residual=40), dict(residual=0, group_k=64)])
def test_lengths_that_differ(paged, kw):
    import torch
    cfg = H.config(2, 4, 4, 2, 1024, untraced_layers=1, **kw)
    pages = cfg.batch * (cfg.max_seq // cfg.group_k)
    deal = torch.randperm(pages + 5, generator=torch.Generator().manual_seed(1))[:pages].view(cfg.batch, -1).int()
    lengths = [[300, 0, 7, 161], [0, 900, 33, 1], [129, 64, 0, 640], [1, 1, 1, 1]]
    total = [sum(n) for n in zip(*lengths)]
    rows = [H.rows_of(cfg, total, layer=layer) for layer in range(2)]
    chunked, single = (KC.RaggedKVCache(cfg, n_pages=pages + 5 if paged else None) for _ in range(2))
    for c in (chunked, single):
        if paged:
            c.page_table.copy_(deal)
        c.set_active([1] * cfg.batch)
    done = [0] * cfg.batch
    for new in lengths:
        starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        for layer in range(2):
            k, v = (torch.from_numpy(np.concatenate([x[b][:, done[b]:done[b] + new[b]].transpose(1, 0, 2)
                                                     for b in range(cfg.batch)])).cuda() for x in rows[layer])
            # (between other columns of one array)
            wide = torch.zeros(k.shape[0], 7, 128, dtype=torch.float16, device="cuda")
            wide[:, 1:3], wide[:, 5:] = k, v
            chunked.extend(layer, wide[:, 1:3], wide[:, 5:], starts, max(new))
        chunked.advance_by(starts, max(new))
        for i in range(max(new)):
            single.set_active([int(i < n) for n in new])
            for layer in range(2):
                k, v = (torch.from_numpy(np.stack([x[b][:, min(done[b] + i, total[b] - 1)] for b in range(cfg.batch)])).cuda()
                        for x in rows[layer])
                single.append(layer, k, v)
            single.advance()
        single.set_active([1] * cfg.batch)
        done = [a + n for a, n in zip(done, new)]
        assert torch.equal(chunked.seq_state, single.seq_state)
        states = [tuple(s[:3]) for s in chunked.seq_state.tolist()]
        assert [s[0] + s[2] for s in states] == done
        H.assert_same(H.live_state(chunked, states), H.live_state(single, states))


def test_sequences_that_are_left_alone():
    import torch
    cfg = H.config(1, 6, 4, 2, 256, residual=32)
    cache = KC.RaggedKVCache(cfg)
    k, v = tokens(cfg, 300)
    starts = torch.arange(0, 6 * 300 + 1, 300, dtype=torch.int32, device="cuda")
    # fits exactly (256 quantized, 44 in the ring); inactive; does not fit; states that no call leaves
    cache.seq_state.copy_(torch.tensor([[0, 0, 0, 1], [0, 0, 0, 0], [32, 0, 32, 1], [16, 0, 0, 1], [0, 5, 0, 1], [0, 0, 64, 1]],
                                       dtype=torch.int32))
    before = {n: getattr(cache, n).clone() for n in ("k_codes", "k_meta", "v_codes", "v_meta", "mask", "k_res", "v_res",
                                                     "pool_k", "pool_v", "pool_idx", "pool_score", "pool_count", "aux_count",
                                                     "frozen", "seq_state")}
    cache.extend(0, k.flatten(0, 1), v.flatten(0, 1), starts, 300)
    cache.advance_by(starts, 300)
    assert cache.seq_state[0].tolist() == [256, 256 % cache.sizes.res_rows, 44, 1]
    assert torch.equal(cache.seq_state[1:], before["seq_state"][1:])
    for name, old in before.items():
        if name != "seq_state":
            per = getattr(cache, name).numel() // cache.sizes.units * 2      # two kv heads of a sequence
            if name in ("pool_k", "pool_v"):
                per = cache.sizes.pool_slots * 256 * 2
            assert torch.equal(getattr(cache, name)[per:], old[per:]), name
            assert not torch.equal(getattr(cache, name)[:per], old[:per]) or name in ("frozen", "aux_count"), name


def test_a_captured_chunk_replays():
    import torch
    cfg = H.config(1, 2, 4, 2, 2048)
    k, v = tokens(cfg, 200)
    want, got = KC.RaggedKVCache(cfg), KC.RaggedKVCache(cfg)
    starts = torch.tensor([0, 200, 400], dtype=torch.int32, device="cuda")
    feed = [torch.zeros(400, 2, 128, dtype=torch.float16, device="cuda") for _ in range(2)]
    for c in (want, got):
        c.set_active([1, 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got.extend(0, feed[0], feed[1], starts, 200)
        got.advance_by(starts, 200)
    for turn in range(4):
        rows = [(x if turn % 2 else x.flip(1)).reshape(400, 2, 128).contiguous() for x in (k, v)]
        want.extend(0, *rows, starts, 200)
        want.advance_by(starts, 200)
        for f, r in zip(feed, rows):
            f.copy_(r)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want.seq_state, got.seq_state)
        states = [tuple(s[:3]) for s in want.seq_state.tolist()]
        H.assert_same(H.live_state(got, states), H.live_state(want, states))
