"""Chunks of tokens, forks, pages and rotations together, as a server would use them: requests behind one system prompt."""
import numpy as np
import pytest

from paper_2505_10938_amd import cache as KC
from tests import chunk_helpers as H
from tests.test_chunk_attention import check
from tests.test_rope_axes import FREQ, rotated, turns

pytestmark = pytest.mark.gpu

AXES = [0] * 16 + [1] * 24 + [2] * 24


class Server:
    """A paged cache of four sequences, and on the host every sequence's rows so far."""

    def __init__(self, cfg, seed):
        import torch
        self.cfg, self.rng = cfg, np.random.default_rng(seed)
        groups = cfg.max_seq // cfg.group_k
        self.cache = KC.RaggedKVCache(cfg, n_pages=cfg.batch * groups)
        self.cache.page_table.copy_(torch.arange(cfg.batch * groups, dtype=torch.int32).flip(0).view(cfg.batch, groups))
        self.cache.set_active([1] * cfg.batch)
        empty = np.zeros((cfg.kv_heads, 0, 128), np.float16)
        self.K = [[empty] * cfg.batch for _ in range(cfg.layers)]
        self.V = [[empty] * cfg.batch for _ in range(cfg.layers)]
        self.freq = torch.from_numpy(FREQ).cuda()

    def lengths(self):
        return [x.shape[1] for x in self.K[0]]

    def positions(self, new):
        """Time, height and width of the new tokens."""
        at = np.concatenate([n0 + np.arange(n) for n0, n in zip(self.lengths(), new)])
        return np.stack([at, at // 7, 3 * (at % 7)]).astype(np.int32)

    def rotate(self, positions, *rows):
        """Rows of one array [tokens, heads, 128] by the cache's rotation, in place of a projection's output."""
        import torch
        q, k = rows
        both = torch.from_numpy(np.concatenate([q, k], 1)).cuda()
        q_at, k_at = both[:, :q.shape[1]], both[:, q.shape[1]:]
        self.cache.rotate(q_at, k_at, torch.from_numpy(positions).cuda(), self.freq, AXES, q_out=q_at, k_out=k_at)
        cos, sin = turns(positions, AXES)
        want = rotated(np.concatenate([q, k], 1), cos, sin)
        size = np.abs(np.concatenate([q, k], 1).astype(np.float64))
        size = np.concatenate([size[..., :64] + size[..., 64:]] * 2, -1)
        err = np.abs(both.cpu().numpy().astype(np.float64) - want)
        # (as in test_rope_axes)
        assert (err <= 7 * 2.0 ** -24 * size + H.HALF * np.abs(want) + 2.0 ** -25).all()
        return q_at, k_at

    def take(self, layer, k, v, new):
        at = 0
        for b, n in enumerate(new):
            for rows, x in ((self.K, k), (self.V, v)):
                rows[layer][b] = np.concatenate([rows[layer][b], x[at:at + n].transpose(1, 0, 2)], 1)
            at += n

    def drawn(self, n):
        c = self.cfg
        return [self.rng.standard_normal((n, h, 128)).astype(np.float16) for h in (c.q_heads, c.kv_heads, c.kv_heads)]

    def chunk(self, new):
        import torch
        c, hist, positions = self.cfg, self.lengths(), self.positions(new)
        starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        for layer in range(c.layers):
            q, k, v = self.drawn(sum(new))
            q, k = self.rotate(positions, q, k)
            vd = torch.zeros(v.shape[0], c.q_heads + c.kv_heads, 128, dtype=torch.float16, device="cuda")
            vd[:, c.q_heads:] = torch.from_numpy(v).cuda()
            vd = vd[:, c.q_heads:]                          # (Keys and Values are equally spaced)
            out = self.cache.attend(layer, q, starts, max(new), k, vd)
            self.cache.extend(layer, k, vd, starts, max(new))
            self.take(layer, k.cpu().numpy(), v, new)
            check(out, c, hist, new, self.K[layer], self.V[layer], q.cpu().numpy())
        self.cache.advance_by(starts, max(new))

    def step(self):
        """A token each: append, advance, decode."""
        import torch
        c, new = self.cfg, [1] * self.cfg.batch
        positions, rows = self.positions(new), []
        for layer in range(c.layers):
            q, k, v = self.drawn(c.batch)
            q, k = self.rotate(positions, q, k)
            self.cache.append(layer, k.contiguous(), torch.from_numpy(v).cuda())
            self.take(layer, k.cpu().numpy(), v, new)
            rows.append(q.contiguous())
        self.cache.advance()
        for layer, q in enumerate(rows):
            out = self.cache.decode(layer, q)
            check(out, c, self.lengths(), new, self.K[layer], self.V[layer], q.cpu().numpy(), cross=True)

    def fork(self, pairs):
        import torch
        self.cache.fork(torch.tensor(pairs, dtype=torch.int32, device="cuda"))
        for rows in self.K + self.V:
            before = list(rows)
            for a, b in pairs:
                rows[b] = before[a]

    def into_another_pool(self, n_pages):
        """Live pages to the front of a pool of another size, the free ones to the groups that have none yet."""
        to = KC.PagePool(self.cfg, n_pages)
        live = int(self.cache.compact_into(to)[1])
        table = to.page_table.cpu().numpy()
        quantized = [H.split(self.cfg, n)[0] // self.cfg.group_k for n in self.lengths()]
        assert [(row >= 0).sum() for row in table] == quantized and len(np.unique(table[table >= 0])) == live
        self.cache.adopt(to)
        free, counts = self.cache.free_pages()
        assert counts.tolist() == [n_pages - live, live]
        import torch
        none = torch.from_numpy(np.argwhere(table < 0)).cuda()[:n_pages - live]
        self.cache.page_table[none[:, 0], none[:, 1]] = free[:len(none)]
        return live


@pytest.mark.parametrize("kw", [dict(outlier_budget=3), dict(bits=4, group_k=64, group_v=128, residual=40)])
def test_requests_behind_one_prompt(kw):
    cfg = H.config(2, 4, 8, 2, 512, **kw)
    s = Server(cfg, 5)
    s.chunk([230, 0, 0, 0])                                 # the system prompt, on an empty cache
    s.fork([(0, 1), (0, 2), (0, 3)])
    s.chunk([0, 5, 130, 64])
    shared = s.into_another_pool(4 * 512 // cfg.group_k + 3)
    each = [H.split(cfg, n)[0] // cfg.group_k for n in s.lengths()]
    assert shared == sum(each) - 3 * each[0]                # (the prompt's groups are there once)
    for _ in range(3):
        s.step()
    s.fork([(2, 0), (3, 2), (2, 3)])                        # beams change places, all at once
    s.chunk([1, 33, 2, 95])
    s.step()
