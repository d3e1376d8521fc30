"""What the calls on chunks, forks, pages and rotations refuse, before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2505_10938_amd import binding as B
from paper_2505_10938_amd import cache as KC
from tests import chunk_helpers as H

BAD, UNSUPPORTED, SPACE = B.KVQ_ERR_INVALID_ARG, B.KVQ_ERR_UNSUPPORTED, B.KVQ_ERR_WORKSPACE
DENSE = B.kvq_qcache(256, 256, 256, 256, 256)
POOL = B.kvq_pool(256, 256, 256, 256, 256, 256, 256)
RES = B.kvq_residual(256, 256)


def paged(**kw):
    a = dict(k=256, table=256, stride=32, pages=50)
    a.update(kw)
    return B.kvq_qcache(a["k"], 256, 256, 256, 256, a["table"], a["stride"], a["pages"])


def cfg(**kw):
    return H.config(1, 2, 8, 2, 1024, **kw)


def attend(c=None, **kw):
    c = c or cfg()
    a = dict(layer=0, q=256, qs=1024, k=256, v=256, ks=256, starts=256, total=40, most=20, qc=DENSE, res=RES, seq=256, nq=64, rs=0,
             nr=100, pool=POOL, out=256, ws=512, bytes=1 << 40)
    a.update(kw)
    return B.load_library().kvq_prompt_attention(
        C.byref(c), a["layer"], a["q"], a["qs"], a["k"], a["v"], a["ks"], B.kvq_chunk(a["starts"], a["total"], a["most"]), a["qc"],
        a["res"], a["seq"], a["nq"], a["rs"], a["nr"], a["pool"], a["out"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw", [
    dict(layer=1), dict(layer=-1), dict(q=None), dict(q=264), dict(qs=1016), dict(qs=1028), dict(k=None), dict(v=None), dict(k=264),
    dict(v=264), dict(ks=248), dict(ks=260), dict(starts=258), dict(total=0), dict(most=0), dict(most=41), dict(starts=None, total=41),
    dict(nq=48), dict(nq=-32), dict(nq=1056), dict(nr=-1), dict(nr=161), dict(seq=264), dict(seq=None, rs=160),
    dict(seq=None, rs=-1), dict(out=None), dict(out=260), dict(qc=B.kvq_qcache(None, 256, 256, 256, 256)),
    dict(qc=B.kvq_qcache(264, 256, 256, 256, 256)), dict(qc=B.kvq_qcache(256, 264, 256, 256, 256)),
    dict(qc=B.kvq_qcache(256, 256, 256, 260, 256)), dict(qc=B.kvq_qcache(256, 256, 256, 256, 258)), dict(qc=paged(pages=0)),
    dict(qc=paged(stride=31)), dict(res=B.kvq_residual(None, 256)), dict(res=B.kvq_residual(256, 264)),
    dict(pool=B.kvq_pool(None, 256, 256, 256, 256, 256, 256)), dict(pool=B.kvq_pool(256, 264, 256, 256, 256, 256, 256)),
    dict(pool=B.kvq_pool(256, 256, 256, 256, None, 256, 256)), dict(pool=B.kvq_pool(256, 256, 256, 256, 256, None, 256))])
def test_attention(kw):
    assert attend(**kw) == BAD


def test_attention_workspace_and_sizes():
    c = cfg()
    need = B.kvq_prompt_workspace_bytes(c, 20, 1024, 160)
    assert need > 0
    for kw in (dict(ws=None), dict(ws=128), dict(bytes=0), dict(bytes=need - 1)):
        assert attend(nq=1024, nr=160, **kw) == SPACE
    with pytest.raises(B.KvqError):
        B.kvq_prompt_workspace_bytes(c, 0, 0, 0)
    with pytest.raises(B.KvqError):
        B.kvq_prompt_workspace_bytes(c, 1, 33, 0)
    with pytest.raises(B.KvqError):
        B.kvq_prompt_workspace_bytes(c, 1, 0, 161)
    # a workspace never shrinks below what a call without new tokens would use
    assert attend(total=1 << 30, most=1 << 29) == UNSUPPORTED
    assert attend(H.config(1, 2, 8, 2, 1024, head_dim=64)) == UNSUPPORTED
    assert attend(H.config(1, 2, 6, 2, 1024)) == UNSUPPORTED


def extend(c=None, **kw):
    c = c or cfg()
    a = dict(layer=0, k=256, v=256, ks=256, starts=256, total=40, most=20, res=RES, seq=256, nq=0, rs=0, nr=0, pool=POOL, sel=256,
             bytes=1 << 30, qc=DENSE)
    a.update(kw)
    return B.load_library().kvq_extend(
        C.byref(c), a["layer"], a["k"], a["v"], a["ks"], B.kvq_chunk(a["starts"], a["total"], a["most"]), a["res"], a["seq"], a["nq"],
        a["rs"], a["nr"], a["pool"], a["sel"], a["bytes"], a["qc"], None)


@pytest.mark.parametrize("kw", [
    dict(layer=1), dict(k=None), dict(v=None), dict(k=264), dict(ks=128), dict(ks=257), dict(total=0), dict(most=0), dict(most=50),
    dict(starts=257), dict(res=B.kvq_residual(256, None)), dict(res=B.kvq_residual(264, 256)), dict(seq=260), dict(sel=None),
    dict(qc=B.kvq_qcache(256, None, 256, 256, 256)), dict(qc=paged(pages=-1)),
    dict(pool=B.kvq_pool(256, 256, None, 256, 256, 256, 256)), dict(pool=B.kvq_pool(256, 256, 256, 256, 256, 256, None)),
    dict(seq=None, nq=16), dict(seq=None, nq=-32), dict(seq=None, rs=16), dict(seq=None, rs=160), dict(seq=None, nr=160),
    dict(seq=None, nr=-1), dict(seq=None, starts=None, nq=1024, nr=150)])
def test_extension(kw):
    assert extend(**kw) == BAD


def test_extension_space_and_settings():
    assert extend(bytes=2 * 2 * 32 - 1) == SPACE
    assert extend(H.config(1, 2, 8, 2, 1024, outlier_budget=0, value_per_step=1)) == UNSUPPORTED
    assert extend(total=1 << 30, most=1 << 30) == UNSUPPORTED
    lib, c = B.load_library(), cfg()
    assert lib.kvq_seq_extend(C.byref(c), None, B.kvq_chunk(256, 40, 20), None) == BAD
    assert lib.kvq_seq_extend(C.byref(c), 264, B.kvq_chunk(256, 40, 20), None) == BAD
    assert lib.kvq_seq_extend(C.byref(c), 256, B.kvq_chunk(256, 40, 0), None) == BAD
    assert lib.kvq_seq_extend(C.byref(H.config(1, 2, 8, 2, 1024, outlier_budget=0, value_per_step=1)), 256,
                              B.kvq_chunk(256, 40, 20), None) == UNSUPPORTED


def fork(c=None, **kw):
    c = c or cfg()
    a = dict(pairs=256, n=2, seq=256, nq=0, rs=0, nr=0, res=RES, pool=POOL, qc=DENSE, table=None)
    a.update(kw)
    return B.load_library().kvq_fork_sequences(C.byref(c), a["pairs"], a["n"], a["seq"], a["nq"], a["rs"], a["nr"], a["res"],
                                               a["pool"], a["qc"], a["table"], None)


@pytest.mark.parametrize("kw", [
    dict(pairs=None), dict(pairs=258), dict(n=0), dict(n=3), dict(seq=264), dict(seq=None, nq=31), dict(seq=None, nq=1056),
    dict(seq=None, rs=160), dict(seq=None, nr=161), dict(res=B.kvq_residual(None, 256)), dict(res=B.kvq_residual(256, 264)),
    dict(pool=B.kvq_pool(256, 264, 256, 256, 256, 256, 256)), dict(pool=B.kvq_pool(256, 256, 258, 256, 256, 256, 256)),
    dict(pool=B.kvq_pool(256, 256, 256, 260, 256, 256, 256)), dict(pool=B.kvq_pool(256, 256, 256, 256, 256, 256, None)),
    dict(qc=paged()), dict(qc=paged(), table=512), dict(table=256), dict(qc=B.kvq_qcache(264, 256, 256, 256, 256)),
    dict(qc=B.kvq_qcache(256, 256, 256, 256, 258)), dict(qc=paged(stride=31), table=256)])
def test_fork(kw):
    assert fork(**kw) == BAD


def test_fork_of_too_many():
    assert fork(H.config(1, 1100, 8, 2, 1024), n=1025) == UNSUPPORTED


def test_pages():
    lib, c = B.load_library(), cfg()
    free = lambda qc=paged(), seq=256, nq=0, out=256, counts=256: lib.kvq_free_pages(C.byref(c), qc, seq, nq, out, counts, None)
    copy = lambda a=paged(), b=paged(k=512), pairs=256, n=1: lib.kvq_copy_pages(C.byref(c), a, b, pairs, n, None)

    def pack(a=paged(), seq=256, nq=0, b=B.kvq_qcache(512, 512, 512, 512, 512, None, 32, 7), table=512, counts=256, ws=256, bytes=200):
        return lib.kvq_compact_pages(C.byref(c), a, seq, nq, b, table, counts, ws, bytes, None)
    for call in (free, pack):
        assert call(DENSE) == BAD and call(paged(pages=0)) == BAD and call(paged(stride=3)) == BAD
        assert call(seq=264) == BAD and call(seq=None, nq=5) == BAD and call(seq=None, nq=2048) == BAD
        assert call(counts=None) == BAD and call(counts=258) == BAD
    assert free(out=None) == BAD and free(out=257) == BAD
    assert copy(DENSE) == BAD and copy(b=DENSE) == BAD and copy(paged(k=264)) == BAD
    assert copy(pairs=None) == BAD and copy(pairs=255) == BAD and copy(n=0) == BAD
    assert pack(b=paged()) == BAD                                            # the same memory
    assert pack(b=B.kvq_qcache(512, 512, 512, 512, 512, None, 31, 7)) == BAD
    assert pack(b=B.kvq_qcache(512, 512, 512, 512, 512, None, 32, 0)) == BAD
    assert pack(table=None) == BAD and pack(table=256) == BAD and pack(table=513) == BAD
    assert pack(ws=None) == SPACE and pack(ws=258) == SPACE and pack(bytes=199) == SPACE


def test_rotation():
    lib, c = B.load_library(), cfg()

    def axes(q=256, qs=1024, k=256, ks=256, n=5, p=256, a=2, of=bytes(64), f=256, qo=256, qos=1024, ko=512, kos=256):
        return lib.kvq_rope_axes(C.byref(c), q, qs, k, ks, n, p, a, of, f, qo, qos, ko, kos, None)

    def rows(n=5, p=256, a=2, of=bytes(64), f=256, out=256):
        return lib.kvq_rope_rows(C.byref(c), n, p, a, of, f, out, None)
    for call in (axes, rows):
        for kw in (dict(n=0), dict(n=-1), dict(p=None), dict(p=258), dict(a=0), dict(a=9), dict(of=None), dict(of=b"\2" * 64),
                   dict(f=None), dict(f=255)):
            assert call(**kw) == BAD, kw
        assert call(n=1 << 30) == UNSUPPORTED
    for kw in (dict(q=None), dict(k=None), dict(q=None, qo=None, k=None, ko=None), dict(qo=None), dict(ko=None), dict(q=264),
               dict(qo=264), dict(ko=260), dict(qs=1000), dict(ks=252), dict(qos=1023), dict(kos=0), dict(qos=2048)):
        assert axes(**kw) == BAD, kw
    assert rows(out=None) == BAD and rows(out=264) == BAD


def test_arguments_of_the_methods():
    cache = KC.KVCache(cfg(), device="cpu")
    ragged = KC.RaggedKVCache(cfg(), device="cpu")
    x = lambda *s, dtype=torch.float16: torch.zeros(s, dtype=dtype)
    q, k = x(2, 3, 8, 128), x(2, 3, 2, 128)
    bad = [lambda: cache.attend(0, q.float()), lambda: cache.attend(0, x(2, 3, 7, 128)), lambda: cache.attend(0, q, k),
           lambda: cache.attend(0, q, k, x(2, 2, 2, 128)), lambda: cache.attend(0, q, k, x(2, 3, 4, 128)[:, :, :2]),
           lambda: cache.attend(0, q, out=x(2, 3, 8, 64)), lambda: cache.attend(0, q, out=q.float()),
           lambda: cache.attend(0, x(2, 0, 8, 128)), lambda: cache.attend(0, x(2, 3, 8, 256)[..., ::2]),
           lambda: cache.extend(0, k, x(2, 1, 2, 128)), lambda: cache.extend(0, k, k.float()),
           lambda: ragged.attend(0, q[0], torch.zeros(3), 3), lambda: ragged.attend(0, q[0], torch.zeros(2, dtype=torch.int32), 3),
           lambda: ragged.extend(0, k[0], k[0], torch.zeros(6, dtype=torch.int32)[::2], 3),
           lambda: ragged.advance_by(torch.zeros(3), 3), lambda: cache.fork(torch.zeros(1, 2)),
           lambda: cache.fork(torch.zeros(2, dtype=torch.int32)), lambda: cache.free_pages(), lambda: cache.compact_into(None),
           lambda: cache.copy_pages(torch.zeros(1, 2, dtype=torch.int32)), lambda: cache.adopt(None),
           lambda: cache.rope_rows(torch.zeros(3), torch.zeros(64)), lambda: cache.rope_rows(torch.zeros(3, dtype=torch.int32), torch.zeros(63)),
           lambda: cache.rotate(q, None, torch.zeros(1, 5, dtype=torch.int32), torch.zeros(64)),
           lambda: cache.rotate(q, None, torch.zeros(6, dtype=torch.int32), torch.zeros(64), q_out=x(2, 2, 8, 128))]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, RuntimeError)):
            call()
            print("not refused:", i)
    with pytest.raises(B.KvqError):
        cache.rope_rows(torch.zeros(3, dtype=torch.int32), torch.zeros(64), [0] * 63)


def test_pools_of_another_configuration():
    c = KC.make_config(2, 2, 8, 2, 512)
    cache = KC.KVCache(c, device="cpu", n_pages=20)
    pairs = torch.zeros(1, 2, dtype=torch.int32)
    for other in (KC.make_config(1, 2, 8, 2, 512), KC.make_config(2, 2, 8, 4, 512), KC.make_config(2, 2, 8, 2, 512, bits=4),
                  KC.make_config(2, 2, 8, 2, 512, group_k=64), KC.make_config(2, 2, 8, 2, 512, group_v=64)):
        to = KC.PagePool(other, 30, device="cpu")
        for call in (lambda: cache.compact_into(to), lambda: cache.adopt(to), lambda: cache.copy_pages(pairs, to)):
            with pytest.raises(ValueError):
                call()
    for other in (KC.make_config(2, 3, 8, 2, 512), KC.make_config(2, 2, 8, 2, 1024)):   # (the tables differ, the pages do not)
        to = KC.PagePool(other, 30, device="cpu")
        for call in (lambda: cache.compact_into(to), lambda: cache.adopt(to)):
            with pytest.raises(ValueError):
                call()
    same = KC.PagePool(c, 30, device="cpu")
    cache.adopt(same)
    assert cache.n_pages == 30 and cache.page_table is same.page_table
