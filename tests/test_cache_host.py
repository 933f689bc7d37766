"""Refusals of the block cache calls: every check runs on the host before anything is enqueued."""
import pytest

import paper_2509_05165_amd as kv
from test_abi_host import FAKE, P, expect

BIG = 1 << 40


def cache(**kw):
    a = dict(format=kv.KVC_E4M3, blocks=8, table_width=4, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, weight=FAKE, table=FAKE)
    a.update(kw)
    return kv.KvcCache(**a)


def fill(p=None, c=None, **kw):
    p = p or P()
    a = dict(k=[FAKE] * 2, v=[FAKE] * 2, idx=FAKE, lengths=FAKE, offsets=FAKE, cu_seqlens=[0, 100], total_budget=10)
    a.update(kw)
    kv.kvc_cache_fill(p, a["k"], a["v"], a["idx"], a["lengths"], a["offsets"], a["cu_seqlens"], a["total_budget"],
                      c or cache(), scores=a.get("scores", 0), workspace=a.get("workspace", 0),
                      workspace_bytes=a.get("workspace_bytes", 0))


def append(p=None, c=None, layer=0, k=FAKE, v=FAKE, lengths=FAKE):
    kv.kvc_cache_append(p or P(window=1), layer, k, v, lengths, c or cache())


def attend(p=None, c=None, layer=0, q=FAKE, lengths=FAKE, most=256, out=FAKE, ws=FAKE, size=BIG, **kw):
    kv.kvc_cache_attend(p or P(window=1), layer, q, lengths, most, c or cache(), out, ws, size, **kw)


def evict(p=None, c=None, lengths=FAKE, keep=FAKE, most=64, table=2 * FAKE, out=2 * FAKE, ws=FAKE, size=BIG):
    kv.kvc_cache_evict(p or P(), lengths, keep, most, c or cache(), table, out, ws, size)


CALLS = [fill, append, attend, evict]


@pytest.mark.parametrize("call", CALLS)
def test_params_and_cache(call):
    expect(1, call, P(hq=6, hkv=4))
    expect(1, call, P(dtype=5))
    expect(2, call, P(head_dim=24))                 # rows of 48 bytes, but codes in pieces of 16
    expect(2, call, P(head_dim=272))
    expect(1, call, c=cache(format=2))
    expect(1, call, c=cache(blocks=0))
    expect(1, call, c=cache(table_width=0))
    expect(2, call, c=cache(table_width=1 << 23))
    for name in ("k", "v", "k_scale", "v_scale", "table"):
        expect(1, call, c=cache(**{name: 0}))
    expect(1, call, c=cache(k=FAKE + 8))
    expect(1, call, c=cache(v=FAKE + 1))


def test_missing_structs():
    expect(1, kv.kvc_cache_append, None, 0, FAKE, FAKE, FAKE, cache())
    expect(1, kv.kvc_cache_append, P(), 0, FAKE, FAKE, FAKE, None)
    expect(1, kv.kvc_cache_attend, None, 0, FAKE, FAKE, 64, cache(), FAKE, FAKE, BIG)
    expect(1, kv.kvc_cache_evict, P(), FAKE, FAKE, 64, None, 2 * FAKE, 2 * FAKE, FAKE, BIG)
    expect(1, kv.kvc_cache_attend_workspace, None, 64)
    expect(1, kv.kvc_cache_evict_workspace, None, 64)


def test_fill():
    expect(1, fill, k=None)
    expect(1, fill, v=[FAKE, 0])
    expect(1, fill, lengths=0)
    expect(1, fill, offsets=0)
    expect(1, fill, cu_seqlens=[1, 100])
    expect(1, fill, total_budget=-1)
    expect(1, fill, total_budget=201)               # more than layers * tokens
    expect(1, fill, c=cache(weight=0), scores=FAKE)
    expect(3, fill, P(order=kv.KVC_ORDER_POSITION))  # the ordered list needs workspace
    fill(total_budget=0)                            # nothing to store: nothing is enqueued


@pytest.mark.parametrize("call", [append, attend])
def test_layer(call):
    expect(1, call, layer=-1)
    expect(1, call, layer=2)


def test_append():
    for name in ("k", "v", "lengths"):
        expect(1, append, **{name: 0})


def test_attend():
    for name in ("q", "lengths", "out"):
        expect(1, attend, **{name: 0})
    expect(1, attend, most=-1)
    expect(1, attend, weight_in=FAKE)               # nowhere to write the sum
    need = kv.kvc_cache_attend_workspace(P(window=1), 256, True)
    assert need > 0
    expect(3, attend, size=need - 1, weight_out=FAKE)
    expect(3, attend, ws=0, weight_out=FAKE)
    expect(3, attend, ws=FAKE + 16, weight_out=FAKE)
    expect(2, attend, P(window=4096, hq=1024, hkv=1, batch=256), weight_out=FAKE)


def test_attend_workspace():
    size = kv.kvc_cache_attend_workspace
    expect(1, size, P(), -1)
    expect(1, size, P(), 1 << 29)
    for p in (P(window=1), P(window=7, batch=3), P(window=1, batch=200)):
        sizes = [size(p, n) for n in (0, 1, 64, 65, 300, 1000, 4097, 60000, 70001, 131072, 1 << 20)]
        assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)
        assert all(size(p, n, True) >= size(p, n) + 4 * n for n in (1, 64, 999, 131072))
    # with one split there is nothing to join
    assert size(P(window=1), 64) == 0 and size(P(window=1), 131072) > 0


def test_evict():
    for name in ("lengths", "keep", "table", "out"):
        expect(1, evict, **{name: 0})
    expect(1, evict, c=cache(weight=0))
    expect(1, evict, table=FAKE)                    # the cache's own table
    expect(1, evict, out=FAKE)                      # the lengths that are read
    expect(1, evict, most=-1)
    expect(1, evict, most=257)
    need = kv.kvc_cache_evict_workspace(P(), 64)
    assert need == 2 * 4 * 64 * 4                   # a position per layer, head and kept token
    expect(3, evict, size=need - 1)
    expect(3, evict, ws=0)
    expect(1, kv.kvc_cache_evict_workspace, P(), -1)
