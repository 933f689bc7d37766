"""kvc_cache_fill and kvc_cache_append against the oracle, bit for bit, the untouched bytes of the pools included."""
import numpy as np
import pytest

import paper_2509_05165_amd as kv
from cache_testlib import Device, dev, empty_cache, params, random_cache, rounded, stream, workspace
from oracle import cache_oracle as orc

pytestmark = pytest.mark.gpu
FORMATS = [orc.E4M3, orc.INT8]


def rows_of(rng, layers, hkv, total, d, dtype):
    """Rows whose size varies by token, with values at the formats' ties and a few zeros."""
    x = rng.standard_normal((layers, hkv, total, d)) * 2.0 ** rng.integers(-4, 5, (layers, hkv, total, 1))
    x[rng.random(x.shape) < 0.05] = 0
    x[rng.random(x.shape) < 0.1] = 0.40625           # a tie of e4m3 and, for many scales, of int8
    return rounded(x, dtype)


def fill_case(rng, fmt, dtype, lens, kept, layers, hkv, d, unstructured=False, order=0, with_idx=True, scores=True,
              weighted=True, offset=0):
    """lens: tokens per sequence; kept: tokens per row."""
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    total = int(cu[-1])
    c = empty_cache(rng, fmt, [-(-n // 64) for n in kept], hkv, d, layers, unstructured=unstructured)
    k, v = (rows_of(rng, layers, hkv, total, d, dtype) for _ in "kv")
    idx = np.concatenate([np.argsort(rng.random((layers, hkv, n)), axis=-1) for n in lens], axis=-1).astype(np.int32)
    s = rng.random((layers, hkv, total)).astype(np.float32)
    device = Device(c, weighted)
    # rows that start `offset` elements into their allocations
    def place(x):
        flat = dev(np.concatenate([np.zeros(offset), x.ravel()]), dtype)
        return flat, flat.data_ptr() + offset * flat.element_size()
    tensors = [place(x) for x in list(k) + list(v)]
    lengths = dev(np.asarray(kept, np.int32))
    offsets = dev(np.concatenate([[0], np.cumsum(kept)]).astype(np.int64))
    p = params(c, len(lens), hkv, dtype, window=16, order=order)
    ws = workspace(kv.kvc_workspace_size(p, total, max(lens)))
    t_idx, t_s = dev(idx), dev(s)
    kv.kvc_cache_fill(p, [a for _, a in tensors[:layers]], [a for _, a in tensors[layers:]],
                      t_idx.data_ptr() if with_idx else 0, lengths.data_ptr(), offsets.data_ptr(), cu, int(sum(kept)),
                      device.struct, stream(), scores=t_s.data_ptr() if scores and weighted else 0,
                      workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    if not with_idx:
        idx = None
    elif order == kv.KVC_ORDER_POSITION:
        for row, hh, b, l, h in c.heads():
            part = idx[l, h, cu[b]:cu[b] + kept[row]]
            idx[l, h, cu[b]:cu[b] + kept[row]] = np.sort(part)
    orc.fill(c, k, v, idx, kept, cu, s if scores else None, weighted)
    device.same(c)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [16, 64, 80, 128, 192, 256])
def test_fill_head_sizes(fmt, dtype, d):
    rng = np.random.default_rng([1, d, fmt])
    fill_case(rng, fmt, dtype, [150, 64], [1, 130, 64, 63], 2, 3, d)


@pytest.mark.parametrize("lens,kept", [
    ([1], [1]), ([0, 5], [0, 5]), ([64], [64]), ([65, 63], [65, 62]), ([300, 0, 20], [0, 0, 7]), ([1000], [129]),
    ([100] * 70, list(range(30, 100)))])               # more rows than a wave probes at once
@pytest.mark.parametrize("fmt", FORMATS)
def test_fill_lengths(fmt, lens, kept):
    rng = np.random.default_rng([2, len(lens), fmt])
    fill_case(rng, fmt, "bf16", lens, kept, 1, 2, 32)


@pytest.mark.parametrize("how", [dict(order=kv.KVC_ORDER_POSITION), dict(with_idx=False), dict(scores=False),
                                 dict(weighted=False), dict(offset=1), dict(offset=3, dtype="f32"),
                                 dict(unstructured=True), dict(unstructured=True, order=kv.KVC_ORDER_POSITION)])
def test_fill_variants(how):
    rng = np.random.default_rng(3)
    how = dict(how)
    dtype = how.pop("dtype", "bf16")
    kept = [40, 70, 3, 65, 0, 90, 64, 12] if how.get("unstructured") else [70, 90]
    fill_case(rng, orc.E4M3, dtype, [90] if not how.get("unstructured") else [100], kept if how.get("unstructured") else kept,
              2, 4 if how.get("unstructured") else 2, 48, **how)


def test_fill_tiny_and_huge_values():
    rng = np.random.default_rng(4)
    for size in (0.0, 1e-37, 2.0 ** -100, 1e30, 3e38):
        c = empty_cache(rng, orc.INT8, [1], 1, 16, 1)
        x = rng.uniform(-1, 1, (1, 1, 20, 16)) * size
        x = x.astype(np.float32).astype(np.float64)
        device, t = Device(c), dev(x, "f32")
        lengths, offsets = dev(np.array([20], np.int32)), dev(np.array([0, 20], np.int64))
        kv.kvc_cache_fill(params(c, 1, 1, "f32"), [t.data_ptr()], [t.data_ptr()], 0, lengths.data_ptr(),
                          offsets.data_ptr(), [0, 20], 20, device.struct, stream())
        orc.fill(c, x, x, None, [20], [0, 20])
        device.same(c)


def test_fill_leaves_out_blocks_that_are_not_there():
    rng = np.random.default_rng(5)
    c = empty_cache(rng, orc.E4M3, [3], 2, 32, 1)
    c.table[0, 1] = -5
    x = rows_of(rng, 1, 2, 170, 32, "bf16")
    device, t = Device(c), dev(x, "bf16")
    lengths, offsets = dev(np.array([170], np.int32)), dev(np.array([0, 170], np.int64))
    kv.kvc_cache_fill(params(c, 1, 2, "bf16"), [t.data_ptr()], [t.data_ptr()], 0, lengths.data_ptr(), offsets.data_ptr(),
                      [0, 170], 170, device.struct, stream())
    orc.fill(c, x, x, None, [170], [0, 170])
    device.same(c)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,d", [(1, 128), (3, 80), (64, 16), (65, 64), (150, 256)])
def test_append(fmt, dtype, window, d):
    """Into rows of every fill level; the new tokens are larger than what is there in some heads."""
    rng = np.random.default_rng([6, fmt, window])
    lens = [window, window + 1, 64, 65, 127, 128, 200, 0, max(window - 1, 0), 333]
    c = random_cache(rng, fmt, [max(0, n) for n in lens], 3, d, 1)
    device = Device(c)
    k, v = (rounded(rng.standard_normal((len(lens), 3, window, d)) * 2.0 ** rng.integers(-5, 6, (len(lens), 3, 1, 1)), dtype)
            for _ in "kv")
    tk, tv, lengths = dev(k, dtype), dev(v, dtype), dev(np.asarray(lens, np.int32))
    p = params(c, len(lens), 3, dtype, window=window)
    orc.append(c, 0, k, v, lens)
    for again in range(2):                            # a repeated call changes nothing
        kv.kvc_cache_append(p, 0, tk.data_ptr(), tv.data_ptr(), lengths.data_ptr(), device.struct, stream())
        device.same(c)


def test_append_layers_heads_and_tables():
    """One layer of several, every head with a row of its own; a row that is full, one of an unknown block, rows of
    lengths that no row has."""
    rng = np.random.default_rng(7)
    for unstructured in (False, True):
        per = 2 if unstructured else 1
        lens = list(rng.integers(1, 150, 3 * 2 * per))
        c = random_cache(rng, orc.E4M3, lens, 2, 32, 2, unstructured=unstructured, width=3)
        lens[per] = 193                               # beyond the table: takes nothing
        lens[3 * per] = -7
        c.table[5 * per, :] = c.table.max() + 9
        device = Device(c, weighted=False)
        k, v = (rounded(rng.standard_normal((3, 2, 2, 32)) * 9, "bf16") for _ in "kv")
        tk, tv, lengths = dev(k, "bf16"), dev(v, "bf16"), dev(np.asarray(lens, np.int32))
        kv.kvc_cache_append(params(c, 3, 4, "bf16", window=2), 1, tk.data_ptr(), tv.data_ptr(), lengths.data_ptr(),
                            device.struct, stream())
        orc.append(c, 1, k, v, lens, weighted=False)
        device.same(c)


def test_append_token_by_token_over_block_ends():
    rng = np.random.default_rng(8)
    c = empty_cache(rng, orc.INT8, [3], 2, 48, 1)
    device = Device(c)
    for n in list(range(1, 70)) + [128, 129]:
        if n == 128:                                  # the slots in between stay what they are
            c.k_scale[c.table[0, 1]] = c.v_scale[c.table[0, 1]] = 0.25
            device = Device(c)
        k, v = (rounded(rng.standard_normal((1, 2, 1, 48)) * 1.1 ** n, "bf16") for _ in "kv")
        tk, tv, lengths = dev(k, "bf16"), dev(v, "bf16"), dev(np.array([n], np.int32))
        if n >= 128:                                  # what is rescaled has to be numbers
            c.k[c.table[0, 1]] = 5
            c.v[c.table[0, 1]] = 251
            device = Device(c)
        kv.kvc_cache_append(params(c, 1, 2, "bf16"), 0, tk.data_ptr(), tv.data_ptr(), lengths.data_ptr(), device.struct, stream())
        orc.append(c, 0, k, v, [n])
    device.same(c)


@pytest.mark.parametrize("seed", range(25))
def test_random_fills(seed):
    rng = np.random.default_rng([31, seed])
    layers, hkv, d = int(rng.integers(1, 5)), int(rng.integers(1, 5)), 16 * int(rng.integers(1, 17))
    unstructured = bool(rng.integers(0, 2))
    lens = [int(x) for x in rng.integers(1, 300, int(rng.integers(1, 5)))]
    per = layers * (hkv if unstructured else 1)
    kept = [int(rng.integers(0, n + 1)) for n in lens for _ in range(per)]
    fill_case(rng, int(rng.integers(0, 2)), str(rng.choice(["bf16", "f32"])), lens, kept, layers, hkv, d, unstructured,
              order=int(rng.integers(0, 2)), scores=bool(rng.integers(0, 2)), offset=int(rng.integers(0, 8)))


@pytest.mark.parametrize("seed", range(25))
def test_random_appends(seed):
    """Steps of any number of tokens one after the other, each of another size."""
    rng = np.random.default_rng([32, seed])
    hkv, d, fmt, dtype = int(rng.integers(1, 4)), 16 * int(rng.integers(1, 17)), int(rng.integers(0, 2)), str(rng.choice(["bf16", "f32"]))
    batch = int(rng.integers(1, 5))
    c = empty_cache(rng, fmt, [5] * batch, hkv, d, 1, width=5)
    device, lens = Device(c), np.zeros(batch, np.int32)
    for _ in range(6):
        m = int(rng.integers(1, 50))
        lens = lens + rng.integers(0, m + 1, batch).astype(np.int32)   # some rows take only the last of the m
        k, v = (rounded(rng.standard_normal((batch, hkv, m, d)) * 2.0 ** rng.integers(-6, 7), dtype) for _ in "kv")
        tk, tv, t_len = dev(k, dtype), dev(v, dtype), dev(lens)
        kv.kvc_cache_append(params(c, batch, hkv, dtype, window=m), 0, tk.data_ptr(), tv.data_ptr(), t_len.data_ptr(),
                            device.struct, stream())
        orc.append(c, 0, k, v, lens)
    device.same(c)
