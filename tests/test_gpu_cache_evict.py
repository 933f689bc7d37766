"""kvc_cache_evict against the oracle, bit for bit."""
import numpy as np
import pytest

import paper_2509_05165_amd as kv
from cache_testlib import Device, dev, params, random_cache, stream, workspace
from oracle import cache_oracle as orc

pytestmark = pytest.mark.gpu
FORMATS = [orc.E4M3, orc.INT8]


def check(rng, c, lens, keep, max_keep=None, first=0, last=0, lose=None):
    """A second table of blocks at the end of the pools takes what is kept."""
    rows, width = c.table.shape
    most = min(max(max(keep), 0), width * 64) if max_keep is None else max_keep
    blocks, extra = len(c.k), rows * -(-max(most, 1) // 64)
    for n in ("k", "v", "k_scale", "v_scale", "weight"):
        a = getattr(c, n)
        setattr(c, n, np.concatenate([a, a[rng.integers(0, blocks, extra)]]))
    table = np.full((rows, width), -3, np.int32)
    table[:, :-(-max(most, 1) // 64)] = blocks + rng.permutation(extra).reshape(rows, -1)
    if lose:
        table[lose] = -1
    device = Device(c)
    t_len, t_keep, t_table = dev(np.asarray(lens, np.int32)), dev(np.asarray(keep, np.int32)), dev(table)
    out = dev(np.full(rows, 77, np.int32))
    batch = rows // (c.layers * (c.hkv if c.unstructured else 1))
    p = params(c, batch, c.hkv, "bf16", keep_first=first, keep_last=last)
    size = kv.kvc_cache_evict_workspace(p, most)
    ws = workspace(size)
    kv.kvc_cache_evict(p, t_len.data_ptr(), t_keep.data_ptr(), most, device.struct, t_table.data_ptr(), out.data_ptr(),
                       ws.data_ptr(), size, stream())
    want = orc.evict(c, lens, keep, table, most, first, last)
    np.testing.assert_array_equal(out.cpu().numpy(), want)
    device.same(c)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [16, 64, 80, 128, 192, 256])
def test_head_sizes(fmt, d):
    rng = np.random.default_rng([20, fmt, d])
    check(rng, random_cache(rng, fmt, [200, 130], 3, d, 1), [200, 130], [100, 65], first=2, last=9)


@pytest.mark.parametrize("lens,keep", [
    ([1], [1]), ([1], [0]), ([0, 64], [5, 64]), ([300], [299]), ([300], [1]), ([300, 100], [64, 1000]), ([129, 2], [128, -4]),
    ([5000], [64]), ([20000], [150])])
@pytest.mark.parametrize("last", [0, 3])
def test_lengths(lens, keep, last):
    rng = np.random.default_rng([21, lens[0], keep[0] + 10])
    check(rng, random_cache(rng, orc.INT8, lens, 2, 16, 1), lens, keep, last=last)


@pytest.mark.parametrize("n", [3000, 40000, 70000])    # weights in registers, and read again in every pass
def test_equal_weights_stay_from_the_front(n):
    rng = np.random.default_rng([22, n])
    c = random_cache(rng, orc.E4M3, [n], 1, 16, 1)
    c.weight[:] = rng.choice(np.array([0.0, -0.0, 0.25, 0.5], np.float32), c.weight.shape)
    for keep in (n // 3, n // 2 + 1, 100):
        check(rng, c, [n], [keep], first=1)
        c = random_cache(rng, orc.E4M3, [n], 1, 16, 1)
        c.weight[:] = 0.5


def test_weights_of_any_size_and_sign():
    rng = np.random.default_rng(23)
    c = random_cache(rng, orc.E4M3, [900], 2, 16, 1)
    w = rng.standard_normal(c.weight.shape) * 10.0 ** rng.integers(-40, 38, c.weight.shape)
    c.weight[:] = w.astype(np.float32)
    c.weight[c.table[0, 2], 0, :5] = np.inf           # beside forced tokens, which count the same
    check(rng, c, [900], [300], first=3, last=3)


@pytest.mark.parametrize("first,last,keep", [(4, 32, 100), (200, 0, 100), (0, 200, 100), (1000, 1000, 100), (60, 60, 100)])
def test_forced_tokens(first, last, keep):
    rng = np.random.default_rng([24, first, last])
    check(rng, random_cache(rng, orc.INT8, [150, 90], 2, 32, 1), [150, 90], [keep, keep], first=first, last=last)


def test_layers_heads_and_bounds():
    rng = np.random.default_rng(25)
    lens = list(rng.integers(0, 250, 2 * 3))
    check(rng, random_cache(rng, orc.E4M3, lens, 2, 32, 3), lens, list(rng.integers(0, 200, 6)), max_keep=120)
    lens = list(rng.integers(0, 250, 2 * 2 * 3))
    check(rng, random_cache(rng, orc.E4M3, lens, 3, 32, 2, unstructured=True), lens, list(rng.integers(0, 200, 12)))


def test_blocks_that_are_not_there():
    """Tokens of a source entry that names no block go first and become zeros if they stay; a target entry that
    names none is left out."""
    rng = np.random.default_rng(26)
    c = random_cache(rng, orc.E4M3, [300, 200], 2, 32, 1)
    c.table[0, 1] = -1
    c.table[1, 2] = 1 << 30
    check(rng, c, [300, 200], [290, 100], lose=(1, 1))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [64, 128, 1088])
def test_kept_tokens_up_to_the_end_of_a_block(fmt, n):
    """The last tokens of a full block stay, and so few of the others go that they end anywhere in a word."""
    rng = np.random.default_rng([28, n, fmt])
    for lost in (1, 2, 3, 5, 30, 62, 63):
        check(rng, random_cache(rng, fmt, [n], 2, 128, 1), [n], [n - lost], last=8)


def test_scales_far_apart():
    """Rows of 2^-90 and 2^60 in one cache, rows of zeros under a large scale."""
    rng = np.random.default_rng(27)
    c = random_cache(rng, orc.INT8, [256], 1, 16, 1)
    for j, e in enumerate((-90, 60, -100, 110)):
        i = c.table[0, j]
        c.k_scale[i] = c.v_scale[i] = np.float32(2.0 ** e)
        c.k[i, 0, ::2] = 0
        c.v[i, 0, :, ::2] = 0
        c.weight[i, 0, ::2] = 1.0 + j % 2
    check(rng, c, [256], [128])


@pytest.mark.parametrize("seed", range(40))
def test_random_caches(seed):
    """Shapes, lengths, shares and weights of every kind; weights rise or fall along the row, so that what stays lies
    in runs."""
    rng = np.random.default_rng([29, seed])
    layers, hkv, d = int(rng.integers(1, 4)), int(rng.integers(1, 5)), 16 * int(rng.integers(1, 17))
    unstructured = bool(rng.integers(0, 2))
    rows = int(rng.integers(1, 4)) * layers * (hkv if unstructured else 1)
    most = int(rng.choice([70, 200, 700, 1500]))
    lens = [int(x) for x in rng.integers(0, most, rows)]
    c = random_cache(rng, int(rng.integers(0, 2)), lens, hkv, d, layers, unstructured=unstructured)
    slope = rng.choice([-1.0, 0.0, 1.0])
    for row, hh, *_ in c.heads():
        for j in range(-(-lens[row] // 64)):
            n = min(64, lens[row] - 64 * j)
            c.weight[c.table[row, j], hh, :n] += np.float32(slope) * (64 * j + np.arange(n, dtype=np.float32)) / 64
            if rng.random() < 0.3:
                c.weight[c.table[row, j], hh, :n] = np.float32(rng.integers(0, 3))
    keep = [int(round(n * s)) for n, s in zip(lens, rng.choice([0.05, 0.5, 0.9, 0.99, 1.1], rows))]
    check(rng, c, lens, keep, first=int(rng.integers(0, 5)), last=int(rng.choice([0, 1, 16, 100])))
