"""kvc_cache_attend with a causal tail and a max_length below the rows' lengths."""
import numpy as np
import pytest

from cache_testlib import attend_bounds, call_attend, random_cache, rounded
from oracle import cache_oracle as orc
from test_gpu_cache_attend import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [2, 6, 9])
@pytest.mark.parametrize("most", [0, 1, 63, 64, 141, 148, 149, 150, 151, 1 << 20])
def test_max_length_about_the_tail(dtype, window, most):
    """Rows that end before, at and behind max_length, rows shorter than the tail and empty ones."""
    rng = np.random.default_rng([80, window, most])
    lens = [150, 148, 64, 3, 0, 400]
    check(rng, random_cache(rng, orc.E4M3, lens, 2, 32, 1), lens, 4, dtype, window, 1, max_length=most)


@pytest.mark.parametrize("weights", ["add", "none"])
@pytest.mark.parametrize("most", [3900, 4096, 4100, 8195])
def test_rows_that_are_split(most, weights):
    rng = np.random.default_rng([81, most])
    lens = [4100, 8200, 3903]
    check(rng, random_cache(rng, orc.INT8, lens, 1, 64, 1), lens, 3, window=8, causal=1, max_length=most, weights=weights)


def test_rows_longer_than_their_table():
    """A length beyond the table is the table's capacity, and the tail ends there."""
    rng = np.random.default_rng(82)
    c = random_cache(rng, orc.E4M3, [192, 192], 2, 64, 1, width=3)
    for most in (100, 190, 192, 1000):
        check(rng, c, [(1 << 31) - 1, 192], 4, window=5, causal=1, max_length=most)


@pytest.mark.parametrize("seed", range(40))
def test_random_calls_within_bounds(seed):
    """Shapes, tails, bounds and layers of every kind, blocks that are not there."""
    rng = np.random.default_rng([83, seed])
    layers, hkv, d = int(rng.integers(1, 3)), int(rng.integers(1, 4)), 16 * int(rng.integers(1, 17))
    unstructured, window, dtype = bool(rng.integers(0, 2)), int(rng.choice([1, 2, 5, 9, 20])), str(rng.choice(["bf16", "f32"]))
    batch = int(rng.integers(1, 4))
    rows = batch * layers * (hkv if unstructured else 1)
    lens = [int(x) for x in rng.integers(0, int(rng.choice([70, 300, 2000])), rows)]
    c = random_cache(rng, int(rng.integers(0, 2)), lens, hkv, d, layers, unstructured=unstructured)
    if rng.random() < 0.3:
        c.table[int(rng.integers(0, rows)), int(rng.integers(0, c.table.shape[1]))] = -1
    most, causal, layer = int(rng.integers(0, max(lens) + 100)), int(rng.integers(0, 2)), int(rng.integers(0, layers))
    q = rounded(rng.standard_normal((batch, hkv * int(rng.integers(1, 9)), window, d)), dtype)
    out, lse, got, mean_abs, largest = orc.attend(c, layer, q, lens, d ** -0.5, bool(causal), most)
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, dtype)
    fine = np.isfinite(lse)
    for weights in (False, True):
        mine, mine_lse, gathered = call_attend(c, q, lens, dtype, causal, max_length=most, layer=layer, weights=weights)
        assert (np.abs(mine - out) <= tol).all()
        assert (np.isneginf(mine_lse) == ~fine).all() and (np.abs(mine_lse[fine] - lse[fine]) <= tol_lse[fine]).all()
    written = np.zeros(gathered.shape, bool)
    heads = q.shape[1] // hkv * window
    for (row, hh), x in got.items():
        for j in range(-(-len(x) // 64)):
            i, part = c.block(row, j), x[64 * j:64 * j + 64]
            if i is None:
                continue
            want = c.weight[i, hh, :len(part)].astype(np.float64) + part
            bound = part * (2 * tol_lse[fine].max(initial=0) + (heads + 8) * 2.0 ** -23) + want * 2.0 ** -23 + 1e-37
            assert (np.abs(gathered[i, hh, :len(part)] - want) <= bound).all()
            written[i, hh, :len(part)] = True
    assert (gathered[~written] == 7).all()
