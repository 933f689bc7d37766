"""kvc_cache_attend with a causal tail and a max_length below the rows' lengths."""
import numpy as np
import pytest

from cache_testlib import random_cache
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
