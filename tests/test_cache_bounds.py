"""What the error bounds of the attention tests can see: mistakes planted in the oracle lie outside them."""
import numpy as np
import pytest

from cache_testlib import attend_bounds, rounded
from oracle import cache_oracle as orc
from test_gpu_cache_precision import far_below, few_tokens, many_tokens


def bf16(x):
    return rounded(x, "bf16")


def rows_of(c, lens, q, scale, terms):
    """Attention with probabilities, in units of the largest one, held in `terms` bf16 terms for the product with V alone."""
    out, group = np.zeros(q.shape), q.shape[1] // c.hkv
    for row, hh, b, _, h in c.heads():
        k, v, _, _ = c.tokens(row, hh, lens[row])
        for g in range(h * group, (h + 1) * group):
            s = (q[b, g] @ k.T) * scale
            e = np.exp(s - s.max(axis=1, keepdims=True))
            held = bf16(e)
            held = held + bf16(e - held) if terms == 2 else held
            out[b, g] = bf16(held @ v / e.sum(axis=1, keepdims=True))
    return out


@pytest.mark.parametrize("group,window,d,fmt", [(4, 8, 64, orc.E4M3), (5, 4, 128, orc.INT8), (1, 1, 64, orc.INT8)])
def test_probabilities_of_eight_bits(group, window, d, fmt):
    c, lens, q = few_tokens(fmt, d, group, window)
    out, lse, _, mean_abs, largest = orc.attend(c, 0, q, lens, d ** -0.5)
    tol, _ = attend_bounds(c, lens, mean_abs, largest, out, lse, "bf16")
    assert (np.abs(rows_of(c, lens, q, d ** -0.5, 2) - out) <= tol).all()
    assert (np.abs(rows_of(c, lens, q, d ** -0.5, 1) - out) > tol).mean() > 0.02


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sum_without_small_probabilities(dtype):
    c, lens, q = far_below(orc.INT8, (1 << 19) - 5, -100, 0)
    q = rounded(q, dtype)
    out, lse, _, mean_abs, largest = orc.attend(c, 0, q, lens, 1.0)
    short, short_lse, _, _, _ = orc.attend(c, 0, q, [64], 1.0)               # all but the first block are missing
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, dtype)
    assert (np.abs(short_lse - lse) > 4 * tol_lse).all()
    if dtype == "f32":
        assert (np.abs(short - out) > tol)[..., 1::2].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_missing_blocks_of_a_million_tokens(dtype):
    c, lens, q = many_tokens()
    q = rounded(q, dtype)

    def run(x, n):
        return orc.attend(x, 0, q, [n], 1.0)

    def without(first, count):
        x = c.copy()
        x.table[0, first:first + count] = -1
        return run(x, lens[0])

    out, lse, got, mean_abs, largest = run(c, lens[0])
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, dtype)
    assert 0.01 < got[0, 0][-17:].sum() / 2 < 0.05
    few = 1 if dtype == "bf16" else 2                                           # blocks that the log-sum-exp shows
    for first in (0, 7777, 16382):
        assert (np.abs(without(first, few)[1] - lse) > tol_lse).all()
    for first in (0, 7200, 16344):                                              # what one workgroup takes: the outputs too
        other = without(first, 36)
        assert (np.abs(other[0] - out) > tol).mean() > 0.5 and (np.abs(other[1] - lse) > 10 * tol_lse).all()
    end = run(c, lens[0] - 17)
    assert (np.abs(end[0] - out) > tol).mean() > 0.8 and (np.abs(end[1] - lse) > 10 * tol_lse).all()
    assert (np.abs(out) > tol).mean() > 0.9                                     # all zeros


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_missing_blocks_of_an_ordinary_row(dtype):
    """Without one of its 24 blocks."""
    c, lens, q = many_tokens(1500, 0)
    q = rounded(q, dtype)
    out, lse, _, mean_abs, largest = orc.attend(c, 0, q, lens, 1.0)
    tol, tol_lse = attend_bounds(c, lens, mean_abs, largest, out, lse, dtype)
    for block in (0, 11, 22):
        x = c.copy()
        x.table[0, block] = -1
        other = orc.attend(x, 0, q, lens, 1.0)
        assert (np.abs(other[1] - lse) > 10 * tol_lse).all()
        if dtype == "f32":                                                      # (bf16: beside a step of the output)
            assert (np.abs(other[0] - out) > tol).mean() > 0.5
    assert (np.abs(out) > tol).mean() > 0.9
