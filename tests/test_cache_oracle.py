"""Pins of the block cache oracle that do not come from itself: the format's published table entries, torch's own
casts, scales worked by hand, softmax of a library, invariants of eviction."""
import numpy as np
import pytest
import torch

from cache_testlib import random_cache
from oracle import cache_oracle as orc


def test_e4m3_numbers():
    v = orc.VALUES[orc.E4M3]
    assert v[0x7E] == 448 and v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and v[0x38] == 1 and v[0xB8] == -1
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF])
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(v, t)


@pytest.mark.parametrize("fmt", [orc.E4M3, orc.INT8])
def test_encode_is_the_nearest_number_halves_to_even(fmt):
    v = orc.VALUES[fmt]
    v = np.unique(v[np.isfinite(v) & (np.abs(v) <= orc.TOP[fmt])])
    mid = (v[1:] + v[:-1]) / 2
    for x in (v, mid, mid * (1 + 1e-9), mid * (1 - 1e-9), np.random.default_rng(1).uniform(-440, 440, 4000) * orc.TOP[fmt] / 448):
        got = orc.decode(orc.encode(x, fmt), fmt)
        if fmt == orc.E4M3:
            want = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
            keep = x.astype(np.float32) == x
            np.testing.assert_array_equal(got[keep], want[keep])
        else:
            np.testing.assert_array_equal(got, np.round(x))
        assert (np.abs(got - x) <= np.abs(v[None, :] - x[:, None]).min(axis=1)).all()


def test_scales_by_hand():
    for fmt, top in ((orc.E4M3, 448.0), (orc.INT8, 127.0)):
        assert orc.scale_of(top, fmt) == 1 and orc.scale_of(np.nextafter(top, 1e9), fmt) == 2
        assert orc.scale_of(top / 2, fmt) == 0.5 and orc.scale_of(0, fmt) == 2.0 ** -100
        assert orc.scale_of(1e-36, fmt) == 2.0 ** -100
    assert orc.scale_of(1.0, orc.INT8) == 2.0 ** -6 and orc.scale_of(1.0, orc.E4M3) == 2.0 ** -8


@pytest.mark.parametrize("fmt", [orc.E4M3, orc.INT8])
def test_attention_is_a_library_softmax(fmt):
    rng = np.random.default_rng(3)
    c = random_cache(rng, fmt, [130, 7], 2, 16, 1)
    q = rng.standard_normal((2, 4, 3, 16))
    out, lse, got, _, _ = orc.attend(c, 0, q, [130, 7], 0.25, causal=True)
    for b, n in ((0, 130), (1, 7)):
        for g in range(4):
            k, v, _, there = c.tokens(b, g // 2, n)
            assert there.all()
            s = torch.from_numpy(k @ q[b, g].T * 0.25).T
            s = s.masked_fill(torch.arange(n)[None] > n - 3 + torch.arange(3)[:, None], -np.inf)
            np.testing.assert_allclose(out[b, g], (torch.softmax(s, -1) @ torch.from_numpy(v)).numpy(), atol=1e-13)
            np.testing.assert_allclose(lse[b, g], torch.logsumexp(s, -1).numpy(), atol=1e-13)
    assert np.isclose(sum(x.sum() for x in got.values()), 2 * 4 * 3)          # every query's probabilities add to 1


def test_append_token_by_token_holds_what_fill_holds():
    """Rows of one magnitude need no rescaling: appended one by one they are the codes of a fill."""
    rng = np.random.default_rng(4)
    x = rng.uniform(1.0, 1.7, (1, 1, 70, 16)) * rng.choice([-1, 1], (1, 1, 70, 16))
    x[..., 0] = 1.7
    filled = orc.Cache(orc.INT8, 4, 1, 16, [[2, 0, 3]], 1)
    orc.fill(filled, x, x, None, [70], [0, 70])
    grown = orc.Cache(orc.INT8, 4, 1, 16, [[2, 0, 3]], 1)
    for t in range(70):
        orc.append(grown, 0, x[:, :, t:t + 1], x[:, :, t:t + 1], [t + 1])
    for i, n in ((2, 64), (0, 6)):
        np.testing.assert_array_equal(grown.k[i, 0, :n], filled.k[i, 0, :n])
        np.testing.assert_array_equal(grown.v[i, 0, :, :n], filled.v[i, 0, :, :n])
        assert grown.k_scale[i, 0] == filled.k_scale[i, 0]


def test_eviction_by_hand():
    c = orc.Cache(orc.INT8, 3, 1, 16, [[0, 1]], 1)
    x = np.arange(1, 7, dtype=np.float64)[:, None] * np.ones(16)
    c.put(0, 0, x, -x, np.array([.1, .5, .2, .5, .5, .0], np.float32))
    n = orc.evict(c, [6], [4], [[2, 1]], 64, keep_last=1)
    assert n.tolist() == [4]
    # the last token is forced, then the three of 0.5
    np.testing.assert_array_equal(orc.decode(c.k[2, 0, :5, 0], orc.INT8) * c.k_scale[2, 0], [2, 4, 5, 6, 0])
    np.testing.assert_array_equal(orc.decode(c.v[2, 0, 3, :5], orc.INT8) * c.v_scale[2, 0], [-2, -4, -5, -6, 0])
    np.testing.assert_array_equal(c.weight[2, 0, :5], np.array([.5, .5, .5, 0, 0], np.float32))


@pytest.mark.parametrize("most", [1, 40, 93, 95, 97, 100, 130])
def test_a_causal_tail_stays_where_the_length_puts_it(most):
    """Query m sees the first length - M + 1 + m tokens, of which those below max_length are read."""
    rng = np.random.default_rng(5)
    c = random_cache(rng, orc.INT8, [100], 1, 16, 1)
    q = rng.standard_normal((1, 1, 6, 16))
    out, lse, got, _, _ = orc.attend(c, 0, q, [100], 0.25, causal=True, max_length=most)
    k, v, _, _ = c.tokens(0, 0, 100)
    gathered = np.zeros(min(100, most))
    for m in range(6):
        n = min(100 - 6 + 1 + m, most)
        s = torch.from_numpy(k[:n] @ q[0, 0, m] * 0.25)
        p = torch.softmax(s, 0).numpy()
        np.testing.assert_allclose(out[0, 0, m], p @ v[:n], atol=1e-13)
        np.testing.assert_allclose(lse[0, 0, m], torch.logsumexp(s, 0).numpy(), atol=1e-13)
        gathered[:n] += p
    np.testing.assert_allclose(got[0, 0], gathered, atol=1e-13)
