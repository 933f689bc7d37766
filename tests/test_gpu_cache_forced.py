"""Forced tokens of the pass have a score of +infinity, which is their first weight in the cache."""
import numpy as np
import pytest

import paper_2509_05165_amd as kv
from cache_testlib import Device, call_attend, dev, params, random_cache, stream, workspace
from oracle import cache_oracle as orc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[300, 90], [5000, 64]])      # whole rows, and rows that are split
def test_infinite_weights_through_attention_and_eviction(lens):
    rng = np.random.default_rng([90, lens[0]])
    c = random_cache(rng, orc.INT8, lens, 2, 32, 1)
    for b, n in enumerate(lens):                               # sinks and a recent window
        for t in [0, 1, 2, 3] + list(range(n - 20, n)):
            c.weight[c.table[b, t // 64], :, t % 64] = np.inf
    q = rng.standard_normal((2, 4, 1, 32)).astype(np.float32).astype(np.float64)
    _, _, got, _, _ = orc.attend(c, 0, q, lens, 32 ** -0.5)
    _, _, gathered = call_attend(c, q, lens, "f32")
    for (row, hh), x in got.items():
        at = c.table[row, :-(-len(x) // 64)]
        was, now = (w[at, hh].ravel()[:len(x)] for w in (c.weight, gathered))
        np.testing.assert_array_equal(np.isposinf(now), np.isposinf(was))
        fine = np.isfinite(was)
        # weights below 1 and two probabilities: roundings of 2^-22 and, for logits below 8, 2^-14 of the probabilities
        assert (np.abs(now[fine] - was[fine] - x[fine]) <= 2.0 ** -22 + x[fine] * 2.0 ** -14).all()
        c.weight[at, hh] = gathered[at, hh].astype(np.float32)
    device, keep = Device(c), [40, 30]
    table = np.full(c.table.shape, -1, np.int32)
    table[:, 0] = np.setdiff1d(np.arange(len(c.k)), c.table)[:2]
    t_len, t_keep, t_table, out = dev(np.asarray(lens, np.int32)), dev(np.asarray(keep, np.int32)), dev(table), dev(np.zeros(2, np.int32))
    p = params(c, 2, 4, "f32", keep_last=8)
    ws = workspace(kv.kvc_cache_evict_workspace(p, 40))
    kv.kvc_cache_evict(p, t_len.data_ptr(), t_keep.data_ptr(), 40, device.struct, t_table.data_ptr(), out.data_ptr(), ws.data_ptr(),
                       ws.numel(), stream())
    np.testing.assert_array_equal(out.cpu().numpy(), orc.evict(c, lens, keep, table, 40, keep_last=8))
    device.same(c)
