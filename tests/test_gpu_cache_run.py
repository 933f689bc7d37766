"""The block cache as a server uses it: a compression pass whose retained rows fill the cache, decoding steps that
append and attend layer by layer, an eviction into fresh blocks, more steps; eagerly, captured in a HIP graph, on
another stream."""
import numpy as np
import pytest
import torch

import paper_2509_05165_amd as kv
import workloads as wl
from cache_testlib import Device, attend_tolerance, dev, empty_cache, params, rounded, stream, workspace
from kvc_testlib import DeviceWorkload, Workload
from oracle import cache_oracle as orc

pytestmark = pytest.mark.gpu


def _bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x).view(np.int16)).view(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("fmt", [orc.E4M3, orc.INT8])
def test_compress_fill_decode_evict(fmt):
    rng = np.random.default_rng([30, fmt])
    cfg = wl.get_config(5, batch=2, layers=3)
    w = Workload(cfg, seed=4, lens=[500, 333])
    dw, p = DeviceWorkload(w), w.params(order=kv.KVC_ORDER_POSITION)
    layers, hkv, d, rows = 3, cfg.hkv, cfg.head_dim, 6
    S = torch.empty((layers, hkv, w.total), device="cuda")
    idx = torch.empty((layers, hkv, w.total), dtype=torch.int32, device="cuda")
    lengths = torch.empty(rows, dtype=torch.int32, device="cuda")
    offsets = torch.empty(rows + 1, dtype=torch.int64, device="cuda")
    tb = sum(w.budgets)
    k_out = torch.empty(tb * hkv * d, dtype=torch.bfloat16, device="cuda")
    v_out = torch.empty_like(k_out)
    size = kv.kvc_workspace_size(p, w.total, 500)
    ws = workspace(size)
    kv.kvc_compress(p, dw.ptrs(dw.q), dw.ptrs(dw.k), dw.ptrs(dw.v), w.cu, w.budgets, k_out.data_ptr(), v_out.data_ptr(),
                    lengths.data_ptr(), offsets.data_ptr(), ws.data_ptr(), size, stream(), scores=S.data_ptr(),
                    idx=idx.data_ptr())
    # room for every row to keep all its tokens and 100 more
    c = empty_cache(rng, fmt, [10] * rows, hkv, d, layers, width=10)
    device = Device(c)
    kv.kvc_cache_fill(p, dw.ptrs(dw.k), dw.ptrs(dw.v), idx.data_ptr(), lengths.data_ptr(), offsets.data_ptr(), w.cu, tb,
                      device.struct, stream(), scores=S.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=size)
    kept, order = lengths.cpu().numpy(), idx.cpu().numpy()
    assert kept.sum() == tb
    for row, hh, b, l, h in c.heads():
        part = order[l, h, w.cu[b]:w.cu[b] + kept[row]]
        order[l, h, w.cu[b]:w.cu[b] + kept[row]] = np.sort(part)
    k, v = (np.stack([_bf16(x) for x in y]) for y in (w.k, w.v))
    orc.fill(c, k, v, order, kept, w.cu, S.cpu().numpy())
    device.same(c)

    def steps(c, device, n, start):
        """n steps of one token, every layer appended to and attended."""
        p1 = params(c, 2, cfg.hq, "bf16")
        t_len = dev(np.asarray(start, np.int32))
        most = c.table.shape[1] * 64
        need = kv.kvc_cache_attend_workspace(p1, most, True)
        ws1 = workspace(need)
        for i in range(n):
            t_len += 1
            for l in range(layers):
                q, kn, vn = (rounded(rng.standard_normal((2, heads, 1, d)), "bf16") for heads in (cfg.hq, hkv, hkv))
                tq, tk, tv = dev(q, "bf16"), dev(kn, "bf16"), dev(vn, "bf16")
                out, weight = torch.empty_like(tq), device.t["weight"]
                kv.kvc_cache_append(p1, l, tk.data_ptr(), tv.data_ptr(), t_len.data_ptr(), device.struct, stream())
                kv.kvc_cache_attend(p1, l, tq.data_ptr(), t_len.data_ptr(), most, device.struct, out.data_ptr(), ws1.data_ptr(),
                                    need, stream(), weight_in=weight.data_ptr(), weight_out=weight.data_ptr())
                now = np.asarray(start) + i + 1
                orc.append(c, l, kn, vn, now)
                ref, _, got, mean_abs, largest = orc.attend(c, l, q, now, d ** -0.5)
                err = np.abs(out.double().cpu().numpy() - ref)
                assert (err <= attend_tolerance(c, q, mean_abs, largest, ref, "bf16")).all()
                # the gathered weights are sums of fp32 probabilities: take the library's for what follows
                mine = weight.cpu().numpy()
                for (row, hh), x in got.items():
                    for j in range(-(-len(x) // 64)):
                        i_blk, part = c.block(row, j), x[j * 64:(j + 1) * 64]
                        want = c.weight[i_blk, hh, :len(part)] + part
                        np.testing.assert_allclose(mine[i_blk, hh, :len(part)], want, rtol=1e-4, atol=1e-9)
                c.weight = mine.copy()
        device.same(c)
        return np.asarray(start) + n

    now = steps(c, device, 3, kept)
    # every row cut back to 60 %, its last 16 tokens kept, into the blocks that nobody owns yet
    blocks, extra = len(c.k), rows * 10
    for n in ("k", "v", "k_scale", "v_scale", "weight"):
        a = getattr(c, n)
        setattr(c, n, np.concatenate([a, np.zeros((extra,) + a.shape[1:], a.dtype)]))
    table = (blocks + rng.permutation(extra).reshape(rows, 10)).astype(np.int32)
    device = Device(c)
    keep = (now * 0.6).astype(np.int32)
    p2 = params(c, 2, cfg.hq, "bf16", keep_last=16)
    need = kv.kvc_cache_evict_workspace(p2, int(keep.max()))
    ws2, t_now, t_keep, t_table = workspace(need), dev(now.astype(np.int32)), dev(keep), dev(table)
    out_len = torch.empty(rows, dtype=torch.int32, device="cuda")
    kv.kvc_cache_evict(p2, t_now.data_ptr(), t_keep.data_ptr(), int(keep.max()), device.struct, t_table.data_ptr(),
                       out_len.data_ptr(), ws2.data_ptr(), need, stream())
    np.testing.assert_array_equal(orc.evict(c, now, keep, table, int(keep.max()), keep_last=16), out_len.cpu().numpy())
    device.same(c)
    c.table = table
    steps(c, Device(c), 2, out_len.cpu().numpy())


def _step(p, layers, qs, ks, vs, t_len, most, device, outs, ws, need, s):
    t_len.add_(1)
    weight = device.t["weight"].data_ptr()
    for l in range(layers):
        kv.kvc_cache_append(p, l, ks[l].data_ptr(), vs[l].data_ptr(), t_len.data_ptr(), device.struct, s)
        kv.kvc_cache_attend(p, l, qs[l].data_ptr(), t_len.data_ptr(), most, device.struct, outs[l].data_ptr(), ws.data_ptr(),
                            need, s, weight_in=weight, weight_out=weight)


def _decode_setup(seed, lens, fmt=orc.E4M3):
    from cache_testlib import random_cache
    rng = np.random.default_rng(seed)
    c = random_cache(rng, fmt, lens, 2, 64, 2, width=12)
    for r, n in enumerate(lens):                      # every row gets blocks of its own up to the table's end
        have = -(-n // 64)
        grown = len(c.k) + np.arange(12 - have)
        for name in ("k", "v", "k_scale", "v_scale", "weight"):
            a = getattr(c, name)
            setattr(c, name, np.concatenate([a, np.zeros((12 - have,) + a.shape[1:], a.dtype)]))
        c.table[r, have:] = grown
    qs = [dev(rng.standard_normal((2, 6, 1, 64)), "bf16") for _ in range(2)]
    ks, vs = ([dev(rng.standard_normal((2, 2, 1, 64)) * 3, "bf16") for _ in range(2)] for _ in "kv")
    return c, qs, ks, vs


def test_decoding_steps_replay_from_a_graph():
    """A step that raises the lengths, appends and attends, recorded once, with another graph of other rows sharing its
    workspace; replays go on where the last one stopped and equal eager steps bit for bit."""
    lens = [[100, 63, 400, 1], [65, 64, 2, 640]]
    sets = [_decode_setup(40 + i, lens[i]) for i in range(2)]
    p = params(sets[0][0], 2, 6, "bf16")
    need = kv.kvc_cache_attend_workspace(p, 768, True)
    ws = workspace(need)
    want = []
    for (c, qs, ks, vs), n in zip(sets, lens):
        device, t_len = Device(c), dev(np.asarray(n, np.int32))
        outs, seen = [torch.empty_like(q) for q in qs], []
        for _ in range(4):
            _step(p, 2, qs, ks, vs, t_len, 768, device, outs, ws, need, stream())
            torch.cuda.synchronize()
            seen.append([o.clone() for o in outs])
        want.append((seen, {k: t.clone() for k, t in device.t.items()}))
    graphs, state = [], []
    for (c, qs, ks, vs), n in zip(sets, lens):
        device, t_len = Device(c), dev(np.asarray(n, np.int32))
        outs = [torch.empty_like(q) for q in qs]
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            _step(p, 2, qs, ks, vs, t_len, 768, device, outs, ws, need, stream())
        graphs.append(g)
        state.append((device, t_len, outs))
    for i in range(4):
        for j in (0, 1):
            graphs[j].replay()
            torch.cuda.synchronize()
            for a, b in zip(state[j][2], want[j][0][i]):
                assert torch.equal(a, b), (i, j)
            ws.fill_(0x5A)                            # the workspace holds nothing that a replay relies on
    for j in (0, 1):
        for name, t in want[j][1].items():
            assert torch.equal(state[j][0].t[name].view(torch.uint8), t.view(torch.uint8)), name


def test_calls_on_another_stream():
    c, qs, ks, vs = _decode_setup(50, [100, 63, 400, 1])
    p = params(c, 2, 6, "bf16")
    need = kv.kvc_cache_attend_workspace(p, 768, True)
    got = []
    for other in (False, True):
        device, t_len, outs, ws = Device(c), dev(np.asarray([100, 63, 400, 1], np.int32)), [torch.empty_like(q) for q in qs], workspace(need)
        torch.cuda.synchronize()
        s = torch.cuda.Stream() if other else torch.cuda.current_stream()
        with torch.cuda.stream(s):
            _step(p, 2, qs, ks, vs, t_len, 768, device, outs, ws, need, s.cuda_stream)
        s.synchronize()
        got.append([o.clone() for o in outs] + [device.t["weight"].clone().nan_to_num()])
    assert all(torch.equal(a, b) for a, b in zip(*got))
