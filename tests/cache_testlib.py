"""Helpers of the block cache tests: a random cache in NumPy, its copy on the GPU, and the comparison."""
import numpy as np
import torch

import paper_2509_05165_amd as kv
from oracle import cache_oracle as orc

GARBAGE = 0x7F        # NaN in e4m3, 127 in int8: what lies in slots and blocks that no token owns
POOLS = ("k", "v", "k_scale", "v_scale", "weight")
DTYPES = {"bf16": (torch.bfloat16, kv.KVC_BF16), "f32": (torch.float32, kv.KVC_F32)}


def rounded(x, dtype):
    """Float64 values as the type holds them."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(DTYPES[dtype][0]).double().numpy()


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t.to(DTYPES[dtype][0]) if dtype else t).cuda()


def empty_cache(rng, fmt, counts, hkv, d, layers, width=None, spare=3, unstructured=False):
    """Pools full of garbage and a table that names `counts` blocks per row in random order; behind them
    entries that name no block."""
    blocks = int(sum(counts)) + spare
    width = width or max(max(counts), 1) + 1
    order, table, at = rng.permutation(blocks), np.empty((len(counts), width), np.int32), 0
    for r, n in enumerate(counts):
        table[r] = rng.choice([-1, blocks, 1 << 30, -(1 << 31)], size=width)
        table[r, :n] = order[at:at + n]
        at += n
    return orc.Cache(fmt, blocks, hkv, d, table, layers, unstructured, fill=GARBAGE)


def random_cache(rng, fmt, lens, hkv, d, layers, unstructured=False, **kw):
    """Rows of `lens` tokens: normal values whose size differs from head to head and block to block."""
    c = empty_cache(rng, fmt, [-(-n // 64) for n in lens], hkv, d, layers, unstructured=unstructured, **kw)
    for row, hh, b, l, h in c.heads():
        for j in range(-(-lens[row] // 64)):
            n = min(64, lens[row] - 64 * j)
            i = c.table[row, j]
            size = 2.0 ** rng.integers(-3, 3)
            for name in ("k", "v"):
                x = rng.standard_normal((n, d)) * size
                s = orc.scale_of(np.abs(x).max(), fmt)
                codes = orc.encode(x / float(s), fmt)
                if name == "k":
                    c.k[i, hh, :n] = codes
                else:
                    c.v[i, hh, :, :n] = codes.T
                getattr(c, name + "_scale")[i, hh] = s
            c.weight[i, hh, :n] = rng.random(n).astype(np.float32) ** 4
    return c


class Device:
    """A cache on the GPU."""

    def __init__(self, c, weighted=True):
        self.t = {n: dev(getattr(c, n)) for n in POOLS + ("table",)}
        self.struct = kv.KvcCache(c.fmt, len(c.k), c.table.shape[1], *[self.t[n].data_ptr() for n in POOLS[:4]],
                                  self.t["weight"].data_ptr() if weighted else 0, self.t["table"].data_ptr())

    def same(self, c):
        """Every byte of the pools."""
        for n in POOLS:
            a, b = self.t[n].cpu().numpy(), getattr(c, n)
            np.testing.assert_array_equal(a.view(np.uint8), np.ascontiguousarray(b).view(np.uint8), err_msg=n)


def params(c, batch, hq, dtype, window=1, **kw):
    return kv.KvcParams(batch, c.layers, hq, c.hkv, c.d, window, DTYPES[dtype][1], unstructured=int(c.unstructured), **kw)


def workspace(size):
    return torch.full((max(size, 256),), 0xAB, dtype=torch.uint8, device="cuda")


def stream():
    return torch.cuda.current_stream().cuda_stream


def attend_tolerance(c, q, mean_abs, largest, out, dtype):
    """Largest error of one output.  A product of d terms summed in fp32 in any order is off by at most
    (d + 2) * 2^-24 of the sum of the terms' magnitudes; scaling it to log2 units, the reference's subtraction and the
    exponential's argument (up to 2 * largest * log2 e in size) round three times more, the exponential itself
    to 2 ulp.  p is off by that relatively, the sums over n tokens by n * 2^-24 at most where they are added one after the
    other; a bf16 call rounds p once to half a step, eps / 2 = 2^-8, and the output once more."""
    n = max(64, c.table.shape[1] * 64)
    rel = largest * 1.4427 * 2.0 ** -24 * (c.d + 2 + 8) + 2.0 ** -22 + 2 * n * 2.0 ** -24
    half = torch.finfo(DTYPES[dtype][0]).eps / 2
    p = half if dtype == "bf16" else 2.0 ** -23
    return mean_abs * (2 * rel[..., None] + p) * 1.01 + np.abs(out) * half + 1e-37


def attend_bounds(c, lens, mean_abs, largest, out, lse, dtype, dims=None):
    """Largest errors of the outputs and of the log-sum-exps, counted by how sums are added up: a wave adds 16
    probabilities of a block per lane and then the blocks that are its own, at most 64 of a row that one workgroup takes and 16 of
    a longer one; a product of the matrix cores adds 32 terms to its accumulator, one after the other at worst; the
    waves (4) and the splits (at most 128 in a chain) come last.  Every addition is off by a step, 2^-23, at most (the matrix
    cores need not round).  Logits are d products (`dims` of them not 0) of `terms` parts, scaled, taken from the reference and
    turned into log2 units; the exponential is within 2 ulp; probabilities of the second product are held in 16
    bits by bf16 calls, in 24 by fp32 ones.  out is rounded once, to half a step of its type."""
    u, bf16 = 2.0 ** -23, dtype == "bf16"
    terms, parts = (1, 2) if bf16 else (3, 3)
    blocks = -(-max(max(lens), 1) // 64)
    deep = min(blocks, 64) if blocks <= 256 else 16
    joins = 4 + (128 if blocks > 4 else 0)
    rel = largest * u * (terms * ((dims or c.d) + 2) + 4) + 2 * u
    sums = (16 + 2 * deep + 2 + joins) * u
    products = (deep * (2 * parts * 32 + 1) + joins) * u
    half = torch.finfo(DTYPES[dtype][0]).eps / 2
    p = 2.0 ** -16 if bf16 else 2.0 ** -24
    tol = mean_abs * (2 * rel[..., None] + sums + products + p) + np.abs(out) * half + 1e-37
    return tol, rel + sums + np.abs(np.where(np.isfinite(lse), lse, 0)) * 2 * u


def call_attend(c, q, lens, dtype, causal=0, scale=0.0, max_length=None, layer=0, weights=True):
    """out, lse and weight_out (7 where nothing is written) of one call, in float64."""
    batch, hq, window, _ = q.shape
    device, lengths, tq = Device(c), dev(np.asarray(lens, np.int32)), dev(q, dtype)
    out, lse = torch.full_like(tq, 7.0), torch.full(q.shape[:3], 7.0, device="cuda")
    gathered = torch.full(c.weight.shape, 7.0, device="cuda")
    p = params(c, batch, hq, dtype, window, causal_tail=causal, softmax_scale=scale)
    most = max(lens) if max_length is None else max_length
    size = kv.kvc_cache_attend_workspace(p, most, weights)
    ws = workspace(size)
    kv.kvc_cache_attend(p, layer, tq.data_ptr(), lengths.data_ptr(), most, device.struct, out.data_ptr(), ws.data_ptr(), size,
                        stream(), lse=lse.data_ptr(), weight_in=device.t["weight"].data_ptr() if weights else 0,
                        weight_out=gathered.data_ptr() if weights else 0)
    device.same(c)
    return tuple(x.double().cpu().numpy() for x in (out, lse, gathered))
