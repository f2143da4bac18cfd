"""Attention where the packed rows are not all of q: a call computes the rows of its own requests and writes no others.

Bounds as for the attention's other tests, with a query's error as its four 6-bit pieces leave it: 2^-15.9 of the largest magnitude of its block of 32, taken here of its largest."""
import numpy as np
import pytest
import torch

import decoder_reference as ref
from test_gpu_cache4_attention import TYPES, Setting

pytestmark = pytest.mark.gpu


def wide(s, first, last, window):
    """(results, bounds) of the rows of requests first .. last, in 64 bits."""
    k, v = (torch.from_numpy(np.nan_to_num(ref.of_cache(c, sc))).cuda() for c, sc in zip(s.codes, s.scales))
    kv, scale = k.shape[1], s.dim ** -0.5
    outs, bounds = [], []
    for i in range(first, last):
        n, (lo, hi) = int(s.lens[i]), s.row_start[i:i + 2]
        t = torch.arange(n, device="cuda")
        pages = torch.from_numpy(s.table[i]).long().cuda()[t // s.page]
        kk, vv = (c[pages, :, t % s.page].transpose(0, 1).repeat_interleave(s.q_heads // kv, 0).contiguous() for c in (k, v))  # [heads][n][dim]
        q = s.q[lo:hi].double().transpose(0, 1).contiguous()
        p = torch.arange(n - int(hi - lo), n, device="cuda")[:, None]
        seen = (t <= p) & ((t > p - window) if window else True)
        w = torch.softmax((torch.matmul(q, kk.transpose(1, 2).contiguous()) * scale).masked_fill(~seen, -np.inf), -1)
        score = torch.matmul(q.abs(), kk.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True) * scale
        pieces = 2.0 ** -15.9 * q.abs().amax(-1, keepdim=True) * kk.abs().sum(-1).amax(-1)[:, None, None] * scale
        want, size = torch.matmul(w, vv), torch.matmul(w, vv.abs())
        _, half, weight, _ = TYPES[s.kind]
        error = (weight + 2 * (s.dim * 2.0 ** -24 * score + pieces) + 2.0 ** -15 + n * 2.0 ** -24) * size
        outs.append(want.transpose(0, 1))
        bounds.append((error + half * (want.abs() + error) + 2.0 ** -25).transpose(0, 1))
    return torch.cat(outs), torch.cat(bounds)


def check(s, first, last, window=0, told=0):
    from paper_2007_12216_amd.decoder import CacheAttention
    out = torch.full_like(s.q, 7.0)
    op = CacheAttention(s.cache, s.q_heads, window=window)
    op.forward(s.q, s.to(s.table[first:last]), s.to(s.lens[first:last]), s.to(s.row_start[first:last + 1]), max_fresh=told, out=out)
    lo, hi = s.row_start[first], s.row_start[last]
    want, bound = wide(s, first, last, window)
    assert ((out[lo:hi].double() - want).abs() <= bound).all()
    assert (out[:lo] == 7.0).all() and (out[hi:] == 7.0).all()
    return op


@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("f16", 64), ("bf16", 96), ("bf16", 128), ("f16", 128), ("bf16", 256)])
@pytest.mark.parametrize("q_heads,kv_heads", [(4, 2), (48, 16)])
@pytest.mark.parametrize("window", [0, 40])
def test_some_of_the_requests(kind, dim, q_heads, kv_heads, window):
    """Requests by their own part of row_start.  (4 and 2 heads: tiles of 16 rows; 48 and 16: of 64 or 128.)"""
    fresh = [30, 1, 200, 7, 3, 150, 60, 90, 33, 300]
    s = Setting(kind, [f + 20 * i for i, f in enumerate(fresh)], fresh, q_heads, kv_heads, dim, 16, seed=21)
    for first, last in ((1, 10), (2, 9), (5, 6), (9, 10), (0, 4)):
        check(s, first, last, window)
    check(s, 3, 5, window, told=7)


def test_some_of_the_requests_over_many_splits():
    """Few rows behind long lengths: a tile's workgroups leave parts, and there are none of the rows in front of the first request."""
    s = Setting("bf16", [60, 3000, 2500], [40, 20, 9], 4, 1, 64, 16, seed=22)
    assert check(s, 1, 3).workspace is not None
