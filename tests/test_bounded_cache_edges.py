"""The cache in 4 bits and the bounded cache where they went wrong before: long runs of tiles under a maximum that stays, block ends beside
the appended row, elements next to a border, queries and scales far from one, calls from two threads, heads that keep fewer rows than are protected."""
import math
import os
import threading
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2506_15724_b200 import binding as mk
from test_bounded_cache import DT, HALF, Cache, attend, config, nibbles, prompt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def packed(code):
    """Codes [rows, d] (uint8) as they lie in the cache."""
    e = code.view(code.shape[0], -1, 8, 2, 2).transpose(1, 2)
    return (e[..., 0] | e[..., 1] << 4).reshape(code.shape[0], -1).contiguous()


def check_attention(dtype, q, k, v, spread, scale, out, lse, least=0.0):
    """One unit's out and lse: logits of d products in fp32 (d + 8 half steps of the products' sum of magnitudes, in both the weight and the
    denominator); bf16: weights times the cells' step rounded (`spread`, the values' distance from mid, times half a step), the result rounded
    once. `least`: what the type's least number takes."""
    want, want_lse, w = attend(q, k, v, scale)
    if not len(k):
        assert not out.any() and np.all(np.isneginf(lse))
        return w
    logit = (q.shape[1] + 8) * 2.0 ** -24 * (np.abs(q) @ np.abs(k).T).max(1, keepdims=True) * scale + 2.0 ** -21
    rounded = HALF[dtype] * (w @ np.abs(spread)) if dtype == "bf16" else 0.0
    most = HALF[dtype] * np.abs(want) + rounded + (2 * logit + (64 + len(k)) ** 0.5 * 2.0 ** -22) * (w @ np.abs(v)) + least
    assert np.all(np.abs(out - want) <= most), float((np.abs(out - want) / most).max())
    off = np.abs(lse - want_lse) / (logit[:, 0] + 2.0 ** -22 * np.maximum(1.0, np.abs(want_lse)))
    assert np.all(off <= 1), float(off.max())
    return w


# ------------------------------------------------------------------------------------------------- ends of blocks
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("units,longest,lens", [(1, 2304, range(1140, 1180)), (32, 4096, range(2490, 2520))])
def test_appended_row_just_behind_a_share(dtype, d, units, longest, lens):
    """A block's rows may end in the middle of a tile whose other rows, the appended one among them, are the next block's (1153 to 1168 rows in 9
    blocks, 2497 to 2512 in 13). The call before leaves NaN wherever blocks keep an appended row in shared memory."""
    many = config(dtype, 1, 1200, 1, 1, d, 8, new=50)
    poison = Cache(many, [1] * 1200)
    qp, kn, _ = poison.step(0)
    nan = torch.full_like(kn, float("nan"))
    cfg = config(dtype, 1, units, 1, 1, d, longest - 8, new=8)
    cache = Cache(cfg, [max(lens)] * units)
    q, kn, vn = (t.cuda() for t in cache.step(1))
    first = torch.arange(units, device="cuda") * (max(lens) + 8)
    bad = []
    for n in lens:
        poison.decode(qp, nan, nan)
        cache.kept_len.fill_(n)
        before = [a[first + n].clone() for a in cache.arrays]
        out, lse = cache.decode(q, kn, vn)
        if out.isnan().any() or lse.isnan().any():
            bad.append(n)
        elif n % 8 == 0:
            k, v, spread = cache.contents()
            for u in (0, units - 1):
                rows = slice(int(first[u]), int(first[u]) + n + 1)
                check_attention(dtype, q[0, u].double().cpu().numpy(), k[rows], v[rows], spread[rows], d ** -0.5,
                                out[0, u].double().cpu().numpy(), lse[0, u].double().cpu().numpy())
        for a, row in zip(cache.arrays, before):
            a[first + n] = row
    assert mk.madakv_poll_status(cache.ws) == 0 and not bad, bad
