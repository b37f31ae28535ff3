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


# ------------------------------------------------------------------------------------------------- sums over many tiles
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,g,units", [("f32", 1, 450), ("bf16", 1, 450), ("bf16", 9, 300)])
def test_sums_do_not_drift_while_the_maximum_stays(dtype, g, units):
    """One block per segment, 47 tiles for each of its warps, logits of 38 to 96 that differ by little: the sums of a tile count the same however
    many tiles come after it. All logits are exact (queries of 1, few bits in K), so what is off is what the softmax rounds.

    In units of 2^-24, the half step of fp32, relative unless said otherwise; Z is the largest logit in the log2 domain:
      a sum l of weights: 4 additions in each of 47 tiles at most, the factors of a new maximum, 3 exchanges, 4 warps: 210; ex2.approx is
        right to 2^-22: 4 for the weight and 4 for each of up to 16 new maxima; its argument, up to 8, is rounded once: 8 ln 2
      lse = (base + log2 l) ln 2, absolute: log2f (up to 13) 32, the sum, the product and ln 2 itself 3 Z ln 2; the scale in the log2 domain (log2 e,
        its product with the softmax scale) 2 Z ln 2
      acc = exp2(logit - lse2): both rounded, 2 Z ln 2; exp2f 4; the scale's error on differences of up to 5: 10
      out: numerator and denominator, and in fp32 the products' sums of 16 rows, cut and not rounded, in three terms: 32; in bf16 the weights' and
        the result's rounding"""
    d, rows, scale = 64, 6000, 0.3
    gen = torch.Generator(device="cuda").manual_seed(units)
    cfg = mk.make_config(DT[dtype], 1, units, g, 1, d, rows, 8, softmax_scale=scale)
    mid = (2 + 3 * torch.arange(units, device="cuda") / units).bfloat16()
    code = torch.randint(0, 16, (units, rows, d), generator=gen, device="cuda", dtype=torch.uint8)
    code[:, 0] = 15  # the largest logit, in the first tile
    k_code = packed(code.view(-1, d))
    k_par = torch.empty((units, rows, 2, 2), dtype=torch.bfloat16, device="cuda")
    k_par[..., 0], k_par[..., 1] = 2.0 ** -6, mid.view(-1, 1, 1)
    v_code = torch.full((units, rows, d // 2), 0xff, dtype=torch.uint8, device="cuda")
    v_code[:, rows // 2:] = 0  # 1.875 in the first half of the rows, -1.875 in the second
    v_par = torch.zeros((units, rows, 2, 2), dtype=torch.bfloat16, device="cuda")
    v_par[..., 0] = 0.25
    cache = [k_code, k_par.view(-1, 2, 2), v_code.view(-1, d // 2), v_par.view(-1, 2, 2)]
    seg_off = torch.arange(units + 1, device="cuda") * rows
    kept_len = torch.full((units,), rows, dtype=torch.int32, device="cuda")
    q = torch.ones((1, units, g, d), dtype=DT[dtype], device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, units, g), device="cuda")
    acc, scratch = torch.zeros(units * rows, device="cuda"), torch.empty((units * rows, g), device="cuda")
    ws = mk.new_workspace(cfg)
    mk.madakv_decode_attn_quant(cfg, -1, q, None, None, *cache, seg_off, kept_len, out, lse, ws, acc, scratch)
    assert mk.madakv_poll_status(ws) == 0

    logit = np.float64(np.float32(scale)) * (d * mid.double().view(-1, 1) + 2.0 ** -6 * (code.sum(2, dtype=torch.int64).double() - 7.5 * d))
    want_lse = torch.logsumexp(logit, 1, keepdim=True)
    w = torch.exp(logit - want_lse)
    half, ln2 = 2.0 ** -24, math.log(2)
    z = logit.amax(1, keepdim=True) / ln2
    l_off = (210 + 4 + 64 + 8 * ln2) * half
    off = (lse.view(units, g).double() - want_lse).abs() / (l_off + (32 + 5 * z * ln2) * half)
    assert float(off.max()) <= 1, float(off.max())
    off = (acc.view(units, rows).double() - g * w).abs() / (g * w * (l_off + (2 * z * ln2 + 32 + 14 + g) * half))
    assert float(off.max()) <= 1, float(off.max())
    want = 1.875 * (w[:, :rows // 2].sum(1) - w[:, rows // 2:].sum(1)).view(units, 1, 1)
    most = 1.875 * (2 * l_off + 42 * half)
    if dtype == "bf16":
        most = most + HALF[dtype] * (1.875 + want.abs())
    off = (out.view(units, g, d).double() - want).abs() / most
    assert float(off.max()) <= 1, float(off.max())


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
