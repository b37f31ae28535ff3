"""The cache in 4 bits and the bounded cache where they went wrong before: long runs of tiles under a maximum that stays, block ends beside
the appended row, elements next to a border, queries and scales far from one, calls from two threads, heads that keep fewer rows than are protected."""
import ctypes
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


# ------------------------------------------------------------------------------------------------- borders
def border_groups(dtype):
    """Groups [n, 32] whose (step, mid) are a power of two and a multiple of it, with elements on the borders, next to them, and next to 0, which
    is a border: as near as the type goes."""
    groups, pars = [], []
    for e in (-3, 20, 110, -110, -60):
        step = 2.0 ** e
        for j in range(-7, 8):
            x = [(j - 7.5) * step, (j + 7.5) * step]
            for tiny in (2.0 ** (e - 20), 2.0 ** (e - 34), 2.0 ** (e - 60), 2.0 ** max(e - 100, -126), 2.0 ** -126):
                x += [tiny, -tiny] if 2.0 ** -126 <= tiny < step else []
            x += [0.0, -0.0, 2.0 ** -133, -2.0 ** -133]
            near = torch.tensor([(j + i) * step for i in (-6, -3, -1, 1, 2, 5)]).to(DT[dtype])
            for way in (math.inf, -math.inf):
                x += torch.nextafter(near, torch.full_like(near, way)).double().tolist()
            x = torch.tensor((x + [j * step] * 32)[:32], dtype=torch.float64)
            groups.append(x.to(DT[dtype]))
            assert torch.equal(groups[-1].double(), x.to(torch.float32).double())  # nothing of them was rounded
            pars.append((step, j * step))
    return torch.stack(groups), pars


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_elements_next_to_a_border_get_the_code_of_the_formula(dtype, d):
    """floor((x - mid) / step) in rational numbers, for compacted rows and for appended ones."""
    groups, pars = border_groups(dtype)
    rows = groups.view(-1, d) if len(groups) * 32 % d == 0 else torch.cat((groups, groups[:1].expand(-len(groups) % (d // 32), 32))).view(-1, d)
    pars += pars[:1] * (rows.numel() // 32 - len(pars))
    want = np.array([[min(15, max(0, math.floor((Fraction(x) - Fraction(m)) / Fraction(s)) + 8)) for x in g]
                     for g, (s, m) in zip(rows.view(-1, 32).double().tolist(), pars)]).reshape(rows.shape)
    n = len(rows)
    par = np.array(pars).reshape(n, d // 32, 2)
    k, v = rows, rows.flip(0)
    # compacted
    cfg = config(dtype, 1, 1, 1, 1, d, n, new=1)
    cache = Cache(cfg, [n])
    cache.kept_idx[:n] = torch.arange(n, dtype=torch.int32, device="cuda")
    for a in cache.arrays:
        a.zero_()
    mk.madakv_compact_quant(cfg, k.view(1, 1, 1, n, d).cuda(), v.contiguous().view(1, 1, 1, n, d).cuda(), cache.kept_idx, cache.seg_off,
                            cache.kept_len, *cache.arrays, cache.ws)
    # appended, one to each of n segments
    cfg = config(dtype, 1, n, 1, 1, d, 4, new=1)
    grown = Cache(cfg, [2] * n)
    grown.decode(grown.step(0)[0], k.reshape(1, n, 1, d), v.reshape(1, n, 1, d))
    at = torch.arange(n, device="cuda") * 3 + 2
    for c, where in ((cache, torch.arange(n, device="cuda")), (grown, at)):
        assert mk.madakv_poll_status(c.ws) == 0
        for i, (code, p) in ((0, (want, par)), (2, (want[::-1], par[::-1]))):
            assert np.array_equal(c.arrays[i + 1][where].double().cpu().numpy(), p)
            got = nibbles(c.arrays[i][where].cpu().numpy(), d)
            assert np.array_equal(got, code), np.argwhere(got != code)[:5]


# ------------------------------------------------------------------------------------------------- queries and scales
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_exp,k_exp,v_exp", [(0, 0, 0), (-60, 60, 0), (-80, 78, 0), (-96, 97, 97), (60, -60, -60), (90, -90, 97), (3, -3, -120)])
def test_queries_keys_and_values_far_from_one(dtype, d, q_exp, k_exp, v_exp):
    """The same numbers times powers of two: as right as without, up to 2^100 in the cache."""
    lens = [40, 1, 700, 129]
    cfg = config(dtype, 1, 2, 6, 2, d, 1024)
    cache = Cache(cfg, lens)
    for i, e in ((1, k_exp), (3, v_exp)):
        cache.arrays[i].mul_(2.0 ** e)
    q, _, _ = cache.step(0, False)
    q = q * 2.0 ** q_exp
    out, lse = cache.decode(q, None, None, track=(cache.acc, cache.scratch))
    k, v, spread = cache.contents()
    assert np.abs(k).max() < 2.0 ** 100 and np.abs(v).max() < 2.0 ** 100
    qs, out, lse = (t.double().cpu().numpy().reshape(4, 3, -1) for t in (q, out, lse))
    for u, n in enumerate(lens):
        a = int(cache.off[u])
        # weights times step are made of bf16 numbers, whose least is 2^-133: the last one is off by up to 2^-134, under 7.5 at most
        check_attention(dtype, qs[u], k[a:a + n], v[a:a + n], spread[a:a + n], d ** -0.5, out[u], lse[u, :, 0], least=n * 2.0 ** -131)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [0.02, 1.0, 3.5, 1e-30, 1e-37, 1e-42])
def test_softmax_scale(dtype, d, scale):
    """Scales other than 1 / sqrt(d), several KV heads, appended rows and tracking; the smallest make all weights alike."""
    lens = [40, 0, 700, 129, 33, 2000]
    cfg = config(dtype, 1, 2, 15, 3, d, 2048, softmax_scale=scale)
    cache = Cache(cfg, lens)
    q, kn, vn = cache.step(0)
    acc = cache.acc.double().cpu().numpy()
    out, lse = cache.decode(q, kn, vn, track=(cache.acc, cache.scratch))
    assert mk.madakv_poll_status(cache.ws) == 0
    k, v, spread = cache.contents()
    qs, out, lse = (t.double().cpu().numpy().reshape(6, 5, -1) for t in (q, out, lse))
    scale = float(np.float32(scale))
    for u, n in enumerate(lens):
        a, n = int(cache.off[u]), n + 1
        w = check_attention(dtype, qs[u], k[a:a + n], v[a:a + n], spread[a:a + n], scale, out[u], lse[u, :, 0])
        old = acc[a:a + n].copy()
        old[-1] = 0.0
        want = old + w.sum(0)
        logit = 2 * ((d + 8) * 2.0 ** -24 * (np.abs(qs[u]) @ np.abs(k[a:a + n]).T).max() * scale + 2.0 ** -20)
        assert np.all(np.abs(cache.acc[a:a + n].double().cpu().numpy() - want) <= logit * w.sum(0) + 7 * 2.0 ** -24 * want + 1e-38)  # (weights below 2^-126 are 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,g", [("bf16", 3), ("bf16", 12), ("f32", 3)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[40, 700], [9000, 1]])
def test_queries_that_are_not_numbers(dtype, g, d, lens):
    """A head with an infinite or missing query element gets NaN in out and lse and adds no weight; the heads beside it stay as they are."""
    cfg = config(dtype, 1, 2, g, 1, d, 9100)
    cache = Cache(cfg, lens)
    q, _, _ = cache.step(0, False)
    for i, odd in enumerate((float("nan"), float("inf"), float("-inf"))):
        results = []
        for head in (None, i):
            x = q.clone()
            if head is not None:
                x[0, :, head, 5 * i + 1] = odd
            acc = torch.zeros_like(cache.acc)
            results.append((*cache.decode(x, None, None, track=(acc, cache.scratch)), acc))
        (a, la, wa), (b, lb, wb) = results
        others = [h for h in range(g) if h != i]
        assert b[0, :, i].isnan().all() and lb[0, :, i].isnan().all()
        assert torch.equal(a[0, :, others], b[0, :, others]) and torch.equal(la[0, :, others], lb[0, :, others])
        for u, n in enumerate(lens):
            at = int(cache.off[u])
            assert abs(float(wb[at:at + n].double().sum()) - (g - 1)) <= 1e-3 and not wb[at:at + n].isnan().any()
    assert mk.madakv_poll_status(cache.ws) == 0


# ------------------------------------------------------------------------------------------------- host side
@pytest.mark.gpu
def test_evictions_of_two_configs_from_two_threads():
    """A call on a long config needs more shared memory than one on a short one; neither may take away what the other has asked for."""
    work = []
    for n in (5000, 1 << 20):
        cfg = mk.make_config(torch.bfloat16, 1, 1, 1, 1, 64, n, 8, max_new_tokens=8)
        t = dict(dtype=torch.bfloat16, device="cuda")
        cap = n + 8
        work.append((cfg, torch.tensor([n], dtype=torch.int32, device="cuda"), torch.zeros(cap, device="cuda"),
                     torch.zeros(cap, dtype=torch.int32, device="cuda"), torch.tensor([0, cap], device="cuda"),
                     torch.tensor([100], dtype=torch.int32, device="cuda"), torch.zeros((cap, 64), **t), torch.zeros((cap, 64), **t),
                     mk.new_workspace(cfg)))
    torch.cuda.synchronize()
    errors = []

    def calls(cfg, limit, acc, idx, seg_off, kept_len, k, v, ws):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20000):
                try:
                    mk.madakv_evict(cfg, -1, limit, 0, acc, idx, seg_off, kept_len, k, v, ws)
                except mk.MadakvError as e:
                    errors.append(e.code)

    threads = [threading.Thread(target=calls, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, (len(errors), set(errors))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,layers,Hq,Hkv,n,w", [("bf16", 16, 4, 4, 2000, 32), ("bf16", 2, 28, 4, 5000, 32), ("f32", 1, 4, 4, 2000, 32)])
def test_first_call_of_a_thread_scores_as_any_other(dtype, layers, Hq, Hkv, n, w):
    """A host thread whose first CUDA call it is gets the same kernels, and the same bits."""
    cfg = mk.make_config(DT[dtype], 1, layers, Hq, Hkv, 128, n, w)
    gen = torch.Generator(device="cuda").manual_seed(layers)
    q = torch.randn((1, layers, Hq, w, 128), generator=gen, device="cuda").to(DT[dtype])
    k = torch.randn((1, layers, Hkv, n, 128), generator=gen, device="cuda").to(DT[dtype])
    seq_len, ws = torch.tensor([n], dtype=torch.int32, device="cuda"), mk.new_workspace(cfg)
    psi = [torch.empty((1, layers, Hkv, n), device="cuda") for _ in range(2)]
    mk.madakv_score(cfg, q, k, seq_len, None, psi[0], ws)
    torch.cuda.synchronize()
    rc = []
    ptrs = [ctypes.c_void_p(t.data_ptr()) for t in (q, k, seq_len, psi[1], ws)]
    strides = [mk.MadakvStrides(*t.stride()[:4]) for t in (q, k)]

    def call():
        rc.append(mk.lib().madakv_score(ctypes.byref(cfg), ptrs[0], strides[0], ptrs[1], strides[1], ptrs[2], None, ptrs[3], ptrs[4], ws.numel(), None))

    t = threading.Thread(target=call)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert rc == [mk.OK] and torch.equal(psi[0], psi[1])


@pytest.mark.gpu
def test_scores_of_two_configs_from_two_threads():
    """Clusters of 8 blocks and of 2 of one kernel, with shared memory for the exchange among as many: every call as if it were alone."""
    work = []
    for layers in (1, 16):
        cfg = mk.make_config(torch.bfloat16, 1, layers, 4, 4, 128, 2000, 32)
        gen = torch.Generator(device="cuda").manual_seed(layers)
        q, k = (torch.randn((1, layers, 4, n, 128), generator=gen, device="cuda").bfloat16() for n in (32, 2000))
        psi = torch.empty((1, layers, 4, 2000), device="cuda")
        work.append((cfg, q, k, torch.tensor([2000], dtype=torch.int32, device="cuda"), None, psi, mk.new_workspace(cfg)))
        mk.madakv_score(*work[-1])
    torch.cuda.synchronize()
    alone = [w[5].clone() for w in work]
    errors, differ = [], []

    def calls(want, cfg, q, k, seq_len, lse, psi, ws):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(3000):
                try:
                    mk.madakv_score(cfg, q, k, seq_len, lse, psi, ws)
                    differ.append((psi != want).any())
                except mk.MadakvError as e:
                    errors.append(e.code)
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=calls, args=(a, *w)) for a, w in zip(alone, work)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, (len(errors), set(errors))
    assert not torch.stack(differ).any(), int(torch.stack(differ).sum())


@pytest.mark.gpu
def test_integers_beyond_32_bits_are_refused():
    cfg = config("bf16", 1, 1, 1, 1, 64, 64)
    cache = Cache(cfg, [40])
    limit = torch.tensor([10], dtype=torch.int32, device="cuda")
    for layer, recent in ((-1, 1 << 32), (-1, (1 << 31)), (1 << 32, 0), (-1 - (1 << 32), 0)):
        with pytest.raises(OverflowError):
            mk.madakv_evict_quant(cfg, layer, limit, recent, cache.acc, cache.kept_idx, cache.seg_off, cache.kept_len, *cache.arrays, cache.ws)
    assert cache.kept_len.tolist() == [40]


def readme_generation():
    text = open(os.path.join(ROOT, "README.md")).read()
    block = text.split("A generation on a cache in 4 bits", 1)[1].split("```", 2)[1]
    assert "run_decode" in block and "run_trim" in block
    return block


@pytest.mark.gpu
@pytest.mark.parametrize("new", [33, 48, 64])
def test_the_generation_in_the_readme(new):
    """It runs as printed, for hundreds of steps, with heads that keep fewer rows than the trims protect: no new token is refused."""
    cfg = config("bf16", 2, 2, 4, 2, 64, 400, new=new)
    q_win, k, v, mask, seq_len, budget = prompt(cfg, 1)
    budget.fill_(5)  # every head keeps few rows
    gen = torch.Generator().manual_seed(0)
    shape = lambda h: torch.randn((2, 2, h, 64), generator=gen).bfloat16().cuda()  # noqa: E731
    names = dict(binding=mk, cfg=cfg, capacity_rows=8 * (400 + new), q_win=q_win, k=k, v=v, mask=mask, seq_len=seq_len, budget=budget, steps=300,
                 q=shape(4), k_new=shape(2), v_new=shape(2), position=seq_len)
    exec(readme_generation(), names)
    buf = names["buf"]
    assert mk.madakv_poll_status(buf.ws) == 0
    off, lens = buf.seg_off.tolist(), buf.kept_len.tolist()
    assert min(names["limit"].view(-1).tolist()) < 32
    for u in range(8):  # the newest tokens are there
        newest = int(seq_len[u // 4]) + 299
        assert set(range(newest - 31, newest + 1)) <= set(buf.kept_idx[off[u]:off[u] + lens[u]].tolist())


def test_trim_without_tracking_is_refused():
    cfg = config("bf16", 1, 1, 1, 1, 64, 64)
    for quant in (False, True):
        buf = mk.EvictionBuffers(cfg, 80, device="cpu", quant=quant)
        with pytest.raises(ValueError):
            buf.run_trim(torch.tensor([10], dtype=torch.int32))


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [False, True])
def test_trim_protects_no_rows_whose_positions_were_not_given(quant):
    cfg = config("bf16", 1, 1, 2, 2, 64, 200, new=6)
    buf = mk.EvictionBuffers(cfg, 2 * 206, quant=quant, track=True)
    given = prompt(cfg, 2)
    buf.run_eviction(*given)
    limit = buf.kept_len.clone()
    gen = torch.Generator().manual_seed(0)
    q, kn, vn = (torch.randn((1, 1, 2, 64), generator=gen).bfloat16().cuda() for _ in range(3))
    position = torch.tensor([200], dtype=torch.int32, device="cuda")
    buf.run_decode(q, kn, vn, position=position)
    buf.run_decode(q)  # (appends nothing)
    buf.run_trim(limit, recent=1)
    assert torch.equal(buf.kept_len, limit)
    buf.run_decode(q, kn, vn)
    with pytest.raises(ValueError):
        buf.run_trim(limit, recent=1)
    assert torch.equal(buf.kept_len, limit + 1)
    buf.run_trim(limit)
    assert torch.equal(buf.kept_len, limit)
    buf.run_eviction(*given)  # positions are known again
    buf.run_decode(q, kn, vn, position=position)
    buf.run_trim(limit, recent=1)
    assert torch.equal(buf.kept_len, limit) and mk.madakv_poll_status(buf.ws) == 0
