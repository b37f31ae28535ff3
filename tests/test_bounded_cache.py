"""The ragged cache in 4 bits, decode steps that accumulate attention weight, and eviction by it, against plain restatements in 64
bits (numpy and torch on the CPU, written from the formulas in the header). What is stored, kept, moved or counted has to be
equal; tolerances of attention are sums of the roundings that the header names."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2506_15724_b200 import binding as mk

FAKE = ctypes.c_void_p(0x10000)  # aligned, never dereferenced: every refusal below comes before a launch
ODD = ctypes.c_void_p(0x10004)
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step of rounding, relative


def config(dtype="bf16", B=1, L=1, Hq=4, Hkv=4, d=128, n=512, new=4, **kw):
    return mk.make_config(DT[dtype], B, L, Hq, Hkv, d, n, 8, max_new_tokens=new, **kw)


# ------------------------------------------------------------------------------------------------- the formulas, in 64 bits
def quantise(x):
    """Codes [rows, d] and (step, mid) [rows, d / 32, 2] as float64, of float64 rows that hold values of the case's type."""
    g = x.reshape(x.shape[0], x.shape[1] // 32, 32)
    with np.errstate(all="ignore"):
        lo, hi = g.min(2), g.max(2)  # (NaN if there is one)
        mid, step = (torch.from_numpy(y).float().bfloat16().double().numpy() for y in ((lo + hi) / 2, (hi - lo) / 15))
        bad = ~(np.isfinite(mid) & np.isfinite(step))
        mid, step = np.where(bad, np.nan, mid), np.where(bad, np.nan, step)
        t = np.floor((g - mid[..., None]) / step[..., None]) + 8
    code = np.where(step[..., None] > 0, np.clip(t, 0, 15), 8).astype(np.int64)
    return code.reshape(x.shape), np.stack((step, mid), 2)


def values(code, par):
    return (par[..., 1:] + (code.reshape(*par.shape[:2], 32) - 7.5) * par[..., :1]).reshape(code.shape)


def nibbles(packed, d):
    """Codes [rows, d] of packed rows [rows, d / 2]."""
    words = packed.astype(np.int64).reshape(-1, d // 4, 2)
    words = words[..., 0] + 256 * words[..., 1]
    e = np.arange(d)
    G, i, nib = e // 32, e % 32 // 4, e % 4
    return words[:, i * (d // 32) + G] >> (4 * nib) & 15


def decoded(code, par, d):
    """Values [rows, d] of a cache's codes and parameters, as they lie on the GPU."""
    return values(nibbles(code.cpu().numpy(), d), par.double().cpu().numpy())


def attend(q, k, v, scale):
    """out [g, d], lse [g], weights [g, rows] in 64 bits."""
    if not len(k):
        return np.zeros_like(q), np.full(len(q), -np.inf), np.zeros((len(q), 0))
    s = q @ k.T * scale
    m = s.max(1, keepdims=True)
    p = np.exp(s - m)
    return p @ v / p.sum(1, keepdims=True), (m + np.log(p.sum(1, keepdims=True)))[:, 0], p / p.sum(1, keepdims=True)


def check_attention(dtype, q, k, v, spread, scale, out, lse):
    """One unit's out and lse. Roundings: logits of d products in fp32 (d + 8 half steps of the products' sum of magnitudes, in both
    the weight and the denominator); bf16: weights times the cells' step rounded before the product with the codes (`spread`, the
    values' distance from mid, times half a step), the result rounded once."""
    want, want_lse, w = attend(q, k, v, scale)
    if not len(k):
        assert not out.any() and np.all(np.isneginf(lse))
        return w
    logit = (q.shape[1] + 8) * 2.0 ** -24 * (np.abs(q) @ np.abs(k).T).max(1, keepdims=True) * scale + 2.0 ** -21
    rounded = HALF[dtype] * (w @ np.abs(spread)) if dtype == "bf16" else 0.0
    most = HALF[dtype] * np.abs(want) + rounded + (2 * logit + (64 + len(k)) ** 0.5 * 2.0 ** -22) * (w @ np.abs(v))
    assert np.all(np.abs(out - want) <= most), float((np.abs(out - want) / most).max())
    assert np.all(np.abs(lse - want_lse) <= logit[:, 0] + 2.0 ** -22 * np.maximum(1.0, np.abs(want_lse)))
    return w


def trimmed(acc, pos, length, limit, recent):
    """(new length, source of every row below it) of one segment."""
    acc, pos = acc[:length].astype(np.float64), pos[:length].astype(np.int64)
    limit = max(0, int(limit))
    if length <= limit:
        return length, np.arange(length)
    safe = pos > pos.max() - recent
    c = max(limit, int(safe.sum()))
    if c >= length:
        return length, np.arange(length)
    weight = np.where(acc > 0, acc, 0.0)  # (NaN is not > 0)
    best = np.sort(np.lexsort((np.arange(length), -weight, ~safe))[:c])
    source = np.arange(c)
    source[np.setdiff1d(np.arange(c), best)] = best[best >= c]
    return c, source


# ------------------------------------------------------------------------------------------------- refusals, on the host
@pytest.fixture(scope="module")
def lib():
    from paper_2506_15724_b200 import build

    build.build()
    return mk.lib()


def test_refusals_before_any_launch(lib):
    c = config()
    need = mk.madakv_workspace_bytes(c)
    st = mk.MadakvStrides(4 * 512 * 128, 4 * 512 * 128, 512 * 128, 128)
    ref = ctypes.byref(c)

    def compact(cfg=ref, k=FAKE, strides=st, idx=FAKE, code=FAKE, par=FAKE, cap=10, ws=FAKE, size=need):
        return lib.madakv_compact_quant(cfg, k, FAKE, strides, idx, FAKE, FAKE, FAKE, FAKE, code, par, cap, ws, size, None)

    assert compact(k=None) == compact(idx=None) == compact(code=None) == compact(par=None) == compact(ws=None) == mk.EINVAL
    assert compact(k=ODD) == compact(code=ODD) == compact(par=ctypes.c_void_p(0x10008)) == mk.EALIGN
    assert compact(strides=mk.MadakvStrides(1, 1, 1, 128)) == compact(ws=ctypes.c_void_p(0x10010)) == mk.EALIGN
    assert compact(cap=0) == mk.ECAPACITY and compact(size=need - 1) == mk.EWORKSPACE
    assert compact(cfg=ctypes.byref(config(d=96))) == mk.EUNSUPPORTED

    def expand(rows=FAKE, n=3, code=FAKE, out=FAKE, cap=10):
        return lib.madakv_expand_quant(ref, rows, n, code, FAKE, FAKE, FAKE, cap, FAKE, out, None)

    assert expand(code=None) == expand(out=None) == mk.EINVAL
    assert expand(n=-1) == mk.ESHAPE and expand(cap=0) == expand(rows=None, n=11) == mk.ECAPACITY
    assert expand(rows=ODD) == expand(out=ODD) == mk.EALIGN
    assert expand(n=0) == mk.OK

    def quant(layer=-1, q=FAKE, k_new=FAKE, v_new=FAKE, par=FAKE, cap=10, acc=None, scratch=None, idx=None, pos=None, decay=1.0,
              ws=FAKE, size=need, cfg=ref):
        return lib.madakv_decode_attn_quant(cfg, layer, q, k_new, v_new, FAKE, par, FAKE, FAKE, FAKE, FAKE, cap, FAKE, None, acc,
                                            scratch, idx, pos, decay, ws, size, None)

    def track(layer=-1, q=FAKE, v_new=FAKE, cap=10, acc=FAKE, scratch=FAKE, idx=FAKE, pos=FAKE, decay=1.0, ws=FAKE, size=need, cfg=ref):
        return lib.madakv_decode_attn_track(cfg, layer, q, FAKE, v_new, FAKE, FAKE, FAKE, FAKE, cap, FAKE, None, acc, scratch, idx,
                                            pos, decay, ws, size, None)

    for f in (quant, track):
        assert f(q=None) == f(v_new=None) == f(ws=None) == mk.EINVAL
        assert f(layer=1) == f(layer=-2) == mk.ESHAPE and f(cap=0) == mk.ECAPACITY and f(size=need - 1) == mk.EWORKSPACE
        assert f(acc=FAKE, scratch=None) == f(acc=FAKE, scratch=FAKE, idx=FAKE, pos=None) == mk.EINVAL
        for decay in (-0.1, 1.1, float("nan")):
            assert f(acc=FAKE, scratch=FAKE, decay=decay) == mk.EINVAL
        assert f(acc=FAKE, scratch=ODD) == f(acc=ctypes.c_void_p(0x10002), scratch=FAKE) == mk.EALIGN
    assert track(acc=None, scratch=None) == mk.EINVAL
    assert quant(scratch=FAKE) == quant(idx=FAKE, pos=FAKE) == mk.EINVAL and quant(par=ODD) == mk.EALIGN
    # more query heads per KV head than the kernels hold: refused before the append
    for dtype, Hq in (("bf16", 17), ("f32", 9)):
        wide = config(dtype, Hq=Hq, Hkv=1)
        size = mk.madakv_workspace_bytes(wide)
        assert quant(cfg=ctypes.byref(wide), size=size) == track(cfg=ctypes.byref(wide), size=size) == mk.EUNSUPPORTED

    def evict(layer=-1, limit=FAKE, recent=0, acc=FAKE, idx=FAKE, cap=10, k=FAKE, ws=FAKE, size=need, cfg=ref):
        return lib.madakv_evict(cfg, layer, limit, recent, acc, idx, FAKE, FAKE, cap, k, FAKE, ws, size, None)

    def evict_quant(layer=-1, limit=FAKE, recent=0, acc=FAKE, idx=FAKE, cap=10, k=FAKE, ws=FAKE, size=need, cfg=ref):
        return lib.madakv_evict_quant(cfg, layer, limit, recent, acc, idx, FAKE, FAKE, cap, k, FAKE, FAKE, FAKE, ws, size, None)

    long = config(n=1 << 20, new=(1 << 19) + 1)
    for f in (evict, evict_quant):
        assert f(limit=None) == f(acc=None) == f(idx=None) == f(k=None) == f(recent=-1) == f(ws=None) == mk.EINVAL
        assert f(layer=1) == mk.ESHAPE and f(cap=0) == mk.ECAPACITY and f(size=need - 1) == mk.EWORKSPACE
        assert f(k=ODD) == f(limit=ctypes.c_void_p(0x10001)) == mk.EALIGN
        assert f(cfg=ctypes.byref(long), size=mk.madakv_workspace_bytes(long)) == mk.EUNSUPPORTED
        assert f(cfg=ctypes.byref(config(d=96))) == mk.EUNSUPPORTED


# ------------------------------------------------------------------------------------------------- GPU: plumbing
class Cache:
    """A ragged cache of given lengths on the GPU, headroom behind every segment."""

    def __init__(self, cfg, lens, seed=0, quant=True, extra=0):
        self.cfg, self.lens, self.d = cfg, np.asarray(lens, np.int64), cfg.head_dim
        self.dtype = {mk.MADAKV_F32: "f32", mk.MADAKV_BF16: "bf16"}[cfg.dtype]
        self.off = np.concatenate([[0], np.cumsum(self.lens + cfg.max_new_tokens)])
        self.cap = int(self.off[-1]) + extra
        gen = torch.Generator().manual_seed(seed)
        self.k, self.v = (torch.randn((self.cap, self.d), generator=gen).to(DT[self.dtype]) for _ in range(2))
        self.seg_off, self.kept_len = torch.from_numpy(self.off).cuda(), torch.from_numpy(self.lens.astype(np.int32)).cuda()
        self.kept_idx = torch.full((self.cap,), -7, dtype=torch.int32)
        for a, n in zip(self.off, self.lens):
            self.kept_idx[a:a + n] = torch.sort(torch.randperm(int(cfg.max_seq_len), generator=gen)[:n])[0].int()
        self.kept_idx = self.kept_idx.cuda()
        self.acc = torch.exp(torch.randn(self.cap, generator=gen)).cuda()
        self.scratch = torch.zeros((self.cap, cfg.n_q_heads // cfg.n_kv_heads), device="cuda")
        self.ws = mk.new_workspace(cfg)
        self.shape = (cfg.batch, cfg.n_layers, cfg.n_q_heads, cfg.head_dim)
        if quant:
            code, par = zip(*(quantise(x.double().numpy()) for x in (self.k, self.v)))
            self.arrays = []
            for c, p in zip(code, par):
                e = c.reshape(self.cap, -1, 8, 2, 2).transpose(0, 2, 1, 3, 4)
                packed = (e[..., 0] | e[..., 1] << 4).reshape(self.cap, -1).astype(np.uint8)
                assert np.array_equal(nibbles(packed, self.d), c)
                self.arrays += [torch.from_numpy(packed).cuda(), torch.from_numpy(p).to(torch.bfloat16).cuda()]
        else:
            self.arrays = [self.k.cuda(), self.v.cuda()]
        self.quant = quant

    def contents(self):
        """K and V rows in 64 bits, and V's distance from its groups' mid."""
        if self.quant:
            k, v = (decoded(*self.arrays[i:i + 2], self.d) for i in (0, 2))
            return k, v, v - np.repeat(self.arrays[3].double().cpu().numpy()[..., 1], 32, 1)
        k, v = (a.double().cpu().numpy() for a in self.arrays)
        return k, v, v

    def step(self, seed, append=True):
        gen = torch.Generator().manual_seed(1000 + seed)
        c = self.cfg
        q = torch.randn(self.shape, generator=gen).to(DT[self.dtype])
        kn, vn = (torch.randn((c.batch, c.n_layers, c.n_kv_heads, self.d), generator=gen).to(DT[self.dtype]) for _ in range(2))
        return q, kn if append else None, vn if append else None

    def decode(self, q, kn, vn, layer=-1, track=(), out=None, lse=None):
        out = torch.full(self.shape, 9.0, dtype=DT[self.dtype], device="cuda") if out is None else out
        lse = torch.full(self.shape[:3], 9.0, device="cuda") if lse is None else lse
        call = mk.madakv_decode_attn_quant if self.quant else mk.madakv_decode_attn_track if track else mk.madakv_decode_attn
        q, kn, vn = (None if t is None else t.cuda() for t in (q, kn, vn))
        call(self.cfg, layer, q, kn, vn, *self.arrays, self.seg_off, self.kept_len, out, lse, self.ws, *track)
        return out, lse

    def tracking(self, position, decay):
        return self.acc, self.scratch, self.kept_idx, position, decay


# ------------------------------------------------------------------------------------------------- GPU: 4 bits
def crafted(rows, d, gen):
    """Rows whose groups are where the quantiser can go wrong."""
    x = torch.randn((rows, d), generator=gen)
    x[1 % rows] = 0.0
    x[2 % rows] = -3.25
    x[3 % rows, ::2] = 0.0  # half of a row at one value
    x[4 % rows] = x[4 % rows].sign() * 0.5  # two values
    x[5 % rows] *= 1e-38
    x[6 % rows] *= 3e-41
    x[7 % rows] = x[7 % rows].clamp(-1, 1) * 3.3e38
    x[8 % rows, 5] = float("inf")
    x[9 % rows, d - 1] = float("nan")
    x[10 % rows, 31], x[10 % rows, 32] = float("-inf"), float("inf")
    x[11 % rows] = 1000.0 + x[11 % rows]  # a shift that swallows the bits of the differences
    grid = torch.arange(32).float() - 15.5
    x[12 % rows] = (grid * 0.25).repeat(d // 32)  # elements on the borders between codes
    x[13 % rows] = (torch.arange(32).float() * 0.5).repeat(d // 32)
    x[14 % rows] = x[14 % rows].abs() + 1e-6
    x[15 % rows, :32] = 1e-20
    x[15 % rows, 0], x[15 % rows, 1], x[15 % rows, 2] = -1.0, 1.0, -1e-20  # elements next to mid = 0
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape,lens", [((1, 1, 1), [1]), ((1, 1, 1), [0]), ((2, 3, 2), [3, 0, 1, 40, 41, 39, 7, 8, 9, 2, 31, 17]),
                                        ((1, 2, 3), [200, 0, 199, 130, 1, 64]), ((3, 1, 1), [150, 256, 255])])
def test_compact_quant_equals_the_formula(dtype, d, shape, lens):
    B, L, H = shape
    n = 256
    cfg = config(dtype, B, L, H, H, d, n, new=3)
    gen = torch.Generator().manual_seed(sum(lens) + d)
    # tokens before heads in memory, as a model's projection leaves them, and rows behind the last token
    k, v = (crafted(B * L * (n + 5) * H, d, gen).to(DT[dtype]).view(B, L, n + 5, H, d) for _ in range(2))
    k[:, :, :, :, 3] *= 7.0
    k, v = (t.cuda().transpose(2, 3) for t in (k, v))
    cache = Cache(cfg, lens, quant=False, extra=11)
    gen2 = torch.Generator().manual_seed(5)
    arrays = [torch.randint(0, 256, (cache.cap, d // 2), generator=gen2, dtype=torch.uint8).cuda(),
              torch.randn((cache.cap, d // 32, 2), generator=gen2).bfloat16().cuda()] * 2
    arrays = [a.clone() for a in arrays]
    before = [a.clone() for a in arrays]
    mk.madakv_compact_quant(cfg, k, v, cache.kept_idx, cache.seg_off, cache.kept_len, *arrays, cache.ws)
    assert mk.madakv_poll_status(cache.ws) == 0
    idx = cache.kept_idx.cpu().numpy()
    written = np.zeros(cache.cap, bool)
    for u, rows in enumerate(lens):
        b, l, h = np.unravel_index(u, (B, L, H))
        a = int(cache.off[u])
        written[a:a + rows] = True
        for src, code, par in ((k, *arrays[:2]), (v, *arrays[2:])):
            want, want_par = quantise(src[b, l, h].double().cpu().numpy()[idx[a:a + rows]])
            assert np.array_equal(par[a:a + rows].double().cpu().numpy(), want_par, equal_nan=True)
            assert np.array_equal(nibbles(code[a:a + rows].cpu().numpy(), d), want)
    for a, b in zip(arrays, before):  # headroom and what lies behind the last segment
        rest = torch.from_numpy(~written).cuda()
        assert torch.equal(a[rest].view(torch.uint8), b[rest].view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_compact_quant_skips_what_selection_refused(d):
    """A segment that would end behind the cache with its headroom, or whose positions lie outside the prompt, is not written."""
    lens = [20, 30, 40]
    cfg = config("bf16", 1, 3, 1, 1, d, 64, new=4)
    cache = Cache(cfg, lens, quant=False)
    k, v = (torch.randn((1, 3, 1, 64, d)).bfloat16().cuda() for _ in range(2))
    cap = int(cache.off[-1]) - 1  # the last segment's headroom lacks a row
    arrays = [torch.full((cap, d // 2), 77, dtype=torch.uint8, device="cuda"), torch.full((cap, d // 32, 2), 5.0, dtype=torch.bfloat16, device="cuda")]
    arrays = [a.clone() for a in arrays * 2]
    cache.kept_idx[3], cache.kept_idx[4] = 64, -1
    mk.madakv_compact_quant(cfg, k, v, cache.kept_idx, cache.seg_off, cache.kept_len, *arrays, cache.ws)
    idx = cache.kept_idx.cpu().numpy()
    for u in range(2):
        a = int(cache.off[u])
        rows = np.array([i for i in range(a, a + lens[u]) if 0 <= idx[i] < 64])
        for src, code, par in ((k, *arrays[:2]), (v, *arrays[2:])):
            want, want_par = quantise(src[0, u, 0].double().cpu().numpy()[idx[rows]])
            assert np.array_equal(nibbles(code.cpu().numpy()[rows], d), want)
            assert np.array_equal(par.double().cpu().numpy()[rows], want_par)
    for code, par in (arrays[:2], arrays[2:]):
        for rows in (slice(3, 5), slice(20, 24), slice(int(cache.off[2]) - 4, cap)):
            assert (code[rows] == 77).all() and (par[rows] == 5.0).all()


@pytest.mark.gpu
def test_quantised_values_are_within_half_a_step():
    cfg = config("f32", n=2000, Hq=1, Hkv=1)
    cache = Cache(cfg, [2000])
    x = cache.k.double().numpy()
    got = decoded(*cache.arrays[:2], 128)
    g, par = x.reshape(len(x), -1, 32), cache.arrays[1].double().cpu().numpy()
    step = par[..., :1]
    # half a step, and at the ends what the roundings to bf16 (half a step of it each) take from mid and from 7.5 steps
    ends = HALF["bf16"] * (np.abs(par[..., 1:]) + 8 * step)
    assert np.all(np.abs(got.reshape(g.shape) - g) <= step / 2 * (1 + 1e-12) + ends)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_expand_quant_equals_the_formula(dtype, d):
    cfg = config(dtype, d=d)
    cache = Cache(cfg, [50, 0, 3, 77])
    cache.arrays[1][4] = float("nan")
    k, v, _ = cache.contents()
    lists = [np.array([0, 5, 5, cache.cap - 1, 4, 3, 60, 0]), np.array([-1, cache.cap, 1 << 40, -(1 << 62), 2]), np.zeros(0, np.int64),
             np.arange(cache.cap)[::-1].copy(), None]
    for rows in lists:
        m = cache.cap if rows is None else len(rows)
        k_out, v_out = (torch.full((m, d), 5.0, dtype=DT[dtype], device="cuda") for _ in range(2))
        mk.madakv_expand_quant(cfg, None if rows is None else torch.from_numpy(rows).cuda(), *cache.arrays, k_out, v_out)
        rows = np.arange(cache.cap) if rows is None else rows
        there = (rows >= 0) & (rows < cache.cap)
        for got, x in ((k_out, k), (v_out, v)):
            want = np.where(there[:, None], x[np.where(there, rows, 0)], 0.0)
            got = got.double().cpu().numpy()
            assert np.array_equal(np.isnan(got), np.isnan(want))
            near = np.abs(got - want) <= (HALF[dtype] + 2.0 ** -23) * np.abs(want)  # rounded to fp32, then to dtype
            assert np.all(near | np.isnan(want))


# heads per KV head of every kernel variant, lengths about the shares and tiles, segments without rows, one segment over many blocks
ATTEND = [("bf16", 128, 1, 3, [0, 1, 2000]), ("bf16", 128, 7, 4, [2048, 33, 1, 700]), ("bf16", 64, 2, 5, [15, 16, 17, 0, 513]),
          ("bf16", 64, 9, 2, [1025, 64]), ("bf16", 128, 16, 3, [129, 300, 31]), ("bf16", 128, 4, 1, [9001]), ("bf16", 64, 8, 2, [63, 65]),
          ("bf16", 128, 1, 70, [1500 - 7 * i for i in range(70)]), ("bf16", 128, 3, 1200, [i % 67 for i in range(1200)]),
          ("f32", 128, 1, 3, [0, 1, 1500]), ("f32", 64, 3, 4, [15, 16, 17, 900]), ("f32", 128, 8, 2, [257, 40]), ("f32", 64, 5, 1, [5003]),
          ("f32", 128, 2, 90, [300 + i for i in range(90)])]


def check_step(cache, dtype, step, layer, before, out, lse, kn, vn, q, track, decay, position):
    """One decode step of the units of `layer` against the formulas; `before`: lens, acc, kept_idx, contents before it."""
    lens, acc0, idx0, arrays0 = before
    k, v, spread = cache.contents()
    c = cache.cfg
    g, scale = c.n_q_heads // c.n_kv_heads, 1 / np.sqrt(cache.d)
    acc, idx = cache.acc.cpu().numpy(), cache.kept_idx.cpu().numpy()
    got_len = cache.kept_len.cpu().numpy()
    out, lse = out.double().cpu().numpy().reshape(-1, g, cache.d), lse.double().cpu().numpy().reshape(-1, g)
    qs = q.double().numpy().reshape(-1, g, cache.d)
    touched = np.zeros(cache.cap, bool)
    for u, n in enumerate(lens):
        if layer >= 0 and u // c.n_kv_heads % c.n_layers != layer:
            assert got_len[u] == n and np.all(out[u] == 9.0)
            continue
        a, n = int(cache.off[u]), int(n)
        if kn is not None:
            for x, new, i in ((k, kn, 0), (v, vn, 1)):
                new = new.double().numpy().reshape(-1, cache.d)[u:u + 1]
                if cache.quant:  # the appended row is quantised as compaction would
                    code, par = quantise(new)
                    assert np.array_equal(nibbles(cache.arrays[2 * i][a + n:a + n + 1].cpu().numpy(), cache.d), code)
                    assert np.array_equal(cache.arrays[2 * i + 1][a + n:a + n + 1].double().cpu().numpy(), par)
                else:
                    assert np.array_equal(x[a + n:a + n + 1], new)
            touched[a + n] = True
            n += 1
        assert got_len[u] == n
        w = check_attention(dtype, qs[u], k[a:a + n], v[a:a + n], spread[a:a + n], scale, out[u], lse[u])
        if track:
            old = acc0[a:a + n].astype(np.float64)
            if kn is not None:
                old[n - 1] = 0.0
                assert idx[a + n - 1] == position[u // (c.n_layers * c.n_kv_heads)]
            want = np.float64(np.float32(decay)) * old + w.sum(0)
            logit = 2 * ((cache.d + 8) * 2.0 ** -24 * (np.abs(qs[u]) @ np.abs(k[a:a + n]).T).max(initial=0) * scale + 2.0 ** -20)
            assert np.all(np.abs(acc[a:a + n] - want) <= logit * w.sum(0) + (g + 2) * 2.0 ** -24 * want + 1e-38)
            acc0[a:a + n], idx0[a:a + n] = acc[a:a + n], idx[a:a + n]
    # nothing else was written
    assert np.array_equal(acc, acc0) and np.array_equal(idx, idx0)
    rest = torch.from_numpy(~touched).cuda()
    for x, y in zip(cache.arrays, arrays0):
        assert torch.equal(x[rest], y[rest])


@pytest.mark.gpu
@pytest.mark.parametrize("quant,track", [(True, False), (True, True), (False, True)])
@pytest.mark.parametrize("dtype,d,g,units,lens", ATTEND)
def test_decode_steps_equal_the_formula(dtype, d, g, units, lens, quant, track):
    """Two appending steps and one without, on one workspace; then one layer alone."""
    B, L = (1, units) if units % 2 else (2, units // 2)
    cfg = config(dtype, B, L, g, 1, d, max(lens) + 1, new=3)
    cache = Cache(cfg, lens, seed=g, quant=quant, extra=5)
    position = np.arange(B) + 100000
    pos = torch.from_numpy(position.astype(np.int32)).cuda()
    for step, (append, layer, decay) in enumerate([(True, -1, 1.0), (True, -1, 0.75), (False, -1, 0.0), (True, L - 1, 0.5)]):
        q, kn, vn = cache.step(step, append)
        before = (cache.kept_len.cpu().numpy(), cache.acc.cpu().numpy(), cache.kept_idx.cpu().numpy(), [a.clone() for a in cache.arrays])
        out, lse = cache.decode(q, kn, vn, layer, cache.tracking(pos, decay) if track else ())
        assert mk.madakv_poll_status(cache.ws) == 0
        check_step(cache, dtype, step, layer, before, out, lse, kn, vn, q, track, decay, position)


# one block per SM for few long segments, in each number of warps that it has; one block per segment beyond the arrival counters
@pytest.mark.gpu
@pytest.mark.parametrize("track", [False, True])
@pytest.mark.parametrize("dtype,d,g,units,lens", [("bf16", 64, 3, 1, [120001]), ("bf16", 64, 11, 2, [90000, 37003]), ("f32", 64, 2, 1, [115007]),
                                                  ("bf16", 128, 1, 4, [29000, 0, 31000, 60001]), ("bf16", 64, 1, 17000, [i % 5 for i in range(17000)])])
def test_decode_on_few_long_and_on_very_many_segments(dtype, d, g, units, lens, track):
    cfg = config(dtype, 1, units, g, 1, d, max(lens) + 1, new=3)
    cache = Cache(cfg, lens, seed=g)
    pos = torch.tensor([123456], dtype=torch.int32, device="cuda")
    q, kn, vn = cache.step(7)
    before = (cache.kept_len.cpu().numpy(), cache.acc.cpu().numpy(), cache.kept_idx.cpu().numpy(), [a.clone() for a in cache.arrays])
    out, lse = cache.decode(q, kn, vn, -1, cache.tracking(pos, 0.25) if track else ())
    assert mk.madakv_poll_status(cache.ws) == 0
    check_step(cache, dtype, 7, -1, before, out, lse, kn, vn, q, track, 0.25, [123456])


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [True, False])
def test_without_decay_old_sums_do_not_matter(quant):
    lens = [700, 0, 33]
    cfg = config("bf16", 1, 3, 2, 1, 128, 1024)
    a, b = Cache(cfg, lens, quant=quant), Cache(cfg, lens, quant=quant)
    b.acc.fill_(float("nan"))
    for c in (a, b):
        c.decode(*c.step(0), track=(c.acc, c.scratch, None, None, 0.0))
    for at, n in zip(a.off, lens):
        assert torch.equal(a.acc[at:at + n + 1], b.acc[at:at + n + 1]) and not a.acc[at:at + n + 1].isnan().any()


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [True, False])
def test_calls_on_two_streams_at_once(quant):
    """Two caches with workspaces and scratch of their own, steps and evictions in flight together: the results of each alone."""
    cfg = config("bf16", 1, 16, 4, 1, 128, 4096, new=8)
    rng = np.random.RandomState(3)
    lens = [rng.randint(1, 4000, size=16), rng.randint(1, 300, size=16)]
    limit = [torch.from_numpy((n // 2).astype(np.int32)).cuda() for n in lens]
    call = mk.madakv_evict_quant if quant else mk.madakv_evict
    pos = torch.tensor([5000], dtype=torch.int32, device="cuda")
    results = []
    for together in (False, True):
        caches = [Cache(cfg, n, seed=i, quant=quant) for i, n in enumerate(lens)]
        steps = [[tuple(t.cuda() for t in c.step(s)) for s in range(6)] for c in caches]
        outs = [[torch.zeros(c.shape, dtype=torch.bfloat16, device="cuda") for _ in range(6)] for c in caches]
        lses = [[torch.zeros(c.shape[:3], device="cuda") for _ in range(6)] for c in caches]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()] if together else [torch.cuda.current_stream()] * 2
        torch.cuda.synchronize()
        for s in range(6):
            for i, c in enumerate(caches):
                with torch.cuda.stream(streams[i]):
                    c.decode(*steps[i][s], track=c.tracking(pos, 0.9), out=outs[i][s], lse=lses[i][s])
                    if s % 3 == 2:
                        call(cfg, -1, limit[i], 2, c.acc, c.kept_idx, c.seg_off, c.kept_len, *c.arrays, c.ws)
        torch.cuda.synchronize()
        for c in caches:
            assert mk.madakv_poll_status(c.ws) == 0
        results.append([t for i, c in enumerate(caches) for t in (*outs[i], *lses[i], c.kept_len, c.kept_idx, c.acc, *c.arrays)])
    for x, y in zip(*results):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.gpu
def test_tracking_where_rows_do_not_arrive(monkeypatch):
    """The copies of cache rows are withheld: the waits run out, results are NaN, sums of weights stay as they were."""
    lens = [300, 2000, 40]
    cfg = config("bf16", 1, 3, 1, 1, 128, 2048)
    cache = Cache(cfg, lens, quant=False)
    q, kn, vn = cache.step(0)
    acc = cache.acc.clone()
    monkeypatch.setenv("MADAKV_TEST_HOLD_COPIES", "200000")
    out, lse = cache.decode(q, kn, vn, track=(cache.acc, cache.scratch))
    assert mk.madakv_poll_status(cache.ws) == mk.ETIMEOUT
    monkeypatch.delenv("MADAKV_TEST_HOLD_COPIES")
    assert out.isnan().all() and lse.isnan().all()
    for a, n in zip(cache.off, lens):
        acc[int(a) + n] = 0.0  # (the appended row's)
    assert torch.equal(cache.acc, acc) and cache.kept_len.tolist() == [n + 1 for n in lens]
    out, lse = cache.decode(q, None, None, track=(cache.acc, cache.scratch))
    assert mk.madakv_poll_status(cache.ws) == 0 and not out.isnan().any() and (cache.acc > acc).any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,g,units,lens", ATTEND)
def test_tracking_changes_nothing_of_the_attention(dtype, d, g, units, lens):
    for quant in (True, False):
        cfg = config(dtype, 1, units, g, 1, d, max(lens) + 1, new=3)
        plain, tracked = Cache(cfg, lens, quant=quant), Cache(cfg, lens, quant=quant)
        for step in range(2):
            q, kn, vn = plain.step(step)
            a, b = plain.decode(q, kn, vn), tracked.decode(q, kn, vn, track=(tracked.acc, tracked.scratch))
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(plain.kept_len, tracked.kept_len)
            for x, y in zip(plain.arrays, tracked.arrays):
                assert torch.equal(x, y)
        assert torch.equal(plain.kept_idx, tracked.kept_idx)  # (no position given: not kept up)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_quant_with_infinite_and_missing_values(dtype, d):
    """Values that are not numbers reach the segment they lie in and no other; rows beside a segment may hold anything; far logits."""
    lens = [40, 100, 5, 300]
    cfg = config(dtype, 1, 4, 2, 1, d, 512)
    cache = Cache(cfg, lens)
    rest = np.ones(cache.cap, bool)
    for a, n in zip(cache.off, lens):
        rest[a:a + n] = False
    rest = torch.from_numpy(rest).cuda()
    for i in (1, 3):
        cache.arrays[i][rest] = float("nan")
    q, _, _ = cache.step(0, False)
    q[0, 1] *= 1e4  # logits thousands apart
    q[0, 3] = 0.0   # all equal
    clean = [a.clone() for a in cache.arrays]
    out, lse = cache.decode(q, None, None, track=(cache.acc, cache.scratch))
    k, v, spread = cache.contents()
    for u, n in enumerate(lens):
        a = int(cache.off[u])
        check_attention(dtype, q[0, u].double().numpy(), k[a:a + n], v[a:a + n], spread[a:a + n], d ** -0.5, out[0, u].double().cpu().numpy(),
                        lse[0, u].double().cpu().numpy())
    # a NaN key: that segment's results are NaN, its weights add nothing; a NaN value reaches its own group of columns alone
    cache.arrays[1][int(cache.off[0]) + 3] = float("nan")
    cache.arrays[3][int(cache.off[2]) + 4, 1] = float("nan")
    acc = cache.acc.clone()
    got, got_lse = cache.decode(q, None, None, track=(cache.acc, cache.scratch, None, None, 0.5))
    assert got[0, 0].isnan().all() and got_lse[0, 0].isnan().all()
    assert torch.equal(got[0, 1], out[0, 1]) and torch.equal(got[0, 3], out[0, 3])
    assert got[0, 2, :, 32:64].isnan().all()
    assert torch.equal(got[0, 2, :, :32], out[0, 2, :, :32]) and torch.equal(got[0, 2, :, 64:], out[0, 2, :, 64:])
    a, n = int(cache.off[0]), lens[0]
    assert torch.equal(cache.acc[a:a + n], 0.5 * acc[a:a + n])
    for x, y in zip(cache.arrays, clean):
        x.copy_(y)


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [True, False])
def test_segments_without_room(quant):
    """A full segment and one that the capacity cuts off: reported, left as they are; the others go on."""
    lens = [10, 20, 30, 6]
    cfg = config("bf16", 1, 4, 2, 1, 128, 64, new=2)
    cache = Cache(cfg, lens, quant=quant)
    off = cache.off.copy()
    off[1:4] = [10, 32, 64]  # the first segment's slot is full
    cache.off = off
    cache.seg_off = torch.from_numpy(off).cuda()
    cache.arrays = [a[: int(off[-1]) - 1].contiguous() for a in cache.arrays]  # the last one's slot ends behind the cache
    cache.cap = int(off[-1]) - 1
    acc, idx = cache.acc.clone(), cache.kept_idx.clone()
    arrays = [a.clone() for a in cache.arrays]
    q, kn, vn = cache.step(0)
    pos = torch.tensor([900], dtype=torch.int32, device="cuda")
    out, lse = cache.decode(q, kn, vn, track=cache.tracking(pos, 1.0))
    assert mk.madakv_poll_status(cache.ws) == mk.ECAPACITY and mk.madakv_poll_status(cache.ws) == 0
    assert cache.kept_len.tolist() == [10, 21, 31, 6]
    assert not out[0, 3].any() and lse[0, 3].isneginf().all()
    k, v, spread = cache.contents()
    for u, n in enumerate([10, 21, 31]):
        a = int(off[u])
        check_attention("bf16", q[0, u].double().numpy(), k[a:a + n], v[a:a + n], spread[a:a + n], 128 ** -0.5,
                        out[0, u].double().cpu().numpy(), lse[0, u].double().cpu().numpy())
    assert torch.equal(cache.acc[64:], acc[64:]) and torch.equal(cache.kept_idx[:10], idx[:10])
    assert (cache.acc[:10] > acc[:10]).all() and int(cache.kept_idx[30]) == 900
    for x, y in zip(cache.arrays, arrays):
        assert torch.equal(x[:10], y[:10]) and torch.equal(x[64:], y[64:])
    # eviction leaves the last one alone, too, and one that is longer than its slot
    cache.kept_len[1] = 23
    limit = torch.tensor([4, 4, 4, 2], dtype=torch.int32, device="cuda")
    call = mk.madakv_evict_quant if quant else mk.madakv_evict
    call(cfg, -1, limit, 0, cache.acc, cache.kept_idx, cache.seg_off, cache.kept_len, *cache.arrays, cache.ws)
    assert cache.kept_len.tolist() == [4, 23, 4, 6]


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [True, False])
def test_offsets_beyond_32_bits(quant):
    """Segments that lie behind 2^32 elements and bytes of the cache."""
    cfg = config("bf16", 1, 2, 2, 1, 64, 400, new=8)
    small = Cache(cfg, [300, 200], quant=quant)
    shift = (1 << 32) // (32 if quant else 64) + 12345
    arrays = [torch.empty((shift + small.cap, *a.shape[1:]), dtype=a.dtype, device="cuda") for a in small.arrays]
    for x, a in zip(arrays, small.arrays):
        x[shift:].copy_(a)
    big = Cache(cfg, [300, 200], quant=quant)
    big.arrays, big.seg_off = arrays, small.seg_off + shift
    big.acc, big.kept_idx = (torch.cat((torch.empty(shift, dtype=t.dtype, device="cuda"), t)) for t in (small.acc, small.kept_idx))
    big.scratch = torch.empty((shift + small.cap, 2), device="cuda")
    pos = torch.tensor([900], dtype=torch.int32, device="cuda")
    limit = torch.tensor([250, 190], dtype=torch.int32, device="cuda")
    got = []
    for c in (small, big):
        q, kn, vn = c.step(0)
        out = c.decode(q, kn, vn, track=c.tracking(pos, 0.5))
        call = mk.madakv_evict_quant if quant else mk.madakv_evict
        call(cfg, -1, limit, 4, c.acc, c.kept_idx, c.seg_off, c.kept_len, *c.arrays, c.ws)
        got.append((*out, c.kept_len, c.acc[-small.cap:], c.kept_idx[-small.cap:], *[a[-small.cap:] for a in c.arrays]))
        assert mk.madakv_poll_status(c.ws) == 0
    for a, b in zip(*got):
        assert torch.equal(a, b)
    if quant:
        rows = small.seg_off[:2] + 7
        outs = [tuple(torch.zeros((2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)) for _ in range(2)]
        mk.madakv_expand_quant(cfg, rows, *small.arrays, *outs[0])
        mk.madakv_expand_quant(cfg, rows + shift, *big.arrays, *outs[1])
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and outs[0][0].any()


# ------------------------------------------------------------------------------------------------- GPU: eviction
def acc_of(kind, cap, gen):
    if kind == "weights":
        return torch.exp(2 * torch.randn(cap, generator=gen))
    if kind == "equal":
        return torch.ones(cap)
    if kind == "zeros":
        return torch.zeros(cap)
    if kind == "few_values":
        return torch.randint(0, 4, (cap,), generator=gen).float() / 8
    x = torch.randn(cap, generator=gen)  # "odd": negative, NaN, infinite and subnormal sums among the others
    x[torch.randint(0, cap, (cap // 8,), generator=gen)] = float("nan")
    x[torch.randint(0, cap, (cap // 8,), generator=gen)] = float("inf")
    x[torch.randint(0, cap, (cap // 8,), generator=gen)] = 1e-42
    x[torch.randint(0, cap, (cap // 8,), generator=gen)] = -0.0
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["weights", "equal", "zeros", "few_values", "odd"])
@pytest.mark.parametrize("dtype,d,quant", [("bf16", 128, False), ("f32", 64, False), ("bf16", 64, True), ("bf16", 128, True)])
@pytest.mark.parametrize("lens,limit,recent", [
    ([1, 2, 3, 0], [0, 1, 5, 0], 0), ([33, 32, 31, 64], [32, 31, 0, 63], 1), ([700, 701, 64, 1025], [350, 700, 70, 1], 16),
    ([5000, 4999, 513, 100], [4999, 100, 512, -3], 40), ([12000, 3, 2047, 2049], [3000, 2, 2046, 1024], 2000), ([40, 40, 40, 40], [5, 10, 39, 40], 1 << 30)])
def test_evict_equals_the_rule(kind, dtype, d, quant, lens, limit, recent):
    cfg = config(dtype, 1, 4, 1, 1, d, max(lens) + 1, new=3)
    cache = Cache(cfg, lens, seed=recent % 97, quant=quant, extra=9)
    gen = torch.Generator().manual_seed(len(kind))
    cache.acc = acc_of(kind, cache.cap, gen).cuda()
    call = mk.madakv_evict_quant if quant else mk.madakv_evict
    state = [cache.acc, cache.kept_idx, *cache.arrays]
    before = [x.clone() for x in state]
    source = np.arange(cache.cap)
    want = []
    for u, n in enumerate(lens):
        a = int(cache.off[u])
        c, src = trimmed(cache.acc[a:].cpu().numpy(), cache.kept_idx[a:].cpu().numpy(), n, limit[u], recent)
        want.append(c)
        source[a:a + c] = a + src[:c]
    source = torch.from_numpy(source).cuda()
    lim = torch.tensor(limit, dtype=torch.int32, device="cuda")
    for layer in (2, -1, -1):  # one layer, all, and once more: nothing is left to do
        call(cfg, layer, lim, recent, cache.acc, cache.kept_idx, cache.seg_off, cache.kept_len, *cache.arrays, cache.ws)
        assert mk.madakv_poll_status(cache.ws) == 0
        if layer == 2:
            assert cache.kept_len.tolist() == [lens[0], lens[1], want[2], lens[3]]
            continue
        assert cache.kept_len.tolist() == want
        for x, y in zip(state, before):
            assert torch.equal(x.view(torch.uint8), y[source].view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,quant", [("bf16", 128, False), ("bf16", 64, True)])
@pytest.mark.parametrize("units,rows,longest", [(400, 300, 300), (320, 1500, 9000), (300, 1, 3), (5, 2500, 7000), (3, 9000, 30000)])
def test_evict_in_every_size_of_block(dtype, d, quant, units, rows, longest):
    """Calls of many segments, of segments that fit the registers and of longer ones beside them; half of them have rows too many."""
    rng = np.random.RandomState(units + rows)
    lens = rng.randint(rows // 2, rows + 1, size=units)
    lens[units // 2] = longest
    cfg = config(dtype, 1, units, 1, 1, d, longest + 1, new=2)
    cache = Cache(cfg, lens, seed=units, quant=quant)
    limit = np.where(rng.rand(units) < 0.5, lens - rng.randint(0, 70, size=units), rng.randint(0, rows + 1, size=units))
    state = [cache.acc, cache.kept_idx, *cache.arrays]
    before = [x.clone() for x in state]
    acc, idx = cache.acc.cpu().numpy(), cache.kept_idx.cpu().numpy()
    source, want = np.arange(cache.cap), []
    for u, n in enumerate(lens.tolist()):
        a = int(cache.off[u])
        c, src = trimmed(acc[a:a + n + 1], idx[a:a + n + 1], n, limit[u], 5)
        want.append(c)
        source[a:a + c] = a + src[:c]
    source = torch.from_numpy(source).cuda()
    call = mk.madakv_evict_quant if quant else mk.madakv_evict
    lim = torch.from_numpy(limit.astype(np.int32)).cuda()
    call(cfg, -1, lim, 5, cache.acc, cache.kept_idx, cache.seg_off, cache.kept_len, *cache.arrays, cache.ws)
    assert mk.madakv_poll_status(cache.ws) == 0 and cache.kept_len.tolist() == want
    for x, y in zip(state, before):
        assert torch.equal(x.view(torch.uint8), y[source].view(torch.uint8))


@pytest.mark.gpu
def test_evict_one_long_segment():
    n = (1 << 20) + 1000
    cfg = config("bf16", 1, 1, 1, 1, 64, 1 << 20, new=1000)
    for limit, recent in ((n - 1, 1), (n // 2, 64), (17, 0)):
        gen = torch.Generator().manual_seed(limit)
        acc = torch.exp(torch.randn(n, generator=gen)).cuda()
        idx = torch.arange(n, dtype=torch.int32, device="cuda")
        k = torch.arange(n, device="cuda").view(-1, 1).float().repeat(1, 32).view(torch.bfloat16).contiguous()  # the row's number
        v = k.clone()
        c, src = trimmed(acc.cpu().numpy(), idx.cpu().numpy(), n, limit, recent)
        kept = torch.tensor([n], dtype=torch.int32, device="cuda")
        ws = mk.new_workspace(cfg)
        want = acc[torch.from_numpy(src).cuda()]
        mk.madakv_evict(cfg, 0, torch.tensor([limit], dtype=torch.int32, device="cuda"), recent, acc, idx,
                        torch.tensor([0, n], device="cuda"), kept, k, v, ws)
        assert int(kept) == c and torch.equal(acc[:c], want)
        assert np.array_equal(idx[:c].cpu().numpy(), src)
        for x in (k, v):
            assert np.array_equal(x.view(torch.float32)[:c, 9].cpu().numpy(), src.astype(np.float32))


# ------------------------------------------------------------------------------------------------- GPU: a run of them together
def prompt(cfg, seed):
    gen = torch.Generator().manual_seed(seed)
    B, L, Hq, Hkv, d, n = cfg.batch, cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.max_seq_len
    dt = torch.float32 if cfg.dtype == mk.MADAKV_F32 else torch.bfloat16
    q = torch.randn((B, L, Hq, cfg.window, d), generator=gen).to(dt)
    k, v = (torch.randn((B, L, Hkv, n, d), generator=gen).to(dt) for _ in range(2))
    mask = (torch.rand((B, n), generator=gen) < 0.6).to(torch.uint8)
    seq_len = torch.tensor([n - 17 * b for b in range(B)], dtype=torch.int32)
    return [t.cuda() for t in (q, k, v, mask, seq_len, torch.full((B,), n // 4, dtype=torch.int32))]


@pytest.mark.gpu
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("dtype,Hq,Hkv,d", [("bf16", 4, 4, 128), ("bf16", 14, 2, 64), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("how", ["eager", "graph", "stream", "layers"])
def test_a_generation_on_a_bounded_cache(quant, dtype, Hq, Hkv, d, how):
    """Prefill eviction, then decode steps with tracking and a trim after every second one, so that no segment ever needs more than
    its headroom: twelve steps with room for three. Every step against the formulas on the state before it."""
    cfg = config(dtype, 2, 2, Hq, Hkv, d, 300, new=3)
    units, L = 2 * 2 * Hkv, 2
    buf = mk.EvictionBuffers(cfg, units * (300 + 3), quant=quant, track=True)
    buf.run_eviction(*prompt(cfg, 3))
    assert mk.madakv_poll_status(buf.ws) == 0
    limit = buf.kept_len.clone()
    assert int(limit.min()) > 0
    cache = Cache.__new__(Cache)  # the same checks on these buffers
    cache.cfg, cache.d, cache.dtype, cache.quant, cache.shape = cfg, d, dtype, quant, (2, L, Hq, d)
    cache.off, cache.cap, cache.arrays = buf.seg_off.cpu().numpy(), buf.kept_idx.numel(), list(buf.cache)
    cache.acc, cache.scratch, cache.kept_idx, cache.kept_len, cache.ws = buf.acc, buf.scratch, buf.kept_idx, buf.kept_len, buf.ws
    q, kn, vn = [t.cuda() for t in cache.step(0)]
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")

    def decode():
        for layer in range(L) if how == "layers" else (-1,):
            buf.run_decode(q, kn, vn, layer, position=pos, decay=0.9)

    def trim():
        for layer in range(L) if how == "layers" else (-1,):
            buf.run_trim(limit, recent=2, layer=layer)

    calls = [decode, trim]
    side = torch.cuda.Stream()
    if how == "graph":
        torch.cuda.synchronize()
        graphs = []
        for call in calls:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call()
            graphs.append(graph.replay)
        calls = graphs
    elif how == "stream":
        def on(call):
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                call()
            torch.cuda.current_stream().wait_stream(side)
        calls = [lambda f=f: on(f) for f in calls]
    for step in range(12):
        hq, hk, hv = cache.step(step)
        q.copy_(hq), kn.copy_(hk), vn.copy_(hv), pos.copy_(torch.tensor([300 + step, 283 + step], dtype=torch.int32))
        buf.out.fill_(9.0)
        before = (buf.kept_len.cpu().numpy(), buf.acc.cpu().numpy(), buf.kept_idx.cpu().numpy(), [a.clone() for a in buf.cache])
        calls[0]()
        assert mk.madakv_poll_status(buf.ws) == 0
        check_step(cache, dtype, step, -1, before, buf.out, buf.lse_dec, hk, hv, hq, True, 0.9, [300 + step, 283 + step])
        if step % 2:
            lens = buf.kept_len.cpu().numpy()
            state = [buf.acc, buf.kept_idx, *buf.cache]
            before = [x.clone() for x in state]
            source = np.arange(cache.cap)
            for u in range(units):
                a = int(cache.off[u])
                c, src = trimmed(buf.acc[a:].cpu().numpy(), buf.kept_idx[a:].cpu().numpy(), int(lens[u]), int(limit[u]), 2)
                assert c == int(limit[u]) or c <= 2
                source[a:a + c], lens[u] = a + src[:c], c
            calls[1]()
            assert buf.kept_len.cpu().numpy().tolist() == lens.tolist()
            source = torch.from_numpy(source).cuda()
            for x, y in zip(state, before):
                assert torch.equal(x.view(torch.uint8), y[source].view(torch.uint8))
    assert mk.madakv_poll_status(buf.ws) == 0


@pytest.mark.gpu
def test_wrong_tensors_are_refused_before_the_launch():
    cfg = config("bf16", 1, 2, 4, 2, 64, 100, new=2)
    cache = Cache(cfg, [10, 20, 30, 40])
    q, kn, vn = [t.cuda() for t in cache.step(0)]
    out, lse = torch.zeros_like(q), torch.zeros(cache.shape[:3], device="cuda")
    good = dict(q=q, kn=kn, vn=vn, arrays=cache.arrays, seg_off=cache.seg_off, kept_len=cache.kept_len, out=out, lse=lse, ws=cache.ws,
                acc=cache.acc, scratch=cache.scratch, idx=cache.kept_idx, pos=torch.zeros(1, dtype=torch.int32, device="cuda"))

    def decode(**kw):
        a = {**good, **kw}
        mk.madakv_decode_attn_quant(cfg, -1, a["q"], a["kn"], a["vn"], *a["arrays"], a["seg_off"], a["kept_len"], a["out"], a["lse"],
                                    a["ws"], a["acc"], a["scratch"], a["idx"], a["pos"])

    def evict(**kw):
        a = {**good, "limit": cache.kept_len, **kw}
        mk.madakv_evict_quant(cfg, -1, a["limit"], 0, a["acc"], a["idx"], a["seg_off"], a["kept_len"], *a["arrays"], a["ws"])

    c = cache.arrays
    both = [dict(arrays=[c[0][:-1], *c[1:]]), dict(arrays=[c[0], c[1].float(), *c[2:]]), dict(arrays=[c[0].cpu(), *c[1:]]),
            dict(arrays=[c[0].repeat(1, 2)[:, ::2], *c[1:]]), dict(seg_off=cache.seg_off[1:]), dict(seg_off=cache.seg_off.int()),
            dict(kept_len=cache.kept_len[1:]), dict(acc=cache.acc[1:]), dict(acc=cache.acc.double()), dict(idx=cache.kept_idx[1:])]
    for kw in both + [dict(q=q.float()), dict(q=q.transpose(2, 3)), dict(kn=kn[:, :1]), dict(out=out[..., :32]), dict(lse=lse[:, 1:]),
                      dict(scratch=cache.scratch[:, :1].contiguous()), dict(pos=cache.seg_off)]:
        with pytest.raises(ValueError):
            decode(**kw)
    for kw in both + [dict(limit=cache.kept_len[1:]), dict(limit=cache.kept_len.long())]:
        with pytest.raises(ValueError):
            evict(**kw)
    with pytest.raises(mk.MadakvError) as e:
        decode(ws=cache.ws[:-256])
    assert e.value.code == mk.EWORKSPACE
    torch.cuda.synchronize()
    assert cache.kept_len.tolist() == [10, 20, 30, 40] and not out.any()
