"""Attention of prompts and of drafted trees, and the commit of an accepted path, against plain restatements in 64 bits written from the
formulas in the header. What is copied or counted has to be equal to the bit; tolerances of attention are sums of the roundings that
the header names."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2506_15724_b200 import binding as mk

FAKE = ctypes.c_void_p(0x10000)  # aligned, never dereferenced: every refusal below comes before a launch
ODD = ctypes.c_void_p(0x10004)
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step of rounding, relative
SENTINEL = 7.0


def config(dtype="bf16", B=1, L=1, Hq=4, Hkv=4, d=128, n=512, w=8, new=4, **kw):
    return mk.make_config(DT[dtype], B, L, Hq, Hkv, d, n, w, max_new_tokens=new, **kw)


def normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(DT[dtype])


# ------------------------------------------------------------------------------------------------- the formulas, in 64 bits
def attend(q, k, v, see, scale):
    """out [m, d], lse [m] and weights [m, n] of q [m, d] on k, v [n, d]; see [m, n] says who sees what. All float64."""
    z = (q @ k.T * scale).masked_fill(~see, -math.inf)
    lse = torch.logsumexp(z, 1) if k.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    w = torch.where(see, torch.exp(z - torch.where(lse.isinf(), 0.0, lse).unsqueeze(1)), 0.0)
    return w @ v, lse, w


def check(dtype, q, k, v, see, scale, out, lse, what=""):
    """Roundings: a logit is a sum of d products in fp32 (each addition off by at most a step, as the tensor core truncates: d + 8
    steps of the products' sum of magnitudes), in the weight and in the sum of weights; bf16: weights rounded before the product with
    v, the result rounded once; sums over the keys: an addition per 16 keys at most, each off by at most a step."""
    q, k, v = q.double(), k.double(), v.double()
    want, want_lse, w = attend(q, k, v, see, scale)
    out, lse = out.double(), lse.double()
    none = ~see.any(1) if k.shape[0] else torch.ones(q.shape[0], dtype=torch.bool, device=q.device)
    assert not out[none].any() and torch.all(lse[none] == -math.inf), what
    far = (w > 0).double()
    mag = (q.abs() @ k.abs().T * far).amax(1) * scale if k.shape[0] else torch.zeros_like(want_lse)
    logit = ((q.shape[1] + 8) * 2.0 ** -23 * mag + 2.0 ** -21).unsqueeze(1)
    sums = (k.shape[0] / 16 + 64) * 2.0 ** -23
    spread = w @ v.abs()
    most = HALF[dtype] * want.abs() + ((HALF[dtype] if dtype == "bf16" else 0.0) + 2 * logit + sums) * spread + 1e-30
    err = (out - want).abs()
    assert torch.all(err[~none] <= most[~none]), (what, float((err / most)[~none].max()))
    off = (lse - want_lse).abs()[~none]
    assert torch.all(off <= logit[~none, 0] + sums + 2.0 ** -22 * want_lse[~none].abs()), (what, float(off.max()))


# ------------------------------------------------------------------------------------------------- refusals, on the host
@pytest.fixture(scope="module")
def lib():
    from paper_2506_15724_b200 import build

    build.build()
    return mk.lib()


def test_prefill_refusals_before_any_launch(lib):
    c = config()
    need, st = mk.madakv_workspace_bytes(c), mk.MadakvStrides(4 * 512 * 128, 4 * 512 * 128, 512 * 128, 128)
    odd = mk.MadakvStrides(1, 1, 1, 128)

    def call(cfg=c, layer=0, q=FAKE, sq=st, rows=512, q_off=None, q_len=None, k=FAKE, sk=st, v=FAKE, sv=st, keys=512, k_off=None, seq=FAKE,
             out=FAKE, so=st, lse=None, q_win=None, lse_win=None, ws=FAKE, size=need):
        return lib.madakv_prefill_attn(ctypes.byref(cfg), layer, q, sq, rows, q_off, q_len, k, sk, v, sv, keys, k_off, seq, out, so, lse,
                                       q_win, lse_win, ws, size, None)

    assert call(q=None) == call(k=None) == call(v=None) == call(out=None) == call(ws=None) == mk.EINVAL
    assert call(seq=None) == call(k_off=FAKE) == call(q_off=FAKE, q_len=FAKE) == mk.EINVAL
    assert call(layer=-1) == call(layer=1) == call(rows=0) == call(keys=0) == mk.ESHAPE
    assert call(rows=1 << 31) == call(keys=1 << 31) == call(config(Hq=65, Hkv=1), size=1 << 40) == call(config(d=96)) == mk.EUNSUPPORTED
    assert call(q=ODD) == call(k=ODD) == call(v=ODD) == call(out=ODD) == call(q_win=ODD) == mk.EALIGN
    assert call(seq=ctypes.c_void_p(0x10002)) == call(lse=ctypes.c_void_p(0x10002)) == call(q_off=ODD) == mk.EALIGN
    assert call(sq=odd) == call(sk=odd) == call(sv=odd) == call(so=odd) == call(ws=ctypes.c_void_p(0x10010)) == mk.EALIGN
    assert call(size=need - 1) == mk.EWORKSPACE


def test_tree_refusals_before_any_launch(lib):
    c = config()
    need, st, odd = mk.madakv_workspace_bytes(c), mk.MadakvStrides(4 * 5 * 128, 4 * 5 * 128, 5 * 128, 128), mk.MadakvStrides(1, 1, 1, 128)

    def attn(cfg=c, layer=-1, nodes=5, q=FAKE, sq=st, k=FAKE, sk=st, v=FAKE, sv=st, mask=FAKE, there=None, kc=FAKE, vc=FAKE, seg=FAKE,
             kept=FAKE, cap=100, out=FAKE, so=st, lse=None, ws=FAKE, size=need):
        return lib.madakv_tree_attn(ctypes.byref(cfg), layer, nodes, q, sq, k, sk, v, sv, mask, there, kc, vc, seg, kept, cap, out, so, lse,
                                    ws, size, None)

    def commit(cfg=c, layer=-1, nodes=5, mask=FAKE, there=None, node=FAKE, k=FAKE, sk=st, v=FAKE, sv=st, kc=FAKE, vc=FAKE, seg=FAKE,
               kept=FAKE, cap=100, acc=None, idx=None, pos=None, ws=FAKE, size=need):
        return lib.madakv_tree_commit(ctypes.byref(cfg), layer, nodes, mask, there, node, k, sk, v, sv, kc, vc, seg, kept, cap, acc, idx,
                                      pos, ws, size, None)

    for call in (attn, commit):
        assert call(k=None) == call(v=None) == call(mask=None) == call(kc=None) == call(vc=None) == call(seg=None) == mk.EINVAL
        assert call(kept=None) == call(ws=None) == mk.EINVAL
        assert call(layer=-2) == call(layer=1) == call(nodes=0) == mk.ESHAPE
        assert call(nodes=65) == call(cfg=config(d=96)) == mk.EUNSUPPORTED
        assert call(cap=0) == mk.ECAPACITY and call(size=need - 1) == mk.EWORKSPACE
        assert call(k=ODD) == call(kc=ODD) == call(mask=ODD) == call(seg=ODD) == call(sk=odd) == call(sv=odd) == mk.EALIGN
    assert attn(q=None) == attn(out=None) == commit(node=None) == commit(idx=FAKE) == commit(pos=FAKE) == mk.EINVAL
    assert attn(q=ODD) == attn(sq=odd) == attn(so=odd) == commit(acc=ctypes.c_void_p(0x10002)) == mk.EALIGN
    assert attn(config(Hq=65, Hkv=1), size=1 << 40) == mk.EUNSUPPORTED


# ------------------------------------------------------------------------------------------------- prompts
def prompt(dtype, lens, Hq, Hkv, d, queries=None, q_form="padded", k_form="padded", causal=1, L=1, layer=0, w=8, fused=False, spread=1.0,
           scale=0.0, seed=0, check_all=True):
    """One call on sequences of `lens` keys (and `queries` queries); every result against the formula."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, g = len(lens), Hq // Hkv
    queries = lens if queries is None else queries
    n, m = max(max(lens), 1), max(max(queries), 1)
    cfg = config(dtype, B, L, Hq, Hkv, d, n, w, causal=causal, softmax_scale=scale)
    scale = scale or 1.0 / math.sqrt(d)

    def rows_of(form, counts, heads, most, extra):
        total = sum(counts) + extra if form == "packed" else most + extra
        if fused:
            x = normal(gen, (1 if form == "packed" else B, L, total, heads + 2, d), dtype).transpose(2, 3)[:, :, :heads]
        else:
            x = normal(gen, (1 if form == "packed" else B, L, heads, total, d), dtype)
        return x

    q = rows_of(q_form, queries, Hq, m, 3) * spread
    k, v = rows_of(k_form, lens, Hkv, n, 2), rows_of(k_form, lens, Hkv, n, 2)
    out = torch.full_like(q, SENTINEL)
    lse = torch.full(q.shape[:4], SENTINEL, device="cuda")
    q_off, k_off = (torch.from_numpy(np.concatenate([[0], np.cumsum(x)])).cuda() for x in (queries, lens))

    def part(x, form, off, counts, b):
        return x[0, layer, :, int(off[b]):int(off[b]) + counts[b]] if form == "packed" else x[b, layer, :, :counts[b]]

    # what stands behind a sequence's keys (padded), or the last one's (packed), is not a number
    if k_form == "packed":
        k[:, :, :, sum(lens):] = math.nan
        v[:, :, :, sum(lens):] = math.nan
    else:
        for b in range(B):
            k[b, :, :, lens[b]:] = math.nan
            v[b, :, :, lens[b]:] = math.nan
    q_win = torch.full((B, L, Hq, w, d), SENTINEL, device="cuda").to(DT[dtype])
    lse_win = torch.full((B, L, Hq, w), SENTINEL, device="cuda")
    ws = mk.new_workspace(cfg)
    args = {"q_off": q_off} if q_form == "packed" else {"q_len": torch.tensor(queries, dtype=torch.int32, device="cuda")}
    args.update({"k_off": k_off} if k_form == "packed" else {"seq_len": torch.tensor(lens, dtype=torch.int32, device="cuda")})
    flat = lambda x, form: x[0] if form == "packed" else x  # noqa: E731
    mk.madakv_prefill_attn(cfg, layer, flat(q, q_form), flat(k, k_form), flat(v, k_form), flat(out, q_form), ws,
                           lse_out=flat(lse, q_form), q_win=q_win, lse_win=lse_win, **args)
    assert mk.madakv_poll_status(ws) == 0
    touched = torch.zeros(q.shape[:4], dtype=torch.bool, device="cuda")
    for b in range(B):
        qb, kb, vb = part(q, q_form, q_off, queries, b), part(k, k_form, k_off, lens, b), part(v, k_form, k_off, lens, b)
        ob, yb = part(out, q_form, q_off, queries, b), part(lse, q_form, q_off, queries, b)
        part(touched, q_form, q_off, queries, b)[:] = True
        at = torch.arange(queries[b], device="cuda").view(-1, 1) + lens[b] - queries[b]
        see = torch.arange(lens[b], device="cuda") <= (at if causal else lens[b])
        see = see.expand(queries[b], lens[b]) if see.dim() == 2 else see.view(1, -1).expand(queries[b], lens[b])
        for h in range(Hq) if check_all else (0, Hq - 1):
            check(dtype, qb[h], kb[h // g], vb[h // g], see, scale, ob[h], yb[h], (b, h))
        x = min(queries[b], w)
        assert torch.equal(q_win[b, layer, :, w - x:], qb[:, queries[b] - x:]) and torch.equal(lse_win[b, layer, :, w - x:], yb[:, queries[b] - x:])
        assert not q_win[b, layer, :, :w - x].any() and torch.all(lse_win[b, layer, :, :w - x] == -math.inf)
    assert torch.all(out[~touched] == SENTINEL) and torch.all(lse[~touched] == SENTINEL)  # rows of no query, other layers
    for x in range(L):
        if x != layer:
            assert torch.all(q_win[:, x] == SENTINEL) and torch.all(lse_win[:, x] == SENTINEL)
    return out, lse


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 511, 700])
def test_prefill_lengths(dtype, n):
    prompt(dtype, [n], 4, 2, 128, seed=n)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (4, 4), (7, 1), (8, 2), (12, 1), (33, 1), (64, 1)])
def test_prefill_head_groups(dtype, d, Hq, Hkv):
    prompt(dtype, [301, 90], Hq, Hkv, d, seed=Hq)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_form,k_form", [("padded", "padded"), ("packed", "packed"), ("packed", "padded"), ("padded", "packed")])
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("causal", [0, 1])
def test_prefill_ragged_batches(dtype, q_form, k_form, fused, causal):
    prompt(dtype, [300, 0, 1, 129, 64, 517], 6, 2, 64, q_form=q_form, k_form=k_form, fused=fused, causal=causal, L=2, layer=1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [0, 1])
def test_prefill_newest_queries(dtype, causal):
    """Chunks: fewer queries than keys, one, none; and more queries than keys, whose first stand before the prompt."""
    prompt(dtype, [900, 400, 257, 128, 5, 0, 33], 8, 2, 128, queries=[70, 1, 257, 0, 9, 4, 33], causal=causal)
    prompt(dtype, [640, 300], 4, 4, 64, queries=[13, 290], q_form="packed", causal=causal)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("queries", [1, 5, 40, 130])
def test_prefill_keys_shared_out(dtype, queries):
    """Few queries on many keys: shares of the keys, joined."""
    prompt(dtype, [20011, 7], 4, 2, 128, queries=[queries, min(queries, 7)], seed=queries, spread=2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [0, 1])
def test_prefill_shares_of_several_items(dtype, causal):
    """Shares of items of one and of two tiles of rows, of unequal sequences, of either head size."""
    prompt(dtype, [9001, 1200, 300], 4, 2, 64, queries=[300, 77, 90], causal=causal, seed=1)
    prompt(dtype, [6007], 7, 1, 128, queries=[57], causal=causal, seed=2)
    prompt(dtype, [3300, 2047], 2, 2, 128, causal=causal, seed=3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_many_sequences(dtype):
    """More sequences than a warp has lanes, some empty, packed and padded."""
    lens = [(i * 37) % 200 for i in range(75)]
    prompt(dtype, lens, 4, 2, 64, q_form="packed", k_form="packed", check_all=False)
    prompt(dtype, lens, 4, 2, 64, check_all=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,spread", [(1e-3, 1.0), (0.3, 1.0), (0.0, 12.0), (1e-4, 40.0)])
def test_prefill_flat_and_steep_weights(dtype, scale, spread):
    """Weights that are nearly equal, and maxima that grow again and again."""
    prompt(dtype, [777], 4, 1, 128, scale=scale, spread=spread)


@pytest.mark.gpu
def test_prefill_long():
    """Many tiles of keys for every block, more items than blocks."""
    prompt("bf16", [5003, 2049], 8, 2, 128, q_form="packed", k_form="packed", check_all=False)
    prompt("bf16", [6000], 7, 1, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_rising_keys(dtype):
    """Every tile of keys holds a larger maximum than those before it: what was summed up is scaled down each time."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    n, d = 1500, 128
    q = torch.ones((1, 1, 2, n, d), device="cuda").to(DT[dtype])
    k = (torch.arange(n, device="cuda").view(1, 1, 1, n, 1) / n * 6.0 + 0.01 * torch.randn((1, 1, 1, n, d), generator=gen, device="cuda")).to(DT[dtype])
    v = normal(gen, (1, 1, 1, n, d), dtype)
    cfg = config(dtype, 1, 1, 2, 1, d, n)
    out, lse = torch.empty_like(q), torch.empty((1, 1, 2, n), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), lse_out=lse, seq_len=torch.tensor([n], dtype=torch.int32, device="cuda"))
    see = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    for h in range(2):
        check(dtype, q[0, 0, h], k[0, 0, 0], v[0, 0, 0], see, d ** -0.5, out[0, 0, h], lse[0, 0, h])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_bad_offsets_and_lengths(dtype):
    """Device data out of range: lengths are used as the nearest bound, stretches that are none count as empty."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    cfg = config(dtype, 3, 1, 2, 2, 64, 100)
    q, k, v = (normal(gen, (1, 2, 150, 64), dtype) for _ in range(3))
    off = torch.tensor([0, 90, 40, 151], device="cuda")  # 90 rows; none (ends before it begins); none (beyond the rows)
    out, ws = torch.full_like(q, SENTINEL), mk.new_workspace(cfg)
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, ws, q_off=off, k_off=off)
    assert torch.all(out[:, :, 90:] == SENTINEL) and not torch.any(out[:, :, :90] == SENTINEL)
    q, k, v = (normal(gen, (3, 1, 2, 80, 64), dtype) for _ in range(3))
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    mk.madakv_prefill_attn(cfg, 0, q, k, v, a, ws, seq_len=i32(-5, 1000, 80), q_len=i32(10, 1000, -1))
    mk.madakv_prefill_attn(cfg, 0, q, k, v, b, ws, seq_len=i32(0, 80, 80), q_len=i32(10, 80, 0))
    assert torch.equal(a, b) and not a[0].any() and a[1].all(dim=-1).all() and not a[2].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_one_key_head_for_all(dtype):
    """Keys and values of one head, expanded over the others: a dimension of stride 0."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    n, d, H = 333, 128, 3
    cfg = config(dtype, 1, 1, 2 * H, H, d, n)
    q, k, v = normal(gen, (1, 1, 2 * H, n, d), dtype), normal(gen, (1, 1, 1, n, d), dtype), normal(gen, (1, 1, 1, n, d), dtype)
    out, lse = torch.empty_like(q), torch.empty((1, 1, 2 * H, n), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k.expand(1, 1, H, n, d), v.expand(1, 1, H, n, d), out, mk.new_workspace(cfg), lse_out=lse,
                           seq_len=torch.tensor([n], dtype=torch.int32, device="cuda"))
    see = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    for h in range(2 * H):
        check(dtype, q[0, 0, h], k[0, 0, 0], v[0, 0, 0], see, d ** -0.5, out[0, 0, h], lse[0, 0, h])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_numbers_that_are_none(dtype):
    """A NaN in a key is in the results of the queries that see it and of no other's; one in a query in that query's alone."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    n, d = 300, 64
    cfg = config(dtype, 1, 1, 2, 1, d, n)
    q, k, v = normal(gen, (1, 1, 2, n, d), dtype), normal(gen, (1, 1, 1, n, d), dtype), normal(gen, (1, 1, 1, n, d), dtype)
    k[0, 0, 0, 170, 5] = math.nan
    q[0, 0, 1, 40, 9] = math.nan
    out, lse = torch.empty_like(q), torch.empty((1, 1, 2, n), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), lse_out=lse, seq_len=torch.tensor([n], dtype=torch.int32, device="cuda"))
    bad = torch.zeros((2, n), dtype=torch.bool, device="cuda")
    bad[:, 170:] = True
    bad[1, 40] = True
    assert torch.equal(lse[0, 0].isnan(), bad) and torch.equal(out[0, 0].isnan(), bad.unsqueeze(2).expand(2, n, d))
    see = torch.ones((170, 170), dtype=torch.bool, device="cuda").tril()
    check(dtype, q[0, 0, 0, :170], k[0, 0, 0, :170], v[0, 0, 0, :170], see, d ** -0.5, out[0, 0, 0, :170], lse[0, 0, 0, :170])


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [260.0, 14.0, -300.0])
def test_prefill_logits_far_apart(d, size):
    """Single keys, at every place of a tile in turn, whose logits stand far above or below all of the tiles before: first tiles of a
    row, later ones, the last. The others stay where they were."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    n = 1300
    cfg = config("bf16", 1, 1, 2, 1, d, n)
    q, k, v = torch.full((1, 1, 2, n, d), d ** -0.5, device="cuda").bfloat16(), normal(gen, (1, 1, 1, n, d), "bf16"), normal(gen, (1, 1, 1, n, d), "bf16")
    q[:, :, 1] *= 0.5
    at = torch.arange(0, n, 37, device="cuda")  # (37 and 128 share no factor)
    k[0, 0, 0, at] = (size * (1.0 + at / n * 0.5)).to(torch.bfloat16).unsqueeze(1)
    out, lse = torch.empty_like(q), torch.empty((1, 1, 2, n), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), lse_out=lse, seq_len=torch.tensor([n], dtype=torch.int32, device="cuda"))
    see = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    for h in range(2):
        check("bf16", q[0, 0, h], k[0, 0, 0], v[0, 0, 0], see, d ** -0.5, out[0, 0, h], lse[0, 0, h])


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [260.0, 14.0, -300.0])
def test_prefill_logits_far_apart_in_fp32(d, size):
    """The same in fp32, with rows whose first keys are the smallest and rows whose first are the largest."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    n = 700
    cfg = config("f32", 1, 1, 2, 1, d, n)
    q, k, v = torch.full((1, 1, 2, n, d), d ** -0.5, device="cuda"), normal(gen, (1, 1, 1, n, d), "f32"), normal(gen, (1, 1, 1, n, d), "f32")
    q[:, :, 1] *= -1.0
    at = torch.arange(0, n, 37, device="cuda")
    k[0, 0, 0, at] = (size * (1.0 + at / n * 0.5)).unsqueeze(1)
    out, lse = torch.empty_like(q), torch.empty((1, 1, 2, n), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), lse_out=lse, seq_len=torch.tensor([n], dtype=torch.int32, device="cuda"))
    see = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    for h in range(2):
        check("f32", q[0, 0, h], k[0, 0, 0], v[0, 0, 0], see, d ** -0.5, out[0, 0, h], lse[0, 0, h])


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [2, 147, 386, 640, 659])
def test_prefill_one_bad_key(d, at):
    """One key of NaN, infinities of both signs, in places of a tile that are computed in different ways."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    n = 700
    cfg = config("bf16", 1, 1, 1, 1, d, n)
    q, k, v = normal(gen, (1, 1, 1, n, d), "bf16").abs() + 0.25, normal(gen, (1, 1, 1, n, d), "bf16"), normal(gen, (1, 1, 1, n, d), "bf16")
    ws, lens = mk.new_workspace(cfg), torch.tensor([n], dtype=torch.int32, device="cuda")
    see = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
    for bad in (math.nan, math.inf, -math.inf):
        k[0, 0, 0, at] = bad
        out, lse = torch.empty_like(q), torch.empty((1, 1, 1, n), device="cuda")
        mk.madakv_prefill_attn(cfg, 0, q, k, v, out, ws, lse_out=lse, seq_len=lens)
        check("bf16", q[0, 0, 0, :at], k[0, 0, 0, :at], v[0, 0, 0, :at], see[:at, :at], d ** -0.5, out[0, 0, 0, :at], lse[0, 0, 0, :at])
        if bad == -math.inf:  # as if it were not there
            rest = torch.arange(n, device="cuda") != at
            check("bf16", q[0, 0, 0, at + 1:], k[0, 0, 0, rest], v[0, 0, 0, rest], see[at + 1:, rest], d ** -0.5, out[0, 0, 0, at + 1:], lse[0, 0, 0, at + 1:])
        else:
            assert out[0, 0, 0, at:].isnan().all() and not lse[0, 0, 0, at:].isfinite().any()


# ------------------------------------------------------------------------------------------------- drafted trees
def tree_masks(rng, B, T, kind):
    """[B, T] masks as Python integers: of random trees, of any bits, or none."""
    masks = []
    for _ in range(B):
        bits = []
        for i in range(T):
            if kind == "tree":
                parent = int(rng.integers(0, i)) if i else -1
                bits.append((bits[parent] if i else 0) | 1 << i)
            else:
                bits.append(int(rng.integers(0, 1 << 62)) & ((1 << T) - 1) if kind == "any" and rng.random() < 0.7 else 0)
        masks.append(bits)
    return masks


def as_int64(masks):
    return torch.from_numpy(np.array(masks, dtype=np.uint64).view(np.int64)).cuda()


class Segments:
    """A ragged cache of segments of `lens` rows with headroom; rows outside the segments are not numbers."""

    def __init__(self, gen, dtype, lens, d, headroom=5, tail=0):
        self.lens = lens
        off = np.concatenate([[0], np.cumsum(np.array(lens) + headroom)])
        self.off, self.cap = off.tolist(), int(off[-1]) + tail
        self.k, self.v = (torch.full((self.cap, d), math.nan, device="cuda").to(DT[dtype]) for _ in range(2))
        for a, n in zip(self.off, lens):
            self.k[a:a + n], self.v[a:a + n] = normal(gen, (n, d), dtype), normal(gen, (n, d), dtype)
        self.seg_off = torch.from_numpy(off).cuda()
        self.kept_len = torch.tensor(lens, dtype=torch.int32, device="cuda")


def strided(gen, shape, dtype, fused):
    """[B, L, H, T, d], contiguous or as a projection of [B, L, T, H, d] leaves it."""
    B, L, H, T, d = shape
    return normal(gen, (B, L, T, H + 1, d), dtype).transpose(2, 3)[:, :, :H] if fused else normal(gen, shape, dtype)


def tree(dtype, B, L, Hq, Hkv, d, T, lens, kind="tree", n_nodes=None, layer=-1, fused=False, seed=0, spread=1.0):
    gen, rng = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    g, units = Hq // Hkv, B * L * Hkv
    lens = [lens[u % len(lens)] for u in range(units)]
    seg = Segments(gen, dtype, lens, d)
    cfg = config(dtype, B, L, Hq, Hkv, d, max(max(lens), 1), new=5)
    q = strided(gen, (B, L, Hq, T, d), dtype, fused) * spread
    k_tree, v_tree = strided(gen, (B, L, Hkv, T, d), dtype, fused), strided(gen, (B, L, Hkv, T, d), dtype, fused)
    masks = tree_masks(rng, B, T, kind)
    counts = [T] * B if n_nodes is None else n_nodes
    for b in range(B):  # rows of nodes that are not there are never used
        k_tree[b, :, :, counts[b]:] = math.nan
        v_tree[b, :, :, counts[b]:] = math.nan
    out, lse, ws = torch.full_like(q, SENTINEL), torch.full((B, L, Hq, T), SENTINEL, device="cuda"), mk.new_workspace(cfg)
    k0, v0 = seg.k.clone(), seg.v.clone()
    mk.madakv_tree_attn(cfg, layer, q, k_tree, v_tree, as_int64(masks), seg.k, seg.v, seg.seg_off, seg.kept_len, out, lse, ws,
                        n_nodes=None if n_nodes is None else torch.tensor(n_nodes, dtype=torch.int32, device="cuda"))
    assert mk.madakv_poll_status(ws) == 0
    assert torch.equal(k0.nan_to_num(9.0), seg.k.nan_to_num(9.0)) and torch.equal(v0.nan_to_num(9.0), seg.v.nan_to_num(9.0))
    touched = torch.zeros((B, L, Hq, T), dtype=torch.bool, device="cuda")
    for u in range(units):
        b, l, h = u // (L * Hkv), u // Hkv % L, u % Hkv
        if layer >= 0 and l != layer:
            continue
        n, a, m = lens[u], seg.off[u], counts[b]
        k = torch.cat((seg.k[a:a + n], k_tree[b, l, h, :m]))
        v = torch.cat((seg.v[a:a + n], v_tree[b, l, h, :m]))
        see = torch.zeros((m, n + m), dtype=torch.bool, device="cuda")
        see[:, :n] = True
        for i in range(m):
            for j in range(m):
                see[i, n + j] = bool(masks[b][i] >> j & 1)
        for j in range(g):
            check(dtype, q[b, l, h * g + j, :m], k, v, see, d ** -0.5, out[b, l, h * g + j, :m], lse[b, l, h * g + j, :m], (u, j))
        touched[b, l, h * g:(h + 1) * g, :m] = True
    assert torch.all(out[~touched] == SENTINEL) and torch.all(lse[~touched] == SENTINEL)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 2, 7, 16, 33, 64])
@pytest.mark.parametrize("Hq,Hkv,d", [(2, 2, 128), (7, 1, 128), (8, 2, 64)])
def test_tree_sizes(dtype, T, Hq, Hkv, d):
    tree(dtype, 1, 2, Hq, Hkv, d, T, [0, 1, 127, 128, 129, 300, 64, 65], seed=T, fused=T % 2 == 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["tree", "any", "none"])
def test_tree_masks_and_node_counts(dtype, kind):
    """Masks that are no trees, that leave nodes nothing to see where the segment is empty; fewer nodes than there is room for, none."""
    tree(dtype, 4, 1, 4, 2, 64, 12, [0, 50, 257], kind=kind, n_nodes=[12, 5, 0, 1], seed=4)
    tree(dtype, 2, 3, 12, 1, 128, 40, [130, 0, 640], kind=kind, n_nodes=[40, 33], layer=1, seed=5, fused=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,Hkv", [(3, 4, 4), (16, 7, 1), (64, 33, 1), (5, 64, 1)])
def test_tree_long_segments(dtype, T, Hq, Hkv):
    """Few long segments: their rows are shared out over blocks."""
    tree(dtype, 1, 1, Hq, Hkv, 128, T, [9001, 4000, 17, 700], seed=T, spread=2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_layers_that_do_not_lie_evenly(dtype):
    """Queries of two of three layers: sequences and layers have strides of their own."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    B, L, H, T, d = 2, 2, 2, 5, 64
    cfg = config(dtype, B, L, H, H, d, 150)
    seg = Segments(gen, dtype, [130, 0, 77, 128, 20, 5, 140, 64], d)
    q, k, v = (normal(gen, (B, L + 1, H, T, d), dtype)[:, 1:] for _ in range(3))
    out, lse, ws = torch.zeros((B, L + 1, H, T, d), device="cuda").to(DT[dtype])[:, :2], torch.empty((B, L, H, T), device="cuda"), mk.new_workspace(cfg)
    mk.madakv_tree_attn(cfg, -1, q, k, v, as_int64([[1, 3, 7, 15, 31]] * B), seg.k, seg.v, seg.seg_off, seg.kept_len, out, lse, ws)
    for u, n in enumerate(seg.lens):
        b, l, h, a = u // (L * H), u // H % L, u % H, seg.off[u]
        see = torch.cat((torch.ones((T, n), device="cuda"), torch.ones((T, T), device="cuda").tril()), 1).bool()
        check(dtype, q[b, l, h], torch.cat((seg.k[a:a + n], k[b, l, h])), torch.cat((seg.v[a:a + n], v[b, l, h])), see, d ** -0.5, out[b, l, h], lse[b, l, h], u)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_copies_that_never_come_end_in_a_status(dtype, monkeypatch):
    """Copies of keys are withheld: every wait for them ends, the call reports it, and the next call on the workspace is whole."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    cfg = config(dtype, 2, 1, 8, 2, 128, 700, new=8)
    ws, n = mk.new_workspace(cfg), torch.tensor([700, 300], dtype=torch.int32, device="cuda")
    q, k, v = normal(gen, (2, 1, 8, 700, 128), dtype), normal(gen, (2, 1, 2, 700, 128), dtype), normal(gen, (2, 1, 2, 700, 128), dtype)
    seg = Segments(gen, dtype, [500, 31, 700, 129], 128, headroom=8)
    qt, kt, mask = normal(gen, (2, 1, 8, 5, 128), dtype), normal(gen, (2, 1, 2, 5, 128), dtype), as_int64([[1, 3, 5, 9, 17]] * 2)
    outs = [torch.zeros_like(q), torch.zeros_like(qt)]

    def calls():
        mk.madakv_prefill_attn(cfg, 0, q, k, v, outs[0], ws, seq_len=n)
        first = mk.madakv_poll_status(ws)
        mk.madakv_tree_attn(cfg, -1, qt, kt, kt, mask, seg.k, seg.v, seg.seg_off, seg.kept_len, outs[1], None, ws)
        return first, mk.madakv_poll_status(ws)

    assert calls() == (0, 0)
    want = [x.clone() for x in outs]
    monkeypatch.setenv("MADAKV_TEST_HOLD_COPIES", "200000")
    assert calls() == (mk.ETIMEOUT, mk.ETIMEOUT)
    monkeypatch.delenv("MADAKV_TEST_HOLD_COPIES")
    assert calls() == (0, 0)
    assert all(torch.equal(x, y) for x, y in zip(outs, want))


@pytest.mark.gpu
def test_tree_many_segments():
    tree("bf16", 2, 20, 8, 8, 128, 6, [200, 31, 129, 0, 402], seed=8)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tree_refused_segments_count_as_empty(dtype):
    gen = torch.Generator(device="cuda").manual_seed(6)
    cfg = config(dtype, 1, 1, 3, 3, 64, 200)
    seg = Segments(gen, dtype, [100, 90, 80], 64)
    seg.seg_off[3] = seg.cap + 1  # the last segment's headroom ends beyond the cache
    seg.kept_len[1] = 96  # longer than its slot
    q, k, v = (normal(gen, (1, 1, 3, 4, 64), dtype) for _ in range(3))
    mask = as_int64([[1, 3, 7, 15]])
    out, lse, ws = torch.empty_like(q), torch.empty((1, 1, 3, 4), device="cuda"), mk.new_workspace(cfg)
    mk.madakv_tree_attn(cfg, -1, q, k, v, mask, seg.k, seg.v, seg.seg_off, seg.kept_len, out, lse, ws)
    see = torch.ones((4, 4), dtype=torch.bool, device="cuda").tril()
    for h in (1, 2):
        check(dtype, q[0, 0, h], k[0, 0, h], v[0, 0, h], see, 0.125, out[0, 0, h], lse[0, 0, h])
    see = torch.cat((torch.ones((4, 100), dtype=torch.bool, device="cuda"), see), 1)
    check(dtype, q[0, 0, 0], torch.cat((seg.k[:100], k[0, 0, 0])), torch.cat((seg.v[:100], v[0, 0, 0])), see, 0.125, out[0, 0, 0], lse[0, 0, 0])


# ------------------------------------------------------------------------------------------------- the accepted path
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layer", [-1, 1])
@pytest.mark.parametrize("T,d", [(1, 128), (9, 64), (64, 128)])
def test_commit_appends_the_accepted_path(dtype, layer, T, d):
    gen, rng = torch.Generator(device="cuda").manual_seed(T), np.random.default_rng(T)
    B, L, H = 5, 2, 3
    lens = [int(x) for x in rng.integers(0, 40, B * L * H)]
    seg = Segments(gen, dtype, lens, d, headroom=min(T, 20))
    cfg = config(dtype, B, L, 2 * H, H, d, 64, new=min(T, 20))
    k_tree, v_tree = strided(gen, (B, L, H, T, d), dtype, True), strided(gen, (B, L, H, T, d), dtype, False)
    masks = tree_masks(rng, B, T, "tree")
    masks[0] = [(1 << (i + 1)) - 1 for i in range(T)]  # a chain: with 64 nodes more than the headroom
    counts, node = [T, T, max(1, T // 2), T, 0], [T - 1, -1, T - 1, T // 2, 0]
    acc = torch.rand(seg.cap, generator=gen, device="cuda")
    idx = torch.full((seg.cap,), -3, dtype=torch.int32, device="cuda")
    position, ws = torch.arange(B, dtype=torch.int32, device="cuda") * 100, mk.new_workspace(cfg)
    want = [x.clone() for x in (seg.k, seg.v, seg.kept_len, acc, idx)]
    capacity = missing = False
    for u in range(B * L * H):
        b, l, h = u // (L * H), u // H % L, u % H
        if (layer >= 0 and l != layer) or node[b] < 0:
            continue
        if node[b] >= counts[b]:
            missing = True
            continue
        path = [j for j in range(counts[b]) if masks[b][node[b]] >> j & 1]
        if len(path) > min(T, 20):
            capacity = True
            continue
        a = seg.off[u] + lens[u]
        for i, j in enumerate(path):
            want[0][a + i], want[1][a + i], want[3][a + i], want[4][a + i] = k_tree[b, l, h, j], v_tree[b, l, h, j], 0.0, 100 * b + i
        want[2][u] += len(path)
    mk.madakv_tree_commit(cfg, layer, as_int64(masks), torch.tensor(node, dtype=torch.int32, device="cuda"), k_tree, v_tree, seg.k, seg.v,
                          seg.seg_off, seg.kept_len, ws, n_nodes=torch.tensor(counts, dtype=torch.int32, device="cuda"), acc=acc, kept_idx=idx,
                          position=position)
    for x, y in zip((seg.k, seg.v, seg.kept_len, acc, idx), want):
        assert torch.equal(x.nan_to_num(9.0) if x.is_floating_point() else x, y.nan_to_num(9.0) if y.is_floating_point() else y)
    status = mk.madakv_poll_status(ws)
    assert status in ([mk.ECAPACITY] if capacity else []) + ([mk.ESHAPE] if missing else []) + ([] if capacity or missing else [0])


# ------------------------------------------------------------------------------------------------- together
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_eviction_and_speculative_steps_together(dtype):
    """Layer by layer through a prompt, eviction by what that left, two speculative steps, a decode step, rows cut back: each stage against the
    formulas on what the stages before it gave."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    B, L, Hq, Hkv, d, n, w, T = 2, 3, 8, 2, 64, 500, 16, 6
    g, lens = Hq // Hkv, [500, 333]
    cfg = config(dtype, B, L, Hq, Hkv, d, n, w, new=24)
    buf = mk.EvictionBuffers(cfg, B * L * Hkv * (n + 24), want_lse=True, track=True)
    q, k, v = normal(gen, (B, L, Hq, n, d), dtype), normal(gen, (B, L, Hkv, n, d), dtype), normal(gen, (B, L, Hkv, n, d), dtype)
    seq_len, mask = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.zeros((B, n), dtype=torch.uint8, device="cuda")
    mask[:, 40:200] = 1
    budget = torch.tensor([60, 45], dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    with pytest.raises(ValueError):
        buf.run_eviction(None, k, v, mask, seq_len, budget)
    for layer in range(L):
        buf.run_prefill(layer, q, k, v, out, seq_len=seq_len)
    for b in range(B):
        see = torch.ones((lens[b], lens[b]), dtype=torch.bool, device="cuda").tril()
        for layer in range(L):
            z = (q[b, layer, 0, :lens[b]].double() @ k[b, layer, 0, :lens[b]].double().T * d ** -0.5).masked_fill(~see, -math.inf)
            check(dtype, q[b, layer, 0, :lens[b]], k[b, layer, 0, :lens[b]], v[b, layer, 0, :lens[b]], see, d ** -0.5, out[b, layer, 0, :lens[b]],
                  torch.logsumexp(z, 1))
    buf.run_eviction(None, k, v, mask, seq_len, budget)
    # the scores of the two-pass stage on the same queries
    q_win = torch.stack([q[b, :, :, lens[b] - w:lens[b]] for b in range(B)])
    assert torch.equal(q_win, buf.q_win)
    psi = torch.zeros_like(buf.psi)
    mk.madakv_score(cfg, q_win, k, seq_len, None, psi, buf.ws)
    assert torch.allclose(psi, buf.psi, rtol=1e-4, atol=1e-7)
    limit = buf.kept_len.clone()
    for step in range(2):
        masks = as_int64([[1, 3, 5, 11, 19, 37]] * B)  # 0 - (1 - (3, 4), 2 - 5)
        node = torch.tensor([4, 5], dtype=torch.int32, device="cuda")
        qt, kt, vt = normal(gen, (B, L, Hq, T, d), dtype), normal(gen, (B, L, Hkv, T, d), dtype), normal(gen, (B, L, Hkv, T, d), dtype)
        ot, yt = torch.zeros_like(qt), torch.zeros((B, L, Hq, T), device="cuda")
        buf.run_tree(qt, kt, vt, masks, ot, yt)
        off, had = buf.seg_off.tolist(), buf.kept_len.tolist()
        before = buf.kept_len.clone()
        buf.run_commit(masks, node, kt, vt, position=seq_len + 3 * step)
        assert torch.equal(buf.kept_len, before + 3)
        for u in range(B * L * Hkv):
            b, l, h = u // (L * Hkv), u // Hkv % L, u % Hkv
            path = [[0, 1, 4], [0, 2, 5]][b]
            a = off[u] + had[u]
            assert torch.equal(buf.k_c[a:a + 3], kt[b, l, h, path]) and torch.equal(buf.v_c[a:a + 3], vt[b, l, h, path])
            assert buf.kept_idx[a:a + 3].tolist() == [lens[b] + 3 * step + i for i in range(3)]
            # the last accepted node attended to what the segment now ends with
            see = torch.ones((1, had[u] + 3), dtype=torch.bool, device="cuda")
            for j in range(g):
                check(dtype, qt[b, l, h * g + j, path[2]:path[2] + 1], buf.k_c[off[u]:a + 3], buf.v_c[off[u]:a + 3], see, d ** -0.5,
                      ot[b, l, h * g + j, path[2]:path[2] + 1], yt[b, l, h * g + j, path[2]:path[2] + 1])
    # a plain decode step sees the committed rows; the same as a tree of one node does
    q1, k1, v1 = normal(gen, (B, L, Hq, 1, d), dtype), normal(gen, (B, L, Hkv, 1, d), dtype), normal(gen, (B, L, Hkv, 1, d), dtype)
    o1, y1 = torch.zeros_like(q1), torch.zeros((B, L, Hq, 1), device="cuda")
    buf.run_tree(q1, k1, v1, torch.ones((B, 1), dtype=torch.int64, device="cuda"), o1, y1)
    buf.run_decode(q1[:, :, :, 0].contiguous(), k1[:, :, :, 0].contiguous(), v1[:, :, :, 0].contiguous(), position=seq_len + 6)
    assert torch.allclose(o1[:, :, :, 0].float(), buf.out.float(), atol=4 * HALF[dtype] * float(v.float().abs().max()) + 1e-5)
    assert torch.allclose(y1[..., 0], buf.lse_dec, atol=1e-5, rtol=1e-5)
    buf.run_trim(limit, recent=4)
    assert torch.equal(buf.kept_len, limit.clamp(min=4)) and mk.madakv_poll_status(buf.ws) == 0  # (the protected rows stay)


@pytest.mark.gpu
def test_buffers_refuse_what_they_cannot_do():
    cfg = config("bf16", n=64)
    four_bits, plain = mk.EvictionBuffers(cfg, 400, quant=True), mk.EvictionBuffers(cfg, 400)
    for call in (lambda: four_bits.run_tree(*[None] * 5), lambda: four_bits.run_commit(*[None] * 4), lambda: plain.run_prefill(0, *[None] * 4)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_bindings_check_their_tensors():
    gen = torch.Generator(device="cuda").manual_seed(1)
    cfg = config("bf16", 2, 1, 4, 2, 64, 32)
    ws, lens = mk.new_workspace(cfg), torch.full((2,), 32, dtype=torch.int32, device="cuda")
    q, k = normal(gen, (2, 1, 4, 32, 64), "bf16"), normal(gen, (2, 1, 2, 32, 64), "bf16")
    ok = dict(q=q, k=k, v=k, out=torch.empty_like(q), ws=ws, seq_len=lens)
    mk.madakv_prefill_attn(cfg, 0, **ok)
    bad = [dict(q=q.float()), dict(q=q.cpu()), dict(q=q[:1]), dict(q=q[:, :, :3]), dict(k=k[..., :32]), dict(v=k[:, :, :, :31]),
           dict(out=torch.empty_like(q)[:, :, :, :31]), dict(q=q.transpose(3, 4)), dict(seq_len=lens[:1]), dict(seq_len=lens.long()),
           dict(lse_out=torch.empty((2, 1, 4, 31), device="cuda")), dict(q_win=torch.empty((2, 1, 4, 7, 64), device="cuda").bfloat16()),
           dict(q_off=torch.zeros(3, dtype=torch.int64, device="cuda")), dict(ws=ws.cpu())]
    for change in bad:
        with pytest.raises(ValueError):
            mk.madakv_prefill_attn(cfg, 0, **{**ok, **change})
    with pytest.raises(mk.MadakvError):
        mk.madakv_prefill_attn(cfg, 0, **{**ok, "seq_len": None})
    with pytest.raises(mk.MadakvError):
        mk.madakv_prefill_attn(cfg, 1, **ok)
    seg = Segments(gen, "bf16", [10, 11, 12, 13], 64)
    mask, node = torch.ones((2, 3), dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    q, k = normal(gen, (2, 1, 4, 3, 64), "bf16"), normal(gen, (2, 1, 2, 3, 64), "bf16")
    attn = dict(q=q, k_tree=k, v_tree=k, mask=mask, k_c=seg.k, v_c=seg.v, seg_off=seg.seg_off, kept_len=seg.kept_len, out=torch.empty_like(q),
                lse_out=None, ws=ws)
    mk.madakv_tree_attn(cfg, -1, **attn)
    commit = dict(mask=mask, node=node, k_tree=k, v_tree=k, k_c=seg.k, v_c=seg.v, seg_off=seg.seg_off, kept_len=seg.kept_len, ws=ws)
    mk.madakv_tree_commit(cfg, -1, **commit)
    shared = [dict(mask=mask[:, :2].contiguous()), dict(mask=mask.int()), dict(k_tree=k[:, :, :, :2]), dict(v_c=seg.v[1:]), dict(v_c=seg.v.float()),
              dict(seg_off=seg.seg_off[:4]), dict(kept_len=seg.kept_len[:3]), dict(n_nodes=node[:1]), dict(k_tree=k[:, :, :1])]
    for change in shared + [dict(q=q[:, :, :2]), dict(lse_out=torch.empty((2, 1, 4, 2), device="cuda"))]:
        with pytest.raises(ValueError):
            mk.madakv_tree_attn(cfg, -1, **{**attn, **change})
    for change in shared + [dict(node=node[:1]), dict(acc=torch.zeros(3, device="cuda"))]:
        with pytest.raises(ValueError):
            mk.madakv_tree_commit(cfg, -1, **{**commit, **change})
    with pytest.raises(mk.MadakvError):
        mk.madakv_tree_commit(cfg, -1, **commit, position=node)


# ------------------------------------------------------------------------------------------------- streams, graphs, repetition
def steps(dtype, seed):
    """A prompt call whose keys are shared out, a whole prompt, a tree call, on one workspace: their tensors and the calls."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cfg = config(dtype, 1, 1, 8, 2, 128, 6000, 8, new=8)
    ws, n = mk.new_workspace(cfg), torch.tensor([6000], dtype=torch.int32, device="cuda")
    k, v = normal(gen, (1, 1, 2, 6000, 128), dtype), normal(gen, (1, 1, 2, 6000, 128), dtype)
    qs = [normal(gen, (1, 1, 8, m, 128), dtype) for m in (9, 700)]
    outs = [torch.zeros_like(x) for x in qs]
    seg = Segments(gen, dtype, [5000, 31], 128, headroom=8)
    qt, kt = normal(gen, (1, 1, 8, 5, 128), dtype), normal(gen, (1, 1, 2, 5, 128), dtype)
    outs.append(torch.zeros_like(qt))
    mask = as_int64([[1, 3, 5, 9, 17]])
    m = [torch.tensor([x.shape[3]], dtype=torch.int32, device="cuda") for x in qs]

    def run():
        for x, y, z in zip(qs, outs, m):
            mk.madakv_prefill_attn(cfg, 0, x, k, v, y, ws, seq_len=n, q_len=z)
        mk.madakv_tree_attn(cfg, -1, qt, kt, kt, mask, seg.k, seg.v, seg.seg_off, seg.kept_len, outs[2], None, ws)

    return run, outs


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_repeated_and_captured_calls_give_the_same_bits(dtype):
    run, outs = steps(dtype, 1)
    run()
    first = [x.clone() for x in outs]
    for _ in range(3):
        for x in outs:
            x.zero_()
        run()
        assert all(torch.equal(x, y) for x, y in zip(outs, first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for x in outs:
            x.zero_()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(outs, first))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_on_two_streams_with_workspaces_of_their_own(dtype):
    sides = [steps(dtype, 1), steps(dtype, 2)]
    want = []
    for run, outs in sides:
        run()
        want.append([x.clone() for x in outs])
        for x in outs:
            x.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sides]
    for _ in range(10):
        for (run, _), s in zip(sides, streams):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for (_, outs), first in zip(sides, want):
        assert all(torch.equal(x, y) for x, y in zip(outs, first))
