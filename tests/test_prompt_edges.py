"""Attention of prompts and drafted trees where no other test goes: huge and infinite numbers in masked places, rows that begin on 16-byte boundaries
only, trees whose logits lie far apart, small workspaces, what is refused."""
import ctypes
import math

import pytest
import torch

from paper_2506_15724_b200 import binding as mk
from test_prompt_and_trees import DT, FAKE, HALF, SENTINEL, Segments, as_int64, attend, check, config, lib, normal  # noqa: F401

BIG_BF16 = 2.0 ** 128 - 2.0 ** 120  # the largest finite bf16 number


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def causal(n):
    return torch.ones((n, n), dtype=torch.bool, device="cuda").tril()


# ------------------------------------------------------------------------------------------------- masked places
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [5, 130, 300, 450, 690])
def test_huge_values_do_not_reach_queries_before_them(dtype, d, at):
    gen = torch.Generator(device="cuda").manual_seed(at)
    n = 700
    cfg = config(dtype, 1, 1, 2, 1, d, n)
    q, k, v = normal(gen, (1, 1, 2, n, d), dtype), normal(gen, (1, 1, 1, n, d), dtype), normal(gen, (1, 1, 1, n, d), dtype)
    ws, outs = mk.new_workspace(cfg), []
    for big in (False, True):
        if big:
            v[..., at:, :] = 3e38
        outs.append(torch.empty_like(q))
        mk.madakv_prefill_attn(cfg, 0, q, k, v, outs[-1], ws, seq_len=i32(n))
    assert torch.equal(outs[0][..., :at, :], outs[1][..., :at, :])
    for h in range(2):
        check(dtype, q[0, 0, h, :at], k[0, 0, 0, :at], v[0, 0, 0, :at], causal(at), d ** -0.5, outs[1][0, 0, h, :at],
              attend(q[0, 0, h, :at].double(), k[0, 0, 0, :at].double(), v[0, 0, 0, :at].double(), causal(at), d ** -0.5)[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_huge_values_do_not_reach_nodes_that_do_not_see_them(dtype, d):
    gen = torch.Generator(device="cuda").manual_seed(3)
    T, seg = 40, Segments(gen, dtype, [200, 0], d)
    cfg = config(dtype, 1, 1, 4, 2, d, 200)
    q, k, v = normal(gen, (1, 1, 4, T, d), dtype), normal(gen, (1, 1, 2, T, d), dtype), normal(gen, (1, 1, 2, T, d), dtype)
    mask, ws, outs = as_int64([[(1 << (i + 1)) - 1 for i in range(T)]]), mk.new_workspace(cfg), []
    for big in (False, True):
        if big:
            v[..., 17:, :] = -3e38
        outs.append(torch.empty_like(q))
        mk.madakv_tree_attn(cfg, -1, q, k, v, mask, seg.k, seg.v, seg.seg_off, seg.kept_len, outs[-1], None, ws)
    assert torch.equal(outs[0][..., :17, :], outs[1][..., :17, :]) and outs[0].isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,d,shift", [(1, 128, 0), (1, 128, 1), (1, 64, 1), (7, 128, 0), (7, 64, 3), (2, 64, 77)])
@pytest.mark.parametrize("at", [255, 260, 639])
def test_a_value_that_is_no_number_reaches_so_far(dtype, Hq, d, shift, at):
    """NaN in a row of V: in the results of the queries that see it, and of none that stands more than 126 + floor(128 / g) positions before it."""
    gen = torch.Generator(device="cuda").manual_seed(at)
    n, g = 700 + shift, Hq
    cfg = config(dtype, 1, 1, Hq, 1, d, n)
    q, k, v = normal(gen, (1, 1, Hq, 700, d), dtype), normal(gen, (1, 1, 1, n, d), dtype), normal(gen, (1, 1, 1, n, d), dtype)
    v[0, 0, 0, at, 3] = math.nan
    out, lse = torch.empty_like(q), torch.empty((1, 1, Hq, 700), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), lse_out=lse, seq_len=i32(n), q_len=i32(700))
    assert lse.isfinite().all() and out[0, 0, :, at - shift:, 3].isnan().all()
    clean = max(0, at - (126 + 128 // g) - shift)  # queries; query i stands at i + shift
    see = torch.arange(n, device="cuda") <= torch.arange(clean, device="cuda").view(-1, 1) + shift
    for h in range(Hq):
        check(dtype, q[0, 0, h, :clean], k[0, 0, 0], v[0, 0, 0].nan_to_num(0.0), see, d ** -0.5, out[0, 0, h, :clean], lse[0, 0, h, :clean])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rise", [0.0, 0.4, 3.0])
@pytest.mark.parametrize("n,m", [(3000, 3000), (30000, 50)])
def test_values_at_the_end_of_their_range(dtype, d, rise, n, m):
    """Values of 2^96, in either sign, on logits that rise slowly: weights add up far beyond the reference that they are taken against."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    cfg = config(dtype, 1, 1, 1, 1, d, n)
    q, k, v = normal(gen, (1, 1, 1, m, d), dtype) * 0.1, normal(gen, (1, 1, 1, n, d), dtype), normal(gen, (1, 1, 1, n, d), dtype)
    q[..., 0] = d ** 0.5
    k[..., 0] = (torch.arange(n, device="cuda") // 128 * rise).to(DT[dtype])  # (a tile's weights are e^rise of the last one's)
    v = (torch.sign(v.float()) * 2.0 ** 96).to(DT[dtype])
    out, lse = torch.empty_like(q), torch.empty((1, 1, 1, m), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), lse_out=lse, seq_len=i32(n), q_len=i32(m))
    see = torch.arange(n, device="cuda") <= torch.arange(m, device="cuda").view(-1, 1) + n - m
    check(dtype, q[0, 0, 0], k[0, 0, 0], v[0, 0, 0], see, d ** -0.5, out[0, 0, 0], lse[0, 0, 0])


# ------------------------------------------------------------------------------------------------- infinities in fp32
@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [2, 147, 386, 640])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_infinite_keys_in_fp32(d, at, sign):
    """An infinite element counts as the largest finite bf16 number: the key has all of the weight, or none. (Queries below 2^-7 in magnitude: the
    products stay finite.)"""
    gen = torch.Generator(device="cuda").manual_seed(at)
    n = 700
    cfg = config("f32", 1, 1, 1, 1, d, n)
    q = (torch.rand((1, 1, 1, n, d), generator=gen, device="cuda") + 0.01) * torch.where(torch.rand((1, 1, 1, n, 1), generator=gen, device="cuda") < 0.5, -1, 1) / 256
    k, v = normal(gen, (1, 1, 1, n, d), "f32"), normal(gen, (1, 1, 1, n, d), "f32")
    k[0, 0, 0, at, 5] = sign * math.inf
    out, lse = torch.empty_like(q), torch.empty((1, 1, 1, n), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), lse_out=lse, seq_len=i32(n))
    qq, kk, vv, oo, yy = q[0, 0, 0], k[0, 0, 0], v[0, 0, 0], out[0, 0, 0], lse[0, 0, 0]
    check("f32", qq[:at], kk[:at], vv[:at], causal(n)[:at, :at], d ** -0.5, oo[:at], yy[:at])
    later = torch.arange(n, device="cuda") >= at
    all_of_it, none = later & (qq[:, 5] * sign > 0), later & (qq[:, 5] * sign < 0)
    want = (qq.double() @ kk.double().nan_to_num(posinf=BIG_BF16, neginf=-BIG_BF16)[at]) * d ** -0.5
    assert all_of_it.sum() > 3 and none.sum() > 3
    assert torch.all((oo[all_of_it] - vv[at]).abs() <= 2.0 ** -22 * vv[at].abs())
    assert torch.all((yy.double() - want).abs()[all_of_it] <= 2.0 ** -20 * want.abs()[all_of_it])
    rest = torch.arange(n, device="cuda") != at
    some = none & (torch.arange(n, device="cuda") > 0)
    check("f32", qq[some], kk[rest], vv[rest], causal(n)[some][:, rest], d ** -0.5, oo[some], yy[some])


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_values_and_queries_in_fp32(d):
    """Values: queries before them are what they were; queries: theirs alone."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    n = 300
    cfg = config("f32", 1, 1, 1, 1, d, n)
    q, k, v = (normal(gen, (1, 1, 1, n, d), "f32") for _ in range(3))
    v[0, 0, 0, 170] = math.inf
    v[0, 0, 0, 171, ::2] = -math.inf
    q[0, 0, 0, 40, 9] = -math.inf
    out, lse = torch.empty_like(q), torch.empty((1, 1, 1, n), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), lse_out=lse, seq_len=i32(n))
    rows = torch.arange(n, device="cuda") != 40
    z = torch.logsumexp((q[0, 0, 0].double().nan_to_num(posinf=0, neginf=0) @ k[0, 0, 0].double().T * d ** -0.5).masked_fill(~causal(n), -math.inf), 1)
    mag = (q[0, 0, 0].double().nan_to_num(posinf=0, neginf=0).abs() @ k[0, 0, 0].double().abs().T * d ** -0.5).amax(1)
    most = (d + 8) * 2.0 ** -23 * mag + (n / 16 + 68) * 2.0 ** -23 + 2.0 ** -22 * z.abs()  # (as in check)
    assert torch.all((lse[0, 0, 0].double() - z).abs()[rows] <= most[rows])
    rows[170:] = False
    check("f32", q[0, 0, 0, rows], k[0, 0, 0, :170], v[0, 0, 0, :170], causal(n)[rows, :170], d ** -0.5, out[0, 0, 0, rows], lse[0, 0, 0, rows])


# ------------------------------------------------------------------------------------------------- logits beyond what exponentials tell apart
def check_ties(dtype, q, k, v, see, scale, out, lse):
    """Logits that are exact and equal or very far apart: what is left are roundings of weights, sums and results (as in check)."""
    z = (q.double() @ k.double().T * scale).masked_fill(~see, -math.inf)
    want_lse, w = torch.logsumexp(z, 1), torch.softmax(z, 1)  # (less the maximum first: a log-sum-exp of 2^58 has no room for the logarithm)
    want = w @ v.double()
    sums = (k.shape[0] / 16 + 64) * 2.0 ** -23
    most = HALF[dtype] * want.abs() + ((HALF[dtype] if dtype == "bf16" else 0.0) + sums) * (w @ v.double().abs()) + 1e-30
    err = (out.double() - want).abs()
    assert torch.all(err <= most), float((err / most).nan_to_num(math.inf).max())
    assert torch.all((lse.double() - want_lse).abs() <= sums + 2.0 ** -21 * want_lse.abs())


def steps_of(gen, n, d, size, low, dtype):
    k = torch.zeros((n, d), device="cuda")
    k[:, 0] = torch.randint(low, low + 6, (n,), generator=gen, device="cuda").float() * size
    return k.to(DT[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [10, 24, 35, 61, 100])
@pytest.mark.parametrize("low", [-6, -2, 1])
@pytest.mark.parametrize("n,m", [(700, 700), (9000, 40)])
def test_prefill_of_huge_logits(dtype, d, power, low, n, m):
    """The keys with the largest logit share the weight equally, also where a logit's rounding is larger than what separates weights."""
    gen = torch.Generator(device="cuda").manual_seed(power)
    cfg = config(dtype, 1, 1, 1, 1, d, n)
    q, v = torch.zeros((1, 1, 1, m, d), device="cuda").to(DT[dtype]), normal(gen, (1, 1, 1, n, d), dtype)
    q[..., 0] = 1.0
    k = steps_of(gen, n, d, 2.0 ** power, low, dtype).view(1, 1, 1, n, d)
    out, lse = torch.empty_like(q), torch.empty((1, 1, 1, m), device="cuda")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), lse_out=lse, seq_len=i32(n), q_len=i32(m))
    see = torch.arange(n, device="cuda") <= torch.arange(m, device="cuda").view(-1, 1) + n - m
    check_ties(dtype, q[0, 0, 0], k[0, 0, 0], v[0, 0, 0], see, d ** -0.5, out[0, 0, 0], lse[0, 0, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("power", [10, 35, 100])
@pytest.mark.parametrize("n", [0, 300, 9000])
def test_trees_of_huge_logits(dtype, d, power, n):
    gen = torch.Generator(device="cuda").manual_seed(power)
    T, seg = 20, Segments(gen, dtype, [n], d)
    cfg = config(dtype, 1, 1, 1, 1, d, max(n, 1))
    q, v = torch.zeros((1, 1, 1, T, d), device="cuda").to(DT[dtype]), normal(gen, (1, 1, 1, T, d), dtype)
    q[..., 0] = 1.0
    seg.k[:n] = steps_of(gen, n, d, 2.0 ** power, -4, dtype)
    k = steps_of(gen, T, d, 2.0 ** power, -3, dtype).view(1, 1, 1, T, d)
    out, lse = torch.empty_like(q), torch.empty((1, 1, 1, T), device="cuda")
    mk.madakv_tree_attn(cfg, -1, q, k, v, as_int64([[(1 << (i + 1)) - 1 for i in range(T)]]), seg.k, seg.v, seg.seg_off, seg.kept_len, out, lse,
                        mk.new_workspace(cfg))
    see = torch.cat((torch.ones((T, n), dtype=torch.bool, device="cuda"), causal(T)), 1)
    check_ties(dtype, q[0, 0, 0], torch.cat((seg.k[:n], k[0, 0, 0])), torch.cat((seg.v[:n], v[0, 0, 0])), see, d ** -0.5, out[0, 0, 0], lse[0, 0, 0])


# ------------------------------------------------------------------------------------------------- strides
def shifted(x):
    """The same numbers in rows that begin on 16-byte boundaries of which no two neighbours are 32-byte ones."""
    e = 16 // x.element_size()
    y = torch.full((*x.shape[:-1], x.shape[-1] + e), SENTINEL, device="cuda").to(x.dtype)[..., e:]
    y.copy_(x)
    return y


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,m", [(400, 400), (90, 90), (9000, 33)])
def test_rows_on_16_byte_boundaries(dtype, d, n, m):
    """Whole tiles and part of one, results that go out at once and shares; proxy tokens' queries behind an odd 16 bytes."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    w = 16
    cfg = config(dtype, 1, 1, 4, 2, d, n, w)
    q, k, v = normal(gen, (1, 1, 4, m, d), dtype), normal(gen, (1, 1, 2, n, d), dtype), normal(gen, (1, 1, 2, n, d), dtype)
    ws, e, got = mk.new_workspace(cfg), 16 // q.element_size(), []
    for f in (lambda x: x, shifted):
        out = f(torch.full_like(q, SENTINEL))
        space = torch.full((4 * w * d + e,), SENTINEL, device="cuda").to(DT[dtype])
        q_win, lse_win = space[0 if f is not shifted else e:][:4 * w * d].view(1, 1, 4, w, d), torch.empty((1, 1, 4, w), device="cuda")
        mk.madakv_prefill_attn(cfg, 0, f(q), f(k), f(v), out, ws, q_win=q_win, lse_win=lse_win, seq_len=i32(n), q_len=i32(m))
        if f is shifted:
            around = out.as_strided((4 * m, e), (d + e, 1), out.storage_offset() - e)
            assert torch.all(around == SENTINEL) and torch.all(space[:e] == SENTINEL)
        got.append((out, q_win, lse_win))
    assert all(torch.equal(x, y) for x, y in zip(*got)) and torch.equal(got[0][1], q[:, :, :, m - w:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_trees_on_16_byte_boundaries(dtype, d):
    gen = torch.Generator(device="cuda").manual_seed(7)
    T, seg = 21, Segments(gen, dtype, [5000, 31], d)
    cfg = config(dtype, 1, 1, 14, 2, d, 5000)
    q, k, v = normal(gen, (1, 1, 14, T, d), dtype), normal(gen, (1, 1, 2, T, d), dtype), normal(gen, (1, 1, 2, T, d), dtype)
    mask, ws, got = as_int64([[(1 << (i + 1)) - 1 for i in range(T)]]), mk.new_workspace(cfg), []
    for f in (lambda x: x, shifted):
        got.append(f(torch.full_like(q, SENTINEL)))
        mk.madakv_tree_attn(cfg, -1, f(q), f(k), f(v), mask, seg.k, seg.v, seg.seg_off, seg.kept_len, got[-1], None, ws)
    assert torch.equal(*got)


@pytest.mark.gpu
def test_results_between_the_rows_of_an_input():
    """Queries and results as two halves of the heads of one tensor: they share its memory and no element."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    n, d = 300, 64
    cfg = config("bf16", 2, 1, 3, 1, d, n)
    x = normal(gen, (2, 1, n, 6, d), "bf16").transpose(2, 3)
    q, out, k, v = x[:, :, :3], x[:, :, 3:], normal(gen, (2, 1, 1, n, d), "bf16"), normal(gen, (2, 1, 1, n, d), "bf16")
    mk.madakv_prefill_attn(cfg, 0, q, k, v, out, mk.new_workspace(cfg), seq_len=i32(n, n))
    want = torch.empty_like(q)
    mk.madakv_prefill_attn(cfg, 0, q, k, v, want, mk.new_workspace(cfg), seq_len=i32(n, n))
    assert torch.equal(out, want) and want.any()


# ------------------------------------------------------------------------------------------------- trees
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [260.0, 14.0, -300.0])
@pytest.mark.parametrize("n", [900, 6000])
def test_tree_logits_far_apart(dtype, d, size, n):
    """Single rows of the segment and single nodes whose logits stand far above or below the others; the longer segment is shared out."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    T, seg = 30, Segments(gen, dtype, [n], d)
    cfg = config(dtype, 1, 1, 2, 1, d, n)
    q, k, v = torch.full((1, 1, 2, T, d), d ** -0.5, device="cuda").to(DT[dtype]), normal(gen, (1, 1, 1, T, d), dtype), normal(gen, (1, 1, 1, T, d), dtype)
    q[:, :, 1] *= -0.5
    at = torch.arange(5, n, 37, device="cuda")
    seg.k[at] = (size * (1.0 + at / n * 0.5)).to(DT[dtype]).unsqueeze(1)
    k[0, 0, 0, 7::9] = size * 1.75
    out, lse = torch.empty_like(q), torch.empty((1, 1, 2, T), device="cuda")
    mk.madakv_tree_attn(cfg, -1, q, k, v, as_int64([[(1 << (i + 1)) - 1 for i in range(T)]]), seg.k, seg.v, seg.seg_off, seg.kept_len, out, lse,
                        mk.new_workspace(cfg))
    see = torch.cat((torch.ones((T, n), dtype=torch.bool, device="cuda"), causal(T)), 1)
    for h in range(2):
        check(dtype, q[0, 0, h], torch.cat((seg.k[:n], k[0, 0, 0])), torch.cat((seg.v[:n], v[0, 0, 0])), see, d ** -0.5, out[0, 0, h], lse[0, 0, h])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [300, 6000])
def test_tree_keys_that_are_no_numbers(dtype, d, n):
    """A NaN in a node's key: in the results of the nodes that see it; one in a row of a segment: in those of its heads and of no other's."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    T, seg = 20, Segments(gen, dtype, [n, n], d)
    cfg = config(dtype, 1, 1, 4, 2, d, n)
    q, k, v = normal(gen, (1, 1, 4, T, d), dtype), normal(gen, (1, 1, 2, T, d), dtype), normal(gen, (1, 1, 2, T, d), dtype)
    k[0, 0, 0, 8, 3] = math.nan
    seg.k[seg.off[1] + n - 7, d - 1] = math.nan
    masks = [[(1 << (i + 1)) - 1 if i % 2 == 0 else 1 << i for i in range(T)]]
    out, lse = torch.empty_like(q), torch.empty((1, 1, 4, T), device="cuda")
    mk.madakv_tree_attn(cfg, -1, q, k, v, as_int64(masks), seg.k, seg.v, seg.seg_off, seg.kept_len, out, lse, mk.new_workspace(cfg))
    assert out[0, 0, 2:].isnan().all() and lse[0, 0, 2:].isnan().all()
    bad = torch.tensor([bool(masks[0][i] >> 8 & 1) for i in range(T)], device="cuda")
    assert bad.any() and not bad.all()
    see = torch.tensor([[bool(masks[0][i] >> j & 1) for j in range(T)] for i in range(T)], device="cuda")
    see = torch.cat((torch.ones((T, n), dtype=torch.bool, device="cuda"), see), 1)[~bad]
    for h in range(2):
        assert out[0, 0, h, bad].isnan().all() and lse[0, 0, h, bad].isnan().all()
        check(dtype, q[0, 0, h, ~bad], torch.cat((seg.k[:n], k[0, 0, 0].nan_to_num(0.0))), torch.cat((seg.v[:n], v[0, 0, 0])), see, d ** -0.5,
              out[0, 0, h, ~bad], lse[0, 0, h, ~bad])


# ------------------------------------------------------------------------------------------------- workspaces
def test_workspaces_of_callers_without_attention_are_small(lib):  # noqa: F811
    """What a layer of 2048 tokens of 28 / 4 heads needs for eviction and decode is a few counters, log-sum-exps and partials."""
    assert mk.madakv_workspace_bytes(config("bf16", 1, 1, 28, 4, 128, 2048, 32)) < 2 << 20
    assert mk.madakv_workspace_bytes(config("f32", 1, 1, 4, 4, 64, 512, 8)) < 2 << 20


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_in_the_smallest_workspace(dtype, d):
    """No room for shares of the keys, room for some, room for all."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    n, m, T = 9000, 30, 9
    cfg = config(dtype, 1, 1, 4, 2, d, n)
    least, most = mk.madakv_workspace_bytes(cfg), mk.new_workspace(cfg).numel()
    q, k, v = normal(gen, (1, 1, 4, m, d), dtype), normal(gen, (1, 1, 2, n, d), dtype), normal(gen, (1, 1, 2, n, d), dtype)
    seg = Segments(gen, dtype, [n, 700], d)
    qt, kt, vt = normal(gen, (1, 1, 4, T, d), dtype), normal(gen, (1, 1, 2, T, d), dtype), normal(gen, (1, 1, 2, T, d), dtype)
    mask = as_int64([[(1 << (i + 1)) - 1 for i in range(T)]])
    for size in (least, least + 4 * m * 3 * (d + 2) * 4, most):
        space = torch.zeros(size + 4096, dtype=torch.uint8, device="cuda")
        space[size:] = 77
        ws = space[:size]
        out, lse, ot, yt = torch.empty_like(q), torch.empty((1, 1, 4, m), device="cuda"), torch.empty_like(qt), torch.empty((1, 1, 4, T), device="cuda")
        mk.madakv_prefill_attn(cfg, 0, q, k, v, out, ws, lse_out=lse, seq_len=i32(n), q_len=i32(m))
        mk.madakv_tree_attn(cfg, -1, qt, kt, vt, mask, seg.k, seg.v, seg.seg_off, seg.kept_len, ot, yt, ws)
        assert mk.madakv_poll_status(ws) == 0 and torch.all(space[size:] == 77)
        see = torch.arange(n, device="cuda") <= torch.arange(m, device="cuda").view(-1, 1) + n - m
        for h in range(4):
            a, rows = seg.off[h // 2], seg.lens[h // 2]
            check(dtype, q[0, 0, h], k[0, 0, h // 2], v[0, 0, h // 2], see, d ** -0.5, out[0, 0, h], lse[0, 0, h])
            check(dtype, qt[0, 0, h], torch.cat((seg.k[a:a + rows], kt[0, 0, h // 2])), torch.cat((seg.v[a:a + rows], vt[0, 0, h // 2])),
                  torch.cat((torch.ones((T, rows), dtype=torch.bool, device="cuda"), causal(T)), 1), d ** -0.5, ot[0, 0, h], yt[0, 0, h])


@pytest.mark.gpu
def test_many_tree_items_in_the_smallest_workspace():
    """More items than blocks: the list of them in the order of what they cost needs room too."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    B, H, T, d, lens = 2, 100, 3, 64, [70, 0, 150, 9]
    seg = Segments(gen, "bf16", [lens[u % 4] for u in range(B * H)], d)
    cfg = config("bf16", B, 1, H, H, d, 150)
    q, k, v = (normal(gen, (B, 1, H, T, d), "bf16") for _ in range(3))
    got = []
    for size in (mk.madakv_workspace_bytes(cfg), mk.new_workspace(cfg).numel()):
        space = torch.zeros(size + 4096, dtype=torch.uint8, device="cuda")
        space[size:] = 77
        got.append(torch.empty_like(q))
        mk.madakv_tree_attn(cfg, -1, q, k, v, as_int64([[1, 3, 7]] * B), seg.k, seg.v, seg.seg_off, seg.kept_len, got[-1], None, space[:size])
        assert mk.madakv_poll_status(space[:size]) == 0 and torch.all(space[size:] == 77)
    assert torch.equal(*got)


# ------------------------------------------------------------------------------------------------- refusals
def test_results_without_strides_are_refused(lib):  # noqa: F811
    """A dimension of out that the call writes and that has stride 0: rows would be written over one another."""
    c = config(B=2, L=2)
    S, short = mk.MadakvStrides, lambda cfg: mk.madakv_workspace_bytes(cfg) - 1  # (so that nothing is launched)
    st = S(2 * 4 * 512 * 128, 4 * 512 * 128, 512 * 128, 128)

    def prefill(so, q_off=None, cfg=c):
        return lib.madakv_prefill_attn(ctypes.byref(cfg), 0, FAKE, st, 512, q_off, None, FAKE, st, FAKE, st, 512, None, FAKE, FAKE, so, None, None, None,
                                       FAKE, short(cfg), None)

    def tree(so, layer=-1, cfg=c):
        return lib.madakv_tree_attn(ctypes.byref(cfg), layer, 5, FAKE, st, FAKE, st, FAKE, st, FAKE, None, FAKE, FAKE, FAKE, FAKE, 100, FAKE, so, None,
                                    FAKE, short(cfg), None)

    for call in (prefill, tree):
        assert call(st) == mk.EWORKSPACE
        assert call(S(0, st.layer, st.head, st.token)) == call(S(st.batch, st.layer, 0, st.token)) == mk.EINVAL
        assert call(S(0, st.layer, st.head, st.token), cfg=config(B=1, L=2)) == mk.EWORKSPACE  # (a dimension of one element)
    assert prefill(S(0, st.layer, st.head, st.token), q_off=FAKE) == mk.EWORKSPACE
    assert tree(S(st.batch, 0, st.head, st.token)) == mk.EINVAL and tree(S(st.batch, 0, st.head, st.token), layer=1) == mk.EWORKSPACE
    assert prefill(S(st.batch, 0, st.head, st.token)) == mk.EWORKSPACE  # (one layer is written)


def test_batch_strides_of_packed_sequences_are_not_used(lib):  # noqa: F811
    c = config(B=2)
    odd, st = mk.MadakvStrides(1, 4 * 512 * 128, 512 * 128, 128), mk.MadakvStrides(4 * 512 * 128, 4 * 512 * 128, 512 * 128, 128)

    def call(sq, skv, so, q_off, k_off):
        return lib.madakv_prefill_attn(ctypes.byref(c), 0, FAKE, sq, 512, q_off, None, FAKE, skv, FAKE, skv, 512, k_off, None if k_off else FAKE, FAKE, so,
                                       None, None, None, FAKE, mk.madakv_workspace_bytes(c) - 1, None)

    assert call(odd, odd, odd, FAKE, FAKE) == call(st, odd, st, None, FAKE) == call(odd, st, odd, FAKE, None) == mk.EWORKSPACE
    assert call(odd, st, st, None, None) == call(st, odd, st, None, None) == call(st, st, odd, None, FAKE) == call(st, odd, st, FAKE, None) == mk.EALIGN


@pytest.mark.gpu
def test_results_that_overlap_are_refused():
    gen = torch.Generator(device="cuda").manual_seed(1)
    cfg = config("bf16", 2, 1, 4, 2, 64, 32)
    q, k = normal(gen, (2, 1, 4, 32, 64), "bf16"), normal(gen, (2, 1, 2, 32, 64), "bf16")
    space = torch.zeros(2 * q.numel(), dtype=torch.bfloat16, device="cuda")
    part = lambda first, like: space[first:first + like.numel()].view(like.shape)  # noqa: E731
    ok = dict(q=part(0, q), k=k, v=k, out=part(q.numel(), q), ws=mk.new_workspace(cfg), seq_len=i32(32, 32))
    mk.madakv_prefill_attn(cfg, 0, **ok)
    win, lse = part(q.numel() - 64, torch.empty((2, 1, 4, 8, 64))), part(q.numel() - 64, torch.empty(2, 1, 4, 64)).view(torch.float32)
    alone = torch.empty((2, 1, 4, 32), device="cuda")
    for change in (dict(out=ok["q"]), dict(out=part(q.numel() - 64, q)), dict(q=k[:, :, :1].expand_as(q), out=part(0, q), v=part(64, k)),
                   dict(out=k.repeat(1, 1, 2, 1, 1), k=k, lse_out=alone, lse_win=alone.view(-1)[:64].view(2, 1, 4, 8)), dict(q_win=win), dict(lse_out=lse)):
        with pytest.raises(ValueError):
            mk.madakv_prefill_attn(cfg, 0, **{**ok, **change})
    with pytest.raises((ValueError, mk.MadakvError)):
        mk.madakv_prefill_attn(cfg, 0, **{**ok, "out": torch.empty_like(q)[:, :, :1].expand_as(q)})
    seg = Segments(gen, "bf16", [10, 11, 12, 13], 64)
    qt, kt = normal(gen, (2, 1, 4, 3, 64), "bf16"), normal(gen, (2, 1, 2, 3, 64), "bf16")
    tree = dict(q=qt, k_tree=kt, v_tree=kt, mask=torch.ones((2, 3), dtype=torch.int64, device="cuda"), k_c=seg.k, v_c=seg.v, seg_off=seg.seg_off,
                kept_len=seg.kept_len, out=torch.empty_like(qt), lse_out=None, ws=ok["ws"])
    mk.madakv_tree_attn(cfg, -1, **tree)
    for change in (dict(out=qt), dict(q=seg.k[:24].view(qt.shape), out=seg.k[:24].view(qt.shape)), dict(out=seg.v[2:26].view(qt.shape)),
                   dict(lse_out=tree["out"].view(-1)[:48].view(torch.float32).view(2, 1, 4, 3))):
        with pytest.raises(ValueError):
            mk.madakv_tree_attn(cfg, -1, **{**tree, **change})
    node = i32(0, 0)
    for change in (dict(k_tree=seg.v[:12].view(kt.shape)), dict(v_tree=seg.v[:12].view(kt.shape))):
        with pytest.raises(ValueError):
            mk.madakv_tree_commit(cfg, -1, tree["mask"], node, **{**{x: tree[x] for x in ("k_tree", "v_tree", "k_c", "v_c", "seg_off", "kept_len", "ws")}, **change})


@pytest.mark.gpu
def test_trims_name_every_call_that_leaves_positions_out():
    cfg = config("bf16", n=64)
    buf = mk.EvictionBuffers(cfg, 400, track=True)
    k = torch.zeros((1, 1, 4, 1, 128), device="cuda").bfloat16()
    buf.run_commit(torch.ones((1, 1), dtype=torch.int64, device="cuda"), i32(-1), k, k)
    with pytest.raises(ValueError, match="run_commit"):
        buf.run_trim(torch.zeros((1, 1, 4), dtype=torch.int32, device="cuda"), recent=2)
