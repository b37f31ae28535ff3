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


# ------------------------------------------------------------------------------------------------- strides
def shifted(x):
    """The same numbers in rows that begin on 16-byte boundaries of which no two neighbours are 32-byte ones."""
    e = 16 // x.element_size()
    y = torch.full((*x.shape[:-1], x.shape[-1] + e), SENTINEL, device="cuda").to(x.dtype)[..., e:]
    y.copy_(x)
    return y
