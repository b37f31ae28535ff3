"""The proxy tokens' queries and log-sum-exps on their way from the attention of a prompt to eviction: prompts in one call and in chunks, what
eviction goes on from, what it refuses. Scores are compared with Eq. 7 in 64 bits; tolerances are sums of roundings."""
import ctypes
import math

import pytest
import torch

from paper_2506_15724_b200 import binding as mk
from test_prompt_and_trees import FAKE, lib  # noqa: F401

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(DT[dtype])


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def scores(q_win, k, lens, w, causal=1, drop=None):
    """Eq. 7 in 64 bits and how far a score may be off: [B, L, H_kv, n] each. drop [B, L, H_q, w]: rows without weight.
    A logit is a sum of d products in fp32, each addition off by at most a step (d + 8 steps of the sum of magnitudes), once in the log-sum-exp and
    once in the scores, where the log-sum-exp is part of the sum; it is rounded itself (four half steps), sums over keys and over rows are an addition
    per 16 at most and 64 more, an exponential is off by less than 8 half steps."""
    B, L, Hq, _, d = q_win.shape
    Hkv, n = k.shape[2], k.shape[3]
    g = Hq // Hkv
    want, most = (torch.zeros((B, L, Hkv, n), dtype=torch.float64, device="cuda") for _ in range(2))
    for b in range(B):
        m = lens[b]
        at = torch.arange(w, device="cuda") + m - w
        see = (torch.arange(m, device="cuda") <= at.view(-1, 1)) if causal else (at >= 0).view(-1, 1).expand(w, m)
        for l in range(L):
            for h in range(Hq):
                q, kk = q_win[b, l, h].double(), k[b, l, h // g, :m].double()
                z = (q @ kk.T * d ** -0.5).masked_fill(~see, -math.inf)
                lse = torch.logsumexp(z, 1) if m else torch.full((w,), -math.inf, dtype=torch.float64, device="cuda")
                gone = lse.isinf() if drop is None else lse.isinf() | drop[b, l, h]
                p = torch.exp(z - lse.masked_fill(gone, 0.0).unsqueeze(1)).masked_fill(gone.unsqueeze(1), 0.0)
                if not m:
                    continue
                mag = (q.abs() @ kk.abs().T * see).amax(1) * d ** -0.5
                size = lse.masked_fill(gone, 0.0).abs()
                off = (d + 8) * 2.0 ** -23 * (2 * mag + size) + 4 * 2.0 ** -24 * size + (m / 16 + g * w / 16 + 136) * 2.0 ** -23
                want[b, l, h // g, :m] += p.sum(0)
                most[b, l, h // g, :m] += (p * off.unsqueeze(1)).sum(0)
    return want, most + 1e-30


def check_scores(psi, want, most):
    err = (psi.double() - want).abs()
    assert torch.all(err <= most), float((err / most).max())  # (a NaN fails)


@pytest.mark.gpu
@pytest.mark.parametrize("path", ["auto", "generic"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,w", [(4, 4, 64, 8), (7, 1, 128, 32)])
def test_rows_without_normaliser_have_no_weight(dtype, path, Hq, Hkv, d, w, monkeypatch):
    """A log-sum-exp of -inf given for rows that do see keys: they add nothing, whichever kernel takes the call."""
    if path == "generic":
        monkeypatch.setenv("MADAKV_SCORE_PATH", "generic")
    gen = torch.Generator(device="cuda").manual_seed(1)
    B, L, n, lens = 2, 2, 300, [300, 190]
    cfg = mk.make_config(DT[dtype], B, L, Hq, Hkv, d, n, w)
    ws = mk.new_workspace(cfg)
    q, k = normal(gen, (B, L, Hq, w, d), dtype), normal(gen, (B, L, Hkv, n, d), dtype)
    lse, psi = torch.zeros((B, L, Hq, w), device="cuda"), torch.zeros((B, L, Hkv, n), device="cuda")
    mk.madakv_score(cfg, q, k, i32(*lens), lse, psi, ws)
    check_scores(psi, *scores(q, k, lens, w))
    drop = torch.rand(lse.shape, generator=gen, device="cuda") < 0.4
    drop[0, 0] = True
    mk.madakv_score_lse(cfg, q, k, i32(*lens), lse.masked_fill(drop, -math.inf), psi, ws)
    check_scores(psi, *scores(q, k, lens, w, drop=drop))
    assert not psi[0, 0].any() and mk.madakv_poll_status(ws) == 0


def test_keeping_windows_refusals_before_any_launch(lib):  # noqa: F811
    c = mk.make_config(torch.bfloat16, 1, 1, 4, 4, 128, 512, 8)
    need, st = mk.madakv_workspace_bytes(c), mk.MadakvStrides(4 * 512 * 128, 4 * 512 * 128, 512 * 128, 128)

    def call(q=FAKE, q_len=None, q_win=FAKE, lse_win=FAKE, win_len=FAKE, size=need - 1):
        return lib.madakv_prefill_attn_keep(ctypes.byref(c), 0, q, st, 512, None, q_len, FAKE, st, FAKE, st, 512, None, FAKE, FAKE, st, None, q_win, lse_win,
                                            win_len, FAKE, size, None)

    assert call() == call(q_len=FAKE) == mk.EWORKSPACE
    assert call(q=None) == call(q_win=None) == call(lse_win=None) == call(win_len=None) == mk.EINVAL
    assert call(win_len=ctypes.c_void_p(0x10002)) == call(lse_win=ctypes.c_void_p(0x10002)) == call(q_win=ctypes.c_void_p(0x10004)) == mk.EALIGN


def test_scores_of_kept_windows_refusals_before_any_launch(lib):  # noqa: F811
    c = mk.make_config(torch.bfloat16, 1, 1, 4, 4, 128, 512, 8)
    need, st = mk.madakv_workspace_bytes(c), mk.MadakvStrides(4 * 512 * 128, 4 * 512 * 128, 512 * 128, 128)

    def call(q=FAKE, k=FAKE, seq=FAKE, lse=FAKE, win_len=FAKE, psi=FAKE, size=need):
        return lib.madakv_score_kept(ctypes.byref(c), q, st, k, st, seq, lse, win_len, psi, FAKE, size, None)

    assert call(q=None) == call(k=None) == call(seq=None) == call(lse=None) == call(win_len=None) == call(psi=None) == mk.EINVAL
    assert call(win_len=ctypes.c_void_p(0x10002)) == call(lse=ctypes.c_void_p(0x10002)) == call(q=ctypes.c_void_p(0x10004)) == mk.EALIGN
    assert call(size=need - 1) == mk.EWORKSPACE


class Prompt:
    """A prompt of several layers, buffers for it, and the calls of a user that goes through it."""

    def __init__(self, dtype, lens, w=16, L=2, Hq=8, Hkv=2, d=64, causal=1, seed=3):
        self.gen, self.dtype, self.lens, self.w, self.L, self.causal = torch.Generator(device="cuda").manual_seed(seed), dtype, lens, w, L, causal
        self.B, self.Hq, self.Hkv, self.d, self.n = len(lens), Hq, Hkv, d, max(lens)
        self.cfg = mk.make_config(DT[dtype], self.B, L, Hq, Hkv, d, self.n, w, causal=causal, max_new_tokens=4)
        self.buf = mk.EvictionBuffers(self.cfg, self.B * L * Hkv * (self.n + 4), want_lse=True)
        self.mask = torch.zeros((self.B, self.n), dtype=torch.uint8, device="cuda")
        self.mask[:, 3:self.n // 2] = 1
        self.budget = i32(*[max(1, x // 5) for x in lens])
        self.new()

    def new(self):  # another prompt of the same lengths
        shape = lambda h: (self.B, self.L, h, self.n, self.d)  # noqa: E731
        self.q, self.k, self.v = (normal(self.gen, shape(h), self.dtype) for h in (self.Hq, self.Hkv, self.Hkv))
        self.out = torch.zeros_like(self.q)

    def chunk(self, layer, begin, end, packed=False):
        """Queries begin .. end - 1 of every sequence that has them; keys that come later are not there yet."""
        keys = [min(x, end) for x in self.lens]
        count = [max(0, x - begin) for x in keys]
        if not packed:
            rows = slice(begin, max(begin + 1, min(end, self.n)))
            return self.buf.run_prefill(layer, self.q[:, :, :, rows], self.k, self.v, self.out[:, :, :, rows], seq_len=i32(*keys), q_len=i32(*count))
        if not sum(count):
            return
        q = torch.cat([self.q[b, :, :, begin:begin + count[b]] for b in range(self.B)], 2)
        off = [sum(count[:b]) for b in range(self.B + 1)]
        out = torch.zeros_like(q)
        self.buf.run_prefill(layer, q, self.k, self.v, out, seq_len=i32(*keys), q_off=torch.tensor(off, device="cuda"))
        for b in range(self.B):
            self.out[b, layer, :, begin:begin + count[b]] = out[layer, :, off[b]:off[b + 1]]

    def whole(self, layers=None):
        for layer in range(self.L) if layers is None else layers:
            self.buf.run_prefill(layer, self.q, self.k, self.v, self.out, seq_len=i32(*self.lens))

    def evict(self, q_win=None, lens=None):
        self.buf.run_eviction(q_win, self.k, self.v, self.mask, i32(*(lens or self.lens)), self.budget)

    def window(self):
        x = torch.zeros((self.B, self.L, self.Hq, self.w, self.d), device="cuda").to(DT[self.dtype])
        for b, m in enumerate(self.lens):
            x[b, :, :, max(0, self.w - m):] = self.q[b, :, :, max(0, m - self.w):m]
        return x

    def check(self):
        """The window and the scores that the last eviction went by are those of the whole prompt."""
        assert mk.madakv_poll_status(self.buf.ws) == 0
        assert torch.equal(self.buf.q_win, self.window())
        check_scores(self.buf.psi, *scores(self.window(), self.k, self.lens, self.w, self.causal))

    def refused(self):
        assert mk.madakv_poll_status(self.buf.ws) == mk.ESHAPE


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,w,ends", [(64, 16, [200, 400, 495, 500]), (128, 16, [497, 498, 500]), (64, 32, [3, 10, 40, 41, 60, 333, 334, 500]),
                                      (64, 1, [499, 500]), (128, 40, [5, 333, 363, 393, 423, 453, 483, 500]), (64, 300, [100, 350, 450, 500])])
def test_eviction_after_a_prompt_in_chunks(dtype, d, w, ends, packed):
    """Chunks shorter than the window, sequences that end in earlier chunks than others, one shorter than the window."""
    p = Prompt(dtype, [500, 333, 9, 41], w=w, d=d)
    for begin, end in zip([0] + ends, ends):
        for layer in range(p.L):
            p.chunk(layer, begin, end, packed)
    p.evict()
    p.check()


@pytest.mark.gpu
def test_eviction_after_a_prompt_token_by_token():
    p = Prompt("bf16", [60, 23], w=24)
    for layer in range(p.L):
        for i in range(60):
            p.chunk(layer, i, i + 1)
    p.evict()
    p.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_longer_prompt_goes_on_from_a_whole_one(dtype):
    """A call of as many queries as keys, then a few tokens more."""
    p = Prompt(dtype, [300, 200])
    for layer in range(p.L):
        p.buf.run_prefill(layer, p.q[:, :, :, :290], p.k[:, :, :, :290], p.v[:, :, :, :290], p.out[:, :, :, :290], seq_len=i32(290, 200))
    for layer in range(p.L):
        p.chunk(layer, 290, 300)
    p.evict()
    p.check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("last", [0, 5, 40])
def test_eviction_after_a_packed_prompt(dtype, last):
    """Queries and keys behind one another, at once or with a last chunk; K and V in padded form for the eviction."""
    p = Prompt(dtype, [300, 9, 120, 200], w=24)
    flat = lambda x, a, e: torch.cat([x[b, :, :, a(m):e(m)] for b, m in enumerate(p.lens)], 2)  # noqa: E731
    off = lambda a, e: torch.tensor([sum(e(m) - a(m) for m in p.lens[:b]) for b in range(p.B + 1)], device="cuda")  # noqa: E731
    first, zero, full = lambda m: max(0, m - last), lambda m: 0, lambda m: m  # noqa: E731
    for begin, end in [(zero, full)] if not last else [(zero, first), (first, full)]:
        q, k, v, k_off = flat(p.q, begin, end), flat(p.k, zero, end), flat(p.v, zero, end), off(zero, end)
        q_off = off(begin, end) if begin is first else k_off
        for layer in range(p.L):
            p.buf.run_prefill(layer, q, k, v, torch.empty_like(q), q_off=q_off, k_off=k_off)
    p.evict()
    p.check()


@pytest.mark.gpu
def test_a_given_window_leaves_the_kept_one_alone():
    """Eviction by queries of the caller's between a prefill and the eviction that goes on from it."""
    p = Prompt("bf16", [300, 200])
    p.whole()
    other = normal(p.gen, p.window().shape, "bf16") * 2.0
    p.evict(other)
    check_scores(p.buf.psi, *scores(other, p.k, p.lens, p.w))
    p.evict()
    p.check()


@pytest.mark.gpu
def test_eviction_refuses_a_layer_that_was_never_run():
    p = Prompt("bf16", [300, 200], L=3)
    with pytest.raises(ValueError):
        p.evict()
    p.whole([0, 2])
    with pytest.raises(ValueError):
        p.evict()
    p.whole([1])
    p.evict()
    p.check()


@pytest.mark.gpu
def test_eviction_reports_windows_of_different_prompts():
    """A second prompt whose prefill has not reached every layer: some windows are still the first prompt's."""
    p = Prompt("bf16", [300, 200], L=3)
    p.whole()
    p.evict()
    p.check()
    first = p.buf.kept_idx.clone()
    p.evict()  # the same again
    p.check()
    assert torch.equal(first, p.buf.kept_idx)
    p.new()
    p.whole([1])
    p.evict()
    p.refused()
    p.evict()  # (it stays refused)
    p.refused()
    p.whole([0, 2])
    p.evict()
    p.check()


@pytest.mark.gpu
def test_eviction_reports_windows_of_other_lengths():
    p = Prompt("bf16", [300, 200])
    p.whole()
    p.evict(lens=[300, 199])
    p.refused()
    p.evict()
    p.check()


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [0, 1])
def test_eviction_reports_incomplete_windows(causal):
    """Fewer new queries than proxy tokens, and nothing before them (or, where every query sees every key, keys that they did not see)."""
    p = Prompt("bf16", [300, 200], causal=causal)
    for layer in range(p.L):
        p.chunk(layer, 290, 300)
    p.evict()
    p.refused()
    for ends in ([300], [100, 290, 300], [150, 300]):
        p.new()
        for layer in range(p.L):
            for begin, end in zip([0] + ends, ends):
                p.chunk(layer, begin, end)
        p.evict()
        if causal == 0 and ends == [100, 290, 300]:
            p.refused()
        else:
            p.check()
    # a prompt whose eviction has been is not gone on from: what stands before may be another's
    p.new()
    for layer in range(p.L):
        p.chunk(layer, 295, 300)
    p.evict()
    p.refused()


@pytest.mark.gpu
def test_captured_chunks_and_evictions():
    """Chunks and eviction in a graph, replayed for other prompts; and chunks in graphs of their own."""
    p = Prompt("bf16", [300, 200])
    ends = [150, 296, 300]
    spans = list(zip([0] + ends, ends))
    counts = [(i32(*[min(x, e) for x in p.lens]), i32(*[max(0, min(x, e) - b) for x in p.lens])) for b, e in spans]
    lens = i32(*p.lens)

    def prefill(span):
        (begin, end), (keys, count) = spans[span], counts[span]
        for layer in range(p.L):
            p.buf.run_prefill(layer, p.q[:, :, :, begin:end], p.k, p.v, p.out[:, :, :, begin:end], seq_len=keys, q_len=count)

    def evict():
        p.buf.run_eviction(None, p.k, p.v, p.mask, lens, p.budget)

    graphs = [torch.cuda.CUDAGraph() for _ in range(5)]
    for graph, calls in zip(graphs, ([lambda i=i: prefill(i) for i in range(3)] + [evict], *[[lambda i=i: prefill(i)] for i in range(3)], [evict])):
        with torch.cuda.graph(graph):
            for call in calls:
                call()
    for run in (graphs[:1], graphs[1:], graphs[:1]):
        q, k = normal(p.gen, p.q.shape, "bf16"), normal(p.gen, p.k.shape, "bf16")
        p.q.copy_(q), p.k.copy_(k)
        for graph in run:
            graph.replay()
        p.check()
