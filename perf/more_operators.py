"""Attention over a prompt, and over a tree of drafted tokens on the ragged cache: the operators, their plain forms and the cases that are timed.

  prefill   causal attention of a prompt (or of its newest part over what is cached), whole or packed, one layer; with the outputs
            come the log-sum-exps, and the queries and log-sum-exps of the proxy tokens, from which eviction goes on
  tree      a speculative step: drafted tokens, a tree per sequence, attend over every head's segment of the ragged cache and their ancestors
  commit    the accepted path of every tree appended to the segments

Query i of a sequence with m queries and n keys stands at position n - m + i and sees the keys up to its position. Node i of a tree sees
the nodes whose bits are set in its mask (its ancestors and itself). A row that sees nothing has the result 0 and the log-sum-exp -inf.

A pass may be repeated on its state: commit puts lengths, positions and accumulated weights back at its start by one copy.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
WINDOW = 32


def _prefill(name, dtype, B, Hq, Hkv, d, n, m, spread=0.0, packed=False, fused=False, causal=True):
    """n keys and m queries a sequence (m = 0: as many as keys); packed: sequences behind one another; fused: q, k and v are parts of
    one projection's rows."""
    return dict(name=name, kind="prefill", dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, d=d, n=n, m=m, spread=spread, packed=packed, fused=fused,
                causal=causal)


def _tree(name, kind, dtype, B, L, Hq, Hkv, d, rows, spread, nodes, path, ragged=False):
    """Segments of about `rows` rows, trees of `nodes` nodes (ragged: fewer in some sequences) whose accepted path has `path`."""
    return dict(name=name, kind=kind, dtype=dtype, B=B, L=L, Hq=Hq, Hkv=Hkv, d=d, rows=rows, spread=spread, nodes=nodes, path=path,
                ragged=ragged)


def listed():
    return [
        # --- prompts
        # one layer of a grouped-query model on a long multimodal prompt: the largest
        _prefill("prefill_qwen", "bf16", 1, 28, 4, 128, 32768, 0),
        # one layer of a dense-attention model
        _prefill("prefill_llava", "bf16", 1, 32, 32, 128, 8192, 0),
        # a serving batch packed into one projection: sequences of different lengths, q, k and v are its columns
        _prefill("prefill_packed", "bf16", 12, 32, 8, 128, 3501, 0, 0.95, packed=True, fused=True),
        # chunked prefill: the newest 67 tokens of a long conversation over its cache; few rows, a long axis
        _prefill("prefill_chunk", "bf16", 2, 32, 8, 128, 100003, 67, 0.2),
        # the smallest prompt of a chat, one layer: latency counts
        _prefill("prefill_short", "bf16", 1, 28, 4, 128, 77, 0),
        # fp32 narrow heads, three prompts, odd lengths
        _prefill("prefill_f32", "f32", 3, 8, 2, 64, 2503, 0, 0.4),
        # --- speculative steps
        # a model's own order, one call per layer: a few segments, a small tree; latency counts
        _tree("tree_layer", "tree", "bf16", 1, 1, 28, 4, 128, 2048, 0.3, 16, 5),
        # dense attention, all layers in one call
        _tree("tree_llava", "tree", "bf16", 1, 32, 32, 32, 128, 1638, 0.3, 26, 5),
        # a serving batch with the largest trees, grouped queries
        _tree("tree_batched", "tree", "bf16", 8, 28, 28, 4, 128, 2512, 0.6, 64, 6, ragged=True),
        # fp32 narrow heads
        _tree("tree_f32", "tree", "f32", 3, 5, 8, 2, 64, 701, 0.6, 11, 3, ragged=True),
        # --- their accepted paths
        # one layer: latency counts
        _tree("commit_layer", "commit", "bf16", 1, 1, 28, 4, 128, 2048, 0.3, 16, 5),
        # all layers of a serving batch
        _tree("commit_batched", "commit", "bf16", 8, 28, 28, 4, 128, 1203, 0.6, 64, 17, ragged=True),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm, odd or even as it falls."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges; none has more work than the largest listed one of its kind."""
    kind = rng.choice(["prefill", "prefill", "prefill", "tree", "tree", "commit"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    Hq, Hkv = rng.choice([(4, 4), (32, 32), (40, 40), (28, 4), (28, 4), (32, 8), (32, 8), (8, 2), (16, 8), (24, 2)])
    d = 64 if rng.random() < 0.25 else 128
    if kind == "prefill":
        form = rng.choice(["whole", "packed", "chunk"])
        most = 28 * 32768 * 16384 // (40 if dtype == "f32" else 1)  # pairs of queries and keys, over all heads
        B = 1 if form == "whole" and rng.random() < 0.6 else rng.choice([1, 2, 3, 5, 8, 13])
        n = _log_int(rng, 1, 32768 if form != "chunk" else 131072)
        m = _log_int(rng, 1, min(n, 4096)) if form == "chunk" else 0
        while B * Hq * (m or n / 2) * n > most or B * n * (Hq + 2 * Hkv) * d > 1 << 30:
            if B > 1:
                B = (B + 1) // 2
            elif m > 16:
                m //= 2
            else:
                n = n * 2 // 3
                m = min(m, n)
        c = _prefill("", dtype, B, Hq, Hkv, d, n, m, round(rng.uniform(0.0, 0.95), 2) if B > 1 else 0.0, form == "packed",
                     form != "chunk" and rng.random() < 0.5, rng.random() < 0.9)
    else:
        B, L = rng.choice([1, 1, 1, 2, 3, 8]), rng.choice([1, 1, 1, 2, 5, 28, 32])
        rows, nodes = _log_int(rng, 1, 40000), _log_int(rng, 1, 64)
        most = 896 * 2512 // (8 if dtype == "f32" else 1)
        while B * L * Hkv * rows > most or B * L * Hq * rows * nodes > most * 7 * 64:
            if B > 1:
                B = (B + 1) // 2
            elif L > 1:
                L = (L + 1) // 2
            else:
                rows = rows * 2 // 3
        c = _tree("", kind, dtype, B, L, Hq, Hkv, d, rows, round(rng.uniform(0.0, 0.6), 2) if rows > 4 else 0.0, nodes,
                  rng.randint(1, min(nodes, 20)), rng.random() < 0.4)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------- inputs
def _uneven(count, around, spread, most):
    """`count` whole numbers around a value, uneven, at least 1."""
    frac = (np.arange(count, dtype=np.float64) + 1) * 0.6180339887498949 % 1.0
    return np.clip(np.floor(around * (1.0 + spread * (2.0 * frac - 1.0))).astype(np.int64), 1, most)


def _lengths(case):
    """Keys and queries of every sequence of a prefill."""
    n = _uneven(case["B"], case["n"], case["spread"], 2 * case["n"])
    return n, (np.minimum(n, case["m"]) if case["m"] else n)


def _node_counts(case):
    """Nodes of every sequence's tree: all, or where ragged between the path's and all."""
    if not case["ragged"]:
        return np.full(case["B"], case["nodes"])
    return case["path"] + np.arange(case["B"]) * 5 % (case["nodes"] - case["path"] + 1)


def _segments(case):
    return _uneven(case["B"] * case["L"] * case["Hkv"], case["rows"], case["spread"], 2 * case["rows"])


def _normal(gen, shape, dtype):
    """N(0, 1) in the case's type, made in pieces (the fp32 image of the largest tensors would not be small)."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 28
    for a in range(0, flat.numel(), step):
        part = flat[a:a + step]
        part.copy_(torch.randn(part.numel(), generator=gen, device="cuda", dtype=torch.float32))
    return out


def _towards(keys, q, g):
    """Adds to keys [H_kv, d] what makes nearly every query of q [H_q, rows, d] attend to them."""
    mean = q.float().mean(1).view(keys.shape[0], g, -1).mean(1)
    norm = (mean * mean).sum(1, keepdim=True)
    keys += (4.0 * math.sqrt(keys.shape[1]) * mean / norm.clamp_min(0.05)).to(keys.dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_prefill if case["kind"] == "prefill" else _prepare_tree)(case, seed, gen)


def _prepare_prefill(case, seed, gen):
    B, Hq, Hkv, d = (case[x] for x in ("B", "Hq", "Hkv", "d"))
    dtype, g = DTYPES[case["dtype"]], Hq // Hkv
    keys, queries = _lengths(case)
    n, m = int(keys.max()), int(queries.max())
    s = dict(case=case, g=g, scale=1.0 / math.sqrt(d))
    tokens = int(keys.sum()) if case["packed"] else n
    groups = 1 if case["packed"] else B  # packed: all sequences behind one another
    if case["fused"]:  # the columns of one projection's rows
        x = _normal(gen, (groups, tokens, Hq + 2 * Hkv, d), dtype)
        q, k, v = (y.transpose(1, 2).unsqueeze(1) for y in x.split([Hq, Hkv, Hkv], dim=2))
        out = torch.zeros((groups, tokens, Hq, d), dtype=dtype, device="cuda").transpose(1, 2).unsqueeze(1)
    else:
        q = _normal(gen, (groups, 1, Hq, tokens if case["packed"] else m, d), dtype)
        k, v = (_normal(gen, (groups, 1, Hkv, tokens, d), dtype) for _ in range(2))
        out = torch.zeros_like(q)
    q += 0.5 * _normal(gen, (Hq, 1, d), dtype)  # heads look into directions of their own
    lse = torch.zeros(q.shape[:4], device="cuda")
    start = np.concatenate([[0], np.cumsum(keys)]) if case["packed"] else np.zeros(B + 1, dtype=np.int64)
    seqs = []
    for b in range(B):  # every sequence's own part of the tensors, as views
        x, a = (0, int(start[b])) if case["packed"] else (b, 0)
        rows, cols = slice(a, a + int(queries[b])), slice(a, a + int(keys[b]))
        seqs.append((q[x, 0, :, rows], k[x, 0, :, cols], v[x, 0, :, cols], out[x, 0, :, rows], lse[x, 0, :, rows]))
        seqs[b][1][:, : int(keys[b]) // 2] += 0.5 * _normal(gen, (Hkv, 1, d), dtype)  # images: shifted per channel
        _towards(seqs[b][1][:, 0], seqs[b][0], g)
    s.update(q=q, k=k, v=v, out=out, lse=lse, seqs=seqs, q_win=torch.zeros((B, 1, Hq, WINDOW, d), dtype=dtype, device="cuda"),
             lse_win=torch.zeros((B, 1, Hq, WINDOW), device="cuda"))
    if case["packed"]:
        s.update(q=q[0], k=k[0], v=v[0], out=out[0], lse=lse[0], off=torch.from_numpy(start).cuda())
    s["seq_len"] = torch.from_numpy(keys.astype(np.int32)).cuda()
    s["q_len"] = torch.from_numpy(queries.astype(np.int32)).cuda()
    if own:
        from paper_2506_15724_b200 import binding as mk

        s["cfg"] = mk.make_config(dtype, B, 1, Hq, Hkv, d, n, WINDOW, causal=int(case["causal"]))
        s["ws"] = mk.new_workspace(s["cfg"])
        s["mk"] = mk
    return s


def _prepare_tree(case, seed, gen):
    B, L, Hq, Hkv, d, T = (case[x] for x in ("B", "L", "Hq", "Hkv", "d", "nodes"))
    dtype, g, units = DTYPES[case["dtype"]], Hq // Hkv, B * L * Hkv
    lens, counts = _segments(case), _node_counts(case)
    headroom = 64
    off = np.concatenate([[0], np.cumsum(lens + headroom)])
    cap, longest = int(off[-1]), int(lens.max())
    s = dict(case=case, g=g, scale=1.0 / math.sqrt(d), seg_off=torch.from_numpy(off).cuda())
    # trees: a chain of `path` nodes that is accepted, the others below any earlier node
    host = np.random.RandomState(seed % (1 << 32))
    mask, node = np.zeros((B, T), dtype=np.int64), np.zeros(B, dtype=np.int32)
    for b in range(B):
        chain = np.sort(host.choice(np.arange(1, counts[b]), case["path"] - 1, replace=False)) if case["path"] > 1 else np.zeros(0, int)
        chain = np.concatenate([[0], chain]).astype(int)
        parent = np.array([-1] + [host.randint(0, i) for i in range(1, counts[b])])
        parent[chain[1:]] = chain[:-1]
        bits = [0] * counts[b]
        for i in range(counts[b]):
            bits[i] = (bits[parent[i]] if i else 0) | 1 << i
        mask[b, :counts[b]] = np.array(bits, dtype=np.uint64).view(np.int64)
        node[b] = chain[-1]
    s.update(mask=torch.from_numpy(mask).cuda(), node=torch.from_numpy(node).cuda(), n_nodes=torch.from_numpy(counts.astype(np.int32)).cuda())
    s["q"] = _normal(gen, (B, L, Hq, T, d), dtype)
    s["q"] += 0.5 * _normal(gen, (L, Hq, 1, d), dtype)
    s["k_tree"], s["v_tree"], s["k_c"], s["v_c"] = (_normal(gen, x, dtype) for x in [(B, L, Hkv, T, d)] * 2 + [(cap, d)] * 2)
    first = s["seg_off"][:-1]
    sink = s["k_c"][first]
    _towards(sink, s["q"].view(B * L * Hq, T, d), g)
    s["k_c"][first] = sink
    # lengths, positions and accumulated weights, in one buffer so that one copy puts them back
    live = torch.zeros(units + 2 * cap, dtype=torch.int32, device="cuda")
    s.update(live=live, kept_len=live[:units], kept_idx=live[units:units + cap], acc=live[units + cap:].view(torch.float32))
    s["kept_len"].copy_(torch.from_numpy(lens))
    s["kept_idx"].copy_(torch.randint(0, 4 * longest, (cap,), generator=gen, device="cuda"))
    s["acc"].copy_(torch.exp(torch.randn(cap, generator=gen, device="cuda")) / case["rows"])
    s["position"] = torch.full((B,), 4 * longest, dtype=torch.int32, device="cuda")
    s["start"] = live.clone()
    if case["kind"] == "tree":
        s.update(out=torch.zeros_like(s["q"]), lse=torch.zeros((B, L, Hq, T), device="cuda"),
                 rows=torch.from_numpy(lens).cuda().view(-1, 1, 1),
                 pad=torch.from_numpy(np.minimum(off[:-1, None] + np.arange(longest), cap - 1)).cuda())
        see = (mask.view(np.uint64)[:, :, None] >> np.arange(T, dtype=np.uint64)) & np.uint64(1)
        s["see"] = torch.from_numpy(see.astype(bool)).cuda().view(B, 1, 1, T, T)  # of a node's row, a column per node
        s["there"] = (torch.arange(T, device="cuda") < s["n_nodes"].view(-1, 1)).view(B, 1, 1, T)
    else:
        # where the accepted rows come from and go to
        seq = np.arange(units) // (L * Hkv)
        path = [np.nonzero(mask[b].view(np.uint64)[node[b]] >> np.arange(T, dtype=np.uint64) & np.uint64(1))[0] for b in range(B)]
        source = np.concatenate([u * T + path[b] for u, b in enumerate(seq)])
        target = np.concatenate([off[u] + lens[u] + np.arange(case["path"]) for u in range(units)])
        s.update(source=torch.from_numpy(source).cuda(), target=torch.from_numpy(target).cuda(),
                 step=torch.arange(case["path"], dtype=torch.int32, device="cuda").repeat(units))
    if own:
        from paper_2506_15724_b200 import binding as mk

        s["cfg"] = mk.make_config(dtype, B, L, Hq, Hkv, d, longest, WINDOW, max_new_tokens=headroom)
        s["ws"] = mk.new_workspace(s["cfg"])
        s["mk"] = mk
    return s


# ------------------------------------------------------------------------------------------------- one pass
def run(s):
    return {"prefill": _run_prefill, "tree": _run_tree, "commit": _run_commit}[s["case"]["kind"]](s)


def _softmax(z):
    """Weights and log-sum-exps of logits z (changed); a row of -inf has weights 0."""
    top = z.amax(-1, keepdim=True).clamp_min_(torch.finfo(z.dtype).min)
    w = z.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    return w.div_(total.clamp_min(torch.finfo(z.dtype).tiny)), (top + total.log()).squeeze(-1)


def _run_prefill(s):
    if own:
        off = s.get("off")
        s["mk"].madakv_prefill_attn(s["cfg"], 0, s["q"], s["k"], s["v"], s["out"], s["ws"], lse_out=s["lse"], q_win=s["q_win"],
                                    lse_win=s["lse_win"], q_off=off, k_off=off, seq_len=None if off is not None else s["seq_len"],
                                    q_len=None if off is not None else s["q_len"])
        return {x: s[x] for x in ("out", "lse", "q_win", "lse_win")}
    case, g = s["case"], s["g"]
    s["q_win"].zero_()
    s["lse_win"].fill_(-math.inf)
    for b, (q, k, v, out, lse) in enumerate(s["seqs"]):
        (Hkv, n, d), m = k.shape, q.shape[1]
        k, v = k.float(), v.float()
        piece = max(1, min(m, (1 << 31) // (q.shape[0] * n)))  # queries at once: the logits of all would not fit
        for i in range(0, m, piece):
            j = min(m, i + piece)
            end = n - m + j if case["causal"] else n
            z = ((q[:, i:j].float() * s["scale"]).reshape(Hkv, g * (j - i), d) @ k[:, :end].mT).view(Hkv, g, j - i, end)
            if case["causal"]:
                at = torch.arange(n - m + i, n - m + j, device="cuda").view(-1, 1)
                z.masked_fill_(torch.arange(end, device="cuda") > at, -math.inf)
            w, y = _softmax(z)
            out[:, i:j] = (w.view(Hkv, g * (j - i), end) @ v[:, :end]).view(Hkv * g, j - i, d).to(out.dtype)
            lse[:, i:j] = y.view(Hkv * g, j - i)
        x = min(m, WINDOW)
        s["q_win"][b, 0, :, WINDOW - x:] = q[:, m - x:]
        s["lse_win"][b, 0, :, WINDOW - x:] = lse[:, m - x:]
    return {x: s[x] for x in ("out", "lse", "q_win", "lse_win")}


def _run_tree(s):
    if own:
        s["mk"].madakv_tree_attn(s["cfg"], -1, s["q"], s["k_tree"], s["v_tree"], s["mask"], s["k_c"], s["v_c"], s["seg_off"],
                                 s["kept_len"], s["out"], s["lse"], s["ws"], n_nodes=s["n_nodes"])
        return {"out": s["out"], "lse": s["lse"]}
    case, g = s["case"], s["g"]
    B, L, Hkv, T, d = s["k_tree"].shape
    units, longest = s["pad"].shape
    q = (s["q"].float() * s["scale"]).view(units, g * T, d)
    rows = s["pad"].view(-1)
    cached = q @ s["k_c"][rows].float().view(units, longest, d).mT
    cached.masked_fill_(torch.arange(longest, device="cuda") >= s["rows"], -math.inf)
    drafted = (q @ s["k_tree"].float().view(units, T, d).mT).view(B, L, Hkv * g, T, T).masked_fill_(~s["see"], -math.inf)
    w, lse = _softmax(torch.cat((cached, drafted.view(units, g * T, T)), dim=2))
    out = w[:, :, :longest] @ s["v_c"][rows].float().view(units, longest, d) + w[:, :, longest:] @ s["v_tree"].float().view(units, T, d)
    s["out"].copy_(torch.where(s["there"].unsqueeze(4), out.view(s["out"].shape).to(s["out"].dtype), s["out"]))
    s["lse"].copy_(torch.where(s["there"], lse.view(s["lse"].shape), s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _run_commit(s):
    s["live"].copy_(s["start"])
    if own:
        s["mk"].madakv_tree_commit(s["cfg"], -1, s["mask"], s["node"], s["k_tree"], s["v_tree"], s["k_c"], s["v_c"], s["seg_off"],
                                   s["kept_len"], s["ws"], acc=s["acc"], kept_idx=s["kept_idx"], position=s["position"])
    else:
        d, B = s["case"]["d"], s["case"]["B"]
        s["k_c"][s["target"]] = s["k_tree"].view(-1, d)[s["source"]]
        s["v_c"][s["target"]] = s["v_tree"].view(-1, d)[s["source"]]
        s["kept_idx"][s["target"]] = s["position"].repeat_interleave(s["step"].numel() // B) + s["step"]
        s["acc"][s["target"]] = 0.0
        s["kept_len"] += s["case"]["path"]
    return {x: s[x] for x in ("k_c", "v_c", "kept_len", "kept_idx", "acc")}


# ------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """What a pass returns, in 64 bits; what is only copied or counted, as all of a commit, has no such value."""
    if case["kind"] == "commit":
        return None
    s = prepare(case, seed)
    return _exact_prefill(s) if case["kind"] == "prefill" else _exact_tree(s)


def _exact_prefill(s):
    case, g = s["case"], s["g"]
    dim = case["d"] ** 0.5
    out, lse = torch.zeros_like(s["out"], dtype=torch.float64), torch.zeros_like(s["lse"], dtype=torch.float64)
    window = torch.full_like(s["lse_win"], -math.inf, dtype=torch.float64)
    at = [0] * case["B"] if "off" not in s else s["off"].tolist()
    for b, (q, k, v, _, _) in enumerate(s["seqs"]):
        (heads, m, d), n = q.shape, k.shape[1]
        for h in range(heads):
            kk, vv = k[h // g].double(), v[h // g].double()
            here = (0, h) if "off" in s else (b, 0, h)
            o, y = out[here], lse[here]
            step = max(1, (1 << 26) // n)
            for i in range(0, m, step):
                j = min(m, i + step)
                z = q[h, i:j].double() @ kk.T / dim
                if case["causal"]:
                    z += torch.full_like(z, -math.inf).triu_(n - m + i + 1)
                y[at[b] + i:at[b] + j] = torch.logsumexp(z, 1)
                o[at[b] + i:at[b] + j] = torch.exp(z - y[at[b] + i:at[b] + j, None]) @ vv
            x = min(m, WINDOW)
            window[b, 0, h, WINDOW - x:] = y[at[b] + m - x:at[b] + m]
    return {"out": out, "lse": lse, "q_win": None, "lse_win": window}


def _exact_tree(s):
    case, g = s["case"], s["g"]
    B, L, H, T, d = s["q"].shape
    out, lse = torch.zeros_like(s["q"], dtype=torch.float64), torch.zeros((B, L, H, T), dtype=torch.float64, device="cuda")
    off, lens, counts = s["seg_off"].tolist(), _segments(case).tolist(), _node_counts(case).tolist()
    hidden = [torch.where(s["see"][b, 0, 0], 0.0, -math.inf).double() for b in range(B)]
    for u, rows in enumerate(lens):
        b, l, h = u // (L * case["Hkv"]), u // case["Hkv"] % L, u % case["Hkv"]
        k = torch.cat((s["k_c"][off[u]:off[u] + rows], s["k_tree"][b, l, h])).double()
        v = torch.cat((s["v_c"][off[u]:off[u] + rows], s["v_tree"][b, l, h])).double()
        z = s["q"][b, l, h * g:(h + 1) * g].double() @ k.T / d ** 0.5
        z[:, :, rows:] += hidden[b]
        y = torch.logsumexp(z, 2)
        o = torch.exp(z - y.unsqueeze(2)) @ v
        lse[b, l, h * g:(h + 1) * g, :counts[b]] = y[:, :counts[b]]
        out[b, l, h * g:(h + 1) * g, :counts[b]] = o[:, :counts[b]]
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------------------------- cost
def work(case):
    d, Hq, Hkv, e = case["d"], case["Hq"], case["Hkv"], 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "prefill":
        # q, k, v read, the results and log-sum-exps written, the proxy tokens' queries and log-sum-exps written
        keys, queries = _lengths(case)
        seen = queries * (keys - (queries - 1) / 2) if case["causal"] else queries * keys
        proxy = np.minimum(queries, WINDOW).sum()
        moved = (2 * Hq * queries.sum() + 2 * Hkv * keys.sum() + Hq * proxy) * d * e + 4 * Hq * (queries.sum() + proxy)
        return {"bytes": float(moved), "flops": float(4 * Hq * d * seen.sum())}
    lens, counts = _segments(case), _node_counts(case)
    if case["kind"] == "commit":
        # accepted rows of K and V read and written, their positions and weights written
        rows = len(lens) * case["path"]
        return {"bytes": float(rows * (4 * d * e + 8)), "flops": float(rows)}
    # segments and drafted rows read; queries read, results and log-sum-exps written
    rows = case["L"] * counts.sum()
    per = counts.repeat(case["L"] * Hkv)
    moved = lens.sum() * 2 * d * e + rows * (2 * Hkv * d * e + Hq * (2 * d * e + 4))
    return {"bytes": float(moved), "flops": float(4 * d * Hq // Hkv * (per * (lens + (per + 1) / 2)).sum())}
