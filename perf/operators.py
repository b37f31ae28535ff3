"""Decode on a bounded ragged cache, in full precision or in 4 bits: the operators, their plain forms and the cases that are timed.

  compact       kept rows of K and V gathered into the ragged cache in 4 bits, and read back
  decode_quant  a decode step on the cache in 4 bits: a row appended per head, attention, weights accumulated where asked
  decode        a decode step on the bf16 or fp32 cache that also accumulates every row's attention weight
  evict         segments cut back to their limit by accumulated weight, in place (bf16, fp32 or 4 bits)

A row of the cache in 4 bits: groups of 32 elements with mid = bf16((lo + hi) / 2), step = bf16((hi - lo) / 15), clamp(floor((x - mid) / step) + 8, 0, 15), value = mid + (code - 7.5) * step. The code of element 32 G + 4 i + e (i < 8, e < 4)
is nibble e of the row's 16-bit word i * (d / 32) + G.

A pass may be repeated on its state: lengths, positions and accumulated weights are put back at its start by one copy, what a
step appends it appends again, and the rows that eviction moves it takes from behind the new end, which it does not write.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 32


def _case(name, kind, dtype, B, L, Hq, Hkv, d, n, rows, spread, **kw):
    c = dict(name=name, kind=kind, dtype=dtype, B=B, L=L, Hq=Hq, Hkv=Hkv, d=d, n=n, rows=rows, spread=spread, append=True,
             track=kind == "decode", quant=kind in ("compact", "decode_quant"), over=0, recent=0)
    c.update(kw)
    return c


def listed():
    return [
        # --- after prefill: the kept rows into 4 bits
        # one layer of a grouped-query model, as it is compacted right after its own prefill
        _case("compact_layer", "compact", "bf16", 1, 1, 28, 4, 128, 32768, 2048, 0.3),
        # the ordinary prompt of a dense-attention model, all layers at once: the largest gather
        _case("compact_llava", "compact", "bf16", 1, 32, 32, 32, 128, 8192, 1638, 0.3),
        # fp32 cache of narrow heads, three prompts, odd lengths
        _case("compact_f32", "compact", "f32", 3, 5, 8, 2, 64, 5003, 701, 0.6),
        # --- decode steps on the cache in 4 bits
        # a model's own order, one call per layer: four segments, 7 query heads per KV head; latency counts
        _case("quant_layer", "decode_quant", "bf16", 1, 1, 28, 4, 128, 32768, 2048, 0.3),
        # dense attention, all layers in one call
        _case("quant_llava", "decode_quant", "bf16", 1, 32, 32, 32, 128, 8192, 1638, 0.3),
        # a serving batch that will evict: weights are accumulated too
        _case("quant_batched", "decode_quant", "bf16", 8, 28, 28, 4, 128, 16384, 2512, 0.6, track=True),
        # nothing evicted: the whole context of one layer of a long prompt, in 4 bits
        _case("quant_full", "decode_quant", "bf16", 1, 1, 32, 8, 128, 131072, 131071, 0.0),
        # fp32 queries on narrow heads
        _case("quant_f32", "decode_quant", "f32", 3, 5, 8, 2, 64, 5003, 701, 0.6, track=True),
        # --- decode steps that accumulate weights on the cache in its own type
        _case("track_layer", "decode", "bf16", 1, 1, 32, 8, 128, 131072, 2952, 0.4),
        _case("track_llava", "decode", "bf16", 1, 32, 32, 32, 128, 8192, 1638, 0.3),
        # --- eviction while decoding
        # one layer, a row too many in each of its segments: done at every step, latency counts
        _case("evict_layer", "evict", "bf16", 1, 1, 28, 4, 128, 32768, 2049, 0.3, quant=True, over=1, recent=32),
        # dense attention, all layers, after 64 steps
        _case("evict_llava", "evict", "bf16", 1, 32, 32, 32, 128, 8192, 1702, 0.3, over=64, recent=32),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], uniform in its logarithm, odd or even as it falls."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges; none has more cache rows than the largest listed ones."""
    kind = rng.choice(["compact", "decode_quant", "decode_quant", "decode_quant", "decode", "decode", "evict", "evict"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    heads = [(4, 4), (32, 32), (40, 40), (28, 4), (28, 4), (32, 8), (32, 8), (8, 2), (16, 8)]
    if dtype == "bf16":
        heads += [(32, 2), (24, 2)]
    Hq, Hkv = rng.choice(heads)
    d = 64 if rng.random() < 0.25 else 128
    B = rng.choice([1, 1, 1, 2, 3, 8])
    L = rng.choice([1, 1, 1, 2, 5, 28, 32, 40])
    rows = _log_int(rng, 1, 40000)
    most = 1024 * 1638 // (2 if dtype == "f32" else 1)
    if Hq // Hkv > 8:
        most //= 4
    while B * L * Hkv * rows > most:
        if B > 1:
            B = (B + 1) // 2
        elif L > 1:
            L = (L + 1) // 2
        else:
            rows = rows * 2 // 3
    spread = round(rng.uniform(0.0, 0.6), 2) if rows > 4 else 0.0
    n = max(rows + 1, int(rows * rng.uniform(1.7, 5.0)))
    if kind == "compact":
        while B * L * Hkv * n * d * (4 if dtype == "f32" else 2) > 1 << 31 and n > 2 * rows:
            n = max(2 * rows, n * 2 // 3)
    c = _case("", kind, dtype, B, L, Hq, Hkv, d, n, rows, spread)
    del c["name"]
    if kind == "decode_quant":
        c.update(track=rng.random() < 0.5)
    if kind.startswith("decode"):
        c.update(append=rng.random() < 0.8)
    if kind == "evict":
        over = min(max(1, rows // 2), _log_int(rng, 1, 256))
        c.update(quant=rng.random() < 0.4, over=over, recent=min(rng.choice([0, 1, 16, 32, 64]), max(0, rows // 4)))
    return c


# ------------------------------------------------------------------------------------------------- the plain quantiser
def _quantise(x):
    """Codes [rows, d] and (step, mid) [rows, d / 32, 2] bf16 of fp32 rows [rows, d]. An element next to a border between two
    codes needs 64 bits."""
    g = x.view(x.shape[0], -1, GROUP).double()
    lo, hi = g.amin(2), g.amax(2)
    mid = ((lo + hi) / 2).float().to(torch.bfloat16)
    step = ((hi - lo) / 15).float().to(torch.bfloat16)
    code = torch.floor((g - mid.double().unsqueeze(2)) / step.double().unsqueeze(2)).add_(8).clamp_(0, 15)
    code = torch.where(step.unsqueeze(2) > 0, code, 8.0).to(torch.uint8)
    return code.view(x.shape), torch.stack((step, mid), dim=2)


def _values(code, par):
    """fp32 values of codes [rows, d] under their (step, mid)."""
    c = code.view(code.shape[0], -1, GROUP).float().sub_(7.5)
    return c.mul_(par[:, :, :1].float()).add_(par[:, :, 1:].float()).view(code.shape)


def _pack(code):
    c = code.view(code.shape[0], -1, 8, 2, 2).transpose(1, 2)
    return (c[..., 0] | (c[..., 1] << 4)).reshape(code.shape[0], -1)


def _unpack(packed, d):
    b = packed.view(packed.shape[0], 8, d // GROUP, 2)
    return torch.stack((b & 15, b >> 4), dim=4).transpose(1, 2).reshape(packed.shape[0], d)


# ------------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """Rows of every (sequence, layer, KV head) before the pass: around case["rows"], uneven from head to head."""
    u = np.arange(case["B"] * case["L"] * case["Hkv"], dtype=np.float64)
    frac = (u + 1) * 0.6180339887498949 % 1.0
    rows = np.floor(case["rows"] * (1.0 + case["spread"] * (2.0 * frac - 1.0))).astype(np.int64)
    return np.clip(rows, 1, case["n"])


def _normal(gen, shape, dtype):
    """N(0, 1) in the case's type, made in pieces (the fp32 image of the largest tensors would not be small)."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 28
    for a in range(0, flat.numel(), step):
        part = flat[a:a + step]
        part.copy_(torch.randn(part.numel(), generator=gen, device="cuda", dtype=torch.float32))
    return out


def _positions(gen, lens, n):
    """Ascending random positions below n, lens[u] of them for every unit, one unit behind the other."""
    r = torch.rand((len(lens), n), generator=gen, device="cuda").argsort(dim=1).to(torch.int32)
    kept = torch.zeros_like(r, dtype=torch.bool)
    lens = torch.from_numpy(lens).cuda().view(-1, 1)
    kept.scatter_(1, r.long(), torch.arange(n, device="cuda").view(1, -1) < lens)
    return kept.nonzero()[:, 1].to(torch.int32)


def prepare(case, seed):
    kind, B, L, Hq, Hkv, d, n = (case[x] for x in ("kind", "B", "L", "Hq", "Hkv", "d", "n"))
    dtype, g, units = DTYPES[case["dtype"]], Hq // Hkv, B * L * Hkv
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = _lengths(case)
    headroom = 16 if kind != "evict" else case["over"] + 1
    before = lens - case["over"] if kind == "evict" else lens  # the rows that were kept at prefill
    before = np.maximum(before, 1)
    off = np.concatenate([[0], np.cumsum(before + headroom)])
    cap, longest = int(off[-1]), int(lens.max()) + 1
    s = dict(case=case, g=g, scale=1.0 / math.sqrt(d), seg_off=torch.from_numpy(off).cuda())
    # plan: the rows of the pass, one unit behind the other, and where they lie
    grown = lens + (1 if kind.startswith("decode") and case["append"] else 0)
    unit = np.repeat(np.arange(units), grown)
    at = np.arange(len(unit)) - np.repeat(np.cumsum(grown) - grown, grown)
    s.update(unit=torch.from_numpy(unit).cuda(), at=torch.from_numpy(at).cuda(),
             flat=torch.from_numpy(off[unit] + at).cuda(), rows=torch.from_numpy(grown).cuda().view(-1, 1),
             pad=torch.from_numpy(np.minimum(off[:-1, None] + np.arange(longest), cap - 1)).cuda())
    # lengths, positions and accumulated weights, in one buffer so that one copy puts them back
    live = torch.zeros(units + 2 * cap, dtype=torch.int32, device="cuda")
    kept_len, kept_idx, acc = live[:units], live[units:units + cap], live[units + cap:].view(torch.float32)
    kept_len.copy_(torch.from_numpy(lens))
    old = np.repeat(off[:-1] - (np.cumsum(before) - before), before) + np.arange(before.sum())
    old = torch.from_numpy(old).cuda()
    kept_idx[old] = _positions(gen, before, n)
    s.update(live=live, kept_len=kept_len, kept_idx=kept_idx, acc=acc)
    if kind == "compact":
        # keys of images are shifted per channel, as in the package's synthetic prompts
        s["k"] = _normal(gen, (B, L, Hkv, n, d), dtype)
        s["k"][:, :, :, : n // 2] += 0.5 * _normal(gen, (L, Hkv, 1, d), dtype)
        s["v"] = _normal(gen, (B, L, Hkv, n, d), dtype)
    else:
        # every segment has a row that nearly every query attends to, as its first
        k = _normal(gen, (cap, d), dtype)
        q = _normal(gen, (B, L, Hq, d), dtype)
        qbar = q.view(units, g, d).float().mean(1)
        k[s["seg_off"][:-1]] += (5.0 * math.sqrt(d) * qbar / (qbar * qbar).sum(1, keepdim=True)).to(dtype)
        v = _normal(gen, (cap, d), dtype)
        s.update(q=q, k_c=k, v_c=v)
    if kind == "evict":
        # heavy-tailed sums; the rows that decoding appended have been there for a few steps only
        acc.copy_(torch.exp(torch.randn(cap, generator=gen, device="cuda")) / case["rows"])
        young = torch.from_numpy(np.maximum(0, at - before[unit] + 1)).cuda()
        rows = s["flat"]
        age = 1.0 - (young - 1).float() / max(1, case["over"])
        acc[rows] *= torch.where(young > 0, age, torch.ones_like(age))
        kept_idx[rows] = torch.where(young > 0, (n - 1 + young).to(torch.int32), kept_idx[rows])
        limit = np.maximum(before, 1)
        final = np.repeat(np.arange(units), limit)
        s.update(limit=torch.from_numpy(limit.astype(np.int32)).cuda(), most=int((lens - limit).max()),
                 final=torch.from_numpy(off[final] + np.arange(len(final)) - np.repeat(np.cumsum(limit) - limit, limit)).cuda())
        del s["q"]
    if kind.startswith("decode"):
        s.update(k_new=_normal(gen, (B, L, Hkv, d), dtype) if case["append"] else None,
                 v_new=_normal(gen, (B, L, Hkv, d), dtype) if case["append"] else None,
                 out=torch.zeros((B, L, Hq, d), dtype=dtype, device="cuda"),
                 lse=torch.zeros((B, L, Hq), device="cuda"), decay=0.98)
        if case["track"]:
            acc.copy_(torch.exp(torch.randn(cap, generator=gen, device="cuda")) * (8.0 * g / case["rows"]))
            s.update(scratch=torch.zeros((cap, g), device="cuda"),
                     position=torch.full((B,), n, dtype=torch.int32, device="cuda"))
        if case["append"]:
            s["fresh"] = s["seg_off"][:-1] + torch.from_numpy(lens).cuda()
    if case["quant"]:
        for x in ("k", "v"):
            s[x + "_code"] = torch.zeros((cap, d // 2), dtype=torch.uint8, device="cuda")
            s[x + "_par"] = torch.zeros((cap, d // GROUP, 2), dtype=torch.bfloat16, device="cuda")
            if kind != "compact":
                dense = s.pop(x + "_c")
                for a in range(0, cap, 1 << 18):
                    code, par = _quantise(dense[a:a + (1 << 18)].float())
                    s[x + "_code"][a:a + (1 << 18)], s[x + "_par"][a:a + (1 << 18)] = _pack(code), par
            m = len(s["flat"]) if kind == "compact" else len(s["final"]) if kind == "evict" else units
            s[x + "_out"] = torch.zeros((m, d), dtype=dtype, device="cuda")
    if kind == "decode" and not case["append"]:
        s["k_new"] = s["v_new"] = None
    s["start"] = live.clone()
    if own:
        from paper_2506_15724_b200 import binding as mk

        s["cfg"] = mk.make_config(dtype, B, L, Hq, Hkv, d, n, 32, max_new_tokens=headroom)
        s["ws"] = mk.new_workspace(s["cfg"])
        s["mk"] = mk
    return s


# ------------------------------------------------------------------------------------------------- one pass
def run(s):
    """One pass: the outputs and the state as it is after it (what is held in 4 bits as the values it stands for)."""
    case = s["case"]
    if case["kind"] == "compact":
        return _run_compact(s)
    s["live"].copy_(s["start"])
    return _run_evict(s) if case["kind"] == "evict" else _run_decode(s)


def _run_compact(s):
    if own:
        mk, cfg = s["mk"], s["cfg"]
        mk.madakv_compact_quant(cfg, s["k"], s["v"], s["kept_idx"], s["seg_off"], s["kept_len"], s["k_code"], s["k_par"],
                                s["v_code"], s["v_par"], s["ws"])
        mk.madakv_expand_quant(cfg, s["flat"], s["k_code"], s["k_par"], s["v_code"], s["v_par"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    n, d = s["case"]["n"], s["case"]["d"]
    src = s["unit"] * n + s["kept_idx"][s["flat"]]
    s["k_out"].copy_(_values(*_quantise(s["k"].view(-1, d)[src].float())))
    s["v_out"].copy_(_values(*_quantise(s["v"].view(-1, d)[src].float())))
    return {"k": s["k_out"], "v": s["v_out"]}


def _run_decode(s):
    case, quant, track = s["case"], s["case"]["quant"], s["case"]["track"]
    if own:
        mk, cfg = s["mk"], s["cfg"]
        if quant:
            tracked = (s["acc"], s["scratch"], s["kept_idx"], s["position"], s["decay"]) if track else ()
            mk.madakv_decode_attn_quant(cfg, -1, s["q"], s["k_new"], s["v_new"], s["k_code"], s["k_par"], s["v_code"],
                                        s["v_par"], s["seg_off"], s["kept_len"], s["out"], s["lse"], s["ws"], *tracked)
            if case["append"]:
                mk.madakv_expand_quant(cfg, s["fresh"], s["k_code"], s["k_par"], s["v_code"], s["v_par"], s["k_out"],
                                       s["v_out"])
        else:
            mk.madakv_decode_attn_track(cfg, -1, s["q"], s["k_new"], s["v_new"], s["k_c"], s["v_c"], s["seg_off"],
                                        s["kept_len"], s["out"], s["lse"], s["ws"], s["acc"], s["scratch"], s["kept_idx"],
                                        s["position"], s["decay"])
    else:
        d, units, g = case["d"], s["pad"].shape[0], s["g"]
        if case["append"]:
            for x in ("k", "v"):
                new = s[x + "_new"].view(units, d)
                if quant:
                    code, s[x + "_par"][s["fresh"]] = _quantise(new.float())
                    s[x + "_code"][s["fresh"]] = _pack(code)
                    s[x + "_out"].copy_(_values(code, s[x + "_par"][s["fresh"]]))
                else:
                    s[x + "_c"][s["fresh"]] = new
            s["kept_len"] += 1
            if track:
                s["acc"][s["fresh"]] = 0.0
                s["kept_idx"][s["fresh"]] = s["position"].repeat_interleave(units // case["B"])
        k, v = _padded(s, "k"), _padded(s, "v")
        score = (s["q"].view(units, g, d).float() * s["scale"]) @ k.mT
        score.masked_fill_((torch.arange(k.shape[1], device="cuda") >= s["rows"]).unsqueeze(1), -math.inf)
        top = score.amax(2, keepdim=True)
        weight = score.sub_(top).exp_()
        total = weight.sum(2, keepdim=True)
        weight /= total
        s["out"].copy_((weight @ v).view(s["out"].shape))
        s["lse"].copy_((top + total.log()).view(s["lse"].shape))
        if track:
            s["acc"][s["flat"]] = s["decay"] * s["acc"][s["flat"]] + weight.sum(1)[s["unit"], s["at"]]
    r = {"out": s["out"], "lse": s["lse"], "kept_len": s["kept_len"]}
    if track:
        r.update(acc=s["acc"], kept_idx=s["kept_idx"])
    if case["append"]:
        r.update({"k_row": s["k_out"], "v_row": s["v_out"]} if quant else {"k_c": s["k_c"], "v_c": s["v_c"]})
    return r


def _padded(s, x):
    """The segments as an fp32 tensor [units, longest, d]; what lies behind a segment's end is masked by the caller."""
    units, longest = s["pad"].shape
    rows = s["pad"].view(-1)
    if s["case"]["quant"]:
        return _values(_unpack(s[x + "_code"][rows], s["case"]["d"]), s[x + "_par"][rows]).view(units, longest, -1)
    return s[x + "_c"][rows].float().view(units, longest, -1)


def _run_evict(s):
    case, quant = s["case"], s["case"]["quant"]
    caches = ("k_code", "k_par", "v_code", "v_par") if quant else ("k_c", "v_c")
    if own:
        mk, cfg = s["mk"], s["cfg"]
        call = mk.madakv_evict_quant if quant else mk.madakv_evict
        call(cfg, -1, s["limit"], case["recent"], s["acc"], s["kept_idx"], s["seg_off"], s["kept_len"],
             *[s[x] for x in caches], s["ws"])
        if quant:
            mk.madakv_expand_quant(cfg, s["final"], s["k_code"], s["k_par"], s["v_code"], s["v_par"], s["k_out"], s["v_out"])
    else:
        units, longest = s["pad"].shape
        at = torch.arange(longest, device="cuda").view(1, -1)
        there = at < s["kept_len"].view(-1, 1)
        position = torch.where(there, s["kept_idx"][s["pad"]], -1).long()
        safe = there & (position > position.amax(1, keepdim=True) - case["recent"])
        acc = s["acc"][s["pad"]]
        key = torch.where(acc > 0, acc, 0.0).view(torch.int32)
        key = torch.where(safe, 0x7fffffff, torch.where(there, key, -1))
        order = key.sort(dim=1, descending=True, stable=True)[1]
        end = torch.minimum(torch.maximum(s["limit"].view(-1, 1), safe.sum(1, keepdim=True)), s["kept_len"].view(-1, 1))
        stays = torch.zeros_like(there).scatter_(1, order, at < end)
        # the j-th hole takes the j-th surviving row from behind the new end; beyond the last hole a row behind the end
        # (which is not written) stands for itself
        holes = ((at < end) & ~stays).to(torch.int8).sort(dim=1, descending=True, stable=True)[1][:, :s["most"]]
        moved = (at >= end) & stays
        movers = moved.to(torch.int8).sort(dim=1, descending=True, stable=True)[1][:, :s["most"]]
        real = at[:, :s["most"]] < moved.sum(1, keepdim=True)
        to = (s["seg_off"][:-1].view(-1, 1) + torch.where(real, holes, end)).view(-1)
        source = (s["seg_off"][:-1].view(-1, 1) + torch.where(real, movers, end)).view(-1)
        for x in caches + ("acc", "kept_idx"):
            s[x][to] = s[x][source]
        s["kept_len"].copy_(end.view(-1))
        if quant:
            for x in ("k", "v"):
                s[x + "_out"].copy_(_values(_unpack(s[x + "_code"][s["final"]], case["d"]), s[x + "_par"][s["final"]]))
    r = {"kept_len": s["kept_len"], "acc": s["acc"], "kept_idx": s["kept_idx"]}
    r.update({"k": s["k_out"], "v": s["v_out"]} if quant else {"k_c": s["k_c"], "v_c": s["v_c"]})
    return r


# ------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """What a pass returns, in 64 bits; what is only copied or counted has no such value."""
    kind, d = case["kind"], case["d"]
    s = prepare(case, seed)
    off = s["seg_off"].tolist()
    lens = _lengths(case).tolist()
    if kind == "evict":
        return _exact_evict(s, off, lens)
    if kind == "compact":
        result = {}
        for x in ("k", "v"):
            parts = []
            for u, rows in enumerate(lens):
                b, rest = divmod(u, case["L"] * case["Hkv"])
                l, h = divmod(rest, case["Hkv"])
                kept = s["kept_idx"][off[u]:off[u] + rows].long()
                parts.append(_nearest_levels(s[x][b, l, h].index_select(0, kept).double()).to(torch.float32))
            result[x] = torch.cat(parts)
        return result
    g, units = s["g"], len(lens)
    out = torch.zeros((units, g, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((units, g), dtype=torch.float64, device="cuda")
    acc = s["acc"].double()
    rows_new = {}
    for u, rows in enumerate(lens):
        a, b = off[u], off[u] + rows
        kv = []
        for x in ("k", "v"):
            y = _stored(s[x + "_code"][a:b], s[x + "_par"][a:b], d) if case["quant"] else s[x + "_c"][a:b].double()
            if case["append"]:
                new = s[x + "_new"].view(units, 1, d)[u].double()
                new = _nearest_levels(new) if case["quant"] else new
                rows_new.setdefault(x, []).append(new)
                y = torch.cat((y, new))
            kv.append(y)
        z = s["q"].view(units, g, d)[u].double() @ kv[0].T / math.sqrt(d)
        lse[u] = torch.logsumexp(z, dim=1)
        p = torch.exp(z - lse[u].unsqueeze(1))
        out[u] = p @ kv[1]
        if case["track"]:
            end = a + p.shape[1]
            if case["append"]:
                acc[end - 1] = 0.0
            acc[a:end] = 0.98 * acc[a:end] + p.sum(0)
    r = {"out": out.view(s["out"].shape), "lse": lse.view(s["lse"].shape), "kept_len": None}
    if case["track"]:
        r.update(acc=acc, kept_idx=None)
    if case["append"]:
        r.update({"k_row": torch.cat(rows_new["k"]), "v_row": torch.cat(rows_new["v"])} if case["quant"]
                 else {"k_c": None, "v_c": None})
    return r


def _exact_evict(s, off, lens):
    """Segment by segment on the host: where every row of the cache comes from, then its contents in 64 bits."""
    acc, at = s["acc"].cpu().numpy(), s["kept_idx"].cpu().numpy()
    limit, recent, d = s["limit"].tolist(), s["case"]["recent"], s["case"]["d"]
    source = np.arange(off[-1])
    for u, rows in enumerate(lens):
        a, p = acc[off[u]:off[u] + rows], at[off[u]:off[u] + rows].astype(np.int64)
        young = p > p.max() - recent
        best = np.lexsort((np.arange(rows), -np.where(a > 0, a.astype(np.float64), 0.0), ~young))
        end = min(rows, max(limit[u], int(young.sum())))
        best = np.sort(best[:end])
        source[off[u] + np.setdiff1d(np.arange(end), best)] = off[u] + best[best >= end]
    source = torch.from_numpy(source).cuda()
    r = {"kept_len": None, "acc": s["acc"].double()[source], "kept_idx": None}
    for x in ("k", "v"):
        if s["case"]["quant"]:
            r[x] = _stored(s[x + "_code"][source[s["final"]]], s[x + "_par"][source[s["final"]]], d)
        else:
            r[x + "_c"] = s[x + "_c"][source].double()
    return r


def _nearest_levels(x):
    """The values that rows (64 bits) have in the cache in 4 bits: the number of borders below an element is its code."""
    result = torch.empty_like(x)
    for a in range(0, x.shape[1], GROUP):
        y = x[:, a:a + GROUP]
        low, high = y.min(dim=1, keepdim=True)[0], y.max(dim=1, keepdim=True)[0]
        mid = ((low + high) / 2).float().bfloat16().double()
        step = ((high - low) / 15).float().bfloat16().double()
        level = torch.zeros_like(y)
        for border in range(-7, 8):
            level += (y >= mid + border * step).double()
        result[:, a:a + GROUP] = mid + (level - 7.5) * step
    return result


def _stored(packed, par, d):
    """The values, in 64 bits, of packed rows."""
    e = torch.arange(d, device="cuda")
    group, rest = e // GROUP, e % GROUP
    byte = 2 * (rest // 4 * (d // GROUP) + group) + rest % 4 // 2
    code = (packed[:, byte].to(torch.int64) >> (4 * (rest % 2))) % 16
    return par[:, group, 1].double() + (code.double() - 7.5) * par[:, group, 0].double()


# ------------------------------------------------------------------------------------------------- cost
def work(case):
    d, g, e = case["d"], case["Hq"] // case["Hkv"], 4 if case["dtype"] == "f32" else 2
    lens = _lengths(case)
    units, rows = len(lens), int(lens.sum())
    small, full = 2 * (d // 2 + d // 8), 2 * d * e  # bytes of a row of K and V in 4 bits and in the case's type
    if case["kind"] == "compact":
        # positions and rows read, the cache and the values read back from it written; about six operations an element
        return {"bytes": float(rows * (4 + 2 * full + small)), "flops": float(rows * 2 * d * 6)}
    if case["kind"] == "evict":
        # weights and positions read, the young rows that stay moved into the holes; the cache in 4 bits is read back
        moved = units * (min(case["recent"], case["over"]) + max(0, case["over"] - case["recent"]) // 2)
        row = small if case["quant"] else full
        back = (rows - units * case["over"]) * (small + full) if case["quant"] else 0
        return {"bytes": float(rows * 8 + moved * 2 * (row + 8) + back), "flops": float(rows)}
    grown = rows + (units if case["append"] else 0)
    row = small if case["quant"] else full
    fixed = units * (2 * g * d * e + 4 * g) + (units * (full + row + (full if case["quant"] else 0)) if case["append"] else 0)
    return {"bytes": float(grown * (row + (8 if case["track"] else 0)) + fixed), "flops": float(grown * g * d * 4)}
