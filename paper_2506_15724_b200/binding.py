"""Thin binding of libmadakv.so: the same names as include/madakv.h, argument marshalling only. The asynchronous calls go
through a small C++ extension (_native.so) that reads the tensors itself, the rest through ctypes.

Every step of the eviction pass runs in the library's CUDA kernels; PyTorch is used for device memory and streams.
There is no CPU fallback: importing this module without the built library, or calling it without a CUDA device,
raises.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmadakv.so")

MADAKV_F32, MADAKV_BF16 = 0, 1
HCC_OFF, HCC_PAPER, HCC_LITERAL, HCC_DEMAND = 0, 1, 2, 3
STATUS_NAMES = ["OK", "EINVAL", "ESHAPE", "EALIGN", "EWORKSPACE", "ECAPACITY", "EUNSUPPORTED", "ECUDA", "ETIMEOUT",
                "ESTATIC"]
(OK, EINVAL, ESHAPE, EALIGN, EWORKSPACE, ECAPACITY, EUNSUPPORTED, ECUDA, ETIMEOUT, ESTATIC) = range(10)
STATIC_SCRATCH_BYTES = 16 << 20

EXPORTS = [
    "madakv_abi_version", "madakv_status_string", "madakv_workspace_bytes", "madakv_workspace_bytes_attn", "madakv_score", "madakv_score_lse",
    "madakv_score_kept",
    "madakv_allocate", "madakv_allocate_layer", "madakv_demand_layer",
    "madakv_select", "madakv_compact", "madakv_decode_attn", "madakv_decode_attn_static", "madakv_poll_status",
    "madakv_compact_quant", "madakv_expand_quant", "madakv_decode_attn_quant", "madakv_decode_attn_track", "madakv_evict",
    "madakv_evict_quant", "madakv_prefill_attn", "madakv_prefill_attn_keep", "madakv_tree_attn", "madakv_tree_commit",
]


class MadakvConfig(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("batch", ctypes.c_int32),
        ("n_layers", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("max_seq_len", ctypes.c_int32), ("window", ctypes.c_int32),
        ("causal", ctypes.c_int32), ("mpa", ctypes.c_int32), ("hcc_mode", ctypes.c_int32),
        ("max_new_tokens", ctypes.c_int32), ("theta", ctypes.c_float), ("softmax_scale", ctypes.c_float),
        ("keep_window", ctypes.c_int32), ("pool_kernel", ctypes.c_int32),
    ]


class MadakvStrides(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("layer", ctypes.c_int64), ("head", ctypes.c_int64),
                ("token", ctypes.c_int64)]


class MadakvError(RuntimeError):
    def __init__(self, where, code):
        self.code = code
        name = STATUS_NAMES[code] if 0 <= code < len(STATUS_NAMES) else str(code)
        super().__init__(f"{where} failed: MADAKV_{name}")


_lib = None


def lib():
    """The loaded C-ABI library (loaded once). Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2506_15724_b200.build` (needs nvcc)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        cfgp = ctypes.POINTER(MadakvConfig)
        L.madakv_abi_version.restype = ctypes.c_int
        L.madakv_status_string.restype = ctypes.c_char_p
        L.madakv_status_string.argtypes = [ctypes.c_int]
        L.madakv_workspace_bytes.argtypes = L.madakv_workspace_bytes_attn.argtypes = [cfgp, ctypes.POINTER(sz)]
        L.madakv_score.argtypes = [cfgp, vp, MadakvStrides, vp, MadakvStrides, vp, vp, vp, vp, sz, vp]
        L.madakv_score_lse.argtypes = [cfgp, vp, MadakvStrides, vp, MadakvStrides, vp, vp, vp, vp, sz, vp]
        L.madakv_score_kept.argtypes = [cfgp, vp, MadakvStrides, vp, MadakvStrides, vp, vp, vp, vp, vp, sz, vp]
        L.madakv_allocate.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.madakv_allocate_layer.argtypes = [cfgp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.madakv_demand_layer.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.madakv_select.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, i64, vp, sz, vp]
        L.madakv_compact.argtypes = [cfgp, vp, vp, MadakvStrides, vp, vp, vp, vp, vp, i64, vp, sz, vp]
        L.madakv_decode_attn.argtypes = [cfgp, i32, vp, vp, vp, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
        L.madakv_decode_attn_static.argtypes = [cfgp, i32, vp, vp, vp, vp, vp, i64, vp, vp, vp]
        f32 = ctypes.c_float
        L.madakv_compact_quant.argtypes = [cfgp, vp, vp, MadakvStrides, vp, vp, vp, vp, vp, vp, vp, i64, vp, sz, vp]
        L.madakv_expand_quant.argtypes = [cfgp, vp, i64, vp, vp, vp, vp, i64, vp, vp, vp]
        L.madakv_decode_attn_quant.argtypes = [cfgp, i32] + [vp] * 9 + [i64] + [vp] * 6 + [f32, vp, sz, vp]
        L.madakv_decode_attn_track.argtypes = [cfgp, i32] + [vp] * 7 + [i64] + [vp] * 6 + [f32, vp, sz, vp]
        L.madakv_evict.argtypes = [cfgp, i32, vp, i32, vp, vp, vp, vp, i64, vp, vp, vp, sz, vp]
        L.madakv_evict_quant.argtypes = [cfgp, i32, vp, i32, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp, sz, vp]
        S = MadakvStrides
        L.madakv_prefill_attn.argtypes = [cfgp, i32, vp, S, i64, vp, vp, vp, S, vp, S, i64, vp, vp, vp, S, vp, vp, vp, vp, sz, vp]
        L.madakv_prefill_attn_keep.argtypes = [*L.madakv_prefill_attn.argtypes[:-3], vp, vp, sz, vp]
        L.madakv_tree_attn.argtypes = [cfgp, i32, i32, vp, S, vp, S, vp, S] + [vp] * 6 + [i64, vp, S, vp, vp, sz, vp]
        L.madakv_tree_commit.argtypes = [cfgp, i32, i32, vp, vp, vp, vp, S, vp, S] + [vp] * 4 + [i64] + [vp] * 4 + [sz, vp]
        L.madakv_poll_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
        for f in EXPORTS:
            if f not in ("madakv_status_string",):
                getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


def make_config(dtype, batch, n_layers, n_q_heads, n_kv_heads, head_dim, max_seq_len, window, causal=1, mpa=1,
                hcc_mode=HCC_PAPER, max_new_tokens=0, theta=0.5, softmax_scale=0.0, keep_window=0, pool_kernel=1):
    code = {torch.float32: MADAKV_F32, torch.bfloat16: MADAKV_BF16}.get(dtype, dtype)
    return MadakvConfig(ctypes.sizeof(MadakvConfig), code, batch, n_layers, n_q_heads, n_kv_heads, head_dim,
                        max_seq_len, window, causal, mpa, hcc_mode, max_new_tokens, theta, softmax_scale, keep_window,
                        pool_kernel)


class _Unbuilt:
    """Stands for the extension where it has not been built: any call raises."""

    def __init__(self, why):
        self.why = why

    def __getattr__(self, name):
        raise ImportError(f"{self.why}: run `python -m paper_2506_15724_b200.build` (needs nvcc and g++)")


# What a call on one layer costs is mostly the host's part. With the tensors' pointers gathered in Python and passed through
# ctypes it was 5.4 us for decode, 5.2-6.4 for allocate_layer, select and compact, 6.8 for score_lse; with the extension, which
# takes the tensors, it is 3.1, 2.5-2.9 and 5.1, most of that the launch.
try:
    from . import _native
except ImportError as e:
    _native = _Unbuilt(e)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check(where, rc):
    if rc != 0:
        raise MadakvError(where, rc)


def madakv_workspace_bytes(cfg):
    out = ctypes.c_size_t(0)
    _check("madakv_workspace_bytes", lib().madakv_workspace_bytes(cfg, ctypes.byref(out)))
    return out.value


def madakv_workspace_bytes_attn(cfg):
    out = ctypes.c_size_t(0)
    _check("madakv_workspace_bytes_attn", lib().madakv_workspace_bytes_attn(cfg, ctypes.byref(out)))
    return out.value


def new_workspace(cfg, device="cuda", attention=True):
    """A zeroed device workspace. attention: with room for the shares of prompt and tree attention, up to 39 MB that other calls do without."""
    return torch.zeros((madakv_workspace_bytes_attn if attention else madakv_workspace_bytes)(cfg), dtype=torch.uint8, device=device)


def madakv_score(cfg, q_win, k, seq_len, lse, psi, ws):
    rc = _native.score(cfg, q_win, k, seq_len, lse, psi, ws)
    if rc:
        raise MadakvError("madakv_score", rc)


def madakv_score_lse(cfg, q_win, k, seq_len, lse, psi, ws):
    rc = _native.score_lse(cfg, q_win, k, seq_len, lse, psi, ws)
    if rc:
        raise MadakvError("madakv_score_lse", rc)


def madakv_score_kept(cfg, q_win, k, seq_len, lse, win_len, psi, ws):
    """The windows of madakv_prefill_attn with win_len; incomplete ones, or those of different prompts, record ESHAPE."""
    rc = _native.score_kept(cfg, q_win, k, seq_len, lse, win_len, psi, ws)
    if rc:
        raise MadakvError("madakv_score_kept", rc)


def madakv_allocate(cfg, psi, mask, seq_len, budget, mass, pref, demand, phi, budgets, ws):
    rc = _native.allocate(cfg, psi, mask, seq_len, budget, mass, pref, demand, phi, budgets, ws)
    if rc:
        raise MadakvError("madakv_allocate", rc)


def madakv_demand_layer(cfg, psi, mask, seq_len, mass, pref, demand, ws):
    rc = _native.demand_layer(cfg, psi, mask, seq_len, mass, pref, demand, ws)
    if rc:
        raise MadakvError("madakv_demand_layer", rc)


def madakv_allocate_layer(cfg, layer, psi, mask, seq_len, budget, mass, pref, demand, phi, budgets, ws):
    """psi may be None: mass, pref and demand then come from madakv_demand_layer."""
    rc = _native.allocate_layer(cfg, int(layer), psi, mask, seq_len, budget, mass, pref, demand, phi, budgets, ws)
    if rc:
        raise MadakvError("madakv_allocate_layer", rc)


def madakv_select(cfg, psi, mask, seq_len, budgets, kept_len, seg_off, kept_idx, ws):
    rc = _native.select(cfg, psi, mask, seq_len, budgets, kept_len, seg_off, kept_idx, ws)
    if rc:
        raise MadakvError("madakv_select", rc)


def madakv_compact(cfg, k, v, kept_idx, seg_off, kept_len, k_c, v_c, ws):
    rc = _native.compact(cfg, k, v, kept_idx, seg_off, kept_len, k_c, v_c, ws)
    if rc:
        raise MadakvError("madakv_compact", rc)


def madakv_decode_attn(cfg, layer, q, k_new, v_new, k_c, v_c, seg_off, kept_len, out, lse_out, ws):
    rc = _native.decode_attn(cfg, layer, q, k_new, v_new, k_c, v_c, seg_off, kept_len, out, lse_out, ws)
    if rc:
        raise MadakvError("madakv_decode_attn", rc)


def madakv_decode_attn_static(cfg, layer, q, k_c, v_c, seg_off, kept_len, out, lse_out):
    """Decode attention without a workspace: the library's built-in scratch is used, nothing is allocated. For
    callers that may not allocate device memory; calls must not overlap on the GPU (they share the scratch)."""
    _check("madakv_decode_attn_static", lib().madakv_decode_attn_static(cfg, layer, _ptr(q), _ptr(k_c),
                                                                        _ptr(v_c), _ptr(seg_off), _ptr(kept_len),
                                                                        k_c.shape[0], _ptr(out), _ptr(lse_out),
                                                                        _stream()))


# The calls from here on check their tensors against the config: a wrong dtype, size or device, or a tensor that is not contiguous
# (k and v of compaction may be strided), raises ValueError before anything is launched.
def madakv_compact_quant(cfg, k, v, kept_idx, seg_off, kept_len, k_code, k_par, v_code, v_par, ws):
    rc = _native.compact_quant(cfg, k, v, kept_idx, seg_off, kept_len, k_code, k_par, v_code, v_par, ws)
    if rc:
        raise MadakvError("madakv_compact_quant", rc)


def madakv_expand_quant(cfg, rows, k_code, k_par, v_code, v_par, k_out, v_out):
    """rows (int64) may be None: all rows of the cache."""
    rc = _native.expand_quant(cfg, rows, k_code, k_par, v_code, v_par, k_out, v_out)
    if rc:
        raise MadakvError("madakv_expand_quant", rc)


def madakv_decode_attn_quant(cfg, layer, q, k_new, v_new, k_code, k_par, v_code, v_par, seg_off, kept_len, out, lse_out, ws,
                             acc=None, scratch=None, kept_idx=None, position=None, decay=1.0):
    """With acc and scratch the call also accumulates every row's attention weight (see madakv_decode_attn_track)."""
    rc = _native.decode_attn_quant(cfg, layer, q, k_new, v_new, k_code, k_par, v_code, v_par, seg_off, kept_len, out, lse_out, ws,
                                   acc, scratch, kept_idx, position, decay)
    if rc:
        raise MadakvError("madakv_decode_attn_quant", rc)


def madakv_decode_attn_track(cfg, layer, q, k_new, v_new, k_c, v_c, seg_off, kept_len, out, lse_out, ws, acc, scratch,
                             kept_idx=None, position=None, decay=1.0):
    rc = _native.decode_attn_track(cfg, layer, q, k_new, v_new, k_c, v_c, seg_off, kept_len, out, lse_out, ws, acc, scratch,
                                   kept_idx, position, decay)
    if rc:
        raise MadakvError("madakv_decode_attn_track", rc)


def madakv_evict(cfg, layer, limit, recent, acc, kept_idx, seg_off, kept_len, k_c, v_c, ws):
    rc = _native.evict(cfg, layer, limit, recent, acc, kept_idx, seg_off, kept_len, k_c, v_c, ws)
    if rc:
        raise MadakvError("madakv_evict", rc)


def madakv_evict_quant(cfg, layer, limit, recent, acc, kept_idx, seg_off, kept_len, k_code, k_par, v_code, v_par, ws):
    rc = _native.evict_quant(cfg, layer, limit, recent, acc, kept_idx, seg_off, kept_len, k_code, k_par, v_code, v_par, ws)
    if rc:
        raise MadakvError("madakv_evict_quant", rc)


def madakv_prefill_attn(cfg, layer, q, k, v, out, ws, lse_out=None, q_win=None, lse_win=None, q_off=None, k_off=None, seq_len=None,
                        q_len=None, win_len=None):
    """Attention of a prompt's layer. q and out [B, L, H_q, rows, d], k and v [B, L, H_kv, rows, d], strided; with q_off (k_off) packed:
    [L, H, rows, d]. Exactly one of k_off and seq_len is given; without q_off and q_len there are as many queries as keys. With win_len [B, L]
    int32 (-1 to begin with) q_win and lse_win keep the rows of earlier chunks (madakv_prefill_attn_keep)."""
    rc = _native.prefill_attn(cfg, int(layer), q, k, v, out, ws, lse_out, q_win, lse_win, q_off, k_off, seq_len, q_len, win_len)
    if rc:
        raise MadakvError("madakv_prefill_attn" if win_len is None else "madakv_prefill_attn_keep", rc)


def madakv_tree_attn(cfg, layer, q, k_tree, v_tree, mask, k_c, v_c, seg_off, kept_len, out, lse_out, ws, n_nodes=None):
    """mask [B, T] int64: the bits of the nodes that a node sees."""
    rc = _native.tree_attn(cfg, int(layer), q, k_tree, v_tree, mask, k_c, v_c, seg_off, kept_len, out, lse_out, ws, n_nodes)
    if rc:
        raise MadakvError("madakv_tree_attn", rc)


def madakv_tree_commit(cfg, layer, mask, node, k_tree, v_tree, k_c, v_c, seg_off, kept_len, ws, n_nodes=None, acc=None, kept_idx=None,
                       position=None):
    rc = _native.tree_commit(cfg, int(layer), mask, node, k_tree, v_tree, k_c, v_c, seg_off, kept_len, ws, n_nodes, acc, kept_idx, position)
    if rc:
        raise MadakvError("madakv_tree_commit", rc)


def madakv_poll_status(ws):
    out = ctypes.c_int32(0)
    _check("madakv_poll_status", lib().madakv_poll_status(_ptr(ws), _stream(), ctypes.byref(out)))
    return out.value


def madakv_status_string(code):
    return lib().madakv_status_string(code).decode()


class EvictionBuffers:
    """Device tensors the calls write (allocated once through torch; no arithmetic here).

    quant: the ragged cache is held in 4 bits (k_code, k_par, v_code, v_par in the place of k_c and v_c).
    track: decode steps accumulate every row's attention weight in `acc`, so that run_trim can cut segments back."""

    def __init__(self, cfg, capacity_rows, device="cuda", want_lse=False, quant=False, track=False):
        B, L, Hq, Hkv = cfg.batch, cfg.n_layers, cfg.n_q_heads, cfg.n_kv_heads
        d, n = cfg.head_dim, cfg.max_seq_len
        units = B * L * Hkv
        dt = torch.float32 if cfg.dtype == MADAKV_F32 else torch.bfloat16
        z = lambda shape, dtype: torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
        self.cfg, self.quant, self.track = cfg, quant, track
        # kept_idx holds the position of every row of the segments. (To be set by who fills it in other ways than run_eviction, a replayed
        # graph of it included, after steps without positions.)
        self.placed = True
        self.ws = new_workspace(cfg, device, attention=want_lse or not quant)  # (neither run_prefill nor run_tree else)
        self.psi = z((B, L, Hkv, n), torch.float32)
        self.lse = z((B, L, Hq, cfg.window), torch.float32) if want_lse else None
        # run_prefill's proxy tokens, and for how many keys they are complete (lse holds the log-sum-exps of queries that run_eviction is given)
        self.q_win = z((B, L, Hq, cfg.window, d), dt) if want_lse else None
        self.lse_win = z((B, L, Hq, cfg.window), torch.float32) if want_lse else None
        self.win_len = torch.full((B, L), -1, dtype=torch.int32, device=device) if want_lse else None
        self.prefilled = set()  # layers that run_prefill has been called for
        self.mass = z((B, L, Hkv, 2), torch.float64)
        self.pref = z((B, L, Hkv, 2), torch.float64)
        self.demand = z((B, L, Hkv, 2), torch.int32)
        self.phi = z((B, L), torch.float64)
        self.budgets = z((B, L, Hkv, 2), torch.int32)
        self.kept_len = z((units,), torch.int32)
        self.seg_off = z((units + 1,), torch.int64)
        self.kept_idx = torch.full((capacity_rows,), -1, dtype=torch.int32, device=device)
        if quant:
            self.k_code, self.v_code = (z((capacity_rows, d // 2), torch.uint8) for _ in range(2))
            self.k_par, self.v_par = (z((capacity_rows, d // 32, 2), torch.bfloat16) for _ in range(2))
            self.cache = (self.k_code, self.k_par, self.v_code, self.v_par)
        else:
            self.k_c = z((capacity_rows, d), dt)
            self.v_c = z((capacity_rows, d), dt)
            self.cache = (self.k_c, self.v_c)
        if track:
            self.acc = z((capacity_rows,), torch.float32)
            self.scratch = z((capacity_rows, Hq // Hkv), torch.float32)
        self.out = z((B, L, Hq, d), dt)
        self.lse_dec = z((B, L, Hq), torch.float32)

    def run_prefill(self, layer, q, k, v, out, **lengths):
        """Attention of a layer's prompt (lengths: q_off, k_off, seq_len, q_len, lse_out of madakv_prefill_attn), whole or in chunks. The proxy
        tokens' queries and log-sum-exps are kept for run_eviction, over chunks shorter than the window too; needs want_lse."""
        if self.lse is None:
            raise ValueError("run_prefill: buffers without want_lse=True keep no log-sum-exps")
        madakv_prefill_attn(self.cfg, layer, q, k, v, out, self.ws, q_win=self.q_win, lse_win=self.lse_win, win_len=self.win_len, **lengths)
        self.prefilled.add(int(layer))

    def run_eviction(self, q_win, k, v, mask, seq_len, budget):
        """Stages 1-4, enqueued on the current stream. q_win None: the queries and log-sum-exps that run_prefill has kept of every layer, with
        which K is read once. ValueError if there is a layer that run_prefill was never called for; what only the device knows (windows that are not
        complete for seq_len keys, layers that a new prompt has not reached) records ESHAPE, and the eviction is not to be used."""
        c = self.cfg
        if q_win is None:
            if len(self.prefilled) < c.n_layers:
                raise ValueError("run_eviction: no q_win, and layers that run_prefill has kept none of")
            madakv_score_kept(c, self.q_win, k, seq_len, self.lse_win, self.win_len, self.psi, self.ws)
        else:
            madakv_score(c, q_win, k, seq_len, self.lse, self.psi, self.ws)
        madakv_allocate(c, self.psi, mask, seq_len, budget, self.mass, self.pref, self.demand, self.phi, self.budgets,
                        self.ws)
        madakv_select(c, self.psi, mask, seq_len, self.budgets, self.kept_len, self.seg_off, self.kept_idx, self.ws)
        compact = madakv_compact_quant if self.quant else madakv_compact
        compact(c, k, v, self.kept_idx, self.seg_off, self.kept_len, *self.cache, self.ws)
        self.placed = True
        if self.track:
            self.acc.zero_()

    def run_decode(self, q, k_new=None, v_new=None, layer=-1, position=None, decay=1.0):
        """One decode step. With tracking, position [B] int32 says where the new tokens stand. None: kept_idx is not kept up, and run_trim
        can protect no recent rows until the next run_eviction. Without tracking position and decay are not used."""
        head = (self.cfg, layer, q, k_new, v_new, *self.cache, self.seg_off, self.kept_len, self.out, self.lse_dec, self.ws)
        if not (self.quant or self.track):
            return madakv_decode_attn(*head)
        tracked = ()
        if self.track:
            tracked = (self.acc, self.scratch, self.kept_idx if position is not None else None, position, decay)
        (madakv_decode_attn_quant if self.quant else madakv_decode_attn_track)(*head, *tracked)
        if k_new is not None and position is None:
            self.placed = False

    def run_tree(self, q, k_tree, v_tree, mask, out, lse_out=None, layer=-1, n_nodes=None):
        """Attention of drafted tokens over the segments and their tree (madakv_tree_attn); the cache is left as it is."""
        if self.quant:
            raise ValueError("run_tree: not on a cache in 4 bits")
        madakv_tree_attn(self.cfg, layer, q, k_tree, v_tree, mask, *self.cache, self.seg_off, self.kept_len, out, lse_out, self.ws, n_nodes)

    def run_commit(self, mask, node, k_tree, v_tree, layer=-1, n_nodes=None, position=None):
        """The path up to node [B] int32 is appended (madakv_tree_commit). position [B] int32 is that of its first node; None: kept_idx is not kept
        up, and run_trim can protect no recent rows until the next run_eviction. With tracking appended rows start without weight: that of
        drafted tokens' attention is not accumulated."""
        if self.quant:
            raise ValueError("run_commit: not on a cache in 4 bits")
        madakv_tree_commit(self.cfg, layer, mask, node, k_tree, v_tree, *self.cache, self.seg_off, self.kept_len, self.ws, n_nodes,
                           self.acc if self.track else None, self.kept_idx if position is not None else None, position)
        if position is None:
            self.placed = False

    def run_trim(self, limit, recent=0, layer=-1):
        """Segments longer than limit [B, L, H_kv] int32 lose their rows of the smallest accumulated weight; needs track. With recent > 0 the
        rows of the newest `recent` positions stay whatever the limit is: a segment keeps up to max(limit, recent) rows, so its headroom
        has to hold max(0, recent - limit) rows and those of the steps until the next trim."""
        if not self.track:
            raise ValueError("run_trim: buffers without track=True accumulate no weights")
        if recent and not self.placed:
            raise ValueError("run_trim: recent rows cannot be told where run_decode or run_commit was given no position")
        call = madakv_evict_quant if self.quant else madakv_evict
        call(self.cfg, layer, limit, recent, self.acc, self.kept_idx, self.seg_off, self.kept_len, *self.cache, self.ws)
