"""Layer-routed KV-cache eviction on AMD MI355X (gfx950): Python binding of librkv.so.

Argument marshalling only: every step of the eviction path runs in the HIP kernels of
librkv.so.  PyTorch provides device memory and the current HIP stream.

    plan = Plan(rules, budgets, window=32, pool_kernel=7)
    out = evict_prefill(plan, q_win, k, v)      # per-layer lists of bf16 device tensors
    out["k_out"][l], out["v_out"][l], out["idx"][l]
"""
from __future__ import annotations

import ctypes as C
import operator
from typing import Sequence

from . import _abi
from ._abi import FULL, STREAMING, SNAPKV, H2O, TOVA, H2O_FULL, PHASE_PREFILL, PHASE_DECODE, T_IDENTITY, T_PPL_CAP  # noqa: F401
from ._abi import SCOPE_PREFILL, SCOPE_DECODE, SCOPE_BOTH, STATUS_TIMEOUT, STATUS_INVALID, STATUS_REPAIRED  # noqa: F401
from ._abi import PAGES_EXHAUSTED, PAGES_INVALID  # noqa: F401
from ._abi import RkvError, check

__all__ = ["Plan", "allocate_budgets", "evict_prefill", "decode_step", "decode_init_from_prefill", "prefill_check",
           "rule_phases", "version", "entropy_profile", "entropy_budgets",
           "PagedCache", "pages_init", "pages_resize", "pages_write", "pages_attend", "pages_init_from_prefill",
           "FULL", "STREAMING", "SNAPKV", "H2O", "TOVA", "H2O_FULL", "SCOPE_PREFILL", "SCOPE_DECODE", "SCOPE_BOTH",
           "RkvError"]


def version() -> int:
    return _abi.lib().rkv_version()


def rule_phases(rule: int) -> int:
    """Phases operator `rule` declares (Section 3.4): bit 0 prefill, bit 1 decode."""
    m = C.c_int32()
    check(_abi.lib().rkv_rule_phases(int(rule), C.byref(m)))
    return m.value


def allocate_budgets(scores: Sequence[float], total: int, b_min: int, transform: int = T_IDENTITY):
    """Per-layer integer budgets summing to `total`, each >= b_min (Section 3.3, Eq. 3)."""
    n = len(scores)
    arr = (C.c_double * n)(*[float(x) for x in scores])
    out = (C.c_int32 * n)()
    check(_abi.lib().rkv_allocate_budgets(arr, n, transform, int(total), int(b_min), out))
    return list(out)


class Plan:
    """Immutable execution plan: per layer an operator and capacity for prefill and decode (Eq. 1)."""

    def __init__(self, rules_prefill, budgets_prefill, rules_decode=None, budgets_decode=None, *,
                 window=32, pool_kernel=7, n_sink=4, recent_num=1, recent_den=2):
        n = len(rules_prefill)
        rules_decode = list(rules_decode) if rules_decode is not None else [FULL] * n
        budgets_decode = list(budgets_decode) if budgets_decode is not None else [0] * n
        if not (len(budgets_prefill) == len(rules_decode) == len(budgets_decode) == n):
            raise ValueError("per-layer lists must have equal length")
        layers = (_abi.Layer * n)()
        for i in range(n):
            layers[i] = _abi.Layer(int(rules_prefill[i]), int(budgets_prefill[i]), int(rules_decode[i]),
                                   int(budgets_decode[i]))
        self.params = _abi.Params(window, pool_kernel, n_sink, recent_num, recent_den)
        handle = C.c_void_p()
        check(_abi.lib().rkv_plan_create(layers, n, C.byref(self.params), C.byref(handle)))
        self._h = handle
        self.n_layers = n
        self.rules_prefill = [int(r) for r in rules_prefill]
        self.rules_decode = rules_decode
        self.window = window

    @classmethod
    def from_route(cls, rules_prefill, weights, total: int, b_min: int, rules_decode=None, *,
                   transform: int = T_IDENTITY, **params):
        """Plan whose per-layer capacities split `total` by allocation `weights` (Eq. 3); decode
        capacities equal the prefill ones."""
        budgets = allocate_budgets(weights, total, b_min, transform)
        return cls(rules_prefill, budgets, rules_decode, budgets if rules_decode is not None else None, **params)

    @classmethod
    def from_scoped_route(cls, rules, scopes, budgets, **params) -> "Plan":
        """Plan of a completed route (Sections 3.1-3.2): layer l runs rules[l] at capacity
        budgets[l] in the phases of scopes[l] (SCOPE_PREFILL, SCOPE_DECODE or SCOPE_BOTH, a tied
        both-phase route) and FULL in the other phase; validated by rkv_plan_from_route."""
        n = len(rules)
        if not (len(scopes) == len(budgets) == n):
            raise ValueError("per-layer lists must have equal length")
        route = (_abi.RouteLayer * n)()
        for i in range(n):
            route[i] = _abi.RouteLayer(int(rules[i]), int(scopes[i]), int(budgets[i]))
        p = dict(window=32, pool_kernel=7, n_sink=4, recent_num=1, recent_den=2)
        p.update(params)
        prm = _abi.Params(p["window"], p["pool_kernel"], p["n_sink"], p["recent_num"], p["recent_den"])
        handle = C.c_void_p()
        check(_abi.lib().rkv_plan_from_route(route, n, C.byref(prm), C.byref(handle)))
        self = cls.__new__(cls)
        self._h = handle
        self.n_layers = n
        self.params = prm
        self.rules_prefill = [int(r) if s != SCOPE_DECODE else FULL for r, s in zip(rules, scopes)]
        self.rules_decode = [int(r) if s != SCOPE_PREFILL else FULL for r, s in zip(rules, scopes)]
        self.window = p["window"]
        return self

    def to_bytes(self) -> bytes:
        """The plan's serialized record (rkv_plan_serialize)."""
        size = C.c_size_t()
        check(_abi.lib().rkv_plan_serialize(self._h, None, 0, C.byref(size)))
        buf = C.create_string_buffer(size.value)
        check(_abi.lib().rkv_plan_serialize(self._h, buf, size.value, C.byref(size)))
        return buf.raw[:size.value]

    @classmethod
    def from_bytes(cls, data: bytes) -> "Plan":
        """A plan from a serialized record, validated by the library (rkv_plan_deserialize)."""
        import struct
        handle = C.c_void_p()
        check(_abi.lib().rkv_plan_deserialize(C.c_char_p(bytes(data)), len(data), C.byref(handle)))
        words = struct.unpack("<%di" % (len(data) // 4), data)
        n = words[2]
        self = cls.__new__(cls)
        self._h = handle
        self.n_layers = n
        self.params = _abi.Params(*words[3:8])
        lay = words[8:]
        self.rules_prefill = [lay[4 * i] for i in range(n)]
        self.rules_decode = [lay[4 * i + 2] for i in range(n)]
        self.window = words[3]
        return self

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None):
            _abi.lib().rkv_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def retained_counts(self, seq_len: int, phase: int = PHASE_PREFILL):
        out = (C.c_int32 * self.n_layers)()
        check(_abi.lib().rkv_plan_retained_counts(self._h, phase, seq_len, out))
        return list(out)

    def workspace_size(self, batch, seq_len, n_q_heads, n_kv_heads, head_dim=128) -> int:
        shape = _abi.Shape(batch, seq_len, n_q_heads, n_kv_heads, head_dim)
        nb = C.c_size_t()
        check(_abi.lib().rkv_prefill_workspace_size(self._h, C.byref(shape), C.byref(nb)))
        return nb.value


_DATA_PTR = operator.methodcaller("data_ptr")


def _parr(ptrs):
    """Pointer table of addresses (None or 0: null); it converts to the C side's void**."""
    return (C.c_void_p * len(ptrs))(*ptrs)


def _table(tensors):
    """Pointer table of a list of tensors (None: null)."""
    try:
        return (C.c_void_p * len(tensors))(*map(_DATA_PTR, tensors))
    except AttributeError:   # some are None
        return _parr([t.data_ptr() if t is not None else None for t in tensors])


def _stream_handle(stream, device):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream(device)
    return s.cuda_stream


def alloc_workspace(plan: Plan, batch, seq_len, n_q_heads, n_kv_heads, device="cuda"):
    import torch
    nb = plan.workspace_size(batch, seq_len, n_q_heads, n_kv_heads)
    return torch.empty(nb, dtype=torch.uint8, device=device)


def evict_prefill(plan: Plan, q_win, k, v, *, out=None, workspace=None, score_out=False, acc_out=False,
                  stream=None, check_status=False):
    """Compress every layer's prompt cache.

    q_win[l]: bf16 [B, Hq, w, d] ([B, Hq, L, d] for H2O_FULL layers; None allowed for FULL /
    STREAMING layers);
    k[l], v[l]: bf16 [B, Hkv, L, d].  Returns dict of per-layer lists: k_out, v_out (bf16
    [B, Hkv, n_l, d]), idx (int32 [B, Hkv, n_l], ascending), and optionally scores (fp32
    [B, Hkv, L]) and acc (fp32 [B, Hkv, n_l]).  Outputs are valid after the stream syncs and
    when the workspace status word (prefill_check) has neither STATUS_TIMEOUT nor STATUS_INVALID;
    check_status=True synchronises and raises RkvError otherwise.
    """
    import torch
    n = plan.n_layers
    if not (len(k) == len(v) == len(q_win) == n):
        raise ValueError("need one q_win / k / v entry per layer")
    B, Hkv, L, d = k[0].shape
    Hq = next((q.shape[1] for q in q_win if q is not None), Hkv)
    dev = k[0].device
    bf16 = torch.bfloat16
    for t in (*k, *v, *q_win):
        if t is not None and (t.dtype != bf16 or not t.is_contiguous() or t.device != dev):
            raise ValueError("inputs must be contiguous bf16 tensors on one device")
    kv_shape = (B, Hkv, L, d)
    for t in (*k, *v):
        if t.shape != kv_shape:
            raise ValueError("every k / v must have shape [B, Hkv, L, d]")
    win_shape, full_shape = (B, Hq, plan.window, d), (B, Hq, L, d)
    for q, r in zip(q_win, plan.rules_prefill):
        if q is not None and q.shape != (full_shape if r == H2O_FULL else win_shape):
            raise ValueError("q_win must have shape [B, Hq, w, d] ([B, Hq, L, d] for H2O_FULL layers)")
    if out is None:
        counts = plan.retained_counts(L)
        out = {
            "k_out": [torch.empty((B, Hkv, c, d), dtype=torch.bfloat16, device=dev) for c in counts],
            "v_out": [torch.empty((B, Hkv, c, d), dtype=torch.bfloat16, device=dev) for c in counts],
            "idx": [torch.empty((B, Hkv, c), dtype=torch.int32, device=dev) for c in counts],
        }
        if score_out:
            out["scores"] = [torch.zeros((B, Hkv, L), dtype=torch.float32, device=dev) for _ in range(n)]
        if acc_out:
            out["acc"] = [torch.empty((B, Hkv, c), dtype=torch.float32, device=dev) for c in counts]
    if workspace is None:
        workspace = alloc_workspace(plan, B, L, Hq, Hkv, dev)
    call = PreparedPrefill(plan, q_win, k, v, out, workspace)
    call(stream)
    out["workspace"] = workspace
    out["io"] = call   # keeps the marshalled pointer tables (decode_init_from_prefill uses them)
    if check_status:
        torch.cuda.synchronize(dev)
        st = prefill_check(workspace)
        if st & (STATUS_TIMEOUT | STATUS_INVALID):
            raise RkvError(7, f"prefill status word {st:#x}: outputs invalid")
    return out


class PreparedPrefill:
    """A prefill call with its pointer tables marshalled once; calling it enqueues the whole
    eviction pass on the stream with a single C call (for loops, benchmarks and graphs)."""

    def __init__(self, plan: Plan, q_win, k, v, out, workspace):
        B, Hkv, L, d = k[0].shape
        Hq = next((q.shape[1] for q in q_win if q is not None), Hkv)
        self._keep = (q_win, k, v, out, workspace)
        self._arrays = [_table(q_win), _table(k), _table(v), _table(out["k_out"]), _table(out["v_out"]), _table(out["idx"]),
                        _table(out["scores"]) if "scores" in out else None,
                        _table(out["acc"]) if "acc" in out else None]
        self.io = _abi.PrefillIO(*self._arrays)
        self.shape = _abi.Shape(B, L, Hq, Hkv, d)
        self.plan = plan
        self.ws_ptr = C.c_void_p(workspace.data_ptr())
        self.ws_bytes = workspace.numel()
        self.device = k[0].device
        self._fn = _abi.lib().rkv_prefill_evict

    def __call__(self, stream=None):
        check(self._fn(self.plan.handle, C.byref(self.shape), C.byref(self.io), self.ws_ptr, self.ws_bytes,
                       C.c_void_p(_stream_handle(stream, self.device))))


def alloc_outputs(plan: Plan, B, Hkv, L, d=128, device="cuda", score_out=False, acc_out=False):
    import torch
    counts = plan.retained_counts(L)
    out = {
        "k_out": [torch.empty((B, Hkv, c, d), dtype=torch.bfloat16, device=device) for c in counts],
        "v_out": [torch.empty((B, Hkv, c, d), dtype=torch.bfloat16, device=device) for c in counts],
        "idx": [torch.empty((B, Hkv, c), dtype=torch.int32, device=device) for c in counts],
    }
    if score_out:
        out["scores"] = [torch.zeros((B, Hkv, L), dtype=torch.float32, device=device) for _ in counts]
    if acc_out:
        out["acc"] = [torch.empty((B, Hkv, c), dtype=torch.float32, device=device) for c in counts]
    return out


STAGE_ZERO, STAGE_SCORE, STAGE_SELECT, STAGE_GATHER, STAGE_DECODE = 0, 1, 2, 3, 4


def profile_enable(stage: int):
    """Record HIP events around every following launch of `stage` (-1 disables)."""
    check(_abi.lib().rkv_profile_enable(int(stage)))


def profile_read():
    """(number of recorded launches, summed milliseconds); synchronises and clears."""
    n = C.c_int32()
    ms = C.c_double()
    check(_abi.lib().rkv_profile_read(C.byref(n), C.byref(ms)))
    return n.value, ms.value


def prefill_check(workspace) -> int:
    """Status word a previous prefill left in `workspace` (0 = clean).  Synchronous."""
    st = C.c_int32()
    check(_abi.lib().rkv_prefill_check(C.c_void_p(workspace.data_ptr()), workspace.numel(), C.byref(st)))
    return st.value


def entropy_profile(q, k, *, stream=None):
    """Attention-entropy layer scores H_l (Section 3.3): q[l] bf16 [B, Hq, n_q, d] (queries of the
    last n_q positions), k[l] bf16 [B, Hkv, L, d].  Returns {"h": fp32 [n_layers] (nats),
    "rows": fp32 [n_layers, B, Hq, n_q], "status": int32 [1] (nonzero: a row was not finite)}.
    Outputs are valid after the stream is synchronised."""
    import torch
    n = len(q)
    assert n == len(k) and n >= 1
    B, Hq, n_q, d = q[0].shape
    Hkv, L = k[0].shape[1], k[0].shape[2]
    dev = k[0].device
    rows = torch.empty((n, B, Hq, n_q), dtype=torch.float32, device=dev)
    h = torch.empty((n,), dtype=torch.float32, device=dev)
    status = torch.empty((1,), dtype=torch.int32, device=dev)
    shape = _abi.Shape(B, L, Hq, Hkv, d)
    nbytes = C.c_size_t()
    check(_abi.lib().rkv_entropy_workspace_size(C.byref(shape), n, n_q, C.byref(nbytes)))
    ws = torch.empty((max(nbytes.value, 8) + 7) // 8, dtype=torch.float64, device=dev)
    check(_abi.lib().rkv_entropy_profile(C.byref(shape), n, n_q, _table(q), _table(k), C.c_void_p(rows.data_ptr()),
                                         C.c_void_p(h.data_ptr()), C.c_void_p(status.data_ptr()),
                                         C.c_void_p(ws.data_ptr()), ws.numel() * 8,
                                         C.c_void_p(_stream_handle(stream, dev))))
    return {"h": h, "rows": rows, "status": status, "workspace": ws}


def entropy_budgets(h, total: int, b_min: int = 32):
    """Entropy allocation: per-layer capacities from H_l by Eq. 3 with the identity transform."""
    return allocate_budgets([float(x) for x in h], total, b_min, T_IDENTITY)


def decode_init_from_prefill(plan: Plan, prefill_out, state=None, *, stream=None):
    """Prefill -> decode hand-off (Section 3.4, rkv_decode_init_from_prefill): the compacted prompt
    cache of an evict_prefill result becomes the decode state of every layer whose decode operator
    is not FULL.  `state` (per-layer lists "k_cache", "v_cache", "pos", "acc") is allocated when
    None; entries of FULL-decode layers stay None, "acc" only for decode H2O layers.  Returns the
    state; valid after the stream syncs."""
    import torch
    call = prefill_out["io"]
    B, L, Hq, Hkv, d = (call.shape.batch, call.shape.seq_len, call.shape.n_q_heads, call.shape.n_kv_heads,
                        call.shape.head_dim)
    dev = call.device
    caps = plan.retained_counts(L, PHASE_DECODE)
    n = plan.n_layers
    if state is None:
        state = {"k_cache": [], "v_cache": [], "pos": [], "acc": []}
        for l in range(n):
            r, c = plan.rules_decode[l], caps[l]
            live = r != FULL
            state["k_cache"].append(torch.empty((B, Hkv, c, d), dtype=torch.bfloat16, device=dev) if live else None)
            state["v_cache"].append(torch.empty((B, Hkv, c, d), dtype=torch.bfloat16, device=dev) if live else None)
            state["pos"].append(torch.empty((B, Hkv, c), dtype=torch.int32, device=dev) if live else None)
            state["acc"].append(torch.empty((B, Hkv, c), dtype=torch.float32, device=dev) if r == H2O else None)
    st = _abi.DecodeState(_table(state["k_cache"]), _table(state["v_cache"]), _table(state["pos"]),
                          _table(state["acc"]))
    check(_abi.lib().rkv_decode_init_from_prefill(plan.handle, C.byref(call.shape), C.byref(call.io), C.byref(st),
                                                  C.c_void_p(_stream_handle(stream, dev))))
    return state


def decode_step(plan: Plan, state, q, k, v, position: int, *, victim_out=None, stream=None):
    """One decode step for every layer with a decode operator.

    state: dict of per-layer lists "k_cache", "v_cache" (bf16 [B, Hkv, C_l, d]), "pos" (int32
    [B, Hkv, C_l]), "acc" (fp32 [B, Hkv, C_l]; None allowed for layers whose decode operator is
    not H2O); updated in place.  q[l]: bf16 [B, Hq, d];
    k[l], v[l]: bf16 [B, Hkv, d].  victim_out: optional per-layer int32 [B, Hkv] tensors.
    """
    n = plan.n_layers
    B, Hkv = k[0].shape[0], k[0].shape[1]
    Hq = q[0].shape[1]
    d = k[0].shape[-1]
    st = _abi.DecodeState(_table(state["k_cache"]), _table(state["v_cache"]), _table(state["pos"]),
                          _table(state["acc"]))
    inp = _abi.DecodeInput(_table(q), _table(k), _table(v),
                           _table(victim_out) if victim_out is not None else None)
    shape = _abi.Shape(B, 1, Hq, Hkv, d)
    dev = k[0].device
    assert len(q) == len(k) == len(v) == n
    check(_abi.lib().rkv_decode_step(plan.handle, C.byref(shape), C.byref(st), C.byref(inp), int(position),
                                     C.c_void_p(_stream_handle(stream, dev))))


# ---- paged caches

_T = None     # torch, imported by the first call that needs it
_I32 = None


def _torch():
    global _T, _I32
    if _T is None:
        import torch
        _T, _I32 = torch, torch.int32
    return _T


def _check_int32(name, t, shape, dev):
    """An int32 tensor on `dev`, dense in its last dimension; shape: its sizes, -1 for any."""
    if t.dtype is _I32 and t.shape == shape and t.is_contiguous() and t.device == dev:
        return
    if t.dtype is not _I32 or t.device != dev:
        raise ValueError(f"{name} must be int32 on the pool's device")
    have = t.shape
    if have != shape and (len(have) != len(shape) or any(n != m and m != -1 for n, m in zip(have, shape))):
        raise ValueError(f"{name} must have shape {list(shape)}, not {list(have)}")
    if t.stride(-1) != 1 and have[-1] > 1:
        raise ValueError(f"{name} must be dense in its last dimension")


def _elsewhere(dev, stream):
    """A context in which `dev` and `stream` are the current ones, or None where they are: what a call allocates then
    belongs to the stream that uses it."""
    torch = _T or _torch()
    if dev.type != "cuda":
        raise ValueError("tensors must be on the GPU")
    if stream is None:
        return None if torch.cuda.current_device() == dev.index else torch.cuda.device(dev)
    if stream.device != dev:
        raise ValueError("the stream is another device's")
    return torch.cuda.stream(stream)


def _raw_stream(dev):
    """The current stream's handle (torch's own accessor for generated code: a Stream object costs ten times as much)."""
    get = getattr(_T._C, "_cuda_getCurrentRawStream", None)
    return get(dev.index) if get else _T.cuda.current_stream(dev).cuda_stream


def _strides(t):
    """Strides, 0 where a dimension has one entry: what stands there is arbitrary."""
    return [0 if n == 1 else s for n, s in zip(t.shape, t.stride())]


def _refuse_gradients(name, *tensors):
    """No backward pass: a result that silently ended the graph would train on wrong gradients."""
    for t in tensors:
        if t is not None and t.requires_grad and _torch().is_grad_enabled():
            raise ValueError(f"{name} has no backward pass: call it under torch.no_grad(), or with detached tensors")


class PagedCache:
    """A pool of K and V pages (rkv_pages): k_pages, v_pages bf16 or fp16 [n_pages, Hkv, page_size, 128], any strides that are
    multiples of 8 with the last dimension dense.  Make one and keep it: its calls then marshal no pool again.  The decode
    caches of `decode_step` ([B, Hkv, C, 128]) are pools of one page per sequence."""

    def __init__(self, k_pages, v_pages):
        torch = _torch()
        if k_pages.dim() != 4 or k_pages.shape != v_pages.shape:
            raise ValueError("k_pages and v_pages must have shape [n_pages, Hkv, page_size, d]")
        if k_pages.dtype != v_pages.dtype or k_pages.dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("pages must be bf16 or fp16")
        if k_pages.stride(3) != 1 or v_pages.stride(3) != 1:
            raise ValueError("pages must be dense in their last dimension")
        if k_pages.device != v_pages.device:
            raise ValueError("pages must be on one device")
        self.k_pages, self.v_pages = k_pages, v_pages
        self.device, self.dtype = k_pages.device, k_pages.dtype
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k_pages.shape
        self._pack = _abi.Pages.pack(k_pages.data_ptr(), v_pages.data_ptr(), *_strides(k_pages)[:3], *_strides(v_pages)[:3], self.n_pages,
                                     self.page_size, self.n_kv_heads, self.head_dim, _abi.BF16 if self.dtype == torch.bfloat16 else _abi.F16)
        self._bytes = {}     # workspace sizes by what they depend on


def pages_init(n_seqs: int, max_pages: int, n_pages: int, page_size: int, device="cuda"):
    """The tables of empty sequences and a full ring of free pages: {"table" int32 [n_seqs, max_pages], "lens" int32 [n_seqs],
    "ring" int32 [n_pages], "cursor" int32 [2] (front of the ring, free pages), "page_size"}."""
    torch = _torch()
    return {"table": torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device),
            "lens": torch.zeros(n_seqs, dtype=torch.int32, device=device),
            "ring": torch.arange(n_pages, dtype=torch.int32, device=device),
            "cursor": torch.tensor([0, n_pages], dtype=torch.int32, device=device), "page_size": int(page_size)}


def pages_resize(pages, new_lens, max_new: int, *, in_place=True, stream=None):
    """Block tables and slot map from request lengths (rkv_pages_resize): sequence s of `pages` (pages_init) gets new_lens[s]
    slots; pages are taken from the ring's front and given back to its end.  Returns {"slots" int32 [max_new] of the new
    tokens, -1 behind the last, "cu_new" int32 [n_seqs + 1], "status" int32 [1] (0, or PAGES_EXHAUSTED / PAGES_INVALID: nothing
    changed), "lens", "cursor"}.  in_place: lens and cursor of `pages` become the new ones; else they stay, and the new ones
    are only returned (the table's entries past the old lengths and the ring's behind the free ones are written all the same)."""
    table, lens, ring, cursor = pages["table"], pages["lens"], pages["ring"], pages["cursor"]
    dev = table.device
    ctx = _elsewhere(dev, stream)
    if ctx is not None:
        with ctx:
            return pages_resize(pages, new_lens, max_new, in_place=in_place)
    n = lens.shape[0]
    width = table.shape[-1]
    _check_int32("table", table, (n, width), dev)
    _check_int32("lens", lens, (n,), dev)
    _check_int32("new_lens", new_lens, (n,), dev)
    _check_int32("ring", ring, (ring.shape[0],), dev)
    _check_int32("cursor", cursor, (2,), dev)
    if max_new < 0:
        raise ValueError("max_new must be >= 0")
    if in_place:
        slots, cu_new, status = new_lens.new_empty(max_new + n + 2).split_with_sizes((max_new, n + 1, 1))
    else:
        slots, cu_new, status, lens, cursor = new_lens.new_empty(max_new + 2 * n + 4).split_with_sizes(
            (max_new, n + 1, 1, n, 2))
    r = _abi.Resize.pack(pages["lens"].data_ptr(), new_lens.data_ptr(), lens.data_ptr(), table.data_ptr(),
                         table.stride(0) if n > 1 else width, ring.data_ptr(), pages["cursor"].data_ptr(), cursor.data_ptr(), slots.data_ptr(), cu_new.data_ptr(), status.data_ptr(), n,
                         width, ring.shape[0], pages["page_size"], max_new)
    check(_abi.lib().rkv_pages_resize(r, _raw_stream(dev)))
    return {"slots": slots, "cu_new": cu_new, "status": status, "lens": lens, "cursor": cursor}


def pages_write(cache: PagedCache, k, v, slots, *, stream=None):
    """Copies new rows to their slots (rkv_pages_write): k, v [T, Hkv, d], or [B, n, Hkv, d] with T = B n, of the pool's type and any
    strides that are multiples of 8; slots int32 [T], distinct; rows with a slot outside the pool (-1) are skipped.  No backward
    pass: tensors that require gradients are refused unless gradients are off."""
    dev = cache.device
    _refuse_gradients("pages_write", k, v, cache.k_pages, cache.v_pages)
    ctx = _elsewhere(dev, stream)
    if ctx is not None:
        with ctx:
            return pages_write(cache, k, v, slots)
    shape = k.shape
    ks, vs = (_strides(k), _strides(v)) if 1 in shape else (k.stride(), v.stride())
    if shape != v.shape or len(shape) not in (3, 4) or shape[-2] != cache.n_kv_heads or shape[-1] != cache.head_dim:
        raise ValueError("k and v must have shape [T, Hkv, d] or [B, n, Hkv, d]")
    if k.dtype != cache.dtype or v.dtype != cache.dtype or ks[-1] != 1 or vs[-1] != 1 or k.device != dev or v.device != dev:
        raise ValueError("k and v must be of the pool's type, on its device and dense in their last dimension")
    if len(shape) == 3:
        outer, n, ks, vs = 1, shape[0], (0, *ks), (0, *vs)
    else:
        outer, n = shape[0], shape[1]
    _check_int32("slots", slots, (outer * n,), dev)
    rows = _abi.Rows.pack(k.data_ptr(), v.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2], slots.data_ptr(), outer, n)
    check(_abi.lib().rkv_pages_write(cache._pack, rows, _raw_stream(dev)))


def pages_attend(cache: PagedCache, q, table, lens, cu_q=None, *, max_q=0, max_kv=0, scale=None, causal=True, window=0, softcap=0.0,
                 slopes=None, prefix_lens=None, first_keys=None, out=None, lse_out=None, return_lse=False, stream=None):
    """Attention of new tokens over a paged cache (rkv_pages_attend).

    q: [T, Hq, d] of the pool's type, any strides that are multiples of 8; table int32 [n_seqs, max_pages]; lens int32 [n_seqs],
    the slots of each sequence with its new tokens' own among them; cu_q int32 [n_seqs + 1]: sequence s has rows cu_q[s] ..
    cu_q[s + 1] - 1 (None: one row each).  max_q, max_kv: the most rows and slots of a sequence, if known: they choose the
    kernel, never the result.  scale: 1 / sqrt(d) by default; window: slots a query sees, its own included (0: all);
    softcap c: scores c tanh(x / c); slopes fp32 [Hq]: scores less slope times distance; prefix_lens int32 [n_seqs]: slots
    every row of the sequence sees; first_keys int32 [T]: the first slot a row sees.  Returns out [T, Hq, d] (`out` if given: rows
    behind the last sequence stay as they are; a row that sees nothing is 0), and with return_lse or lse_out also fp32
    [T, Hq], the logarithm of the sum of exponentials (-inf for a row that sees nothing).  No backward pass: tensors that
    require gradients are refused unless gradients are off."""
    dev = cache.device
    _refuse_gradients("pages_attend", q, cache.k_pages, cache.v_pages, slopes, out, lse_out)
    ctx = _elsewhere(dev, stream)
    if ctx is not None:
        with ctx:
            return pages_attend(cache, q, table, lens, cu_q, max_q=max_q, max_kv=max_kv, scale=scale, causal=causal, window=window,
                                softcap=softcap, slopes=slopes, prefix_lens=prefix_lens, first_keys=first_keys, out=out, lse_out=lse_out,
                                return_lse=return_lse)
    torch = _T
    shape = q.shape
    if len(shape) != 3 or shape[2] != cache.head_dim or q.dtype != cache.dtype or q.stride(2) != 1 or q.device != dev:
        raise ValueError("q must have shape [T, Hq, d], the pool's type and device and a dense last dimension")
    T, Hq, d = shape
    q_token, q_head, _ = q.stride()
    n = lens.shape[0]
    width = table.shape[-1]
    _check_int32("table", table, (n, width), dev)
    _check_int32("lens", lens, (n,), dev)
    cu = prefix = first = slope = lse_ptr = 0
    if cu_q is not None:
        _check_int32("cu_q", cu_q, (n + 1,), dev)
        cu = cu_q.data_ptr()
    if prefix_lens is not None:
        _check_int32("prefix_lens", prefix_lens, (n,), dev)
        prefix = prefix_lens.data_ptr()
    if first_keys is not None:
        _check_int32("first_keys", first_keys, (T,), dev)
        first = first_keys.data_ptr()
    if slopes is not None:
        if slopes.dtype != torch.float32 or slopes.shape != (Hq,) or not slopes.is_contiguous() or slopes.device != dev:
            raise ValueError("slopes must be contiguous fp32 [Hq] on the pool's device")
        slope = slopes.data_ptr()
    if out is None:
        out = torch.empty_like(q) if q.is_contiguous() else torch.empty(shape, dtype=q.dtype, device=dev)
    elif out.shape != shape or out.dtype != q.dtype or out.stride(2) != 1 or out.device != dev:
        raise ValueError("out must have q's shape, type and device and a dense last dimension")
    lse = lse_out
    if lse is None:
        if return_lse:
            lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    elif lse.shape != (T, Hq) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.device != dev:
        raise ValueError("lse_out must be contiguous fp32 [T, Hq] on the pool's device")
    if lse is not None:
        lse_ptr = lse.data_ptr()
    out_token, out_head, _ = out.stride()
    if T == 1:      # what stands there says nothing
        q_token = out_token = 0
    if Hq == 1:
        q_head = out_head = 0
    a = _abi.Attend.pack(q.data_ptr(), out.data_ptr(), lse_ptr, q_token, q_head, out_token, out_head, table.data_ptr(), table.stride(0) if n > 1 else width,
                         lens.data_ptr(), cu, prefix, first, slope, n, T, Hq, width, max_q, max_kv, bool(causal), window,
                         d ** -0.5 if scale is None else scale, softcap)
    L = _abi.lib()
    key = (T, Hq, n, width, max_q, max_kv, cu != 0)
    nbytes = cache._bytes.get(key)
    if nbytes is None:
        size = C.c_size_t()
        check(L.rkv_pages_attend_workspace_size(cache._pack, a, C.byref(size)))
        if len(cache._bytes) >= 1024:
            cache._bytes.clear()
        nbytes = cache._bytes[key] = size.value
    ws = lens.new_empty(nbytes // 4) if nbytes else None
    check(L.rkv_pages_attend(cache._pack, a, ws.data_ptr() if nbytes else None, nbytes, _raw_stream(dev)))
    return out if lse is None else (out, lse)


def pages_init_from_prefill(plan: Plan, prefill_out, *, page_size=16, extra=0, stream=None):
    """Prefill -> paged caches: the compacted prompt cache of every layer of an evict_prefill result moves into pages, of which a
    layer takes as many as its retained rows need, and `extra` more slots' worth per sequence stay free for new tokens.
    Returns, per layer, (cache, pages): a PagedCache and its tables (pages_init) with lens at the layer's retained count."""
    if page_size < 1 or extra < 0:
        raise ValueError("page_size must be >= 1 and extra >= 0")
    torch = _torch()
    got = []
    dev = prefill_out["k_out"][0].device
    ctx = _elsewhere(dev, stream)
    if ctx is not None:
        with ctx:
            return pages_init_from_prefill(plan, prefill_out, page_size=page_size, extra=extra)
    for k, v in zip(prefill_out["k_out"], prefill_out["v_out"]):
        B, Hkv, n, d = k.shape
        per = -(-(n + extra) // page_size)
        pages = pages_init(B, max(1, per), max(1, B * per), page_size, dev)
        pool = torch.empty((2, max(1, B * per), Hkv, page_size, d), dtype=k.dtype, device=dev)
        cache = PagedCache(pool[0], pool[1])
        step = pages_resize(pages, torch.full((B,), n, dtype=torch.int32, device=dev), B * n)
        pages_write(cache, k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3), step["slots"])
        got.append((cache, pages))
    return got
