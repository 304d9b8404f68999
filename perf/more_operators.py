"""Workloads of caches held in 8 bits and of batches that share a prefix, for timing them and comparing their outputs.

Every case is one call of a program that serves a decoder from a paged cache: `pages_write` of new rows into a
`QuantizedCache` (e4m3 codes, a power of two for each row of 128 values), `pages_read` of rows back, `pages_attend` over
such a cache, and `pages_attend_shared`, attention of sequences whose first slots are one common prefix.  Sizes are those
of `synth/workloads.py`, `bench.py` and `perf/operators.py` (32 query and 8 KV heads of 128, prompts to 32K, decode batches
of 64, evicted caches of 1024) and ragged ones around them.

With `own` false `run` computes the operators in elementary torch operations, in 32 bits.
"""
import math
import random

import torch

own = False

D = 128
DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EXPONENTS = {"bf16": (-117, 120), "fp16": (-15, 8)}     # of a row's scale: code 2^e is then a value of the type
E4M3 = torch.float8_e4m3fn
ATTEND = {"kind": "attend", "quant": True, "type": "bf16", "hq": 32, "hkv": 8, "page": 16, "singles": 0, "q_min": 1, "q_max": 1, "window": 0,
          "cap": 0.0, "alibi": False, "prefix": False, "lse": False, "pad": 0, "sizes": 1}
SHARED = {**ATTEND, "kind": "shared", "quant": False, "groups": 1, "alone": 0}


def listed():
    return [
        # the new rows of one decode step
        {"name": "write8_tick", "kind": "write", "type": "bf16", "rows": 64, "pad": 0, "hkv": 8, "page": 16, "slots": 1 << 17, "layout": "rows"},
        # a chunk of 16K tokens, K and V slices of a fused projection, some padding rows behind it
        {"name": "write8_chunk", "kind": "write", "type": "bf16", "rows": 16371, "pad": 13, "hkv": 8, "page": 64, "slots": 1 << 17, "layout": "fused"},
        # one short sequence's cache leaves its pages
        {"name": "read8_short", "kind": "read", "quant": True, "type": "fp16", "batch": 1, "rows": 301, "hkv": 8, "page": 16, "slots": 1 << 15, "layout": "rows"},
        # four prompts of 8K come back as the matrices that an eviction takes
        {"name": "read8_prompts", "kind": "read", "quant": True, "type": "bf16", "batch": 4, "rows": 8192, "hkv": 8, "page": 64, "slots": 1 << 17, "layout": "heads"},
        # one token of one interactive sequence, the smallest call
        {**ATTEND, "name": "token8_1k", "seqs": 1, "kv_min": 1024, "kv_max": 1024},
        # a decode step of 64 ragged sequences
        {**ATTEND, "name": "token8_batch_64", "seqs": 64, "kv_min": 512, "kv_max": 8192, "sizes": 3},
        # few very long sequences, eight query heads per KV head
        {**ATTEND, "name": "token8_long", "hq": 64, "page": 64, "seqs": 4, "kv_min": 131072, "kv_max": 131072, "lse": True},
        # a prompt's next 512 tokens after 32K
        {**ATTEND, "name": "chunk8_on_32k", "page": 64, "seqs": 1, "kv_min": 33280, "kv_max": 33280, "q_min": 512, "q_max": 512, "lse": True},
        # decoding sequences and entering prompts in one call: capped scores, a window, prefixes seen from both sides,
        # pages that end inside a tile, rows behind the last sequence
        {**ATTEND, "name": "mixed8_batch", "type": "fp16", "hq": 16, "page": 40, "seqs": 28, "singles": 24, "kv_min": 1024, "kv_max": 6007,
         "q_min": 6007, "q_max": 6007, "window": 4096, "cap": 50.0, "prefix": True, "pad": 9, "sizes": 4},
        # a decode step of 64 requests to one long system prompt
        {**SHARED, "name": "shared_batch_64", "seqs": 64, "shared_min": 8192, "shared_max": 8192, "kv_min": 64, "kv_max": 2048, "lse": True, "sizes": 2},
        # several prompts with a few requests each and some without, a few tokens each (drafts to verify), scores that fall with
        # distance, a window that cuts the longer prefixes
        {**SHARED, "name": "shared_groups", "type": "fp16", "hq": 16, "page": 48, "seqs": 41, "groups": 5, "alone": 4, "shared_min": 900, "shared_max": 9001,
         "kv_min": 20, "kv_max": 1501, "q_min": 2, "q_max": 9, "alibi": True, "window": 6000, "sizes": 6},
        # 128 requests to a document of 32K, all in 8 bits
        {**SHARED, "name": "shared8_on_32k", "quant": True, "page": 64, "seqs": 128, "shared_min": 32768, "shared_max": 32768, "kv_min": 16, "kv_max": 1024,
         "sizes": 7},
    ]


MOST_BYTES, MOST_FLOPS, MOST_PAIRS = 1.1e9, 2.9e11, 3.5e7     # of the largest listed cases


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    kind = rng.choice(["write", "read", "token", "token", "chunk", "mixed", "shared", "shared", "shared"])
    sizes = rng.randrange(1 << 30)
    page = rng.choice([1, 8, 16, 16, 32, 48, 64, 100, 128, 256, _log(rng, 2, 400)])
    dtype = rng.choice(["bf16", "fp16"])
    if kind == "write":
        return {"kind": "write", "type": dtype, "rows": _log(rng, 1, 16384), "pad": rng.choice([0, 0, _log(rng, 1, 200)]),
                "hkv": rng.choice([1, 2, 4, 8, 8, 16]), "page": page, "slots": 1 << 17, "layout": rng.choice(["rows", "fused", "heads"])}
    if kind == "read":
        batch = rng.choice([1, 1, _log(rng, 1, 16)])
        return {"kind": "read", "quant": rng.random() < 0.7, "type": dtype, "batch": batch, "rows": min(60000 // batch, _log(rng, 1, 8192)),
                "hkv": rng.choice([1, 2, 4, 8, 8]), "page": page, "slots": 1 << 16, "layout": rng.choice(["rows", "heads"])}
    hkv = rng.choice([1, 2, 4, 8, 8, 8])
    more = {"type": dtype, "hkv": hkv, "hq": hkv * rng.choice([1, 2, 3, 4, 4, 6, 8]), "page": page, "lse": rng.random() < 0.5,
            "cap": rng.choice([0.0, 0.0, 0.0, 30.0, 50.0]), "alibi": rng.random() < 0.2, "sizes": sizes}
    if kind == "token":
        lo, hi = sorted((_log(rng, 1, 32768), _log(rng, 1, 131072)))
        case = {**ATTEND, **more, "seqs": _log(rng, 1, 128), "kv_min": lo, "kv_max": hi, "window": rng.choice([0, 0, 0, _log(rng, 1, 8192)])}
        if rng.random() < 0.25:
            case.update(q_min=2, q_max=_log(rng, 2, 16))
    elif kind == "chunk":
        lo, hi = sorted((_log(rng, 32, 33000), _log(rng, 32, 33000)))
        case = {**ATTEND, **more, "seqs": _log(rng, 1, 8), "kv_min": lo, "kv_max": hi, "q_min": _log(rng, 4, 500), "q_max": _log(rng, 501, 8192),
                "window": rng.choice([0, 0, _log(rng, 1, 8192)])}
    elif kind == "mixed":
        n = _log(rng, 2, 64)
        case = {**ATTEND, **more, "seqs": n, "singles": rng.randrange(1, n), "kv_min": _log(rng, 1, 500), "kv_max": _log(rng, 501, 8192),
                "q_min": 8192, "q_max": 8192, "prefix": rng.random() < 0.6, "window": rng.choice([0, _log(rng, 64, 8192)]),
                "pad": rng.choice([0, _log(rng, 1, 64)])}
    else:
        n = _log(rng, 1, 128)
        lo, hi = sorted((_log(rng, 1, 32768), _log(rng, 16, 32768)))
        a, b = sorted((_log(rng, 1, 2048), _log(rng, 1, 2048)))
        case = {**SHARED, **more, "quant": rng.random() < 0.5, "seqs": n, "groups": _log(rng, 1, n), "shared_min": lo, "shared_max": hi, "kv_min": a,
                "kv_max": b, "window": rng.choice([0, 0, 0, _log(rng, 1, 16384)]), "pad": rng.choice([0, 0, _log(rng, 1, 64)])}
        case["alone"] = rng.choice([0, 0, rng.randrange(n - case["groups"] + 1)])
        if rng.random() < 0.4:
            case.update(q_min=1, q_max=_log(rng, 2, 300))
    while True:      # a drawn case costs no more than the largest listed one
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS and _plain_pairs(case) <= MOST_PAIRS:
            return case
        if case["seqs"] > case.get("groups", 0) + 1:
            case["seqs"] = max(1, case.get("groups", 0), case["seqs"] // 2)
            case["singles"] = min(case["singles"], case["seqs"])
            if "alone" in case:
                case["alone"] = min(case["alone"], case["seqs"] - case["groups"])
        elif case.get("shared_max", 0) > case["kv_max"]:
            case["shared_max"] //= 2
            case["shared_min"] = min(case["shared_min"], case["shared_max"])
        else:
            case["kv_max"] //= 2
            case["kv_min"] = min(case["kv_min"], case["kv_max"])


# ---- the sizes of a case, the same for every seed

def _lens(case):
    """(queries, keys) of each sequence: the keys hold the queries' own rows."""
    rng = random.Random(case["sizes"])
    got = []
    for s in range(case["seqs"]):
        n = _log(rng, case["kv_min"], case["kv_max"])
        q = 1 if s < case["singles"] else min(n, _log(rng, case["q_min"], max(case["q_min"], case["q_max"])))
        got.append((q, n))
    return got


def _groups(case):
    """(prefix, first sequence, behind the last) of each group; the last `alone` sequences have none."""
    if case["kind"] != "shared":
        return []
    rng = random.Random(case["sizes"] + 1)
    n, g = case["seqs"] - case["alone"], case["groups"]
    cuts = [0] + sorted(rng.sample(range(1, n), g - 1)) + [n]
    return [(_log(rng, case["shared_min"], case["shared_max"]), a, b) for a, b in zip(cuts, cuts[1:])]


def _before(case):
    """The slots of each sequence's shared prefix."""
    got = [0] * case["seqs"]
    for n, a, b in _groups(case):
        got[a:b] = [n] * (b - a)
    return got


def _spans(case, q, n, before):
    """(first, behind the last) visible key of each query, the shared prefix's first among them."""
    prefix = n // 4 if case["prefix"] else 0
    at = [before + n - q + i for i in range(q)]
    return [max(0, p - case["window"] + 1) if case["window"] else 0 for p in at], [before + max(p - before + 1, prefix) for p in at]


def _plain_pairs(case):
    return sum(q * (n + b) for (q, n), b in zip(_lens(case), _before(case))) * case["hq"] / 32


def work(case):
    if case["kind"] == "write":
        return {"bytes": case["rows"] * (case["hkv"] * (2 * D * 2 + 2 * (D + 1)) + 4), "flops": 0}
    row = 2 * (D + 1) if case["quant"] else 2 * 2 * D       # of K and V
    if case["kind"] == "read":
        return {"bytes": case["batch"] * case["rows"] * (case["hkv"] * (row + 2 * D * 2) + 4), "flops": 0}
    nbytes, pairs, need = 0, 0, {}
    for (q, n), before in zip(_lens(case), _before(case)):
        lo, hi = _spans(case, q, n, before)
        pairs += sum(hi) - sum(lo)
        nbytes += (max(hi) - max(before, min(lo))) * case["hkv"] * row + q * case["hq"] * (D * 2 * 2 + (4 if case["lse"] else 0)) + 4 * -(-n // case["page"])
    for n, a, b in _groups(case):
        first = min(min(_spans(case, q, m, n)[0]) for q, m in _lens(case)[a:b])
        nbytes += max(0, n - first) * case["hkv"] * row
    return {"bytes": nbytes, "flops": 4 * D * case["hq"] * pairs}


# ---- inputs

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, g):
    return torch.randn(shape, dtype=dtype, device=DEVICE, generator=g)


def _rows(shape, g, dtype):
    """K or V rows [..., D]: some channels are larger than others, and some rows."""
    channel = 1 + 7 * (torch.rand(D, device=DEVICE, generator=g) < 0.05)
    row = torch.exp(0.5 * _normal((*shape[:-1], 1), torch.float32, g))
    return (_normal(shape, torch.float32, g) * channel * row).to(dtype)


def _encode(x, dtype):
    """Codes and exponent bytes of rows [..., D], in elementary operations."""
    lo, hi = EXPONENTS[dtype]
    x = x.float()
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    f, e = torch.frexp(top)                              # f in [0.5, 1): 448 is 0.875 of 2^9
    e = torch.where(top > 0, e - 9 + (f > 0.875), lo).clamp(lo, hi)
    most = 240.0 * 2.0 ** hi
    y = torch.ldexp(x.clamp(-most, most), -e.unsqueeze(-1))
    return torch.where(torch.isfinite(x), y, math.nan).to(E4M3), (e + 127).to(torch.uint8)


def _decode(codes, scales):
    return codes.float() * (scales.int() << 23).view(torch.float32).unsqueeze(-1)


def _pools(case, n_pages, g):
    """K and V pools [n_pages, heads, page, D] of the case's kind: {"k", "v"} or also their exponents."""
    got = {}
    for x in ("k", "v"):
        if not case["quant"]:
            got[x] = _rows((n_pages, case["hkv"], case["page"], D), g, TYPES[case["type"]])
            continue
        got[x] = torch.empty((n_pages, case["hkv"], case["page"], D), dtype=E4M3, device=DEVICE)
        got[x + "_scale"] = torch.empty((n_pages, case["hkv"], case["page"]), dtype=torch.uint8, device=DEVICE)
        step = max(1, (1 << 27) // (case["hkv"] * case["page"] * D))
        for i in range(0, n_pages, step):
            m = min(step, n_pages - i)
            got[x][i:i + m], got[x + "_scale"][i:i + m] = _encode(_rows((m, case["hkv"], case["page"], D), g, TYPES[case["type"]]), case["type"])
    return got


def _handle(state):
    if own:
        import paper_2606_15157_amd as rkv
        p = state["pools"]
        if "k_scale" in p:
            state["cache"] = rkv.QuantizedCache(p["k"], p["v"], p["k_scale"], p["v_scale"], dtype=TYPES[state["case"]["type"]])
        else:
            state["cache"] = rkv.PagedCache(p["k"], p["v"])
    return state


def _slots(case, count, g):
    page = case["page"]
    first = torch.randperm(case["slots"] // page, generator=g, device=DEVICE)[:-(-count // page)] * page
    return (first.repeat_interleave(page) + torch.arange(first.numel() * page, device=DEVICE) % page)[:count].to(torch.int32)


def _prepare_write(case, seed):
    g = _generator(seed)
    t, h, dtype = case["rows"] + case["pad"], case["hkv"], TYPES[case["type"]]
    if case["layout"] == "heads":         # what an eviction returns: [1, heads, rows, D]
        k, v = (_rows((1, h, t, D), g, dtype).permute(0, 2, 1, 3) for _ in range(2))
    elif case["layout"] == "fused":       # slices of one projection's output
        x = _rows((t, 6 * h, D), g, dtype)
        k, v = x[:, 4 * h:5 * h], x[:, 5 * h:]
    else:
        k, v = (_rows((t, h, D), g, dtype) for _ in range(2))
    slots = _slots(case, t, g)
    slots[case["rows"]:] = -1
    shape, pools = (case["slots"] // case["page"], h, case["page"], D), {}
    for x in ("k", "v"):
        pools[x] = torch.randint(0, 127, shape, dtype=torch.uint8, device=DEVICE, generator=g).view(E4M3)
        pools[x + "_scale"] = torch.randint(112, 136, shape[:3], dtype=torch.uint8, device=DEVICE, generator=g)
    return _handle({"case": case, "pools": pools, "k": k, "v": v, "slots": slots})


def _prepare_read(case, seed):
    g = _generator(seed)
    b, n, h, dtype = case["batch"], case["rows"], case["hkv"], TYPES[case["type"]]
    state = {"case": case, "pools": _pools(case, case["slots"] // case["page"], g), "slots": _slots(case, b * n, g), "out": None}
    if b > 1 or case["layout"] == "heads":
        state["slots"] = state["slots"].view(b, n)
    if case["layout"] == "heads":         # what an eviction takes: [batch, heads, rows, D]
        state["out"] = [torch.empty((b, h, n, D), dtype=dtype, device=DEVICE) for _ in range(2)]
    return _handle(state)


def _tables(counts, ids, at):
    table = torch.full((len(counts), max(counts) + 1), -1, dtype=torch.int32, device=DEVICE)
    for s, k in enumerate(counts):
        table[s, :k] = ids[at:at + k]
        at += k
    return table, at


def _prepare_attend(case, seed):
    g = _generator(seed)
    lens, groups, p, hq, hkv, dtype = _lens(case), _groups(case), case["page"], case["hq"], case["hkv"], TYPES[case["type"]]
    counts, shared = [-(-n // p) for _, n in lens], [-(-n // p) for n, _, _ in groups]
    n_pages = sum(counts) + sum(shared) + 3
    ids = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)
    table, at = _tables(counts, ids, 0)
    rows = sum(q for q, _ in lens)
    cu = [0]
    for n_q, _ in lens:
        cu.append(cu[-1] + n_q)
    q = _normal((rows + case["pad"], hq, D), torch.float32, g).mul_(0.5).to(dtype)
    state = {"case": case, "pools": _pools(case, n_pages, g), "table": table, "q": q, "lens": _ints([n for _, n in lens]), "cu": _ints(cu),
             "counts": lens, "slopes": None, "prefix": None, "out": None}
    if groups:
        state["shared_table"], _ = _tables(shared, ids, at)
        state["shared_lens"] = _ints([n for n, _, _ in groups])
        state["cu_seqs"] = _ints([0] + [b for _, _, b in groups])
    if case["alibi"]:
        state["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device=DEVICE)
    if case["prefix"]:
        state["prefix"] = _ints([n // 4 for _, n in lens])
    if case["pad"]:      # a captured step's static output: rows behind the last sequence stay as they are
        state["out"] = torch.zeros_like(q)
        state["lse_out"] = torch.zeros((q.shape[0], hq), dtype=torch.float32, device=DEVICE)
    return _handle(state)


def prepare(case, seed):
    return {"write": _prepare_write, "read": _prepare_read}.get(case["kind"], _prepare_attend)(case, seed)


# ---- one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own(state, kind)
    return {"write": _plain_write, "read": _plain_read}.get(kind, _plain_attend)(state)


def _own(state, kind):
    import paper_2606_15157_amd as rkv
    if kind == "write":
        rkv.pages_write(state["cache"], state["k"], state["v"], state["slots"])
        return state["pools"]
    if kind == "read":
        if state["out"] is None:
            k, v = rkv.pages_read(state["cache"], state["slots"])
        else:
            k, v = rkv.pages_read(state["cache"], state["slots"], k_out=state["out"][0].permute(0, 2, 1, 3), v_out=state["out"][1].permute(0, 2, 1, 3))
        return {"k": k, "v": v}
    case, lens = state["case"], state["counts"]
    kw = {"max_q": max(n for n, _ in lens), "max_kv": max(n for _, n in lens), "window": case["window"], "softcap": case["cap"], "slopes": state["slopes"]}
    if state["out"] is not None:
        kw["out"] = state["out"]
        if case["lse"]:
            kw["lse_out"] = state["lse_out"]
    elif case["lse"]:
        kw["return_lse"] = True
    if kind == "shared":
        got = rkv.pages_attend_shared(state["cache"], state["q"], state["shared_table"], state["shared_lens"], state["cu_seqs"], state["table"],
                                      state["lens"], state["cu"], max_shared=case["shared_max"], **kw)
    else:
        got = rkv.pages_attend(state["cache"], state["q"], state["table"], state["lens"], state["cu"], prefix_lens=state["prefix"], **kw)
    return {"out": got[0], "lse": got[1]} if case["lse"] else {"out": got}


def _plain_write(state):
    case, p, rows = state["case"], state["case"]["page"], state["case"]["rows"]
    slots = state["slots"][:rows].long()
    page, at = slots // p, slots % p
    for x in ("k", "v"):
        new = state[x][0] if state[x].dim() == 4 else state[x]
        codes, scales = _encode(new[:rows], case["type"])
        state["pools"][x].view(torch.uint8)[page, :, at] = codes.view(torch.uint8)
        state["pools"][x + "_scale"][page, :, at] = scales
    return state["pools"]


def _plain_read(state):
    case, p, got = state["case"], state["case"]["page"], {}
    slots = state["slots"].long()
    for i, x in enumerate(("k", "v")):
        rows = _gathered(state["pools"], x, slots // p, slots % p).to(TYPES[case["type"]])
        if state["out"] is not None:
            state["out"][i].copy_(rows.permute(0, 2, 1, 3))
            rows = state["out"][i].permute(0, 2, 1, 3)
        got[x] = rows
    return got


def _gathered(pools, x, page, at):
    """Rows [..., heads, D] of (page, slot) in 32 bits."""
    if x + "_scale" in pools:
        return _decode(pools[x].view(torch.uint8)[page, :, at].view(E4M3), pools[x + "_scale"][page, :, at])
    return pools[x][page, :, at].float()


def _plain_part(state, q, ids, n, lo, hi, pos):
    """Sums of a batch of sequences, padded to one size: q [S, m, hq, D] in 32 bits, page ids [S, pages], n slots at most, of
    which row (s, i), at pos[s, i], sees lo[s, i] to hi[s, i].  Returns the sum of exp(x - top) v, that of exp(x - top), and top."""
    case = state["case"]
    hq, hkv, p = case["hq"], case["hkv"], case["page"]
    g, (S, m) = hq // hkv, q.shape[:2]
    at = torch.arange(n, device=DEVICE)
    k, v = (_gathered(state["pools"], x, ids[:, at // p].clamp(min=0).long(), at % p).transpose(1, 2) for x in ("k", "v"))
    k, v = k.transpose(2, 3).contiguous(), v.contiguous()
    parts = []
    step = max(1, (1 << 29) // max(1, S * hq * n))
    for r in range(0, m, step):      # rows whose scores fit the memory
        y = q[:, r:r + step]
        w = y.shape[1]
        y = y.reshape(S, w, hkv, g, D).permute(0, 2, 3, 1, 4).reshape(S, hkv, g * w, D)
        x = (torch.matmul(y, k) / math.sqrt(D)).view(S, hkv, g, w, n)
        if case["cap"]:
            x = torch.tanh(x / case["cap"]) * case["cap"]
        if state["slopes"] is not None:
            x = x - state["slopes"].view(hkv, g, 1, 1) * (pos[:, r:r + step, None] - at).abs().float()[:, None, None]
        seen = (at >= lo[:, r:r + step, None]) & (at < hi[:, r:r + step, None])
        x = x.masked_fill_(~seen[:, None, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        x = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
        total = x.sum(-1, keepdim=True)
        o = torch.matmul(x.view(S, hkv, g * w, n), v).view(S, hkv, g, w, D)
        parts.append([z.permute(0, 3, 1, 2, 4).reshape(S, w, hq, -1) for z in (o, total, top)])
    return [torch.cat(z, 1) for z in zip(*parts)]


def _plain_sums(state, table, lens, before, causal):
    """(sum of exp(x - top) v, sum of exp(x - top), top) of all rows over the sequences `lens` of (queries, keys), one behind the other,
    whose rows' positions begin `before` further on."""
    case, q = state["case"], state["q"]
    rows = sum(m for m, _ in lens)
    got = [torch.zeros((rows, case["hq"], w), dtype=torch.float32, device=DEVICE) for w in (D, 1, 1)]
    got[2].fill_(-math.inf)
    s, row = 0, 0
    while s < len(lens):     # as many sequences at once as fit the memory, padded
        e, m, n = s + 1, max(1, lens[s][0]), max(1, lens[s][1])
        while e < len(lens):
            m2, n2 = max(m, lens[e][0]), max(n, lens[e][1])
            if (e + 1 - s) * n2 * max(m2 * case["hq"], case["hkv"] * D) > 1 << 29:
                break
            e, m, n = e + 1, m2, n2
        n_q, n_k = (torch.tensor([x[i] for x in lens[s:e]], device=DEVICE)[:, None] for i in range(2))
        i = torch.arange(m, device=DEVICE)
        there = i < n_q
        at = row + torch.cumsum(n_q, 0) - n_q + i
        at = torch.where(there, at, 0)
        pos = before[at]
        hi = torch.minimum(pos + 1, n_k) if causal else n_k.expand(-1, m)
        if state["prefix"] is not None:
            hi = torch.maximum(hi, state["prefix"][s:e, None])
        lo = (pos - case["window"] + 1).clamp(min=0) if case["window"] else torch.zeros_like(pos)
        parts = _plain_part(state, q[at].float(), table[s:e], n, lo, torch.where(there, hi, 0), pos)
        for to, x in zip(got, parts):
            to[at[there]] = x[there]
        row += sum(x[0] for x in lens[s:e])
        s = e
    return got


def _plain_attend(state):
    case, q, lens = state["case"], state["q"], state["counts"]
    rows = sum(m for m, _ in lens)
    count, ends = (torch.tensor(x, device=DEVICE) for x in ([m for m, _ in lens], [n for _, n in lens]))
    pos = torch.arange(rows, device=DEVICE) + torch.repeat_interleave(ends - torch.cumsum(count, 0), count)   # of each row among its own keys
    o, total, top = _plain_sums(state, state["table"], lens, pos, True)
    groups = _groups(case)
    if groups:
        whole = [(sum(m for m, _ in lens[a:b]), n) for n, a, b in groups]
        first = torch.repeat_interleave(torch.tensor([n for n, _, _ in groups], device=DEVICE), torch.tensor([m for m, _ in whole], device=DEVICE))
        o2, total2, top2 = _plain_sums(state, state["shared_table"], whole, pos[:first.numel()] + first, False)
        m = first.numel()
        both = torch.maximum(top[:m], top2)
        ref = torch.where(both == -math.inf, 0.0, both)
        f, f2 = torch.exp(top[:m] - ref), torch.exp(top2 - ref)
        o[:m], total[:m], top[:m] = o[:m] * f + o2 * f2, total[:m] * f + total2 * f2, both
    out = torch.empty_like(q) if state["out"] is None else state["out"]
    out[:rows] = (o / torch.where(total == 0, 1.0, total)).to(q.dtype)
    if not case["lse"]:
        return {"out": out}
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=DEVICE) if state["out"] is None else state["lse_out"]
    lse[:rows] = (top + total.log())[..., 0]
    return {"out": out, "lse": lse}


# ---- the definitions in 64 bits

def exact(case, seed):
    if case["kind"] == "write":
        return _exact_write(case, seed)
    if case["kind"] == "read":
        return _exact_read(case, seed)
    return _exact_attend(case, seed)


def _values():
    """The 256 values of e4m3: sign, four bits of exponent (bias 7), three of mantissa; the last of each sign is no number."""
    v = [(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)]
    v[127] = math.nan
    return torch.tensor(v + [-x for x in v], dtype=torch.float64, device=DEVICE)


def _exact_write(case, seed):
    """Codes by search among the values, a piece of the rows at a time; the other slots as they were."""
    state = _prepare_write(case, seed)
    grid = _values()[:127]
    between = (grid[1:] + grid[:-1]) / 2
    lo, hi = EXPONENTS[case["type"]]
    got = {x: t.clone() for x, t in state["pools"].items()}
    for x in ("k", "v"):
        new = state[x].reshape(-1, case["hkv"], D)[:case["rows"]].double()
        top = new.abs().amax(-1)
        e = torch.full(top.shape, lo, dtype=torch.int64, device=DEVICE)
        for step in (128, 64, 32, 16, 8, 4, 2, 1):      # the least exponent whose largest value covers the row
            e = torch.where((e + step <= hi) & (top > 448.0 * torch.exp2((e + step - 1).double())), e + step, e)
        for i in range(0, case["rows"], 2048):
            y = new[i:i + 2048].abs() / torch.exp2(e[i:i + 2048].double())[..., None]
            c = torch.searchsorted(between, y.contiguous())                                # a tie has found the lower code
            tie = (c < 126) & (y == between[c.clamp(max=125)]) & (c % 2 == 1)
            code = c + tie.long() + 128 * torch.signbit(new[i:i + 2048]).long()
            slot = state["slots"][i:i + code.shape[0]].long()
            where = (slot // case["page"], slice(None), slot % case["page"])
            got[x].view(torch.uint8)[where] = code.to(torch.uint8)
            got[x + "_scale"][where] = (e[i:i + 2048] + 127).to(torch.uint8)
    return got


def _exact_rows(state, x, slots):
    p = state["case"]["page"]
    page, at = torch.div(slots, p, rounding_mode="floor").long(), torch.remainder(slots, p).long()
    pool = state["pools"]
    if x + "_scale" not in pool:
        return pool[x][page, :, at].double()
    codes = pool[x].view(torch.uint8)[page, :, at].long()
    return _values()[codes] * torch.exp2(pool[x + "_scale"][page, :, at].double() - 127).unsqueeze(-1)


def _exact_read(case, seed):
    state = _prepare_read(case, seed)
    return {x: _exact_rows(state, x, state["slots"]) for x in ("k", "v")}


def _exact_attend(case, seed):
    state = _prepare_attend(case, seed)
    p, hq, hkv = case["page"], case["hq"], case["hkv"]
    q = state["q"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device=DEVICE)

    def cached(table, n):
        j = torch.arange(n, device=DEVICE)
        slots = table[j // p] * p + j % p
        return [_exact_rows(state, x, slots) for x in ("k", "v")]

    group = {s: (g, n) for g, (n, a, b) in enumerate(_groups(case)) for s in range(a, b)}
    done, held, last = 0, None, -1
    for s, (n_q, n) in enumerate(state["counts"]):
        k, v = cached(state["table"][s], n)
        g, before = group.get(s, (-1, 0))
        if g >= 0:
            if g != last:
                held, last = cached(state["shared_table"][g], before), g
            k, v = torch.cat([held[0], k]), torch.cat([held[1], v])
        where = torch.arange(before + n, device=DEVICE)
        lo, hi = (_ints(x).long() for x in _spans(case, n_q, n, before))
        for h in range(hkv):
            kt, vh = k[:, h].t().contiguous(), v[:, h].contiguous()
            for e in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                for i in range(0, n_q, 4096):
                    j = min(n_q, i + 4096)
                    z = (q[done + i:done + j, e].double() @ kt) * D ** -0.5
                    if case["cap"] > 0:
                        z = case["cap"] * (z / case["cap"]).tanh()
                    if case["alibi"]:
                        far = torch.arange(before + n - n_q + i, before + n - n_q + j, device=DEVICE).view(-1, 1) - where
                        z = z - 2.0 ** (-8.0 * (e + 1) / hq) * far.abs()
                    z[(where < lo[i:j].view(-1, 1)) | (where >= hi[i:j].view(-1, 1))] = -math.inf
                    total = torch.logsumexp(z, dim=1)
                    lse[done + i:done + j, e] = total
                    out[done + i:done + j, e] = torch.nan_to_num((z - total.view(-1, 1)).exp(), nan=0.0) @ vh
        done += n_q
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
