"""GPU parity of attention over shared prefixes against the float64 oracle, in 16-bit and 8-bit pools."""
import math

import numpy as np
import pytest
import torch

import paper_2606_15157_amd as rkv
from oracle import pages as OG
from test_gpu_paged import Case, HALF, NAN, compare, f64, ints
from test_gpu_quantized import QCase

pytestmark = pytest.mark.gpu

SLOPES = [2.0 ** -(i + 1) for i in range(8)]


class Shared:
    """Sequences `lens` of (rows, own slots) whose groups' prefixes hold `prefixes` slots; group g has sizes[g] sequences, `before` come
    before the first group and whatever is left follows the last.  Prefixes and sequences are sequences of one Case."""

    def __init__(self, lens, prefixes, sizes, before=0, quant=False, **kw):
        n = len(lens)
        pad = kw.pop("pad", 0)
        self.c = (QCase if quant else Case)([*lens, *((0, p) for p in prefixes)], **kw)
        self.lens, self.prefixes, self.cu_seqs = lens, prefixes, np.cumsum([before, *sizes]).tolist()
        self.table, self.shared = self.c.table[:n], self.c.table[n:]
        self.cu, self.q, self.dtype = self.c.cu[:n + 1], self.c.q, self.c.dtype
        self.pad = pad
        if pad:
            self.q = torch.cat([self.q, torch.randn((pad, *self.q.shape[1:]), device="cuda").to(self.dtype)])

    def args(self):
        return (self.q, ints(self.shared.tolist()).view(len(self.prefixes), -1), ints(self.prefixes), ints(self.cu_seqs), ints(self.table.tolist()),
                ints([n for _, n in self.lens]), ints(self.cu))

    def oracle(self, **kw):
        return OG.attend_shared(f64(self.c.k), f64(self.c.v), f64(self.q), self.shared, self.prefixes, self.cu_seqs, self.table, [n for _, n in self.lens],
                                self.cu, **kw)

    def check(self, cu=True, **kw):
        dev = dict(kw)
        if "slopes" in kw:
            dev["slopes"] = torch.tensor(kw["slopes"], device="cuda", dtype=torch.float32)
        args = self.args() if cu else self.args()[:-1]
        out, lse = rkv.pages_attend_shared(self.c.cache, *args, return_lse=True, **dev)
        drop = {k: x for k, x in kw.items() if k not in ("max_q", "max_kv", "max_shared", "out", "lse_out")}
        want, log, weight, reach = self.oracle(**drop)
        n = self.cu[-1]
        most = max([n for _, n in self.lens] + [1]) + max(self.prefixes + [0])
        compare(out[:n], lse[:n], want[:n], log[:n], weight[:n], reach[:n], self.dtype, kw.get("softcap", 0.0), kw.get("slopes"), most)
        return out, lse


DECODE = dict(lens=[(1, 1), (1, 2), (1, 63), (1, 64), (1, 65), (1, 500), (1, 16), (1, 33)], prefixes=[300, 64, 1], sizes=[4, 2, 1])
DRAFTS = dict(lens=[(4, 4), (2, 130), (7, 20), (0, 9), (3, 3), (1, 1), (5, 70), (2, 2)], prefixes=[100, 0, 700], sizes=[3, 1, 2], before=1)
PROMPTS = dict(lens=[(70, 70), (33, 100), (1, 50), (129, 300), (2, 2), (0, 0), (40, 41)], prefixes=[257, 90], sizes=[3, 4])
SETS = {"decode": DECODE, "drafts": DRAFTS, "prompts": PROMPTS}


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page", [1, 7, 16, 48, 100])
@pytest.mark.parametrize("what", SETS)
def test_over_any_page_size(what, page, dtype, quant):
    Shared(**SETS[what], hq=4, hkv=2, page=page, dtype=dtype, seed=page, quant=quant).check()


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (6, 2), (8, 1), (24, 1), (33, 1), (200, 1)])
def test_over_head_layouts(hq, hkv, quant):
    Shared(**DECODE, hq=hq, hkv=hkv, seed=hq, quant=quant).check(max_q=1)
    Shared(**DRAFTS, hq=hq, hkv=hkv, seed=hq, quant=quant).check()


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
@pytest.mark.parametrize("width", [0, 16384], ids=["tiles", "shares"])
@pytest.mark.parametrize("what", SETS)
@pytest.mark.parametrize("kw", [dict(), dict(window=1), dict(window=64), dict(window=150), dict(softcap=2.0), dict(scale=-0.2), dict(slopes=SLOPES[:6]),
                                dict(softcap=3.0, slopes=SLOPES[:6], window=200), dict(causal=False), dict(scale=0.0)],
                         ids=lambda d: "-".join(f"{k}{v}" if k != "slopes" else k for k, v in d.items()) or "plain")
def test_masks_and_scores(what, kw, width, quant):
    Shared(**SETS[what], hq=6, hkv=2, page=16, seed=11, width=width // 16, quant=quant).check(**kw)


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
@pytest.mark.parametrize("width", [0, 16384], ids=["tiles", "shares"])
@pytest.mark.parametrize("page", [16, 30])
@pytest.mark.parametrize("kw", [dict(), dict(window=64), dict(window=200, slopes=[0.3] * 16), dict(softcap=3.0), dict(causal=False, window=100)],
                         ids=lambda d: "-".join(d) or "plain")
def test_more_rows_than_go_at_once(kw, page, width, quant):
    """Over 2048 rows of a KV head: the prefixes first, then the own slots from those sums on."""
    Shared(**PROMPTS, hq=16, hkv=1, page=page, seed=17, width=width // page, quant=quant).check(**kw)


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_long_prefixes_that_share_the_chip(dtype, quant):
    """Prefixes and own slots both split over shares, more rows than a tile, and a group of one sequence."""
    lens = [(1, 30 + 37 * s % 900) for s in range(50)] + [(3, 2000)]
    s = Shared(lens, [5003, 3000], [50, 1], hq=4, hkv=1, page=16, width=1024, seed=3, quant=quant, dtype=dtype)
    s.check(max_q=3, max_kv=2000, max_shared=5003)
    s.check(window=1500, slopes=[0.1, 0.01, 0.001, 0.0])


def test_decode_without_cu_q_and_bounds_that_change_no_result():
    lens = [(1, 1 + 7 * s % 90) for s in range(40)]
    s = Shared(lens, [600, 30, 77], [20, 3, 15], before=1, hq=8, hkv=2, seed=4)
    for kw in (dict(), dict(max_q=1), dict(max_q=300, max_kv=1, max_shared=1), dict(max_q=10 ** 6, max_kv=10 ** 6, max_shared=10 ** 6)):
        s.check(cu=False, **kw)
    s.check(cu=False, window=40, slopes=SLOPES)


def test_more_row_tiles_than_are_listed():
    lens = [(1, 1 + 7 * s % 50) for s in range(1100)]
    Shared(lens, [20 + g % 30 for g in range(1060)], [1] * 1060, hq=2, hkv=1, page=8, seed=22).check()
    Shared(lens, [70], [1100], hq=2, hkv=1, page=8, seed=23, quant=True).check()


def test_calls_of_nothing():
    s = Shared([(1, 5), (1, 7)], [20], [2], hq=4, hkv=2, seed=5)
    q, shared, plens, cu_seqs, table, lens, cu = s.args()
    # no groups; groups without sequences; sequences in no group
    want = rkv.pages_attend(s.c.cache, q, table, lens, cu)
    for sh, pl, cs in ((shared[:0], ints([]), ints([0])), (shared, plens, ints([0, 0])), (shared, plens, ints([2, 2]))):
        assert torch.equal(rkv.pages_attend_shared(s.c.cache, q, sh, pl, cs, table, lens, cu), want)
    # a prefix of no slots, and a table of no pages
    assert torch.equal(rkv.pages_attend_shared(s.c.cache, q, shared, ints([0]), cu_seqs, table, lens, cu), want)
    assert torch.equal(rkv.pages_attend_shared(s.c.cache, q, shared[:, :0], plens, cu_seqs, table, lens, cu), want)
    # own slots of none: the prefix alone
    got = rkv.pages_attend_shared(s.c.cache, q, shared, plens, cu_seqs, table, ints([0, 0]), cu)
    assert torch.allclose(got.float(), rkv.pages_attend(s.c.cache, q, shared.expand(2, -1).contiguous(), ints([20, 20]), causal=False).float(), atol=2.0 ** -6)
    # nothing at all: rows that see nothing
    out, lse = rkv.pages_attend_shared(s.c.cache, q, shared, ints([0]), cu_seqs, table, ints([0, 0]), cu, return_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()
    none = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    assert rkv.pages_attend_shared(s.c.cache, none, shared, plens, ints([0, 0]), table[:0], ints([]), ints([0])).shape == (0, 4, 128)


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
def test_strided_tensors_and_rows_behind_the_last_sequence(quant):
    s = Shared([(3, 50), (1, 200), (20, 20)], [77], [3], hq=4, hkv=2, seed=9, pad=5, quant=quant)
    wide = torch.randn((29, 9, 128), device="cuda").to(torch.bfloat16)
    wide[:, 2:6] = s.q
    s.q = wide[:, 2:6]
    held = torch.full((29, 7, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((29, 4), 7.0, device="cuda")
    s.check(out=held[:, 1:5, 128:], lse_out=lse)
    assert (held[24:] == 7).all() and (lse[24:] == 7).all()
    assert (held[:, 0] == 7).all() and (held[:, 5:] == 7).all() and (held[..., :128] == 7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
def test_sinks_in_the_prefix_and_in_the_own_slots(dtype, quant):
    """The running maximum lies in the prefix for some rows, and in their own slots for others, by hundreds."""
    s = Shared([(1, 70), (1, 300), (4, 90), (60, 80)], [900], [4], hq=4, hkv=2, seed=6, dtype=dtype, quant=quant)
    c = s.c
    for table, j, row in ((s.shared[0], 850, 0), (s.table[1], 200, 1), (s.table[2], 3, 3), (s.table[3], 30, 9)):
        c.k[int(table[j // 16]), :, j % 16] = 20 * s.q[row, ::2]
    if quant:
        c.quantize()
    s.check()


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
@pytest.mark.parametrize("window", [0, 120])
@pytest.mark.parametrize("width", [0, 16384])
@pytest.mark.parametrize("hq", [4, 64], ids=["at-once", "in-two"])
def test_nan_reaches_only_the_rows_that_see_it(hq, window, width, quant):
    """V of a few slots of the prefix and of the own slots is NaN: windows hide the prefix's from some rows of a tile."""
    lens = [(40, 60), (1, 30), (30, 200), (3, 5)]
    s = Shared(lens, [100], [4], hq=hq, hkv=2, seed=31, width=width // 16, quant=quant)
    kw = dict(window=window) if window else {}
    want, log, weight, reach = s.oracle(**kw)
    bad = [(-1, 40, 5), (-1, 95, 9), (0, 50, 64), (2, 150, 0), (3, 4, 33)]
    for q, j, d in bad:
        table = s.shared[0] if q < 0 else s.table[q]
        if quant:
            s.c.cache.v_pages.view(torch.uint8)[int(table[j // 16]), :, j % 16, d] = 127
        else:
            s.c.v[int(table[j // 16]), :, j % 16, d] = NAN
    got, lse = rkv.pages_attend_shared(s.c.cache, *s.args(), return_lse=True, **kw)
    filled, row = got.clone(), 0
    for q, (m, n) in enumerate(lens):
        for i in range(m):
            p = 100 + n - m + i
            lo = max(0, p - window + 1) if window else 0
            hit = [d for t, j, d in bad if (t < 0 and lo <= j) or (t == q and lo <= 100 + j <= p)]
            assert torch.isnan(got[row][:, hit]).all()
            filled[row][:, hit] = torch.from_numpy(want[row][:, hit]).to("cuda", torch.bfloat16)
            row += 1
    compare(filled, lse, want, log, weight, reach, torch.bfloat16, most=300)


def test_pages_outside_the_pool_and_queries_before_the_first_slot():
    s = Shared([(2, 64), (9, 4)], [64, 32], [1, 1], hq=4, hkv=2, seed=12)
    s.shared[0, 1], s.table[1, 0] = 1 << 30, -5
    s.check()


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
@pytest.mark.parametrize("kw", [dict(), dict(window=30), dict(slopes=SLOPES[:4]), dict(causal=False), dict(causal=False, window=30)],
                         ids=lambda d: "-".join(d) or "plain")
@pytest.mark.parametrize("width", [0, 16384], ids=["tiles", "shares"])
@pytest.mark.parametrize("hq,hkv", [(4, 2), (16, 1)], ids=["at-once", "in-two"])
def test_queries_among_the_prefix(hq, hkv, kw, width, quant):
    """More rows than own slots: the first ones' positions lie in the prefix, or before its first slot."""
    if "slopes" in kw:
        kw = dict(kw, slopes=[SLOPES[i % 4] for i in range(hq)])
    s = Shared([(40, 4), (1, 0), (3, 0), (2, 1), (90, 3), (1, 30)], [70, 20], [4, 2], hq=hq, hkv=hkv, seed=13, width=width // 16, quant=quant)
    s.check(**kw)


def test_cu_seqs_outside_their_range_are_cut():
    """Groups past the sequences hold the last ones; nothing else is read."""
    s = Shared([(1, 40), (1, 30), (1, 20)], [50], [3], hq=4, hkv=2, seed=8)
    q, shared, plens, _, table, lens, cu = s.args()
    want = rkv.pages_attend_shared(s.c.cache, q, shared, plens, ints([0, 3]), table, lens, cu)
    assert torch.equal(rkv.pages_attend_shared(s.c.cache, q, shared, plens, ints([-5, 1 << 30]), table, lens, cu), want)


@pytest.mark.parametrize("what", SETS)
@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
def test_pages_behind_4_gib(quant, what):
    """The same pages at the end of a pool of more than 2^32 bytes give the same bits, few rows and many."""
    s = Shared(**SETS[what], hq=8, hkv=2, quant=quant, seed=41)
    small, held = s.c.cache, ("k_pages", "v_pages") + (("k_scales", "v_scales") if quant else ())
    pools = [getattr(small, x) for x in held]
    first = 2 ** 32 // (pools[0][0].numel() * pools[0].element_size()) + 1
    far = [torch.empty((first + small.n_pages, *x.shape[1:]), dtype=x.dtype, device="cuda") for x in pools]
    for x, y in zip(far, pools):
        x.view(torch.uint8)[first:] = y.contiguous().view(torch.uint8)
    cache = rkv.QuantizedCache(*far, s.dtype) if quant else rkv.PagedCache(*far)
    q, shared, plens, cu_seqs, table, lens, cu = s.args()
    for kw in (dict(), dict(window=40)):
        want = rkv.pages_attend_shared(small, *s.args(), return_lse=True, **kw)
        got = rkv.pages_attend_shared(cache, q, shared + first, plens, cu_seqs, table + first, lens, cu, return_lse=True, **kw)
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
def test_repeats_graphs_and_streams_give_the_same_bits(quant):
    """Eager, on a side stream, and in two captured graphs that run beside each other, with other work between replays."""
    s = Shared([(1, 30 + 37 * i % 300) for i in range(30)], [3000, 100], [20, 9], hq=8, hkv=2, seed=15, width=512, quant=quant)
    args = s.args()
    call = lambda: rkv.pages_attend_shared(s.c.cache, *args, return_lse=True)  # noqa: E731
    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = rkv.pages_attend_shared(s.c.cache, *args, return_lse=True, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graphs, held = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            held.append(call())
    for i in range(4):
        for x in held:
            x[0].zero_()
        args[0].copy_(torch.randn_like(args[0], dtype=torch.float32).to(args[0].dtype))
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        want = call()
        for x in held:
            assert all(torch.equal(a, b) for a, b in zip(want, x)), i


def test_a_served_prompt_with_many_answers():
    """A prompt's pages and its answers' in one set of tables: the prompt enters once, every answer decodes behind it."""
    Hq, Hkv, P, n, steps = 8, 2, 150, 5, 20
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = lambda t, h: torch.randn((t, h, 128), device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    pages = rkv.pages_init(n + 1, 16, 60, 16)
    pool = torch.full((2, 60, Hkv, 16, 128), NAN, dtype=torch.bfloat16, device="cuda")
    cache = rkv.PagedCache(pool[0], pool[1])
    k, v = rows(P, Hkv), rows(P, Hkv)
    new = ints([P] + [0] * n)
    step = rkv.pages_resize(pages, new, max_new=P)
    rkv.pages_write(cache, k, v, step["slots"])
    own = []
    for t in range(steps):
        new = ints([P] + [t + 1] * n)
        step = rkv.pages_resize(pages, new, max_new=n)
        kt, vt, qt = rows(n, Hkv), rows(n, Hkv), rows(n, Hq)
        rkv.pages_write(cache, kt, vt, step["slots"])
        own.append((kt, vt))
        y, lse = rkv.pages_attend_shared(cache, qt, pages["table"][:1], pages["lens"][:1], ints([0, n]), pages["table"][1:], pages["lens"][1:], max_q=1,
                                         return_lse=True)
    full = [torch.cat([x.expand(n, -1, -1, -1), torch.stack([o[i] for o in own], 1)], 1).transpose(1, 2) for i, x in enumerate((k[None], v[None]))]
    want, log, weight, reach = OG.attend(f64(full[0]), f64(full[1]), f64(qt), [[b] for b in range(n)], [P + steps] * n)
    compare(y, lse, want, log, weight, reach, torch.bfloat16, most=P + steps)


def near(a, b, size, dtype, steps=2):
    """Two results of one definition: each is off by half a step of its type of itself, and by half a step of the probabilities' of
    sum p |v| (`size`, which is itself a result in that type: 1.02 times); sums in 32 bits are far below both."""
    half = HALF[dtype]
    assert ((a.float() - b.float()).abs() <= steps * half * 1.02 * (1.02 * size.float() + b.float().abs()) + 2.0 ** -20).all()


@pytest.mark.parametrize("quant", [False, True], ids=["rows", "codes"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,groups,own,kw", [(64, 3, 900, dict()), (256, 2, 40, dict()), (100, 90, 700, dict(window=3000)), (40, 2, 2500, dict(softcap=20.0)),
                                             (48, 2, 300, dict(q=7)), (48, 2, 300, dict(q=40)), (70, 60, 500, dict(q=16, window=2000))],
                         ids=["few", "many", "groups", "capped", "drafts", "in-two", "groups-in-two"])
def test_large_batches_equal_attention_over_whole_caches(n, groups, own, kw, dtype, quant):
    """Shares of many items, of both kinds, whose sizes count: against calls in which every sequence's table begins with its prefix's pages."""
    kw = dict(kw)
    m, hq, hkv, page, g = kw.pop("q", 1), 32, 8, 16, torch.Generator(device="cuda").manual_seed(n)
    rng = np.random.default_rng(n)
    prefixes = [int(x) * page for x in rng.integers(64, 300, groups)]
    lens = [int(x) for x in rng.integers(m, own + m, n)]
    cuts = [0, *sorted(rng.choice(np.arange(1, n), groups - 1, replace=False).tolist()), n]
    total = sum(prefixes) // page + sum(-(-x // page) for x in lens)
    k, v = (torch.randn((total, hkv, page, 128), device="cuda", generator=g).to(dtype) for _ in range(2))
    if quant:
        cache = rkv.QuantizedCache.empty(total, hkv, page, dtype)
        slots = torch.arange(total * page, device="cuda", dtype=torch.int32)
        rkv.pages_write(cache, *(x.transpose(1, 2).reshape(-1, hkv, 128) for x in (k, v)), slots)
        k, v = (x.view(total, page, hkv, 128).transpose(1, 2) for x in rkv.pages_read(cache, slots))
    plain, sizes = rkv.PagedCache(k, v), rkv.PagedCache(k, v.abs())
    cache = cache if quant else plain
    ids, width = iter(rng.permutation(total).tolist()), max(prefixes) // page + (own + m) // page + 2
    shared = [[next(ids) for _ in range(p // page)] for p in prefixes]
    table = [[next(ids) for _ in range(-(-x // page))] for x in lens]
    group = np.repeat(np.arange(groups), np.diff(cuts))
    pad = lambda rows, w: ints([r + [-1] * (w - len(r)) for r in rows])  # noqa: E731
    whole, all_lens = pad([shared[x] + t for x, t in zip(group, table)], width), ints([prefixes[x] + y for x, y in zip(group, lens)])
    q = torch.randn((n * m, hq, 128), device="cuda", generator=g).to(dtype)
    cu = ints([m * i for i in range(n + 1)])
    want, log = rkv.pages_attend(plain, q, whole, all_lens, cu, return_lse=True, **kw)
    size = rkv.pages_attend(sizes, q, whole, all_lens, cu, **kw)
    args = (q, pad(shared, max(prefixes) // page), ints(prefixes), ints(cuts), pad(table, (own + m) // page + 2), ints(lens), cu)
    got, lse = rkv.pages_attend_shared(cache, *args, return_lse=True, max_q=m, **kw)
    near(got, want, size, dtype)
    assert (lse - log).abs().max() <= 1e-4
    if quant:      # and the same call without sharing, in 8 bits
        got, lse = rkv.pages_attend(cache, q, whole, all_lens, cu, return_lse=True, max_q=m, **kw)
        near(got, want, size, dtype)
        assert (lse - log).abs().max() <= 1e-4


def test_gradients_are_refused():
    s = Shared([(1, 5)], [3], [1], seed=1)
    q, *rest = s.args()
    with pytest.raises(ValueError, match="backward"):
        rkv.pages_attend_shared(s.c.cache, q.clone().requires_grad_(), *rest)
