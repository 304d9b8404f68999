"""GPU parity of the paged caches (block tables and slot maps, rows to slots, attention over pages) against the float64
oracle, and of a program that uses them together."""
import math

import numpy as np
import pytest
import torch

import paper_2606_15157_amd as rkv
from oracle import pages as OG

pytestmark = pytest.mark.gpu

NAN = float("nan")
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step, relative


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


# ------------------------------------------------------------------ block tables and slot maps

def run_resize(pages, new, max_new, **kw):
    """One call against the oracle; returns what it returned."""
    old = {k: pages[k].cpu().tolist() for k in ("table", "lens", "ring", "cursor")}
    want = OG.resize(old["table"], old["lens"], old["ring"], old["cursor"], new, pages["page_size"], max_new)
    got = rkv.pages_resize(pages, ints(new), max_new, **kw)
    assert got["status"].tolist() == [want["status"]]
    for k in ("slots", "cu_new", "lens", "cursor"):
        assert got[k].tolist() == want[k], k
    assert pages["table"].tolist() == want["table"]
    assert pages["ring"].tolist() == want["ring"]
    return got


@pytest.mark.parametrize("n,page,most", [(1, 16, 100), (1, 1, 1), (7, 5, 33), (64, 16, 500), (65, 64, 3000), (200, 7, 900), (1025, 16, 60),
                                         (8192, 16, 40)])
def test_resize_follows_the_oracle_turn_by_turn(n, page, most):
    """Requests grow, shrink, end and enter over several turns on one state."""
    rng = np.random.default_rng(n * 31 + page)
    width = -(-most // page)
    pages = rkv.pages_init(n, width, n * width + 3, page)
    lens = [0] * n
    for turn in range(6):
        new = [int(x) for x in rng.integers(0, most + 1, n)]
        keep = rng.random(n) < 0.5
        new = [min(most, a + 1) if k else b for a, b, k in zip(lens, new, keep)]
        max_new = sum(max(0, b - a) for a, b in zip(lens, new)) + int(rng.integers(0, 9))
        got = run_resize(pages, new, max_new)
        if got["status"].item() == 0:
            lens = new
            rows = [pages["table"][s, :-(-x // page)].tolist() for s, x in enumerate(lens)]
            held = [p for r in rows for p in r]
            assert len(set(held)) == len(held)


def test_resize_without_in_place_leaves_lengths_and_cursor():
    pages = rkv.pages_init(3, 8, 20, 4)
    run_resize(pages, [5, 9, 1], 15)
    before = pages["lens"].tolist(), pages["cursor"].tolist()
    got = run_resize(pages, [6, 0, 30], 30, in_place=False)
    assert (pages["lens"].tolist(), pages["cursor"].tolist()) == before and got["lens"].tolist() == [6, 0, 30]


@pytest.mark.parametrize("what", ["pages", "slots", "long", "negative", "head", "count", "old"])
def test_resize_changes_nothing_when_it_cannot_serve_all(what):
    pages = rkv.pages_init(4, 4, 9, 8)
    run_resize(pages, [8, 3, 0, 17], 28)
    new, max_new = [9, 3, 4, 17], 5
    if what == "pages":
        new, max_new = [32, 32, 32, 17], 100
    elif what == "slots":
        max_new = 4
    elif what == "long":
        new = [33, 3, 4, 17]
    elif what == "negative":
        new = [9, -1, 4, 17]
    elif what == "head":
        pages["cursor"][0] = 9
    elif what == "count":
        pages["cursor"][1] = -1
    else:
        pages["lens"][2] = 40
    got = run_resize(pages, new, max_new)
    assert got["status"].item() == (1 if what == "pages" else 2)
    assert got["slots"].tolist() == [-1] * max_new


def test_resize_of_many_new_tokens_and_a_ring_that_wraps():
    """More slots than one workgroup fills, pages given back around the ring's end."""
    pages = rkv.pages_init(40, 600, 40 * 40, 16)
    rng = np.random.default_rng(5)
    for turn in range(5):
        new = [int(x) for x in rng.integers(0, 640, 40)]
        run_resize(pages, new, 40 * 640)
    new = [0] * 40
    run_resize(pages, new, 0)
    run_resize(pages, [9600, 9600] + [0] * 38, 20000)


def test_resize_of_no_sequences():
    pages = rkv.pages_init(0, 4, 9, 8)
    got = rkv.pages_resize(pages, ints([]), 3)
    assert got["slots"].tolist() == [-1] * 3 and got["cu_new"].tolist() == [0] and got["status"].item() == 0


# ------------------------------------------------------------------ rows to slots

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,hkv,page,layout", [(1, 8, 16, "rows"), (7, 1, 1, "rows"), (300, 3, 7, "fused"), (130, 8, 100, "heads"),
                                               (4099, 2, 64, "fused")])
def test_write_puts_every_row_in_its_slot_and_touches_no_other(T, hkv, page, layout, dtype):
    g = torch.Generator(device="cuda").manual_seed(T)
    n_pages = -(-2 * T // page) + 2
    pool = torch.randn((2, n_pages, hkv, page, 128), device="cuda", generator=g).to(dtype)
    if layout == "heads":
        k, v = (torch.randn((2, hkv, T // 2, 128), device="cuda", generator=g).to(dtype).permute(0, 2, 1, 3) for _ in range(2))
    elif layout == "fused":
        x = torch.randn((T, 2 * hkv + 4, 128), device="cuda", generator=g).to(dtype)
        k, v = x[:, 4:4 + hkv], x[:, 4 + hkv:]
    else:
        k, v = (torch.randn((T, hkv, 128), device="cuda", generator=g).to(dtype) for _ in range(2))
    slots = torch.randperm(n_pages * page, device="cuda", generator=g)[:T].to(torch.int32)
    if T > 5:
        slots[3], slots[T - 1], slots[4] = -1, n_pages * page, -7
    want = pool.cpu().clone()
    for x, src in ((want[0], k), (want[1], v)):
        src = src.reshape(T, hkv, 128).cpu()
        for t, s in enumerate(slots.tolist()):
            if 0 <= s < n_pages * page:
                x[s // page, :, s % page] = src[t]
    rkv.pages_write(rkv.PagedCache(pool[0], pool[1]), k, v, slots)
    assert torch.equal(pool.cpu().view(torch.int16), want.view(torch.int16))


def test_write_and_attend_past_32_bit_offsets():
    """A pool of more than 2^32 elements: the last page's rows."""
    page, n_pages = 1024, (1 << 25) // 1024 + 2
    pool = torch.empty((n_pages, 1, page, 128), dtype=torch.bfloat16, device="cuda")
    k = torch.randn((70, 1, 128), device="cuda").to(torch.bfloat16)
    slots = torch.arange(n_pages * page - 70, n_pages * page, dtype=torch.int32, device="cuda")
    cache = rkv.PagedCache(pool, pool)
    rkv.pages_write(cache, k, k, slots)
    assert torch.equal(pool[-1, 0, -70:], k[:, 0])
    q = torch.randn((1, 1, 128), device="cuda").to(torch.bfloat16)
    out = rkv.pages_attend(cache, q, ints([[n_pages - 1]]), ints([page]), window=70)
    small = rkv.PagedCache(k.view(1, 1, 70, 128), k.view(1, 1, 70, 128))
    want = rkv.pages_attend(small, q, ints([[0]]), ints([70]))
    assert (out - want).abs().max() <= 2 * 2.0 ** -8 * want.abs().max() + 2.0 ** -8 * k.abs().max()


# ------------------------------------------------------------------ attention

class Case:
    """Pools whose every slot outside the sequences holds NaN, tables, and queries."""

    def __init__(self, lens, hq=4, hkv=2, page=16, dtype=torch.bfloat16, seed=0, pad=0, spread=1.0, nhd=False, width=0):
        rng = np.random.default_rng(seed)
        self.lens, self.page, self.dtype = lens, page, dtype
        counts = [-(-n // page) for _, n in lens]
        n_pages = sum(counts) + 2
        ids = rng.permutation(n_pages)
        self.table = np.full((len(lens), max(counts + [width]) + 1), -1, dtype=np.int32)
        shape = (n_pages, page, hkv, 128) if nhd else (n_pages, hkv, page, 128)
        self.k, self.v = (torch.full(shape, NAN, dtype=dtype, device="cuda") for _ in range(2))
        if nhd:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        at = 0
        for s, (c, (_, n)) in enumerate(zip(counts, lens)):
            self.table[s, :c] = ids[at:at + c]
            at += c
            for j in range(c):
                m = min(page, n - j * page)
                for x in (self.k, self.v):
                    x[int(self.table[s, j]), :, :m] = torch.from_numpy(rng.standard_normal((hkv, m, 128)) * spread).to("cuda", dtype)
        self.rows = sum(m for m, _ in lens)
        self.q = torch.from_numpy(rng.standard_normal((self.rows + pad, hq, 128)) * spread).to("cuda", dtype)
        self.cu = np.cumsum([0] + [m for m, _ in lens]).tolist()
        self.cache = rkv.PagedCache(self.k, self.v)

    def check(self, q=None, rows=None, **kw):
        """The call against the oracle, every element within what the roundings may move it by."""
        q = self.q if q is None else q
        dev = {k: torch.tensor(np.asarray(x), device="cuda", dtype=torch.float32 if k == "slopes" else torch.int32)
               for k, x in kw.items() if k in ("slopes", "prefix_lens", "first_keys") and x is not None}
        same = {k: x for k, x in kw.items() if k not in dev}
        lens = [n for _, n in self.lens]
        out, lse = rkv.pages_attend(self.cache, q, ints(self.table.tolist()), ints(lens), ints(self.cu), return_lse=True, **{**same, **dev})
        drop = {k: x for k, x in kw.items() if k not in ("max_q", "max_kv", "out", "lse_out")}
        want, log, weight, reach = OG.attend(f64(self.k), f64(self.v), f64(q), self.table, lens, self.cu, **drop)
        n = self.rows
        compare(out[:n], lse[:n], want[:n], log[:n], weight[:n], reach[:n], self.dtype, kw.get("softcap", 0.0), kw.get("slopes"),
                max([x for x in lens] + [1]))
        return out, lse


def compare(out, lse, want, log, weight, reach, dtype, softcap=0.0, slopes=None, most=1):
    """A score is off by the fp32 sum of 128 products (each addition half a step of 2^-23 of what has been summed, at most
    `reach`), its scaling, the cap (a few steps of the cap itself) and the bias (a step of slope times distance); the reference's
    subtraction and the exponential add steps of the score's size and one of the result.  A probability's relative error is
    that, plus half a step of its type where it is rounded for the product; the output's is half a step again."""
    top = reach + (np.max(np.abs(slopes)) * most if slopes is not None else 0.0)
    score = 2.0 ** -24 * (140 * reach + 8 * top + 16 * softcap + 8)
    assert not torch.isnan(out).any() and not torch.isnan(lse).any()
    got, empty = f64(lse), np.isneginf(log)
    assert (np.isneginf(got) == empty).all()
    # sums of up to 2^18 terms in 32 bits, in parts of at most a few thousand: below 2^-13 relative in all
    off = np.where(empty, 0.0, got - np.where(empty, 0.0, log))
    assert (np.abs(np.where(empty, 0.0, off)) <= score + 2.0 ** -13 * 0.01 + 2.0 ** -22 * np.abs(np.where(empty, 0.0, log))).all(), np.abs(off[~empty]).max()
    u = HALF[dtype]
    # a probability below the type's normal range keeps an absolute step only (fp16: 2^-25 of the largest one)
    tiny = 2.0 ** -25 * most if dtype == torch.float16 else 0.0
    bound = u * (weight + np.abs(want)) * 1.01 + (2 * score[..., None] + 2.0 ** -15) * weight + tiny
    bad = np.abs(f64(out) - want) - bound
    assert (bad <= 0).all(), (bad.max(), np.argwhere(bad > 0)[:4])


FEW = [(4, 4), (2, 300), (3, 64), (1, 900), (4, 1030), (2, 1)]
ONE = [(1, 1), (1, 2), (1, 63), (1, 64), (1, 65), (1, 500), (1, 1025), (1, 16)]
MANY = [(5, 5), (1, 130), (70, 200), (33, 33), (0, 40), (129, 300), (2, 2), (0, 0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("page", [1, 7, 16, 48, 64, 100, 2000])
def test_attention_over_any_page_size(page, dtype):
    Case(ONE, page=page, dtype=dtype, seed=page).check(max_q=1)
    Case(MANY, page=page, dtype=dtype, seed=page + 1).check()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (6, 2), (10, 2), (8, 1), (16, 2), (24, 1), (40, 1), (33, 1), (200, 1)])
def test_attention_over_head_layouts(hq, hkv):
    Case(ONE, hq=hq, hkv=hkv, seed=hq).check()
    Case([(1, 300), (3, 70), (40, 200), (0, 3)], hq=hq, hkv=hkv, seed=hq + 1).check()


@pytest.mark.parametrize("lens", [ONE, MANY, FEW], ids=["one", "many", "few"])
@pytest.mark.parametrize("kw", [
    dict(causal=False), dict(window=1), dict(window=64), dict(window=50), dict(softcap=2.0), dict(softcap=50.0), dict(scale=0.5),
    dict(scale=-0.2), dict(scale=0.0), dict(softcap=3.0, window=50), dict(softcap=3.0, slopes=True, window=50),
    dict(prefix_lens=1000), dict(prefix_lens=37), dict(prefix_lens=37, window=20), dict(slopes=True),
    dict(slopes=True, softcap=5.0, prefix_lens=64), dict(first_keys="half"), dict(first_keys="beyond"), dict(causal=False, window=33)],
    ids=lambda d: "-".join(f"{k}{v}" for k, v in d.items()))
def test_attention_masks_and_scores(lens, kw):
    kw = dict(kw)
    c = Case(lens, hq=6, hkv=2, page=16, seed=11)
    if "slopes" in kw:
        kw["slopes"] = np.array([2.0 ** -(i + 1) for i in range(6)], dtype=np.float32)
    if "prefix_lens" in kw:
        kw["prefix_lens"] = [kw["prefix_lens"]] * len(lens)
    if "first_keys" in kw:
        at = [n - m + i for m, n in lens for i in range(m)]
        # half of them begin halfway, the others nowhere a row sees: its own slot's next
        kw["first_keys"] = [p // 2 if kw["first_keys"] == "half" or t % 2 else p + 1 for t, p in enumerate(at)]
    out, lse = c.check(**kw)
    if kw.get("first_keys") and kw["first_keys"][0] > 0:
        assert (out[0] == 0).all() and torch.isneginf(lse[0]).all()


@pytest.mark.parametrize("lens", [MANY, [(300, 4000)], [(1, 2000), (200, 260), (1, 1), (70, 3000), (0, 9), (129, 129), (1, 700)]], ids=["many", "chunk", "mixed"])
@pytest.mark.parametrize("kw", [dict(), dict(window=70), dict(prefix_lens=50), dict(first_keys="half"), dict(softcap=4.0, slopes=True)],
                         ids=lambda d: "-".join(f"{k}{v}" for k, v in d.items()) or "plain")
@pytest.mark.parametrize("page", [16, 30])
def test_row_tiles_that_share_the_chip(lens, kw, page):
    """Tables wide enough for sequences of 16K slots: the tiles' keys are shared out, and split rows joined."""
    kw = dict(kw)
    c = Case(lens, hq=4, hkv=1, page=page, seed=21, width=16384 // page)
    if "slopes" in kw:
        kw["slopes"] = np.array([0.5, 0.1, 0.02, 0.003], dtype=np.float32)
    if "prefix_lens" in kw:
        kw["prefix_lens"] = [kw["prefix_lens"]] * len(lens)
    if "first_keys" in kw:
        kw["first_keys"] = [(n - m + i) // 2 for m, n in lens for i in range(m)]
    c.check(**kw)


def test_more_row_tiles_than_are_listed():
    """1100 sequences: a workgroup per tile, decoding sequences before chunks, in either numbering of the tiles."""
    lens = [(1, 1 + 7 * s % 90) for s in range(1098)]
    Case(lens + [(100, 300), (65, 65)], hq=2, hkv=1, seed=22).check()
    Case([(130, 140)] * 40 + [(1, 33)] * 3, hq=2, hkv=1, seed=23).check()


def test_calls_of_nothing():
    c = Case([(1, 4)], seed=45)
    none = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    out, lse = rkv.pages_attend(c.cache, none, ints([]).view(0, 5), ints([]), ints([0]), return_lse=True)
    assert out.shape == (0, 4, 128) and lse.shape == (0, 4)
    held = torch.full((3, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    rkv.pages_attend(c.cache, held.clone(), ints([]).view(0, 5), ints([]), ints([0]), out=held)
    assert (held == 7).all()
    out, lse = rkv.pages_attend(c.cache, c.q, ints([]).view(1, 0), ints([4]), return_lse=True)      # a table of no pages
    assert (out == 0).all() and torch.isneginf(lse).all()
    rkv.pages_write(c.cache, none[:, :2], none[:, :2], ints([]))


def test_pages_that_a_window_has_left_behind():
    """Ids of pages below every window are no longer pages."""
    c = Case([(1, 700), (5, 300)], seed=46)
    c.table[0, :700 // 16 - 4] = -1
    c.table[1, :300 // 16 - 5] = 1 << 20
    c.check(window=50)


def test_queries_before_the_first_slot_see_nothing():
    """More rows than slots: the first ones' positions are negative."""
    out, lse = Case([(9, 4), (3, 0), (1, 20)], seed=2).check()
    assert (out[:5] == 0).all() and torch.isneginf(lse[9:12]).all()


@pytest.mark.parametrize("hints", [dict(), dict(max_q=1), dict(max_q=300, max_kv=400), dict(max_q=1, max_kv=1), dict(max_q=10 ** 6, max_kv=10 ** 6)])
def test_bounds_change_no_result(hints):
    """max_q and max_kv choose kernels only, wrong ones too."""
    Case(MANY, seed=3).check(**hints)
    Case([(1, 900), (1, 5), (1, 0)], seed=4, hq=8).check(**hints)


def test_large_scores_and_sinks():
    """Scores far apart: the running maximum moves late, early and by hundreds."""
    Case([(1, 700), (40, 333)], seed=5, spread=4.0).check()
    c = Case([(1, 4000), (20, 1000)], seed=6)
    for s, j in ((0, 3900), (1, 3), (1, 970)):
        c.k[int(c.table[s, j // 16]), :, j % 16] = 20 * c.q[0, ::2]
    c.check()


def test_long_sequences_in_few_rows():
    Case([(1, 40000), (1, 17), (1, 9001)], hq=8, hkv=1, page=64, seed=7).check(max_q=1, max_kv=40000)
    Case([(30, 20011)], hq=4, hkv=1, page=32, seed=8).check()


@pytest.mark.parametrize("nhd", [False, True])
def test_strided_tensors(nhd):
    """Queries sliced from a fused projection, an output with gaps, pools of either order; rows behind the last sequence and gaps
    stay as they were."""
    c = Case([(3, 50), (1, 200), (20, 20)], hq=4, hkv=2, seed=9, pad=5, nhd=nhd)
    wide = torch.randn((29, 9, 128), device="cuda").to(torch.bfloat16)
    wide[:, 2:6] = c.q
    held = torch.full((29, 7, 256), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((29, 4), 7.0, device="cuda")
    out, _ = c.check(q=wide[:, 2:6], out=held[:, 1:5, 128:], lse_out=lse)
    assert (held[24:] == 7).all() and (lse[24:] == 7).all()
    assert (held[:, 0] == 7).all() and (held[:, 5:] == 7).all() and (held[..., :128] == 7).all()


def test_dimensions_of_one_have_no_stride():
    """Pools of one page, head or slot and calls of one row, whose strides there say nothing; the widest window."""
    pool = torch.randn((2, 40, 1, 1, 128), device="cuda").to(torch.bfloat16)
    odd = pool.as_strided((2, 40, 1, 1, 128), (40 * 128, 128, 3, 1 << 40, 1))
    q = torch.randn((1, 2, 128), device="cuda").to(torch.bfloat16)
    odd_q = q.as_strided((1, 2, 128), (5, 128, 1))
    table = torch.arange(40, dtype=torch.int32, device="cuda").view(1, 40)
    odd_table = table.as_strided((1, 40), (0, 1))
    want = rkv.pages_attend(rkv.PagedCache(*pool), q, table, ints([40]))
    assert torch.equal(rkv.pages_attend(rkv.PagedCache(*odd), odd_q, odd_table, ints([40]), window=2 ** 31 - 1), want)
    rkv.pages_write(rkv.PagedCache(*odd), pool[0, :1, 0].as_strided((1, 1, 128), (7, 9, 1)), pool[1, :1, 0], ints([3]))
    assert torch.equal(pool[0, 3], pool[0, 0]) and torch.equal(pool[1, 3], pool[1, 0])
    Case([(9, 4), (3, 3)], seed=32).check(causal=False, window=2 ** 31 - 1)


def test_nan_and_infinity_where_no_row_looks():
    """Slots before the window and behind the row's own hold NaN and infinities."""
    c = Case([(1, 300), (1, 77)], seed=10)
    want = c.check(window=40)[0]
    for s, n in ((0, 300), (1, 77)):
        for j in range(n - 40):
            for x, bad in ((c.k, NAN), (c.v, math.inf if j % 2 else -math.inf)):
                x[int(c.table[s, j // 16]), :, j % 16] = bad
    got = rkv.pages_attend(c.cache, c.q, ints(c.table.tolist()), ints([300, 77]), window=40, max_q=1)
    assert not torch.isnan(got).any() and torch.equal(got, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kw", [dict(), dict(first_keys=True), dict(window=30), dict(prefix_lens=[20, 40, 0, 89])], ids=["causal", "documents", "window", "prefix"])
@pytest.mark.parametrize("wide", [0, 16384])
def test_nan_and_infinity_reach_only_the_rows_that_see_them(kw, dtype, wide):
    """V of a few slots is not finite: columns of rows that do not see those slots are as without them, though others of the
    same tiles do; rows that see them are not finite where V is not."""
    kw = dict(kw)
    lens = [(150, 150), (40, 200), (1, 70), (3, 90)]
    c = Case(lens, hq=4, hkv=2, page=16, seed=31, dtype=dtype, width=wide // 16)
    if "first_keys" in kw:
        kw["first_keys"] = [(n - m + i) // 50 * 50 for m, n in lens for i in range(m)]
    want, log, weight, reach = OG.attend(f64(c.k), f64(c.v), f64(c.q), c.table, [n for _, n in lens], c.cu, **kw)
    bad = [(0, 70, NAN, 5), (0, 70, math.inf, 9), (0, 140, -math.inf, 127), (1, 180, NAN, 64), (1, 10, math.inf, 0), (2, 3, NAN, 1), (3, 88, NAN, 33), (3, 55, -math.inf, 34)]
    for s, j, x, d in bad:
        c.v[int(c.table[s, j // 16]), :, j % 16, d] = x
    dev = {k: ints(x) if isinstance(x, list) else x for k, x in kw.items()}
    got, lse = rkv.pages_attend(c.cache, c.q, ints(c.table.tolist()), ints([n for _, n in lens]), ints(c.cu), return_lse=True, **dev)
    filled, row = got.clone(), 0
    for s, (m, n) in enumerate(lens):
        for i in range(m):
            p = n - m + i
            lo = max(0, p - kw["window"] + 1 if "window" in kw else 0, kw["first_keys"][row] if "first_keys" in kw else 0)
            hi = max(p + 1, min(n, kw["prefix_lens"][s])) if "prefix_lens" in kw else p + 1
            hit = [d for t, j, _, d in bad if t == s and lo <= j < hi]
            assert not torch.isfinite(got[row][:, hit]).any()
            filled[row][:, hit] = torch.from_numpy(want[row][:, hit]).to("cuda", dtype)
            row += 1
    compare(filled, lse, want, log, weight, reach, dtype, most=200)


def test_pages_outside_the_pool_read_as_zeros():
    """Page ids that are no page: rows of zeros, and no fault; the other sequence's results are its own."""
    c = Case([(2, 64), (2, 64)], seed=12)
    c.table[0, 1], c.table[0, 2] = 1 << 30, -5
    c.check()


def test_sequences_that_share_pages():
    c = Case([(1, 100), (4, 90)], seed=13)
    c.table[1, :4] = c.table[0, :4]
    c.check()


def test_repeats_are_bit_equal_and_a_side_stream_serves():
    c = Case([(1, 5000), (70, 900), (1, 1)], hq=8, seed=14)
    args = (c.cache, c.q, ints(c.table.tolist()), ints([5000, 900, 1]), ints(c.cu))
    want = rkv.pages_attend(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [rkv.pages_attend(*args, stream=side) for _ in range(3)]
    side.synchronize()
    for x in got:
        assert torch.equal(x, want)


def test_two_calls_at_once():
    """Calls whose keys are shared out, on two streams side by side, each with a workspace of its own."""
    cases = [Case([(1, 9000), (1, 300), (2, 4000)], hq=8, seed=41), Case([(40, 5000), (1, 2000)], hq=8, seed=42)]
    args = [(c.cache, c.q, ints(c.table.tolist()), ints([n for _, n in c.lens]), ints(c.cu)) for c in cases]
    want = [rkv.pages_attend(*a) for a in args]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            got[i].append(rkv.pages_attend(*args[i], stream=s))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(x, w) for x in g)


def test_captured_calls_replay_with_other_lengths():
    """Calls of both kinds in one graph, replayed with other lengths and queries, against eager calls."""
    long = Case([(1, 9000), (1, 300), (1, 4000)], hq=8, seed=43)
    chunk = Case([(40, 500), (70, 200)], hq=8, seed=44)
    state = [(c, ints(c.table.tolist()), ints([n for _, n in c.lens]), ints(c.cu)) for c in (long, chunk)]
    call = lambda: [rkv.pages_attend(c.cache, c.q, t, n, cu, return_lse=True) for c, t, n, cu in state]  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    g = torch.Generator(device="cuda").manual_seed(4)
    for turn in range(4):
        for c, _, n, _ in state:
            c.q.copy_(torch.randn(c.q.shape, device="cuda", generator=g))
            n.copy_(torch.tensor([max(m, x - 97 * turn) for m, x in c.lens], device="cuda"))
        graph.replay()
        got = [(o.clone(), l.clone()) for o, l in held]
        for (o, l), (eo, el) in zip(got, call()):
            assert torch.equal(o, eo) and torch.equal(l, el)


# ------------------------------------------------------------------ together

def test_evicted_prompt_moves_into_pages_and_is_attended():
    """evict_prefill, its caches into pages, new tokens written and attended, layer by layer with their own capacities."""
    g = torch.Generator(device="cuda").manual_seed(1)
    B, hkv, hq, L = 2, 2, 8, 400
    rules, budgets = [rkv.SNAPKV, rkv.STREAMING, rkv.H2O, rkv.FULL], [77, 40, 130, 0]
    plan = rkv.Plan(rules, budgets, window=32)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    k, v, q = ([rand(B, h, n, 128) for _ in rules] for h, n in ((hkv, L), (hkv, L), (hq, 32)))
    out = rkv.evict_prefill(plan, q, k, v, check_status=True)
    layers = rkv.pages_init_from_prefill(plan, out, page_size=16, extra=3)
    for l, (cache, pages) in enumerate(layers):
        n = plan.retained_counts(L)[l]
        assert pages["lens"].tolist() == [n] * B
        new_k, new_v, new_q = rand(B * 3, hkv, 128), rand(B * 3, hkv, 128), rand(B * 3, hq, 128)
        step = rkv.pages_resize(pages, pages["lens"] + 3, B * 3)
        rkv.pages_write(cache, new_k, new_v, step["slots"])
        got, lse = rkv.pages_attend(cache, new_q, pages["table"], pages["lens"], step["cu_new"], return_lse=True)
        rows_k, rows_v = (torch.cat([out[x][l], new.view(B, 3, hkv, 128).transpose(1, 2)], 2) for x, new in (("k_out", new_k), ("v_out", new_v)))
        want = OG.attend(f64(rows_k), f64(rows_v), f64(new_q), [[0], [1]], [n + 3] * B, [0, 3, 6])
        compare(got, lse, *want, torch.bfloat16, most=n + 3)


def test_decode_caches_are_read_in_place():
    """The caches of decode_step as pools of one page a sequence."""
    g = torch.Generator(device="cuda").manual_seed(2)
    B, hkv, hq, L = 3, 2, 4, 300
    plan = rkv.Plan([rkv.TOVA], [50], [rkv.TOVA], [50], window=32)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    out = rkv.evict_prefill(plan, [rand(B, hq, 32, 128)], [rand(B, hkv, L, 128)], [rand(B, hkv, L, 128)], check_status=True)
    state = rkv.decode_init_from_prefill(plan, out)
    cache = rkv.PagedCache(state["k_cache"][0], state["v_cache"][0])
    table, lens = torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1), ints([50] * B)
    for t in range(3):
        q = rand(B, hq, 128)
        rkv.decode_step(plan, state, [q], [rand(B, hkv, 128)], [rand(B, hkv, 128)], L + t)
        got, lse = rkv.pages_attend(cache, q, table, lens, return_lse=True)
        want = OG.attend(f64(state["k_cache"][0]), f64(state["v_cache"][0]), f64(q), table.tolist(), [50] * B)
        compare(got, lse, *want, torch.bfloat16, most=50)


def test_a_captured_step_replays():
    """One decode step (tables, rows, attention) in a graph, replayed with eager work between, against the oracle."""
    n, hkv, hq, page = 5, 2, 8, 4
    pages = rkv.pages_init(n, 20, 100, page)
    pool = torch.full((2, 100, hkv, page, 128), NAN, dtype=torch.bfloat16, device="cuda")
    cache = rkv.PagedCache(pool[0], pool[1])
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    start = [1, 0, 7, 30, 4]
    step = rkv.pages_resize(pages, ints(start), 42)
    seen = [rand(42, hkv, 128), rand(42, hkv, 128)]
    rkv.pages_write(cache, *seen, step["slots"])
    hist = [[[x[i] for i in range(sum(start[:s]), sum(start[:s + 1]))] for s in range(n)] for x in seen]
    q, k, v = rand(n, hq, 128), rand(n, hkv, 128), rand(n, hkv, 128)
    new_lens = torch.empty_like(pages["lens"])

    def tick():
        torch.add(pages["lens"], 1, out=new_lens)
        step = rkv.pages_resize(pages, new_lens, n)
        rkv.pages_write(cache, k, v, step["slots"])
        return rkv.pages_attend(cache, q, pages["table"], pages["lens"], step["cu_new"], max_q=1, return_lse=True)

    saved = {x: pages[x].clone() for x in ("table", "lens", "ring", "cursor")}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = tick()
    for x, t in saved.items():
        pages[x].copy_(t)
    for turn in range(6):
        q.copy_(rand(n, hq, 128)), k.copy_(rand(n, hkv, 128)), v.copy_(rand(n, hkv, 128))
        for x, src in zip(hist, (k, v)):
            for s in range(n):
                x[s].append(src[s].clone())
        if turn % 2:
            tick_out, tick_lse = tick()      # the program's own eager step
        else:
            graph.replay()
            tick_out, tick_lse = out, lse
        torch.cuda.synchronize()
        lens = [a + turn + 1 for a in start]
        assert pages["lens"].tolist() == lens
        dense = [np.zeros((n, hkv, max(lens), 128)) for _ in range(2)]
        for d, x in zip(dense, hist):
            for s in range(n):
                d[s, :, :lens[s]] = f64(torch.stack(x[s])).transpose(1, 0, 2)
        want = OG.attend(*dense, f64(q), [[s] for s in range(n)], lens)
        compare(tick_out, tick_lse, *want, torch.bfloat16, most=max(lens))


def test_refusals_reach_python():
    c = Case([(1, 4)], seed=15)
    table, lens = ints(c.table.tolist()), ints([4])
    with pytest.raises(rkv.RkvError):       # six heads over two is fine, three is not
        rkv.pages_attend(c.cache, torch.zeros((1, 3, 128), dtype=torch.bfloat16, device="cuda"), table, lens)
    odd = torch.zeros(1 * 4 * 128 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(1, 4, 128)
    with pytest.raises(rkv.RkvError):
        rkv.pages_attend(c.cache, odd, table, lens)
    for bad in (dict(lens=lens.long()), dict(table=table.t()), dict(cu_q=ints([0])), dict(first_keys=ints([0, 0])),
                dict(slopes=torch.zeros(4, device="cuda", dtype=torch.float64)), dict(out=c.q[:, :2])):
        kw = {"table": table, "lens": lens, **bad}
        with pytest.raises(ValueError):
            rkv.pages_attend(c.cache, c.q, kw.pop("table"), kw.pop("lens"), **kw)


@pytest.mark.parametrize("hq,hkv,lens,each", [(1, 1, [(1, 9000)], True), (3, 1, [(1, 9000)], True), (3, 1, [(1, 9000)], False),
                                              (6, 2, [(1, 5000), (1, 9001)], True), (1, 1, [(17, 9000)], False), (3, 3, [(19, 4001), (2, 6000)], False),
                                              (5, 1, [(5, 9000)], False), (1, 1, [(127, 3001)], False)])
def test_split_rows_of_odd_numbers(hq, hkv, lens, each):
    """Calls whose keys are shared out and whose tiles have an odd number of rows, with cu_q and (each) without."""
    c = Case(lens, hq=hq, hkv=hkv, seed=51)
    out, lse = c.check()
    if each:
        got = rkv.pages_attend(c.cache, c.q, ints(c.table.tolist()), ints([n for _, n in lens]), return_lse=True)
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)


@pytest.mark.parametrize("lens,width,page", [([(1, 40000)], 0, 64), ([(1, 900), (2, 700)], 0, 16), ([(40, 3000)], 16384, 16), ([(150, 3001)], 0, 30),
                                             ([(150, 3001)], 16384, 48)], ids=["split", "few", "chunk", "pages-of-30", "split-chunk"])
@pytest.mark.parametrize("kw", [dict(), dict(softcap=40.0), dict(softcap=40.0, slopes=True)], ids=["plain", "cap", "cap-slopes"])
@pytest.mark.parametrize("gap,sink", [(17.5, 0), (13.0, 0), (17.5, 600), (13.0, 600), (5.5, 600)])
def test_fp16_keeps_the_mass_behind_a_sink(lens, width, page, kw, gap, sink):
    """Every key but one lies `gap` below it, and that one's value is 0: the output is what the others' small probabilities hold.
    A row's largest probability is held at 2^7 or more, where half a step of fp16's smallest values is 2^-25: each key is off by
    at most 2^-32 of the largest or 2^-11 of itself, the output by half a step (2^-25 below the normal range) again."""
    kw = dict(kw)
    c = Case(lens, hq=4, hkv=2, page=page, dtype=torch.float16, seed=61, width=width // page)
    rng = np.random.default_rng(62)
    c.q.zero_()
    c.q[..., 0] = 8.0
    for s, (_, n) in enumerate(lens):
        for j in range(-(-n // page)):
            m, at = min(page, n - j * page), int(c.table[s, j])
            c.k[at, :, :m] = 0
            c.v[at, :, :m] = torch.from_numpy(rng.uniform(0.5, 1.5, (2, m, 128))).to("cuda", torch.float16)
        c.k[int(c.table[s, sink // page]), :, sink % page, 0] = 2.0      # a score of 16 times the scale
        c.v[int(c.table[s, sink // page]), :, sink % page] = 0
    top = gap if not kw else 40.0 * math.atanh(gap / 40.0)
    kw["scale"] = top / 16.0
    if "slopes" in kw:
        kw["slopes"] = np.array([0.0, 2.0 ** -16, 0.0, 2.0 ** -15], dtype=np.float32)
    dev = {k: torch.tensor(x, device="cuda") if k == "slopes" else x for k, x in kw.items()}
    n_kv = [n for _, n in lens]
    out, lse = rkv.pages_attend(c.cache, c.q, ints(c.table.tolist()), ints(n_kv), ints(c.cu), return_lse=True, **dev)
    want, log, weight, reach = OG.attend(f64(c.k), f64(c.v), f64(c.q), c.table, n_kv, c.cu, **kw)
    # scores as in compare(): products are exact here, the cap's steps are of 40
    score = 2.0 ** -24 * (140 * reach + 8 * (reach + 2) + 16 * kw.get("softcap", 0.0) + 8)
    mass = 1.5 * max(n_kv)
    bound = 2.0 ** -32 * mass + 2.0 ** -11 * 1.01 * (weight + np.abs(want)) + (2 * score[..., None] + 2.0 ** -15) * weight + 2.0 ** -25
    bad = np.abs(f64(out) - want) - bound
    assert (bad <= 0).all(), (bad.max(), np.argwhere(bad > 0)[:4])
    assert (np.abs(f64(lse) - log) <= score + 2.0 ** -13 * 0.01 + 2.0 ** -22 * np.abs(log)).all()


@pytest.mark.parametrize("scale", [0.0, 1e-12])
@pytest.mark.parametrize("slopes", [None, np.array([0.0, 0.5, 0.0, 0.1], dtype=np.float32)], ids=["cap", "cap-slopes"])
def test_the_smallest_caps_beside_hidden_nan(scale, slopes):
    """A cap whose reciprocal is past fp32: scores are 0, also for rows summed up by themselves beside a NaN that they do not see."""
    c = Case([(40, 60), (1, 30)], hq=4, hkv=2, seed=71)
    c.v[int(c.table[0, 3]), :, 2] = NAN      # slot 50
    kw = dict(scale=scale, softcap=1e-39)
    dev = {**kw, "slopes": None if slopes is None else torch.tensor(slopes, device="cuda")}
    out, lse = rkv.pages_attend(c.cache, c.q, ints(c.table.tolist()), ints([60, 30]), ints(c.cu), return_lse=True, **dev)
    want, log, weight, reach = OG.attend(f64(c.k), f64(c.v), f64(c.q), c.table, [60, 30], c.cu, slopes=slopes, **kw)
    rows = [*range(30), 40]
    assert torch.isnan(out[30:40]).all()
    compare(out[rows], lse[rows], want[rows], log[rows], weight[rows], reach[rows], c.dtype, 1e-39, slopes, 60)


@pytest.mark.parametrize("shape,strides", [((2, 2, 32, 128), (1 << 31, 32 * 128, 128, 1)), ((2, 1, 20, 128), ((1 << 31) + 8, 0, 128, 1)),
                                           ((1, 1, 16, 128), (0, 0, (1 << 27) - 8, 1)), ((1, 1, 48, 128), (0, 0, 1 << 26, 1)),
                                           ((2, 2, 16, 128), (128, 1 << 31, 256, 1))], ids=["pages", "odd-pages", "slots", "more-slots", "heads"])
def test_strides_whose_bytes_pass_32_bits(shape, strides):
    """Rows written to and read from pools of 4 to 9 GB whose pages, slots or heads lie 2 to 4 GB apart, against a dense pool."""
    need = sum((n - 1) * s for n, s in zip(shape, strides)) + 1
    far = [torch.empty(need, dtype=torch.bfloat16, device="cuda").as_strided(shape, strides) for _ in range(2)]
    near = [torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    n_pages, hkv, page, _ = shape
    T = n_pages * page
    g = torch.Generator(device="cuda").manual_seed(81)
    k, v, q = (torch.randn((T, h, 128), device="cuda", generator=g).to(torch.bfloat16) for h in (hkv, hkv, 2 * hkv))
    slots = torch.randperm(T, device="cuda", generator=g).to(torch.int32)
    got = []
    for pool in (far, near):
        cache = rkv.PagedCache(*pool)
        rkv.pages_write(cache, k, v, slots)
        got.append([rkv.pages_attend(cache, x, torch.arange(n_pages, dtype=torch.int32, device="cuda").view(1, -1), ints([T]), ints([0, x.shape[0]]))
                    for x in (q, q[:1])])
    for a, b in zip(far, near):
        assert torch.equal(a, b)
    for a, b in zip(*got):
        # both within half a step for P and half a step for the output, of the largest value at most
        assert (a.float() - b.float()).abs().max() <= 4 * 2.0 ** -8 * v.float().abs().max()
