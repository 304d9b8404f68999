"""Caches in 8 bits and shared prefixes without a GPU: the oracle against hand cases, and every refusal of the C entry points and
of the binding (each before any HIP call, with pointers that are never followed)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2606_15157_amd as rkv
from paper_2606_15157_amd import _abi
from oracle import pages as OG
from test_paged_cpu import P, attend, pages, refused, rows

E4M3 = torch.float8_e4m3fn


def test_oracle_values_are_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(E4M3).double().numpy()
    assert np.array_equal(OG.e4m3_values(), want, equal_nan=True)


@pytest.mark.parametrize("kind,dtype", [("bf16", torch.bfloat16), ("fp16", torch.float16)])
def test_oracle_rows_by_hand(kind, dtype):
    lo, hi = OG.EXPONENTS[kind]
    most = torch.finfo(dtype).max
    x = np.zeros((9, 128))
    x[1, 0], x[2, 0] = 448.0, 449.0                      # the largest code, and the next exponent
    x[3, :3] = 448.0, 17.0, 19.0                         # ties to even: 16 and 20
    x[4, :2] = 1.0, 2.0 ** -19                           # 1 is 256 2^-8: half the smallest code 2^-9 2^-8 is 2^-18
    x[5, 0], x[6, 0] = most, -most
    x[7, :4] = np.nan, np.inf, -np.inf, 1.0
    x[8, 0] = 2.0 ** -30 if kind == "fp16" else 2.0 ** -133
    codes, scales = OG.encode(x, kind)
    y = OG.decode(codes, scales)
    assert scales.tolist() == [lo + 127, 127, 128, 127, 119, hi + 127, hi + 127, 119, lo + 127]
    assert y[1, 0] == 448 and y[2, 0] == 448 and y[3, :3].tolist() == [448, 16, 20] and y[4, :2].tolist() == [1, 0]
    assert y[5, 0] == 240 * 2.0 ** hi == -y[6, 0] and most * (1 - 2.0 ** -4) <= y[5, 0] <= most
    assert np.isnan(y[7, :3]).all() and y[7, 3] == 1 and (y[8] == 0).all() and (y[0] == 0).all()
    back = torch.from_numpy(y).to(dtype).double().numpy()      # every value is one of the type's
    assert np.array_equal(back, y, equal_nan=True)


@pytest.mark.parametrize("kind,dtype", [("bf16", torch.bfloat16), ("fp16", torch.float16)])
def test_oracle_codes_are_torchs_roundings(kind, dtype):
    rng = np.random.default_rng(0)
    lo, hi = OG.EXPONENTS[kind]
    x = rng.standard_normal((300, 128)) * np.exp2(rng.integers(-20, 12, (300, 1)))
    x = torch.from_numpy(x).to(dtype).double().numpy()
    codes, scales = OG.encode(x, kind)
    e = scales.astype(int) - 127
    top = np.abs(x).max(-1)
    assert (top <= 448 * np.exp2(e)).all() and ((top > 448 * np.exp2(e - 1.0)) | (e == lo)).all()
    assert np.array_equal(torch.from_numpy(x * np.exp2(-e)[:, None]).float().to(E4M3).view(torch.uint8).numpy(), codes)
    y = OG.decode(codes, scales)
    assert (np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), np.exp2(e - 10.0)[:, None])).all()
    assert np.array_equal(torch.from_numpy(y).to(dtype).double().numpy(), y)


def test_oracle_shared_prefix_is_attention_over_the_whole():
    """Three sequences, two of which begin with one prefix, against caches that hold prefix and own slots themselves."""
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 9, 2, 4, 128))
    q = rng.standard_normal((4, 4, 128))
    got = OG.attend_shared(k, v, q, [[8, 0]], [7], [1, 3], [[1, 2], [3, 4], [5, 6]], [6, 5, 2], [0, 1, 3, 4], window=9)
    flat = [x.transpose(0, 2, 1, 3).reshape(36, 2, 128) for x in (k, v)]
    slots = [list(range(4, 10)), [32, 33, 34, 35, 0, 1, 2, 12, 13, 14, 15, 16], [32, 33, 34, 35, 0, 1, 2, 20, 21]]
    whole = [np.zeros((3, 2, 12, 128)) for _ in range(2)]
    for s, at in enumerate(slots):
        for x, f in zip(whole, flat):
            x[s, :, :len(at)] = f[at].transpose(1, 0, 2)
    want = OG.attend(whole[0], whole[1], q, [[0], [1], [2]], [6, 12, 9], [0, 1, 3, 4], window=9)
    for a, b in zip(got, want):
        np.testing.assert_allclose(a, b, atol=1e-12)


# ------------------------------------------------------------------ refusals

def qpages(**kw):
    f = dict(k=P, v=P, k_scale=P + 1, v_scale=P + 2, k_page=4096, k_head=2048, k_slot=128, v_page=4096, v_head=2048, v_slot=128, ks_page=32, ks_head=16,
             ks_slot=1, vs_page=32, vs_head=16, vs_slot=1, n_pages=4, page_size=16, n_kv_heads=2, head_dim=128, dtype=0)
    f.update(kw)
    return _abi.QPages(**f)


def shared(**kw):
    f = dict(table=P, table_stride=4, lens=P, cu_seqs=P, n_groups=2, max_pages=4, max_len=0)
    f.update(kw)
    return _abi.Shared(**f)


@pytest.mark.parametrize("status,bad", [
    (1, dict(k=None)), (1, dict(v=None)), (1, dict(k_scale=None)), (1, dict(v_scale=None)), (1, dict(n_pages=0)), (1, dict(page_size=0)),
    (1, dict(n_kv_heads=0)), (1, dict(dtype=2)), (1, dict(dtype=-1)), (1, dict(k_slot=-16)), (1, dict(ks_slot=-1)), (1, dict(vs_page=-32)),
    (4, dict(head_dim=64)), (4, dict(k=P + 8)), (4, dict(v=P + 1)), (4, dict(k_head=2056)), (4, dict(v_page=8)), (4, dict(v_slot=136)),
    (4, dict(n_pages=1 << 20, page_size=1 << 11))])
def test_bad_pools_are_refused(status, bad):
    L, n = _abi.lib(), C.c_size_t()
    p = C.byref(qpages(**bad))
    refused(status, L.rkv_qpages_write(p, C.byref(rows()), None))
    refused(status, L.rkv_qpages_read(p, C.byref(rows()), None))
    refused(status, L.rkv_qpages_attend(p, C.byref(attend()), None, 0, None))
    refused(status, L.rkv_qpages_attend_workspace_size(p, C.byref(attend()), C.byref(n)))
    refused(status, L.rkv_qpages_attend_shared(p, C.byref(attend()), C.byref(shared()), None, 0, None))
    refused(status, L.rkv_qpages_attend_shared_workspace_size(p, C.byref(attend()), C.byref(shared()), C.byref(n)))


@pytest.mark.parametrize("status,bad", [
    (1, dict(k=None)), (1, dict(v=None)), (1, dict(slots=None)), (1, dict(n_tokens=-1)), (1, dict(n_outer=-1)), (1, dict(v_token=-128)),
    (4, dict(k=P + 4)), (4, dict(k_token=130)), (4, dict(v_outer=9)), (4, dict(n_outer=1 << 15, n_tokens=1 << 15))])
def test_bad_rows_are_refused(status, bad):
    L = _abi.lib()
    refused(status, L.rkv_qpages_write(C.byref(qpages()), C.byref(rows(**bad)), None))
    refused(status, L.rkv_qpages_read(C.byref(qpages()), C.byref(rows(**bad)), None))
    refused(status, L.rkv_pages_read(C.byref(pages()), C.byref(rows(**bad)), None))


def test_k_and_v_are_not_read_into_the_same_rows():
    for call, pool in ((_abi.lib().rkv_qpages_read, qpages()), (_abi.lib().rkv_pages_read, pages())):
        refused(1, call(C.byref(pool), C.byref(rows()), None), "same")


@pytest.mark.parametrize("bad", [dict(k_token=128), dict(k_head=64), dict(v_token=0), dict(n_outer=2), dict(n_outer=2, k_outer=768, v_outer=512)])
def test_rows_that_run_into_each_other_are_not_read_into(bad):
    for call, pool in ((_abi.lib().rkv_qpages_read, qpages()), (_abi.lib().rkv_pages_read, pages())):
        refused(1, call(C.byref(pool), C.byref(rows(**{"v": 2 * P, **bad})), None), "overlap")


LAYOUTS = [
    (0, dict(v=2 * P)), (1, dict(v=P + 2 * 64)), (1, dict(v=P + 2 * 384)), (1, dict(v=P + 2 * 760)), (0, dict(v=P + 2 * 768)), (0, dict(v=P - 2 * 768)), (1, dict(v=P - 2 * 760)),
    # heads 2 .. 3 and 1 .. 2 of one buffer of four; 0 .. 1 and 2 .. 3
    (1, dict(k=P + 512, v=P + 256, k_token=512, v_token=512)), (0, dict(v=P + 512, k_token=512, v_token=512)),
    # [tokens, heads, 2, d], even and odd tokens, and even ones with later even ones
    (0, dict(v=P + 256, k_head=256, v_head=256, k_token=512, v_token=512)), (0, dict(v=P + 2 * 256 * 5, k_token=512, v_token=512, n_tokens=40)),
    (1, dict(v=P + 2 * 256 * 6, k_token=512, v_token=512, n_tokens=40)), (1, dict(v=P - 2 * 256 * 6, k_token=512, v_token=512, n_tokens=40)),
    # [batch, heads, tokens, d] of one allocation, and the second beginning in the first's last row
    (0, dict(v=P + 2 * 768, k_head=384, k_token=128, v_head=384, v_token=128)), (1, dict(v=P + 2 * 640, k_head=384, k_token=128, v_head=384, v_token=128)),
    # the same memory by other strides; strides of dimensions of one do not count
    (1, dict(v=P + 2 * 128, v_token=128, v_head=512)), (0, dict(v=P + 512, k_token=512, v_token=512, k_outer=8, v_outer=1 << 40))]


@pytest.mark.parametrize("met,layout", [x for x in LAYOUTS if x[0]])
def test_rows_of_k_are_not_read_into_those_of_v(met, layout):
    for call, pool in ((_abi.lib().rkv_qpages_read, qpages()), (_abi.lib().rkv_pages_read, pages())):
        refused(1, call(C.byref(pool), C.byref(rows(**layout)), None), "overlap")


def elements(at, counts, strides):
    got = np.array([at])
    for n, s in zip(counts, strides):
        got = (got[:, None] + s * np.arange(n)).ravel()
    return (got[:, None] + np.arange(128)).ravel()


@pytest.mark.skipif(torch.cuda.is_available(), reason="without a GPU a call that is not refused ends at its launch")
def test_rows_are_refused_for_an_element_that_k_and_v_share_and_for_no_other_reason():
    """All layouts above, and drawn ones of equal strides, against the sets of their elements."""
    rng = np.random.default_rng(7)
    names = [("k_outer", "v_outer"), ("k_token", "v_token"), ("k_head", "v_head")]
    tried = [(2, rows(**x)) for _, x in LAYOUTS]
    for _ in range(600):
        counts = [int(x) for x in rng.integers(1, 5, 3)]
        strides, extent = [0] * 3, 128
        for i in rng.permutation(3):
            strides[i] = extent + 8 * int(rng.integers(0, 40))
            extent += strides[i] * (counts[i] - 1)
        far = 8 * int(rng.integers(-extent // 8 - 8, extent // 8 + 8))      # elements from k to v
        if rng.random() < 0.5:
            far = sum(int(d) * s for d, s in zip(rng.integers(-4, 5, 3), strides)) + 8 * int(rng.integers(-17, 18))
        tried.append((counts[2], rows(v=P + 2 * far, n_outer=counts[0], n_tokens=counts[1], **{x: s for pair, s in zip(names, strides) for x in pair})))
    seen = [0, 0]
    for heads, r in tried:
        counts = (r.n_outer, r.n_tokens, heads)
        meet = np.intersect1d(*(elements((getattr(r, "kv"[i]) - P) // 2, counts, [getattr(r, pair[i]) for pair in names]) for i in range(2))).size > 0
        got = _abi.lib().rkv_pages_read(C.byref(pages(n_kv_heads=heads)), C.byref(r), None)
        assert got == (1 if meet else 6), (meet, got, [(n, getattr(r, n)) for n, _ in r._fields_])
        seen[meet] += 1
    assert min(seen) >= 100, seen


@pytest.mark.parametrize("bad", [dict(k_slot=0), dict(v_slot=112), dict(k_head=0), dict(v_page=2048), dict(ks_slot=0), dict(vs_head=8), dict(ks_page=16),
                                 dict(vs_slot=2)])
def test_overlapping_pools_are_not_written(bad):
    refused(1, _abi.lib().rkv_qpages_write(C.byref(qpages(**bad)), C.byref(rows()), None), "overlap")


# Pools of 4 pages of 2 heads of 16 slots: 16 KiB of codes (32 KiB in 16 bits) and 128 scales.
APART = dict(v=2 * P, v_scale=P // 2 + 128, k_scale=P // 2)


@pytest.mark.parametrize("bad", [dict(v=P + 128), dict(v=P + 16384 - 16), dict(v=P - 16384 + 128), dict(v_scale=P // 2), dict(v_scale=P // 2 + 127),
                                 dict(v_scale=P + 5), dict(k_scale=P + 16383), dict(k_scale=2 * P, v_scale=2 * P + 128), dict(v=P), dict(v=P, v_scale=P // 2, k_page=8192),
                                 dict(k_slot=144, k_head=2304, k_page=4608, k_scale=P + 127, ks_slot=144, ks_head=2304, ks_page=4608)])
def test_written_pools_of_k_and_v_do_not_run_into_each_other(bad):
    refused(1, _abi.lib().rkv_qpages_write(C.byref(qpages(**{**APART, **bad})), C.byref(rows()), None), "overlap")


@pytest.mark.parametrize("bad", [dict(v=P + 256), dict(v=P + 32768 - 16), dict(v=P - 32768 + 16), dict(v=P, v_slot=256, v_head=128 * 32, v_page=128 * 64)])
def test_written_16_bit_pools_do_not_run_into_each_other(bad):
    pool = dict(k_page=4096, k_head=2048, k_slot=128, v_page=4096, v_head=2048, v_slot=128)
    refused(1, _abi.lib().rkv_pages_write(C.byref(pages(**{**pool, **bad})), C.byref(rows()), None), "overlap")


@pytest.mark.skipif(torch.cuda.is_available(), reason="without a GPU a call that is not refused ends at its launch")
def test_pools_that_share_no_byte_are_written():
    """Codes and scales in one piece of memory: a record a slot, a block a page, K and V by turns; and a pool whose values are its keys."""
    slot = dict(k_slot=144, k_head=2304, k_page=4608, k_scale=P + 128, ks_slot=144, ks_head=2304, ks_page=4608)
    block = dict(k_page=8192 + 64, v=P + 4096, v_page=8192 + 64, k_scale=P + 8192, ks_page=8192 + 64, v_scale=P + 8192 + 32, vs_page=8192 + 64)
    pairs = dict(k_slot=256, k_head=4096, k_page=8192, v=P + 128, v_slot=256, v_head=4096, v_page=8192)
    one = dict(v=P, v_scale=P // 2)
    for good in (dict(), dict(v=P + 16384), dict(v=P - 16384, v_scale=P // 2 - 128), slot, block, pairs, one):
        assert _abi.lib().rkv_qpages_write(C.byref(qpages(**{**APART, **good})), C.byref(rows()), None) == 6, good
    pool = dict(k_page=4096, k_head=2048, k_slot=128, v_page=4096, v_head=2048, v_slot=128)
    for good in (dict(), dict(v=P + 32768), dict(k_page=8192, v=P + 8192, v_page=8192), dict(k_slot=256, k_head=4096, k_page=8192, v=P + 256, v_slot=256, v_head=4096, v_page=8192)):
        assert _abi.lib().rkv_pages_write(C.byref(pages(**{**pool, **good})), C.byref(rows()), None) == 6, good


@pytest.mark.parametrize("status,bad", [
    (1, dict(q=None)), (1, dict(out=None)), (1, dict(lens=None)), (1, dict(table=None)), (1, dict(n_seqs=-1)), (1, dict(window=-1)), (1, dict(causal=2)),
    (1, dict(scale=float("nan"))), (1, dict(softcap=-1.0)), (4, dict(softcap=600.0)), (1, dict(out_token=0)), (2, dict(n_q_heads=3)), (2, dict(cu_q=None)),
    (2, dict(table_stride=3)), (4, dict(q=P + 8)), (4, dict(q_head=130)), (4, dict(max_pages=1 << 27, table_stride=1 << 27)), (4, dict(n_rows=1 << 29))])
def test_bad_attention_calls_are_refused(status, bad):
    L = _abi.lib()
    refused(status, L.rkv_qpages_attend(C.byref(qpages()), C.byref(attend(**bad)), None, 0, None))
    for call, pool in ((L.rkv_qpages_attend_shared, qpages()), (L.rkv_pages_attend_shared, pages())):
        refused(status, call(C.byref(pool), C.byref(attend(**bad)), C.byref(shared()), None, 0, None))


@pytest.mark.parametrize("status,bad", [
    (1, dict(n_groups=-1)), (1, dict(max_pages=-1)), (1, dict(max_len=-1)), (1, dict(table_stride=-4)), (2, dict(table_stride=3)),
    (1, dict(table=None)), (1, dict(lens=None)), (1, dict(cu_seqs=None)), (4, dict(max_pages=1 << 27, table_stride=1 << 27)),
    (4, dict(max_pages=(1 << 27) - 64, table_stride=1 << 27)), (4, dict(n_groups=1 << 23))])
def test_bad_prefixes_are_refused(status, bad):
    """Pages of 16 slots and 4 pages a sequence: 2^31 - 1024 slots are 2^27 - 64 pages."""
    L = _abi.lib()
    for call, pool in ((L.rkv_qpages_attend_shared, qpages()), (L.rkv_pages_attend_shared, pages())):
        refused(status, call(C.byref(pool), C.byref(attend()), C.byref(shared(**bad)), None, 0, None))


@pytest.mark.parametrize("bad", [dict(prefix_lens=P), dict(first_keys=P)])
def test_masks_that_do_not_go_with_prefixes_are_refused(bad):
    refused(4, _abi.lib().rkv_pages_attend_shared(C.byref(pages()), C.byref(attend(**bad)), C.byref(shared()), None, 0, None), "prefix_lens")


def test_null_structs_are_refused():
    L, n = _abi.lib(), C.c_size_t()
    q, r, a, g = C.byref(qpages()), C.byref(rows()), C.byref(attend()), C.byref(shared())
    for call in (L.rkv_qpages_write, L.rkv_qpages_read, L.rkv_pages_read):
        refused(1, call(None, r, None))
    refused(1, L.rkv_qpages_write(q, None, None))
    refused(1, L.rkv_qpages_read(q, None, None))
    refused(1, L.rkv_qpages_attend(None, a, None, 0, None))
    refused(1, L.rkv_qpages_attend(q, None, None, 0, None))
    refused(1, L.rkv_qpages_attend_shared(q, a, None, None, 0, None))
    refused(1, L.rkv_qpages_attend_shared(q, None, g, None, 0, None))
    refused(1, L.rkv_qpages_attend_shared(None, a, g, None, 0, None))
    refused(1, L.rkv_qpages_attend_shared_workspace_size(q, a, g, None))
    refused(1, L.rkv_qpages_attend_workspace_size(q, a, None))


def test_calls_of_nothing_need_no_gpu():
    L = _abi.lib()
    none = rows(n_tokens=0, k=None, v=None, slots=None)
    for call in (L.rkv_qpages_write, L.rkv_qpages_read):
        assert call(C.byref(qpages()), C.byref(none), None) == 0
    assert L.rkv_pages_read(C.byref(pages()), C.byref(none), None) == 0
    assert L.rkv_qpages_attend(C.byref(qpages()), C.byref(attend(n_rows=0)), None, 0, None) == 0
    assert L.rkv_qpages_attend_shared(C.byref(qpages()), C.byref(attend(n_rows=0)), C.byref(shared()), None, 0, None) == 0
    assert L.rkv_pages_attend_shared(C.byref(pages()), C.byref(attend(n_seqs=0)), C.byref(shared(n_groups=0)), None, 0, None) == 0


@pytest.mark.parametrize("cu_q", [None, P])
def test_the_workspace_of_a_shared_call_holds_its_sums_and_is_checked(cu_q):
    """528 bytes a row and head for the prefixes and for the own slots, rounded up to 256; then 1024 partial sums of up to 128 rows, all
    rows of a group among them, also where sequences have one row each, and 4096 of at most 16."""
    L, n = _abi.lib(), C.c_size_t()
    a = attend(n_seqs=40, n_rows=40, cu_q=cu_q)
    g = shared(max_pages=4000, table_stride=4000)
    for call, size, pool in ((L.rkv_qpages_attend_shared, L.rkv_qpages_attend_shared_workspace_size, qpages()),
                             (L.rkv_pages_attend_shared, L.rkv_pages_attend_shared_workspace_size, pages())):
        assert size(C.byref(pool), C.byref(a), C.byref(g), C.byref(n)) == 0
        assert n.value == (2 * 528 * 40 * 4 + 255) // 256 * 256 + (1024 * 80 + 4096 * 16) * 130 * 4
        refused(5, call(C.byref(pool), C.byref(a), C.byref(g), None, n.value, None))
        refused(5, call(C.byref(pool), C.byref(a), C.byref(g), C.c_void_p(P + 16), n.value, None))
        refused(5, call(C.byref(pool), C.byref(a), C.byref(g), C.c_void_p(P), n.value - 1, None))
        # no groups: what the plain call needs
        assert size(C.byref(pool), C.byref(a), C.byref(shared(n_groups=0)), C.byref(n)) == 0 and n.value == 0


def test_binding_refuses_what_the_library_would_misread():
    x, s = torch.zeros(2, 3, 16, 128, dtype=torch.uint8).view(E4M3), torch.zeros(2, 3, 16, dtype=torch.uint8)
    cache = rkv.QuantizedCache(x, x.clone(), s, s.clone())
    assert (cache.n_pages, cache.n_kv_heads, cache.page_size, cache.dtype) == (2, 3, 16, torch.bfloat16)
    for bad in ((x[0], x[0], s, s), (x, x[:1], s, s), (x.view(torch.uint8), x.view(torch.uint8), s, s), (x, x, s[:1], s), (x, x, s, s.int()),
                (x.transpose(2, 3), x.transpose(2, 3), s, s), (x, x, s.unsqueeze(-1), s)):
        with pytest.raises(ValueError):
            rkv.QuantizedCache(*bad)
    with pytest.raises(ValueError):
        rkv.QuantizedCache(x, x, s, s, dtype=torch.float32)
    k, one = torch.zeros(1, 3, 128, dtype=torch.bfloat16), torch.ones(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        rkv.pages_write(cache, k, k, one)
    with pytest.raises(ValueError, match="on the GPU"):
        rkv.pages_read(cache, one)
    with pytest.raises(ValueError, match="on the GPU"):
        rkv.pages_attend(cache, k, one.view(1, 1), one)
    with pytest.raises(ValueError, match="on the GPU"):
        rkv.pages_attend_shared(cache, k, one.view(1, 1), one, torch.zeros(2, dtype=torch.int32), one.view(1, 1), one)


def test_packed_structs_are_the_c_ones():
    for cls, kinds in ((_abi.QPages, _abi._QPAGES[1]), (_abi.Shared, _abi._SHARED[1])):
        values = [i + 1 for i in range(len(kinds))]
        got = cls.from_buffer_copy(cls.pack(*values))
        assert [getattr(got, name) for name, _ in cls._fields_] == values
        with pytest.raises(ValueError):
            cls.pack(*([1 << 70] * len(kinds)))


@pytest.mark.parametrize("which", ["q", "k", "v", "slopes", "out", "k_out"])
def test_calls_that_would_drop_gradients_are_refused(which):
    def make(name, *shape):
        return torch.zeros(shape, dtype=torch.float32 if name == "slopes" else torch.bfloat16, requires_grad=which == name)
    x, s = torch.zeros(2, 3, 16, 128, dtype=torch.uint8).view(E4M3), torch.zeros(2, 3, 16, dtype=torch.uint8)
    cache, one = rkv.QuantizedCache(x, x.clone(), s, s), torch.ones(1, dtype=torch.int32)
    if which in ("k", "v"):
        calls = [lambda: rkv.pages_write(cache, make("k", 1, 3, 128), make("v", 1, 3, 128), one)]
    elif which == "k_out":
        calls = [lambda: rkv.pages_read(cache, one, k_out=make("k_out", 1, 3, 128))]
    else:
        kw = dict(slopes=make("slopes", 3), out=make("out", 1, 3, 128))
        calls = [lambda: rkv.pages_attend(cache, make("q", 1, 3, 128), one.view(1, 1), one, **kw),
                 lambda: rkv.pages_attend_shared(cache, make("q", 1, 3, 128), one.view(1, 1), one, one[:1].repeat(2), one.view(1, 1), one, **kw)]
    for call in calls:
        with pytest.raises(ValueError, match="no backward pass"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on the GPU"):
            call()
