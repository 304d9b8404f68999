"""Paged caches without a GPU: the oracle against hand cases, and every refusal of the C entry points (each before any HIP
call, with pointers that are never followed)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2606_15157_amd as rkv
from paper_2606_15157_amd import _abi
from oracle import pages as OG

P = 1 << 20          # a 16-byte aligned address that no refused call follows


def test_oracle_resize_by_hand():
    table = [[-1] * 3 for _ in range(3)]
    got = OG.resize(table, [0, 0, 0], [0, 1, 2, 3, 4], [0, 5], [5, 0, 4], 4, 12)
    assert got["table"] == [[0, 1, -1], [-1] * 3, [2, -1, -1]]
    assert got["slots"] == [0, 1, 2, 3, 4, 8, 9, 10, 11, -1, -1, -1] and got["cu_new"] == [0, 5, 5, 9] and got["cursor"] == [3, 2]
    got = OG.resize(got["table"], got["lens"], got["ring"], got["cursor"], [0, 9, 4], 4, 9)      # three pages, two free
    assert got["status"] == 1 and got["lens"] == [5, 0, 4]
    got = OG.resize(got["table"], got["lens"], got["ring"], got["cursor"], [0, 8, 5], 4, 9)      # the given ones come later
    assert got["status"] == 1
    got = OG.resize(got["table"], got["lens"], got["ring"], got["cursor"], [0, 8, 4], 4, 9)
    assert got["status"] == 0 and got["cursor"] == [0, 2] and got["ring"][:2] == [0, 1] and got["table"][1][:2] == [3, 4]


def test_oracle_attention_by_hand():
    """Equal keys: the mean of the visible values; one visible key: its value."""
    rng = np.random.default_rng(0)
    k, v = np.ones((3, 1, 2, 128)), rng.standard_normal((3, 1, 2, 128))
    q = rng.standard_normal((3, 2, 128))
    out, lse, _, _ = OG.attend(k, v, q, [[2, 0, 1]], [5], [0, 3])
    seq = np.concatenate([v[2, 0], v[0, 0], v[1, 0]])
    for i in range(3):
        np.testing.assert_allclose(out[i, 1], seq[:3 + i].mean(0), atol=1e-12)
    out, _, _, _ = OG.attend(k, v, q, [[2, 0, 1]], [5], [0, 3], window=1)
    np.testing.assert_allclose(out[1, 0], seq[3], atol=1e-12)
    out, lse, _, _ = OG.attend(k, v, q, [[2, 0, 1]], [1], [0, 3])
    assert np.isneginf(lse[:2]).all() and (out[:2] == 0).all() and np.allclose(out[2, 0], seq[0])


def pages(**kw):
    f = dict(k=P, v=P, k_page=2048, k_head=128, k_slot=128, v_page=2048, v_head=128, v_slot=128, n_pages=4, page_size=16,
             n_kv_heads=2, head_dim=128, dtype=0)
    f.update(kw)
    return _abi.Pages(**f)


def refused(status, call, *words):
    assert call == status
    message = _abi.lib().rkv_last_error().decode()
    assert message
    for w in words:
        assert w in message, message


BAD_PAGES = [
    (1, dict(k=None)), (1, dict(v=None)), (1, dict(n_pages=0)), (1, dict(page_size=0)), (1, dict(n_kv_heads=0)), (1, dict(dtype=2)),
    (1, dict(dtype=-1)), (1, dict(k_slot=-8)), (4, dict(head_dim=64)), (4, dict(k=P + 8)), (4, dict(v=P + 2)), (4, dict(k_head=132)),
    (4, dict(v_page=4)), (4, dict(k_slot=1 << 27)), (4, dict(v_slot=1 << 40)), (4, dict(n_pages=1 << 20, page_size=1 << 11))]


def rows(**kw):
    f = dict(k=P, v=P, k_outer=0, k_token=256, k_head=128, v_outer=0, v_token=256, v_head=128, slots=P, n_outer=1, n_tokens=3)
    f.update(kw)
    return _abi.Rows(**f)


@pytest.mark.parametrize("status,bad", BAD_PAGES)
def test_bad_pools_are_refused(status, bad):
    L = _abi.lib()
    refused(status, L.rkv_pages_write(C.byref(pages(**bad)), C.byref(rows()), None))
    refused(status, L.rkv_pages_attend(C.byref(pages(**bad)), C.byref(attend()), None, 0, None))
    n = C.c_size_t()
    refused(status, L.rkv_pages_attend_workspace_size(C.byref(pages(**bad)), C.byref(attend()), C.byref(n)))


@pytest.mark.parametrize("status,bad", [
    (1, dict(k=None)), (1, dict(v=None)), (1, dict(slots=None)), (1, dict(n_tokens=-1)), (1, dict(n_outer=-1)), (1, dict(v_token=-128)),
    (4, dict(k=P + 4)), (4, dict(k_token=130)), (4, dict(v_outer=9)), (4, dict(n_outer=1 << 15, n_tokens=1 << 15))])
def test_bad_rows_are_refused(status, bad):
    refused(status, _abi.lib().rkv_pages_write(C.byref(pages()), C.byref(rows(**bad)), None))


@pytest.mark.parametrize("bad", [dict(k_slot=0), dict(v_slot=64), dict(k_head=0), dict(v_page=120)])
def test_overlapping_pools_are_not_written(bad):
    refused(1, _abi.lib().rkv_pages_write(C.byref(pages(**bad)), C.byref(rows()), None), "overlap")


def test_no_rows_need_no_gpu():
    L = _abi.lib()
    assert L.rkv_pages_write(C.byref(pages()), C.byref(rows(n_tokens=0, k=None, v=None, slots=None)), None) == 0
    assert L.rkv_pages_attend(C.byref(pages()), C.byref(attend(n_rows=0)), None, 0, None) == 0
    assert L.rkv_pages_attend(C.byref(pages()), C.byref(attend(n_seqs=0, n_rows=5)), None, 0, None) == 0


def attend(**kw):
    f = dict(q=P, out=P, lse=None, q_token=512, q_head=128, out_token=512, out_head=128, table=P, table_stride=4, lens=P, cu_q=P,
             prefix_lens=None, first_keys=None, slopes=None, n_seqs=2, n_rows=6, n_q_heads=4, max_pages=4, max_q=0, max_kv=0, causal=1,
             window=0, scale=0.1, softcap=0.0)
    f.update(kw)
    return _abi.Attend(**f)


@pytest.mark.parametrize("status,bad", [
    (1, dict(q=None)), (1, dict(out=None)), (1, dict(lens=None)), (1, dict(table=None)), (1, dict(n_seqs=-1)), (1, dict(n_rows=-1)),
    (1, dict(max_pages=-1)), (1, dict(max_q=-1)), (1, dict(max_kv=-2)), (1, dict(window=-1)), (1, dict(causal=2)),
    (1, dict(scale=float("nan"))), (1, dict(scale=float("inf"))), (1, dict(softcap=-1.0)), (1, dict(softcap=float("inf"))), (1, dict(softcap=1e-35)), (4, dict(softcap=600.0)),
    (1, dict(q_token=-8)), (1, dict(out_token=0)), (1, dict(out_head=64)), (2, dict(n_q_heads=3)), (2, dict(n_q_heads=0)), (2, dict(cu_q=None)), (2, dict(table_stride=3)),
    (4, dict(q=P + 8)), (4, dict(out=P + 4)), (4, dict(q_head=130)), (4, dict(out_token=513)),
    (4, dict(max_pages=1 << 27, table_stride=1 << 27)), (4, dict(n_rows=1 << 29))])
def test_bad_attention_calls_are_refused(status, bad):
    refused(status, _abi.lib().rkv_pages_attend(C.byref(pages()), C.byref(attend(**bad)), None, 0, None))


def resize(**kw):
    f = dict(lens=P, new_lens=P, lens_out=P, table=P, table_stride=4, ring=P, cursor=P, cursor_out=P, slots=P, cu_new=P, status=P,
             n_seqs=3, max_pages=4, n_pages=8, page_size=16, max_new=5)
    f.update(kw)
    return _abi.Resize(**f)


@pytest.mark.parametrize("status,bad", [(1, {name: None}) for name in
                                        "lens new_lens lens_out table ring cursor cursor_out slots cu_new status".split()] + [
    (1, dict(n_seqs=-1)), (1, dict(max_pages=-1)), (1, dict(max_new=-1)), (1, dict(n_pages=0)), (1, dict(page_size=0)),
    (1, dict(table_stride=-4)), (2, dict(table_stride=3)), (4, dict(n_seqs=8193)), (4, dict(n_pages=1 << 28)),
    (4, dict(max_pages=1 << 27, table_stride=1 << 27))])
def test_bad_resizes_are_refused(status, bad):
    refused(status, _abi.lib().rkv_pages_resize(C.byref(resize(**bad)), None))


def test_null_structs_are_refused():
    L, n = _abi.lib(), C.c_size_t()
    refused(1, L.rkv_pages_resize(None, None))
    refused(1, L.rkv_pages_write(None, C.byref(rows()), None))
    refused(1, L.rkv_pages_write(C.byref(pages()), None, None))
    refused(1, L.rkv_pages_attend(None, C.byref(attend()), None, 0, None))
    refused(1, L.rkv_pages_attend(C.byref(pages()), None, None, 0, None))
    refused(1, L.rkv_pages_attend_workspace_size(C.byref(pages()), C.byref(attend()), None))
    assert L.rkv_pages_attend_workspace_size(C.byref(pages()), C.byref(attend(q=None, out=None, lens=None)), C.byref(n)) == 0


def test_binding_refuses_what_the_library_would_misread():
    pool = torch.zeros(2, 3, 16, 128, dtype=torch.bfloat16)
    cache = rkv.PagedCache(pool, pool.clone())
    assert (cache.n_pages, cache.n_kv_heads, cache.page_size) == (2, 3, 16)
    for k, v in ((pool[0], pool[0]), (pool, pool[:1]), (pool, pool.half()), (pool.float(), pool.float()),
                 (pool.transpose(2, 3), pool.transpose(2, 3))):
        with pytest.raises(ValueError):
            rkv.PagedCache(k, v)
    with pytest.raises(ValueError):      # no fallback for tensors that are not on the GPU
        rkv.pages_write(cache, torch.zeros(1, 3, 128, dtype=torch.bfloat16), torch.zeros(1, 3, 128, dtype=torch.bfloat16),
                        torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        rkv.pages_attend(cache, torch.zeros(1, 3, 128, dtype=torch.bfloat16), torch.zeros(1, 1, dtype=torch.int32),
                         torch.ones(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        rkv.pages_resize(rkv.pages_init(1, 2, 4, 16, device="cpu"), torch.ones(1, dtype=torch.int32), 4)


def test_workspace_is_checked():
    L, n = _abi.lib(), C.c_size_t()
    assert L.rkv_pages_attend_workspace_size(C.byref(pages()), C.byref(attend(max_pages=100, table_stride=100)), C.byref(n)) == 0
    assert n.value > 0
    refused(5, L.rkv_pages_attend(C.byref(pages()), C.byref(attend(max_pages=100, table_stride=100)), None, n.value, None))
    refused(5, L.rkv_pages_attend(C.byref(pages()), C.byref(attend(max_pages=100, table_stride=100)), C.c_void_p(P + 16), n.value, None))
    refused(5, L.rkv_pages_attend(C.byref(pages()), C.byref(attend(max_pages=100, table_stride=100)), C.c_void_p(P), n.value - 1, None))
    assert L.rkv_pages_attend_workspace_size(C.byref(pages()), C.byref(attend(n_rows=0, max_pages=100, table_stride=100)), C.byref(n)) == 0 and n.value == 0
    refused(4, L.rkv_pages_attend(C.byref(pages()), C.byref(attend(n_seqs=1 << 30)), None, 0, None))
    # short sequences are not split: nothing to keep
    assert L.rkv_pages_attend_workspace_size(C.byref(pages()), C.byref(attend()), C.byref(n)) == 0 and n.value == 0


def test_packed_structs_are_the_c_ones():
    for cls, kinds in ((_abi.Pages, _abi._PAGES[1]), (_abi.Resize, _abi._RESIZE[1]), (_abi.Rows, _abi._ROWS[1]), (_abi.Attend, _abi._ATTEND[1])):
        values = [float(i) if k == "f" else i + 1 for i, k in enumerate(kinds)]
        got = cls.from_buffer_copy(cls.pack(*values))
        assert [getattr(got, name) for name, _ in cls._fields_] == values
        with pytest.raises(ValueError):
            cls.pack(*([1 << 70] * len(kinds)))


@pytest.mark.parametrize("group,rows,cu_q", [(1, 1, None), (1, 1, P), (3, 1, None), (3, 3, P), (5, 5, P), (1, 129, P), (2, 4, P)])
def test_partial_sums_are_16_byte_aligned(group, rows, cu_q):
    """512 records of 16 bytes, then 1024 partial sums of one size, which are written and read 16 bytes at a time."""
    L, n = _abi.lib(), C.c_size_t()
    seqs = 1 if cu_q else rows
    a = attend(n_seqs=seqs, n_rows=rows, n_q_heads=2 * group, cu_q=cu_q, out_token=256 * group, max_pages=400, table_stride=400)
    assert L.rkv_pages_attend_workspace_size(C.byref(pages()), C.byref(a), C.byref(n)) == 0
    parts = n.value - 512 * 16
    assert parts >= 1024 * min(128, (rows if cu_q else 1) * group) * 130 * 4 and parts % (1024 * 16) == 0


@pytest.mark.parametrize("bad", [
    dict(k_page=128, k_head=128, k_slot=128), dict(v_page=128, v_head=128, v_slot=128), dict(k_slot=128, k_head=128), dict(v_head=1920, v_slot=128),
    dict(k_page=128, k_head=384, k_slot=1024), dict(k_page=1920, n_kv_heads=1), dict(v_page=4080, v_head=2048), dict(k_slot=120, n_pages=1, n_kv_heads=1)])
def test_pools_whose_dimensions_run_into_each_other_are_not_written(bad):
    refused(1, _abi.lib().rkv_pages_write(C.byref(pages(**{**NESTED, **bad})), C.byref(rows()), None), "overlap")


NESTED = dict(k_page=4096, k_head=2048, k_slot=128, v_page=4096, v_head=2048, v_slot=128)


@pytest.mark.parametrize("bad", [dict(out_token=128, out_head=128), dict(out_token=384, out_head=128), dict(out_token=128, out_head=640),
                                 dict(out_token=504), dict(out_token=1 << 62, out_head=120)])
def test_out_rows_that_run_into_each_other_are_refused(bad):
    n = C.c_size_t()
    refused(1, _abi.lib().rkv_pages_attend_workspace_size(C.byref(pages()), C.byref(attend(**bad)), C.byref(n)), "overlap")
    refused(1, _abi.lib().rkv_pages_attend(C.byref(pages()), C.byref(attend(**bad)), None, 0, None), "overlap")


@pytest.mark.parametrize("good", [dict(out_token=128, out_head=768), dict(out_token=512, out_head=128), dict(out_token=1 << 62, out_head=1 << 58),
                                  dict(out_token=0, n_rows=1), dict(out_head=0, n_q_heads=1, out_token=128)])
def test_out_rows_of_either_order_are_taken(good):
    n = C.c_size_t()
    pool = pages(n_kv_heads=1) if "n_q_heads" in good else pages()
    a = attend(**good)
    assert _abi.lib().rkv_pages_attend_workspace_size(C.byref(pool), C.byref(a), C.byref(n)) == 0


@pytest.mark.parametrize("bad", [dict(n_tokens=1 << 27), dict(n_tokens=(1 << 27) - 7), dict(n_outer=1 << 13, n_tokens=1 << 14), dict(n_outer=1 << 15, n_tokens=1 << 13)])
def test_more_rows_than_a_launch_takes_are_refused(bad):
    """16 rows a workgroup of 256 threads, fewer than 2^32 threads; two heads a row here."""
    refused(4, _abi.lib().rkv_pages_write(C.byref(pages(**NESTED)), C.byref(rows(**bad)), None), "rows")


@pytest.mark.parametrize("status,kw", [
    (0, dict(n_seqs=(1 << 23) - 1)), (4, dict(n_seqs=1 << 23)), (4, dict(n_seqs=1 << 24)), (4, dict(n_seqs=1 << 23, n_rows=1 << 23, cu_q=None)),
    (0, dict(n_seqs=1, n_rows=(1 << 28) - 1)), (4, dict(n_seqs=1 << 22, n_rows=(1 << 28) - 1)), (0, dict(n_seqs=0, n_rows=(1 << 28) - 1))])
def test_more_row_tiles_than_a_launch_takes_are_refused(status, kw):
    """A workgroup of 256 threads per place and KV head, two of which are here."""
    L, n = _abi.lib(), C.c_size_t()
    got = L.rkv_pages_attend_workspace_size(C.byref(pages()), C.byref(attend(**kw)), C.byref(n))
    assert got == status
    if status:
        refused(status, L.rkv_pages_attend(C.byref(pages()), C.byref(attend(**kw)), None, 0, None), "sequences")


@pytest.mark.parametrize("seqs,split", [(1, True), (100, True), (252, True), (256, False), (512, False), (1000, False)])
def test_lists_whose_key_tiles_32_bits_may_not_hold_are_not_split(seqs, split):
    """Tables of 2^29 slots a sequence, 2^23 key tiles: up to 255 row tiles (three here are the long sequences' room)."""
    a = attend(n_seqs=seqs, n_rows=192, max_pages=1 << 16, table_stride=1 << 16)
    n = C.c_size_t()
    assert _abi.lib().rkv_pages_attend_workspace_size(C.byref(pages(page_size=1 << 13)), C.byref(a), C.byref(n)) == 0
    assert (n.value > 0) == split


@pytest.mark.parametrize("which", ["q", "k", "v", "pool", "slopes", "out"])
def test_calls_that_would_drop_gradients_are_refused(which):
    """Before anything else is looked at; with gradients off the call goes on (here to the refusal of tensors off the GPU)."""
    def make(name, *shape):
        return torch.zeros(shape, dtype=torch.float32 if name == "slopes" else torch.bfloat16, requires_grad=which == name)
    cache = rkv.PagedCache(make("pool", 2, 3, 16, 128), torch.zeros(2, 3, 16, 128, dtype=torch.bfloat16))
    one = torch.ones(1, dtype=torch.int32)
    calls = []
    if which in ("k", "v", "pool"):
        calls.append(lambda: rkv.pages_write(cache, make("k", 1, 3, 128), make("v", 1, 3, 128), one))
    if which not in ("k", "v"):
        calls.append(lambda: rkv.pages_attend(cache, make("q", 1, 3, 128), one.view(1, 1), one, slopes=make("slopes", 3), out=make("out", 1, 3, 128)))
    for call in calls:
        with pytest.raises(ValueError, match="no backward pass"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on the GPU"):
            call()


@pytest.mark.parametrize("kw", [dict(extra=-1), dict(extra=-16), dict(page_size=0), dict(page_size=-16)])
def test_a_hand_over_without_room_is_refused(kw):
    """Fewer pages than the retained rows need would leave every layer's cache empty."""
    x = [torch.zeros(1, 2, 20, 128, dtype=torch.bfloat16)]
    with pytest.raises(ValueError, match="extra"):
        rkv.pages_init_from_prefill(None, {"k_out": x, "v_out": x}, **kw)
