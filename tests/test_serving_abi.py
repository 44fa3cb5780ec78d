"""The calls around the indexer without a GPU: what they refuse, before anything is launched.  (Pointers are fake
non-null values: a call that got past its checks here would fail the test by its status.)"""
import copy
import ctypes as C

import pytest
import torch

from paper_2603_28458_amd import hisa
from tests.test_abi import lib  # noqa: F401  (the fixture)

F = 0x1000
BF16, FP8, F32 = hisa.HISA_BF16, hisa.HISA_FP8_E4M3, hisa.HISA_F32
OK, NULL, SHAPE, DTYPE, WS, ALIGN = 0, 1, 2, 3, 5, 6


def cache(**kw):
    a = dict(k=F, v=F, k_scale=F, v_scale=F, block_table=F, seq_len=F, page_stride=64 * 2 * 128, token_stride=2 * 128,
             head_stride=128, n_pages=100, page=64, n_seq=4, max_pages=16, H_kv=2, d=128, dtype=BF16)
    a.update(kw)
    return hisa._Cache(**a)


def queries(**kw):
    a = dict(q=F, w=None, q_seq=None, q_pos=None, q_lo=None, T=4, H=8, q_pos0=0, q_dtype=BF16)
    a.update(kw)
    return hisa._Queries(**a)


BAD_CACHES = [
    (dict(k=None), NULL), (dict(dtype=FP8, k_scale=None), NULL), (dict(dtype=FP8, v_scale=None), NULL),
    (dict(dtype=3), DTYPE), (dict(dtype=-1), DTYPE), (dict(n_pages=0), SHAPE), (dict(page=0), SHAPE),
    (dict(H_kv=0), SHAPE), (dict(H_kv=257), SHAPE), (dict(d=0), SHAPE), (dict(n_pages=1 << 26), SHAPE),
    (dict(page_stride=-128), SHAPE), (dict(token_stride=-128), SHAPE), (dict(head_stride=-128), SHAPE),
    (dict(k=F + 8), ALIGN), (dict(v=F + 8), ALIGN), (dict(page_stride=4), ALIGN), (dict(token_stride=260), ALIGN),
    (dict(head_stride=132), ALIGN),
]


def paged(lib, q, c, start=F, scale=0.1, out=F, ws=F, n=1 << 40):
    return lib.hisa_paged_attention(C.byref(q) if q else None, C.byref(c) if c else None, start, scale, out, None, ws, n, None)


def sparse(lib, q, c, k=64, lists=F, scale=0.1, out=F, ws=F, n=1 << 40):
    return lib.hisa_sparse_attention(C.byref(q) if q else None, C.byref(c) if c else None, lists, k, scale, out, None, ws, n,
                                     None)


@pytest.mark.parametrize("kw,status", BAD_CACHES + [
    (dict(v=None), NULL), (dict(block_table=None), NULL), (dict(seq_len=None), NULL), (dict(n_seq=0), SHAPE),
    (dict(n_seq=65536), SHAPE), (dict(max_pages=0), SHAPE), (dict(page=48), SHAPE), (dict(H_kv=3), SHAPE),
    (dict(max_pages=1 << 25), SHAPE), (dict(d=96), SHAPE), (dict(d=256), SHAPE), (dict(dtype=F32), DTYPE),
    (dict(dtype=FP8, head_stride=136), ALIGN)])
def test_attention_refuses_caches(lib, kw, status):  # noqa: F811
    assert paged(lib, queries(), cache(**kw)) == status
    assert sparse(lib, queries(), cache(**kw)) == status
    q, c = queries(), cache(**kw)
    assert lib.hisa_attention_workspace_bytes(C.byref(q), C.byref(c), 0) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), NULL), (dict(T=0), SHAPE), (dict(T=(1 << 22) + 1), SHAPE), (dict(H=0), SHAPE), (dict(H=258), SHAPE),
    (dict(H=7), SHAPE), (dict(q=F + 2), ALIGN), (dict(q_dtype=F32), DTYPE), (dict(q_dtype=FP8), DTYPE)])
def test_attention_refuses_queries(lib, kw, status):  # noqa: F811
    assert paged(lib, queries(**kw), cache()) == status
    assert sparse(lib, queries(**kw), cache()) == status


def test_attention_refuses_the_rest(lib):  # noqa: F811
    q, c = queries(), cache()
    assert paged(lib, None, c) == NULL and paged(lib, q, None) == NULL
    assert paged(lib, q, c, start=None) == NULL and paged(lib, q, c, out=None) == NULL
    assert sparse(lib, q, c, lists=None) == NULL and sparse(lib, q, c, out=None) == NULL
    assert paged(lib, q, c, out=F + 4) == ALIGN
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert paged(lib, q, c, scale=scale) == SHAPE and sparse(lib, q, c, scale=scale) == SHAPE
    for k in (0, -1, 65537):
        assert sparse(lib, q, c, k=k) == SHAPE
    # a long cache and few queries: split, through a workspace
    c = cache(max_pages=2048)
    need = lib.hisa_attention_workspace_bytes(C.byref(q), C.byref(c), 0)
    assert need > 0
    assert paged(lib, q, c, ws=None, n=0) == WS and paged(lib, q, c, n=need - 1) == WS
    assert paged(lib, q, c, ws=F + 4, n=need) == ALIGN
    need = lib.hisa_attention_workspace_bytes(C.byref(q), C.byref(c), 8192)
    assert need > 0 and sparse(lib, q, c, k=8192, n=need - 1) == WS
    # fp32: its own head sizes
    for d, status in ((6, SHAPE), (260, SHAPE)):
        assert paged(lib, queries(q_dtype=F32), cache(dtype=F32, d=d)) == status


def test_launches_beyond_32_bits_of_threads_are_refused(lib):  # noqa: F811
    many = queries(T=1 << 22, H=64)
    assert sparse(lib, many, cache(H_kv=8, head_stride=128, token_stride=1024), k=1) == SHAPE
    assert paged(lib, queries(T=131070, H=256), cache(H_kv=256, n_seq=65535, token_stride=256 * 128, max_pages=1)) == SHAPE
    assert append(lib, cache(H_kv=64, d=512, token_stride=64 * 512, head_stride=512), stride=64 * 512, T=1 << 22) == SHAPE


def append(lib, c, slots=F, k=F, v=F, dt=BF16, stride=256, T=4):
    return lib.hisa_cache_append(C.byref(c) if c else None, slots, k, v, dt, stride, T, None)


@pytest.mark.parametrize("kw,status", BAD_CACHES + [(dict(d=12), SHAPE), (dict(d=520), SHAPE), (dict(dtype=F32), DTYPE)])
def test_append_refuses_caches(lib, kw, status):  # noqa: F811
    assert append(lib, cache(**kw)) == status


def test_append_refuses_the_rest(lib):  # noqa: F811
    c = cache()
    assert append(lib, None) == NULL and append(lib, c, slots=None) == NULL and append(lib, c, k=None) == NULL
    assert append(lib, c, v=None) == NULL and append(lib, cache(v=None)) == NULL      # values on one side only
    assert append(lib, c, dt=FP8) == DTYPE and append(lib, c, dt=7) == DTYPE
    assert append(lib, c, T=-1) == SHAPE and append(lib, c, T=(1 << 22) + 1) == SHAPE
    assert append(lib, c, stride=248) == SHAPE and append(lib, c, stride=1 << 31) == SHAPE
    assert append(lib, c, stride=260) == ALIGN and append(lib, c, k=F + 8) == ALIGN and append(lib, c, v=F + 8) == ALIGN
    assert append(lib, c, T=0) == OK                                                  # nothing to do, no launch


def tables(lib, **kw):
    a = dict(ctx=F, new=F, n_seq=4, table=F, max_pages=16, page=64, free=F, n_free=9, rows=32, s_max=0, seq_len=F,
             q_start=F, page_start=F, q_seq=F, q_pos=F, slots=F, key_rows=None)
    a.update(kw)
    return lib.hisa_page_tables(a["ctx"], a["new"], a["n_seq"], a["table"], a["max_pages"], a["page"], a["free"],
                                a["n_free"], a["rows"], a["s_max"], a["seq_len"], a["q_start"], a["page_start"],
                                a["q_seq"], a["q_pos"], a["slots"], a["key_rows"], None)


@pytest.mark.parametrize("kw,status", [
    *[({n: None}, NULL) for n in ("ctx", "new", "table", "free", "seq_len", "q_start", "page_start", "q_seq", "q_pos", "slots")],
    (dict(n_seq=0), SHAPE), (dict(n_seq=65536), SHAPE), (dict(max_pages=0), SHAPE), (dict(page=0), SHAPE),
    (dict(n_free=-1), SHAPE), (dict(rows=0), SHAPE), (dict(rows=(1 << 22) + 1), SHAPE), (dict(max_pages=1 << 30), SHAPE),
    (dict(page=1 << 28), SHAPE), (dict(key_rows=F), SHAPE), (dict(key_rows=F, s_max=1 << 30), SHAPE),
    (dict(ctx=F + 64, new=F + 128, seq_len=F + 64), SHAPE), (dict(ctx=F + 64, new=F + 128, seq_len=F + 128), SHAPE)])
def test_tables_refuse(lib, kw, status):  # noqa: F811
    assert tables(lib, **kw) == status


# ---- the binding: tensors that no kernel may be given
def test_the_binding_refuses_tensors_that_are_not_on_the_gpu(lib):  # noqa: F811
    k = torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="not on the GPU"):
        hisa.Cache(k=k, v=k, dtype=BF16)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="not on the GPU"):
        hisa.hisa_page_tables(i, i, torch.zeros((3, 2), dtype=torch.int32), 4, i, 3)


class OnGpu:
    """Tensors of the CPU that say they are on the GPU, for the checks behind that one."""

    def __init__(self, monkeypatch):
        monkeypatch.setattr(hisa, "_on_gpu", lambda t: True)


def test_the_binding_refuses_types_shapes_and_strides(lib, monkeypatch):  # noqa: F811
    OnGpu(monkeypatch)
    bf, i32 = torch.bfloat16, torch.int32
    k = torch.zeros((2, 4, 2, 64), dtype=bf)
    i3 = torch.zeros(3, dtype=i32)
    table = torch.zeros((3, 2), dtype=i32)
    with pytest.raises(ValueError, match="k: torch.float32"):
        hisa.Cache(k=k.float(), v=k, dtype=BF16)
    with pytest.raises(ValueError, match="v: shape"):
        hisa.Cache(k=k, v=k[:1], dtype=BF16)
    with pytest.raises(ValueError, match="strides"):
        hisa.Cache(k=k, v=torch.zeros((2, 2, 4, 64), dtype=bf).permute(0, 2, 1, 3), dtype=BF16)
    with pytest.raises(ValueError, match="last dimension"):
        hisa.Cache(k=torch.zeros((2, 4, 64, 2), dtype=bf).permute(0, 1, 3, 2), v=None, dtype=BF16)
    with pytest.raises(ValueError, match=r"needed is \[n_pages"):
        hisa.Cache(k=k[0], v=None, dtype=BF16)
    with pytest.raises(ValueError, match="dtype"):
        hisa.Cache(k=k, v=k, dtype=9)
    with pytest.raises(ValueError, match="k_scale"):
        hisa.Cache(k=k.view(torch.uint8), v=None, dtype=FP8, k_scale=torch.zeros((2, 4, 1)))
    with pytest.raises(ValueError, match="seq_len"):
        hisa.Cache(k=k, v=k, dtype=BF16, block_table=table, seq_len=torch.zeros(4, dtype=i32))
    c = hisa.Cache(k=k, v=k, dtype=BF16, block_table=table, seq_len=i3)
    q = hisa.Queries(q=torch.zeros((5, 4, 64), dtype=bf), w=None, dtype=BF16)
    start = torch.zeros(4, dtype=i32)
    with pytest.raises(ValueError, match="q_start"):
        hisa.hisa_paged_attention(q, c, i3)
    with pytest.raises(ValueError, match="q_start"):
        hisa.hisa_paged_attention(q, c, start.long())
    with pytest.raises(ValueError, match="out"):
        hisa.hisa_paged_attention(q, c, start, out=torch.zeros((5, 4, 64)))
    with pytest.raises(ValueError, match="lse"):
        hisa.hisa_paged_attention(q, c, start, lse=torch.zeros((5, 3)))
    with pytest.raises(ValueError, match="q_lo"):
        hisa.hisa_paged_attention(hisa.Queries(q=q.q, w=None, dtype=BF16, q_lo=i3), c, start)
    with pytest.raises(ValueError, match="q: shape"):
        hisa.hisa_paged_attention(hisa.Queries(q=q.q[:, :, :32].contiguous(), w=None, dtype=BF16), c, start)
    with pytest.raises(ValueError, match="ws"):
        hisa.hisa_paged_attention(q, c, start, ws=torch.zeros(64))
    with pytest.raises(ValueError, match="topk_idx"):
        hisa.hisa_sparse_attention(q, c, torch.zeros((4, 8), dtype=i32))
    with pytest.raises(ValueError, match="topk_idx"):
        hisa.hisa_sparse_attention(q, c, torch.zeros((5, 0), dtype=i32))
    with pytest.raises(ValueError, match="block_table"):
        hisa.hisa_paged_attention(q, hisa.Cache(k=k, v=k, dtype=BF16), start)
    with pytest.raises(ValueError, match="k_new"):
        hisa.hisa_cache_append(c, i3, torch.zeros((3, 2, 32), dtype=bf), torch.zeros((3, 2, 32), dtype=bf))
    with pytest.raises(ValueError, match="contiguous"):
        hisa.hisa_cache_append(c, i3, torch.zeros((3, 64, 2), dtype=bf).transpose(1, 2), torch.zeros((3, 2, 64), dtype=bf))
    with pytest.raises(ValueError, match="v_new"):
        hisa.hisa_cache_append(c, i3, torch.zeros((3, 2, 64), dtype=bf), torch.zeros((3, 2, 64)))
    with pytest.raises(ValueError, match="elements apart"):
        hisa.hisa_cache_append(c, i3, torch.zeros((3, 2, 64), dtype=bf), torch.zeros((3, 3, 64), dtype=bf)[:, :2])
    with pytest.raises(ValueError, match="new_len"):
        hisa.hisa_page_tables(i3, torch.zeros(2, dtype=i32), table, 4, i3, 3)
    with pytest.raises(ValueError, match="block_table"):
        hisa.hisa_page_tables(i3, i3, table[:2], 4, i3, 3)
    with pytest.raises(ValueError, match="slots"):
        hisa.hisa_page_tables(i3, i3, table, 4, i3, 3, out=hisa.PageTables(i3, start, start, i3, i3, start))


def test_another_gpu_than_the_current_one_is_made_current_for_the_call(monkeypatch):
    seen = []

    class Guard:
        def __init__(self, index):
            seen.append(index)

        def __enter__(self):
            seen.append("in")

        def __exit__(self, *exc):
            seen.append("out")

    monkeypatch.setattr(hisa.torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(hisa.torch.cuda, "device", Guard)
    monkeypatch.setattr(hisa, "_stream", lambda stream: seen.append("stream") or 5)
    assert hisa._call(lambda *a: a, 1, None, 7, 8) == (7, 8, 5)
    assert seen == [1, "in", "stream", "out"]
    del seen[:]
    assert hisa._call(lambda *a: a, 0, None, 7) == (7, 5)
    assert seen == ["stream"]


def test_a_cache_is_checked_again_after_a_change(monkeypatch):
    monkeypatch.setattr(hisa, "_on_gpu", lambda t: True)
    k = torch.zeros((4, 16, 2, 128), dtype=torch.bfloat16)
    cache = hisa.Cache(k=k, v=k.clone(), dtype=hisa.HISA_BF16, block_table=torch.zeros((3, 2), dtype=torch.int32),
                       seq_len=torch.zeros(3, dtype=torch.int32))
    c = cache.c()
    assert (c.n_pages, c.page, c.H_kv, c.d, c.n_seq, c.max_pages) == (4, 16, 2, 128, 3, 2)
    cache.block_table = torch.zeros((3, 5), dtype=torch.int32)
    assert cache.c().max_pages == 5 and cache.c().block_table == cache.block_table.data_ptr()
    cache.block_table = torch.zeros((2, 5), dtype=torch.int32)
    with pytest.raises(ValueError, match="seq_len"):
        cache.c()
    cache.seq_len = torch.zeros(2, dtype=torch.int32)
    assert cache.c().n_seq == 2
    other = copy.deepcopy(cache)
    assert other.c().k == other.k.data_ptr() != cache.c().k
    assert copy.copy(cache).c() is not cache.c()
    cache.k.resize_(8, 8, 2, 128)
    with pytest.raises(ValueError, match="v: shape"):
        cache.c()
    cache.v = cache.v.float()
    with pytest.raises(ValueError, match="v: "):
        cache.c()


# ---- the oracle against a few numbers worked out by hand
def test_the_oracle():
    import numpy as np
    from oracle import serving_oracle as SO
    t = SO.page_tables([3, 0, 4], [2, 3, 0], [[7, -1], [-1, -1], [5, 6]], 4, [9, 8, 1], 7, s_max=4)
    assert t["seq_len"].tolist() == [5, 3, 4] and t["q_start"].tolist() == [0, 2, 5, 5]
    assert t["page_start"].tolist() == [0, 1, 2, 2] and t["block_table"].tolist() == [[7, 9], [8, -1], [5, 6]]
    assert t["q_seq"].tolist() == [0, 0, 1, 1, 1, 0, 0] and t["q_pos"].tolist() == [3, 4, 0, 1, 2, -1, -1]
    assert t["slots"].tolist() == [31, 36, 32, 33, 34, -1, -1] and t["key_rows"].tolist() == [3, -1, 4, 5, 6, -1, -1]
    k = np.array([[[1.0, 0.0]], [[0.0, 2.0]], [[9.0, 9.0]], [[0.0, 0.0]]])
    v = np.array([[[1.0, 2.0]], [[3.0, -4.0]], [[9.0, 9.0]], [[5.0, 6.0]]])
    q = np.log(2.0) * np.array([[[1.0, 0.5]], [[0.0, 0.0]], [[1.0, 1.0]]])
    table = np.array([[3, 0, 1, -1]])
    out, lse, mag = SO.attention(q, k, v, table, [4], 1, lambda t: 0 if t < 2 else None,
                                 lambda t: [0, 1, 2, 3][:3 if t == 0 else 0], 1.0)
    # positions 0, 1, 2 are rows 3, 0, 1: weights 1, 2, 2
    assert np.allclose(out[0, 0], [(5 + 2 + 6) / 5, (6 + 4 - 8) / 5]) and np.isclose(lse[0, 0], np.log(5.0))
    assert np.allclose(mag[0, 0], [(5 + 2 + 6) / 5, (6 + 4 + 8) / 5])
    assert out[1, 0].tolist() == [0, 0] and np.isneginf(lse[1, 0]) and np.isnan(lse[2, 0])


# ---- what the attention rounds its weights to
@pytest.mark.parametrize("weights", [-1, 2, 7])
def test_unknown_weights_are_refused(lib, monkeypatch, weights):  # noqa: F811
    assert paged(lib, queries(), cache(weights=weights)) == DTYPE and sparse(lib, queries(), cache(weights=weights)) == DTYPE
    monkeypatch.setattr(hisa, "_on_gpu", lambda t: True)
    k = torch.zeros((2, 4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="weights"):
        hisa.Cache(k=k, v=k, dtype=BF16, weights=weights)
    c = hisa.Cache(k=k, v=k, dtype=BF16)
    assert c.c().weights == hisa.HISA_WEIGHTS_16BIT and C.sizeof(hisa._Cache) == 104
    c.weights = hisa.HISA_WEIGHTS_8BIT
    assert c.c().weights == hisa.HISA_WEIGHTS_8BIT
    c.weights = weights
    with pytest.raises(ValueError, match="weights"):
        c.c()


# ---- tensors that change in place behind a descriptor's back
@pytest.mark.parametrize("change,match", [
    (lambda c: c.v.resize_(4, 8, 2, 128), "v: shape"),
    (lambda c: c.v.as_strided_((4, 16, 2, 128), (4096, 128, 2048, 1)), "strides"),
    (lambda c: c.k.as_strided_((4, 16, 2, 128), (4096, 128, 2048, 1)), "strides"),
    (lambda c: c.k_scale.resize_(3, 16, 2), "k_scale: shape"),
    (lambda c: c.v_scale.resize_(4, 16, 1), "v_scale: shape"),
    (lambda c: c.k_scale.as_strided_((4, 16, 2), (32, 1, 16)), "k_scale: not contiguous"),
    (lambda c: c.seq_len.resize_(2), "seq_len: shape"),
    (lambda c: c.seq_len.as_strided_((3,), (0,)), "seq_len: not contiguous"),
    (lambda c: c.block_table.t_(), "block_table: not contiguous"),
    (lambda c: c.block_table.resize_(2, 3), "seq_len: shape")])
def test_a_change_in_place_of_any_tensor_is_seen(monkeypatch, change, match):
    monkeypatch.setattr(hisa, "_on_gpu", lambda t: True)
    k = torch.zeros((4, 16, 2, 128), dtype=torch.uint8)
    cache = hisa.Cache(k=k, v=k.clone(), dtype=FP8, block_table=torch.zeros((3, 3), dtype=torch.int32),
                       seq_len=torch.zeros(3, dtype=torch.int32), k_scale=torch.ones((4, 16, 2)),
                       v_scale=torch.ones((4, 16, 2)))
    c = cache.c()
    assert cache.c() is c and [c.k, c.v, c.k_scale, c.v_scale, c.block_table, c.seq_len] == [
        t.data_ptr() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.block_table, cache.seq_len)]
    change(cache)
    for _ in range(2):
        with pytest.raises(ValueError, match=match):
            cache.c()


def test_a_cache_of_keys_alone_and_its_copies(monkeypatch):
    monkeypatch.setattr(hisa, "_on_gpu", lambda t: True)
    cache = hisa.Cache(k=torch.zeros((4, 16, 2, 128)), v=None, dtype=F32)
    c = cache.c()
    assert c.k == cache.k.data_ptr() and [c.v, c.k_scale, c.v_scale, c.block_table, c.seq_len] == [None] * 5
    other = copy.copy(cache)
    cache.k = torch.zeros((4, 8, 2, 128))
    assert cache.c().page == 8 and other.c().page == 16 and other.c() is not cache.c()
    cache.v = torch.zeros((4, 8, 2, 128))
    assert cache.c().v == cache.v.data_ptr() and cache.c().seq_len is None


def test_tables_whose_layout_changes_in_place_are_refused(monkeypatch):
    monkeypatch.setattr(hisa, "_on_gpu", lambda t: True)
    t = hisa.PageTables.empty(3, 5, "cpu", key_rows=True)
    device = torch.device("cpu")
    assert t.pointers(3, 5, -1, device) == t.pointers(3, 5, -1, device)
    t.q_pos.as_strided_((5,), (0,))
    with pytest.raises(ValueError, match="q_pos: not contiguous"):
        t.pointers(3, 5, -1, device)


# ---- workspaces
def test_a_workspace_is_sized_by_shapes_alone_and_for_each_batch_size(lib):  # noqa: F811
    def need(T, k=0, at=F, **kw):
        q, c = queries(T=T, H=64, q=at), cache(max_pages=2048, n_seq=1, H_kv=8, token_stride=1024, page_stride=65536, k=at,
                                               v=at, block_table=at, seq_len=at, **kw)
        return lib.hisa_attention_workspace_bytes(C.byref(q), C.byref(c), k)

    # (as the header says)
    assert [need(T) for T in (64, 256, 1024)] == [34078720, 34078720, 0]
    for T in (1, 2, 3, 17, 64, 65, 255, 256, 300, 1023, 1024, 4096):
        for k in (0, 1, 100, 2048, 65536):
            for kw in (dict(), dict(dtype=FP8), dict(weights=hisa.HISA_WEIGHTS_8BIT)):
                size = need(T, k, **kw)
                assert size == need(T, k, at=1 << 40, **kw)             # (whatever the addresses are)
                q, c = queries(T=T, H=64), cache(max_pages=2048, n_seq=1, H_kv=8, token_stride=1024, page_stride=65536, **kw)
                if size:                                                # what is a byte less is refused, before any launch
                    status = paged(lib, q, c, n=size - 1) if k == 0 else sparse(lib, q, c, k=k, n=size - 1)
                    assert status == WS


def test_scales_that_overflow_are_refused(lib):  # noqa: F811
    """(In units of log2 a scale is 1.44 times as large.)"""
    q, c = queries(), cache()
    for scale in (2.4e38, 3.4e38, 2.0 ** 128):
        assert paged(lib, q, c, scale=scale) == SHAPE and sparse(lib, q, c, scale=scale) == SHAPE
    # the largest that header allows passes this check (and fails a later one: there is no workspace)
    assert paged(lib, q, cache(max_pages=2048), scale=1.7e38, ws=None, n=0) == WS
