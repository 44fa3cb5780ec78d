"""hisa_paged_attention against the plain 64-bit form: head layouts, lengths from nothing to long, pages that end inside a
tile, positions and first visible positions of every kind, rows that are nobody's, NaN in everything unseen."""
import numpy as np
import pytest
import torch

from paper_2603_28458_amd import hisa
from tests.serving import Batch

pytestmark = pytest.mark.gpu


def run(b, positions=None, lo=None, scale=None, q_pos="given", what=""):
    pos = b.pos if positions is None else positions
    if q_pos == "given":
        b.queries.q_pos = b.put(pos)
    else:
        b.queries.q_pos = None
    b.queries.q_lo = None if lo is None else b.put(lo)
    out = torch.full_like(b.queries.q, 7.25)
    lse = torch.full((b.T, b.H), 123.0, dtype=torch.float32, device=b.dev)
    print(f"\n[paged] {what} lens={b.lens[:6]} H={b.H}/{b.H_kv} d={b.d} kv={b.kv} page={b.page}", flush=True)
    hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, scale=scale, out=out, lse=lse)
    torch.cuda.synchronize()
    first = np.zeros(b.T, np.int64) if lo is None else np.maximum(0, lo)
    want = b.want(lambda t: np.arange(first[t], max(first[t], int(pos[t]) + 1)), scale)
    mine = b.check(out, lse, want, int(b.seq_len.max()), scale, what)
    nobody = ~mine[:, 0]
    assert (out[torch.from_numpy(nobody).to(b.dev)] == 7.25).all(), "rows of nobody were written"
    assert (lse[torch.from_numpy(nobody).to(b.dev)] == 123.0).all(), "rows of nobody were written"
    return out, lse


HEADS = [(8, 8), (8, 2), (32, 4), (64, 1), (40, 8), (7, 1), (1, 1)]


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("H,H_kv", HEADS)
def test_single_tokens(kv, H, H_kv):
    run(Batch([(0, 1), (1, 1), (31, 1), (32, 1), (63, 1), (64, 1), (300, 1), (1029, 1)], H=H, H_kv=H_kv, kv=kv, seed=H),
        what="decode")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 8, 16, 64, 256])
def test_pages(kv, d, page):
    run(Batch([(5, 3), (0, 17), (129, 1), (70, 33)], d=d, kv=kv, page=page, seed=page + d), what="pages")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("layout", ["token", "head", "apart"])
def test_cache_layouts(kv, layout):
    run(Batch([(5, 3), (0, 17), (129, 1), (70, 33)], kv=kv, layout=layout, seed=3), what=layout)


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("H,H_kv,d", [(8, 2, 128), (4, 4, 64), (16, 1, 64), (40, 8, 128), (6, 2, 128)])
def test_chunks(kv, H, H_kv, d):
    run(Batch([(0, 200), (513, 131), (64, 64), (1, 255)], H=H, H_kv=H_kv, d=d, kv=kv, page=32, seed=H + d), what="chunks")


@pytest.mark.parametrize("d", [4, 36, 100, 256])
def test_fp32_head_sizes(d):
    run(Batch([(0, 9), (100, 2), (65, 1)], H=6, H_kv=2, d=d, kv="f32", seed=d), what="fp32")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_a_long_sequence_beside_short_ones(kv):
    run(Batch([(20000, 2), (3, 1), (0, 1), (777, 5)], kv=kv, page=64, seed=1), what="long")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("new", [1, 90])
def test_positions_follow_from_the_lengths(kv, new):
    b = Batch([(33, new), (0, new), (500, new)], kv=kv, seed=5)
    given = run(b, what="given")
    derived = run(b, q_pos="derived", what="derived")
    assert torch.equal(given[0], derived[0]) and torch.equal(given[1], derived[1])


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("window", [1, 5, 64, 100])
def test_windows(kv, window):
    b = Batch([(300, 1), (90, 150), (0, 40), (1000, 3)], kv=kv, seed=window)
    run(b, lo=b.pos - window + 1, what=f"window {window}")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_documents_and_prefixes(kv):
    b = Batch([(40, 260), (0, 130)], kv=kv, seed=9)
    # documents of 50 tokens
    run(b, lo=b.pos // 50 * 50, what="documents")
    # the first 100 positions see each other whole
    run(b, positions=np.maximum(b.pos, np.where(b.pos >= 0, 99, -1)).astype(np.int32), what="prefix")
    # positions beyond the sequence see the sequence
    run(b, positions=b.pos + 1000, what="beyond")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("new", [1, 7, 150])
def test_rows_that_see_nothing(kv, new):
    b = Batch([(50, new), (0, new), (200, new)], kv=kv, seed=11)
    pos = b.pos.copy()
    pos[::3] = -1
    out, lse = run(b, positions=pos, what="before position 0")
    assert (out[::3] == 0).all() and torch.isneginf(lse[::3]).all()
    lo = np.zeros(b.T, np.int64)
    lo[1::2] = b.pos[1::2] + 1
    run(b, lo=lo, what="first visible behind the last")
    run(b, positions=np.full(b.T, -1, np.int32), what="nothing at all")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("new", [1, 40])
def test_rows_of_nobody_are_left_alone(kv, new):
    run(Batch([(50, new), (0, 0), (0, new), (9, 0)], kv=kv, seed=13, spare_rows=37, first_row=5), what="padded")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_pages_that_are_none_hold_nothing(kv):
    b = Batch([(200, 1), (90, 60)], kv=kv, page=16, seed=17)
    for n, j, bad in ((0, 2, -1), (0, 12, 1 << 20), (1, 0, -5), (1, 7, b.cache.k.shape[0])):
        b.table[n, j] = bad
    b.cache.block_table.copy_(torch.from_numpy(b.table))
    run(b, what="bad pages")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_unseen_rows_do_not_matter_whatever_they_hold(kv, new, bad):
    """Rows of the same sequence, in the same tiles, that some queries see and others do not."""
    b = Batch([(150, new), (20, new)], kv=kv, seed=19)
    lo = np.maximum(0, b.pos - 30)
    b.queries.q_pos, b.queries.q_lo = b.put(b.pos), b.put(lo)
    clean, clean_lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
    # one position before the windows (a tile's neighbour of theirs), and the last one of each chunk
    changed = {0: [100] + [150 + new - 1] * (new > 1), 1: [3] + [20 + new - 1] * (new > 1)}
    for n, p in ((n, p) for n in changed for p in changed[n]):
        page, o = int(b.table[n, p // b.page]), p % b.page
        for t, s in ((b.cache.k, b.cache.k_scale), (b.cache.v, b.cache.v_scale)):
            if b.kv == "fp8":
                t[page, o].view(torch.uint8).fill_(0x7f)
                s[page, o] = bad
            else:
                t[page, o, :, ::2] = bad
    out, lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
    torch.cuda.synchronize()
    blind = np.array([all(not (lo[t] <= p <= b.pos[t]) for p in changed[int(b.q_seq[t])]) for t in range(b.T)])
    assert blind.any()
    sel = torch.from_numpy(blind).to(b.dev)
    # (the wording of the contract: nothing at an unseen position affects a result)
    assert torch.equal(out[sel], clean[sel]) and torch.equal(lse[sel], clean_lse[sel])


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("new", [1, 70])
def test_infinite_values_that_are_seen(kv, new):
    if kv == "fp8":
        pytest.skip("e4m3 has no infinity")
    b = Batch([(40, new)], H=4, H_kv=1, kv=kv, seed=23)
    p = 40
    page, o = int(b.table[0, p // b.page]), p % b.page
    b.cache.v[page, o, 0, 3] = float("inf")
    b.cache.v[page, o, 0, 4] = -float("inf")
    b.cache.v[page, o, 0, 5] = float("nan")
    b.queries.q_pos = b.put(b.pos)
    out, _ = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start)
    assert (out[:, :, 3] == float("inf")).all() and (out[:, :, 4] == -float("inf")).all()
    assert out[:, :, 5].isnan().all()
    assert out[:, :, 6:].isfinite().all() and out[:, :, :3].isfinite().all()


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("gain,shift", [(60.0, 0.0), (8.0, 30.0), (0.0, 0.0)])
@pytest.mark.parametrize("new", [1, 80])
def test_large_and_equal_scores(kv, gain, shift, new):
    run(Batch([(700, new), (64, new)], kv=kv, q_gain=gain, k_shift=shift, seed=29), what=f"gain {gain} shift {shift}")


@pytest.mark.parametrize("scale", [1e-3, 0.5])
def test_scale(scale):
    run(Batch([(100, 1), (64, 90)], seed=31), scale=scale, what="scale")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_the_same_call_gives_the_same_bits_without_lse_too(kv):
    b = Batch([(3000, 1), (10, 1), (64, 90)], kv=kv, seed=37)
    b.queries.q_pos = b.put(b.pos)
    out, lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
    for _ in range(3):
        again, none = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start)
        assert none is None and torch.equal(again, out)


def test_strides_beyond_32_bits():
    """A pool whose later pages begin more than 2^32 bytes behind its first."""
    dev = torch.device("cuda:0")
    page, H_kv, d = 64, 1, 128
    n_pages = 1 << 19                                              # 4 Gi elements, 8 GiB each for keys and values
    k = torch.zeros((n_pages, page, H_kv, d), dtype=torch.bfloat16, device=dev)
    v = torch.zeros((n_pages, page, H_kv, d), dtype=torch.bfloat16, device=dev)
    g = torch.Generator(device=dev).manual_seed(3)
    ids = torch.tensor([[n_pages - 1, 1, n_pages // 2 + 7, n_pages - 9]], dtype=torch.int32, device=dev)
    for i in ids[0].tolist():
        k[i], v[i] = (torch.randn((page, H_kv, d), generator=g, device=dev).bfloat16() for _ in range(2))
    q = torch.randn((3, 8, d), generator=g, device=dev).bfloat16()
    small = ids[0].long()
    ref = hisa.Cache(k=k[small].clone(), v=v[small].clone(), dtype=hisa.HISA_BF16,
                     block_table=torch.arange(4, dtype=torch.int32, device=dev)[None],
                     seq_len=torch.tensor([250], dtype=torch.int32, device=dev))
    big = hisa.Cache(k=k, v=v, dtype=hisa.HISA_BF16, block_table=ids, seq_len=ref.seq_len)
    Q = hisa.Queries(q=q, w=None, dtype=hisa.HISA_BF16)
    start = torch.tensor([0, 3], dtype=torch.int32, device=dev)
    a, _ = hisa.hisa_paged_attention(Q, big, start)
    b, _ = hisa.hisa_paged_attention(Q, ref, start)
    assert torch.equal(a, b) and a.float().abs().sum() > 0
    lists = torch.arange(250, dtype=torch.int32, device=dev)[None].repeat(3, 1).contiguous()
    a, _ = hisa.hisa_sparse_attention(Q, big, lists)
    b, _ = hisa.hisa_sparse_attention(Q, ref, lists)
    assert torch.equal(a, b) and a.float().abs().sum() > 0
