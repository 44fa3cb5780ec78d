"""The attention calls on either side of the sizes at which they take another way: weights in one or two parts, one token at
a time or tiles of rows, many parts to join, waves without rows, fp32 heads of any number and size."""
import numpy as np
import pytest
import torch

from paper_2603_28458_amd import hisa
from tests import test_paged_attention_gpu as paged
from tests import test_sparse_attention_gpu as sparse
from tests.serving import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,H,H_kv", [([(40, 1)], 7, 1), ([(700, 1), (64, 1)], 8, 2), ([(2000, 1)], 64, 1),
                                         ([(300, 9), (20, 30)], 8, 2), ([(0, 8)], 128, 2)])
def test_few_rows_are_as_good_as_their_own_rounding(kv, d, lens, H, H_kv):
    b = Batch(lens, H=H, H_kv=H_kv, d=d, kv=kv, seed=H + d)
    assert b.T * H <= 1024
    b.queries.q_pos = b.put(b.pos)
    out, lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
    want = b.want(lambda t: np.arange(int(b.pos[t]) + 1))
    b.check(out, lse, want, int(b.seq_len.max()), what="few rows", weights=2.0 ** -15)
    k = int(b.seq_len.max())
    lists = sparse.draw(b, k, 1)                                     # (all positions that a query sees)
    out, lse = hisa.hisa_sparse_attention(b.queries, b.cache, b.put(lists), want_lse=True)
    b.check(out, lse, want, k, what="few lists", weights=2.0 ** -15)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("tokens", [2, 3, 4, 5, 8, 9, 33])
@pytest.mark.parametrize("H,H_kv", [(8, 2), (64, 1), (40, 8)])
def test_a_few_new_tokens(kv, tokens, H, H_kv):
    """T at and around two, four tokens a sequence, lengths unequal; T * H on both sides of 1024."""
    b = Batch([(90, tokens), (513, 1), (0, tokens), (31, 0), (5, 2)], H=H, H_kv=H_kv, kv=kv, seed=tokens)
    paged.run(b, what=f"{tokens} tokens")
    paged.run(b, lo=np.maximum(0, b.pos - 40), what=f"{tokens} tokens, windows")


@pytest.mark.parametrize("kv,d,H,H_kv", [("bf16", 128, 8, 8), ("fp8", 64, 8, 1), ("bf16", 64, 64, 1), ("f32", 128, 8, 2),
                                         ("f32", 20, 3, 1), ("f32", 64, 4, 4), ("f32", 256, 2, 1)])
def test_many_parts_of_one_row(kv, d, H, H_kv):
    """One token over a long sequence beside a short one: up to 256 parts of the long row, most of the short one's empty."""
    b = Batch([(33000, 1), (70, 1)], H=H, H_kv=H_kv, d=d, kv=kv, page=64, seed=d, q_gain=1.0)
    paged.run(b, what="parts")
    b = Batch([(9000, 70)], H=H, H_kv=H_kv, d=d, kv=kv, page=64, seed=d + 1, q_gain=1.0)
    paged.run(b, what="parts of a chunk")


@pytest.mark.parametrize("k", [2048, 9000])
@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_many_parts_of_one_list(kv, k):
    b = Batch([(9500, 1), (100, 1)], H=16, H_kv=1, kv=kv, page=64, seed=k, q_gain=1.0)
    sparse.run(b, sparse.draw(b, k, 5, holes=0.1), what="parts")


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("new,H", [(1, 4), (1, 128), (9, 8), (9, 128), (70, 2), (70, 32), (300, 8)])
def test_infinite_values_stay_what_they_are(kv, new, H):
    b = Batch([(40, new)], H=H, H_kv=1 if H < 128 else 2, kv=kv, seed=new)
    page, o = int(b.table[0, 40 // b.page]), 40 % b.page
    for e, x in ((3, float("inf")), (4, -float("inf")), (5, float("nan"))):
        b.cache.v[page, o, :, e] = x
    b.queries.q_pos = b.put(b.pos)
    lists = b.put(np.tile(np.arange(41, dtype=np.int32), (b.T, 1)))
    for out, _ in (hisa.hisa_paged_attention(b.queries, b.cache, b.q_start),
                   hisa.hisa_sparse_attention(b.queries, b.cache, lists)):
        assert (out[:, :, 3] == float("inf")).all() and (out[:, :, 4] == -float("inf")).all()
        assert out[:, :, 5].isnan().all()
        assert out[:, :, 6:].isfinite().all() and out[:, :, :3].isfinite().all()


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("H", [4, 64])
@pytest.mark.parametrize("new", [6, 20, 61])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_unseen_rows_do_not_matter_in_tiles_with_idle_waves(kv, H, new, bad):
    b = Batch([(150, new)], H=H, H_kv=2, kv=kv, seed=new)
    b.queries.q_pos = b.put(b.pos)
    clean, clean_lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
    p = 150 + new // 2                                              # seen by the later half of the tokens
    page, o = int(b.table[0, p // b.page]), p % b.page
    for t, s in ((b.cache.k, b.cache.k_scale), (b.cache.v, b.cache.v_scale)):
        if kv == "fp8":
            s[page, o] = bad
        else:
            t[page, o, :, 1::3] = bad
    out, lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
    blind = new // 2
    assert torch.equal(out[:blind], clean[:blind]) and torch.equal(lse[:blind], clean_lse[:blind])
    assert not out[blind:].isfinite().all(dim=2).any()


@pytest.mark.parametrize("d", [8, 64, 96, 128, 200, 256])
@pytest.mark.parametrize("H,H_kv", [(40, 1), (70, 2), (3, 3)])
def test_fp32_groups(d, H, H_kv):
    b = Batch([(130, 3), (0, 40), (31, 1), (64, 0)], H=H, H_kv=H_kv, d=d, kv="f32", layout="apart", seed=d)
    paged.run(b, what="fp32")
    sparse.run(b, sparse.draw(b, 77, 1, holes=0.2), what="fp32")


@pytest.mark.parametrize("kv,d", [("bf16", 128), ("fp8", 64), ("f32", 36), ("f32", 128)])
@pytest.mark.parametrize("lens,H,H_kv", [([(3000, 1), (70, 1)], 8, 2), ([(700, 33), (0, 5), (9, 0)], 14, 2), ([(5000, 1)], 100, 1),
                                         ([(60, 300)], 4, 1)])
def test_nothing_beside_the_outputs_and_the_workspace_is_written(kv, d, lens, H, H_kv):
    b = Batch(lens, H=H, H_kv=H_kv, d=d, kv=kv, page=64, seed=d)
    b.queries.q_pos = b.put(b.pos)
    lists = b.put(sparse.draw(b, 600, 3))
    for k in (0, 600):
        size = hisa.hisa_attention_workspace_bytes(b.queries, b.cache, k)
        sizes = (b.T * H * d * b.queries.q.element_size(), b.T * H * 4, max(size, 16))
        bufs = [torch.full((n + 2048,), 0xA5, dtype=torch.uint8, device=b.dev) for n in sizes]
        out, lse, ws = (x[1024:1024 + n] for x, n in zip(bufs, sizes))
        out, lse = out.view(b.queries.q.dtype).view(b.T, H, d), lse.view(torch.float32).view(b.T, H)
        if k:
            hisa.hisa_sparse_attention(b.queries, b.cache, lists, out=out, lse=lse, ws=ws)
        else:
            hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, out=out, lse=lse, ws=ws)
        torch.cuda.synchronize()
        for x in bufs:
            assert (x[:1024] == 0xA5).all() and (x[-1024:] == 0xA5).all()
        want = (hisa.hisa_sparse_attention(b.queries, b.cache, lists) if k
                else hisa.hisa_paged_attention(b.queries, b.cache, b.q_start))[0]
        assert torch.equal(out, want)


@pytest.mark.parametrize("how", ["stream", "handle", "default"])
def test_what_a_call_allocates_belongs_to_its_stream(how, monkeypatch):
    b = Batch([(3000, 1), (70, 1)], seed=2)
    b.queries.q_pos = b.put(b.pos)
    want, wlse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    stream, handle = {"stream": (side, side.cuda_stream), "handle": (side.cuda_stream, side.cuda_stream), "default": (0, 0)}[how]
    seen = []
    for name in ("empty", "empty_like"):
        real = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, real=real, **kw: seen.append(torch.cuda.current_stream().cuda_stream)
                            or real(*a, **kw))
    with torch.cuda.stream(torch.cuda.Stream()):                     # (the caller's own stream is a third one)
        out, lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True, stream=stream)
        ctx, new = b.put([3000, 70]), b.put([1, 1])
        torch.cuda.synchronize()
        before = len(seen)
        assert seen == [handle] * before and before == 3             # out, lse, workspace
        t = hisa.hisa_page_tables(ctx, new, b.cache.block_table.clone(), b.page, b.put([0] * 9), 2, stream=stream)
        assert seen == [handle] * len(seen) and len(seen) > before
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wlse) and t.seq_len.tolist() == [3001, 71]


@pytest.mark.parametrize("kv,d", [("bf16", 128), ("fp8", 64), ("f32", 36), ("f32", 128)])
@pytest.mark.parametrize("new", [1, 3, 150])
def test_sequences_that_end_at_the_last_position(kv, d, new):
    """A table of 2^31 - 16 positions, of which the last 496 have pages: what is seen there is what a short sequence sees."""
    b = Batch([(496 - new, new)], H=8, H_kv=2, d=d, kv=kv, page=16, seed=new + d)
    lo = np.maximum(0, b.pos.astype(np.int64) - 99)
    want = b.want(lambda t: np.arange(lo[t], int(b.pos[t]) + 1))
    shift = 2 ** 31 - 512
    table = torch.full((1, 2 ** 27 - 1), -1, dtype=torch.int32, device=b.dev)
    table[0, shift // 16:] = b.cache.block_table[0, :31]
    b.cache.block_table, b.cache.seq_len = table, b.put([2 ** 31 - 16])
    b.queries.q_lo = b.put(lo + shift)
    print(f"\n[last position] kv={kv} d={d} new={new}", flush=True)
    for q_pos in (b.put(b.pos.astype(np.int64) + shift), None, b.put(np.full(b.T, 2 ** 31 - 1))):
        b.queries.q_pos = q_pos
        out, lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
        torch.cuda.synchronize()
        if q_pos is not None and int(q_pos[0]) == 2 ** 31 - 1:
            want = b.want(lambda t: np.arange(lo[t], 496))
        b.check(out, lse, want, 496, what="last position", weights=2.0 ** -15)
    lists = lo[:, None] + np.arange(130)
    out, lse = hisa.hisa_sparse_attention(b.queries, b.cache, b.put(lists + shift), want_lse=True)
    b.check(out, lse, b.want(lambda t: lists[t]), 496, what="last position, lists", weights=2.0 ** -15)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("far", [-2 ** 31, -2 ** 31 + 70, -2 ** 30, -2])
def test_positions_far_before_the_first_see_nothing(kv, new, far):
    """Beside rows of the same tile that see their prefix."""
    b = Batch([(200, new), (0, new), (31, new)], H=8, H_kv=2, kv=kv, seed=new)
    pos = b.pos.copy()
    pos[::3] = far
    out, lse = paged.run(b, positions=pos, what=f"position {far}")
    assert (out[::3] == 0).all() and torch.isneginf(lse[::3]).all()


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("chunk", [20, 90])
def test_a_mixed_batch_as_one_call_and_as_calls_of_its_parts(kv, chunk):
    """Single tokens, idle sequences and a chunk; each part with the same queries and outputs and its share of the tables."""
    b = Batch([(300 + i, 1) for i in range(9)] + [(0, 0)] * 20 + [(500, chunk)], kv=kv, spare_rows=11, first_row=2, seed=chunk)
    whole, whole_lse = paged.run(b, what="mixed")
    b.queries.q_pos = None
    out, lse = torch.full_like(b.queries.q, 7.25), torch.full((b.T, b.H), 123.0, device=b.dev)
    for first, last in ((0, 9), (29, 30)):
        part = hisa.Cache(k=b.cache.k, v=b.cache.v, dtype=b.cache.dtype, k_scale=b.cache.k_scale, v_scale=b.cache.v_scale,
                          block_table=b.cache.block_table[first:last], seq_len=b.cache.seq_len[first:last])
        hisa.hisa_paged_attention(b.queries, part, b.q_start[first:last + 1], out=out, lse=lse)
    torch.cuda.synchronize()
    mine = b.check(out, lse, b.want(lambda t: np.arange(int(b.pos[t]) + 1)), int(b.seq_len.max()), what="parts", weights=2.0 ** -15)
    nobody = torch.from_numpy(~mine[:, 0]).to(b.dev)
    assert (out[nobody] == 7.25).all() and (lse[nobody] == 123.0).all()


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_tokens_beyond_the_rows_with_the_tables_positions(kv):
    """More new tokens than rows: the rows there are stand for the first of them, which the tables' q_pos says."""
    b = Batch([(40, 30), (10, 125)], kv=kv, seed=3)
    rows = 70
    t = hisa.hisa_page_tables(b.put([40, 10]), b.put([30, 125]), b.cache.block_table.clone(), b.page, b.put(range(20)), rows)
    assert t.q_start.tolist() == [0, 30, 70] and torch.equal(t.seq_len, b.cache.seq_len)
    b.T, b.starts, b.q_start = rows, np.array([0, 30, 70], np.int32), t.q_start
    b.q64, b.q_seq, b.pos = b.q64[:rows], b.q_seq[:rows], b.pos[:rows]
    assert t.q_pos.tolist() == b.pos.tolist()
    b.queries = hisa.Queries(q=b.queries.q[:rows].contiguous(), w=None, dtype=b.queries.dtype)
    paged.run(b, positions=t.q_pos.cpu().numpy(), what="cut short")
