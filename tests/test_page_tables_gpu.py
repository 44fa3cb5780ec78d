"""hisa_page_tables against the plain loop over sequences: whole numbers, equal to the last one."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as SO
from paper_2603_28458_amd import hisa

pytestmark = pytest.mark.gpu

FIELDS = ("seq_len", "q_start", "page_start", "q_seq", "q_pos", "slots", "key_rows")


def run(ctx, new, max_pages, page, rows, n_free=None, s_max=0, seed=0):
    g = np.random.default_rng(seed)
    n_seq = len(ctx)
    ids = g.permutation(4 * n_seq * max_pages + 16).astype(np.int32)
    table = ids[:n_seq * max_pages].reshape(n_seq, max_pages).copy()      # (entries behind a sequence's end too)
    free = ids[n_seq * max_pages:]
    free = free[:len(free) if n_free is None else n_free]
    dev = torch.device("cuda:0")

    def put(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)

    bt = put(table)
    # guard words on both sides of every output
    sizes = [n_seq, n_seq + 1, n_seq + 1, rows, rows, rows, rows]
    bufs = [torch.full((n + 128,), -77, dtype=torch.int32, device=dev) for n in sizes]
    parts = [b[64:64 + n] for b, n in zip(bufs, sizes)]
    out = hisa.PageTables(*parts[:6], parts[6] if s_max else None)
    print(f"\n[tables] n_seq={n_seq} page={page} max_pages={max_pages} rows={rows} free={len(free)}", flush=True)
    got = hisa.hisa_page_tables(put(ctx), put(new), bt, page, put(free), rows, s_max=s_max, out=out)
    torch.cuda.synchronize()
    want = SO.page_tables(ctx, new, table, page, free, rows, s_max)
    for f in FIELDS:
        if f == "key_rows" and not s_max:
            continue
        assert np.array_equal(getattr(got, f).cpu().numpy(), want[f]), f
    assert np.array_equal(bt.cpu().numpy(), want["block_table"])
    assert int(got.pages_used) == want["page_start"][-1]
    for b, n in zip(bufs, sizes):
        assert (b[:64] == -77).all() and (b[64 + n:] == -77).all()
    return got


@pytest.mark.parametrize("n_seq", [1, 2, 63, 64, 65, 1000, 1023, 1024, 1025, 3000, 5000])
@pytest.mark.parametrize("page", [1, 16, 100])
def test_ragged_batches(n_seq, page):
    g = np.random.default_rng(n_seq + page)
    ctx, new = g.integers(0, 200, n_seq), g.integers(0, 9, n_seq)
    new[g.random(n_seq) < 0.3] = 0
    ctx[g.random(n_seq) < 0.2] = 0
    ctx[g.random(n_seq) < 0.2] = 160                              # ends of pages
    rows = max(1, int(new.sum())) + int(g.integers(0, 70))
    run(ctx, new, 210 // page + 2, page, rows, s_max=230, seed=n_seq)


@pytest.mark.parametrize("n_seq", [1, 7, 1100])
def test_prompts(n_seq):
    g = np.random.default_rng(n_seq)
    new = g.integers(1, 5000 // n_seq + 2, n_seq)
    run(np.zeros(n_seq, int), new, -(-int(new.max()) // 16), 16, int(new.sum()))


@pytest.mark.parametrize("n_seq", [3, 1200])
def test_nothing_new(n_seq):
    got = run(np.full(n_seq, 33), np.zeros(n_seq, int), 5, 16, 10)
    assert (got.slots == -1).all() and (got.q_pos == -1).all() and int(got.pages_used) == 0


@pytest.mark.parametrize("n_seq", [4, 1030])
def test_free_pages_run_out(n_seq):
    run(np.full(n_seq, 30), np.full(n_seq, 20), 8, 16, 20 * n_seq, n_free=n_seq // 2 + 1)
    run(np.full(n_seq, 30), np.full(n_seq, 20), 8, 16, 20 * n_seq, n_free=0)


@pytest.mark.parametrize("n_seq", [4, 1030])
def test_tokens_beyond_the_table_or_the_rows(n_seq):
    ctx, new = np.arange(n_seq) % 60, np.arange(n_seq) % 23
    run(ctx, new, 3, 16, int(new.sum()), s_max=40)                # more tokens than three pages hold
    run(ctx + 100, new, 3, 16, int(new.sum()))                    # more cached than the table can say
    run(ctx, new, 8, 16, max(1, int(new.sum()) // 2))             # more tokens than rows


@pytest.mark.parametrize("n_seq", [4, 1030])
def test_negative_and_huge_lengths(n_seq):
    ctx, new = np.arange(n_seq) % 40, np.arange(n_seq) % 5
    ctx[1], new[2] = -7, -9
    run(ctx, new, 8, 16, int(np.maximum(new, 0).sum()))
    ctx[3], new[0] = 2 ** 31 - 1, 2 ** 31 - 1
    run(ctx, new, 8, 16, 500)


@pytest.mark.parametrize("n_seq", [4, 1030])
def test_positions_and_slots_past_31_bits(n_seq):
    ctx, new = np.arange(n_seq) % 40, np.full(n_seq, 3)
    ctx[1] = ctx[n_seq - 1] = 2 ** 31 - 2
    run(ctx, new, 8, 16, 3 * n_seq + 5, s_max=100)
    dev = torch.device("cuda:0")
    put = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)  # noqa: E731
    table = put([2 ** 27, -1], [7, -1])
    t = hisa.hisa_page_tables(put(15, 3), put(2, 1), table, 16, put(2 ** 27 - 1), 4)
    torch.cuda.synchronize()
    assert t.slots.tolist() == [-1, (2 ** 27 - 1) * 16, 7 * 16 + 3, -1]


def test_without_an_output_given():
    dev = torch.device("cuda:0")
    ctx, new = torch.tensor([5, 0], dtype=torch.int32, device=dev), torch.tensor([1, 3], dtype=torch.int32, device=dev)
    table = torch.full((2, 4), -1, dtype=torch.int32, device=dev)
    table[0, 0] = 9
    t = hisa.hisa_page_tables(ctx, new, table, 8, torch.tensor([3, 4], dtype=torch.int32, device=dev), 6)
    assert t.key_rows is None and t.slots.tolist() == [77, 24, 25, 26, -1, -1]
    t = hisa.hisa_page_tables(ctx, new, table, 8, torch.tensor([3, 4], dtype=torch.int32, device=dev), 6, s_max=32)
    assert t.key_rows.tolist() == [5, 32, 33, 34, -1, -1] and t.q_seq.tolist() == [0, 1, 1, 1, 0, 0]


@pytest.mark.parametrize("n_seq,new,page,rows,n_free", [
    (4, 2000, 1, 1000, None), (1, 5000, 1, 100, None), (1, 32000, 16, 512, None), (32, 4096, 16, 4096, None),
    (4, 2000, 1, 1000, 5000), (3, 1025, 1, 1, None),
    (2000, 160, 16, 8192, None), (2000, 160, 16, 8192, 12345), (1100, 7, 1, 1, None), (1025, 300, 7, 257, 40000)])
def test_more_new_pages_than_rows(n_seq, new, page, rows, n_free):
    """Every page of every new token is taken and named, whether the token has a row or not; in one launch and in two."""
    ctx = np.arange(n_seq) * 7 % 50
    run(ctx, np.full(n_seq, new), (new + 50) // page + 2, page, rows, n_free=n_free, seed=n_seq)
    # some sequences grow far past the rows, others not at all
    g = np.random.default_rng(n_seq)
    some = np.where(g.random(n_seq) < 0.4, 0, g.integers(0, 2 * new, n_seq))
    run(ctx, some, (new + 50) // page + 2, page, rows, n_free=n_free, s_max=64, seed=n_seq + 1)


@pytest.mark.parametrize("n_seq", [1, 1025])
def test_more_than_a_billion_new_pages(n_seq):
    """A table of more than 2^30 entries, all of them new."""
    dev = torch.device("cuda:0")
    most = (2 ** 30 + 12345) // n_seq
    table = torch.full((n_seq, most + 1), 7, dtype=torch.int32, device=dev)
    length = torch.full((n_seq,), most, dtype=torch.int32, device=dev)
    free = torch.tensor([11, 12, 13], dtype=torch.int32, device=dev)
    if n_seq > 1:
        length[0] += 1                                              # (into the last column)
    total = int(length.long().sum())
    assert total > 2 ** 30
    t = hisa.hisa_page_tables(torch.zeros_like(length), length, table, 1, free, 1 << 22)
    torch.cuda.synchronize()
    assert int(t.pages_used) == total and torch.equal(t.seq_len, length)
    assert table[0, :3].tolist() == [11, 12, 13] and int((table == -1).sum()) == total - 3
    assert int((table == 7).sum()) == n_seq * (most + 1) - total and int(table[-1, -1]) == 7
