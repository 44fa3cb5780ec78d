"""hisa_sparse_attention against the plain 64-bit form: lists of every length, padding anywhere, positions outside the
sequence, positions named twice, all head layouts and cache types."""
import numpy as np
import pytest
import torch

from paper_2603_28458_amd import hisa
from tests.serving import Batch

pytestmark = pytest.mark.gpu


def run(b, lists, scale=None, what=""):
    out = torch.full_like(b.queries.q, 7.25)
    lse = torch.full((b.T, b.H), 123.0, dtype=torch.float32, device=b.dev)
    print(f"\n[sparse] {what} lens={b.lens[:6]} k={lists.shape[1]} H={b.H}/{b.H_kv} d={b.d} kv={b.kv} page={b.page}",
          flush=True)
    hisa.hisa_sparse_attention(b.queries, b.cache, b.put(lists), scale=scale, out=out, lse=lse)
    torch.cuda.synchronize()
    want = b.want(lambda t: lists[t], scale, everybody=True)
    b.check(out, lse, want, lists.shape[1], scale, what)
    return out, lse


def draw(b, k, seed, holes=0.0):
    """Ascending distinct positions of each query's prefix, then -1; holes: some entries -1 wherever they stand."""
    g = np.random.default_rng(seed)
    lists = np.full((b.T, k), -1, np.int32)
    for t in range(b.T):
        n = int(b.pos[t]) + 1
        pick = np.sort(g.permutation(n)[:k])
        lists[t, :len(pick)] = pick
    lists[g.random(lists.shape) < holes] = -1
    return lists


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("H,H_kv", [(64, 1), (32, 1), (32, 2), (16, 4), (48, 8), (7, 1), (8, 8), (100, 1)])
def test_head_layouts(kv, H, H_kv):
    b = Batch([(700, 1), (90, 3), (0, 2)], H=H, H_kv=H_kv, kv=kv, seed=H)
    run(b, draw(b, 256, 1), what="heads")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("k", [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 500, 1000])
def test_list_lengths(kv, k):
    b = Batch([(900, 2), (30, 1), (0, 3)], H=32, H_kv=1, kv=kv, seed=k)
    run(b, draw(b, k, 2), what="lengths")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,layout", [(1, "token"), (8, "apart"), (64, "head")])
def test_pages_and_layouts(kv, d, page, layout):
    b = Batch([(400, 5), (77, 2)], H=16, H_kv=2, d=d, kv=kv, page=page, layout=layout, seed=d)
    run(b, draw(b, 200, 3), what=layout)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_padding_anywhere_order_and_repeats(kv):
    b = Batch([(400, 4), (77, 3)], H=32, H_kv=1, kv=kv, seed=5)
    lists = draw(b, 150, 4, holes=0.4)
    run(b, lists, what="holes")
    g = np.random.default_rng(6)
    run(b, np.stack([g.permutation(r) for r in lists]), what="any order")
    twice = lists.copy()
    twice[:, 75:] = twice[:, :75]
    run(b, twice, what="named twice")
    lists[2] = -1
    lists[5] = -1
    out, lse = run(b, lists, what="empty rows")
    assert (out[2] == 0).all() and torch.isneginf(lse[5]).all()


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_positions_outside_the_sequence_and_no_sequence(kv):
    b = Batch([(100, 2), (30, 2)], H=32, H_kv=2, kv=kv, seed=7)
    lists = draw(b, 64, 5)
    lists[:, 3] = 102
    lists[:, 7] = 2 ** 31 - 1
    lists[:, 9] = -(2 ** 31)
    lists[:, 60] = 60                                             # outside the second sequence, inside the first
    run(b, lists, what="outside")
    b.q_seq[:] = [0, 5, -1, 1]
    b.queries.q_seq.copy_(torch.from_numpy(b.q_seq))
    out, _ = run(b, lists, what="no sequence")
    assert (out[1] == 0).all() and (out[2] == 0).all()
    b.q_seq[:] = 0
    b.queries.q_seq = None
    run(b, lists, what="sequence 0")


@pytest.mark.parametrize("kv", ["bf16", "fp8", "f32"])
def test_unlisted_rows_do_not_matter(kv):
    b = Batch([(300, 3)], H=32, H_kv=1, kv=kv, seed=9)
    lists = draw(b, 100, 6, holes=0.2)
    clean, _ = hisa.hisa_sparse_attention(b.queries, b.cache, b.put(lists))
    for p in set(range(303)) - set(lists[lists >= 0].tolist()):
        page, o = int(b.table[0, p // b.page]), p % b.page
        for t in (b.cache.k, b.cache.v):
            t[page, o].view(torch.uint8).fill_(0x7f) if kv == "fp8" else t[page, o].fill_(float("nan"))
    # what a skipped entry is read from instead, if anything, is NaN as well
    out, _ = hisa.hisa_sparse_attention(b.queries, b.cache, b.put(lists))
    assert torch.equal(out, clean) and out.isfinite().all()


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("T,k", [(300, 384), (1, 8192), (40, 2048)])
def test_sizes_of_real_calls(kv, T, k):
    b = Batch([(9000 - T, T)], H=64, H_kv=1, kv=kv, page=64, seed=T)
    run(b, draw(b, k, 8), what="real")


def test_all_positions_listed_is_the_attention_over_the_cache():
    b = Batch([(250, 50), (0, 40)], H=16, H_kv=2, seed=41)
    b.queries.q_pos = b.put(b.pos)
    whole, whole_lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
    lists = np.full((b.T, 320), -1, np.int32)
    for t in range(b.T):
        lists[t, :b.pos[t] + 1] = np.arange(b.pos[t] + 1)
    out, lse = run(b, lists, what="whole")
    # both within half a bf16 step of the same numbers, each with weights rounded to bf16
    assert (out.float() - whole.float()).abs().max() <= 4 * 2.0 ** -8 * whole.float().abs().max()
    assert (lse - whole_lse).abs().max() <= 1e-4
