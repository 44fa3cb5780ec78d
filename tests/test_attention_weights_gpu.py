"""How far the attention's results over bf16 and fp8 caches are from the 64-bit form in the mean square, in every kernel, with
many rows and few, alone and in a batch of padding: what a query gets does not hang on who else is in its call.

The tolerance.  A result rounded to bf16 is off by r, which the oracle's own result, rounded, says.  Weights in two parts
add at most 2^-15 of sum p |v| / sum p = mag, scores of d fp32 terms a few 2^-24 of their size each; with |out| of mag / 10 and
more in the mean square (the batches below: checked) and r of 2^-9.3 |out| (half a step of 2^-8..2^-9, evenly spread) the first
is at most 0.2 r, which adds to r as squares do: 1.02 r.  Weights of 8 bits are off by as much as the result's rounding, 1.41 r.
So two parts have to stay below 1.15 r, and 8 bits below the bound of each value (tests/serving.py)."""
import numpy as np
import pytest
import torch

from paper_2603_28458_amd import hisa
from tests import test_sparse_attention_gpu as sparse
from tests.serving import Batch, f64

pytestmark = pytest.mark.gpu


def ratio(got, want):
    """Root mean square error of `got` as a multiple of the rounded oracle's."""
    out, lse, mag = want
    mine = np.isfinite(lse)
    rounded = f64(torch.from_numpy(np.where(mine[..., None], out, 0)).to(torch.float32).to(torch.bfloat16))
    assert np.mean(out[mine] ** 2) >= 0.01 * np.mean(mag[mine] ** 2)
    return np.sqrt(np.mean((f64(got)[mine] - out[mine]) ** 2) / np.mean((rounded[mine] - out[mine]) ** 2))


def both(b, k=0, lo=None):
    """(result, the oracle's) over all that a query sees, or over lists of k."""
    b.queries.q_pos = b.put(b.pos)
    print(f"\n[weights] lens={b.lens[:6]} T={b.T} H={b.H}/{b.H_kv} d={b.d} kv={b.kv} k={k}", flush=True)
    if k:
        lists = sparse.draw(b, k, 1)
        out, lse = hisa.hisa_sparse_attention(b.queries, b.cache, b.put(lists), want_lse=True)
        want = b.want(lambda t: lists[t])
    else:
        out, lse = hisa.hisa_paged_attention(b.queries, b.cache, b.q_start, want_lse=True)
        want = b.want(lambda t: np.arange(int(b.pos[t]) + 1))
    return out, lse, want


SHAPES = [([(300 + 7 * i, 1) for i in range(40)], 32, 4, 0),       # single tokens
          ([(300 + 7 * i, 1) for i in range(20)], 64, 1, 0),       # 64 heads a workgroup
          ([(700, 30), (40, 90)], 16, 2, 0),                       # chunks
          ([(0, 300)], 8, 8, 0),
          ([(900, 70)], 32, 2, 200),                               # lists
          ([(900, 70)], 64, 1, 200)]


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,H,H_kv,k", SHAPES)
def test_many_rows_are_as_good_as_their_own_rounding(kv, d, lens, H, H_kv, k):
    b = Batch(lens, H=H, H_kv=H_kv, d=d, kv=kv, page=32, seed=H + d)
    assert b.T * H > 1024
    out, lse, want = both(b, k)
    b.check(out, lse, want, int(b.seq_len.max()), what="many rows", weights=2.0 ** -15)
    assert ratio(out, want) <= 1.15


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_rows_of_padding_change_nothing(kv):
    b = Batch([(300, 1), (90, 1), (513, 1), (64, 1)], H=16, H_kv=2, kv=kv, spare_rows=156, seed=3)
    assert b.T * b.H > 1024
    out, lse, want = both(b)
    b.check(out, lse, want, int(b.seq_len.max()), what="padded", weights=2.0 ** -15)
    assert ratio(out, want) <= 1.15


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,H,H_kv,k", SHAPES + [([(2000, 1)], 8, 2, 0), ([(2000, 1)], 8, 2, 600), ([(60, 9)], 64, 1, 0)])
def test_weights_of_8_bits_where_they_are_asked_for(kv, d, lens, H, H_kv, k):
    b = Batch(lens, H=H, H_kv=H_kv, d=d, kv=kv, page=32, seed=H + d)
    fine, fine_lse, want = both(b, k)
    b.cache.weights = hisa.HISA_WEIGHTS_8BIT
    out, lse, _ = both(b, k)
    b.check(out, lse, want, int(b.seq_len.max()), what="8 bits", weights=2.0 ** -8)
    assert torch.equal(lse, fine_lse) and not torch.equal(out, fine)      # (the sum of the weights is not rounded)
    b.cache.weights = hisa.HISA_WEIGHTS_16BIT
    assert torch.equal(both(b, k)[0], fine)
