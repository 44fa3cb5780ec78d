"""Batches for the tests of the paged cache and its attention, with the oracle's answer and the tolerances.

Every slot that no sequence holds is filled with NaN, and so are the rows of the last page behind a sequence's end: a
kernel that lets an unseen row into a result shows it.

Tolerances, from the arithmetic (u = half a step of the output type relative to the value: bf16 2^-8, fp32 2^-24):
  scores    dot products of d terms in fp32 are off by at most (d + 8) * 2^-24 * sum |q k|, which shifts a weight by
            that much, times the scale, relatively: E (the largest over the batch, plus 2^-19 for the exponential of an
            fp32 argument of magnitude up to 2^6);
  weights   rounded to bf16 for the second product: 2^-8 each (bf16 and fp8 caches), nothing in fp32.  In two parts the
            first is cut (off by 2^-7 at most) and the second, what is left, rounded to bf16: 2^-7 2^-8 = 2^-15 each;
  sums      n terms in fp32 in any order: n * 2^-24, at most 2^-11 for n <= 8192, of sum p |v| / sum p = mag; this
            is far above what a tree or a matrix unit makes of it, so a quarter of it is asked for;
  output    u * |out|.
So |got - want| <= u |want| + (2 E + w + n 2^-26 + 2^-20) mag, with w = 2^-8 or 0, and for the log-sum-exp
2 E + n 2^-26 + 2^-20 + 2^-23 |lse|."""
from __future__ import annotations

import numpy as np
import torch

from oracle import serving_oracle as SO
from paper_2603_28458_amd import hisa

CODE = {"f32": hisa.HISA_F32, "bf16": hisa.HISA_BF16, "fp8": hisa.HISA_FP8_E4M3}


def f64(t):
    return t.detach().float().cpu().double().numpy() if t.dtype != torch.float64 else t.cpu().numpy()


class Batch:
    """Sequences of the given (cached, new) lengths in a scattered cache."""

    def __init__(self, lens, H=8, H_kv=2, d=128, kv="bf16", page=16, layout="token", seed=0, spare_rows=0, first_row=0,
                 q_gain=2.0, k_shift=0.0, device="cuda:0"):
        g = np.random.default_rng(seed)
        self.lens, self.H, self.H_kv, self.d, self.kv, self.page = lens, H, H_kv, d, kv, page
        total = [c + n for c, n in lens]
        need = [-(-t // page) for t in total]
        n_pages = sum(need) + 3
        ids = g.permutation(n_pages)
        width = max(need + [1]) + 1
        table = np.full((len(lens), width), -1, np.int32)
        at = 0
        for n, c in enumerate(need):
            table[n, :c] = ids[at:at + c]
            at += c
        held = np.zeros(n_pages * page, bool)
        for n, t in enumerate(total):
            p = np.arange(t)
            held[table[n, p // page].astype(np.int64) * page + p % page] = True
        self.table, self.held = table, held
        rows = {}
        scales = {}
        for name in ("k", "v"):
            x = torch.from_numpy(g.standard_normal((n_pages * page, H_kv, d)).astype(np.float32))
            if name == "k":
                x += k_shift
            if kv == "fp8":
                s = x.abs().amax(dim=2) / 448.0
                code = (x / s[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
                code.view(torch.uint8)[~torch.from_numpy(held)] = 0x7f           # NaN
                s[~torch.from_numpy(held)] = float("nan")
                rows[name], scales[name] = code, s
            else:
                x = x.to(torch.bfloat16 if kv == "bf16" else torch.float32)
                x[~torch.from_numpy(held)] = float("nan")
                rows[name] = x
        self.rows64 = {}
        for name in ("k", "v"):
            x = f64(rows[name])
            if kv == "fp8":
                x = x * f64(scales[name])[..., None]
            self.rows64[name] = x
        shape = (n_pages, page, H_kv, d)
        dev = torch.device(device)
        k, v = rows["k"].view(shape), rows["v"].view(shape)

        def move(t):                                   # (float8 copies go through bytes)
            return t.view(torch.uint8).to(dev).view(t.dtype) if t.dtype == torch.float8_e4m3fn else t.to(dev)

        if layout == "token":
            k, v = move(k), move(v)
        elif layout == "head":                         # [n_pages, H_kv, page, d]
            k, v = (move(t.permute(0, 2, 1, 3).contiguous()).permute(0, 2, 1, 3) for t in (k, v))
        else:                                          # keys and values of a page beside each other, rows apart
            both = torch.zeros((n_pages, 2, page, H_kv, d + 16), dtype=k.dtype)
            both[:, 0, :, :, :d], both[:, 1, :, :, :d] = k, v
            both = move(both)
            k, v = both[:, 0, :, :, :d], both[:, 1, :, :, :d]
        self.new = [n for _, n in lens]
        self.starts = np.concatenate([[first_row], first_row + np.cumsum(self.new)]).astype(np.int32)
        self.T = int(self.starts[-1]) + spare_rows
        qt = torch.float32 if kv == "f32" else torch.bfloat16
        q = (torch.from_numpy(g.standard_normal((self.T, H, d)).astype(np.float32)) * q_gain).to(qt)
        self.q64 = f64(q)
        self.seq_len = np.array(total, np.int32)
        self.cache = hisa.Cache(k=k, v=v, dtype=CODE[kv], block_table=torch.from_numpy(table).to(dev),
                                seq_len=torch.from_numpy(self.seq_len).to(dev),
                                k_scale=scales["k"].view(shape[:3]).to(dev) if scales else None,
                                v_scale=scales["v"].view(shape[:3]).to(dev) if scales else None)
        self.q_start = torch.from_numpy(self.starts).to(dev)
        self.q_seq = np.zeros(self.T, np.int32)
        self.pos = np.full(self.T, -1, np.int32)
        for n, (c, m) in enumerate(lens):
            self.q_seq[self.starts[n]:self.starts[n + 1]] = n
            self.pos[self.starts[n]:self.starts[n + 1]] = c + np.arange(m)
        self.dev = dev
        self.queries = hisa.Queries(q=q.to(dev), w=None, dtype=CODE["f32" if kv == "f32" else "bf16"],
                                    q_seq=torch.from_numpy(self.q_seq).to(dev))

    def put(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(self.dev)

    def want(self, positions_of, scale=None, everybody=False):
        """Oracle: positions_of(t); everybody: rows outside the sequences too (lists)."""
        scale = self.d ** -0.5 if scale is None else scale

        def seq_of(t):
            return int(self.q_seq[t]) if everybody or self.starts[0] <= t < self.starts[-1] else None

        return SO.attention(self.q64, self.rows64["k"], self.rows64["v"], self.table, self.seq_len, self.page, seq_of,
                            positions_of, scale)

    def check(self, got, lse, want, n_max, scale=None, what="", weights=2.0 ** -8):
        out, wlse, mag = want
        scale = self.d ** -0.5 if scale is None else scale
        kmax = np.nanmax(np.where(np.isfinite(self.rows64["k"]), np.abs(self.rows64["k"]), 0).sum(axis=2))
        E = (self.d + 8) * 2.0 ** -24 * scale * np.abs(self.q64).max() * kmax + 2.0 ** -19
        u = 2.0 ** -24 if self.kv == "f32" else 2.0 ** -8
        w = 0.0 if self.kv == "f32" else weights
        g = f64(got)
        mine = ~np.isnan(wlse)                                       # (rows that are somebody's)
        rel = 2 * E + w + n_max * 2.0 ** -26 + 2.0 ** -20
        bound = u * np.abs(out) + rel * mag
        err = np.abs(g - out)
        bad = ~(err <= bound) & mine[..., None]
        assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} values out of tolerance, first at "
                               f"{np.argwhere(bad)[0]}, got {g[bad][0]}, want {out[bad][0]}, bound {bound[bad][0]}")
        if lse is not None:
            l = f64(lse)
            empty = np.isneginf(wlse) & mine
            assert np.array_equal(np.isneginf(l) & mine, empty), f"{what}: empty rows of lse"
            seen = mine & ~empty
            lb = 2 * E + n_max * 2.0 ** -26 + 2.0 ** -20 + 2.0 ** -23 * np.abs(np.where(seen, wlse, 0))
            assert (np.abs(np.where(seen, l - np.where(seen, wlse, 0), 0)) <= lb).all(), f"{what}: lse"
        return mine
