"""The calls around the indexer run together, as a serving loop uses them: lengths -> tables and slots -> rows into the
caches (keys and values in pages, the indexer's keys in their padded array) -> pooled keys -> Stage 1 -> Stage 2 -> the
attention over the selected tokens, and over everything; prompts, chunks and single tokens, in a batch padded to a fixed
number of rows; eagerly, on another stream, and as a captured graph."""
import numpy as np
import pytest
import torch

from oracle import serving_oracle as SO
from paper_2603_28458_amd import hisa
from tests.serving import f64

pytestmark = pytest.mark.gpu

H_IDX, D, B, M_KEEP, K = 32, 128, 32, 4, 96
H, HKV, PAGE, ROWS, SMAX = 16, 2, 16, 160, 512


class Server:
    """Buffers of a program that serves `n` sequences; every step's inputs go into the same tensors."""

    def __init__(self, n, kv, seed=0):
        dev = self.dev = torch.device("cuda:0")
        self.n, self.kv = n, kv
        code = {"bf16": hisa.HISA_BF16, "fp8": hisa.HISA_FP8_E4M3}[kv]
        i32 = dict(dtype=torch.int32, device=dev)
        n_pages = n * SMAX // PAGE + 7
        g = torch.Generator().manual_seed(seed)
        self.free_all = torch.randperm(n_pages, generator=g).to(torch.int32).to(dev)
        self.taken = 0
        self.ctx, self.new = torch.zeros(n, **i32), torch.zeros(n, **i32)
        self.table = torch.full((n, SMAX // PAGE), -1, **i32)
        self.tables = hisa.PageTables.empty(n, ROWS, dev, key_rows=True)
        self.pages_left = torch.zeros(n_pages, **i32)
        store = torch.bfloat16 if kv == "bf16" else torch.uint8
        fill = float("nan") if kv == "bf16" else 0x7f

        def rows(*shape):
            return torch.full((*shape,), fill, dtype=store, device=dev)

        def scales(*shape):
            return torch.full(shape, float("nan"), device=dev) if kv == "fp8" else None

        self.cache = hisa.Cache(k=rows(n_pages, PAGE, HKV, D), v=rows(n_pages, PAGE, HKV, D), dtype=code,
                                block_table=self.table, seq_len=self.tables.seq_len,
                                k_scale=scales(n_pages, PAGE, HKV), v_scale=scales(n_pages, PAGE, HKV))
        self.keys = hisa.Keys(k=rows(n, SMAX, D), seq_len=self.tables.seq_len, dtype=code, k_scale=scales(n, SMAX))
        self.key_rows = hisa.Cache(k=self.keys.k.view(n, SMAX, 1, D), v=None, dtype=code,
                                   k_scale=None if kv == "bf16" else self.keys.k_scale.view(n, SMAX, 1))
        self.pooled = torch.zeros((n, SMAX // B, D), dtype=torch.bfloat16, device=dev)
        bf = dict(dtype=torch.bfloat16, device=dev)
        self.k_new, self.v_new = torch.zeros((ROWS, HKV, D), **bf), torch.zeros((ROWS, HKV, D), **bf)
        self.i_new = torch.zeros((ROWS, 1, D), **bf)
        self.queries = hisa.Queries(q=torch.zeros((ROWS, H, D), **bf), w=None, dtype=hisa.HISA_BF16,
                                    q_seq=self.tables.q_seq, q_pos=self.tables.q_pos)
        self.index = hisa.Queries(q=torch.zeros((ROWS, H_IDX, D), **bf),
                                  w=torch.zeros((ROWS, H_IDX), device=dev), dtype=hisa.HISA_BF16,
                                  q_seq=self.tables.q_seq, q_pos=self.tables.q_pos)
        self.blocks = torch.zeros((ROWS, M_KEEP), **i32)
        self.topk = torch.zeros((ROWS, K), **i32)
        self.dense, self.sparse = torch.zeros((ROWS, H, D), **bf), torch.zeros((ROWS, H, D), **bf)
        self.dense_lse, self.sparse_lse = torch.zeros((ROWS, H), device=dev), torch.zeros((ROWS, H), device=dev)

        def ws(n):
            return torch.empty(max(1, n), dtype=torch.uint8, device=dev)

        self.ws1 = ws(hisa.hisa_workspace_bytes(hisa.OP_BLOCK_SCORE_TOPK, self.index, self.keys, B, M_KEEP))
        self.ws2 = ws(hisa.hisa_workspace_bytes(hisa.OP_TOKEN_REFINE_TOPK, self.index, self.keys, B, M_KEEP, K))
        self.wsa = ws(max(hisa.hisa_attention_workspace_bytes(self.queries, self.cache, k) for k in (0, K)))

    def feed(self, ctx, new, seed):
        g = torch.Generator().manual_seed(seed)
        self.ctx.copy_(torch.tensor(ctx, dtype=torch.int32))
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        self.pages_left[:self.free_all.numel() - self.taken] = self.free_all[self.taken:]
        self.taken += sum(-(-(c + m) // PAGE) + (-c // PAGE) for c, m in zip(ctx, new))
        for t in (self.k_new, self.v_new, self.i_new, self.queries.q, self.index.q):
            t.copy_(torch.randn(t.shape, generator=g))
        self.index.w.copy_(torch.rand(self.index.w.shape, generator=g))

    def step(self):
        t = self.tables
        hisa.hisa_page_tables(self.ctx, self.new, self.table, PAGE, self.pages_left, ROWS, s_max=SMAX, out=t)
        hisa.hisa_cache_append(self.cache, t.slots, self.k_new, self.v_new)
        hisa.hisa_cache_append(self.key_rows, t.key_rows, self.i_new)
        hisa.hisa_pool_append(self.keys, B, self.ctx, SMAX, self.pooled)
        hisa.hisa_block_score_topk(self.index, self.keys, self.pooled, hisa.HISA_BF16, B, M_KEEP, block_idx=self.blocks,
                                   ws=self.ws1)
        hisa.hisa_token_refine_topk(self.index, self.keys, B, M_KEEP, self.blocks, K, topk_idx=self.topk, ws=self.ws2)
        hisa.hisa_sparse_attention(self.queries, self.cache, self.topk, out=self.sparse, lse=self.sparse_lse, ws=self.wsa)
        hisa.hisa_paged_attention(self.queries, self.cache, t.q_start, out=self.dense, lse=self.dense_lse, ws=self.wsa)

    def outputs(self):
        n = int(self.tables.q_start[-1])
        t = self.tables
        return [x.clone() for x in (t.slots, t.key_rows, t.q_seq, t.q_pos, self.table, self.topk[:n], self.sparse[:n],
                                    self.sparse_lse[:n], self.dense[:n], self.dense_lse[:n])]


STEPS = [([0, 0, 0, 0], [60, 1, 33, 0]), ([60, 1, 33, 0], [70, 40, 1, 49]), ([130, 41, 34, 49], [1, 1, 1, 1]),
         ([131, 42, 35, 50], [3, 0, 150, 1]), ([134, 42, 185, 51], [1, 1, 1, 1])]


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_a_serving_loop_against_the_oracle(kv):
    s = Server(4, kv)
    kept = {n: {"k": [], "v": [], "i": []} for n in range(4)}          # what each sequence's rows have to be
    for at, (ctx, new) in enumerate(STEPS):
        s.feed(ctx, new, seed=at)
        s.step()
        torch.cuda.synchronize()
        t0 = 0
        for n, m in enumerate(new):
            for name, x in (("k", s.k_new), ("v", s.v_new), ("i", s.i_new)):
                kept[n][name].append(x[t0:t0 + m].float().cpu())
            t0 += m
        topk = s.topk.cpu().numpy()
        q = f64(s.queries.q)
        t = 0
        for n, (c, m) in enumerate(zip(ctx, new)):
            rows = {name: torch.cat(kept[n][name]) for name in ("k", "v", "i")}
            if kv == "fp8":
                for name, x in rows.items():
                    scale = x.abs().amax(dim=-1, keepdim=True) / torch.tensor(448.0)
                    rows[name] = (x / scale).clamp(-448, 448).to(torch.float8_e4m3fn).float() * scale
            # the indexer's own array, as it reads it
            have = s.keys.k[n, :c + m]
            have = have.float() if kv == "bf16" else have.view(torch.float8_e4m3fn).float() * s.keys.k_scale[n, :c + m, None]
            assert torch.equal(have.cpu(), rows["i"][:, 0])
            k64, v64 = rows["k"].double().numpy(), rows["v"].double().numpy()
            for i in range(m):
                pos = c + i
                picks = topk[t][topk[t] >= 0]
                assert len(picks) == min(K, pos + 1) and picks.max() <= pos
                for pick, out, lse in ((picks, s.sparse, s.sparse_lse), (np.arange(pos + 1), s.dense, s.dense_lse)):
                    for h in range(HKV):
                        sl = slice(h * (H // HKV), (h + 1) * (H // HKV))
                        want, wl, mag = SO.attend(q[t, sl], k64[pick][:, h], v64[pick][:, h], D ** -0.5)
                        # (output and weights rounded to bf16: half a step each; fp32 sums: 2^-14 is far above them)
                        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -14) * mag
                        assert (np.abs(f64(out[t, sl]) - want) <= bound).all()
                        assert (np.abs(f64(lse[t, sl]) - wl) <= 2.0 ** -14 * (1 + np.abs(wl))).all()
                t += 1
        # rows behind the last token: nothing selected, nothing written by the attention over the cache
        assert (s.tables.slots[t:] == -1).all() and (topk[t:] == -1).all()
        assert (s.sparse[t:] == 0).all()


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_the_loop_as_one_graph_and_on_another_stream(kv):
    eager = Server(4, kv)
    want = []
    for at, (ctx, new) in enumerate(STEPS):
        eager.feed(ctx, new, seed=at)
        eager.step()
        torch.cuda.synchronize()
        want.append(eager.outputs())

    side = torch.cuda.Stream()
    other = Server(4, kv)
    with torch.cuda.stream(side):
        for at, (ctx, new) in enumerate(STEPS):
            other.feed(ctx, new, seed=at)
            other.step()
            for a, b in zip(other.outputs(), want[at]):
                assert torch.equal(a, b)
    torch.cuda.synchronize()

    s = Server(4, kv)
    s.feed([0, 0, 0, 0], [0, 0, 0, 0], seed=99)                        # a batch of padding: warms up, changes nothing
    with torch.cuda.stream(side):
        s.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    for at, (ctx, new) in enumerate(STEPS):
        s.feed(ctx, new, seed=at)
        assert torch.randn(1 << 18, device=s.dev).square().sum().item() > 0     # the program's own eager work
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(s.outputs(), want[at])):
            assert torch.equal(a, b), f"step {at}: output {i} of the replay differs from the eager one"


def test_two_graphs_with_workspaces_of_their_own_replayed_side_by_side():
    """Each call without a workspace given takes one of its own: graphs captured that way may overlap."""
    graphs = []
    for seed in (1, 2):
        s = Server(4, "bf16", seed=seed)
        for at, (ctx, new) in enumerate(STEPS):
            s.feed(ctx, new, seed=10 * seed + at)
            s.step()
        torch.cuda.synchronize()
        out = torch.zeros_like(s.dense)
        want, _ = hisa.hisa_paged_attention(s.queries, s.cache, s.tables.q_start, out=torch.zeros_like(out))
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            hisa.hisa_paged_attention(s.queries, s.cache, s.tables.q_start, out=out)
        graphs.append((s, graph, stream, out, want))
    for replay in range(3):
        for s, graph, stream, out, want in graphs:
            out.zero_()
        torch.cuda.synchronize()
        for s, graph, stream, out, want in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for s, graph, stream, out, want in graphs:
            assert torch.equal(out, want)
