"""The serving operators around the indexer, timed: building block tables and slot maps from request lengths, writing
new rows into a paged cache, attention of new tokens over the paged cache, and attention over the tokens that the
indexer selected.

`own` False computes them in plain torch operations, in fp32; `own` True makes the calls of
`paper_2603_28458_amd.hisa` that a serving program makes.
"""
import math

import torch

own = False

DEV = "cuda"
F8 = torch.float8_e4m3fn
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": F8}
BYTES = {"f32": 4, "bf16": 2, "fp8": 1}
ROWS_AT_ONCE = 1 << 30          # elements of an intermediate array of the plain forms


# ---------------------------------------------------------------------------------------------- cases
def _tables(name, *, n_seq, page, ctx, new, pad=0):
    """ctx, new: largest context and largest number of new tokens of a sequence; pad: token rows behind the last."""
    c = {"op": "tables", "n_seq": n_seq, "page": page, "ctx": ctx, "new": new, "pad": pad}
    return dict(c, name=name) if name else c


def _append(name, *, T, R, d, src, dst, page, values=True):
    """T rows of R heads of d elements; values False: one array (the indexer's keys), True: keys and values."""
    c = {"op": "append", "T": T, "R": R, "d": d, "src": src, "dst": dst, "page": page, "values": values}
    return dict(c, name=name) if name else c


def _paged(name, *, n_seq, new, ctx, H, Hkv, d, kv, page, ragged=True, window=0, lse=False):
    """new tokens at the end of ctx cached ones, per sequence (the longest; ragged: the others shorter); window > 0: a
    token sees that many positions."""
    c = {"op": "paged", "n_seq": n_seq, "new": new, "ctx": ctx, "H": H, "Hkv": Hkv, "d": d, "kv": kv, "page": page,
         "ragged": ragged, "window": window, "lse": lse}
    return dict(c, name=name) if name else c


def _sparse(name, *, n_seq, T, L, k, H, Hkv, d, kv, page, lse=False):
    """T queries (the last of each sequence's tokens) over k selected tokens each, contexts up to L."""
    c = {"op": "sparse", "n_seq": n_seq, "T": T, "L": L, "k": k, "H": H, "Hkv": Hkv, "d": d, "kv": kv, "page": page,
         "lse": lse}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the bookkeeping of a decode step of the benchmark's batch: one new token in each of 32 long sequences
        _tables("tables_decode32", n_seq=32, page=64, ctx=131072, new=1),
        # many requests at once, prompts of every length beside running ones, in a batch padded to a fixed size
        _tables("tables_mixed1000", n_seq=1000, page=16, ctx=20011, new=131, pad=777),
        # a decode step of 200 sequences into an fp8 cache
        _append("append_decode200_fp8", T=200, R=4, d=128, src="bf16", dst="fp8", page=64),
        # a prefill chunk into a bf16 cache
        _append("append_chunk16k_bf16", T=16384, R=8, d=128, src="bf16", dst="bf16", page=64),
        # the indexer's own keys of that chunk, as codes and scales in its padded key array
        _append("append_keys16k_fp8", T=16384, R=1, d=128, src="bf16", dst="fp8", page=65536, values=False),
        # one user's decode step on a short context: the smallest call of a serving loop
        _paged("paged_decode1_bf16", n_seq=1, new=1, ctx=1009, H=32, Hkv=8, d=128, kv="bf16", page=64),
        # the decode batch of the benchmark: 32 sequences of 96K to 128K tokens
        _paged("paged_decode32_bf16", n_seq=32, new=1, ctx=131071, H=64, Hkv=8, d=128, kv="bf16", page=64),
        # a wide decode batch on an fp8 cache, ragged, lengths that are no multiple of anything
        _paged("paged_decode200_fp8", n_seq=200, new=1, ctx=20011, H=32, Hkv=4, d=128, kv="fp8", page=16),
        # 1024 new tokens at the end of 64K: a chunk of a long prompt
        _paged("paged_chunk1024_64k_bf16", n_seq=1, new=1024, ctx=64512, H=64, Hkv=8, d=128, kv="bf16", page=64, lse=True),
        # several prompts prefilled at once behind short cached prefixes, windowed, fp8, small heads
        _paged("paged_ragged11_fp8", n_seq=11, new=2777, ctx=1500, H=32, Hkv=2, d=64, kv="fp8", page=32, window=1024),
        # the decode batch on the indexer's selection, all heads on one key row per token
        _sparse("sparse_decode32_bf16", n_seq=32, T=32, L=131072, k=2048, H=64, Hkv=1, d=128, kv="bf16", page=64),
        # the chunk on the indexer's selection
        _sparse("sparse_chunk1024_64k_bf16", n_seq=1, T=1024, L=65536, k=2048, H=64, Hkv=1, d=128, kv="bf16", page=64,
                lse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges, none costlier than the decode batch of 32."""
    op = rng.choice(["tables", "append", "paged", "paged", "paged", "sparse", "sparse"])
    page = rng.choice([16, 32, 64, 128])
    if op == "tables":
        n_seq = _log(rng, 1, 4096)
        new = 1 if rng.random() < 0.4 else _log(rng, 2, max(3, min(8192, 262144 // n_seq)))
        return _tables(None, n_seq=n_seq, page=page, ctx=_log(rng, 1, min(131072, (1 << 27) // n_seq)), new=new,
                       pad=rng.choice([0, 0, rng.randint(1, 2000)]))
    if op == "append":
        src, dst = rng.choice([("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "fp8"), ("f32", "f32"), ("f32", "bf16"),
                               ("f32", "fp8")])
        values = rng.random() < 0.7
        return _append(None, T=_log(rng, 1, 32768), R=rng.choice([1, 2, 4, 8]) if values else 1, d=rng.choice([64, 128]),
                       src=src, dst=dst, page=page if values else 65536, values=values)
    kv = rng.choice(["bf16", "bf16", "fp8", "fp8", "f32"])
    d = rng.choice([64, 128, 128])
    if op == "sparse":
        H, Hkv = rng.choice([(64, 1), (64, 1), (32, 1), (32, 2), (16, 4), (48, 8), (7, 1)])
        L = _log(rng, 64, 131072)
        n_seq = rng.choice([1, 1, _log(rng, 2, 64)])
        T = n_seq if rng.random() < 0.4 else n_seq * _log(rng, 1, max(1, min(2048 // n_seq, L)))
        k = rng.choice([2048, 1024, 512, rng.randint(1, 700)])
        if kv == "f32":
            T, L, k = min(T, 256), min(L, 8192), min(k, 512)
            n_seq = min(n_seq, T)
            T = T // n_seq * n_seq
        return _sparse(None, n_seq=n_seq, T=T, L=L, k=min(k, L), H=H, Hkv=Hkv, d=d, kv=kv, page=page,
                       lse=rng.random() < 0.5)
    H, Hkv = rng.choice([(64, 8), (32, 8), (32, 2), (64, 1), (16, 16), (40, 8), (7, 1)])
    if kv == "f32":
        return _paged(None, n_seq=rng.randint(1, 8), new=_log(rng, 1, 100), ctx=_log(rng, 1, 3000), H=H, Hkv=Hkv, d=d,
                      kv=kv, page=page, window=rng.choice([0, 0, 200]), lse=rng.random() < 0.5)
    kind = rng.choice(["decode", "decode", "few", "chunk"])
    if kind == "decode":                       # one new token a sequence; at most 4 GB of cache
        n_seq = _log(rng, 1, 256)
        ctx = _log(rng, 1, min(131071, (1 << 32) // (n_seq * Hkv * d * 2 * BYTES[kv])))
        return _paged(None, n_seq=n_seq, new=1, ctx=ctx, H=H, Hkv=Hkv, d=d, kv=kv, page=page,
                      window=rng.choice([0, 0, 0, 1024]), lse=rng.random() < 0.3)
    if kind == "few":                          # a few tokens a sequence: speculative steps, tails of prompts
        n_seq = _log(rng, 1, 64)
        ctx = _log(rng, 1, min(131071, (1 << 32) // (n_seq * Hkv * d * 2 * BYTES[kv])))
        return _paged(None, n_seq=n_seq, new=rng.randint(2, 77), ctx=ctx, H=H, Hkv=Hkv, d=d, kv=kv, page=page,
                      window=rng.choice([0, 0, 0, 1024]), lse=rng.random() < 0.3)
    new = _log(rng, 78, 8192)                  # a chunk of a prompt; at most the work of 1024 tokens at 64K
    ctx = _log(rng, 1, max(2, min(65536, (1 << 31) * 128 // (H * d) // new - new // 2)))
    n_seq = rng.choice([1, 1, rng.randint(2, 6)])
    return _paged(None, n_seq=n_seq, new=max(1, new // n_seq), ctx=ctx, H=H, Hkv=Hkv, d=d, kv=kv, page=page,
                  window=rng.choice([0, 0, 0, 1000]), lse=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------- shapes of a case
def _lens(case):
    """(cached tokens, new tokens) of each sequence: plain lists, the same for every seed."""
    n = case["n_seq"]
    ctx, new = [], []
    for i in range(n):
        f = ((i * 2654435761 + 12345) % 4096) / 4096.0           # ragged, and the longest first
        if case["op"] == "tables":
            ctx.append(case["ctx"] if i == 0 else int(case["ctx"] * f) if i % 7 else 0)
            new.append(case["new"] if i == 0 or case["new"] == 1 else int(case["new"] * (1.0 - f)))
        elif case["op"] == "sparse":
            ctx.append(case["L"] if i == 0 else max(case["T"] // n, int(case["L"] * (0.75 + 0.25 * f))))
            new.append(case["T"] // n)
        else:
            low = 0.75 if n <= 64 else 0.05
            f = 1.0 if i == 0 or not case["ragged"] else low + (1.0 - low) * f
            ctx.append(int(case["ctx"] * f))
            new.append(max(1, int(case["new"] * f)))
    if case["op"] == "sparse":
        ctx = [max(0, c - m) for c, m in zip(ctx, new)]
    return ctx, new


def _visible(case):
    """Keys that the new tokens of each sequence see, summed over its tokens."""
    out = []
    for c, n in zip(*_lens(case)):
        w = case.get("window", 0)
        full = n * c + n * (n + 1) // 2
        if w:
            full = sum(min(w, c + i + 1) for i in range(n)) if n < 4096 else min(full, n * w)
        out.append(full)
    return out


def work(case):
    op = case["op"]
    if op == "tables":
        ctx, new = _lens(case)
        pages = sum(-(-(c + n) // case["page"]) + (-c // case["page"]) for c, n in zip(ctx, new))
        touched = sum((c + n - 1) // case["page"] - c // case["page"] + 1 if n else 0 for c, n in zip(ctx, new))
        rows = sum(new) + case["pad"]
        return {"bytes": case["n_seq"] * 16 + pages * 8 + (touched - pages) * 4 + rows * 16, "flops": 0}
    if op == "append":
        n = case["T"] * case["R"] * (2 if case["values"] else 1)
        return {"bytes": n * case["d"] * (BYTES[case["src"]] + BYTES[case["dst"]]) + (4 * n if case["dst"] == "fp8" else 0)
                + 4 * case["T"], "flops": 0}
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    ctx, new = _lens(case)
    T = sum(new)
    qb = 4 if case["kv"] == "f32" else 2
    row = Hkv * 2 * (d * BYTES[case["kv"]] + (4 if case["kv"] == "fp8" else 0))
    io = T * H * (d * 2 * qb + (4 if case["lse"] else 0))
    if op == "paged":
        w = case["window"]
        keys = sum(min(c + n, w + n - 1) if w else c + n for c, n in zip(ctx, new))
        return {"bytes": keys * row + io + keys // case["page"] * 4, "flops": sum(_visible(case)) * H * 4 * d}
    picked = sum(min(case["k"], c + i + 1) for c, n in zip(ctx, new) for i in range(n))
    distinct = sum(min(c + n, n * case["k"]) for c, n in zip(ctx, new))
    return {"bytes": distinct * row + io + T * case["k"] * 4, "flops": picked * H * 4 * d}


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed((seed * 1000003 + stream * 7919 + 17) & 0x7fffffff)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _normal(shape, gen, dtype):
    """Unit normal rows; for large arrays drawn in pieces, so that no fp32 copy of the whole is needed."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    step = 1 << 28
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=gen, device=DEV, dtype=torch.bfloat16 if dtype == torch.bfloat16
                                    else torch.float32)
    return out


def _quantised(shape, gen):
    """Codes and scales of rows of the given shape, as a serving program holds them."""
    codes = torch.empty(shape, dtype=F8, device=DEV)
    scale = torch.empty(shape[:-1], dtype=torch.float32, device=DEV)
    c, s = codes.view(-1, shape[-1]), scale.view(-1)
    step = (1 << 27) // shape[-1]
    for i in range(0, s.numel(), step):
        n = min(step, s.numel() - i)
        x = torch.randn((n, shape[-1]), generator=gen, device=DEV)
        a = x.abs().amax(dim=1) / 448.0
        c[i:i + n] = (x / a[:, None]).clamp(-448.0, 448.0).to(F8)
        s[i:i + n] = a
    return codes, scale


def _cache(case, seed, lens):
    """A pool of pages, scattered over the sequences at random, with room behind the longest."""
    page, Hkv, d, kv = case["page"], case["Hkv"], case["d"], case["kv"]
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=_gen(seed, 1), device=DEV).to(torch.int32)
    width = max(need) + 1
    col = torch.arange(width, device=DEV)[None, :]
    need_t = torch.tensor(need, device=DEV)
    first = torch.cumsum(need_t, 0) - need_t
    table = torch.where(col < need_t[:, None], order[(first[:, None] + col).clamp(max=n_pages - 1)], -1).to(torch.int32)
    st = {"block_table": table.contiguous(), "seq_len": _ints(lens)}
    shape = (n_pages, page, Hkv, d)
    if kv == "fp8":
        st["k"], st["k_scale"] = _quantised(shape, _gen(seed, 2))
        st["v"], st["v_scale"] = _quantised(shape, _gen(seed, 3))
    else:
        st["k"], st["v"] = _normal(shape, _gen(seed, 2), TORCH[kv]), _normal(shape, _gen(seed, 3), TORCH[kv])
    return st


def prepare(case, seed):
    op = case["op"]
    st = {"case": case}
    if op == "tables":
        ctx, new = _lens(case)
        page = case["page"]
        g = _gen(seed, 0)
        # lengths differ from seed to seed by less than a page, their sums' bounds do not
        jitter = torch.randint(0, page, (len(ctx),), generator=g, device=DEV).to(torch.int32)
        ctx_t = (_ints(ctx) - jitter).clamp(min=0)
        width = -(-(max(c + n for c, n in zip(ctx, new))) // page) + 1
        bound = sum(-(-(c + n) // page) + 1 for c, n in zip(ctx, new))
        order = torch.randperm(bound + 5, generator=g, device=DEV).to(torch.int32)
        had = (ctx_t + page - 1) // page
        first = torch.cumsum(had, 0) - had
        col = torch.arange(width, device=DEV)[None, :]
        take = (first[:, None] + col).clamp(max=bound)
        st["block_table"] = torch.where(col < had[:, None], order[take], -1).to(torch.int32).contiguous()
        rest = torch.arange(bound + 5, device=DEV) >= had.sum()
        # the pages that no sequence holds, in the order in which they became free
        st["free_pages"] = order[torch.argsort((~rest).to(torch.int32), stable=True)].contiguous()
        st["ctx_len"], st["new_len"] = ctx_t, _ints(new)
        st["rows"] = sum(new) + case["pad"]
        st["s_max"] = width * page
        # (their number is not known to the host: the list is long enough for every sequence's growth)
    elif op == "append":
        T, R, d, page = case["T"], case["R"], case["d"], case["page"]
        n_pages = -(-T // page) + (2 if case["values"] else 1)
        g = _gen(seed, 0)
        st["k_new"] = _normal((T, R, d), g, TORCH[case["src"]])
        st["v_new"] = _normal((T, R, d), g, TORCH[case["src"]]) if case["values"] else None
        slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:T].to(torch.int32)
        if T > 64:                                        # chunks lie in runs; a few rows are padding
            pages = torch.randperm(n_pages, generator=g, device=DEV)
            t = torch.arange(T, device=DEV)
            slots = (pages[t // page] * page + t % page).to(torch.int32)
            slots[-3:] = -1
        st["slots"] = slots.contiguous()
        for name in ("k", "v") if case["values"] else ("k",):
            st[name] = torch.zeros((n_pages, page, R, d), dtype=TORCH[case["dst"]], device=DEV)
            if case["dst"] == "fp8":
                st[name + "_scale"] = torch.ones((n_pages, page, R), dtype=torch.float32, device=DEV)
    else:
        ctx, new = _lens(case)
        lens = [c + n for c, n in zip(ctx, new)]
        st.update(_cache(case, seed, lens))
        T, H, d = sum(new), case["H"], case["d"]
        qt = torch.float32 if case["kv"] == "f32" else torch.bfloat16
        # scores of standard deviation 2: a few tokens carry most of a row's weight
        st["q"] = (_normal((T, H, d), _gen(seed, 4), torch.float32) * 2.0).to(qt)
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        st["ctx"], st["new"], st["starts"] = ctx, new, starts
        st["q_start"] = _ints(starts)
        q_seq = torch.repeat_interleave(torch.arange(len(new), device=DEV), torch.tensor(new, device=DEV))
        pos = torch.arange(T, device=DEV) - torch.tensor(starts[:-1], device=DEV)[q_seq] + torch.tensor(ctx, device=DEV)[q_seq]
        st["q_seq"], st["q_pos"] = q_seq.to(torch.int32), pos.to(torch.int32)
        if op == "paged":
            st["q_lo"] = (pos - case["window"] + 1).clamp(min=0).to(torch.int32) if case["window"] else None
        else:
            st["topk_idx"] = _selection(case["k"], pos, _gen(seed, 5))
    if own:
        st["own"] = _handles(st)
    return st


def _selection(k, pos, gen):
    """[T, k] distinct positions <= pos, ascending, then -1: half of them from a few blocks of 128 tokens, as a
    selection by blocks gives them, the rest anywhere."""
    out = torch.full((pos.numel(), k), -1, dtype=torch.int32, device=DEV)
    L = int(pos.max()) + 1
    step = max(1, (1 << 27) // L)
    for i in range(0, pos.numel(), step):
        p = pos[i:i + step]
        key = torch.rand((p.numel(), L), generator=gen, device=DEV)
        hot = torch.rand((p.numel(), -(-L // 128)), generator=gen, device=DEV) < 0.125
        key += hot.repeat_interleave(128, dim=1)[:, :L] * 0.2
        key.masked_fill_(torch.arange(L, device=DEV)[None, :] > p[:, None], -1.0)
        top = torch.topk(key, min(k, L), dim=1)
        ids = torch.where(top.values >= 0, top.indices, L).sort(dim=1).values
        out[i:i + step, :ids.shape[1]] = torch.where(ids < L, ids, -1).to(torch.int32)
    return out


# ---------------------------------------------------------------------------------------------- the framework's calls
def _handles(st):
    """What a serving program sets up once: descriptors, outputs and the workspace."""
    from paper_2603_28458_amd import hisa
    case = st["case"]
    op = case["op"]
    if op == "tables":
        n, rows = case["n_seq"], st["rows"]
        return {"out": hisa.PageTables.empty(n, rows, DEV, key_rows=True)}
    code = {"f32": hisa.HISA_F32, "bf16": hisa.HISA_BF16, "fp8": hisa.HISA_FP8_E4M3}
    cache = hisa.Cache(k=st["k"], v=st.get("v"), dtype=code[case["dst" if op == "append" else "kv"]],
                       block_table=st.get("block_table"), seq_len=st.get("seq_len"), k_scale=st.get("k_scale"),
                       v_scale=st.get("v_scale"))
    if op == "append":
        return {"cache": cache}
    q = hisa.Queries(q=st["q"], w=None, dtype=code["f32" if case["kv"] == "f32" else "bf16"], q_seq=st["q_seq"],
                     q_pos=st["q_pos"], q_lo=st.get("q_lo"))
    k = case["k"] if op == "sparse" else 0
    nbytes = hisa.hisa_attention_workspace_bytes(q, cache, k)
    return {"cache": cache, "q": q, "out": torch.empty_like(st["q"]),
            "lse": torch.empty(st["q"].shape[:2], dtype=torch.float32, device=DEV) if case["lse"] else None,
            "ws": torch.empty(nbytes, dtype=torch.uint8, device=DEV) if nbytes else None}


def _run_own(st):
    from paper_2603_28458_amd import hisa
    case = st["case"]
    op = case["op"]
    h = st.get("own")
    if h is None:
        h = st["own"] = _handles(st)
    if op == "tables":
        t = hisa.hisa_page_tables(st["ctx_len"], st["new_len"], st["block_table"], case["page"], st["free_pages"],
                                  st["rows"], s_max=st["s_max"], out=h["out"])
        return {"seq_len": t.seq_len, "q_start": t.q_start, "q_seq": t.q_seq, "q_pos": t.q_pos, "slots": t.slots,
                "key_rows": t.key_rows, "pages_used": t.pages_used, "block_table": st["block_table"]}
    if op == "append":
        hisa.hisa_cache_append(h["cache"], st["slots"], st["k_new"], st["v_new"])
        return _held(st)
    if op == "paged":
        hisa.hisa_paged_attention(h["q"], h["cache"], st["q_start"], out=h["out"], lse=h["lse"], ws=h["ws"])
    else:
        hisa.hisa_sparse_attention(h["q"], h["cache"], st["topk_idx"], out=h["out"], lse=h["lse"], ws=h["ws"])
    return [h["out"], h["lse"]] if case["lse"] else [h["out"]]


def _held(st):
    return {n: st[n] for n in ("k", "v", "k_scale", "v_scale") if n in st}


# ---------------------------------------------------------------------------------------------- the plain forms
def _run_tables(st):
    case = st["case"]
    page, rows, n = case["page"], st["rows"], case["n_seq"]
    ctx, new = st["ctx_len"].long(), st["new_len"].long()
    seq_len = ctx + new
    ends = torch.cumsum(new, 0)
    q_start = torch.cat([torch.zeros_like(ends[:1]), ends])
    had, need = (ctx + page - 1) // page, (seq_len + page - 1) // page
    grown = need - had
    first = torch.cumsum(grown, 0) - grown
    col = torch.arange(st["block_table"].shape[1], device=DEV)[None, :]
    fresh = (col >= had[:, None]) & (col < need[:, None])
    source = (first[:, None] + col - had[:, None]).clamp(0, st["free_pages"].numel() - 1)
    table = torch.where(fresh, st["free_pages"][source], st["block_table"])
    t = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(ends, t, right=True)
    real = seq < n
    seq = torch.where(real, seq, 0)
    pos = torch.where(real, ctx[seq] + t - q_start[seq], -1)
    slot = torch.where(real, table[seq, pos.clamp(min=0) // page].long() * page + pos % page, -1)
    key_row = torch.where(real, seq * st["s_max"] + pos, -1)
    i32 = torch.int32
    return {"seq_len": seq_len.to(i32), "q_start": q_start.to(i32), "q_seq": seq.to(i32), "q_pos": pos.to(i32),
            "slots": slot.to(i32), "key_rows": key_row.to(i32), "pages_used": grown.sum().to(i32).reshape(1),
            "block_table": table}


def _run_append(st):
    case = st["case"]
    n_slots = st["k"].shape[0] * st["k"].shape[1]
    slot = st["slots"].long()
    # the row that every slot of the pool receives (one more, for the rows without a slot)
    row = torch.full((n_slots + 1,), -1, dtype=torch.int64, device=DEV)
    row[torch.where(slot >= 0, slot, n_slots)] = torch.arange(slot.numel(), device=DEV)
    row = row[:n_slots]
    new, row = row >= 0, row.clamp(min=0)
    for name in ("k", "v") if case["values"] else ("k",):
        x = st[name + "_new"].float()
        dst = st[name].view(-1, case["R"], case["d"])
        if case["dst"] == "fp8":
            amax = x.abs().amax(dim=2)
            scale = torch.where(amax > 0, amax / torch.full_like(amax, 448.0), 1.0)
            y = (x / scale[:, :, None]).clamp(-448.0, 448.0).to(F8)
            s = st[name + "_scale"].view(-1, case["R"])
            s.copy_(torch.where(new[:, None], scale[row], s))
            y, dst = y.view(torch.uint8), dst.view(torch.uint8)
        else:
            y = x.to(dst.dtype)
        dst.copy_(torch.where(new[:, None, None], y[row], dst))
    return _held(st)


def _rows_of(st, n, length, name, dt):
    """[length, Hkv, d] rows of sequence n in their order, widened."""
    page = st["case"]["page"]
    ids = st["block_table"][n, :-(-length // page)].long()
    x = st[name][ids].to(dt)
    if name + "_scale" in st:
        x = x * st[name + "_scale"][ids].to(dt)[..., None]
    return x.reshape(-1, *x.shape[2:])[:length]


def _run_paged(st):
    case = st["case"]
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    G = H // Hkv
    out = torch.empty_like(st["q"])
    lse = torch.empty(st["q"].shape[:2], dtype=torch.float32, device=DEV)
    for n, (c, m, t0) in enumerate(zip(st["ctx"], st["new"], st["starts"])):
        length = c + m
        keys, values = _rows_of(st, n, length, "k", torch.float32), _rows_of(st, n, length, "v", torch.float32)
        step = max(1, ROWS_AT_ONCE // (length * G))
        for a in range(t0, t0 + m, step):
            b = min(a + step, t0 + m)
            s = torch.arange(length, device=DEV)[None, :]
            hidden = s > st["q_pos"][a:b, None]
            if st["q_lo"] is not None:
                hidden |= s < st["q_lo"][a:b, None]
            for h in range(Hkv):
                q = st["q"][a:b, h * G:(h + 1) * G].float().reshape(-1, d)
                x = (q @ keys[:, h].t().contiguous()) * d ** -0.5
                x = x.view(b - a, G, length).masked_fill_(hidden[:, None, :], -math.inf)
                top = x.amax(dim=2, keepdim=True)
                p = torch.exp(x.sub_(top))
                total = p.sum(dim=2, keepdim=True)
                o = (p.view(-1, length) @ values[:, h].contiguous()).view(b - a, G, d) / total
                out[a:b, h * G:(h + 1) * G] = o.to(out.dtype)
                lse[a:b, h * G:(h + 1) * G] = (top + torch.log(total))[..., 0]
    return [out, lse] if case["lse"] else [out]


def _run_sparse(st):
    case = st["case"]
    H, Hkv, d, k, page = case["H"], case["Hkv"], case["d"], case["k"], case["page"]
    G = H // Hkv
    T = st["q"].shape[0]
    out = torch.empty_like(st["q"])
    lse = torch.empty(st["q"].shape[:2], dtype=torch.float32, device=DEV)
    step = max(1, ROWS_AT_ONCE // 2 // (k * Hkv * d))
    for a in range(0, T, step):
        b = min(a + step, T)
        ids = st["topk_idx"][a:b].long()
        absent = ids < 0
        ids = ids.clamp(min=0)
        slot = st["block_table"][st["q_seq"][a:b, None].long(), ids // page].long() * page + ids % page
        kv = []
        for name in ("k", "v"):
            x = st[name].view(-1, Hkv, d)
            x = (x.view(torch.uint8)[slot].view(F8) if x.dtype == F8 else x[slot]).float()
            if name + "_scale" in st:
                x = x * st[name + "_scale"].view(-1, Hkv)[slot][..., None]
            kv.append(x.transpose(1, 2).contiguous())                              # [b, Hkv, k, d]
        q = st["q"][a:b].float().view(b - a, Hkv, G, d)
        x = torch.matmul(q, kv[0].transpose(2, 3).contiguous()) * d ** -0.5        # [b, Hkv, G, k]
        x.masked_fill_(absent[:, None, None, :], -math.inf)
        top = x.amax(dim=3, keepdim=True)
        p = torch.exp(x - top)
        total = p.sum(dim=3, keepdim=True)
        out[a:b] = (torch.matmul(p, kv[1]) / total).reshape(b - a, H, d).to(out.dtype)
        lse[a:b] = (top + torch.log(total)).reshape(b - a, H)
    return [out, lse] if case["lse"] else [out]


def run(state):
    if own:
        return _run_own(state)
    return {"tables": _run_tables, "append": _run_append, "paged": _run_paged,
            "sparse": _run_sparse}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions in 64 bits: softmax of the scaled products over the keys that a token sees."""
    op = case["op"]
    if op == "tables":
        return None                                          # whole numbers only
    st = prepare(case, seed)
    st.pop("own", None)
    if op == "append":
        held = _held(st)
        there = st["slots"] >= 0
        at = st["slots"][there].long()
        for name in ("k", "v") if case["values"] else ("k",):
            x = st[name + "_new"][there].double()
            if case["dst"] == "fp8":                         # the numbers that the codes stand for, unrounded
                scale = held[name + "_scale"].double().view(-1, case["R"])
                most = x.abs().max(dim=2).values
                scale[at] = torch.where(most > 0, most / 448, torch.ones_like(most))
                x = x / scale[at][..., None]
                held[name + "_scale"] = scale.view(held[name + "_scale"].shape)
            flat = held[name].double().view(-1, case["R"], case["d"])
            flat[at] = x
            held[name] = flat.view(held[name].shape)
        return held
    H, Hkv, d, page = case["H"], case["Hkv"], case["d"], case["page"]
    G = H // Hkv
    T = st["q"].shape[0]
    out = torch.empty((T, H, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((T, H), dtype=torch.float64, device=DEV)
    for n, (c, m, t0) in enumerate(zip(st["ctx"], st["new"], st["starts"])):
        length = c + m
        for h in range(Hkv):
            ids = st["block_table"][n, :-(-length // page)].long()
            kv = []
            for name in ("k", "v"):
                x = st[name][ids, :, h].double().reshape(-1, d)[:length]
                if name + "_scale" in st:
                    x = x * st[name + "_scale"][ids, :, h].double().reshape(-1, 1)[:length]
                kv.append(x)
            step = max(1, (1 << 28) // ((length if op == "paged" else case["k"] * d) * G))
            for a in range(t0, t0 + m, step):
                b = min(a + step, t0 + m)
                q = st["q"][a:b, h * G:(h + 1) * G].double()
                if op == "paged":
                    s = torch.matmul(q.reshape(-1, d), kv[0].t().contiguous()).view(b - a, G, length) / math.sqrt(d)
                    t = torch.arange(length, device=DEV)
                    seen = t[None, :] <= st["q_pos"][a:b, None]
                    if case["window"]:
                        seen &= t[None, :] > st["q_pos"][a:b, None] - case["window"]
                    s = torch.where(seen[:, None, :], s, -math.inf)
                    p = torch.softmax(s, dim=2)
                    out[a:b, h * G:(h + 1) * G] = torch.matmul(p.view(-1, length), kv[1]).view(b - a, G, d)
                else:
                    picks = st["topk_idx"][a:b].long()
                    kk, vv = kv[0][picks.clamp(min=0)], kv[1][picks.clamp(min=0)]
                    s = (q[:, :, None, :] * kk[:, None]).sum(3) / math.sqrt(d) if G == 1 else \
                        torch.matmul(q, kk.transpose(1, 2).contiguous()) / math.sqrt(d)
                    s = torch.where((picks >= 0)[:, None, :], s, -math.inf)
                    p = torch.softmax(s, dim=2)
                    out[a:b, h * G:(h + 1) * G] = torch.matmul(p, vv)
                lse[a:b, h * G:(h + 1) * G] = torch.logsumexp(s, dim=2)
    return [out, lse] if case["lse"] else [out]
