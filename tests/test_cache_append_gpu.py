"""hisa_cache_append: every slot holds its row converted, every other byte of the cache is what it was."""
import numpy as np
import pytest
import torch

from paper_2603_28458_amd import hisa

pytestmark = pytest.mark.gpu
CODE = {"f32": hisa.HISA_F32, "bf16": hisa.HISA_BF16, "fp8": hisa.HISA_FP8_E4M3}
STORE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}
PAIRS = [("f32", "f32"), ("f32", "bf16"), ("f32", "fp8"), ("bf16", "bf16"), ("bf16", "fp8")]


def quantised(x):
    """Codes (bytes) and scales by correctly rounded fp32 divisions, on the CPU."""
    finite = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).amax(dim=-1)
    scale = torch.where(finite > 0, torch.maximum(finite / torch.tensor(448.0), torch.tensor(2.0 ** -126)), torch.tensor(1.0))
    y = torch.where(x.isfinite(), (x / scale[..., None]).clamp(-448, 448), torch.tensor(float("nan")))
    return y.to(torch.float8_e4m3fn).view(torch.uint8), scale


def run(T, R, d, src, dst, page=16, n_pages=None, layout="token", values=True, special=False, apart=0, seed=0):
    g = torch.Generator().manual_seed(seed)
    n_pages = n_pages or -(-T // page) + 2
    dev = torch.device("cuda:0")
    print(f"\n[append] T={T} R={R} d={d} {src}->{dst} page={page} {layout}", flush=True)
    slots = torch.randperm(n_pages * page, generator=g)[:T].to(torch.int32)
    if T > 2:
        slots[1] = -1
    if T > 5:
        slots[4] = n_pages * page
    new = {}
    for name in ("k", "v") if values else ("k",):
        x = torch.randn((T, R, d), generator=g) * (10.0 ** torch.randint(-3, 4, (T, R, 1), generator=g))
        if special:
            x[0] = 0.0
            x[T // 2, :, 0] = float("inf")
            x[T // 2, :, 1] = float("nan")
            x[T // 3] = 1e-41
            x[T - 1, :, :] = -448.0 * 3.5
        new[name] = x.to(torch.float32 if src == "f32" else torch.bfloat16)
    fill = {n: torch.randint(0, 120, (n_pages, page, R, d), generator=g).to(STORE[dst]) for n in new}
    sfill = {n: torch.rand((n_pages, page, R), generator=g) for n in new}
    if layout == "head":
        arr = {n: fill[n].permute(0, 2, 1, 3).contiguous().to(dev).permute(0, 2, 1, 3) for n in new}
    elif layout == "apart":
        both = torch.full((n_pages, 2, page, R, d + 16), 3, dtype=STORE[dst], device=dev)
        arr = {n: both[:, i, :, :, :d] for i, n in enumerate(new)}
        for n in new:
            arr[n].copy_(fill[n])
    else:
        arr = {n: fill[n].to(dev) for n in new}
    sc = {n: sfill[n].to(dev) for n in new}
    cache = hisa.Cache(k=arr["k"], v=arr.get("v"), dtype=CODE[dst], k_scale=sc["k"] if dst == "fp8" else None,
                       v_scale=sc.get("v") if dst == "fp8" else None)
    dnew = {}
    for n, x in new.items():
        if apart:
            wide = torch.zeros((T, R * d + apart), dtype=x.dtype, device=dev)
            wide[:, :R * d] = x.reshape(T, R * d).to(dev)
            dnew[n] = wide[:, :R * d].view(T, R, d)
        else:
            dnew[n] = x.to(dev)
    hisa.hisa_cache_append(cache, slots.to(dev), dnew["k"], dnew.get("v"))
    torch.cuda.synchronize()
    ok = (slots >= 0) & (slots < n_pages * page)
    at = slots[ok].long()
    for n, x in new.items():
        want, swant = fill[n].clone().view(-1, R, d), sfill[n].clone().view(-1, R)
        if dst == "fp8":
            codes, scale = quantised(x.float())
            want[at], swant[at] = codes[ok], scale[ok]
        else:
            want[at] = x.to(STORE[dst])[ok]
        got = arr[n].cpu().contiguous().view(-1, R, d)
        bits = torch.uint8 if dst == "fp8" else torch.int16 if dst == "bf16" else torch.int32
        same = (got.view(bits) == want.view(bits)) | (got.float().isnan() & want.float().isnan() & (dst != "fp8"))
        assert same.all(), (n, int((~same).sum()))
        assert torch.equal(sc[n].cpu().view(-1, R), swant)
    if layout == "apart":
        assert (both[:, :, :, :, d:] == 3).all()


@pytest.mark.parametrize("src,dst", PAIRS)
@pytest.mark.parametrize("T,R,d", [(1, 1, 8), (1, 4, 128), (3, 1, 64), (37, 5, 24), (200, 8, 128), (65, 3, 256), (9, 2, 512),
                                   (1025, 1, 128), (70, 7, 72)])
def test_shapes(src, dst, T, R, d):
    run(T, R, d, src, dst, seed=T + d)


@pytest.mark.parametrize("src,dst", PAIRS)
@pytest.mark.parametrize("layout", ["token", "head", "apart"])
@pytest.mark.parametrize("page", [1, 7, 64])
def test_layouts(src, dst, layout, page):
    run(50, 4, 128, src, dst, page=page, layout=layout, apart=48, seed=page)


@pytest.mark.parametrize("src,dst", PAIRS)
def test_special_values(src, dst):
    run(40, 3, 64, src, dst, special=True, seed=1)


@pytest.mark.parametrize("src,dst", PAIRS)
def test_keys_alone(src, dst):
    run(77, 1, 128, src, dst, page=500, n_pages=3, values=False)


def test_offsets_beyond_32_bits():
    dev = torch.device("cuda:0")
    n_pages, page, d = 1 << 17, 64, 512                            # 4 Gi elements
    k = torch.zeros((n_pages, page, 1, d), dtype=torch.bfloat16, device=dev)
    cache = hisa.Cache(k=k, v=None, dtype=hisa.HISA_BF16)
    slots = torch.tensor([n_pages * page - 1, 5, n_pages * page - 70], dtype=torch.int32, device=dev)
    x = torch.randn((3, 1, d), device=dev).bfloat16()
    hisa.hisa_cache_append(cache, slots, x)
    assert torch.equal(k.view(-1, 1, d)[slots.long()], x)
    assert int((k.view(-1, d)[::1].abs().amax(dim=1) > 0).sum()) == 3


def test_no_rows_is_no_launch():
    dev = torch.device("cuda:0")
    k = torch.zeros((2, 4, 1, 8), device=dev)
    hisa.hisa_cache_append(hisa.Cache(k=k, v=None, dtype=hisa.HISA_F32), torch.empty(0, dtype=torch.int32, device=dev),
                           torch.empty((0, 1, 8), device=dev))
    assert (k == 0).all()
