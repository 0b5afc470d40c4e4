"""harts_gen_cache_write / _read on the GPU: what a cache holds, bit for bit, against the definition in 64 bits on the CPU."""
import pytest
import torch

import paper_2608_28158_b200 as H

pytestmark = pytest.mark.gpu


def quantised(x):
    """(values, biased exponents) of bf16 rows by the definition, in 64 bits: smallest e >= -126 with max |x| <= 448 2^e, x 2^-e rounded to
    4 significant bits (steps of 2^-9 below 2^-6), ties to even."""
    x = x.double()
    bad = ~torch.isfinite(x).all(-1)
    top = torch.where(bad[..., None], torch.zeros_like(x), x).abs().amax(-1)
    e = torch.full(top.shape, -126, dtype=torch.int64)
    for i in range(-126, 128):
        e = torch.where(top > 448 * 2.0 ** i, i + 1, e)
    y = torch.where(bad[..., None], torch.zeros_like(x), x) * (-e[..., None]).double().exp2()
    _, p = torch.frexp(y)
    step = ((p - 1).clamp(min=-6) - 3).double().exp2()
    y = torch.round(y / step) * step
    y = torch.where((e == 120)[..., None], y.clamp(-240, 240), y)          # 256 2^120 would be 2^128
    return y, torch.where(bad, 255, e + 127).to(torch.uint8)


def rows(n, hkv, seed, ld=0):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, hkv, 128, generator=gen) * torch.exp(2 * torch.randn(n, hkv, 1, generator=gen))).to(torch.bfloat16)
    return x


def special(x):
    """Rows of a first token's heads and of some others where the scale can go wrong."""
    flat = x.view(-1, 128)
    values = [0.0, 448.0, 450.0, 2.0 ** -133, 2.0 ** -126, 3.3895e38, 447.0, 1.75, 1.7578125, -1.75 * 2.0 ** 40]
    for i, v in enumerate(values[:len(flat)]):
        flat[i] = flat[i].clamp(-1, 1) * 0 if v == 0 else (flat[i].clamp(-1, 1) * v).to(torch.bfloat16)
        flat[i, 17] = v
    if len(flat) > 13:
        flat[11, 3], flat[12, 127], flat[13, 0] = float("inf"), float("nan"), float("-inf")
    return x


def cache(kind, n_pages, hkv, page):
    k, v = ((torch.randint(0, 256, (n_pages, hkv, page, 128 * (1 if kind == "e4m3" else 2)), dtype=torch.uint8, device="cuda"))
            .view(torch.float8_e4m3fn if kind == "e4m3" else torch.bfloat16) for _ in range(2))
    exps = [torch.randint(1, 250, (n_pages, hkv, page), dtype=torch.uint8, device="cuda") if kind == "e4m3" else None for _ in range(2)]
    return k, v, *exps


def at(t, slot, page):
    return t[slot // page, :, slot % page]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,hkv,page", [(1, 1, 16), (14, 1, 16), (61, 8, 64), (1000, 3, 128), (333, 5, 32)])
def test_written_rows_and_nothing_else(kind, n, hkv, page):
    n_pages = n // page + 3
    c = cache(kind, n_pages, hkv, page)
    before = [None if x is None else x.clone() for x in c]
    x = {s: special(rows(n, hkv, i)) for i, s in enumerate("kv")}
    slot = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(n))[:n].to(torch.int32)
    slot[::7] = -1
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    H.harts_gen_cache_write(x["k"].cuda(), x["v"].cuda(), slot.cuda(), *c, dev_status=status)
    H.harts_la_check(status)
    kept = slot >= 0
    left = torch.ones(n_pages * page, dtype=torch.bool)
    left[slot[kept].long()] = False
    for i, s in enumerate("kv"):
        got, was = c[i].cpu(), before[i].cpu()
        raw = lambda t: t.view(torch.uint8)  # noqa: E731
        assert torch.equal(raw(got).transpose(1, 2).reshape(n_pages * page, -1)[left], raw(was).transpose(1, 2).reshape(n_pages * page, -1)[left])
        if kind == "bf16":
            assert torch.equal(at(raw(got), slot[kept].long(), page), raw(x[s][kept].contiguous()))
        else:
            y, e = quantised(x[s][kept])
            assert torch.equal(at(c[2 + i].cpu(), slot[kept].long(), page), e)
            assert torch.equal(at(raw(got), slot[kept].long(), page).view(torch.float8_e4m3fn).double(), y)
            assert torch.equal(c[2 + i].cpu().transpose(1, 2).reshape(n_pages * page, -1)[left], before[2 + i].cpu().transpose(1, 2).reshape(n_pages * page, -1)[left])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,hkv,page", [(1, 1, 16), (14, 1, 16), (61, 8, 64), (1000, 3, 128)])
def test_read_back(kind, n, hkv, page):
    n_pages = n // page + 3
    c = cache(kind, n_pages, hkv, page)
    x = {s: special(rows(n, hkv, i)) for i, s in enumerate("kv")}
    slot = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(n))[:n].to(torch.int32)
    H.harts_gen_cache_write(x["k"].cuda(), x["v"].cuda(), slot.cuda(), *c)
    slot[::5] = -1
    got = [torch.full((n, hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    H.harts_gen_cache_read(c[0], c[1], slot.cuda(), *got, *c[2:], dev_status=status)
    H.harts_la_check(status)
    for s, y in zip("kv", got):
        ref = x[s].double()
        if kind == "e4m3":
            v, e = quantised(x[s])
            ref = torch.where(e[..., None] == 255, torch.nan, v * (e[..., None].double() - 127).exp2())
        ref[slot < 0] = 0
        assert torch.equal(torch.nan_to_num(y.cpu().double(), nan=12345.0), torch.nan_to_num(ref.to(torch.bfloat16).double(), nan=12345.0))
        fine = torch.isfinite(ref).all(-1, keepdim=True) & (x[s].abs().amax(-1, keepdim=True) > 1e-30)
        if kind == "e4m3":        # a value is off by half a step of its 4 bits, or half the smallest step of the row: 2^-10 of 448
            off = (y.cpu().double() - x[s].double()).abs()
            top = x[s].double().abs().amax(-1, keepdim=True)
            assert bool(((off <= torch.maximum(x[s].double().abs() * 2.0 ** -4, top * 2.0 ** -17)) | ~fine | (slot < 0)[:, None, None]).all())
    only = torch.zeros_like(got[1])
    H.harts_gen_cache_read(c[0], c[1], slot.cuda(), None, only, *c[2:])
    assert torch.equal(only.view(torch.int16), got[1].view(torch.int16))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_slots_beyond_the_cache_are_left_out_and_reported(kind):
    c = cache(kind, 4, 2, 16)
    k, v = rows(3, 2, 0).cuda(), rows(3, 2, 1).cuda()
    for bad in (64, 2 ** 31 - 1):
        status = torch.zeros(2, dtype=torch.int32, device="cuda")
        slot = torch.tensor([5, bad, 63], dtype=torch.int32, device="cuda")
        before = c[0].view(torch.uint8).clone()
        H.harts_gen_cache_write(k, v, slot, *c, dev_status=status)
        with pytest.raises(H.HartsError) as e:
            H.harts_la_check(status)
        assert e.value.code == -1 and int(status[1]) == 1
        other = [s for s in range(64) if s not in (5, 63)]
        flat = lambda t: t.transpose(1, 2).reshape(64, -1)[other]  # noqa: E731
        assert torch.equal(flat(before), flat(c[0].view(torch.uint8)))
        status.zero_()
        y = [torch.full((3, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        H.harts_gen_cache_read(c[0], c[1], slot, *y, *c[2:], dev_status=status)
        assert int(status[1]) == 1 and not y[0][1].any() and not y[1][1].any() and y[0][0].any()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_rows_of_a_wider_tensor_and_another_stream(kind):
    """Keys and values as parts of one projection's output."""
    n, hkv = 77, 4
    qkv = torch.randn(n, 3 * hkv * 128 + 64, device="cuda").to(torch.bfloat16)
    k, v = (qkv[:, 64 + i * hkv * 128:64 + (i + 1) * hkv * 128].view(n, hkv, 128) for i in (0, 2))
    slot = torch.arange(n, dtype=torch.int32, device="cuda")
    a, b = cache(kind, 5, hkv, 32), cache(kind, 5, hkv, 32)
    for x in (*a, *b):
        if x is not None:
            x.view(torch.uint8).zero_()
    H.harts_gen_cache_write(k.contiguous(), v.contiguous(), slot, *a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    H.harts_gen_cache_write(k, v, slot, *b, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


def test_a_large_cache_has_offsets_beyond_32_bits():
    n_pages, hkv, page = 70000, 4, 128                      # 4.6 GB of 8-bit keys
    k_cache = torch.empty(n_pages, hkv, page, 128, dtype=torch.float8_e4m3fn, device="cuda")
    v_cache = torch.empty_like(k_cache)
    exps = [torch.empty(n_pages, hkv, page, dtype=torch.uint8, device="cuda") for _ in range(2)]
    k, v = rows(64, hkv, 0).cuda(), rows(64, hkv, 1).cuda()
    slot = (n_pages * page - 64 + torch.arange(64, device="cuda")).to(torch.int32)
    H.harts_gen_cache_write(k, v, slot, k_cache, v_cache, *exps)
    y, e = quantised(k.cpu())
    assert torch.equal(exps[0][-1, :, -64:].cpu().transpose(0, 1), e)
    assert torch.equal(k_cache[-1, :, -64:].cpu().double().transpose(0, 1), y)
    back = [torch.empty_like(k) for _ in range(2)]
    H.harts_gen_cache_read(k_cache, v_cache, slot, *back, *exps)
    assert torch.equal(back[0].cpu().double(), y * (e[..., None].double() - 127).exp2())
