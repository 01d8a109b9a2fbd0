"""GPU tests of the paged 4-bit cache: written values against the format's
definition bit by bit, the layout of fgd.h byte by byte, and slots outside the
cache, of pages in any order, and past 4 GiB."""

import numpy as np
import pytest

from oracle import attention as ref
from oracle import operators

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    import paper_2606_22768_amd as fgd

    return fgd, torch


def _np(t):
    return t.detach().double().cpu().numpy()


def _heads(torch, T, H, D, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, H, D), generator=g) * torch.exp(3 * torch.randn((T, H, D // 32, 1), generator=g)).expand(
        -1, -1, -1, 32).reshape(T, H, D)
    return x.to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).cuda()


def _same(got, want):
    got = _np(got)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.nan_to_num(got, nan=7.0), np.nan_to_num(want, nan=7.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H, D, page, T", [(1, 32, 16, 1), (2, 64, 16, 50), (3, 96, 32, 33), (8, 128, 64, 200),
                                           (1, 160, 128, 17), (5, 192, 16, 16), (2, 224, 256, 100), (4, 256, 16, 31)])
def test_written_values(env, H, D, page, T, dtype):
    fgd, torch = env
    k, v = _heads(torch, T, H, D, dtype, 1), _heads(torch, T, H, D, dtype, 2)
    k[0, 0, :32] = 0
    k[T // 2, 0, 5] = float("inf")
    v[T // 2, 0, 31] = float("nan")
    v[T - 1] *= 1e-38
    pages = -(-T // page) + 2
    cache = fgd.Mx4Cache(pages, page, H, D)
    cache.data.fill_(0xA5)
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(T))[:T].cuda()
    fgd.mx4_cache_write(cache, k, v, slots)
    for out in ("f32", "bf16"):
        got = fgd.mx4_cache_read(cache, slots, out)
        _same(got[0], ref.cached(_np(k)))
        _same(got[1], ref.cached(_np(v)))
    # Bytes of other slots are as they were.
    others = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    others[slots] = False
    codes = _decode(cache.data.cpu().numpy(), pages, page, H, D)
    for part in codes:
        assert (part[others.cpu().numpy()] == 0xA5).all()


def _decode(data, pages, page, H, D):
    """(keys' codes, values' codes, keys' scales, values' scales) by slot, as
    fgd.h lays them out: bytes [slots][H][..], codes two to a byte."""
    NB, G = D // 32, page // 16
    d = data.reshape(pages, H, G, 17 * D)
    kc, vc = np.zeros((2, pages, page, H, D // 2), np.uint8)
    ks, vs = np.zeros((2, pages, page, H, NB), np.uint8)
    for t in range(page):
        g, i = d[:, :, t // 16], t % 16
        for e in range(0, D, 2):
            h, j = divmod(e, D // 4)
            kc[:, t, :, e // 2] = g[..., (i + 16 * h) * (D // 8) + j // 2]
            b, n = e // 32, e % 32 // 2
            vc[:, t, :, e // 2] = g[..., 8 * D + (n + 16 * (i // 4)) * (D // 8) + 4 * b + i % 4]
        for b in range(NB):
            ks[:, t, :, b] = g[..., 16 * D + i * NB + b]
            vs[:, t, :, b] = g[..., 16 * D + D // 2 + i // 4 * 4 * NB + 4 * b + i % 4]
    return [a.reshape(pages * page, H, -1) for a in (kc, vc, ks, vs)]


@pytest.mark.parametrize("D", [32, 96, 128, 256])
def test_layout(env, D):
    fgd, torch = env
    H, page, pages = 2, 32, 3
    k, v = _heads(torch, pages * page, H, D, "f32", 3), _heads(torch, pages * page, H, D, "f32", 4)
    cache = fgd.Mx4Cache(pages, page, H, D)
    fgd.mx4_cache_write(cache, k, v, torch.arange(pages * page, device="cuda"))
    codes = _decode(cache.data.cpu().numpy(), pages, page, H, D)
    for x, c, s in ((k, codes[0], codes[2]), (v, codes[1], codes[3])):
        assert np.array_equal(s, operators.mx4_scale_bytes(_np(x)))
        want = operators.GRID[np.stack((c & 7, c >> 4 & 7), -1).reshape(*c.shape[:-1], D)]
        assert np.array_equal(want * np.repeat(np.ldexp(1.0, s.astype(int) - 127), 32, -1), abs(ref.cached(_np(x))))


@pytest.mark.parametrize("run", [1, 3, 4, 15, 64])
@pytest.mark.parametrize("first", [0, 1, 2, 13])
def test_runs_of_slots(env, run, first):
    # Prompts are written as runs of neighbouring slots from anywhere in a page.
    fgd, torch = env
    H, D, page = 3, 128, 16
    T = 5 * run
    k, v = _heads(torch, T, H, D, "bf16", run), _heads(torch, T, H, D, "bf16", first)
    each = -(-(run + first) // page)
    cache = fgd.Mx4Cache(5 * each, page, H, D)
    cache.data.fill_(0x5A)
    order = torch.randperm(5 * each)
    at = torch.cat([i * each * page + first + torch.arange(run) for i in range(5)])
    slots = (order[at // page] * page + at % page).cuda()
    fgd.mx4_cache_write(cache, k, v, slots)
    got = fgd.mx4_cache_read(cache, slots)
    _same(got[0], ref.cached(_np(k)))
    _same(got[1], ref.cached(_np(v)))
    others = np.ones(5 * each * page, bool)
    others[slots.cpu().numpy()] = False
    for part in _decode(cache.data.cpu().numpy(), 5 * each, page, H, D):
        assert (part[others] == 0x5A).all()


def test_slots_outside_the_cache(env):
    fgd, torch = env
    cache = fgd.Mx4Cache(2, 16, 2, 64)
    cache.data.fill_(0xA5)
    k = _heads(torch, 6, 2, 64, "f32")
    fgd.mx4_cache_write(cache, k, k, torch.tensor([-1, 32, -2 ** 62, 2 ** 62, 33, -33], device="cuda"))
    assert (cache.data == 0xA5).all()
    slots = torch.tensor([3, -1, 31, 32, 2 ** 40, 8], device="cuda")
    fgd.mx4_cache_write(cache, k, k, slots)
    got = fgd.mx4_cache_read(cache, slots)
    want = ref.cached(_np(k))
    want[[1, 3, 4]] = 0
    _same(got[0], want)
    _same(got[1], want)
    empty = fgd.Mx4Cache(0, 16, 2, 64)
    fgd.mx4_cache_write(empty, k, k, slots)
    assert (fgd.mx4_cache_read(empty, slots)[0] == 0).all()
    none = slots[:0]
    fgd.mx4_cache_write(cache, k[:0], k[:0], none)
    assert fgd.mx4_cache_read(cache, none)[0].shape == (0, 2, 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_and_unaligned_heads(env, dtype):
    fgd, torch = env
    T, H, D = 21, 2, 96
    k, v = _heads(torch, T, H, D, dtype, 5), _heads(torch, T, H, D, dtype, 6)
    wide = torch.zeros((T, 2 * H * D + 3), dtype=k.dtype, device="cuda")
    wide[:, 1:1 + H * D] = k.flatten(1)
    wide[:, 2 + H * D:2 + 2 * H * D] = v.flatten(1)
    slots = torch.arange(T, device="cuda")
    a, b = fgd.Mx4Cache(2, 16, H, D), fgd.Mx4Cache(2, 16, H, D)
    a.data.zero_()
    b.data.zero_()
    fgd.mx4_cache_write(a, k, v, slots)
    fgd.mx4_cache_write(b, wide[:, 1:1 + H * D].unflatten(1, (H, D)),
                        wide[:, 2 + H * D:2 + 2 * H * D].unflatten(1, (H, D)), slots)
    assert torch.equal(a.data, b.data)
    swapped = k.transpose(0, 1).contiguous().transpose(0, 1)
    b.data.zero_()
    fgd.mx4_cache_write(b, swapped, v, slots)
    assert torch.equal(a.data, b.data)


def test_past_four_gigabytes(env):
    fgd, torch = env
    cache = fgd.Mx4Cache(70_000, 64, 8, 128)  # 4.9 GB
    assert cache.nbytes > 2 ** 32 + 2 ** 29
    k, v = _heads(torch, 6, 8, 128, "bf16", 7), _heads(torch, 6, 8, 128, "bf16", 8)
    slots = torch.tensor([0, 63, 61_681 * 64 - 1, 61_681 * 64 + 5, 70_000 * 64 - 1, 70_000 * 64 - 17], device="cuda")
    fgd.mx4_cache_write(cache, k, v, slots)
    got = fgd.mx4_cache_read(cache, slots)
    _same(got[0], ref.cached(_np(k)))
    _same(got[1], ref.cached(_np(v)))
    # Attention reads there too: each of three sequences has one of the pages.
    q = torch.randn((3, 8, 128), device="cuda")
    for i, page in ((3, 61_681), (5, 69_999)):
        table = torch.full((3, 1), page, dtype=torch.int32, device="cuda")
        at = int(slots[i]) % 64
        fill = page * 64 + torch.arange(at, device="cuda")
        zeros = torch.zeros((at, 8, 128), device="cuda")
        fgd.mx4_cache_write(cache, zeros, zeros, fill)
        out = fgd.mx4_attend(q, cache, table, torch.full((3,), at + 1, dtype=torch.int32, device="cuda"), window=1)
        assert np.array_equal(_np(out), np.broadcast_to(ref.cached(_np(v))[i], (3, 8, 128)))
    del cache


def test_kept_data_and_streams(env):
    fgd, torch = env
    cache = fgd.Mx4Cache(4, 16, 2, 64)
    k = _heads(torch, 9, 2, 64, "f32")
    slots = torch.arange(9, device="cuda") * 5
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    fgd.mx4_cache_write(cache, k, k, slots, stream=s)
    got = fgd.mx4_cache_read(cache, slots, stream=s)
    s.synchronize()
    _same(got[0], ref.cached(_np(k)))
    again = fgd.Mx4Cache(4, 16, 2, 64, data=cache.data.clone())
    assert torch.equal(fgd.mx4_cache_read(again, slots)[0], got[0])


def test_data_on_the_current_gpu(env):
    fgd, torch = env
    data = torch.empty(fgd.Mx4Cache(3, 16, 2, 64).nbytes, dtype=torch.uint8, device="cuda")
    k = _heads(torch, 5, 2, 64, "f32")
    slots = torch.arange(5, device="cuda") * 7
    for device in ("cuda", "cuda:0", torch.device("cuda")):
        cache = fgd.Mx4Cache(3, 16, 2, 64, device=device, data=data)
        fgd.mx4_cache_write(cache, k, k, slots)
        _same(fgd.mx4_cache_read(cache, slots)[0], ref.cached(_np(k)))
    for device in ("cpu", "cuda:1"):
        with pytest.raises(ValueError, match="data: expected a tensor on"):
            fgd.Mx4Cache(3, 16, 2, 64, device=device, data=data)
