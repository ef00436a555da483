"""Keys and values into a cache in 4 bits and back: every value is the nearest one of the format, for
all bf16 bit patterns, on the middles of neighbouring values and at both ends of the scale; rows
that are left alone; and the way back with and without positions."""

import numpy as np
import pytest
import torch

from paper_2602_02579_amd import api
from tests import attention64 as A

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def cfg(dtype, hkv, d, theta=1e4):
    return api.LayerCfg(2 * hkv, hkv, d, 64, theta, dtype)


def indices(cache):
    """Indices [Hkv, rows, D] and scale bytes [Hkv, rows, D / 16] of keys and of values."""
    t = {n: x.cpu().numpy() for n, x in cache.tensors.items()}
    vs = t["v_scales"].transpose(0, 1, 3, 2).reshape(t["k_scales"].shape)
    return [(np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1), s)
            for c, s in ((t["k_codes"], t["k_scales"]), (t["v_codes"], vs))]


def hard_values(dtype):
    """All bf16 patterns, every middle of two values at many scales with its neighbours, and blocks at the
    ends of the range; [n, 1, 16]."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(torch.bfloat16).float()
    order = torch.randperm(65536, generator=torch.Generator().manual_seed(3))
    parts = [bits.view(-1, 16), bits[order].view(-1, 16)]
    mid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5])
    eps = torch.finfo(DT[dtype]).eps
    for e in (-130, -97, -96, -95, -94, -40, 0, 1, 60, 120, 122, 123, 124, 125):
        for lead in (4.0, 6.0, 6.9, 6.9921875, 7.0, 7.5):
            for near in (1.0, 1 - eps / 2, 1 + eps):
                b = torch.cat((mid * near, -mid * near))
                b[15] = lead
                parts.append(torch.ldexp(b, torch.tensor(e)).unsqueeze(0))
    parts.append(torch.zeros(1, 16))
    parts.append(-torch.zeros(1, 16))
    return torch.cat(parts).to(DT[dtype]).unsqueeze(1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_element_becomes_the_nearest_value(gpu_device, dtype):
    x = hard_values(dtype)
    n = x.shape[0]
    c = cfg(dtype, 1, 16)
    cache = api.QCache.empty(c, n, gpu_device)
    dev = x.to(gpu_device)
    api.pkv_qcache_store(c, dev, dev.flip(0).contiguous(), cache)
    want, byte = A.encode(x.double().numpy()[:, 0])
    for (got, scales), w, b in zip(indices(cache), (want, want[::-1]), (byte, byte[::-1])):
        assert np.array_equal(scales[0, :n], b)
        nan = np.repeat(b == 255, 16, -1)
        assert np.array_equal(np.where(nan, 0, got[0, :n]), np.where(nan, 0, w))
    back = torch.empty_like(dev), torch.empty_like(dev)
    api.pkv_qcache_restore(c, cache, *back, rotate=False)
    for y, w, b in zip(back, (want, want[::-1]), (byte, byte[::-1])):
        np.testing.assert_array_equal(y[:, 0].cpu().double().numpy(), A.decode(w, b))


@pytest.mark.parametrize("dtype,hkv,d,n", [("bf16", 8, 128, 1000), ("f32", 4, 64, 333),
                                           ("bf16", 3, 48, 77), ("f32", 1, 16, 1),
                                           ("bf16", 2, 256, 65), ("f32", 5, 112, 31)])
def test_rows_go_where_they_are_sent(gpu_device, dtype, hkv, d, n):
    gen = torch.Generator(device=gpu_device).manual_seed(n)
    c = cfg(dtype, hkv, d)
    k, v = (torch.randn((n, hkv, d), generator=gen, device=gpu_device).to(DT[dtype])
            for _ in range(2))
    cache = api.QCache.empty(c, 2 * n + 40, gpu_device)
    rows = cache.rows
    for t in cache.tensors.values():
        t.random_(0, 256, generator=gen)
    before = {name: t.clone() for name, t in cache.tensors.items()}
    dst = torch.randperm(rows, generator=gen, device=gpu_device)[:n].int()
    outside = dst.clone()
    outside[::5] = torch.where(outside[::5] % 2 == 0, -1 - outside[::5], rows + outside[::5])
    kept = (outside >= 0) & (outside < rows)
    api.pkv_qcache_store(c, k, v, cache, outside)
    for (got, scales), x in zip(indices(cache), (k, v)):
        want, byte = A.encode(x.cpu().double().numpy())
        at, i = outside[kept].cpu().numpy(), kept.cpu().numpy()
        assert np.array_equal(got[:, at], want[i].transpose(1, 0, 2))
        assert np.array_equal(scales[:, at], byte[i].transpose(1, 0, 2))
    for name, t in cache.tensors.items():          # no other row is touched
        other = torch.ones(rows, dtype=torch.bool, device=gpu_device)
        other[outside[kept].long()] = False
        if name == "v_scales":
            t, was = (x.transpose(2, 3).reshape(hkv, rows, -1) for x in (t, before[name]))
        else:
            was = before[name]
        assert torch.equal(t[:, other], was[:, other])


def turned(x, pos, theta):
    half = x.shape[-1] // 2
    freq = float(np.float32(theta)) ** (-torch.arange(half, dtype=torch.float64, device=x.device) / half)
    a = (pos.double()[:, None] * freq)[:, None]
    return torch.cat((x[..., :half] * a.cos() - x[..., half:] * a.sin(),
                      x[..., half:] * a.cos() + x[..., :half] * a.sin()), -1)


@pytest.mark.parametrize("dtype,hkv,d,stored,m", [
    ("bf16", 8, 128, 4096, 1500), ("f32", 4, 64, 700, 700), ("bf16", 1, 16, 32, 1),
    ("bf16", 2, 48, 100, 201), ("f32", 3, 256, 64, 65), ("bf16", 5, 80, 96, 33)])
@pytest.mark.parametrize("given", ["rows and positions", "positions", "neither", "unturned"])
def test_rows_come_back(gpu_device, dtype, hkv, d, stored, m, given):
    gen = torch.Generator(device=gpu_device).manual_seed(7)
    c = cfg(dtype, hkv, d, 5e5)
    cache = api.QCache.empty(c, stored, gpu_device)
    new = lambda n: torch.randn((n, hkv, d), generator=gen, device=gpu_device).to(DT[dtype])  # noqa: E731
    api.pkv_qcache_store(c, new(stored), new(stored), cache)
    if given != "rows and positions":
        m = min(m, cache.rows)
    rows = torch.arange(m, device=gpu_device)
    pos = torch.arange(m, device=gpu_device) + (3 if given == "neither" else 0)
    kw = {} if given == "unturned" else dict(pos_base=3)
    if given == "rows and positions":      # any order, some twice, one outside
        rows = torch.randint(0, stored, (m,), generator=gen, device=gpu_device)
        rows[0] = stored if stored == cache.rows else -7
        kw["row_idx"] = rows.int()
    if given in ("rows and positions", "positions"):
        pos = torch.randint(-1000, 300000, (m,), generator=gen, device=gpu_device)
        kw["pos"] = pos.int()
    out = [torch.full((m, hkv, d), 9.0, dtype=DT[dtype], device=gpu_device) for _ in range(2)]
    api.pkv_qcache_restore(c, cache, *out, rotate=given != "unturned", **kw)
    inside = (rows >= 0) & (rows < cache.rows)
    k, v = A.stored(cache, rows.clamp(0, cache.rows - 1))
    if given != "unturned":
        k = turned(k, pos, 5e5)
    k[~inside], v[~inside] = 9.0, 9.0
    assert torch.equal(out[1].double(), v)
    if given == "unturned":
        assert torch.equal(out[0].double(), k)
    # one rounding; cosine, sine and the reduced angle (up to pi) in fp32: 8 half steps of the pair
    pair = torch.hypot(k[..., :d // 2], k[..., d // 2:]).repeat(1, 1, 2)
    tol = A.HALF_STEP[dtype] * k.abs() + 8 * 2.0 ** -24 * pair
    assert ((out[0].double() - k).abs() <= tol).all()


def test_no_rows_are_no_work(gpu_device):
    c = cfg("bf16", 2, 64)
    cache = api.QCache.empty(c, 32, gpu_device)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=gpu_device)
    api.pkv_qcache_store(c, none, none, cache)
    api.pkv_qcache_restore(c, cache, none, none)
    assert all(int(t.sum()) == 0 for t in cache.tensors.values())
