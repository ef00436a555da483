"""Attention over a cache in 4 bits whose values reach the end of the format's range: sums of them stay finite
where the result is, whenever a wave meets the first of them, and smaller values beside them keep
their accuracy."""

import pytest
import torch

from paper_2602_02579_amd import api
from tests import attention64 as A
from tests.test_gpu_qcache_attn import DT, check, queries, run

pytestmark = pytest.mark.gpu

MOST = 1.5 * 2.0 ** 127      # the largest that the format holds: 6 * 2^125


def stored_values(cfg, rows, device, large, grow=False):
    """Rows of normal values, of which those of ``large`` (row, factor) have every second block of 16 elements
    at the end of the range times factor, all of one sign; ``grow``: keys that grow along the rows."""
    gen = torch.Generator(device=device).manual_seed(rows)
    cache = api.QCache.empty(cfg, rows, device)
    k, v = (torch.randn((cache.rows, cfg.n_kv_heads, cfg.head_dim), generator=gen, device=device)
            for _ in range(2))
    if grow:
        k = k.abs() * torch.linspace(0.01, 6, cache.rows, device=device)[:, None, None]
    for rows_of, factor in large:
        even = torch.arange(cfg.head_dim, device=device) % 32 < 16
        v[rows_of] = torch.where(even, MOST * factor, v[rows_of])
    api.pkv_qcache_store(cfg, k.to(DT[cfg.dtype]), v.to(DT[cfg.dtype]), cache)
    return cache, A.stored(cache, torch.arange(cache.rows, device=device))


PLACES = {"all": [(slice(None), 1.0)], "first": [(slice(0, 40), 1.0)], "last": [(slice(-40, None), 1.0)],
          "one": [(slice(900, 901), 1.0)], "both signs": [(slice(0, 300), -1.0), (slice(600, None), 1.0)],
          "near 2^65": [(slice(0, 500), 2.0 ** -62), (slice(500, None), 2.0 ** -64)]}


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 8, 128), ("bf16", 8, 2, 64), ("bf16", 40, 1, 128),
                                           ("bf16", 6, 2, 48), ("bf16", 4, 1, 256), ("f32", 4, 4, 64),
                                           ("f32", 8, 2, 128), ("f32", 3, 1, 96), ("f32", 2, 1, 256)])
@pytest.mark.parametrize("place", PLACES)
def test_large_values(gpu_device, dtype, hq, hkv, d, place):
    cfg = api.LayerCfg(hq, hkv, d, 64, 1e4, dtype)
    for rows, grow in ((1100, False), (4100, False), (4100, True)):
        cache, values = stored_values(cfg, rows, gpu_device, PLACES[place], grow)
        q = queries(cfg, 1, gpu_device)
        q = q.abs() if grow else q
        pos = torch.tensor([cache.rows - 1], dtype=torch.int32, device=gpu_device)
        check(cfg, q, cache, values, pos, run(cfg, q, cache, pos))
        n = 5
        start = torch.tensor([0, 300, 890, 17, 2000 % cache.rows], dtype=torch.int32, device=gpu_device)
        pos = torch.tensor([700, 900, 40, -1, 3000, 2, 1100, 63, -1, 0], dtype=torch.int32,
                           device=gpu_device)
        q = queries(cfg, 2 * n, gpu_device)
        check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, n), start, n)
