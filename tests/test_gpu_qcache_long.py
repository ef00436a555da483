"""Attention over a cache in 4 bits with several steps a workgroup and many parts a row: for every head some
keys that outweigh the others, spread over all tiles, so that a tile which is lost, or counted twice,
is off by far more than the tolerance."""

import pytest
import torch

from paper_2602_02579_amd import api
from tests import attention64 as A
from tests.test_gpu_qcache_attn import DT, check, queries, run

pytestmark = pytest.mark.gpu

PLANTED = 48    # keys a head; each has a weight of some 2 %


def problem(cfg, rows, m, device, seed):
    gen = torch.Generator(device=device).manual_seed(seed)
    q = queries(cfg, m, device, seed=seed)
    cache = api.QCache.empty(cfg, rows, device)
    k, v = (torch.randn((cache.rows, cfg.n_kv_heads, cfg.head_dim), generator=gen, device=device)
            for _ in range(2))
    group = cfg.n_q_heads // cfg.n_kv_heads
    strong = torch.log(torch.tensor(float(rows))) + 3      # their scores
    for h in range(cfg.n_q_heads):
        i = h % m                       # for one of the rows
        at = torch.randint(0, rows, (PLANTED,), generator=gen, device=device)
        at[:2] = torch.tensor([max(0, rows - 1 - 31 * (h % 9)), 33 * (h % 9) % rows], device=device)
        d = q[i, h].float()
        k[at, h // group] = d * strong.to(device) * cfg.head_dim ** 0.5 / d.square().sum()
    api.pkv_qcache_store(cfg, k.to(DT[cfg.dtype]), v.to(DT[cfg.dtype]), cache)
    return q, cache, A.stored(cache, torch.arange(cache.rows, device=device))


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 40, 2, 128), ("bf16", 8, 2, 64),
                                           ("bf16", 40, 2, 64), ("bf16", 6, 2, 96), ("bf16", 40, 2, 112),
                                           ("bf16", 4, 1, 256), ("bf16", 4, 1, 208), ("f32", 4, 4, 64),
                                           ("f32", 8, 2, 128), ("f32", 2, 1, 256), ("f32", 3, 1, 48),
                                           ("f32", 3, 1, 176)])
@pytest.mark.parametrize("rows", [800, 1100, 1537, 2040])
@pytest.mark.parametrize("m", [1, 3])
def test_one_workgroup_of_several_steps(gpu_device, dtype, hq, hkv, d, rows, m):
    cfg = api.LayerCfg(hq, hkv, d, 64, 1e4, dtype)
    q, cache, values = problem(cfg, rows, m, gpu_device, seed=rows + d)
    pos = torch.full((m,), rows - 1, dtype=torch.int32, device=gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos))
    start = torch.full((1,), 45, dtype=torch.int32, device=gpu_device)
    check(cfg, q, cache, values, pos - 45, run(cfg, q, cache, pos - 45, start), start)


@pytest.mark.parametrize("dtype,hq,hkv,d,rows", [
    ("bf16", 32, 8, 128, 40000), ("bf16", 4, 1, 128, 20000), ("bf16", 4, 1, 128, 70000),
    ("bf16", 8, 2, 128, 70000), ("bf16", 40, 2, 128, 30000), ("bf16", 4, 1, 64, 70000),
    ("bf16", 40, 2, 64, 20000), ("bf16", 2, 1, 80, 30000), ("bf16", 2, 1, 256, 30000), ("f32", 4, 1, 64, 40000),
    ("f32", 8, 2, 128, 20000), ("f32", 2, 1, 256, 20000), ("f32", 2, 1, 48, 70000)])
def test_many_parts_and_steps(gpu_device, dtype, hq, hkv, d, rows):
    cfg = api.LayerCfg(hq, hkv, d, 64, 1e4, dtype)
    q, cache, values = problem(cfg, rows, 1, gpu_device, seed=d)
    for last in (rows - 1, rows // 2 + 77):
        pos = torch.tensor([last], dtype=torch.int32, device=gpu_device)
        check(cfg, q, cache, values, pos, run(cfg, q, cache, pos))
    q = torch.cat((q, q, q, q))      # a sequence and its parts
    start = torch.tensor([0, rows // 3, rows - 900, 5], dtype=torch.int32, device=gpu_device)
    pos = torch.tensor([rows - 1, rows // 2, 899, rows // 4], dtype=torch.int32, device=gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, 4), start, 4)
