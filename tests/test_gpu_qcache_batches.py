"""Batches of sequences whose groups of keys are dealt out evenly between workgroups: lengths that make
pieces begin and end everywhere, in front of a sequence's first group too, against the attention in
64 bits over the values that the cache holds."""

import pytest
import torch

from paper_2602_02579_amd import api
from tests.test_gpu_qcache_attn import check, filled, queries, run

pytestmark = pytest.mark.gpu

LENGTHS = [0, 0, 1, 2, 31, 32, 33, 255, 256, 257, 300, 511, 513, 800, 1500, 2700]


@pytest.mark.parametrize("dtype,hq,hkv,d,each", [("bf16", 8, 2, 128, 1), ("bf16", 8, 8, 128, 3),
                                                 ("bf16", 32, 2, 64, 2), ("bf16", 2, 1, 256, 1),
                                                 ("bf16", 4, 4, 96, 1), ("f32", 4, 4, 64, 1),
                                                 ("f32", 4, 1, 256, 2)])
@pytest.mark.parametrize("n_seq", [2, 3, 5, 9, 17, 40, 70])
def test_lengths_of_all_kinds(gpu_device, dtype, hq, hkv, d, each, n_seq):
    cfg = api.LayerCfg(hq, hkv, d, 64, 1e4, dtype)
    gen = torch.Generator().manual_seed(n_seq + d)
    lens = [LENGTHS[i] for i in torch.randint(len(LENGTHS), (n_seq,), generator=gen).tolist()]
    cache, values = filled(cfg, max(1, sum(lens)), gpu_device)
    start = torch.tensor([sum(lens[:i]) for i in range(n_seq)], dtype=torch.int32,
                         device=gpu_device)
    n = torch.tensor(lens, dtype=torch.int32, device=gpu_device)[:, None]
    pos = (n - each + torch.arange(each, dtype=torch.int32, device=gpu_device)).flatten()
    q = queries(cfg, n_seq * each, gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, n_seq), start, n_seq)


@pytest.mark.parametrize("lens", [[256] * 33, [257] * 31, [1] * 64, [5000, 1, 1, 1], [1, 1, 1, 5000],
                                  [0, 0, 3000, 0, 0], [0] * 5, [768] * 10 + [0] * 10])
def test_even_and_lopsided_batches(gpu_device, lens):
    cfg = api.LayerCfg(8, 8, 128, 64, 1e4, "bf16")
    cache, values = filled(cfg, max(1, sum(lens)), gpu_device)
    start = torch.tensor([sum(lens[:i]) for i in range(len(lens))], dtype=torch.int32,
                         device=gpu_device)
    pos = torch.tensor(lens, dtype=torch.int32, device=gpu_device) - 1
    q = queries(cfg, len(lens), gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, len(lens)), start, len(lens))


def test_beginnings_outside_of_the_cache_count_as_its_ends(gpu_device):
    cfg = api.LayerCfg(4, 2, 128, 64, 1e4, "bf16")
    cache, values = filled(cfg, 640, gpu_device)
    start = torch.tensor([-5, -2 ** 31, 640, 2 ** 31 - 1], dtype=torch.int32, device=gpu_device)
    pos = torch.tensor([300, 639, 10, 10], dtype=torch.int32, device=gpu_device)
    q = queries(cfg, 4, gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, 4), start, 4)
    got = run(cfg, q[:1].contiguous(), cache, pos[:1], start[:1])
    check(cfg, q[:1], cache, values, pos[:1], got, start[:1])
