"""Attention over a cache held in 4 bits against the attention in 64 bits over the values that it
stands for: one sequence and batches, one row and many, sequences that begin anywhere, share rows,
are empty or reach the end of the cache, and what lies in rows that nobody attends."""

import pytest
import torch

from paper_2602_02579_amd import api
from tests import attention64 as A

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def filled(cfg, rows, device, seed=0, spread=1.0):
    """A cache full of stored rows and the values that it holds."""
    gen = torch.Generator(device=device).manual_seed(seed)
    cache = api.QCache.empty(cfg, rows, device)
    k, v = (torch.randn((cache.rows, cfg.n_kv_heads, cfg.head_dim), generator=gen,
                        device=device).to(DT[cfg.dtype]) for _ in range(2))
    api.pkv_qcache_store(cfg, k * spread, v, cache)
    return cache, A.stored(cache, torch.arange(cache.rows, device=device))


def queries(cfg, m, device, seed=1, spread=1.0):
    gen = torch.Generator(device=device).manual_seed(seed)
    return (torch.randn((m, cfg.n_q_heads, cfg.head_dim), generator=gen, device=device)
            * spread).to(DT[cfg.dtype])


def run(cfg, q, cache, pos, start=None, n_seq=1, scale=0.0, out=None):
    m = q.shape[0]
    out = torch.full_like(q, float("nan")) if out is None else out
    lse = torch.full((m, cfg.n_q_heads), float("nan"), device=q.device)
    need = api.pkv_qcache_attn_workspace_bytes(cfg, cache.rows, m, n_seq)
    ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device=q.device) if need else None
    api.pkv_qcache_attn(cfg, q, cache, pos, out, start, n_seq, lse, scale, ws=ws)
    return out, lse


def ranges(cache, pos, start, n_seq):
    each = len(pos) // n_seq
    lo = torch.zeros_like(pos).long() if start is None else \
        start.long().clamp(0, cache.rows).repeat_interleave(each)
    hi = (lo + pos.long() + 1).clamp(max=cache.rows)
    return lo, torch.maximum(hi, lo)


def check(cfg, q, cache, values, pos, got, start=None, n_seq=1, scale=None):
    lo, hi = ranges(cache, pos, start, n_seq)
    want = A.attention(q, *values, lo, hi, scale)
    A.agree(got[0], got[1], want, cfg.dtype, int((hi - lo).max()), cfg.head_dim)


GEOMETRIES = [("bf16", 32, 8, 128), ("bf16", 10, 2, 128), ("bf16", 8, 2, 64), ("bf16", 4, 4, 16),
              ("bf16", 6, 2, 48), ("bf16", 4, 1, 256), ("bf16", 40, 1, 128), ("bf16", 5, 5, 80),
              ("f32", 4, 4, 64), ("f32", 8, 2, 128), ("f32", 3, 1, 48), ("f32", 2, 1, 256),
              ("f32", 34, 2, 32), ("bf16", 4, 2, 144)]


@pytest.mark.parametrize("dtype,hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 500, 4097])
def test_one_row_over_a_cache(gpu_device, dtype, hq, hkv, d, n):
    cfg = api.LayerCfg(hq, hkv, d, 64, 1e4, dtype)
    cache, values = filled(cfg, n + 5, gpu_device)
    q = queries(cfg, 1, gpu_device)
    pos = torch.tensor([n - 1], dtype=torch.int32, device=gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos))


@pytest.mark.parametrize("dtype,hq,hkv,d", GEOMETRIES)
@pytest.mark.parametrize("each", [1, 3])
def test_a_batch_of_sequences(gpu_device, dtype, hq, hkv, d, each):
    cfg = api.LayerCfg(hq, hkv, d, 64, 1e4, dtype)
    lens = [700, 1, 64, 0, 1033, 7, 0, 129, 33]
    cache, values = filled(cfg, sum(lens) + 100, gpu_device)
    start = torch.tensor([sum(lens[:i]) for i in range(len(lens))], dtype=torch.int32,
                         device=gpu_device)
    n = torch.tensor(lens, dtype=torch.int32, device=gpu_device)[:, None]
    pos = (n - each + torch.arange(each, dtype=torch.int32, device=gpu_device)).flatten()
    q = queries(cfg, len(pos), gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, len(lens)), start, len(lens))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 112)])
@pytest.mark.parametrize("m", [2, 5, 16, 17, 40, 150])
def test_many_rows_of_one_sequence(gpu_device, dtype, d, m):
    cfg = api.LayerCfg(8, 2, d, 64, 1e4, dtype)
    cache, values = filled(cfg, 3000, gpu_device)
    gen = torch.Generator(device=gpu_device).manual_seed(2)
    pos = torch.randint(-3, 3000, (m,), generator=gen, device=gpu_device).int()   # in any order
    q = queries(cfg, m, gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos))


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 8, 2, 128), ("f32", 4, 4, 64)])
@pytest.mark.parametrize("n_seq", [64, 65, 300])
def test_many_sequences(gpu_device, dtype, hq, hkv, d, n_seq):
    cfg = api.LayerCfg(hq, hkv, d, 64, 1e4, dtype)
    cache, values = filled(cfg, 5000, gpu_device)
    gen = torch.Generator(device=gpu_device).manual_seed(n_seq)
    start = torch.randint(0, 5000, (n_seq,), generator=gen, device=gpu_device).int()
    pos = torch.randint(-2, 1200, (n_seq,), generator=gen, device=gpu_device).int()
    pos[n_seq // 2] = 4999
    q = queries(cfg, n_seq, gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, n_seq), start, n_seq)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_ranges_out_of_the_cache(gpu_device, dtype, d):
    """Positions behind the end and sequences that begin outside end where the cache does; shared rows."""
    cfg = api.LayerCfg(4, 2, d, 64, 1e4, dtype)
    cache, values = filled(cfg, 256, gpu_device)
    big = 2 ** 31 - 1
    start = torch.tensor([0, 250, 256, 300, big, 17, 17, 255], dtype=torch.int32, device=gpu_device)
    pos = torch.tensor([big, 100, 3, 5, big, 40, 90, 0], dtype=torch.int32, device=gpu_device)
    q = queries(cfg, 8, gpu_device)
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, 8), start, 8)
    pos[:] = -2 ** 31
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, 8), start, 8)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 48)])
def test_rows_that_nobody_attends_do_not_matter(gpu_device, dtype, d):
    """Bytes of any value around the sequences, scales that stand for NaN among them."""
    cfg = api.LayerCfg(4, 2, d, 64, 1e4, dtype)
    cache, values = filled(cfg, 1024, gpu_device)
    start = torch.tensor([37, 500], dtype=torch.int32, device=gpu_device)
    pos = torch.tensor([400, 61], dtype=torch.int32, device=gpu_device)
    q = queries(cfg, 2, gpu_device)
    used = torch.zeros(cache.rows, dtype=torch.bool, device=gpu_device)
    used[37:438], used[500:562] = True, True
    for fill in (255, 0, 254):
        for name, t in cache.tensors.items():
            if name == "v_scales":
                flat = t.permute(1, 3, 0, 2).reshape(cache.rows, 2, d // 16).clone()
                flat[~used] = fill
                t.copy_(flat.view(cache.rows // 8, 8, 2, d // 16).permute(2, 0, 3, 1))
            else:
                t[:, ~used] = fill
        check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, start, 2), start, 2)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_scores_of_any_size(gpu_device, dtype, d):
    cfg = api.LayerCfg(4, 2, d, 64, 1e4, dtype)
    pos = torch.tensor([2999], dtype=torch.int32, device=gpu_device)
    for spread in (0.0, 0.01, 20.0, 300.0):
        cache, values = filled(cfg, 3000, gpu_device, spread=spread)
        q = queries(cfg, 1, gpu_device, spread=3.0)
        check(cfg, q, cache, values, pos, run(cfg, q, cache, pos))
    check(cfg, q, cache, values, pos, run(cfg, q, cache, pos, scale=0.003), scale=0.003)


def test_values_that_are_not_finite_reach_the_rows_that_attend_them(gpu_device):
    cfg = api.LayerCfg(4, 2, 128, 64, 1e4, "bf16")
    cache, values = filled(cfg, 512, gpu_device)
    v = torch.zeros((1, 2, 128), dtype=torch.bfloat16, device=gpu_device)
    v[0, 1, 16] = float("inf")
    api.pkv_qcache_store(cfg, torch.zeros_like(v), v, cache,
                         torch.tensor([100], dtype=torch.int32, device=gpu_device))
    q = queries(cfg, 2, gpu_device)
    pos = torch.tensor([99, 100], dtype=torch.int32, device=gpu_device)
    out, _ = run(cfg, q, cache, pos)
    nan = torch.zeros_like(out, dtype=torch.bool)
    nan[1, 2:, 16:32] = True
    assert torch.equal(torch.isnan(out), nan)


def test_results_may_replace_the_queries_and_repeat(gpu_device):
    for dtype, d in (("bf16", 128), ("f32", 64)):
        cfg = api.LayerCfg(8, 2, d, 64, 1e4, dtype)
        cache, _ = filled(cfg, 6000, gpu_device)
        pos = torch.tensor([5999, 3, 700], dtype=torch.int32, device=gpu_device)
        q = queries(cfg, 3, gpu_device)
        want = run(cfg, q, cache, pos)
        again = run(cfg, q, cache, pos)
        mine = q.clone()
        over = run(cfg, mine, cache, pos, out=mine)
        for a, b in ((again, want), (over, want)):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_offsets_beyond_32_bits(gpu_device):
    """16 GB of codes a tensor: heads, rows and scales whose byte offsets need more than 32 bits."""
    cfg = api.LayerCfg(8, 8, 128, 64, 1e4, "bf16")
    rows = 1 << 25
    cache = api.QCache.empty(cfg, rows, gpu_device)
    n = 300
    gen = torch.Generator(device=gpu_device).manual_seed(5)
    k, v = (torch.randn((n, 8, 128), generator=gen, device=gpu_device).bfloat16()
            for _ in range(2))
    at = torch.arange(rows - n, rows, dtype=torch.int32, device=gpu_device)
    api.pkv_qcache_store(cfg, k, v, cache, at)
    out = torch.empty_like(k), torch.empty_like(v)
    api.pkv_qcache_restore(cfg, cache, *out, row_idx=at, rotate=False)
    for x, y in zip((k, v), out):
        want = A.decode(*A.encode(x.cpu().double().numpy()))
        assert torch.equal(y.cpu().double(), torch.from_numpy(want))
    q = queries(cfg, 1, gpu_device)
    start = torch.tensor([rows - n], dtype=torch.int32, device=gpu_device)
    pos = torch.tensor([n - 1], dtype=torch.int32, device=gpu_device)
    got = run(cfg, q, cache, pos, start)
    want = A.attention(q, *out, torch.zeros(1, device=gpu_device).long(),
                       torch.full((1,), n, device=gpu_device))
    A.agree(got[0], got[1], want, "bf16", n, 128)


def test_two_calls_at_once_and_a_captured_step(gpu_device):
    """A decoding step - the new row stored, the attention - as a graph whose lengths grow from replay to
    replay, beside eager calls on another stream."""
    cfg = api.LayerCfg(32, 8, 128, 64, 1e4, "bf16")
    cache, _ = filled(cfg, 3000, gpu_device)
    other, _ = filled(cfg, 700, gpu_device, seed=9)
    start = torch.tensor([0, 1500], dtype=torch.int32, device=gpu_device)
    pos = torch.tensor([1000, 40], dtype=torch.int32, device=gpu_device)
    dst = start + pos
    q, kv = queries(cfg, 2, gpu_device), torch.randn((2, 2, 8, 128), device=gpu_device).bfloat16()
    out, lse = torch.empty_like(q), torch.empty((2, 32), device=gpu_device)
    ws = torch.empty(max(256, api.pkv_qcache_attn_workspace_bytes(cfg, cache.rows, 2, 2)),
                     dtype=torch.uint8, device=gpu_device)

    def step():
        api.pkv_qcache_store(cfg, kv[0], kv[1], cache, dst)
        api.pkv_qcache_attn(cfg, q, cache, pos, out, start, 2, lse, ws=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    pos2 = torch.tensor([650], dtype=torch.int32, device=gpu_device)
    want2 = run(cfg, q[:1].contiguous(), other, pos2)
    side = torch.cuda.Stream()
    for n in range(4):
        pos += torch.tensor([1, 300 if n == 1 else 1], dtype=torch.int32, device=gpu_device)
        dst.copy_(start + pos)
        kv.normal_()
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            got2 = run(cfg, q[:1].contiguous(), other, pos2)
        torch.cuda.synchronize()
        eager = run(cfg, q, cache, pos, start, 2)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        assert torch.equal(got2[0], want2[0]) and torch.equal(got2[1], want2[1])
