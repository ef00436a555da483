"""Attention over a packed prompt against the same in 64 bits: lengths of one and of none, rows that
attend nothing, odd sizes and head layouts, windows, positions out of range, keys that are not
finite where nobody looks, several calls at once, and a captured call."""

import pytest
import torch

from paper_2602_02579_amd import api
from tests import attention64 as A

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def problem(device, dtype, hq, hkv, d, lens, seed=0, spread=1.0):
    gen = torch.Generator(device=device).manual_seed(seed)
    m = sum(lens)
    q, k, v = (torch.randn((m, h, d), generator=gen, device=device) for h in (hq, hkv, hkv))
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).to(device) if lens else \
        torch.empty(0, dtype=torch.int32, device=device)
    return api.LayerCfg(hq, hkv, d, 64, 1e4, dtype), (q * spread).to(DT[dtype]), k.to(DT[dtype]), \
        v.to(DT[dtype]), pos


def run(cfg, q, k, v, pos, scale=0.0, out=None, ws=None):
    m = q.shape[0]
    out = torch.full_like(q, float("nan")) if out is None else out
    lse = torch.full((m, cfg.n_q_heads), float("nan"), device=q.device)
    need = api.pkv_packed_attn_workspace_bytes(cfg, m)
    if ws is None and need:
        ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device=q.device)
    api.pkv_packed_attn(cfg, q, k, v, pos, out, lse, scale, ws=ws)
    return out, lse


def check(cfg, q, k, v, pos, got, scale=None):
    at = torch.arange(q.shape[0], device=q.device)
    lo = torch.where(pos < 0, at + 1, (at - pos).clamp(min=0))
    n_keys = int((at + 1 - lo).max()) if len(at) else 0
    want = A.attention(q, k, v, lo, at + 1, scale)
    A.agree(got[0], got[1], want, cfg.dtype, n_keys, cfg.head_dim)


LENS = {"one row": [1], "ones": [1] * 70, "short": [3, 1, 64, 65, 63, 2, 128, 17],
        "one": [777], "ragged": [512, 487, 1, 333, 500, 61, 130],
        "long first": [2049, 5, 40], "long last": [5, 40, 2049]}


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("dtype,hq,hkv,d", [
    ("bf16", 32, 8, 128), ("bf16", 10, 2, 128), ("bf16", 8, 8, 64), ("bf16", 7, 1, 128),
    ("bf16", 6, 3, 48), ("bf16", 2, 1, 256), ("bf16", 3, 3, 16), ("bf16", 4, 2, 80),
    ("f32", 4, 4, 64), ("f32", 6, 2, 128), ("f32", 5, 1, 48), ("f32", 2, 2, 256), ("f32", 3, 1, 32)])
def test_sequences_attend_within_themselves(gpu_device, dtype, hq, hkv, d, lens):
    p = problem(gpu_device, dtype, hq, hkv, d, LENS[lens])
    check(*p, run(*p))


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 8, 128), ("bf16", 4, 2, 64),
                                           ("f32", 4, 2, 64)])
def test_many_jobs(gpu_device, dtype, hq, hkv, d):
    p = problem(gpu_device, dtype, hq, hkv, d, [4100, 9, 1500, 700, 1, 2222], seed=4)
    check(*p, run(*p))


def test_groups_wider_than_a_tile(gpu_device):
    for hq, d in ((300, 128), (130, 64), (257, 16)):
        p = problem(gpu_device, "bf16", hq, 1, d, [9, 1, 40])
        check(*p, run(*p))
    p = problem(gpu_device, "f32", 71, 1, 32, [9, 1, 40])
    check(*p, run(*p))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("bf16", 96), ("f32", 64)])
def test_padding_windows_and_positions_out_of_range(gpu_device, dtype, d):
    cfg, q, k, v, pos = problem(gpu_device, dtype, 8, 2, d, [300, 41, 700])
    pos[5:9] = -1                       # padding inside, whole tiles of it, and at the end
    pos[320:600] = -5
    pos[-3:] = -2 ** 31
    pos[0], pos[10], pos[700] = 2 ** 31 - 1, 11, 5000      # further back than there are rows
    check(cfg, q, k, v, pos, run(cfg, q, k, v, pos))
    window = torch.arange(len(pos), dtype=torch.int32, device=gpu_device).clamp(max=99)
    check(cfg, q, k, v, window, run(cfg, q, k, v, window))
    nothing = torch.full_like(pos, -1)
    check(cfg, q, k, v, nothing, run(cfg, q, k, v, nothing))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("bf16", 32), ("f32", 64)])
def test_scores_of_any_size(gpu_device, dtype, d):
    """Scores far from zero, far below it only, growing along the keys, and all alike; a scale of one's own."""
    cfg, q, k, v, pos = problem(gpu_device, dtype, 4, 2, d, [700, 130], spread=30.0)
    check(cfg, q, k, v, pos, run(cfg, q, k, v, pos))
    low = k.clone()
    low[:] = -q[:, ::2].abs().amax() / 8
    check(cfg, q.abs(), low, v, pos, run(cfg, q.abs(), low, v, pos))
    grow = (k.abs() * torch.linspace(0.01, 8, len(pos), device=gpu_device)[:, None, None]).to(k.dtype)
    check(cfg, q.abs(), grow, v, pos, run(cfg, q.abs(), grow, v, pos))
    fall = grow.flip(0).contiguous()
    check(cfg, q.abs(), fall, v, pos, run(cfg, q.abs(), fall, v, pos))
    same = torch.zeros_like(k)
    check(cfg, q, same, v, pos, run(cfg, q, same, v, pos))
    check(cfg, q, k, v, pos, run(cfg, q, k, v, pos, 0.01), 0.01)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("bf16", 48), ("f32", 64)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_a_row_does_not_see_does_not_reach_it(gpu_device, dtype, d, bad):
    """A sequence of values that are not finite between two others, and rows behind a row of its own."""
    lens = [100, 70, 333]
    cfg, q, k, v, pos = problem(gpu_device, dtype, 4, 2, d, lens)
    k2, v2 = k.clone(), v.clone()
    k2[100:170], v2[100:170] = bad, bad
    k2[-1], v2[-1] = bad, bad
    got = run(cfg, q, k2, v2, pos)
    clean = torch.ones(len(pos), dtype=torch.bool, device=gpu_device)
    clean[100:170], clean[-1] = False, False
    at = torch.arange(len(pos), device=gpu_device)
    want = A.attention(q, k, v, at - pos, at + 1)
    A.agree(got[0][clean], got[1][clean], [x[clean] for x in want], dtype, 333, d)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("bf16", 80), ("f32", 64)])
def test_results_may_replace_the_queries(gpu_device, dtype, d):
    cfg, q, k, v, pos = problem(gpu_device, dtype, 8, 2, d, [700, 3, 200])
    want, lse = run(cfg, q, k, v, pos)
    mine = q.clone()
    _, lse2 = run(cfg, mine, k, v, pos, out=mine)
    assert torch.equal(mine, want) and torch.equal(lse, lse2)
    again = run(cfg, q, k, v, pos)
    assert torch.equal(again[0], want) and torch.equal(again[1], lse)


def test_nothing_else_is_written(gpu_device):
    cfg, q, k, v, pos = problem(gpu_device, "bf16", 4, 2, 128, [130, 5])
    room = torch.full((140, 4, 128), 7.0, dtype=q.dtype, device=gpu_device)
    norm = torch.full((140, 4), 7.0, device=gpu_device)
    ws = torch.empty(max(256, api.pkv_packed_attn_workspace_bytes(cfg, 135)), dtype=torch.uint8,
                     device=gpu_device)
    api.pkv_packed_attn(cfg, q, k, v, pos, room[:135], norm[:135], ws=ws)
    assert (room[135:] == 7).all() and (norm[135:] == 7).all()
    plain = torch.empty_like(q)
    api.pkv_packed_attn(cfg, q, k, v, pos, plain, ws=ws)      # without the normalisers
    assert torch.equal(plain, room[:135])
    none = q[:0]
    api.pkv_packed_attn(cfg, none, k[:0], v[:0], pos[:0], none.clone())


def test_two_calls_at_once_and_a_captured_one(gpu_device):
    cfg, q, k, v, pos = problem(gpu_device, "bf16", 32, 8, 128, [2100, 33, 1800])
    cfg2, q2, k2, v2, pos2 = problem(gpu_device, "bf16", 8, 2, 128, [150, 33], seed=8)
    want, want2 = run(cfg, q, k, v, pos), run(cfg2, q2, k2, v2, pos2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got2 = run(cfg2, q2, k2, v2, pos2)
    got = run(cfg, q, k, v, pos)
    torch.cuda.synchronize()
    for a, b in zip(got + got2, want + want2):
        assert torch.equal(a, b)

    out, lse = torch.empty_like(q), torch.empty_like(want[1])
    ws = torch.empty(max(256, api.pkv_packed_attn_workspace_bytes(cfg, len(pos))),
                     dtype=torch.uint8, device=gpu_device)
    api.pkv_packed_attn(cfg, q, k, v, pos, out, lse, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.pkv_packed_attn(cfg, q, k, v, pos, out, lse, ws=ws)
    for n in range(3):
        other = (pos.clone() + 0) if n != 1 else pos.clamp(max=40)
        pos.copy_(other)
        ws.random_(0, 256)
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        eager = run(cfg, q, k, v, pos)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
