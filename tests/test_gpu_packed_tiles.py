"""Attention over a packed prompt with more tiles than run at once, and with as few as leave CUs idle (whose
keys are split within a workgroup): what the smaller problems check, in both forms of the kernel."""

import pytest
import torch

from paper_2602_02579_amd import api
from tests import attention64 as A
from tests.test_gpu_packed_attn import DT, check, problem, run

pytestmark = pytest.mark.gpu

# 12000 or 70000 (row, head) pairs: less and more than 256 (head_dim 64: 512) tiles of 64
LAYOUTS = [("bf16", 32, 8, 128), ("bf16", 24, 8, 48), ("bf16", 16, 4, 96), ("bf16", 40, 8, 64),
           ("bf16", 8, 8, 112), ("bf16", 7, 1, 128),
           ("f32", 8, 8, 64), ("f32", 16, 4, 128), ("f32", 10, 2, 48), ("f32", 12, 4, 112), ("f32", 8, 2, 256)]


def lengths(hq, many):
    unit = [300, 1, 41, 64, 128, 17, 509]
    rows = (70000 if many else 12000) // hq
    out = []
    while sum(out) < rows:
        out.append(min(unit[len(out) % len(unit)], rows - sum(out)))
    return out


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("dtype,hq,hkv,d", LAYOUTS)
def test_sequences(gpu_device, dtype, hq, hkv, d, many):
    p = problem(gpu_device, dtype, hq, hkv, d, lengths(hq, many))
    got = run(*p)
    check(*p, got)
    mine = p[1].clone()
    over = run(p[0], mine, *p[2:], out=mine)
    assert torch.equal(over[0], got[0]) and torch.equal(over[1], got[1])


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("dtype,hq,hkv,d", LAYOUTS)
def test_padding_windows_and_one_sequence(gpu_device, dtype, hq, hkv, d, many):
    cfg, q, k, v, pos = problem(gpu_device, dtype, hq, hkv, d, lengths(hq, many), spread=3.0)
    at = torch.arange(len(pos), dtype=torch.int32, device=gpu_device)
    gaps = torch.where((at % 97 < 40) | (at > len(pos) - 30), -1, pos)
    check(cfg, q, k, v, gaps, run(cfg, q, k, v, gaps))
    window = at.clamp(max=70)
    check(cfg, q, k, v, window, run(cfg, q, k, v, window))
    one = at.clone()
    check(cfg, q, k, v, one, run(cfg, q, k, v, one))


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_a_row_does_not_see_does_not_reach_it(gpu_device, many, bad):
    lens = lengths(32, many)
    cfg, q, k, v, pos = problem(gpu_device, "bf16", 32, 8, 128, lens)
    k2, v2 = k.clone(), v.clone()
    k2[301:342], v2[301:342] = bad, bad
    got = run(cfg, q, k2, v2, pos)
    clean = torch.ones(len(pos), dtype=torch.bool, device=gpu_device)
    clean[301:342] = False
    at = torch.arange(len(pos), device=gpu_device)
    want = A.attention(q, k, v, at - pos, at + 1)
    A.agree(got[0][clean], got[1][clean], [x[clean] for x in want], "bf16", max(lens), 128)
    assert torch.isnan(got[0][301:342]).all()


@pytest.mark.parametrize("dtype,hkv", [("bf16", 16), ("f32", 8)])
def test_offsets_beyond_32_bits(gpu_device, dtype, hkv):
    """Tensors of more than 4 GB: a window of 41 rows for every row, looked at where they end."""
    m = (1 << 20) + 4099
    cfg = api.LayerCfg(hkv, hkv, 128, 64, 1e4, dtype)
    gen = torch.Generator(device=gpu_device).manual_seed(1)
    q, k, v = (torch.empty((m, hkv, 128), dtype=DT[dtype], device=gpu_device).normal_(generator=gen)
               for _ in range(3))
    pos = torch.arange(m, dtype=torch.int32, device=gpu_device).clamp(max=40)
    out, lse = run(cfg, q, k, v, pos)
    for a in (0, m // 2 + 1, m - 500):
        rows, seen = slice(a, a + 500), slice(max(0, a - 40), a + 500)
        at = torch.arange(a, a + 500, device=gpu_device) - seen.start
        want = A.attention(q[rows], k[seen], v[seen], at - pos[rows], at + 1)
        A.agree(out[rows], lse[rows], want, dtype, 41, 128)
