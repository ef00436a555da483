"""Attention over a packed prompt with values that are not finite: they reach the elements of the rows that
see them and no others, large values do not overflow on the way to a finite result, and none of it
costs many times what finite values do."""

import pytest
import torch

from tests import attention64 as A
from tests.test_gpu_packed_attn import check, problem, run

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
# the second: more tiles of bf16 than the form for few tiles takes
LENS = {"few": [200, 1, 333, 70], "many": [700, 1, 900, 333, 70, 300]}
LAYOUTS = [("bf16", 32, 8, 128), ("bf16", 7, 1, 128), ("bf16", 8, 2, 64), ("bf16", 40, 8, 64), ("bf16", 4, 2, 80),
           ("bf16", 3, 3, 16), ("bf16", 4, 2, 256), ("f32", 4, 2, 64), ("f32", 6, 2, 128),
           ("f32", 5, 1, 48), ("f32", 4, 2, 112), ("f32", 4, 2, 256), ("f32", 2, 1, 144)]


def starts_of(pos):
    at = torch.arange(len(pos), device=pos.device)
    return at, torch.where(pos < 0, at + 1, (at - pos).clamp(min=0))


def check_elements(cfg, q, k, v, pos, bad, in_place=False):
    """``bad``: (row, kv head, element, value) of values put into v; everything else as without them."""
    v2 = v.clone()
    at, lo = starts_of(pos)
    plus = torch.zeros(q.shape, dtype=torch.bool, device=q.device)
    minus = plus.clone()
    group = cfg.n_q_heads // cfg.n_kv_heads
    for row, head, d, x in bad:
        v2[row, head, d] = x
        seen = ((lo <= row) & (at >= row))[:, None]
        heads = slice(head * group, (head + 1) * group)
        if not x < 0:
            plus[:, heads, d] |= seen
        if not x > 0:
            minus[:, heads, d] |= seen
    mine = q.clone()
    out, lse = run(cfg, mine, k, v2, pos, out=mine if in_place else None)
    assert torch.equal(torch.isnan(out), plus & minus)
    assert torch.equal(out == INF, plus & ~minus) and torch.equal(out == -INF, minus & ~plus)
    want = A.attention(q, k, v, lo, at + 1)
    out = torch.where(plus | minus, want[0].to(out.dtype), out)
    A.agree(out, lse, want, cfg.dtype, int((at + 1 - lo).max()), cfg.head_dim)


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("dtype,hq,hkv,d", LAYOUTS)
def test_elements_that_are_not_finite(gpu_device, dtype, hq, hkv, d, lens):
    p = problem(gpu_device, dtype, hq, hkv, d, LENS[lens])
    n = p[1].shape[0]
    bad = [(5, 0, 3, NAN), (150, hkv - 1, d - 1, INF), (199, 0, 3, INF), (201, 0, 0, -INF),
           (260, hkv - 1, d - 1, -INF), (263, hkv - 1, d - 1, INF), (300, 0, d // 2, NAN), (n - 1, 0, 1, -INF),
           (n - 40, 0, 1, -INF)]
    check_elements(*p, bad)
    check_elements(*p, bad[1:3], in_place=True)


@pytest.mark.parametrize("dtype,hq,hkv,d", LAYOUTS)
def test_padding_of_any_bytes(gpu_device, dtype, hq, hkv, d):
    """Rows of padding between, in front of and behind the sequences, whose queries, keys and values are NaN."""
    cfg, q, k, v, pos = problem(gpu_device, dtype, hq, hkv, d, [30, 200, 41, 3, 29, 300, 7])
    pos[:30], pos[230:271], pos[274:303], pos[-7:] = -1, -1, -1, -1
    pad = pos < 0
    for t in (q, k, v):
        t[pad] = NAN
    got = run(cfg, q, k, v, pos)
    assert (got[0][pad] == 0).all()
    q[pad], k[pad], v[pad] = 0, 0, 0
    check(cfg, q, k, v, pos, got)


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("dtype,hq,hkv,d", LAYOUTS)
def test_large_values_do_not_overflow_on_the_way(gpu_device, dtype, hq, hkv, d, lens):
    cfg, q, k, v, pos = problem(gpu_device, dtype, hq, hkv, d, LENS[lens])
    v = torch.where(v > 0.5, 1.5 * 2.0 ** 126, 2.0 ** 127).to(v.dtype)
    check(cfg, q, k, v, pos, run(cfg, q, k, v, pos))
    v[:, :, ::3] *= -1
    check(cfg, q, k, v, pos, run(cfg, q, k, v, pos))


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 8, 2, 64), ("f32", 4, 4, 64)])
@pytest.mark.parametrize("where", ["key", "value", "both ends"])
def test_time(gpu_device, dtype, hq, hkv, d, where):
    """One bad value that thousands of rows see: another pass over the keys, one that is not pipelined (and in
    fp32 not shared by four waves), some 10 times the first.  Column by column it took 70 to 1100 times as long."""
    cfg, q, k, v, pos = problem(gpu_device, dtype, hq, hkv, d, [4096])
    k2, v2 = k.clone(), v.clone()
    if where == "key":
        k2[0, 0, 0] = NAN
    else:
        v2[0, 0, 0] = NAN
        if where == "both ends":
            v2[4000, hkv - 1, 5] = INF

    def least(k, v):
        times = []
        for _ in range(6):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            run(cfg, q, k, v, pos)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)
    clean, bad = least(k, v), least(k2, v2)
    assert bad < 20 * clean, (clean, bad)
