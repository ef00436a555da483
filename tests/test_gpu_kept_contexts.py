"""The calls on packed prompts and on caches in 4 bits as a program uses them together: chunks of any
lengths prefilled side by side, kept in 4 bits, put together in another order, selected from and
recomputed, and the answer decoded over the result.

Against the oracles, which take over what was stored (a value near the middle of two codes may go
either way): the stored values themselves are checked against the oracle's to half the distance of
two codes.  Bars as for the rest of the model: fp32 1e-4, bf16 2e-2 of the largest element for a
call, twice that behind several layers."""

import numpy as np
import pytest
import torch

from oracle import pkv_diag_oracle as DG
from oracle import pkv_model_oracle as MO
from oracle import pkv_oracle as O
from paper_2602_02579_amd import api, diagnostics, model, synth
from tests import attention64 as A
from tests.test_gpu_diagnostics import geo_of, make_model, to_dev
from tests.test_gpu_model import CASES, EPS, TOL, geometry, host, rel_err

pytestmark = pytest.mark.gpu

LENGTHS = {"f32-small": [1, 60, 2, 37, 28], "bf16-tiles": [200, 1, 33, 64, 128, 86],
           "bf16-odd": [130, 7, 96, 67]}


def as64(blocks):
    return [{k: v.astype(np.float64) for k, v in b.items()} for b in blocks]


def chunks_of(lens):
    ends = np.cumsum(lens)
    return [(e - n, e) for n, e in zip(lens, ends)]


def produced(name, device):
    cfg, inter = CASES[name]
    embed, blocks = make_model(cfg, inter)
    d_embed, d_blocks = to_dev(cfg, embed, blocks, device)
    dg = diagnostics.Diagnostics(cfg, inter, EPS, device)
    return cfg, inter, embed, blocks, d_embed, d_blocks, dg


@pytest.mark.parametrize("name", list(LENGTHS))
def test_chunks_of_any_lengths(gpu_device, name):
    cfg, inter, embed, blocks, d_embed, d_blocks, dg = produced(name, gpu_device)
    got = dg.chunk_isolated_cache(d_embed, d_blocks, LENGTHS[name])
    for a, b in chunks_of(LENGTHS[name]):
        alone = DG.chunk_isolated_cache(embed[a:b].astype(np.float64), as64(blocks), b - a, b - a,
                                        **geo_of(cfg))
        for g, w in zip(got, alone):
            for li in range(cfg.n_layers):
                bar = TOL[cfg.dtype] * (1 if li == 0 else 2)
                assert rel_err(host(g[li][a:b]), w[li]) <= bar, (a, b, li)


@pytest.mark.parametrize("name", ["f32-small", "bf16-tiles"])
def test_equal_chunks_as_lengths(gpu_device, name, monkeypatch):
    """The same chunks named one by one, in one group and in several: the same rows, up to the
    order of the sums."""
    cfg, inter, embed, blocks, d_embed, d_blocks, dg = produced(name, gpu_device)
    n = 32
    want = dg.chunk_isolated_cache(d_embed, d_blocks, n)
    for rows in (diagnostics.GROUP_ROWS, 70):
        monkeypatch.setattr(diagnostics, "GROUP_ROWS", rows)
        got = dg.chunk_isolated_cache(d_embed, d_blocks, [n] * (cfg.n_ctx // n))
        for g, w in zip(got, want):
            for a, b in zip(g, w):
                assert rel_err(host(a), host(b)) <= 2 * TOL[cfg.dtype]


@pytest.mark.parametrize("name", list(LENGTHS))
def test_a_kept_context_is_selected_from_and_recomputed(gpu_device, name):
    cfg, inter, embed, blocks, d_embed, d_blocks, dg = produced(name, gpu_device)
    n, qn = cfg.n_ctx, cfg.n_query
    kept = model.keep_caches(cfg, *dg.chunk_isolated_cache(d_embed, d_blocks, LENGTHS[name]))
    parts = chunks_of(LENGTHS[name])[::-1]           # the chunks in another order
    order = torch.cat([torch.arange(a, b) for a, b in parts])
    rows = order.to(torch.int32).to(gpu_device)
    d_embed[:n] = d_embed[:n][rows.long()]
    embed = np.concatenate([embed[:n][order.numpy()], embed[n:]])
    layers, oracle = [], []
    for li, (d, b) in enumerate(zip(d_blocks, blocks)):
        k, v = (torch.full((n + qn, cfg.n_kv_heads, cfg.head_dim), float("nan"), device=gpu_device,
                           dtype=d["wq"].dtype) for _ in range(2))
        # the first layer: its chunks already in order, without a table
        kr, vr = A.stored(kept[li], rows.long())
        layer = dict(d, k_cache=k, v_cache=v, kept=kept[li], kept_rows=rows)
        if li == 0:
            lc = model.layer_cfg(cfg)
            layer["kept"] = api.QCache.empty(lc, n, gpu_device)
            api.pkv_qcache_store(lc, kr.to(k.dtype), vr.to(v.dtype), layer["kept"])
            del layer["kept_rows"]
        layers.append(layer)
        oracle.append(dict(as64([b])[0], k_nope=host(kr), v=host(vr)))
    cr = model.CarriedRows(cfg, inter, EPS, gpu_device)
    h = cr.run(d_embed, layers)
    torch.cuda.synchronize()
    sel = np.sort(cr.rows[:cr.k].cpu().numpy())
    _, score, want = MO.prophetkv_model(embed, oracle, qn, cr.k, cfg.n_score_layers, eps=EPS,
                                        dtype=cfg.dtype, sel=sel, **geometry(cfg))
    tol = TOL[cfg.dtype]
    assert rel_err(host(cr.score), score) <= tol
    # tokens are selected by a score that is off by tol of the largest: none may be left out that
    # lies further above one that was taken
    left = np.setdiff1d(np.arange(n), sel)
    assert score[left].max() - score[sel].min() <= 2 * tol * score.max()
    assert rel_err(host(h), want["h_final"]) <= 2 * tol
    for li, L in enumerate(layers):
        assert rel_err(host(L["k_cache"]), want["k_cache"][li]) <= 2 * tol
        assert rel_err(host(L["v_cache"]), want["v_cache"][li]) <= 2 * tol
        assert np.array_equal(host(L["v_cache"])[left], oracle[li]["v"][left])


def decode_oracle(cfg, h, blocks, caches, pos, start, each):
    """One step for rows of one or several sequences over what the caches hold after it; the stored
    rows against those that the oracle projects."""
    h = O.round_to_storage(h, cfg.dtype)
    used = pos >= 0
    where = start.repeat(each) + pos
    for b, cache in zip(as64(blocks), caches):
        x = MO.rmsnorm_rows(h, None, b["w_in"], EPS, cfg.dtype)
        q, k, v = O.project_qkv_rows(x, np.arange(len(pos)), pos, b["wq"], b["wk"], b["wv"],
                                     dtype=cfg.dtype, **geometry(cfg))
        held = [host(t) for t in A.stored(cache, torch.arange(cache.rows))]
        for new, t in ((k, held[0]), (v, held[1])):
            # two codes are at most 2 scales apart and a scale at most 1 / 3.5 of the largest of the
            # 16 elements; a value that is off by d itself may also raise the largest by d
            top = np.abs(new).reshape(*new.shape[:2], -1, 16).max(-1).repeat(16, -1)
            off = 2 * TOL[cfg.dtype] * np.abs(new).max()
            assert (np.abs(t[where] - new) <= (top + off) / 3.5 + off)[used].all()
        attn = np.zeros_like(q)
        for i in np.nonzero(used)[0]:
            s = slice(start[i // each], where[i] + 1)
            attn[i] = O.sparse_row_attn(q[i:i + 1], held[0][s], held[1][s], pos[i:i + 1],
                                        dtype=cfg.dtype)[0][0]
        h = MO.attention_block_tail(h, attn, b["wo"], cfg.dtype)
        h = MO.mlp_block(h, b["w_post"], EPS, b["w_gate"], b["w_up"], b["w_down"], cfg.dtype)
    return h


def inputs(cfg, m, device, seed):
    h = np.random.default_rng(seed).standard_normal((m, cfg.hidden)).astype(np.float32)
    h = torch.from_numpy(h).to(model.layer_cfg(cfg).torch_dtype)
    return h.to(device), host(h)


@pytest.mark.parametrize("name", list(LENGTHS))
def test_an_answer_over_the_recomputed_caches(gpu_device, name):
    cfg, inter, embed, blocks, d_embed, d_blocks, dg = produced(name, gpu_device)
    n, t = cfg.n_ctx, cfg.n_ctx + cfg.n_query
    layers = dg._layers_with_cache(d_blocks, *dg.chunk_isolated_cache(d_embed, d_blocks,
                                                                      LENGTHS[name]))
    model.CarriedRows(cfg, inter, EPS, gpu_device).run(d_embed, layers)
    caches = model.keep_caches(cfg, [L["k_cache"] for L in layers], [L["v_cache"] for L in layers],
                               room=6)
    one = model.AnswerRows(cfg, inter, EPS, caches, gpu_device)
    three = model.AnswerRows(cfg, inter, EPS, caches, gpu_device, rows_each=3)
    start = torch.zeros(1, dtype=torch.int32, device=gpu_device)
    at = t
    for step, rows in enumerate((one, three, one)):
        pos = torch.arange(at, at + rows.m, dtype=torch.int32, device=gpu_device)
        h, h64 = inputs(cfg, rows.m, gpu_device, step)
        assert rows.step(h, d_blocks, pos, start) is h
        want = decode_oracle(cfg, h64, blocks, caches, pos.cpu().numpy(), np.zeros(1, np.int64),
                             rows.m)
        assert rel_err(host(h), want) <= 2 * TOL[cfg.dtype]
        at += rows.m


def batch(cfg, device, room):
    """Sequences of several lengths in one cache for every layer, the last one empty."""
    lens = np.array([40, 1, 130, 0])
    start = np.concatenate([[0], np.cumsum(lens + room)[:-1]])
    lc, caches = model.layer_cfg(cfg), []
    gen = torch.Generator(device=device).manual_seed(5)
    for _ in range(cfg.n_layers):
        caches.append(api.QCache.empty(lc, int((lens + room).sum()), device))
        k, v = (torch.randn((caches[-1].rows, lc.n_kv_heads, lc.head_dim), generator=gen,
                            device=device).to(lc.torch_dtype) for _ in range(2))
        api.pkv_qcache_store(lc, k, v, caches[-1])
    return lens, start, caches


@pytest.mark.parametrize("name", list(LENGTHS))
@pytest.mark.parametrize("each", [1, 2])
def test_answers_to_a_batch(gpu_device, name, each):
    cfg, inter, embed, blocks, _, d_blocks, _ = produced(name, gpu_device)
    lens, start, caches = batch(cfg, gpu_device, 4)
    rows = model.AnswerRows(cfg, inter, EPS, caches, gpu_device, len(lens), each)
    pos = (lens[:, None] + np.arange(each)).reshape(-1)
    pos[-1] = -1                                     # a slot that is not used
    d_pos, d_start = (torch.from_numpy(a.astype(np.int32)).to(gpu_device) for a in (pos, start))
    before = [[t.clone() for t in A.stored(c, torch.arange(c.rows))] for c in caches]
    h, h64 = inputs(cfg, rows.m, gpu_device, 3)
    rows.step(h, d_blocks, d_pos, d_start)
    want = decode_oracle(cfg, h64, blocks, caches, pos, start, each)
    assert rel_err(host(h), want) <= 2 * TOL[cfg.dtype]
    written = (start.repeat(each) + pos)[pos >= 0]
    kept = np.setdiff1d(np.arange(caches[0].rows), written)
    for c, old in zip(caches, before):
        for a, b in zip(A.stored(c, torch.arange(c.rows)), old):
            assert torch.equal(a[kept], b[kept])


def test_a_step_is_captured_and_allocates_nothing(gpu_device):
    cfg, inter, _, _, _, d_blocks, _ = produced("bf16-tiles", gpu_device)
    lens, start, caches = batch(cfg, gpu_device, 8)
    _, _, again = batch(cfg, gpu_device, 8)
    d_start = torch.from_numpy(start.astype(np.int32)).to(gpu_device)
    hs = [inputs(cfg, len(lens), gpu_device, s)[0] for s in range(4)]

    def positions(step):
        return torch.from_numpy((lens + step).astype(np.int32)).to(gpu_device)

    eager = model.AnswerRows(cfg, inter, EPS, again, gpu_device, len(lens))
    want = [eager.step(h.clone(), d_blocks, positions(s), d_start) for s, h in enumerate(hs)]
    rows = model.AnswerRows(cfg, inter, EPS, caches, gpu_device, len(lens))
    h, pos = hs[0].clone(), positions(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        rows.step(h, d_blocks, pos, d_start)         # stores what the first replay stores again
        torch.cuda.synchronize()
        count = torch.cuda.memory_stats()["allocation.all.allocated"]
        rows.step(h, d_blocks, pos, d_start)
        assert torch.cuda.memory_stats()["allocation.all.allocated"] == count
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rows.step(h, d_blocks, pos, d_start)
    for s, x in enumerate(hs):
        h.copy_(x)
        pos.copy_(positions(s))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, want[s]), s
    for a, b in zip(caches, again):
        for name in a.tensors:
            assert torch.equal(a.tensors[name], b.tensors[name])
