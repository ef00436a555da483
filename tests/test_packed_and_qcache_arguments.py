"""What the calls on packed prompts and on the cache in 4 bits refuse, before any launch: no GPU
is needed, and nothing is enqueued on account of a bad argument."""

import ctypes
import os

import pytest
import torch

from paper_2602_02579_amd import api, diagnostics, model, synth

CFG = api.LayerCfg(8, 2, 128, 256, 1e4, "bf16")
P = 4096          # a pointer that is aligned and never followed


@pytest.fixture
def lib():
    if not os.path.exists(api.library_path()):
        pytest.skip("libpkv.so not built")
    return api.load_library()


def cache(rows=64, **over):
    c = api._CQCache(P, P, P, P, rows)
    for name, value in over.items():
        setattr(c, name, value)
    return ctypes.byref(c)


def test_packed_attn(lib):
    def status(q=P, k=P, v=P, pos=P, out=P, lse=None, m=4, scale=0.0, cfg=CFG, ws=None, ws_bytes=0):
        return lib.pkv_packed_attn(cfg and cfg._ref, q, k, v, pos, out, lse, m, scale, ws, ws_bytes,
                                   None)
    assert status(cfg=None) == 1
    assert status(m=0, q=None, k=None, v=None, pos=None, out=None) == 0
    for name in ("q", "k", "v", "pos", "out"):
        assert status(**{name: None}) == 1
    for name in ("q", "k", "v", "out"):
        assert status(**{name: P + 8}) == 3
    assert status(m=-1) == 2 and status(m=(1 << 30) + 1) == 2
    assert status(m=1 << 28) == 3                              # 2^31 (row, head) pairs
    assert status(scale=-1.0) == 2 and status(scale=float("nan")) == 2
    assert status(cfg=api.LayerCfg(8, 3, 128, 256, 1e4, "bf16")) == 2
    assert status(cfg=api.LayerCfg(8, 2, 72, 256, 1e4, "bf16")) == 3
    big = 1 << 18
    need = api.pkv_packed_attn_workspace_bytes(CFG, big)
    if need:
        assert need % 256 == 0
        assert status(m=big) == 4 and status(m=big, ws=P, ws_bytes=need - 1) == 4
    assert api.pkv_packed_attn_workspace_bytes(CFG, 0) == 0
    assert api.pkv_packed_attn_workspace_bytes(CFG, -1) == 0
    assert api.pkv_packed_attn_workspace_bytes(CFG, 1 << 28) == 0


def test_qcache_store_and_restore(lib):
    def store(k=P, v=P, dst=None, c=cache(), m=4, cfg=CFG):
        return lib.pkv_qcache_store(cfg and cfg._ref, k, v, dst, c, m, None)

    def restore(c=cache(), idx=None, pos=None, base=0, k=P, v=P, m=4, cfg=CFG):
        return lib.pkv_qcache_restore(cfg and cfg._ref, c, idx, pos, base, 1, k, v, m, None)
    for call in (store, restore):
        assert call(cfg=None) == 1 and call(c=None) == 1
        assert call(m=0, k=None, v=None) == 0
        assert call(k=None) == 1 and call(v=None) == 1
        assert call(k=P + 8) == 3 and call(v=P + 4) == 3
        assert call(m=-1) == 2
        assert call(m=65) == 2                                 # more rows than the cache has
        assert call(c=cache(rows=0)) == 2 and call(c=cache(rows=40)) == 2
        assert call(c=cache(rows=-32)) == 2 and call(c=cache(rows=(1 << 30) + 32)) == 2
        for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
            assert call(c=cache(**{name: None})) == 1
            assert call(c=cache(**{name: P + 8})) == 3
        assert call(cfg=api.LayerCfg(8, 2, 8, 256, 1e4, "bf16")) == 3
    assert restore(base=1 << 31) == 2 and restore(base=-(1 << 31)) == 2


def test_qcache_attn(lib):
    def status(q=P, c=cache(), pos=P, start=None, out=P, m=4, n_seq=1, scale=0.0, cfg=CFG, ws=None,
               ws_bytes=0):
        return lib.pkv_qcache_attn(cfg and cfg._ref, q, c, pos, start, out, None, m, n_seq, scale, ws,
                                   ws_bytes, None)
    assert status(cfg=None) == 1 and status(c=None) == 1
    assert status(m=0, q=None, pos=None, out=None) == 0
    for name in ("q", "pos", "out"):
        assert status(**{name: None}) == 1
    assert status(q=P + 8) == 3 and status(out=P + 8) == 3
    assert status(m=-4) == 2 and status(n_seq=0) == 2 and status(n_seq=-1) == 2
    assert status(n_seq=3) == 2 and status(n_seq=8) == 2
    assert status(scale=-1.0) == 2 and status(scale=float("inf")) == 2
    assert status(c=cache(rows=33)) == 2 and status(c=cache(v_scales=None)) == 1
    assert status(m=1 << 28) == 3
    need = api.pkv_qcache_attn_workspace_bytes(CFG, 1 << 20, 1, 1)
    if need:
        assert need % 256 == 0
        assert status(c=cache(rows=1 << 20), m=1) == 4
        assert status(c=cache(rows=1 << 20), m=1, ws=P, ws_bytes=need - 1) == 4
    for rows, m, n_seq in ((0, 1, 1), (33, 1, 1), (64, 0, 1), (64, 3, 2), (64, 1, 0), (64, 1 << 28, 1)):
        assert api.pkv_qcache_attn_workspace_bytes(CFG, rows, m, n_seq) == 0


def test_shapes_are_checked_by_the_binding():
    new = lambda *s: torch.zeros(s, dtype=torch.bfloat16)          # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)             # noqa: E731
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)              # noqa: E731
    good = (new(3, 8, 128), new(3, 2, 128), new(3, 2, 128), i32(3), new(3, 8, 128))
    for i, bad in ((0, new(2, 8, 128)), (1, new(3, 8, 128)), (2, new(3, 2, 64)), (3, i32(4)),
                   (3, i32(3, 1)), (4, new(3, 2, 128))):
        with pytest.raises(ValueError, match="must be"):
            api.pkv_packed_attn(CFG, *good[:i], bad, *good[i + 1:])
    with pytest.raises(ValueError, match="lse_out"):
        api.pkv_packed_attn(CFG, *good, torch.zeros(3, 2))
    with pytest.raises(ValueError, match="GPU tensor"):
        api.pkv_packed_attn(CFG, *good)
    parts = [u8(2, 64, 64), u8(2, 64, 8), u8(2, 64, 64), u8(2, 8, 8, 8)]
    for i, bad in ((0, u8(2, 63, 64)), (0, u8(2, 0, 64)), (0, u8(64, 64)), (1, u8(2, 64, 16)),
                   (2, u8(2, 64, 128)), (3, u8(2, 64, 8))):
        with pytest.raises(ValueError, match="must be"):
            api.QCache(CFG, *parts[:i], bad, *parts[i + 1:])
    with pytest.raises(ValueError, match="GPU tensor"):
        api.QCache(CFG, *parts)
    c = object.__new__(api.QCache)
    c.heads, c.head_dim, c.rows, c.device = 2, 64, 64, -1
    with pytest.raises(ValueError, match="GPU tensor"):
        api.pkv_qcache_store(CFG, new(3, 2, 128), new(3, 2, 128), c)
    with pytest.raises(ValueError, match="other heads"):
        api._of_cache(CFG, c, -1)
    c.head_dim = 128
    for call in (lambda: api.pkv_qcache_store(CFG, new(3, 2, 128), new(4, 2, 128), c),
                 lambda: api.pkv_qcache_store(CFG, new(3, 2, 128), new(3, 2, 128), c, i32(4)),
                 lambda: api.pkv_qcache_restore(CFG, c, new(3, 2, 128), new(3, 2, 64)),
                 lambda: api.pkv_qcache_restore(CFG, c, new(3, 2, 128), new(3, 2, 128), i32(2)),
                 lambda: api.pkv_qcache_restore(CFG, c, new(3, 2, 128), new(3, 2, 128), None, i32(2)),
                 lambda: api.pkv_qcache_attn(CFG, new(3, 8, 128), c, i32(2), new(3, 8, 128)),
                 lambda: api.pkv_qcache_attn(CFG, new(3, 8, 128), c, i32(3), new(3, 8, 128), i32(2)),
                 lambda: api.pkv_qcache_attn(CFG, new(3, 8, 128), c, i32(3), new(3, 8, 128),
                                             lse_out=torch.zeros(3, 2))):
        with pytest.raises(ValueError, match="must be"):
            call()


def test_layer_rows_packed(lib):
    def status(**over):
        c = api.LayerCall()
        c.m = c.n_cache = 4
        for name, value in over.items():
            setattr(c, name, value)
        return lib.pkv_layer_rows_packed(CFG._ref, ctypes.byref(c), None)
    assert lib.pkv_layer_rows_packed(None, None, None) == 1
    assert lib.pkv_layer_rows_packed(CFG._ref, None, None) == 1
    assert status(n_cache=5) == 2 and status(chunk_len=4) == 2 and status(chunk_len=-1) == 2
    assert status(score=P) == 2 and status(stop=3) == 2
    assert status() == 1                                       # none of its buffers


def test_chunk_lengths_make_up_the_context():
    cfg = synth.Config("lengths", "bf16", 2, 8, 4, 2, 1, 16, 32, 1e4)
    dg = diagnostics.Diagnostics(cfg, 32, 1e-5, torch.device("cpu"))
    embed = torch.zeros((cfg.n_ctx + cfg.n_query, 32), dtype=torch.bfloat16)
    for lens in ([], [15], [8, 9], [16, 0], [20, -4], (17,)):
        with pytest.raises(ValueError, match="positive lengths"):
            dg.chunk_isolated_cache(embed, [], lens)
    with pytest.raises(ValueError, match="positive lengths"):
        dg.chunk_isolated_cache(embed[:15], [], [8, 8])
    for bad in (2.5, [8.0, 8.0], None):
        with pytest.raises(TypeError):
            dg.chunk_isolated_cache(embed, [], bad)
    assert dg.chunk_isolated_cache(embed, [], torch.tensor([7, 9])) == ([], [])
    assert dg.chunk_isolated_cache(embed, [], [1] * 16) == ([], [])


def test_answer_rows_check_their_counts():
    cfg = synth.Config("answer", "bf16", 2, 8, 4, 2, 1, 16, 32, 1e4)
    for n_seq, each in ((0, 1), (1, 0), (-1, 1)):
        with pytest.raises(ValueError):
            model.AnswerRows(cfg, 32, 1e-5, [], torch.device("cpu"), n_seq, each)
    rows = model.AnswerRows(cfg, 32, 1e-5, [], torch.device("cpu"), 2)
    i32 = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="layers"):
        rows.step(torch.zeros((2, 32), dtype=torch.bfloat16), [{}], i32, i32)
