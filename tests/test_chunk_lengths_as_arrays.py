"""Lengths of chunks as lists, arrays and tensors mean the same, a single one too."""

import numpy as np
import pytest
import torch

from paper_2602_02579_amd import diagnostics
from tests.test_gpu_model import CASES, EPS


@pytest.mark.parametrize("make", [list, tuple, np.array, torch.tensor])
@pytest.mark.parametrize("lens", [[40], [39, 1], [41], [20], [20, 21], [40, 0]])
def test_lengths(monkeypatch, make, lens):
    cfg, inter = CASES[sorted(CASES)[0]]
    dg = diagnostics.Diagnostics(cfg.with_(n_chunks=1, chunk_len=40), inter, EPS, torch.device("cpu"))
    embed = torch.zeros((40, cfg.hidden), dtype=dg.dt)
    got = []
    monkeypatch.setattr(dg, "_prefill_into", lambda e, b, k, v, chunks: got.append((len(e), chunks)))
    if sum(lens) != 40 or 0 in lens:
        with pytest.raises(ValueError, match="positive lengths"):
            dg.chunk_isolated_cache(embed, [{}], make(lens))
        assert got == []
    else:
        dg.chunk_isolated_cache(embed, [{}], make(lens))
        assert got == [(40, lens)]
