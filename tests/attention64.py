"""Attention of rows over ranges of keys in 64 bits, with the sizes that tolerances are made of, and
the 4-bit format of a cache written out element by element."""

import numpy as np
import torch

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def attention(q, k, v, lo, hi, scale=None):
    """q [m, Hq, D], k, v [n, Hkv, D]; row i sees the keys lo[i] <= t < hi[i].  Returns out, lse, the same
    sum over |v| and the largest sum of |q||k| over a row's keys, all fp64 on the inputs' device."""
    q, k, v = q.double(), k.double(), v.double()
    m, hq, d = q.shape
    n, hkv = k.shape[:2]
    scale = d ** -0.5 if scale is None else scale
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((m, hq), float("-inf"), dtype=torch.float64, device=q.device)
    most = torch.zeros_like(lse)
    at = torch.arange(n, device=q.device)
    for r in range(0, m, 512):
        rows = slice(r, min(m, r + 512))
        a, b = int(lo[rows].min()), max(int(hi[rows].max()), int(lo[rows].min()))
        if a >= b:
            continue
        seen = (at[a:b] >= lo[rows, None]) & (at[a:b] < hi[rows, None])
        some = seen.any(1)
        for h in range(hq):
            kh, vh = k[a:b, h * hkv // hq].contiguous(), v[a:b, h * hkv // hq].contiguous()
            s = (q[rows, h] @ kh.t().contiguous() * scale).masked_fill(~seen, float("-inf"))
            norm = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(some, norm, 0.0)[:, None])
            vh = torch.where(torch.isfinite(vh) | seen.any(0)[:, None], vh, 0.0)
            out[rows, h], size[rows, h], lse[rows, h] = p @ vh, p @ vh.abs(), norm
            qk = q[rows, h].abs() @ kh.abs().t().contiguous() * scale
            most[rows, h] = qk.masked_fill(~seen, 0.0).amax(1)
    return out, lse, size, most


def tolerance(dtype, out, size, most, n_keys, d):
    """Of the output: its own rounding; bf16: the rounding of the weights, half a step of each; fp32 sums
    over d products for a score (off by d half steps of the sum of |q||k|, which goes into the
    weight as it is) and over the keys for the numerator and the denominator."""
    s = 2.0 ** -24
    weight = (d + 8) * s * most.unsqueeze(-1) + 2 * n_keys * s + 8 * s
    if dtype == "bf16":
        weight = weight + HALF_STEP["bf16"]
    return HALF_STEP[dtype] * out.abs() + 2 * size * weight * 1.01 + 1e-30


def lse_tolerance(lse, most, n_keys, d):
    s = 2.0 ** -24
    return (d + 8) * s * most + (2 * n_keys + 8) * s + 4 * s * lse.abs().nan_to_num(0, 0, 0)


def agree(got, lse, want, dtype, n_keys, d):
    """The elements of ``got`` (and ``lse``) against what ``attention`` returned."""
    out, norm, size, most = want
    off = (got.double() - out).abs() - tolerance(dtype, out, size, most, n_keys, d)
    assert not torch.isnan(got).any()
    assert off.max() <= 0, (float(off.max()), int(off.argmax()))
    if lse is not None:
        empty = torch.isinf(norm)
        assert torch.equal(lse.double()[empty], norm[empty])
        off = ((lse.double() - norm).abs() - lse_tolerance(norm, most, n_keys, d))[~empty]
        assert off.numel() == 0 or off.max() <= 0, float(off.max())


# ---- the format ---------------------------------------------------------------------------------

def encode(x):
    """Indices 0..15 and scale bytes of x [.., D] (numpy, any float type), element by element."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(-1, 16)
    index, byte = np.zeros(blocks.shape, np.uint8), np.zeros(len(blocks), np.uint8)
    middles = [(a + b) / 2 for a, b in zip(VALUES, VALUES[1:])]
    for n, b in enumerate(blocks):
        if not np.isfinite(b).all():
            byte[n] = 255
            continue
        top = np.abs(b).max()
        e = -200
        if top > 0:
            e = int(np.floor(np.log2(top)))
            e += int(2.0 ** (e + 1) <= top) - int(2.0 ** e > top)      # log2 may round across a power
            e -= 2
            e += int(top >= 7 * 2.0 ** e)
        e = min(max(e, 32 - 127), 252 - 127)
        byte[n] = e + 127
        for j, y in enumerate(np.abs(b) / 2.0 ** e):
            i = 0
            for i, mid in enumerate(middles):     # past the middle, or in it with an even index above
                if y < mid or (y == mid and i % 2 == 0):
                    break
            else:
                i = 7
            index[n, j] = i + 8 * np.signbit(b[j])
    return index.reshape(x.shape), byte.reshape(*x.shape[:-1], -1)


def decode(index, byte):
    table = np.array(VALUES + tuple(-a for a in VALUES))
    with np.errstate(invalid="ignore"):
        scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return table[index] * np.repeat(scale, 16, -1)


def stored(cache, rows):
    """Values fp64 [n, Hkv, D] that the tensors of a QCache hold in the given rows (a tensor)."""
    t = {name: x.cpu().numpy() for name, x in cache.tensors.items()}
    r = rows.cpu().numpy()
    both = []
    for codes, scales in ((t["k_codes"], t["k_scales"]),
                          (t["v_codes"], t["v_scales"].transpose(0, 1, 3, 2).reshape(
                              t["k_scales"].shape))):
        c = codes[:, r]
        index = np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1)
        both.append(torch.from_numpy(decode(index, scales[:, r]).transpose(1, 0, 2).copy()).to(
            rows.device))
    return both
