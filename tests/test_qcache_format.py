"""The 4-bit format as the tests write it out, against its definition: the nearest of the values, the
even index in the middle, and a scale that keeps the largest magnitude within half a step."""

import numpy as np

from tests import attention64 as A


def test_the_nearest_value_and_the_even_index():
    rng = np.random.default_rng(0)
    x = np.concatenate((rng.standard_normal((300, 16)) * 2.0 ** rng.integers(-40, 40, (300, 1)),
                        np.arange(320).reshape(20, 16) / 8.0))
    index, byte = A.encode(x)
    scale = 2.0 ** (byte.astype(float) - 127)
    table = np.array(A.VALUES)
    far = np.abs(np.abs(x)[..., None] / scale[..., None] - table)
    best = far.min(-1)
    for i in range(len(x)):
        for j in range(16):
            near = np.flatnonzero(far[i, j] == best[i, j])
            want = near[0] if len(near) == 1 else near[near % 2 == 0][0]
            assert index[i, j] % 8 == want
            assert (index[i, j] >= 8) == np.signbit(x[i, j])
    top = np.abs(x).max(-1, keepdims=True) / scale
    assert (top < 7).all() and ((top >= 3.5) | (top == 0)).all()
    back = A.decode(index, byte)
    assert np.array_equal(back, np.sign(x) * table[index % 8] * scale)


def test_the_ends_of_the_scale():
    x = np.zeros((5, 16))
    x[0, 3], x[1, 3], x[2, 0], x[3, 5], x[4, 0] = 3e38, 2.0 ** -120, np.inf, np.nan, 2.0 ** 127 * 1.75
    index, byte = A.encode(x)
    assert byte[:, 0].tolist() == [252, 32, 255, 255, 252]
    back = A.decode(index, byte)
    assert back[0, 3] == 6 * 2.0 ** 125 and back[1, 3] == 0 and np.isnan(back[2:4]).all()
    assert np.isfinite(back[0].astype(np.float32)).all()
