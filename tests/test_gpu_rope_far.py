"""rope_axes_forward at positions near 2^31: the angle is as exact there as near 0."""
from fractions import Fraction

import numpy as np
import pytest

from tests.sampling_util import STEP, U32, gpu, host, round_to

pytestmark = pytest.mark.gpu

PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def cos_sin(pos, freq):
    """Of pos * freq radians, reduced in exact arithmetic."""
    angle = Fraction(int(pos)) * Fraction(float(freq))
    turns = angle / (2 * PI)
    rest = float((turns - round(turns)) * 2 * PI)     # |rest| <= pi, off by 2^-53 of itself
    return np.cos(rest), np.sin(rest)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("top", [1.0, 3.7, 1000.0])
def test_far_positions_are_exact(dtype, layout, top):
    """A turned element errs by 4 units of 2^-24 of its pair for sine and cosine and three more for the products and their sum (the bounds of the
    rotation at near positions), and one rounding to the data type; nothing grows with the angle, which reaches 2^31 * top."""
    import torch
    import paper_2507_07966_amd as pa
    T, H, pairs = 48, 2, 16
    rng = np.random.default_rng(int(top))
    pos = np.concatenate([rng.integers((1 << 31) - 100000, 1 << 31, size=T // 2), -rng.integers((1 << 31) - 100000, (1 << 31) + 1, size=T // 2)])
    pos[0], pos[-1] = (1 << 31) - 1, -(1 << 31)
    freq = (top * rng.uniform(0.5, 1.0, size=pairs)).astype(np.float32)
    freq[:2] = top, 0.7 * top
    x = round_to(rng.standard_normal((T, H, 2 * pairs)), dtype)
    rope = pa.rope_axes((pairs,), 2 * pairs, layout=layout)
    out = torch.empty_like(gpu(x, dtype))
    pa.rope_axes_forward(rope, gpu(x, dtype), None, gpu(pos.astype(np.int32)[None]), gpu(freq), out, None)
    got = host(out)
    turn = np.array([[cos_sin(p, f) for f in freq] for p in pos])
    c, s = turn[:, None, :, 0], turn[:, None, :, 1]
    first, second = (slice(0, pairs), slice(pairs, None)) if layout == "halves" else (slice(0, None, 2), slice(1, None, 2))
    a, b = x[:, :, first], x[:, :, second]
    worst = 0.0
    for part, want in ((first, a * c - b * s), (second, b * c + a * s)):
        bound = (7 * U32 * (np.abs(a) + np.abs(b)) + STEP[dtype] * np.abs(want)) * (1 + 2.0 ** -7)
        worst = max(worst, float((np.abs(got[:, :, part] - want) / bound).max()))
    print(f"error / bound {worst:.3f}", flush=True)
    assert worst <= 1
