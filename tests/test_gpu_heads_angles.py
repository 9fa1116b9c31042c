"""Angles of positions on the GPU against exact arithmetic: cos and sin alone, of rows whose first pair of channels is (1, 0)."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2607_07724_amd as ugbs

pytestmark = pytest.mark.gpu

TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510")
FAR = [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30 + 12345, 2 ** 28 + 1, 2 ** 20, 3, 0, -1, -2 ** 28, -2 ** 31]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need an MI355X (gfx950) visible to torch")
    ugbs.lib()


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_far_positions_of_slow_and_negative_frequencies(sign):
    """The angle is off by at most 2^-51 |t| + 2^-23.  The second channel becomes 0 cos t + 1 sin t, the first 1 cos t - 0 sin t,
    without rounding; the series are off by 2^-28, three fp32 roundings of numbers up to one by 2^-23, where the
    number is small by 2^-23 of it; half a step of bf16 is 2^-8 of the result at most."""
    freqs = sign * np.concatenate([10.0 ** np.linspace(-15, 0, 30), [5e-15, 7.7e-12]])
    x = torch.zeros((1, len(FAR), 1, 64), dtype=torch.bfloat16, device="cuda")
    x[..., :32] = 1.0                                         # channels j and j + 32 are a pair
    h = ugbs.Heads.make(1, 1, 1, 64, len(FAR))
    Q, K, V = (torch.zeros((1, 1, len(FAR), 64), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    ugbs.ugbs_heads_split(h, x, x, x, torch.tensor(freqs, device="cuda"), Q, K, V,
                          positions=torch.tensor(FAR, dtype=torch.int32, device="cuda").view(1, 1, -1))
    got = Q[0, 0].double().cpu().numpy()
    for i, pos in enumerate(FAR):
        for j, f in enumerate(freqs.tolist()):
            t = Fraction(f) * pos
            rest = float(t - TWO_PI * round(t / TWO_PI))
            angle = 2.0 ** -51 * abs(float(t)) + 2.0 ** -23
            for c, want, slope in ((j, math.cos(rest), math.sin(rest)), (j + 32, math.sin(rest), math.cos(rest))):
                tol = (2.0 ** -8 + 2.0 ** -23) * abs(want) + angle * (abs(slope) + angle) + 2.0 ** -28
                assert abs(got[i, c] - want) <= tol, (pos, f, c >= 32, got[i, c], want, tol)
