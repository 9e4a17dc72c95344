"""The operators on a K/V cache where launches, masks, memory and values meet:
against the definitions in 64 bits with the tolerances of test_gpu_cache.py."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import test_gpu_cache as T  # noqa: E402
from test_gpu_cache import Case, S, check, ints  # noqa: E402


# ---- large values ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("t", [1, 20, 100, 200])
def test_large_values_behind_a_rising_score(dtype, d, t):
    # a slot's score is above those before it by a factor of 2^7.2 of its weight, and
    # its values are a hundredth of the largest number: no weight may exceed 1
    c = Case(dtype, d, b=1, hkv=1, g=1, cap=140, lens=(140,), t=t)
    c.q[:], c.k[:], c.kn[:] = 0, 0, 0
    c.q[..., 0] = math.sqrt(d)
    c.k[0, 0, 130, 0] = 5.0
    c.v[0, 0, 130] = 3e36 * torch.sign(c.v[0, 0, 130].float()).to(c.v.dtype)
    for x, y in ((c.dq, c.q), (c.dk, c.k), (c.dkn, c.kn), (c.dv, c.v)):
        x.copy_(y)
    T.run_attend(c)
