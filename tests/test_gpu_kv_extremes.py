"""8-bit pages at the ends of the types' ranges."""
import math

import pytest
import torch

from test_gpu_kv_ops import DEV, Pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h", [32, 64, 128])
def test_eight_bits_hold_the_largest_numbers(dtype, h):
    """Finite rows come back finite, each value within half a step (2^-4 of it), up to the largest number of the type."""
    p = Pool(dtype, "fp8", 1, 1, h, 64, [(0, 70)])
    top = float(torch.finfo(p.t).max)
    x = p.normal(70, 1, h, scale=top / 40)
    x[0], x[1], x[2, 0, ::2], x[3, 0, 1::2] = top, -top, top, -top
    x[4] = torch.linspace(0.9, 1.0, h, device=DEV).mul(top).to(p.t)
    x[5, 0, 0], x[5, 0, 1], x[6, 0, 0] = top, math.inf, math.nan
    # borders: 247.9 and 248 times 2^120, of which the first lies below the middle of 240 and 256
    x[7:10] = torch.tensor([247.0, 248.0, -248.0], device=DEV).view(3, 1, 1).mul(2.0 ** 120).to(p.t)
    b = p.batch([70], [70])
    p.cache.append(b, None, x, x)
    for got in p.cache.read(b):
        fine = x.isfinite()
        assert torch.equal(got.isfinite(), fine) and torch.equal(got.isnan(), ~fine)
        assert bool(((got.double() - x.double()).abs() <= x.double().abs() * 2.0 ** -4)[fine & (x.abs() > top / 64)].all())
        assert bool((got[7].double() == 240 * 2.0 ** 120).all())
    b.check()
