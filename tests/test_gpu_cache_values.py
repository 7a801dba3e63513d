"""GPU tests of dspark_verify_attn_scaled where a block's scale says little about its values:
blocks of zeros, or of codes far below the largest, that take most of the probability.

Tolerances are those of test_gpu_cache.py, per row in the 2-norm.  bf16: 4e-3.  The output's
rounding is at most 2^-9 of each value and a probability's 2^-11; what lies below fp16's normal
numbers may cost every value 2^-9 of the row's largest if the roundings of all keys meet, which
those of different keys do not.  fp32: 1e-5, and what the block's own score is off by, which every
row's sum of probabilities has: its D products are of one sign, so their sum, `above` in the end,
is off by at most D roundings of it, D * 2^-24 * above (256 and 8: 1.2e-4).
"""
import numpy as np
import pytest
import torch

from gpu_helpers import dev, log, to_f64
from test_gpu_cache import Case, attend, check_attention

pytestmark = pytest.mark.gpu


def e4m3(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float64)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def with_a_block(c, values, scale, exp, above):
    """c's scores normally distributed and its values around 88 * 2^exp, but in one block of 16 tokens of
    each context: scores that lie `above` around it, these values and this scale of theirs."""
    D = c.Dqk
    q = (0.5 + torch.from_numpy(c.rng.random((c.rows, c.Hq, D), dtype=np.float32))).to(c.dt).to(dev())
    c.scale["k"][:] = np.where(np.isnan(c.scale["k"]), np.nan, np.float32(1 / 88))
    c.scale["v"][:] = np.where(np.isnan(c.scale["v"]), np.nan, np.float32(2.0 ** exp))
    for r in range(c.R):
        at = int(c.kv[r]) // 32 * 16  # first token of the block
        pg, sl = c.table[r, at // c.page], at % c.page
        c.code["k"][pg, :, sl:sl + 16] = e4m3(np.full((c.Hkv, 16, D), 64.0))
        c.scale["k"][pg, :, sl // 16] = np.float32(above / 64 / D ** 0.5)
        c.code["v"][pg, :, sl:sl + 16] = e4m3(values(c.rng, (c.Hkv, 16, c.Dv)))
        c.scale["v"][pg, :, sl // 16] = scale
    return q


ZERO = lambda rng, shape: np.zeros(shape)  # noqa: E731
LOW = lambda rng, shape: 2.0 ** -9 * rng.integers(-1, 2, shape)  # noqa: E731
ONE_DIM = lambda rng, shape: np.where(np.arange(shape[-1]) == 3, rng.normal(0, 0.5, shape), 0.0)  # noqa: E731


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group,D", [(2, 64), (9, 64), (4, 128), (8, 128), (3, 256), (12, 256)])  # one wave a range; four
@pytest.mark.parametrize("exp", [-13, -17, -21, -30])
@pytest.mark.parametrize("values", [ZERO, LOW, ONE_DIM], ids=["zero", "low", "one_dim"])
def test_a_large_scale_of_small_values(values, exp, group, D, dt):
    c = Case([5, 2, 1], [2100, 130, 40], 2 * group, 2, D, D, 64, 16, dt, seed=40)
    q = with_a_block(c, values, 1.0, exp, 8.0)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse, tol=4e-3 if dt == torch.bfloat16 else 1e-5 + D * 2.0 ** -24 * 8.0)


@pytest.mark.parametrize("group,D", [(2, 64), (8, 128), (12, 256)])
@pytest.mark.parametrize("above", [0.0, 4.0, 16.0])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** 40])
def test_scores_of_the_block(scale, above, group, D):
    c = Case([5, 2, 1], [700, 130, 40], 2 * group, 2, D, D, 16, 16, torch.bfloat16, seed=41)
    q = with_a_block(c, ZERO, scale, -12, above)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [2, 8])
def test_values_that_are_all_zeros_of_any_scale(group, dt):
    c = Case([5, 2, 1], [700, 130, 40], 2 * group, 2, 128, 128, 64, 16, dt, seed=42)
    c.code["v"][:] = np.where(c.rng.random(c.code["v"].shape) < 0.5, 0, 0x80)
    c.scale["v"][:] = np.where(np.isnan(c.scale["v"]), np.nan, np.float32(1.0))
    q = torch.from_numpy(c.rng.normal(0, 1, (c.rows, c.Hq, 128)).astype(np.float32)).to(dt).to(dev())
    out, lse = attend(c, c.on_device(), q)
    assert bool((out == 0).all()) and bool(torch.isfinite(lse).all())
    # one value, in the last block that a row sees
    c.code["v"][c.table[0, (700 - 1) // 64], 1, (700 - 1) % 64, 5] = 0x38  # 1.0
    out, _ = attend(c, c.on_device(), q)
    o = to_f64(out)
    assert (o[4, group:, 5] > 0).all()
    o[4, group:, 5] = 0
    assert (o == 0).all()


@pytest.mark.parametrize("size", [0.003, 0.05])
@pytest.mark.parametrize("group,D", [(2, 64), (9, 64), (8, 128), (12, 256)])
def test_small_values_under_one_scale(group, D, size):
    c = Case([5, 2, 1], [2100, 130, 40], 2 * group, 2, D, D, 16, 16, torch.bfloat16, seed=44)
    c.code["v"] = np.where(c.code["v"] == 0x7f, 0x7f, e4m3(c.rng.normal(0, size, c.code["v"].shape)))
    c.scale["v"][:] = np.where(np.isnan(c.scale["v"]), np.nan, np.float32(1.0))
    q = torch.from_numpy(c.rng.normal(0, 1, (c.rows, c.Hq, D)).astype(np.float32)).to(c.dt).to(dev())
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("below", [20, 22, 24, 26, 28, 30])
def test_values_far_below_the_rows_largest(below):
    # values of 448 in one dim, and blocks whose p * s is 2^-below of those tokens': subnormal in fp16
    # at last, an error of 2^-25 where that is 2^7 or more, for 64 tokens' codes of at most 448
    c = Case([1], [64 + 16], 1, 1, 64, 64, 16, 16, torch.bfloat16, seed=43)
    q = torch.ones(1, 1, 64, dtype=torch.bfloat16, device=dev())
    c.code["k"][:] = 0
    c.scale["k"][:] = 1.0
    for i in range(5):
        c.scale["v"][c.table[0, i]] = 2.0 ** (0 if i == 2 else -below)
    c.code["v"][c.table[0, 2]] = 0
    c.code["v"][c.table[0, 2], :, :, 0] = 0x7e
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)
    v = c.values("v", 0)[0]
    want, got = v.mean(0), to_f64(out)[0, 0]
    log(f"[scaled] 2^-{below} below: worst of the other dims {np.abs(got[1:] / want[1:] - 1).max():.2e}")
    assert np.abs(got[1:] - want[1:]).max() <= 64 * 448 * 2.0 ** -25 / 2 ** 7 / 80 + 2.0 ** -9 * np.abs(want[1:]).max()
