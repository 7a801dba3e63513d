"""GPU tests of dspark_cache_append without values: codes and scales, both exact (a latent cache,
whose values are a part of its keys)."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from gpu_helpers import to_f64
from paper_2607_05147_amd import dspark
from test_gpu_cache import Case, expected, fill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,page,block,layout,wide", [(576, 16, 16, "hnd", 0), (576, 64, 32, "nhd", 64), (64, 32, 16, "hnd", 8), (72, 16, 16, "hnd", 3)])
def test_keys_alone_have_their_codes_and_scales(D, page, block, layout, wide, dt):
    c = Case([3, 5, 0, 40], [40, 7, 20, 100], 2, 2, D, D, page, block, dt, layout, seed=45)
    x = fill(c, dt, wide)
    want, d = expected(c, x), c.on_device()
    values, scales = d["vc"].clone(), d["vs"].clone()
    for _ in range(2):  # the same rows again: the same cache
        dspark.dspark_cache_append(x["k"], None, d["kc"], None, c.strides["k"], None, d["ks"], None, c.block, d["table"], d["kv"], d["cu"],
                                   c.max_q, c.page)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(ref.VALUES[c.unflat("k", d["kc"].cpu().numpy())], want["k"])
        np.testing.assert_array_equal(d["ks"].cpu().numpy(), want["ks"])
    assert torch.equal(d["vc"], values) and np.array_equal(to_f64(d["vs"]), to_f64(scales), equal_nan=True)


@pytest.mark.parametrize("old", [2.0 ** -20, 2.0 ** 3, 0.3])
def test_keys_alone_behind_tokens_of_any_scale(old):
    c = Case([3], [20 + 3], 1, 1, 576, 576, 32, 32, torch.bfloat16, seed=46)
    c.scale["k"][:] = np.float32(old)
    x = fill(c, torch.bfloat16)
    want, d = expected(c, x), c.on_device()
    dspark.dspark_cache_append(x["k"], None, d["kc"], None, c.strides["k"], None, d["ks"], None, c.block, d["table"], d["kv"], d["cu"], c.max_q, c.page)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(ref.VALUES[c.unflat("k", d["kc"].cpu().numpy())], want["k"])
    np.testing.assert_array_equal(d["ks"].cpu().numpy(), want["ks"])
