"""GPU tests of dspark_verify_attn_scaled on the vector ALUs where a large batch is cut into fewer
splits than its contexts ask for, and with a workspace that a larger batch sized."""
import numpy as np
import pytest
import torch

from gpu_helpers import dev
from paper_2607_05147_amd import dspark
from test_gpu_cache import Case, attend, check_attention, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,splits", [(90, 8), (110, 6), (300, 2), (800, 1)])
def test_fewer_splits_of_large_batches(R, splits, dt):
    rng = np.random.default_rng(R)
    kv, ql = rng.integers(17, 60, R), rng.integers(1, 3, R)
    long = [0, R // 2, R - 1]
    kv[long], ql[long] = [8100, 1025, 3000], [17, 1, 5]
    assert min(8, max(1, 786432 // (R * 17 * 64))) == splits
    c = Case(ql, kv, 64, 2, 24, 40, 64, 16, dt, seed=R)
    q, d = queries(c), c.on_device()
    out, lse = attend(c, d, q)
    check_attention(c, q, out, lse, requests=[*long, 1, R // 3])
    # the workspace of twice the batch
    n = dspark.dspark_verify_attn_scaled_workspace_size(2 * R, c.max_q, 64, 2, 24, 40, c.table.shape[1], 64, 16, dt)
    again, _ = attend(c, d, q, ws=torch.empty(n, dtype=torch.uint8, device=dev()))
    assert torch.equal(again, out)
