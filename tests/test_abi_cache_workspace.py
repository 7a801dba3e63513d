"""Workspace sizes of dspark_verify_attn_scaled (no GPU): what the vector-ALU path's partials
may take stops growing with the batch, and never shrinks with it."""
import os

import pytest
import torch

from paper_2607_05147_amd import dspark


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(dspark.LIB_PATH):
        from paper_2607_05147_amd import build
        build.build()


def size(R, max_q=17, Hq=64, Hkv=8, D=128, max_pages=256, page=64, dt=torch.bfloat16):
    return dspark.dspark_verify_attn_scaled_workspace_size(R, max_q, Hq, Hkv, D, D, max_pages, page, 16, dt)


def test_a_large_batch_needs_little_more_than_its_rows():
    row = (128 + 2) * 4
    bound = 786432 * row
    assert size(128) <= bound and size(512) <= bound  # 8 splits of each: 579 MB, 2.3 GB
    # from there on a partial for each row
    assert size(2048) == 2048 * 17 * 64 * row


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 72, 128, 576])
def test_a_workspace_serves_the_smaller_batches(D, dt):
    for max_q in (1, 9, 17):
        sizes = [size(R, max_q, D=D, dt=dt) for R in range(1, 1500)]
        assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
    sizes = [size(300, max_q, D=D, dt=dt) for max_q in range(1, 66)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
