"""GPU tests of what debug mode finds before pages are given back twice."""
import pytest
import torch

from gpu_helpers import dev
from paper_2607_05147_amd import dspark
from test_gpu_pages import Both, I

pytestmark = pytest.mark.gpu


def a_step(b, q_len, **kw):
    cu = torch.cat([I([0]), I(q_len).cumsum(0).int()])
    return cu, dspark.dspark_pages_reserve(b.table, b.kv, cu, 16, b.ref, b.bufs, **kw)


@pytest.mark.parametrize("stale", ["committed", "trimmed", "foreign"])
def test_debug_mode_looks_at_a_commit(stale, monkeypatch):
    monkeypatch.setenv("DSPARK_DEBUG", "1")
    b = Both([20, 7, 33], 16, 20, 4, seed=31)
    cu, step = a_step(b, [14, 30, 2])
    if stale == "committed":
        dspark.dspark_pages_commit(b.table, b.kv, step, cu, 16, b.ref, accepted_len=I([0, 0, 0]))
    elif stale == "trimmed":
        dspark.dspark_pages_trim(b.table, b.kv, I([64, 0, 64]), 16, b.ref)
    else:
        step[1] = 65
    before = [t.clone() for t in (b.table, b.kv, b.ref)]
    with pytest.raises(dspark.DSparkError, match="dspark_pages_commit.*request [01]"):
        dspark.dspark_pages_commit(b.table, b.kv, step, cu, 16, b.ref, accepted_len=I([0, 0, 0]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, t) for a, t in zip(before, (b.table, b.kv, b.ref)))


def test_debug_mode_passes_a_life(monkeypatch):
    monkeypatch.setenv("DSPARK_DEBUG", "1")
    b = Both([20, 0, 33, 16], 16, 20, 6, seed=32)
    b.fork([0], [1], [18])
    for accepted in ([0, 1, 2, 3], None, [-1, -1, -1, -1]):
        b.reserve([3, 4, 0, 17])
        b.commit(accepted)
    b.trim([5, 64, 0, 64])
    b.compact()
