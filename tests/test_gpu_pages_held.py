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


@pytest.mark.parametrize("num_pages", [20, 8192, 8193, 30000])
def test_a_page_that_more_entries_name_than_its_ref(num_pages):
    find = lambda: dspark.check_page_inputs(b.table, b.kv, 16, b.ref)  # noqa: E731
    b = Both([20, 0, 33, 0, 64], 16, num_pages, 4, seed=33)
    b.fork([0, 2], [1, 3])
    assert find() is None
    shared = int(b.table[2, 1])
    assert int(b.ref[shared]) == 2
    b.ref[shared] = 1
    assert find()[:4] == (4, 2, 1, shared)
    b.ref[int(b.table[2, 2])] = 1   # a later page of the same request
    assert find()[:4] == (4, 2, 1, shared)
    other = int(b.table[0, 1])
    b.ref[other] = 1                # an earlier request's
    assert find()[:4] == (4, 0, 1, other)
    b.ref[other] = 3                # more holders than entries may be a step's
    assert find()[:4] == (4, 2, 1, shared)
    b.ref[int(b.table[4, 3])] = 0   # the other rules come first, whatever the request
    assert find()[:4] == (3, 4, 3, int(b.table[4, 3]))


def test_a_page_given_back_twice_and_handed_out_again(monkeypatch):
    # request 0's step is committed a second time after request 1 took the page that it gave back
    b = Both([16, 16], 16, 4, 4, seed=34)
    cu, step = a_step(b, [9, 0])
    dspark.dspark_pages_commit(b.table, b.kv, step, cu, 16, b.ref, accepted_len=I([-1, -1]))
    assert b.kv.tolist() == [16, 16]
    cu2, step2 = a_step(b, [0, 9])
    dspark.dspark_pages_commit(b.table, b.kv, step2, cu2, 16, b.ref)
    assert int(b.table[0, 1]) == int(b.table[1, 1])
    monkeypatch.setenv("DSPARK_DEBUG", "1")
    # (request 1's step has its page, so that both name it)
    stale = torch.stack([step[0], step2[1]])
    with pytest.raises(dspark.DSparkError, match="request 0.*more entries"):
        dspark.dspark_pages_commit(b.table, b.kv, stale, I([0, 9, 18]), 16, b.ref, accepted_len=I([-1, 8]))


def test_as_many_requests_and_entries_as_a_server_has():
    R, n = 8192, 20000
    b = Both([16 * (1 + r % 3) if r % 2 == 0 else 0 for r in range(R)], 16, n, 4, seed=35, sizes=())
    dspark.dspark_pages_fork(b.table, b.kv, 16, b.ref, I(range(0, R, 2)), I(range(1, R, 2)))
    assert dspark.check_page_inputs(b.table, b.kv, 16, b.ref) is None
    at = int(b.table[8191, 0])
    b.ref[at] = 1
    assert dspark.check_page_inputs(b.table, b.kv, 16, b.ref)[:4] == (4, 8190, 0, at)
