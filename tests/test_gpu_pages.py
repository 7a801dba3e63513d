"""GPU tests of dspark_pages_* against the page-at-a-time bookkeeping of
cache_reference.Pages: tables, holders, lengths and page contents, all exact."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from gpu_helpers import dev, log
from paper_2607_05147_amd import dspark

pytestmark = pytest.mark.gpu

T = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev())  # noqa: E731
I = lambda a: T(np.asarray(a, np.int32))  # noqa: E731


class Both:
    """The same state on the device and in the reference."""

    def __init__(self, kv, page, num_pages, max_pages, seed=0, sizes=(48, 7, 4), shift=0):
        rng = np.random.default_rng(seed)
        kv = np.asarray(kv, np.int32)
        R = len(kv)
        held = -(-kv // page)
        perm = rng.permutation(num_pages)
        table = rng.integers(-5, num_pages + 5, (R, max_pages)).astype(np.int32)  # entries past the held ones mean nothing
        at = 0
        for r in range(R):
            table[r, :held[r]] = perm[at:at + held[r]]
            at += held[r]
        self.m = ref.Pages(table, kv, page, num_pages, [rng.integers(0, 256, (num_pages, b), dtype=np.uint8) for b in sizes])
        self.page = page
        self.table, self.kv, self.ref = T(self.m.table), T(self.m.kv), T(self.m.ref)
        self.contents = [T(c) for c in self.m.contents]
        self.bufs = dspark.page_buffers(self.contents, num_pages)
        self.step = self.step_ref = None

    def same(self, what):
        torch.cuda.synchronize()
        np.testing.assert_array_equal(self.table.cpu().numpy(), self.m.table, err_msg=what + ": table")
        np.testing.assert_array_equal(self.kv.cpu().numpy(), self.m.kv, err_msg=what + ": kv_len")
        np.testing.assert_array_equal(self.ref.cpu().numpy(), self.m.ref, err_msg=what + ": ref")
        for i, (a, b) in enumerate(zip(self.contents, self.m.contents)):
            np.testing.assert_array_equal(a.cpu().numpy(), b, err_msg=f"{what}: buffer {i}")

    def fork(self, parent, child, length=None):
        dspark.dspark_pages_fork(self.table, self.kv, self.page, self.ref, I(parent), I(child), None if length is None else I(length))
        self.m.fork(parent, child, length)
        self.same("fork")

    def reserve(self, q_len):
        self.q_len, self.cu = np.asarray(q_len), I(np.concatenate([[0], np.cumsum(q_len)]))
        self.step = dspark.dspark_pages_reserve(self.table, self.kv, self.cu, self.page, self.ref, self.bufs)
        self.step_ref = self.m.reserve(self.q_len)
        torch.cuda.synchronize()
        np.testing.assert_array_equal(self.step.cpu().numpy(), self.step_ref, err_msg="reserve: step_len")
        self.same("reserve")

    def commit(self, accepted=None):
        dspark.dspark_pages_commit(self.table, self.kv, self.step, self.cu, self.page, self.ref, None if accepted is None else I(accepted))
        self.m.commit(self.step_ref, self.q_len, accepted)
        self.same("commit")

    def trim(self, new_len):
        dspark.dspark_pages_trim(self.table, self.kv, I(new_len), self.page, self.ref)
        self.m.trim(new_len)
        self.same("trim")

    def compact(self):
        used = dspark.dspark_pages_compact(self.table, self.kv, self.page, self.ref, self.bufs)
        want = self.m.compact()
        self.same("compact")
        assert int(used) == want


@pytest.mark.parametrize("R,page,num_pages", [(1, 16, 12), (5, 16, 60), (70, 32, 1100), (300, 16, 5000), (1500, 16, 12000), (8192, 16, 40000)])
def test_a_life_of_steps(R, page, num_pages):
    rng = np.random.default_rng(R)
    most = min(num_pages // (2 * R) + 3, 40) * page
    b = Both(rng.integers(0, most // 2, R), page, num_pages, most // page + 8, seed=R)
    for step in range(6):
        empty = np.flatnonzero(b.m.kv == 0)
        full = np.flatnonzero(b.m.kv > 0)
        if len(empty) and len(full):
            n = min(len(empty), R // 3 + 1)
            parent = rng.choice(full, n)
            b.fork(parent, rng.choice(empty, n, replace=False), None if step % 2 else rng.integers(0, most, n))
        q = rng.integers(0, 18, R)
        q = np.where(b.m.kv + q <= b.m.table.shape[1] * page, q, 0)
        b.reserve(q)
        b.commit(None if step == 2 else rng.integers(-1, 18, R))
        b.trim(np.where(rng.random(R) < 0.25, rng.integers(0, most, R) * (rng.random(R) < 0.5), 1 << 30))
        if step % 2:
            b.compact()
    log(f"[pages] R={R}: {int((b.m.ref > 0).sum())} of {num_pages} pages in use")


@pytest.mark.parametrize("grow", [[1, 1, 1], [1, 1, 0], [0, 1, 1], [1, 0, 0], [0, 0, 0], [17, 1, 40]])
def test_who_copies_a_shared_page(grow):
    # three holders of a partly filled page: all grow, some, one
    b = Both([21, 0, 0, 5], 16, 20, 8, seed=1)
    b.fork([0, 0], [1, 2])
    b.reserve(grow + [1])
    b.commit()
    b.reserve([1] * 4)
    b.commit([0] * 4)
    b.trim([0, 0, 0, 0])
    assert not b.m.ref.any()


def test_forks_that_end_inside_a_parents_page():
    b = Both([40, 0, 0, 0], 16, 20, 8, seed=2)
    b.fork([0, 0, 0], [1, 2, 3], [21, 32, 0])
    b.reserve([1, 3, 2, 1])
    b.commit()


@pytest.mark.parametrize("free", range(0, 9))
def test_shortage_serves_in_order(free):
    # needs 1 + copy, 1 + copy, (keeps), 2, 0, 1 pages with 0 .. 8 of them free
    held = 2 + 0 + 0 + 1 + 1 + 1
    b = Both([30, 0, 0, 16, 3, 16], 16, held + free, 8, seed=3)
    b.fork([0, 0], [1, 2])
    b.reserve([10, 10, 2, 32, 2, 1])
    b.commit()


def test_no_page_free_and_nothing_needed():
    b = Both([16, 15, 0], 16, 2, 4, seed=4)
    b.reserve([0, 1, 0])
    b.commit()
    b.reserve([1, 1, 1])
    assert b.step_ref.tolist() == [0, 0, 0]
    b.commit()


def test_fork_pairs_that_are_skipped():
    b = Both([20, 7, 0, 0, 0], 16, 20, 4, seed=5)
    b.fork([0, 0, 1, 3, 9], [1, 2, 2, 3, 4])
    b.fork([2, 3, -1, 0], [3, 4, 0, 1 << 20])


def test_compact_edges():
    for kv, n in (([], 0), ([16], 1), ([16] * 3, 3), ([16, 16], 1025), ([0], 5)):
        if not len(kv):
            continue
        b = Both(kv, 16, max(n, 1), 3, seed=6)
        b.compact()
        b.compact()


@pytest.mark.parametrize("sizes", [(16384 * 3 + 16, 64), (1, 2, 3, 5, 20), (16,) * 70, (512, 516, 511, 16384, 8, 528, 513),
                                   tuple(1024 + 16 * i if i % 3 else 12 + i for i in range(130))], ids=range(5))
def test_copies_of_every_size(sizes):
    b = Both([5, 0, 70, 3], 16, 40, 8, seed=7, sizes=sizes)
    b.fork([0], [1])
    b.reserve([1, 1, 1, 1])
    b.compact()


def test_buffers_of_pages_that_lie_apart():
    # page_stride above page_bytes, through the C struct
    n, stride, size = 12, 80, 48
    base = torch.randint(0, 256, (n, stride), dtype=torch.uint8, device=dev())
    before = base.clone()
    b = Both([5, 0], 16, n, 4, seed=8, sizes=())
    b.fork([0], [1])
    bufs = dspark.page_buffers([base], n)
    bufs.array[0].page_bytes = size
    old = int(b.m.table[0, 0])
    b.cu = I([0, 1, 2])
    dspark.dspark_pages_reserve(b.table, b.kv, b.cu, 16, b.ref, bufs)
    torch.cuda.synchronize()
    new = int(b.table[0, 0])
    assert new != old and int(b.table[1, 0]) == old  # the last holder keeps it
    before[new, :size] = before[old, :size]
    assert torch.equal(base, before)


def test_malformed_state_is_passed_over():
    b = Both([20, 20, 20, 20, 20, 20], 16, 40, 4, seed=9)
    b.kv[0], b.kv[1] = -4, 10 ** 6
    b.table[2, 1] = 40          # the partly filled page is outside the cache
    b.table[3, 1] = -1
    cu = I([0, 1, 2, 3, 4, 3, 4])  # request 4: a negative count
    ref0 = b.ref.clone()
    step = dspark.dspark_pages_reserve(b.table, b.kv, cu, 16, b.ref, b.bufs)
    torch.cuda.synchronize()
    assert step.cpu().tolist() == [0, 0, 0, 0, 0, 21] and torch.equal(b.ref, ref0)
    kv = b.kv.clone()
    dspark.dspark_pages_commit(b.table, b.kv, step, cu, 16, b.ref)
    kv[5] = 21
    torch.cuda.synchronize()
    assert torch.equal(b.kv, kv) and torch.equal(b.ref, ref0)
    dspark.dspark_pages_trim(b.table, b.kv, I([0] * 6), 16, b.ref)
    used = dspark.dspark_pages_compact(b.table, b.kv, 16, b.ref, b.bufs)
    torch.cuda.synchronize()
    # requests 0 and 1 were never ended, of 2 and 3 a page each was not named
    assert b.kv.cpu().tolist() == [-4, 10 ** 6, 0, 0, 0, 0] and int(used) == 6


def test_a_step_of_pages_in_a_graph():
    rng = np.random.default_rng(10)
    R, page, n = 40, 16, 900
    b = Both(np.where(np.arange(R) % 4 == 0, rng.integers(1, 200, R), 0), page, n, 20, seed=10)
    parent, child = I(np.repeat(np.arange(0, R, 4), 3)), I(np.setdiff1d(np.arange(R), np.arange(0, R, 4)))
    q_len = rng.integers(1, 9, R)
    acc = rng.integers(0, q_len)
    new = np.where(np.arange(R) % 4 == 1, 1 << 30, 0)
    cu, accd, newd = I(np.concatenate([[0], np.cumsum(q_len)])), I(acc), I(new)
    ws = torch.empty(dspark.dspark_pages_workspace_size(R, n), dtype=torch.uint8, device=dev())
    step, used = torch.zeros(R, dtype=torch.int32, device=dev()), torch.zeros(1, dtype=torch.int32, device=dev())
    state = [b.table, b.kv, b.ref, *b.contents]
    start = [t.clone() for t in state]

    def life():
        dspark.dspark_pages_fork(b.table, b.kv, page, b.ref, parent, child, ws=ws)
        dspark.dspark_pages_reserve(b.table, b.kv, cu, page, b.ref, b.bufs, step_len=step, ws=ws)
        dspark.dspark_pages_commit(b.table, b.kv, step, cu, page, b.ref, accepted_len=accd)
        dspark.dspark_pages_trim(b.table, b.kv, newd, page, b.ref)
        dspark.dspark_pages_compact(b.table, b.kv, page, b.ref, b.bufs, used=used, ws=ws)

    life()
    b.m.fork(parent.cpu().numpy(), child.cpu().numpy())
    st = b.m.reserve(q_len)
    b.m.commit(st, q_len, acc)
    b.m.trim(new)
    want = b.m.compact()
    b.same("eager")
    g = torch.cuda.CUDAGraph()
    for t, s in zip(state, start):
        t.copy_(s)
    with torch.cuda.graph(g):
        life()
    for rep in range(3):
        for t, s in zip(state, start):
            t.copy_(s)
        float(torch.ones(100, device=dev()).sum())
        g.replay()
        b.same(f"replay {rep}")
        assert int(used) == want


def test_checks_and_refusals(monkeypatch):
    b = Both([20, 7, 33], 16, 20, 4, seed=11)
    find = lambda: dspark.check_page_inputs(b.table, b.kv, 16, b.ref)  # noqa: E731
    assert find() is None
    b.ref[b.table[2, 1].long()] = 0
    assert find()[:4] == (3, 2, 1, int(b.table[2, 1]))
    b.table[2, 0] = 20
    assert find()[:4] == (2, 2, 0, 20)
    b.kv[0] = 65
    assert find()[:4] == (1, 0, 0, 65)
    monkeypatch.setenv("DSPARK_DEBUG", "1")
    for call in (lambda: dspark.dspark_pages_reserve(b.table, b.kv, I([0, 1, 2, 3]), 16, b.ref, b.bufs),
                 lambda: dspark.dspark_pages_trim(b.table, b.kv, I([0, 0, 0]), 16, b.ref),
                 lambda: dspark.dspark_pages_fork(b.table, b.kv, 16, b.ref, I([0]), I([1])),
                 lambda: dspark.dspark_pages_compact(b.table, b.kv, 16, b.ref, b.bufs)):
        with pytest.raises(dspark.DSparkError, match="request 0"):
            call()
    monkeypatch.delenv("DSPARK_DEBUG")
    for call in (lambda: dspark.dspark_pages_reserve(b.table, b.kv, I([0, 1, 2]), 16, b.ref, b.bufs),
                 lambda: dspark.dspark_pages_reserve(b.table, b.kv, I([0, 1, 2, 3]), 16, b.ref, b.bufs, step_len=b.kv),
                 lambda: dspark.dspark_pages_reserve(b.table, b.kv, I([0, 1, 2, 3]), 16, b.ref[:5], b.bufs),
                 lambda: dspark.dspark_pages_reserve(b.table, b.kv, I([0, 1, 2, 3]), 24, b.ref, b.bufs),
                 lambda: dspark.dspark_pages_reserve(b.table, b.kv, I([0, 1, 2, 3]), 16, b.ref, b.bufs, ws=torch.empty(8, dtype=torch.uint8, device=dev())),
                 lambda: dspark.dspark_pages_trim(b.table, b.kv, I([0, 0]), 16, b.ref),
                 lambda: dspark.dspark_pages_fork(b.table, b.kv, 16, b.ref, I([0, 0, 0, 0]), I([1, 1, 1, 1])),
                 lambda: dspark.dspark_pages_fork(b.table, b.kv, 16, b.ref, I([0]), I([1, 2])),
                 lambda: dspark.page_buffers([torch.zeros(7, device=dev())], 20),
                 lambda: dspark.page_buffers([torch.zeros(40)], 20)):
        with pytest.raises(dspark.DSparkError):
            call()
