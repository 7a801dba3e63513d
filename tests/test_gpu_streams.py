"""GPU tests of calls on another stream than the current one that allocate what they were not
given: it has to be memory of the call's stream, since the allocator hands out a block of the
current stream's as soon as it is freed there, before the kernels that use it have run."""
import numpy as np
import pytest
import torch

from gpu_helpers import dev
from paper_2607_05147_amd import dspark
from test_gpu_cache import Case, attend, queries

pytestmark = pytest.mark.gpu

I = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev())  # noqa: E731
F = lambda *n: torch.rand(*n, device=dev())  # noqa: E731
B = lambda *n: (torch.rand(*n, device=dev()) - 0.5).bfloat16()  # noqa: E731


def _pages():
    return torch.arange(8, dtype=torch.int32, device=dev()).view(2, 4), I(20, 7), 16, I(1, 1, 0, 0, 1, 0, 0, 0)


def _attention(s):
    st = (2 * 16 * 64, 16 * 64, 64)
    return dspark.dspark_verify_attn(B(3, 4, 64), B(8 * 2 * 16 * 64), B(8 * 2 * 16 * 64), st, st, _pages()[0], I(20, 7), I(0, 1, 3), 2, 2, 64, 16,
                                     0.1, want_lse=True, stream=s)


def _scaled(s):
    c = Case([3, 1], [300, 90], 16, 2, 128, 128, 64, 64, torch.bfloat16, seed=19)
    return attend(c, c.on_device(), queries(c), stream=s)


def _fork(s):
    table, kv, page, ref = _pages()
    kv[1] = 0
    return dspark.dspark_pages_fork(table, kv, page, ref, I(0), I(1), stream=s)


def _draft(s, rnn):
    R, K, V, rank = 2, 3, 256, 64
    more = (B(3 * rank, 2 * rank),) if rnn else ()
    f = dspark.dspark_rnn_draft if rnn else dspark.dspark_markov_draft
    return f(I(1, 2), B(R * K, V), B(V, rank), B(V, rank), *more, F(rank), F(R, K), K, stream=s)


CALLS = {
    "schedule": lambda s: dspark.dspark_schedule(F(4, 3), torch.arange(17, 0, -1, device=dev()).double(), want_tok_req=True, stream=s),
    "capacity": lambda s: dspark.dspark_schedule_capacity(F(4, 3), torch.arange(17, 0, -1, device=dev()).double(), stream=s),
    "topk": lambda s: dspark.dspark_schedule_topk(F(4, 3), I(9), want_tok_req=True, stream=s),
    "verify_attn": _attention,
    "verify_attn_scaled": _scaled,
    "reserve": lambda s: dspark.dspark_pages_reserve(*_pages()[:2], I(0, 1, 2), *_pages()[2:], stream=s),
    "fork": _fork,
    "compact": lambda s: dspark.dspark_pages_compact(*_pages(), stream=s),
    "accept": lambda s: dspark.dspark_accept(I(1, 2, 3, 4).view(2, 2), F(6, 100), I(0, 3, 6), draft_p=F(2, 2, 100) / 50, u=F(2, 3), want_rate=True,
                                             stream=s),
    "markov": lambda s: _draft(s, False),
    "rnn": lambda s: _draft(s, True),
    "check_verify": lambda s: dspark.check_verify_inputs(_pages()[0], I(20, 7), I(0, 1, 2), 1, 16, 8, stream=s),
    "check_accept": lambda s: dspark.check_accept_inputs(I(0, 1, 2), None, 2, stream=s),
    "check_schedule": lambda s: dspark.check_schedule_inputs(F(2, 2), stream=s),
    "check_draft": lambda s: dspark.check_draft_inputs(F(2, 2), stream=s),
    "check_page": lambda s: dspark.check_page_inputs(*_pages(), stream=s),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_what_a_call_allocates_is_its_streams(name, monkeypatch):
    s = torch.cuda.Stream()
    # (inputs come from the current stream, with a wait before the library's call)
    lib, made, empty = dspark.lib(), [], torch.empty

    def seen(*a, **kw):
        made.append(torch.cuda.current_stream().cuda_stream)
        return empty(*a, **kw)

    class Waiting:
        def __getattr__(self, f):
            torch.cuda.synchronize()
            return getattr(lib, f)

    monkeypatch.setattr(dspark, "lib", lambda: Waiting())
    monkeypatch.setattr(dspark.torch, "empty", seen)
    out = CALLS[name](s)
    torch.cuda.synchronize()
    assert made and set(made) == {s.cuda_stream}
    # the allocator's own account of the tensors that came back
    segments = torch.cuda.memory_snapshot()
    for t in out if isinstance(out, tuple) else [out]:
        if isinstance(t, torch.Tensor):
            (owner,) = [g["stream"] for g in segments if g["address"] <= t.data_ptr() < g["address"] + g["total_size"]]
            assert owner == s.cuda_stream


def test_a_block_that_the_current_stream_still_writes():
    c = Case([3, 1], [300, 90], 16, 2, 128, 128, 64, 64, torch.bfloat16, seed=19)
    d, q = c.on_device(), queries(c)
    want, want_lse = attend(c, d, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    need = dspark.dspark_verify_attn_scaled_workspace_size(c.R, c.max_q, c.Hq, c.Hkv, 128, 128, d["table"].shape[1], c.page, c.block, c.dt)
    for _ in range(3):
        late = [torch.empty(n, dtype=torch.uint8, device=dev()) for n in (need, want.numel() * 2, want_lse.numel() * 4)]
        torch.cuda._sleep(1 << 20)
        for t in late:
            t.fill_(0xff)
        del late, t
        out, lse = dspark.dspark_verify_attn_scaled(q, d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], c.block, d["table"],
                                                    d["kv"], d["cu"], c.max_q, c.Dv, c.page, c.Dqk ** -0.5, want_lse=True, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_results_read_on_the_current_stream_live_until_it_has_read_them():
    # the other way round: freed while the current stream still reads, not handed to the call's stream
    c = Case([3, 1], [300, 90], 16, 2, 128, 128, 64, 64, torch.bfloat16, seed=19)
    d, q = c.on_device(), queries(c)
    want, _ = attend(c, d, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, _ = dspark.dspark_verify_attn_scaled(q, d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], c.block, d["table"], d["kv"],
                                              d["cu"], c.max_q, c.Dv, c.page, c.Dqk ** -0.5, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    at = out.data_ptr()
    torch.cuda._sleep(1 << 24)
    got = out.clone()
    del out
    with torch.cuda.stream(s):
        other = torch.full(want.shape, 7.0, dtype=want.dtype, device=dev())
    assert other.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_captured_call_on_a_side_stream_that_allocates():
    c = Case([3, 1], [300, 90], 16, 2, 128, 128, 64, 64, torch.bfloat16, seed=19)
    d, q = c.on_device(), queries(c)
    want, want_lse = attend(c, d, q)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.wait_stream(torch.cuda.current_stream())
        out, lse = dspark.dspark_verify_attn_scaled(q, d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], c.block, d["table"],
                                                    d["kv"], d["cu"], c.max_q, c.Dv, c.page, c.Dqk ** -0.5, want_lse=True, stream=s)
        torch.cuda.current_stream().wait_stream(s)
    for _ in range(3):
        out.zero_(), lse.zero_()
        float((q.float() * q.float()).sum())  # eager work and a synchronization between replays
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
