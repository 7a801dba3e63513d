"""GPU test of a whole verify step on the 8-bit paged cache, as a server runs it: schedule,
reserve pages, append the new rows, attend, accept, commit.  Each stage against its reference
(the oracle's lengths and tokens, the pages' bookkeeping, the cache's codes and scales, all
exact; attention within its tolerance), then captured in a graph and replayed."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from gpu_helpers import dev, to_dev
from oracle import guard
from paper_2607_05147_amd import dspark, synth
from test_gpu_cache import Case, check_append, check_attention, expected, fill

pytestmark = pytest.mark.gpu

T = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev())  # noqa: E731


@pytest.mark.parametrize("name,R,lo,hi", [("serving", 8, 100, 3000), ("highconc", 24, 1, 400), ("tiny", 4, 20, 60)])
def test_a_verify_step_on_the_8_bit_cache(name, R, lo, hi):
    w = synth.scaled(synth.WORKLOADS[name], R=R)
    case = guard.build_case(w, 3, with_kv=False)
    bf16 = w.dtype == "bf16"
    dt = torch.bfloat16 if bf16 else torch.float32
    K, block = w.K, 16
    rng = np.random.default_rng(5)
    kv0 = rng.integers(lo, hi, R)
    # contexts as an earlier append left them, and a second holder of the first one's pages:
    # appending behind a shared, partly filled page copies it
    kv0[1] = kv0[0]
    c = Case(np.zeros(R, np.int64), kv0, w.Hq, w.Hkv, w.Dqk, w.Dv, w.page, block, dt, seed=5, max_q=K + 1, extra=R * (K // w.page + 2))
    max_pages = (int(kv0.max()) + K + 1 + w.page - 1) // w.page
    c.table = np.pad(c.table, ((0, 0), (0, max_pages - c.table.shape[1])), constant_values=-1)
    c.table[1] = c.table[0]
    parts = lambda: [c.code["k"], c.code["v"], c.scale["k"], c.scale["v"]]  # noqa: E731
    pages = ref.Pages(c.table, kv0.astype(np.int32), w.page, c.num_pages, parts())

    d = c.on_device()
    held = T(pages.ref)
    bufs = dspark.page_buffers([d["kc"], d["vc"], d["ks"], d["vs"]], c.num_pages)
    rows = R * (K + 1)
    c.rows = rows
    x = fill(c, dt)
    q = T(rng.normal(0, 1, (rows, w.Hq, w.Dqk)).astype(np.float32)).to(dt)
    conf, sps = to_dev(case.conf), to_dev(case.sps)
    logits, tok = to_dev(case.logits, w.logit_dtype == "bf16"), to_dev(case.drafts.draft_tok)
    dp = None if case.drafts.draft_p is None else to_dev(case.drafts.draft_p)
    u = None if case.drafts.u is None else to_dev(case.drafts.u)
    i32 = lambda *n: torch.empty(*n, dtype=torch.int32, device=dev())  # noqa: E731
    u8 = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device=dev())  # noqa: E731
    ln, cu, step_len, acc, nxt = i32(R), i32(R + 1), i32(R), i32(R), i32(R)
    out, lse = torch.empty(rows, w.Hq, w.Dv, dtype=dt, device=dev()), torch.empty(rows, w.Hq, device=dev())
    ws_s, ws_p = u8(dspark.dspark_schedule_workspace_size(R, K)), u8(dspark.dspark_pages_workspace_size(R, c.num_pages))
    ws_a = u8(dspark.dspark_verify_attn_scaled_workspace_size(R, K + 1, w.Hq, w.Hkv, w.Dqk, w.Dv, max_pages, w.page, block, dt))
    ws_c = u8(dspark.dspark_accept_workspace_size(R, K, w.V))

    def step():
        dspark.dspark_schedule(conf, sps, 0, len_out=ln, cu_q=cu, ws=ws_s)
        dspark.dspark_pages_reserve(d["table"], d["kv"], cu, w.page, held, bufs, step_len=step_len, ws=ws_p)
        dspark.dspark_cache_append(x["k"], x["v"], d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], block, d["table"],
                                   step_len, cu, K + 1, w.page)
        dspark.dspark_verify_attn_scaled(q, d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], block, d["table"], step_len, cu,
                                         K + 1, w.Dv, w.page, w.scale, out=out, lse=lse, ws=ws_a)
        dspark.dspark_accept(tok, logits, cu, draft_p=dp, u=u, accepted_len=acc, next_tok=nxt, ws=ws_c)
        dspark.dspark_pages_commit(d["table"], d["kv"], step_len, cu, w.page, held, accepted_len=acc)

    state = [d[n] for n in ("kc", "vc", "ks", "vs", "table", "kv")] + [held]
    start = [t.clone() for t in state]
    step()
    torch.cuda.synchronize()

    # lengths and tokens
    assert np.array_equal(ln.cpu().numpy(), case.len) and np.array_equal(cu.cpu().numpy(), case.cu_q)
    good = np.ones(R, bool)
    good[case.unguarded] = False
    assert np.array_equal(acc.cpu().numpy()[good], case.accepted_len[good])
    assert np.array_equal(nxt.cpu().numpy()[good], case.next_tok[good])
    # pages
    q_len = np.diff(case.cu_q)
    want_len = pages.reserve(q_len)
    assert np.array_equal(step_len.cpu().numpy(), want_len) and (want_len == kv0 + q_len).all()
    c.table = pages.table.copy()
    c.code["k"], c.code["v"], c.scale["k"], c.scale["v"] = [t.copy() for t in pages.contents]
    pages.commit(want_len, q_len, acc.cpu().numpy())
    assert np.array_equal(d["table"].cpu().numpy(), pages.table) and np.array_equal(d["kv"].cpu().numpy(), pages.kv)
    assert np.array_equal(held.cpu().numpy(), pages.ref)
    assert np.array_equal(pages.kv, kv0 + 1 + acc.cpu().numpy())
    # the cache and what was read from it
    c.kv, c.q_len, c.cu = want_len, q_len, case.cu_q
    check_append(c, d, expected(c, x))
    for n in ("k", "v"):
        c.code[n], c.scale[n] = c.unflat(n, d[n + "c"].cpu().numpy()), d[n + "s"].cpu().numpy()
    total = int(case.cu_q[-1])
    check_attention(c, q[:total], out[:total], lse[:total])

    results = state + [ln, cu, step_len, acc, nxt]
    want = [t.clone() for t in results] + [out[:total].clone(), lse[:total].clone()]
    g = torch.cuda.CUDAGraph()
    for t, s in zip(state, start):
        t.copy_(s)
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for t, s in zip(state, start):
            t.copy_(s)
        out.zero_()
        float((logits[:4].float() ** 2).sum())  # eager work and a synchronization between replays
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(results + [out[:total], lse[:total]], want):
            assert torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b)
