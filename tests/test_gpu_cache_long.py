"""GPU tests of dspark_verify_attn_scaled where a worker's range of keys is longer than the 128 pages
whose ids it holds: it reads the next ids and starts its copies again in the middle of the range.

A card's workers, 4 to 12 of a CU, share a batch's keys equally, so the batch has to have
millions; requests name the pages of a small pool again and again.  Tolerances are those of
test_gpu_cache.py: scores of a standard deviation of 2 leave a row's sum of 100000 values as
much weight as 2000 equally probable ones, and its rounding errors are random as theirs.
"""
import numpy as np
import pytest
import torch

from gpu_helpers import dev, log
from paper_2607_05147_amd import dspark
from test_gpu_cache import TOL

pytestmark = pytest.mark.gpu

CUS, MAX_WORKERS = 256, 12  # of a CU: registers allow no more (four waves of a SIMD at most, three for single ones)


def codes(g, *shape):
    x = torch.randn(*shape, generator=g, device=dev()).mul_(88).clamp_(-448, 448)
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,layout", [(16, "hnd"), (16, "nhd"), (48, "hnd")])
@pytest.mark.parametrize("D,Hkv,group,max_q", [(64, 1, 8, 1), (64, 2, 8, 3), (64, 2, 9, 8), (128, 2, 4, 2), (128, 1, 8, 4), (128, 2, 9, 8), (256, 1, 2, 2), (256, 1, 8, 5)],
                         ids=lambda x: str(x))
def test_ranges_of_more_pages_than_a_worker_holds(D, Hkv, group, max_q, page, layout, dt):
    rng = np.random.default_rng(page + D + group)
    g = torch.Generator(device=dev())
    g.manual_seed(D + group)
    pool, most = 500, 131072 // page * page
    keys = 0.9 * most  # of a request, on average
    R = int(130 * page * CUS * MAX_WORKERS / (Hkv * keys)) + 2
    kv = rng.integers(int(0.8 * most), most + 1, R)
    kv[1] = 40
    ql = rng.integers(1, max_q + 1, R)
    ql[0] = max_q
    table = rng.integers(0, pool, (R, most // page)).astype(np.int32)
    cu = np.concatenate([[0], np.cumsum(ql)]).astype(np.int32)
    strides = (Hkv * page * D, page * D, D) if layout == "hnd" else (page * Hkv * D, D, Hkv * D)
    view = (pool, Hkv, page, D) if layout == "hnd" else (pool, page, Hkv, D)
    cache = {n: codes(g, *view) for n in "kv"}
    scale = {n: torch.exp2(torch.randint(-2, 1, (pool, Hkv, page // 16), generator=g, device=dev()).float()) * (2 / 88 if n == "k" else 1 / 88)
             for n in "kv"}
    q = torch.randn(int(cu[-1]), Hkv * group, D, generator=g, device=dev()).to(dt)
    I = lambda a: torch.from_numpy(np.asarray(a, np.int32)).to(dev())  # noqa: E731
    out, lse = dspark.dspark_verify_attn_scaled(q, cache["k"].view(-1), cache["v"].view(-1), strides, strides, scale["k"], scale["v"], 16, I(table), I(kv),
                                                I(cu), max_q, D, page, D ** -0.5, want_lse=True)
    torch.cuda.synchronize()
    values = {n: (c if layout == "hnd" else c.transpose(1, 2)).contiguous().view(torch.float8_e4m3fn).double() *
              scale[n].double().repeat_interleave(16, 2)[..., None] for n, c in cache.items()}  # page, head, slot, dim
    worst = 0.0
    for r in [0, 1, R // 3, R // 2, R - 2, R - 1]:
        n, a = int(kv[r]), int(cu[r])
        ids = torch.from_numpy(table[r, : -(-n // page)]).to(dev()).long()
        for h in range(Hkv):
            k, v = (values[x][ids, h].reshape(-1, D)[:n] for x in "kv")
            qq = q[a:a + int(ql[r]), h * group:(h + 1) * group].double()
            z = qq.reshape(-1, D) @ k.T * D ** -0.5
            t = torch.arange(int(ql[r]), device=dev()).repeat_interleave(group)
            z.masked_fill_(torch.arange(n, device=dev())[None] > n - int(ql[r]) + t[:, None], float("-inf"))
            want_lse = torch.logsumexp(z, 1)
            want = torch.exp(z - want_lse[:, None]) @ v
            got = out[a:a + int(ql[r]), h * group:(h + 1) * group].double().reshape(-1, D)
            worst = max(worst, float(((got - want).norm(dim=1) / want.norm(dim=1)).max()))
            got_lse = lse[a:a + int(ql[r]), h * group:(h + 1) * group].double().reshape(-1)
            # scores up to about 12: 2^-24 of D terms' sum each (test_gpu_cache.py)
            assert float((got_lse - want_lse).abs().max()) <= 1e-4 * 2
    log(f"[long] R={R} {Hkv * group}/{Hkv} D={D} page {page} {layout} {dt}: worst row {worst:.2e}")
    assert worst <= TOL[dt]
