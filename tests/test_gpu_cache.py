"""GPU tests of the paged cache in 8 bits: dspark_cache_append and
dspark_verify_attn_scaled against plain fp64 implementations.

Tolerances.  Appending is compared exactly: with scales that are powers of two a
code is one rounding of an exact quotient.  Attention: codes and scales are exact,
so the error is that of the arithmetic.  bf16: the output's rounding is at most
2^-8 / 2 per value (half a step of 2^-8 relative, eps / 2 = 2^-9 on the mean of a
binade's two ends), a probability times its value's scale is rounded once to fp16,
2^-11 of itself or 2^-25, where the row's largest is 2^7 or more: 2^-12 in the mean
of squares; per row in the 2-norm the output's rounding alone is below 2^-8: 4e-3.
fp32: three bf16 terms are exact to 2^-24, a score sums up to 256 products in fp32,
256 * 2^-24 * sum |q k| at worst and its square root in practice; with |scores| up to
about 8 the probabilities move by at most a few 1e-6 relative: 1e-5, the existing fp32
tolerance of this attention.
"""
import numpy as np
import pytest
import torch

import cache_reference as ref
from gpu_helpers import dev, log, to_f64
from paper_2607_05147_amd import dspark

pytestmark = pytest.mark.gpu

TOL = {torch.bfloat16: 4e-3, torch.float32: 1e-5}


class Case:
    """Contexts in a paged cache of codes, in shuffled pages; page 0 .. and slots past the
    contexts hold NaN codes and their scales NaN."""

    def __init__(self, q_len, kv, Hq, Hkv, Dqk, Dv, page, block, dt=torch.bfloat16, layout="hnd", pad=0, seed=0, extra=2,
                 scale_exp=(-8, -5), max_q=None):
        rng = self.rng = np.random.default_rng(seed)
        self.q_len, self.kv = np.asarray(q_len), np.asarray(kv)
        self.Hq, self.Hkv, self.Dqk, self.Dv, self.page, self.block, self.dt = Hq, Hkv, Dqk, Dv, page, block, dt
        R = self.R = len(self.kv)
        self.max_q = max(int(self.q_len.max()), 1) if max_q is None else max_q
        npg = -(-self.kv // page)
        self.num_pages = int(npg.sum()) + extra
        perm = rng.permutation(self.num_pages)
        self.table = np.full((R, max(1, int(npg.max()))), -1, np.int32)
        at = 0
        for r in range(R):
            self.table[r, :npg[r]] = perm[at:at + npg[r]]
            at += npg[r]
        self.cu = np.concatenate([[0], np.cumsum(self.q_len)]).astype(np.int32)
        self.rows = int(self.cu[-1])
        self.code, self.scale, self.strides = {}, {}, {}
        for name, D in (("k", Dqk), ("v", Dv)):
            # [page, head, slot, dim], every slot NaN until a context fills it
            c = np.full((self.num_pages, Hkv, page, D), 0x7f, np.uint8)
            s = np.full((self.num_pages, Hkv, page // block), np.nan, np.float32)
            x = np.clip(rng.normal(0, 88, (int(self.kv.sum()), Hkv, D)), -448, 448)
            x = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
            at = 0
            for r in range(R):
                for j in range(int(self.kv[r])):
                    c[self.table[r, j // page], :, j % page] = x[at]
                    if j % block == 0:
                        s[self.table[r, j // page], :, j % page // block] = 2.0 ** rng.integers(*scale_exp, Hkv)
                    at += 1
            self.code[name], self.scale[name] = c, s
            row = D + pad
            self.strides[name] = (Hkv * page * row, page * row, row) if layout == "hnd" else (page * Hkv * row, row, Hkv * row)

    def flat(self, name):
        """The codes as the strides lay them out."""
        c = self.code[name]
        s0, s1, s2 = self.strides[name]
        out = np.full(self.num_pages * s0, 0x7f, np.uint8)
        v = np.lib.stride_tricks.as_strided(out, c.shape, (s0, s1, s2, 1))
        v[:] = c
        return out

    def unflat(self, name, flat):
        return np.lib.stride_tricks.as_strided(flat, self.code[name].shape, (*self.strides[name], 1)).copy()

    def on_device(self):
        T = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev())  # noqa: E731
        i32 = lambda a: T(np.asarray(a, np.int32))  # noqa: E731
        return dict(kc=T(self.flat("k")), vc=T(self.flat("v")), ks=T(self.scale["k"]), vs=T(self.scale["v"]), table=i32(self.table),
                    kv=i32(self.kv), cu=i32(self.cu))

    def values(self, name, r):
        """[Hkv, kv, D] of request r, fp64."""
        j = np.arange(int(self.kv[r]))
        pg, sl = self.table[r, j // self.page], j % self.page
        x = ref.VALUES[self.code[name][pg, :, sl]] * self.scale[name][pg, :, sl // self.block][..., None].astype(np.float64)
        return x.transpose(1, 0, 2)


def attend(c, d, q, **kw):
    out, lse = dspark.dspark_verify_attn_scaled(q, d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], c.block, d["table"],
                                                d["kv"], d["cu"], c.max_q, c.Dv, c.page, c.Dqk ** -0.5, want_lse=True, **kw)
    torch.cuda.synchronize()
    return out, lse


def queries(c):
    x = torch.from_numpy(c.rng.normal(0, 1, (c.rows, c.Hq, c.Dqk)).astype(np.float32))
    return x.to(c.dt).to(dev())


def check_attention(c, q, out, lse, requests=None, tol=None):
    o, q64, l = to_f64(out), to_f64(q), to_f64(lse)
    worst = 0.0
    for r in range(c.R) if requests is None else requests:
        a, ql = int(c.cu[r]), int(c.q_len[r])
        if ql == 0:
            continue
        want, want_lse = ref.attention(q64[a:a + ql], c.values("k", r), c.values("v", r), int(c.kv[r]), ql, c.Hq // c.Hkv, c.Dqk ** -0.5)
        err = np.linalg.norm(o[a:a + ql] - want, axis=2) / np.linalg.norm(want, axis=2)
        worst = max(worst, float(err.max()))
        # a score is a sum of Dqk fp32 products: 2^-24 of its terms' sum each, and 2^-23 in exp2 units
        assert (np.abs(l[a:a + ql] - want_lse) <= 1e-4 * np.maximum(1.0, np.abs(want_lse) / 8)).all()
    log(f"[scaled] R={c.R} {c.Hq}/{c.Hkv} {c.Dqk}/{c.Dv} page {c.page} block {c.block} {c.dt}: worst row {worst:.2e}")
    assert worst <= (TOL[c.dt] if tol is None else tol)


SHAPES = [
    # Hq, Hkv, Dqk, Dv, page, block, dt, layout, pad
    (8, 2, 64, 64, 16, 16, torch.float32, "hnd", 0),
    (8, 2, 64, 64, 16, 16, torch.bfloat16, "nhd", 0),
    (16, 2, 128, 128, 64, 64, torch.bfloat16, "hnd", 0),
    (16, 2, 128, 128, 64, 32, torch.float32, "nhd", 0),
    (10, 2, 80, 80, 48, 16, torch.bfloat16, "hnd", 0),
    (6, 2, 96, 96, 32, 32, torch.bfloat16, "nhd", 16),
    (4, 4, 192, 128, 64, 16, torch.bfloat16, "hnd", 0),
    (8, 1, 256, 256, 16, 16, torch.bfloat16, "hnd", 0),
    (8, 2, 256, 192, 32, 16, torch.float32, "nhd", 0),
    (5, 1, 16, 32, 16, 16, torch.float32, "hnd", 0),
    (16, 2, 128, 128, 64, 64, torch.bfloat16, "hnd", 8),   # strides that the matrix-core path does not take
    (4, 2, 72, 40, 32, 16, torch.bfloat16, "nhd", 0),
    (8, 1, 576, 512, 32, 32, torch.bfloat16, "hnd", 0),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x).replace("torch.", "") for x in s))
def test_attention_matches_fp64(shape):
    Hq, Hkv, Dqk, Dv, page, block, dt, layout, pad = shape
    # contexts of one token, of a page less and more one, of a step of 64 keys less and more one; long ones
    kv = [1, 5, page - 1, page, page + 1, 63, 64, 65, 127, 129, 200, 700]
    q_len = [1, 5, 2, 9, 3, 1, 9, 4, 7, 9, 0, 9]
    c = Case(q_len, kv, Hq, Hkv, Dqk, Dv, page, block, dt, layout, pad, seed=1)
    q = queries(c)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("kv,ql", [([17], [17]), ([1] * 70, [1] * 70), ([65] * 3, [65] * 3), ([256, 250, 3], [1, 2, 3]),
                                   ([257, 1], [17, 1]), ([5000], [1]), ([4097, 12000, 64], [17, 4, 17]), ([300] * 130, [1] * 130)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_attention_lengths(kv, ql, dt):
    c = Case(ql, kv, 16, 2, 128, 128, 64, 64, dt, seed=2)
    q = queries(c)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse, requests=range(0, c.R, max(1, c.R // 8)))


@pytest.mark.parametrize("group,ql", [(1, 1), (1, 17), (3, 5), (5, 13), (8, 17), (16, 9)])
def test_attention_groups_and_chunks(group, ql):
    # rows of one chunk less one, exactly, and several chunks
    c = Case([ql, 1, ql], [500, 300, 1100], 2 * group, 2, 64, 64, 16, 16, torch.bfloat16, seed=3)
    q = queries(c)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)


def test_rows_past_the_batch_and_skipped_requests_stay():
    c = Case([3, 2, 4, 1], [100, 40, 90, 30], 4, 2, 64, 64, 16, 16, torch.bfloat16, seed=4)
    d, q = c.on_device(), queries(c)
    q = torch.cat([q, q[:5]])  # rows behind the last sequence
    d["kv"][1] = 1           # fewer keys than queries: skipped
    d["kv"][2] = 10 ** 6     # past the table: skipped
    out = torch.full((q.shape[0], c.Hq, c.Dv), 7.0, dtype=c.dt, device=dev())
    lse = torch.full((q.shape[0], c.Hq), 7.0, device=dev())
    attend(c, d, q, out=out, lse=lse)
    check_attention(c, q, out, lse, requests=[0, 3])
    left = torch.ones(q.shape[0], dtype=torch.bool)
    for r in (0, 3):
        left[int(c.cu[r]):int(c.cu[r + 1])] = False
    assert bool((out.cpu()[left] == 7.0).all()) and bool((lse.cpu()[left] == 7.0).all())


@pytest.mark.parametrize("kv", [40, 48])  # 40: the pages read instead are in part empty, NaN
@pytest.mark.parametrize("D", [64, 128])
def test_table_entries_outside_the_cache_read_a_page_inside(D, kv):
    c = Case([1, 1], [kv, kv], 4, 2, D, D, 16, 16, torch.bfloat16, seed=5, extra=0)
    d, q = c.on_device(), queries(c)
    d["table"][1, 0], d["table"][1, 1] = -3, 10 ** 9
    out, lse = attend(c, d, q)
    c.table[1, 0], c.table[1, 1] = 0, c.num_pages - 1
    nan = bool(np.isnan(c.values("k", 1)).any())
    assert nan == (kv == 40)
    check_attention(c, q, out, lse, requests=[0] if nan else None)
    if nan:
        assert bool(torch.isnan(out[1].float()).all())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("what", ["k", "v", "k_scale", "v_scale", "v_inf"])
@pytest.mark.parametrize("group,D", [(2, 64), (9, 64), (8, 128), (20, 128), (12, 256), (2, 72)])  # 10 rows; 40 to 100; on the vector ALUs
def test_what_is_not_finite_reaches_only_the_rows_that_see_it(dt, what, group, D):
    # the last verify token's key, value or scales: earlier rows do not see it
    page = 16
    c = Case([5, 5], [320 + 5, 33], 2 * group, 2, D, D, page, 16, dt, seed=6)
    c.kv[1] = 33
    j = int(c.kv[0]) - 1
    pg, sl = c.table[0, j // page], j % page
    q = queries(c)
    good, _ = attend(c, c.on_device(), q)
    if what in ("k", "v"):
        c.code[what][pg, 0, sl, 3] = 0x7f
        sees = [4]
    else:
        # a whole block's scale: rows from its first token on see it
        c.scale[what[0]][pg, 0, sl // 16] = np.inf if what == "v_inf" else np.nan
        first = j // 16 * 16
        sees = [t for t in range(5) if 320 + t >= first]
    out, _ = attend(c, c.on_device(), q)
    bad = ~torch.isfinite(out.float()).all(2).cpu().numpy()  # [rows, heads]
    rows = [int(c.cu[0]) + t for t in sees]
    assert bad[rows][:, :group].all()
    rest = np.ones_like(bad)
    rest[np.ix_(rows, range(group))] = False
    assert not bad[rest].any()
    same = out.float().cpu().numpy()[rest] - good.float().cpu().numpy()[rest]
    assert np.abs(same).max() <= 2e-2 * np.abs(good.float().cpu().numpy()).max()


def test_every_code_widens_exactly():
    # one key, so the output is its value: 254 finite codes, both as fp32 and bf16
    for dt in (torch.float32, torch.bfloat16):
        c = Case([1] * 4, [1] * 4, 1, 1, 64, 64, 16, 16, dt, seed=7)
        codes = np.array([x for x in range(256) if x & 127 != 127] + [0, 0], np.uint8).reshape(4, 64)
        for r in range(4):
            c.code["v"][c.table[r, 0], 0, 0] = codes[r]
            c.scale["v"][c.table[r, 0], 0, 0] = 2.0 ** -3
        out, _ = attend(c, c.on_device(), queries(c))
        assert np.array_equal(to_f64(out)[:, 0], ref.VALUES[codes] * 2.0 ** -3)


def test_scales_that_are_no_powers_of_two():
    c = Case([2, 3], [150, 77], 4, 2, 64, 64, 32, 16, torch.float32, seed=8)
    for n in ("k", "v"):
        c.scale[n] *= c.rng.uniform(0.5, 2.0, c.scale[n].shape).astype(np.float32)
    q = queries(c)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("group", [1, 5])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_references_that_keep_moving(D, group, dt):
    # scores and values that grow from block to block, by up to 2^30 each: the running
    # maximum and the values' reference move at every block, inside a step too
    c = Case([9, 1], [600, 250], 2 * group, 2, D, D, 16, 16, dt, seed=22)
    for r in range(c.R):
        n = -(-int(c.kv[r]) // 16)
        for i in range(n):
            c.scale["k"][c.table[r, i], :, 0] = 2.0 ** (-14 + 12 * i / n)
            c.scale["v"][c.table[r, i], :, 0] = 2.0 ** (-20 + 30 * i / n)
    q = queries(c)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse, tol=8e-3 if dt == torch.bfloat16 else 1e-4)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [1, 4, 24])
@pytest.mark.parametrize("what", [float("inf"), 2.0 ** 100, float("nan")])
def test_scales_of_blocks_without_tokens_may_be_anything(what, group, dt):
    # page 0 too, which stands in for table entries past a context
    c = Case([1, 2], [33, 70], 8 * group, 8, 64, 64, 64, 16, dt, seed=23)
    used = {(int(c.table[r, j // 64]), j % 64 // 16) for r in range(c.R) for j in range(int(c.kv[r]))}
    q = queries(c)
    for n in ("k", "v"):
        for pg in range(c.num_pages):
            for b in range(4):
                if (pg, b) not in used:
                    c.scale[n][pg, :, b] = what
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group,D", [(2, 64), (9, 64), (4, 128), (8, 128), (12, 256)])
@pytest.mark.parametrize("ratio", [20, 40])
def test_large_values_that_the_scores_leave_out(ratio, group, D, dt):
    # the first 64 keys score far below the rest and their values' scales are 2^ratio larger:
    # what counts is the product of both (2^-18 and less of the others' here)
    c = Case([5, 1], [400, 90], 2 * group, 2, D, D, 16, 16, dt, seed=24)
    low = (ratio + 18) * np.log(2.0)
    q = (0.5 + torch.from_numpy(c.rng.random((c.rows, c.Hq, D), dtype=np.float32))).to(dt).to(dev())
    for r in range(c.R):
        for i in range(-(-int(c.kv[r]) // 16)):
            at = c.table[r, i]
            # (the others' scores lie around 2, those of the first near -low)
            mean = 4.0 if i >= 4 else -2.0 * low
            x = np.clip(c.rng.normal(64, 8, (2, 16, D)), 0, 128) * np.sign(mean)
            c.code["k"][at] = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
            c.scale["k"][at] = np.float32(abs(mean) / (64 * D * D ** -0.5))
            if i < 4:
                c.scale["v"][at] = 2.0 ** (ratio - 6)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [2, 8])
@pytest.mark.parametrize("exps", [(-100,), (-60,), (60,), (110,), (-100, 60), (-3, 90)])
def test_values_scales_of_any_size(exps, group, dt):
    # block by block in turn; the second request's keys and scales are small enough for one range
    c = Case([5, 2], [3000, 130], 2 * group, 2, 128, 128, 64, 16, dt, seed=25)
    for r in range(c.R):
        for b in range(-(-int(c.kv[r]) // 16)):
            c.scale["v"][c.table[r, b // 4], :, b % 4] = 2.0 ** exps[b % len(exps)]
    q = queries(c)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("group", [2, 8])
def test_negative_scales_and_scales_of_zero(group, dt):
    c = Case([5, 2], [700, 130], 2 * group, 2, 128, 128, 64, 16, dt, seed=26)
    for n in ("k", "v"):
        c.scale[n] *= c.rng.choice(np.array([-1.0, 1.0, 1.0, 0.0], np.float32), c.scale[n].shape)
    q = queries(c)
    out, lse = attend(c, c.on_device(), q)
    check_attention(c, q, out, lse)


def test_values_that_are_all_zero():
    for group in (2, 8):
        c = Case([5, 2], [700, 130], 2 * group, 2, 128, 128, 64, 16, torch.bfloat16, seed=27)
        c.scale["v"][:] = 0.0
        out, lse = attend(c, c.on_device(), queries(c))
        assert bool((out == 0).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("page,tail", [(16, 1), (64, 700)])  # contexts of a few steps; cut into ranges
def test_as_many_requests_as_there_may_be(page, tail):
    rng = np.random.default_rng(29)
    kv = rng.integers(1, 30, 8192)
    kv[-1] = tail
    c = Case([1] * 8192, kv, 4, 2, 64, 64, page, 16, torch.bfloat16, seed=29)
    x, q, d = fill(c, torch.bfloat16), queries(c), c.on_device()
    out, lse = attend(c, d, q)
    check_attention(c, q, out, lse, requests=[0, 1, 63, 64, 4095, 8190, 8191])
    want = expected(c, x)
    append(c, d, x)
    check_append(c, d, want)


def test_values_that_alias_the_keys():
    c = Case([3, 2], [130, 50], 8, 1, 128, 96, 32, 32, torch.bfloat16, seed=9)
    c.code["v"], c.scale["v"] = c.code["k"][..., :96], c.scale["k"]
    d, q = c.on_device(), queries(c)
    out, lse = dspark.dspark_verify_attn_scaled(q, d["kc"], d["kc"], c.strides["k"], c.strides["k"], d["ks"], d["ks"], c.block, d["table"],
                                                d["kv"], d["cu"], c.max_q, 96, c.page, c.Dqk ** -0.5, want_lse=True)
    check_attention(c, q, out, lse)


# ------------------------------------------------------------------ append

def fill(c, dt, wide=0, magnitude=1.0):
    """New rows [rows, Hkv, D] for c's verify tokens, part of rows `wide` values wider."""
    out = {}
    for name, D in (("k", c.Dqk), ("v", c.Dv)):
        x = torch.from_numpy(c.rng.normal(0, magnitude, (c.rows, c.Hkv * D + wide)).astype(np.float32)).to(dt).to(dev())
        out[name] = x[:, wide // 2: wide // 2 + c.Hkv * D].unflatten(1, (c.Hkv, D))
    return out


def append(c, d, x, **kw):
    dspark.dspark_cache_append(x["k"], x["v"], d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], c.block, d["table"], d["kv"],
                               d["cu"], c.max_q, c.page, **kw)
    torch.cuda.synchronize()


def expected(c, x, skip=()):
    """Codes (as values) and scales after the append."""
    got = {}
    for name in ("k", "v"):
        v, s, new = ref.VALUES[c.code[name]], c.scale[name].copy(), to_f64(x[name])
        for r in range(c.R):
            kv, ql = int(c.kv[r]), int(c.q_len[r])
            if r in skip or ql == 0:
                continue
            kv0 = kv - ql
            for lo in range(kv0 // c.block * c.block, kv, c.block):
                pg, sl = c.table[r, lo // c.page], lo % c.page
                first, end = max(lo, kv0), min(kv, lo + c.block)
                rows = slice(int(c.cu[r]) + first - kv0, int(c.cu[r]) + end - kv0)
                for h in range(c.Hkv):
                    vals, sc = ref.append_block(v[pg, h, sl:sl + first - lo], s[pg, h, sl // c.block], new[rows, h])
                    v[pg, h, sl:sl + end - lo] = vals
                    s[pg, h, sl // c.block] = sc
        got[name], got[name + "s"] = v, s
    return got


def check_append(c, d, want):
    for name in ("k", "v"):
        codes = c.unflat(name, d[name + "c"].cpu().numpy())
        np.testing.assert_array_equal(ref.VALUES[codes], want[name])
        np.testing.assert_array_equal(d[name + "s"].cpu().numpy(), want[name + "s"])


APPENDS = [
    # q_len, kv, Hkv, Dqk, Dv, page, block, layout, pad, wide
    ([1, 5, 17, 16, 3, 0, 2], [1, 5, 17, 48, 66, 30, 200], 2, 64, 64, 16, 16, "hnd", 0, 0),
    ([4, 9, 1], [70, 64, 129], 4, 128, 128, 64, 64, "hnd", 0, 64),
    ([4, 9, 17], [70, 100, 129], 2, 128, 128, 64, 32, "nhd", 0, 64),
    ([300, 1, 1000], [300, 90, 1100], 2, 128, 64, 64, 16, "nhd", 0, 0),   # prompts
    ([600], [1000], 1, 256, 256, 256, 256, "hnd", 0, 0),                  # a block too large for the registers
    ([5, 3], [37, 18], 3, 40, 24, 16, 16, "hnd", 3, 1),                   # no alignment
    ([5, 3], [37, 18], 1, 576, 512, 32, 32, "hnd", 0, 8),
]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("spec", APPENDS, ids=range(len(APPENDS)))
def test_append_matches_the_definition(spec, dt):
    q_len, kv, Hkv, Dqk, Dv, page, block, layout, pad, wide = spec
    c = Case(q_len, kv, Hkv, Hkv, Dqk, Dv, page, block, dt, layout, pad, seed=11, scale_exp=(-8, -5))
    x = fill(c, dt, wide)
    want = expected(c, x)
    d = c.on_device()
    append(c, d, x)
    check_append(c, d, want)
    append(c, d, x)  # the same rows again: the same cache
    check_append(c, d, want)


def test_append_roundings_at_the_borders():
    # maxima on both sides of 448 * 2^k, values on the midpoints between codes
    c = Case([4] * 6, [4, 4, 20, 20, 4, 4], 1, 1, 16, 16, 16, 16, torch.float32, seed=12)
    x = fill(c, torch.float32)
    up, down = np.nextafter(np.float32(448), np.float32(1e9)), np.nextafter(np.float32(448), np.float32(0))
    for r, m in enumerate((448.0, up, down, 448 * 2.0 ** -9, 3.4e38, 1e-38)):
        v = np.asarray(ref.VALUES[:120:4][:16], np.float32) * np.float32(m / 448)
        mid = ((ref.VALUES[1:17] + ref.VALUES[2:18]) / 2).astype(np.float32) * np.float32(m / 448)
        rows = torch.from_numpy(np.stack([v, mid, -mid, np.full(16, m, np.float32)]).astype(np.float32)).to(dev())
        for n in ("k", "v"):
            x[n][4 * r:4 * r + 4, 0] = rows
    want = expected(c, x)
    d = c.on_device()
    append(c, d, x)
    check_append(c, d, want)


def test_append_of_zeros_infinities_and_nan():
    c = Case([3, 3, 3, 2], [3, 3, 19, 2], 2, 2, 32, 32, 16, 16, torch.float32, seed=13)
    x = fill(c, torch.float32)
    for n in ("k", "v"):
        x[n][0:3] = 0.0
        x[n][3, 0, 5], x[n][4, 1, 7] = float("inf"), float("nan")
        x[n][6, 0, 0] = float("-inf")
        x[n][9:11] = float("nan")
    want = expected(c, x)
    d = c.on_device()
    append(c, d, x)
    check_append(c, d, want)
    assert float(d["ks"][int(c.table[0, 0]), 0, 0]) == 1.0


@pytest.mark.parametrize("old", [2.0 ** -12, 2.0 ** 3, 0.3, -0.01, 0.0, float("nan"), float("inf"), 2.0 ** 126, 1e-38])
def test_append_behind_tokens_of_any_scale(old):
    c = Case([3], [20 + 3], 2, 2, 32, 32, 32, 32, torch.float32, seed=14)
    for n in ("k", "v"):
        c.scale[n][:] = np.float32(old)
    x = fill(c, torch.float32)
    want = expected(c, x)
    d = c.on_device()
    append(c, d, x)
    check_append(c, d, want)


def test_append_block_by_block_equals_append_at_once():
    # a prompt token by token and whole: the same codes wherever the scale did not end lower than
    # a token's smallest values need
    c = Case([40], [40], 2, 2, 64, 64, 16, 16, torch.float32, seed=15)
    x = fill(c, torch.float32)
    d = c.on_device()
    append(c, d, x)
    e = c.on_device()
    for t in range(40):
        one = {n: x[n][t:t + 1] for n in ("k", "v")}
        dspark.dspark_cache_append(one["k"], one["v"], e["kc"], e["vc"], c.strides["k"], c.strides["v"], e["ks"], e["vs"], c.block, e["table"],
                                   torch.tensor([t + 1], dtype=torch.int32, device=dev()), torch.tensor([0, 1], dtype=torch.int32, device=dev()), 1, c.page)
    torch.cuda.synchronize()
    assert torch.equal(d["ks"].nan_to_num(), e["ks"].nan_to_num())
    for n in ("k", "v"):
        a, b = (ref.VALUES[c.unflat(n, t[n + "c"].cpu().numpy())] for t in (d, e))
        # twice rounded below 2^-6: at most a step of 2^-9 apart
        np.testing.assert_allclose(a, b, rtol=0, atol=2.0 ** -9)


def test_append_skips_what_it_must_not_write():
    c = Case([3, 2, 4, 1], [40, 20, 50, 30], 2, 2, 64, 64, 16, 16, torch.bfloat16, seed=16)
    x = fill(c, torch.bfloat16)
    kv, table = c.kv.copy(), c.table.copy()
    want = expected(c, x, skip=(0, 1, 3))
    d = c.on_device()
    d["kv"][0] = 2                                # fewer tokens than rows
    d["kv"][1] = 10 ** 6
    d["table"][3, (30 - 1) // 16] = c.num_pages   # outside the cache
    append(c, d, x)
    check_append(c, d, want)


def test_keys_alone():
    c = Case([3, 5], [40, 7], 1, 1, 576, 576, 16, 16, torch.bfloat16, seed=17)
    x = fill(c, torch.bfloat16)
    want = expected(c, x)
    d = c.on_device()
    dspark.dspark_cache_append(x["k"], None, d["kc"], None, c.strides["k"], None, d["ks"], None, c.block, d["table"], d["kv"], d["cu"], c.max_q,
                               c.page)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(ref.VALUES[c.unflat("k", d["kc"].cpu().numpy())], want["k"])


def test_offsets_past_32_bits():
    # a pool of more than 4 GB: pages on both sides of 2^32 bytes
    page, Hkv, D = 64, 8, 128
    per = Hkv * page * D
    n = (1 << 32) // per + 40
    ids = [0, n - 1, (1 << 32) // per - 1, (1 << 32) // per, (1 << 31) // per, n - 2]
    kc = torch.zeros(n * per, dtype=torch.uint8, device=dev())
    vc = torch.zeros(n * per, dtype=torch.uint8, device=dev())
    ks, vs = torch.ones(n, Hkv, 1, device=dev()), torch.ones(n, Hkv, 1, device=dev())
    table = torch.tensor([ids[:3], ids[3:]], dtype=torch.int32, device=dev())
    kv = torch.tensor([150, 192], dtype=torch.int32, device=dev())
    cu = torch.tensor([0, 150, 342], dtype=torch.int32, device=dev())
    g = torch.Generator(device=dev())
    g.manual_seed(3)
    x = [torch.randn(342, Hkv, D, generator=g, device=dev()).bfloat16() for _ in range(2)]
    st = (per, page * D, D)
    dspark.dspark_cache_append(x[0], x[1], kc, vc, st, st, ks, vs, 64, table, kv, cu, 192, page)
    got = kc.view(torch.float8_e4m3fn).view(n, Hkv, page, D)[table.long()].float() * ks[table.long()][..., None]
    got = got.transpose(2, 3).reshape(2, 192, Hkv, D)
    for r, (a, b) in enumerate(((0, 150), (150, 342))):
        want = x[0][a:b].float()
        assert bool(((got[r, :b - a] - want).abs() <= want.abs() * 2.0 ** -4 + 2.0 ** -9 * 2.0 ** -6).all())
    # attention over those pages against the same contexts in a small pool
    small = torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32, device=dev())
    pick = lambda t: t.view(n, -1)[table.long().view(-1)].contiguous()  # noqa: E731
    q = torch.randn(4, 32, D, generator=g, device=dev()).bfloat16()
    cu2 = torch.tensor([0, 1, 4], dtype=torch.int32, device=dev())
    far, _ = dspark.dspark_verify_attn_scaled(q, kc, vc, st, st, ks, vs, 64, table, kv, cu2, 3, D, page, D ** -0.5)
    near, _ = dspark.dspark_verify_attn_scaled(q, pick(kc).view(-1), pick(vc).view(-1), st, st, pick(ks).view(6, Hkv, 1), pick(vs).view(6, Hkv, 1),
                                               64, small, kv, cu2, 3, D, page, D ** -0.5)
    torch.cuda.synchronize()
    assert torch.equal(far, near)


# ------------------------------------------------------------------ graphs, streams, refusals

@pytest.mark.parametrize("group", [8, 16])  # one wave a range; four
def test_append_and_attention_in_a_graph(group):
    c = Case([3, 1, 4], [300, 1000, 64], 2 * group, 2, 128, 128, 64, 64, torch.bfloat16, seed=18)
    x, q, d = fill(c, torch.bfloat16), queries(c), c.on_device()
    need = dspark.dspark_verify_attn_scaled_workspace_size(c.R, c.max_q, c.Hq, c.Hkv, 128, 128, d["table"].shape[1], c.page, c.block, c.dt)
    ws = torch.empty(need, dtype=torch.uint8, device=dev())
    out, lse = torch.empty(c.rows, c.Hq, 128, dtype=c.dt, device=dev()), torch.empty(c.rows, c.Hq, device=dev())
    start = {n: d[n].clone() for n in ("kc", "vc", "ks", "vs")}

    def step():
        append(c, d, x) if not torch.cuda.is_current_stream_capturing() else dspark.dspark_cache_append(
            x["k"], x["v"], d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], c.block, d["table"], d["kv"], d["cu"], c.max_q, c.page)
        dspark.dspark_verify_attn_scaled(q, d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], c.block, d["table"], d["kv"], d["cu"],
                                         c.max_q, c.Dv, c.page, c.Dqk ** -0.5, out=out, lse=lse, ws=ws)

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (out, lse, d["kc"], d["ks"])]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(3):
        for n, t in start.items():
            d[n].copy_(t)
        out.zero_()
        float((q.float() * q.float()).sum())
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(d["kc"], want[2])
        assert torch.equal(d["ks"].nan_to_num(), want[3].nan_to_num())


def test_another_stream():
    c = Case([3, 1], [300, 90], 16, 2, 128, 128, 64, 64, torch.bfloat16, seed=19)
    d, q = c.on_device(), queries(c)
    want, _ = attend(c, d, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse = attend(c, d, q, stream=s)
    assert torch.equal(out, want)


def test_two_calls_at_once():
    # each with its own workspace and outputs, over one cache
    c = Case([3, 1, 9], [3000, 90, 5000], 32, 2, 128, 128, 64, 64, torch.bfloat16, seed=28)
    d, q = c.on_device(), queries(c)
    want, lse = attend(c, d, q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(dspark.dspark_verify_attn_scaled(q, d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], c.block, d["table"],
                                                            d["kv"], d["cu"], c.max_q, c.Dv, c.page, c.Dqk ** -0.5, want_lse=True))
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) and torch.equal(x, lse) for o, x in got)


def test_refusals():
    c = Case([2, 1], [40, 20], 4, 2, 64, 64, 32, 16, torch.bfloat16, seed=20)
    d, q, x = c.on_device(), queries(c), fill(c, torch.bfloat16)

    def bad(**kw):
        e = dict(d, **{k: v for k, v in kw.items() if k in d})
        with pytest.raises(dspark.DSparkError):
            dspark.dspark_verify_attn_scaled(kw.get("q", q), e["kc"], e["vc"], c.strides["k"], c.strides["v"], e["ks"], e["vs"], kw.get("block", c.block),
                                             e["table"], e["kv"], e["cu"], c.max_q, kw.get("Dv", c.Dv), kw.get("page", c.page), 0.1, ws=kw.get("ws"))
        if "q" not in kw and "Dv" not in kw and "ws" not in kw:
            with pytest.raises(dspark.DSparkError):
                dspark.dspark_cache_append(kw.get("k", x["k"]), x["v"], e["kc"], e["vc"], c.strides["k"], c.strides["v"], e["ks"], e["vs"],
                                           kw.get("block", c.block), e["table"], e["kv"], e["cu"], c.max_q, kw.get("page", c.page))

    bad(q=q.half())
    bad(q=q.cpu())
    bad(kc=d["kc"][:-1])                                   # fewer pages than scales
    bad(kc=d["kc"].view(torch.int8))
    bad(ks=d["ks"].double())
    bad(vs=d["vs"][1:])
    bad(block=24)
    bad(block=8)
    bad(page=16)
    bad(table=d["table"].long())
    bad(kv=d["kv"][:1])
    bad(ws=torch.empty(256, dtype=torch.uint8, device=dev()))
    bad(Dv=60)
    with pytest.raises(dspark.DSparkError):
        dspark.dspark_cache_append(x["k"].transpose(0, 1).contiguous().transpose(0, 1), x["v"], d["kc"], d["vc"], c.strides["k"], c.strides["v"],
                                   d["ks"], d["vs"], c.block, d["table"], d["kv"], d["cu"], c.max_q, c.page)
    with pytest.raises(dspark.DSparkError):
        dspark.dspark_cache_append(x["k"], None, d["kc"], d["vc"], c.strides["k"], c.strides["v"], d["ks"], d["vs"], c.block, d["table"], d["kv"],
                                   d["cu"], c.max_q, c.page)


def test_debug_mode_raises_first(monkeypatch):
    c = Case([2, 1], [40, 20], 4, 2, 64, 64, 32, 16, torch.bfloat16, seed=21)
    d, q, x = c.on_device(), queries(c), fill(c, torch.bfloat16)
    monkeypatch.setenv("DSPARK_DEBUG", "1")
    attend(c, d, q)
    d["table"][1, 0] = c.num_pages
    with pytest.raises(dspark.DSparkError, match="request 1"):
        attend(c, d, q)
    with pytest.raises(dspark.DSparkError, match="request 1"):
        append(c, d, x)
