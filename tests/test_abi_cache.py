"""C ABI checks of the 8-bit cache and its pages that need no GPU: what validation
refuses before anything touches HIP, and workspace sizes."""
import ctypes as C
import os

import numpy as np
import pytest

import cache_reference as ref
from paper_2607_05147_amd import dspark

EINVAL, ESHAPE, EDTYPE, EUNSUPPORTED, EWORKSPACE = 1, 2, 3, 4, 5
FAKE, ODD = C.c_void_p(1 << 20), C.c_void_p((1 << 20) + 2)  # never dereferenced


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(dspark.LIB_PATH):
        from paper_2607_05147_amd import build
        build.build()
    return dspark.lib()


def st(*v):
    return (C.c_int64 * 3)(*v)


def _append(L, **kw):
    a = dict(k=FAKE, v=FAKE, k_ld=1024, v_ld=1024, dt=1, kc=FAKE, vc=FAKE, ks=st(65536, 8192, 128), vs=st(65536, 8192, 128), ksc=FAKE, vsc=FAKE,
             block=64, bt=FAKE, max_pages=4, num_pages=10, kv=FAKE, cu=FAKE, R=4, max_q=9, Hkv=8, Dqk=128, Dv=128, page=64)
    a.update(kw)
    return L.dspark_cache_append(*a.values(), None)


def test_append_validation(L):
    assert _append(L, R=0) == EINVAL
    assert _append(L, max_q=0) == EINVAL
    assert _append(L, max_q=(1 << 20) + 1) == EINVAL
    assert _append(L, num_pages=0) == EINVAL
    assert _append(L, dt=5) == EDTYPE
    assert _append(L, Dqk=100) == EUNSUPPORTED
    assert _append(L, page=24, block=24) == EUNSUPPORTED
    assert _append(L, block=48) == EUNSUPPORTED
    assert _append(L, block=8) == EUNSUPPORTED
    assert _append(L, block=0) == EUNSUPPORTED
    assert _append(L, k_ld=1023) == ESHAPE
    assert _append(L, v_ld=1000) == ESHAPE
    assert _append(L, ks=st(65536, 8192, 120)) == ESHAPE
    assert _append(L, vs=st(65536, -1, 128)) == EINVAL
    assert _append(L, max_pages=1 << 25) == EUNSUPPORTED
    assert _append(L, R=8192, max_q=1 << 20) == EUNSUPPORTED
    for name in ("k", "kc", "ks", "ksc", "bt", "kv", "cu", "v", "vc", "vs", "vsc"):
        assert _append(L, **{name: None}) == EINVAL, name
    for name in ("ksc", "vsc", "bt", "kv", "cu"):
        assert _append(L, **{name: ODD}) == EINVAL, name
    assert _append(L, k=C.c_void_p((1 << 20) + 1)) == EINVAL


def _attn(L, **kw):
    a = dict(q=FAKE, kc=FAKE, vc=FAKE, ks=st(65536, 8192, 128), vs=st(65536, 8192, 128), ksc=FAKE, vsc=FAKE, block=64, bt=FAKE, max_pages=4,
             num_pages=10, kv=FAKE, cu=FAKE, R=4, max_q=9, Hq=32, Hkv=8, Dqk=128, Dv=128, page=64, scale=0.1, dt=1, out=FAKE, lse=None, ws=FAKE,
             ws_bytes=0)
    a.update(kw)
    return L.dspark_verify_attn_scaled(*a.values(), None)


def test_attention_validation(L):
    assert _attn(L, R=0) == EINVAL
    assert _attn(L, max_q=66) == EINVAL
    assert _attn(L, num_pages=0) == EINVAL
    assert _attn(L, Hq=30) == ESHAPE
    assert _attn(L, dt=2) == EDTYPE
    assert _attn(L, Dv=1024) == EUNSUPPORTED
    assert _attn(L, block=48) == EUNSUPPORTED
    assert _attn(L, scale=0.0) == EINVAL
    assert _attn(L, scale=float("nan")) == EINVAL
    assert _attn(L, ks=st(65536, 8192, 64)) == ESHAPE
    for name in ("q", "kc", "vc", "ks", "vs", "ksc", "vsc", "bt", "kv", "cu", "out"):
        assert _attn(L, **{name: None}) == EINVAL, name
    assert _attn(L, lse=ODD) == EINVAL
    need = L.dspark_verify_attn_scaled_workspace_size(4, 9, 32, 8, 128, 128, 4, 64, 64, 1)
    assert need == 0 or _attn(L, ws_bytes=need - 1) == EWORKSPACE
    need = L.dspark_verify_attn_scaled_workspace_size(4, 9, 32, 8, 128, 128, 64, 64, 64, 1)
    assert need > 0
    assert _attn(L, max_pages=64, ws_bytes=need - 1) == EWORKSPACE
    assert _attn(L, max_pages=64, ws=None, ws_bytes=need) == EWORKSPACE
    assert _attn(L, max_pages=64, ws=C.c_void_p((1 << 20) + 64), ws_bytes=need) == EWORKSPACE


def test_attention_workspace_size(L):
    f = L.dspark_verify_attn_scaled_workspace_size
    assert f(0, 9, 32, 8, 128, 128, 64, 64, 64, 1) == 0
    assert f(4, 9, 32, 8, 128, 128, 64, 64, 24, 1) == 0
    for dt in (0, 1):
        prev = 0
        for R in range(1, 200):  # one sized for the largest batch serves the smaller ones
            n = f(R, 9, 32, 8, 64, 64, 256, 16, 16, dt)
            assert n >= prev > -1
            prev = n


class Buf(C.Structure):
    _fields_ = [("base", C.c_void_p), ("page_stride", C.c_int64), ("page_bytes", C.c_int64)]


def bufs(*v):
    return (Buf * len(v))(*[Buf(*x) for x in v])


def test_pages_validation(L):
    need = L.dspark_pages_workspace_size(4, 100)
    assert need > 0 and need % 256 == 0
    assert L.dspark_pages_workspace_size(0, 100) == 0 and L.dspark_pages_workspace_size(4, (1 << 24) + 1) == 0

    def reserve(bt=FAKE, mp=8, kv=FAKE, cu=FAKE, R=4, page=16, r=FAKE, n=100, b=None, nb=0, step=C.c_void_p(1 << 21), ws=FAKE, wb=need):
        return L.dspark_pages_reserve(bt, mp, kv, cu, R, page, r, n, b, nb, step, ws, wb, None)

    def commit(bt=FAKE, mp=8, kv=FAKE, step=FAKE, cu=FAKE, acc=None, R=4, page=16, r=FAKE, n=100):
        return L.dspark_pages_commit(bt, mp, kv, step, cu, acc, R, page, r, n, None)

    def trim(bt=FAKE, mp=8, kv=FAKE, new=FAKE, R=4, page=16, r=FAKE, n=100):
        return L.dspark_pages_trim(bt, mp, kv, new, R, page, r, n, None)

    def fork(bt=FAKE, mp=8, kv=FAKE, R=4, page=16, r=FAKE, n=100, p=FAKE, c=FAKE, ln=None, k=2, ws=FAKE, wb=need):
        return L.dspark_pages_fork(bt, mp, kv, R, page, r, n, p, c, ln, k, ws, wb, None)

    def compact(bt=FAKE, mp=8, kv=FAKE, R=4, page=16, r=FAKE, n=100, b=None, nb=0, used=FAKE, ws=FAKE, wb=need):
        return L.dspark_pages_compact(bt, mp, kv, R, page, r, n, b, nb, used, ws, wb, None)

    def check(bt=FAKE, mp=8, kv=FAKE, R=4, page=16, r=FAKE, n=100, rep=FAKE):
        return L.dspark_check_page_inputs(bt, mp, kv, R, page, r, n, rep, None)

    for f in (reserve, commit, trim, fork, compact, check):
        assert f(R=0) == EINVAL and f(R=8193) == EINVAL
        assert f(mp=0) == EINVAL
        assert f(n=0) == EINVAL and f(n=(1 << 24) + 1) == EINVAL
        assert f(page=8) == EUNSUPPORTED and f(page=24) == EUNSUPPORTED
        assert f(mp=1 << 27) == EUNSUPPORTED
        for name in ("bt", "kv", "r"):
            assert f(**{name: None}) == EINVAL, (f, name)
            assert f(**{name: ODD}) == EINVAL, (f, name)
    for f in (reserve, fork, compact):
        assert f(ws=None) == EWORKSPACE
        assert f(wb=need - 1) == EWORKSPACE
        assert f(ws=C.c_void_p((1 << 20) + 64)) == EWORKSPACE
    for f in (reserve, compact):
        assert f(nb=-1) == EINVAL and f(nb=1025, b=bufs((1 << 20, 16, 16))) == EINVAL
        assert f(nb=1) == EINVAL
        assert f(nb=1, b=bufs((0, 16, 16))) == EINVAL
        assert f(nb=2, b=bufs((1 << 20, 16, 16), (1 << 20, 16, 0))) == EINVAL
        assert f(nb=1, b=bufs((1 << 20, 15, 16))) == ESHAPE
        assert f(nb=1, b=bufs((1 << 20, (1 << 31) + 1, 16))) == ESHAPE
    assert reserve(cu=None) == EINVAL and reserve(step=None) == EINVAL
    assert reserve(step=FAKE) == EINVAL  # kv_len itself
    assert commit(step=None) == EINVAL and commit(cu=None) == EINVAL and commit(acc=ODD) == EINVAL
    assert trim(new=None) == EINVAL
    assert fork(p=None) == EINVAL and fork(c=None) == EINVAL and fork(k=5) == EINVAL and fork(k=-1) == EINVAL and fork(ln=ODD) == EINVAL
    assert fork(k=0, p=None, c=None) == 0  # nothing to do
    assert compact(used=None) == EINVAL
    assert check(rep=None) == EINVAL


def test_pages_workspace_grows(L):
    for n in (1, 1000, 1025, 70000):
        prev = 0
        for R in (1, 2, 100, 1000, 8192):
            need = L.dspark_pages_workspace_size(R, n)
            assert need >= prev and need >= L.dspark_pages_workspace_size(R, max(1, n // 2))
            prev = need


# ------------------------------------------------------------------ the reference itself

def test_reference_rounding_is_the_types():
    import torch
    x = np.concatenate([np.random.default_rng(0).normal(0, s, 5000) for s in (1e-3, 0.02, 1, 100)] +
                       [(ref.VALUES[:126] + ref.VALUES[1:127]) / 2, -ref.VALUES[:127]]).astype(np.float32)
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(ref.e4m3_round(x), want)
    assert np.array_equal(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(), ref.VALUES, equal_nan=True)


def test_reference_scales():
    for k in range(-99, 120):
        a = 448 * 2.0 ** k
        assert ref.pow2_scale(a) == 2.0 ** k and ref.pow2_scale(np.nextafter(a, 0)) == 2.0 ** k
        assert ref.pow2_scale(np.nextafter(a, np.inf)) == 2.0 ** (k + 1)
    assert ref.pow2_scale(0.0) == 0.0 and ref.pow2_scale(1e-40) == 2.0 ** -100


def test_reference_pages_keep_count():
    # holders' counts are those of the held entries, whatever happened
    rng = np.random.default_rng(1)
    R, n, page = 9, 60, 16
    p = ref.Pages(rng.permutation(n)[:R * 6].reshape(R, 6).astype(np.int32), rng.integers(0, 60, R).astype(np.int32), page, n, [np.arange(n)[:, None]])
    for _ in range(60):
        empty, full = np.flatnonzero(p.kv == 0), np.flatnonzero(p.kv > 0)
        if len(empty) and len(full):
            p.fork(rng.choice(full, len(empty)), empty, rng.integers(0, 96, len(empty)))
        q = np.minimum(rng.integers(0, 20, R), 96 - p.kv)
        st = p.reserve(q)
        p.commit(st, q, rng.integers(-1, 20, R))
        p.trim(rng.integers(0, 200, R) * (rng.random(R) < 0.7))
        used = p.compact()
        count = np.zeros(n, int)
        for r in range(R):
            np.add.at(count, p.table[r, :p.held(r)], 1)
        assert np.array_equal(count, p.ref) and (p.ref[:used] > 0).all() and (p.ref[used:] == 0).all()
