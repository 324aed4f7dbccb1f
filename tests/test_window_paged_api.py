"""The entry points of moa_window.h and moa_paged.h on the CPU: they are exported and bound, and reject
invalid calls before touching the GPU (no compute calls here)."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADERS = {"moa_window.h": ["moa_win_attn_bwd", "moa_win_attn_bwd_workspace_bytes", "moa_win_attn_fwd",
                            "moa_win_attn_num_splits", "moa_win_attn_workspace_bytes"],
           "moa_paged.h": ["moa_paged_append", "moa_paged_attn_fwd", "moa_paged_attn_num_splits",
                           "moa_paged_attn_workspace_bytes"]}

moa = pytest.importorskip("paper_2606_07713_amd", reason="HIP library not built")
from paper_2606_07713_amd import paged, window  # noqa: E402

_SAN = os.environ.get("MOA_TEST_SANITIZED_API_LIB")
if _SAN:   # the same checks against a build under sanitizers
    lib = ctypes.CDLL(_SAN)
    for f in [*(x for m in (window, paged) for x in vars(m).values() if isinstance(x, (window.Function, window.Packed)))]:
        f.f = getattr(lib, f.name)
        f.f.argtypes, f.f.restype = f.argtypes, f.restype

P = 1 << 24          # addresses that nothing is read at: every call here is refused, or has no rows
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("header", HEADERS)
def test_headers_and_exports(header, tmp_path):
    path = os.path.join(ROOT, "include", header)
    text = re.sub(r"/\*.*?\*/", "", open(path).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(moa_\w+)\s*\(", text))) == HEADERS[header]
    lib = ctypes.CDLL(moa.LIB_PATH)
    for name in HEADERS[header]:
        assert hasattr(lib, name) and hasattr(moa, name) and name in moa.__all__
    c = tmp_path / "t.c"
    c.write_text(f'#include "{header}"\nint main(void){{return MOA_OK;}}\n')
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(path), str(c), "-o", str(tmp_path / "t")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    for name in ("win_attn_fwd", "win_attn_bwd", "paged_cache", "paged_append", "paged_attn_fwd"):
        assert hasattr(moa, name) and name in moa.__all__


def _i64(v):
    return None if v is None else (ctypes.c_int64 * len(v))(*v)


def _strided(a, names):
    for k in names:
        a[k] = _i64(a[k])
    return a.values()


def _fwd(**kw):
    a = dict(Q=P, K=2 * P, V=3 * P, O=4 * P, LSE=5 * P, B=2, Hq=4, Hk=2, Nq=8, Nk=8, d=64, qs=None, ks=None, vs=None, os=None,
             left=-1, right=0, sinks=0, scale=1.0, dt=moa.MOA_BF16, ws=None, wsn=0, splits=1)
    a.update(kw)
    return moa.moa_win_attn_fwd(*_strided(a, ("qs", "ks", "vs", "os")), None)


FWD_BAD = [
    (dict(Q=None), 1), (dict(K=None), 1), (dict(V=None), 1), (dict(O=None), 1), (dict(Q=P + 8), 1), (dict(O=4 * P + 2), 1),
    (dict(LSE=5 * P + 2), 1), (dict(ws=6 * P + 8, wsn=1 << 20), 1),
    (dict(B=-1), 1), (dict(Hq=-4), 1), (dict(Hk=0), 1), (dict(Hq=5), 1), (dict(Nq=-1), 1), (dict(Nk=-1), 1), (dict(d=0), 1),
    (dict(d=96), 2), (dict(sinks=-1), 1), (dict(splits=-1), 1), (dict(splits=257), 1), (dict(dt=2), 1),
    (dict(scale=NAN), 1), (dict(scale=INF), 1), (dict(scale=3e38), 2),
    (dict(Nk=(1 << 30) + 1), 2), (dict(Nq=(1 << 30) + 1), 2), (dict(Nq=1 << 23), 2), (dict(B=1 << 25, Nq=1), 2),
    (dict(B=1 << 13, Hk=4, Nq=2000, splits=256), 2),
    (dict(qs=[-512, 64, 64]), 1), (dict(qs=[4096, 512, 63]), 2), (dict(ks=[1 << 41, 512, 64]), 2),
    (dict(ks=[1 << 30, 1 << 29, (1 << 25) + 8]), 2), (dict(os=[512, 64, 0]), 1), (dict(os=[2048, 512, 32]), 1),
    (dict(O=P), 1), (dict(O=2 * P), 1), (dict(O=3 * P + 1024), 1), (dict(LSE=P), 1), (dict(LSE=4 * P + 64), 1),
    (dict(splits=2), 3), (dict(splits=2, ws=6 * P, wsn=64), 3), (dict(splits=2, ws=4 * P, wsn=1 << 20), 1),
    (dict(splits=2, ws=2 * P, wsn=1 << 20), 1),
]


@pytest.mark.parametrize("kw,status", FWD_BAD, ids=str)
def test_win_attn_fwd_refuses(kw, status):
    assert _fwd(**kw) == status


@pytest.mark.parametrize("kw", [dict(B=0), dict(Hq=0), dict(Nq=0), dict(B=0, Q=None, K=None, V=None, O=None),
                                dict(Nq=0, Q=None, O=None)], ids=str)
def test_win_attn_fwd_without_rows(kw):
    assert _fwd(**kw) == 0


def _bwd(**kw):
    a = dict(Q=P, K=2 * P, V=3 * P, O=4 * P, dO=5 * P, LSE=6 * P, dQ=7 * P, dK=8 * P, dV=9 * P, B=2, Hq=4, Hk=2, Nq=8, Nk=8, d=64,
             qs=None, ks=None, vs=None, os=None, gs=None, dqs=None, dks=None, dvs=None, left=-1, right=0, sinks=0, scale=1.0,
             dt=moa.MOA_BF16, ws=10 * P, wsn=1 << 22)
    a.update(kw)
    return moa.moa_win_attn_bwd(*_strided(a, ("qs", "ks", "vs", "os", "gs", "dqs", "dks", "dvs")), None)


BWD_BAD = [
    *[({k: None}, 1) for k in ("Q", "K", "V", "O", "dO", "LSE", "dQ", "dK", "dV")],
    (dict(dO=5 * P + 8), 1), (dict(LSE=6 * P + 1), 1), (dict(ws=10 * P + 4), 1), (dict(Hq=3), 1), (dict(d=32), 2), (dict(dt=5), 1),
    (dict(scale=NAN), 1), (dict(scale=-3e38), 2), (dict(sinks=-4), 1), (dict(Nk=1 << 24), 2),
    (dict(gs=[1 << 28, 1 << 27, (1 << 23) + 8]), 2), (dict(dks=[1024, 64, 64]), 1), (dict(dqs=[2048, 512, -64]), 1),
    (dict(dQ=P), 1), (dict(dQ=5 * P), 1), (dict(dK=8 * P, dV=8 * P), 1), (dict(dV=3 * P), 1), (dict(dK=6 * P), 1),
    (dict(ws=7 * P), 1), (dict(ws=6 * P), 1), (dict(ws=None), 3), (dict(wsn=100), 3),
    # more workgroups of the join than one launch takes
    (dict(B=1 << 20, Hq=1, Hk=1, Nq=40, Nk=40, left=3, sinks=4, **{k: i * P << 16 for i, k in enumerate(("Q", "K", "V", "O", "dO", "LSE", "dQ", "dK", "dV", "ws"), 1)}), 2),
]


@pytest.mark.parametrize("kw,status", BWD_BAD, ids=str)
def test_win_attn_bwd_refuses(kw, status):
    assert _bwd(**kw) == status


def test_win_attn_bwd_without_rows():
    assert _bwd(B=0) == 0
    assert _bwd(Nq=0, Nk=0, Q=None, K=None, V=None, O=None, dO=None, LSE=None, dQ=None, dK=None, dV=None) == 0


def _append(**kw):
    a = dict(Q=P, K=2 * P, V=3 * P, Qo=4 * P, kp=5 * P, vp=6 * P, wq=7 * P, wk=8 * P, pos=9 * P, freq=10 * P, lens=11 * P,
             new=12 * P, table=13 * P, B=2, Hq=4, Hk=2, N=8, d=64, rot=64, page=16, num=20, most=4, qs=None, ks=None, vs=None,
             qos=None, kps=None, vps=None, axes=1, sec=None, il=0, eps=1e-6, dt=moa.MOA_BF16, wdt=moa.MOA_F32)
    a.update(kw)
    return moa.moa_paged_append(*_strided(a, ("qs", "ks", "vs", "qos", "kps", "vps", "sec")), None)


APPEND_BAD = [
    *[({k: None}, 1) for k in ("Q", "K", "V", "Qo", "kp", "vp", "freq", "lens")],
    (dict(kp=5 * P + 8), 1), (dict(lens=11 * P + 2), 1), (dict(table=13 * P + 1), 1), (dict(pos=9 * P + 4), 1),
    (dict(table=None), 1), (dict(table=None, most=1, num=1), 1), (dict(page=0), 1), (dict(page=8), 2), (dict(page=48), 2),
    (dict(page=1 << 21), 2), (dict(num=-1), 1), (dict(most=-1), 1), (dict(most=1 << 27), 2), (dict(num=1 << 30), 2),
    (dict(B=-1), 1), (dict(N=-1), 1), (dict(Hk=-1), 1), (dict(d=80), 2), (dict(rot=24), 2), (dict(rot=80), 1), (dict(axes=5), 1),
    (dict(axes=2, sec=[1, 2]), 1), (dict(il=2), 1), (dict(eps=-1.0), 1), (dict(dt=3), 1), (dict(wdt=3), 1),
    (dict(B=1 << 20, N=1 << 7), 2), (dict(B=1 << 14, N=1 << 12, Hq=8, Hk=13), 2),
    (dict(kps=[2048, 1024, 0]), 1), (dict(kps=[1024, 1024, 64]), 1), (dict(vps=[1 << 30, 1 << 29, (1 << 25) + 8]), 2),
    (dict(kps=[2048, 1024, 60]), 2), (dict(qos=[2048, 512, 32]), 1),
    (dict(kp=6 * P + 128), 1), (dict(kp=2 * P), 1), (dict(vp=P), 1), (dict(Qo=5 * P), 1), (dict(Qo=2 * P), 1), (dict(Qo=P + 16), 1),
    (dict(Qo=P, dt=moa.MOA_F32), 1), (dict(kp=11 * P - 64), 1), (dict(vp=7 * P), 1), (dict(Qo=9 * P), 1), (dict(kp=10 * P), 1),
]


@pytest.mark.parametrize("kw,status", APPEND_BAD, ids=str)
def test_paged_append_refuses(kw, status):
    assert _append(**kw) == status


def test_paged_append_without_rows():
    for kw in (dict(B=0), dict(N=0), dict(Hq=0, Hk=0, Q=None, K=None, V=None, Qo=None, kp=None, vp=None)):
        assert _append(**kw) == 0


def _attn(**kw):
    a = dict(Q=P, kp=2 * P, vp=3 * P, O=4 * P, LSE=5 * P, lens=6 * P, new=7 * P, table=8 * P, B=2, Hq=4, Hk=2, N=8, d=64, page=16,
             num=20, most=4, max_len=0, qs=None, kps=None, vps=None, os=None, left=-1, right=0, sinks=0, scale=1.0,
             dt=moa.MOA_BF16, ws=None, wsn=0, splits=1)
    a.update(kw)
    return moa.moa_paged_attn_fwd(*_strided(a, ("qs", "kps", "vps", "os")), None)


ATTN_BAD = [
    *[({k: None}, 1) for k in ("Q", "kp", "vp", "O", "lens", "table")],
    (dict(kp=2 * P + 4), 1), (dict(lens=6 * P + 1), 1), (dict(Hk=0), 1), (dict(Hq=3), 1), (dict(page=24), 2), (dict(page=-16), 1),
    (dict(max_len=-1), 1), (dict(sinks=-1), 1), (dict(scale=INF), 1), (dict(dt=9), 1), (dict(d=256), 2), (dict(N=-2), 1),
    (dict(num=-1), 1), (dict(most=1 << 28), 2), (dict(N=1 << 24), 2), (dict(os=[2048, 512, 60]), 2), (dict(kps=[2048, -1024, 64]), 1),
    (dict(O=2 * P), 1), (dict(O=6 * P - 64), 1), (dict(LSE=8 * P), 1), (dict(O=P), 1), (dict(splits=3), 3),
    (dict(splits=3, ws=3 * P, wsn=1 << 20), 1), (dict(splits=3, ws=7 * P, wsn=1 << 20), 1), (dict(splits=300), 1),
]


@pytest.mark.parametrize("kw,status", ATTN_BAD, ids=str)
def test_paged_attn_fwd_refuses(kw, status):
    assert _attn(**kw) == status


def test_paged_attn_fwd_without_rows():
    for kw in (dict(B=0), dict(N=0), dict(Hq=0)):
        assert _attn(**kw) == 0


def test_splits_and_workspaces():
    n, w = moa.moa_win_attn_num_splits, moa.moa_win_attn_workspace_bytes
    assert n(1, 32, 8, 200, 20000, 128, -1, 0, 0, 0) > 1 and n(8, 32, 8, 4096, 4096, 128, -1, 0, 0, 0) == 1
    assert n(1, 32, 8, 200, 20000, 128, -1, 0, 0, 7) == 7 and n(1, 32, 8, 0, 20000, 128, -1, 0, 0, 7) == 1
    assert w(1, 32, 8, 200, 20000, 128, -1, 0, 0, 7) >= 32 * 200 * 7 * 130 * 4 and w(1, 32, 8, 200, 20000, 128, -1, 0, 0, 1) == 0
    assert w(1, 32, 7, 200, 20000, 128, -1, 0, 0, 7) == 0 and n(1, 32, 7, 200, 20000, 128, -1, 0, 0, 7) == 1
    # a window leaves nothing to split where all keys would
    assert n(4, 32, 8, 1, 100000, 128, 127, 0, 0, 0) == 1 < n(4, 32, 8, 1, 100000, 128, -1, 0, 0, 0)
    m, x = moa.moa_paged_attn_num_splits, moa.moa_paged_attn_workspace_bytes
    assert m(1, 32, 8, 1, 128, 16, 1000, 0, -1, 0, 0, 0) > m(1, 32, 8, 1, 128, 16, 1000, 100, -1, 0, 0, 0)
    assert x(1, 32, 8, 1, 128, 16, 1000, 0, -1, 0, 0, 5) >= 32 * 5 * 130 * 4 and x(1, 32, 8, 1, 128, 24, 1000, 0, -1, 0, 0, 5) == 0
    b = moa.moa_win_attn_bwd_workspace_bytes
    assert b(2, 8, 2, 100, 100, 64, -1, 0, 0) >= 2 * 8 * 100 * 4 and b(2, 8, 3, 100, 100, 64, -1, 0, 0) == 0
    assert b(1, 32, 8, 8192, 8192, 128, 1023, 0, 4) > b(1, 32, 8, 8192, 8192, 128, 1023, 0, 0)
    # many first keys, few of them, one more query than a window: sizes stay in bounds
    for sinks in (1, 127, 128, 129, 5000, 1 << 40):
        for left in (0, 1, 1000, 1 << 40):
            for N in (1, 64, 65, 5000):
                assert b(1, 4, 2, N, 5000, 64, left, 0, sinks) < 1 << 30


@pytest.mark.parametrize("far", [1 << 30, 1 << 62, (1 << 63) - 1])
def test_windows_longer_than_any_sequence(far):
    """They are no limit, however long: the same choices as without one, and no sum of them overflows."""
    for N, Nk, sinks in ((1, 5000, 0), (300, 9000, 4), (4096, 4096, 200)):
        for left, right in ((far, 0), (far, far), (-1, far), (100, far)):
            plain = [-1 if x == far else x for x in (left, right)]
            for f, more in ((moa.moa_win_attn_num_splits, [0]), (moa.moa_win_attn_workspace_bytes, [0]),
                            (moa.moa_win_attn_bwd_workspace_bytes, [])):
                assert f(1, 8, 2, N, Nk, 64, left, right, sinks, *more) == f(1, 8, 2, N, Nk, 64, *plain, sinks, *more)
                assert f(1, 8, 2, N, Nk, 64, left, right, far, *more) == f(1, 8, 2, N, Nk, 64, *plain, 1 << 30, *more)
            a = [moa.moa_paged_attn_num_splits(1, 8, 2, N, 64, 16, 1000, 0, *w, s, 0) for w, s in (((left, right), sinks), (plain, sinks))]
            assert a[0] == a[1]


def test_wrappers_refuse():
    torch = pytest.importorskip("torch")
    q = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    with pytest.raises((ValueError, TypeError)):
        moa.win_attn_fwd(q, q, q)                      # not on a device
    with pytest.raises((ValueError, TypeError)):
        moa.paged_attn_fwd(q, q, q, torch.zeros(1, dtype=torch.int32))
    with pytest.raises((ValueError, TypeError)):
        moa.paged_append(q, q, q, q, q, torch.zeros(1, dtype=torch.int32))
    with pytest.raises((ValueError, TypeError)):
        moa.win_attn_bwd(q, q, q, q, q, torch.zeros(1, 2, 3))
    for bad in (dict(page=8), dict(page=48), dict(d=96)):
        with pytest.raises(ValueError):
            moa.paged_cache(**{**dict(num_pages=2, heads=1, page=16, d=64, device="cpu"), **bad})
    k, v = moa.paged_cache(2, 3, 32, 64, device="cpu")
    assert k.shape == v.shape == (2, 3, 32, 64) and k.dtype is torch.bfloat16
