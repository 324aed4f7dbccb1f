"""The entry points of moa_rope.h and moa_kv4.h on the CPU: they are exported and bound, and reject
invalid calls before touching the GPU (no compute calls here)."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADERS = {"moa_rope.h": ["moa_qk_norm_rope", "moa_qk_norm_rope_bwd", "moa_qk_norm_rope_bwd_workspace_bytes"],
           "moa_kv4.h": ["moa_kv4_attn_fwd", "moa_kv4_attn_num_splits", "moa_kv4_attn_workspace_bytes",
                         "moa_kv4_page_bytes", "moa_kv4_read", "moa_kv4_write"]}

moa = pytest.importorskip("paper_2606_07713_amd", reason="HIP library not built")
from paper_2606_07713_amd import kv4, rope  # noqa: E402

P = 1 << 20          # addresses that nothing is read at: every call here is refused, or has no rows


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


def _i64(v):
    return None if v is None else (ctypes.c_int64 * len(v))(*v)


def _rope(**kw):
    a = dict(Q=P, K=2 * P, Qo=3 * P, Ko=4 * P, wq=5 * P, wk=6 * P, pos=7 * P, freq=8 * P, B=2, Hq=4, Hk=2, N=8, d=64, rot=64,
             qs=None, ks=None, qos=None, kos=None, axes=1, sec=None, il=0, eps=1e-6, dt=moa.MOA_BF16, wdt=moa.MOA_F32)
    a.update(kw)
    for k in ("qs", "ks", "qos", "kos", "sec"):
        a[k] = _i64(a[k])
    return moa.moa_qk_norm_rope(*a.values(), None)


ROPE_BAD = [
    (dict(Q=None), 1), (dict(Ko=None), 1), (dict(Q=P + 8), 1), (dict(pos=7 * P + 4), 1), (dict(freq=None), 1),
    (dict(B=-1), 1), (dict(N=-1), 1), (dict(d=0), 1), (dict(d=96), 2), (dict(rot=-16), 1), (dict(rot=80), 1),
    (dict(rot=24), 2), (dict(axes=0), 1), (dict(axes=5), 1), (dict(axes=2), 1), (dict(axes=2, sec=[16, 15]), 1),
    (dict(axes=2, sec=[33, -1]), 1), (dict(sec=[31]), 1), (dict(sec=[33]), 1), (dict(il=2), 1), (dict(eps=float("nan")), 1), (dict(eps=-1.0), 1), (dict(dt=2), 1),
    (dict(wdt=7), 1), (dict(Qo=2 * P), 1), (dict(Ko=3 * P), 1), (dict(Qo=P + 16), 1), (dict(Qo=5 * P), 1),
    (dict(Ko=7 * P), 1), (dict(Ko=8 * P), 1), (dict(qs=[-64, 64, 64]), 1), (dict(qs=[4096, 512, 63]), 2),
    (dict(qos=[512, 64, 0]), 1), (dict(qos=[512, 64, 32]), 1), (dict(Qo=P, qos=[4096, 64, 256]), 1),
    (dict(B=1 << 20, N=1 << 7), 2), (dict(B=1 << 20, N=64, Hq=40), 2), (dict(Hq=1 << 40), 2),
    (dict(B=1, N=1, Hq=(1 << 30) - 2), 2), (dict(qs=[1 << 41, 64, 64]), 2),
]


@pytest.mark.parametrize("kw,status", ROPE_BAD, ids=[str(i) for i in range(len(ROPE_BAD))])
def test_norm_rope_refusals(kw, status):
    assert _rope(**kw) == status


def test_norm_rope_without_rows_and_buffers_that_take_turns():
    for kw in (dict(B=0), dict(N=0), dict(Hq=0, Hk=0)):
        assert _rope(Q=None, K=None, Qo=None, Ko=None, pos=None, freq=None, **kw) == moa.MOA_OK
    # in place, and heads of one packed buffer: not refused (there is no device here, or the call would run)
    import torch
    if torch.cuda.is_available():
        pytest.skip("would run on the GPU")
    packed = dict(qs=[8 * 512, 64, 512], ks=[8 * 512, 64, 512], K=P + 256 * 2)
    for kw in (dict(Qo=P, Ko=2 * P), dict(Qo=P, Ko=P + 512, qos=packed["qs"], kos=packed["ks"], **packed),
               dict(wq=None, wk=None), dict(rot=0, freq=None, pos=None)):
        assert _rope(**kw) == moa.MOA_ERR_HIP
    # rows that take turns, but the heads of one reach into the other's
    assert _rope(Qo=P, Ko=P + 256, qos=packed["qs"], kos=packed["ks"], **dict(packed, K=P + 256)) == 1


def _rope_bwd(**kw):
    a = dict(Q=P, K=2 * P, dQo=3 * P, dKo=4 * P, wq=5 * P, wk=6 * P, pos=7 * P, freq=8 * P, dQ=9 * P, dK=10 * P, dwq=11 * P,
             dwk=12 * P, B=2, Hq=4, Hk=2, N=8, d=64, rot=64, qs=None, ks=None, dqos=None, dkos=None, dqs=None, dks=None,
             axes=1, sec=None, il=0, eps=1e-6, dt=moa.MOA_F32, wdt=moa.MOA_F32, ws=16 * P, n=1 << 20)
    a.update(kw)
    for k in ("qs", "ks", "dqos", "dkos", "dqs", "dks", "sec"):
        a[k] = _i64(a[k])
    return moa.moa_qk_norm_rope_bwd(*a.values(), None)


ROPE_BWD_BAD = [
    (dict(Q=None), 1), (dict(dKo=None), 1), (dict(dQ=None), 1), (dict(dwq=None), 1), (dict(dwk=12 * P + 4), 1),
    (dict(ws=None), 3), (dict(n=1000), 3), (dict(ws=16 * P + 8), 1), (dict(dQ=P), 1), (dict(dQ=4 * P), 1), (dict(dK=9 * P), 1),
    (dict(dwq=12 * P), 1), (dict(dwq=P), 1), (dict(ws=9 * P), 1), (dict(dwk=16 * P), 1), (dict(dwk=5 * P), 1), (dict(rot=8), 2),
]


@pytest.mark.parametrize("kw,status", ROPE_BWD_BAD, ids=[str(i) for i in range(len(ROPE_BWD_BAD))])
def test_norm_rope_bwd_refusals(kw, status):
    assert _rope_bwd(**kw) == status


def _rows(fn, **kw):
    a = dict(a=P, b=2 * P, c=4 * P, lens=8 * P, new=9 * P, table=10 * P, B=2, Hk=2, N=8, d=64, page=64, num=4, max=2, ks=None,
             vs=None, dt=moa.MOA_BF16)
    a.update(kw)
    for k in ("ks", "vs"):
        a[k] = _i64(a[k])
    if fn is moa.moa_kv4_read:      # the cache comes first
        a = {"c": a.pop("c"), **a}
    return fn(*a.values(), None)


KV4_BAD = [
    (dict(a=None), 1), (dict(b=None), 1), (dict(c=None), 1), (dict(lens=None), 1), (dict(a=P + 8), 1), (dict(c=4 * P + 8), 1),
    (dict(lens=8 * P + 2), 1), (dict(table=10 * P + 1), 1), (dict(B=-1), 1), (dict(N=-1), 1), (dict(num=-1), 1), (dict(page=0), 1),
    (dict(d=32), 2), (dict(page=48), 2), (dict(page=96), 2), (dict(page=1 << 21), 2), (dict(max=1 << 26), 2),
    (dict(N=(1 << 29) - 10), 2), (dict(B=1 << 20, Hk=1 << 12), 2), (dict(table=None), 1), (dict(table=None, max=1, num=1), 1),
    (dict(dt=2), 1), (dict(ks=[1024, -512, 64]), 1), (dict(ks=[1024, 512, 60]), 2), (dict(c=P), 1),
    (dict(c=2 * P - 16), 1),
]


@pytest.mark.parametrize("kw,status", KV4_BAD, ids=[str(i) for i in range(len(KV4_BAD))])
@pytest.mark.parametrize("name", ["moa_kv4_write", "moa_kv4_read"])
def test_kv4_rows_refusals(name, kw, status):
    assert _rows(getattr(moa, name), **kw) == status


def test_kv4_overlaps_and_no_rows():
    assert _rows(moa.moa_kv4_write, c=8 * P) == 1                           # the pool over the lengths
    assert _rows(moa.moa_kv4_read, b=P) == 1                                # keys and values in one place
    assert _rows(moa.moa_kv4_read, ks=[1024, 512, 0]) == 1                  # a row written twice
    assert _rows(moa.moa_kv4_read, a=9 * P) == 1
    for fn in (moa.moa_kv4_read, moa.moa_kv4_write):
        for kw in (dict(B=0), dict(N=0), dict(Hk=0), dict(num=0)):
            assert _rows(fn, **kw) == moa.MOA_OK


def _attn(**kw):
    a = dict(Q=P, c=4 * P, O=2 * P, lse=3 * P, lens=8 * P, new=None, table=10 * P, B=2, Hq=4, Hk=2, N=3, d=64, page=64, num=4,
             max=100, max_len=0, qs=None, os=None, scale=0.1, causal=1, odt=moa.MOA_BF16, ws=16 * P, n=1 << 24, splits=0)
    a.update(kw)
    for k in ("qs", "os"):
        a[k] = _i64(a[k])
    return moa.moa_kv4_attn_fwd(*a.values(), None)


ATTN_BAD = [
    (dict(Q=None), 1), (dict(c=None), 1), (dict(O=None), 1), (dict(lens=None), 1), (dict(Hq=3), 1), (dict(Hk=0), 1),
    (dict(scale=float("inf")), 1), (dict(causal=2), 1), (dict(odt=3), 1), (dict(splits=-1), 1), (dict(splits=257), 1),
    (dict(max_len=-1), 1), (dict(lse=3 * P + 2), 1), (dict(ws=16 * P + 4), 1), (dict(ws=None), 3), (dict(n=100), 3),
    (dict(d=96), 2), (dict(page=100), 2), (dict(N=1 << 23), 2), (dict(N=1 << 18, splits=256), 2), (dict(O=P), 1), (dict(O=4 * P), 1), (dict(lse=2 * P), 1),
    (dict(ws=2 * P), 1), (dict(ws=4 * P - 16), 1), (dict(O=8 * P), 1), (dict(qs=[768, 192, 33]), 2), (dict(os=[768, 0, 64]), 1),
    (dict(Q=P + 2), 1),
]


@pytest.mark.parametrize("kw,status", ATTN_BAD, ids=[str(i) for i in range(len(ATTN_BAD))])
def test_kv4_attn_refusals(kw, status):
    assert _attn(**kw) == status


def test_sizes():
    assert moa.moa_kv4_page_bytes(64, 128) == 64 * 136 and moa.moa_kv4_page_bytes(192, 64) == 192 * 68
    for page, d in ((0, 64), (63, 64), (64, 96), (96, 128), ((1 << 20) + 64, 64), (-64, 64)):
        assert moa.moa_kv4_page_bytes(page, d) == 0
    assert moa.moa_qk_norm_rope_bwd_workspace_bytes(2, 4, 2, 8, 64) > 0
    assert moa.moa_qk_norm_rope_bwd_workspace_bytes(2, 4, 2, 8, 96) == 0
    shape = (1, 32, 8, 1, 128, 64, 128)
    s = moa.moa_kv4_attn_num_splits(*shape, 0, 0)
    assert s > 1 and moa.moa_kv4_attn_num_splits(*shape, 0, 5) == 5 and moa.moa_kv4_attn_num_splits(*shape, 0, 300) == 1
    assert moa.moa_kv4_attn_workspace_bytes(*shape, 0, 0) >= 32 * s * 130 * 4
    assert moa.moa_kv4_attn_workspace_bytes(*shape, 0, 1) == 0
    assert moa.moa_kv4_attn_num_splits(*shape, 100, 0) == 1          # few keys are not split
    assert moa.moa_kv4_attn_num_splits(64, 32, 8, 1, 128, 64, 128, 0, 0) <= 2
    for kw in (dict(B=0), dict(N=0), dict(Hq=0)):
        assert _attn(Q=None, O=None, lse=None, ws=None, n=0, **kw) == moa.MOA_OK


def test_c_functions_without_torch():
    # the C entry points need no torch, as those of moa_attn.h
    import sys
    code = ("import sys; sys.modules['torch'] = None\n"
            "import paper_2606_07713_amd as moa\n"
            "assert moa.moa_kv4_page_bytes(64, 128) == 8704 and moa.moa_attn_status_string(0) == 'ok'\n"
            "assert moa.moa_qk_norm_rope_bwd_workspace_bytes(1, 1, 1, 1, 64) > 0\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_torch_wrappers_refuse():
    import torch
    x = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    lens = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        moa.qk_norm_rope(x)
    with pytest.raises(ValueError):
        moa.qk_norm_rope(x[0])
    with pytest.raises(ValueError, match="device"):
        moa.kv4_write(x, x, torch.zeros((1, 2, 64 * 68), dtype=torch.uint8), lens)
    with pytest.raises(ValueError, match="device"):
        moa.kv4_attn_fwd(x, torch.zeros((1, 2, 64 * 68), dtype=torch.uint8), lens)
    with pytest.raises(ValueError):
        moa.kv4_cache(1, 1, 48, 64, device="cpu")
    assert moa.kv4_cache(3, 2, 64, 128, device="cpu").shape == (3, 2, 64 * 136)


def test_torch_wrappers_refuse_a_stream_of_another_device():
    import types
    import torch
    x = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16)
    lens, cache = torch.zeros(1, dtype=torch.int32), torch.zeros((1, 2, 64 * 68), dtype=torch.uint8)
    stream = types.SimpleNamespace(device=torch.device("cuda", 1))
    for call in (lambda: moa.qk_norm_rope(x, stream=stream), lambda: moa.qk_norm_rope_bwd(x, None, x, None, stream=stream),
                 lambda: moa.kv4_write(x, x, cache, lens, stream=stream), lambda: moa.kv4_read(cache, 1, 64, lens, stream=stream),
                 lambda: moa.kv4_attn_fwd(x, cache, lens, stream=stream)):
        with pytest.raises(ValueError, match="stream of cuda:1"):
            call()


# entry point: its record's function; which argument counts the heads of each strides argument; those of
# tokens and head size; that of the sections
RECORDS = {
    "moa_qk_norm_rope": (rope._fwd, {14: 9, 15: 10, 16: 9, 17: 10}, 11, 12, 19),
    "moa_qk_norm_rope_bwd": (rope._bwd, {18: 13, 19: 14, 20: 13, 21: 14, 22: 13, 23: 14}, 15, 16, 25),
    "moa_kv4_write": (kv4._write, {13: 7, 14: 7}, 8, 9, None),
    "moa_kv4_read": (kv4._read, {13: 7, 14: 7}, 8, 9, None),
    "moa_kv4_attn_fwd": (kv4._attn, {16: 8, 17: 8}, 10, 11, None),
}


def _as_record(name):
    """The entry point ``name``, called through the record that the torch wrappers hand over."""
    packed, strides, tokens, size, sections = RECORDS[name]

    def call(*args):
        words = []
        for i, x in enumerate(args):
            if i in strides:
                h, n, d = args[strides[i]], args[tokens], args[size]
                words += [*(x or (h * n * d, n * d, d)), 1]
            elif i == sections:
                words += (1, *x, 0, 0, 0, 0)[:5] if x else (0,) * 5
            else:
                words.append(0 if x is None else x)
        return packed(packed.pack(*words))
    return call


@pytest.mark.parametrize("name,call,bad", [
    ("moa_qk_norm_rope", _rope, ROPE_BAD), ("moa_qk_norm_rope_bwd", _rope_bwd, ROPE_BWD_BAD),
    ("moa_kv4_write", lambda **kw: _rows(moa.moa_kv4_write, **kw), KV4_BAD),
    ("moa_kv4_read", lambda **kw: _rows(moa.moa_kv4_read, **kw), KV4_BAD), ("moa_kv4_attn_fwd", _attn, ATTN_BAD)])
def test_records_hand_over_every_argument(monkeypatch, name, call, bad):
    monkeypatch.setattr(moa, name, _as_record(name))
    for kw, status in bad:
        if not any(isinstance(x, int) and abs(x) >= 1 << 31 for x in kw.values()):   # strides of such sizes pass 64 bits
            assert call(**kw) == status, kw
