"""The calls of a layer's step around the paged cache reject bad arguments on the
host, before anything is launched (no GPU here: the pointers are host memory that no
call dereferences), also with the host layer under the address and
undefined-behaviour sanitizers."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest
import torch

from paper_2608_26806_amd import avtp as A
from paper_2608_26806_amd.paged import PagedCache
from paper_2608_26806_amd.rotary import Rotary

BUF = torch.zeros(4096 + 256, dtype=torch.uint8)
BASE = (BUF.data_ptr() + 255) // 256 * 256
P, OTHER, THIRD, FOURTH, FIFTH, ODD = (ctypes.c_void_p(BASE + x) for x in (0, 64, 128, 192, 256, 8))
I, U, W = A.ERR_INVALID_ARG, A.ERR_UNSUPPORTED, A.ERR_WORKSPACE
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")


def _pages(**patch):
    f = dict(k=BASE, v=BASE, dtype=A.BF16, n_pages=10, page_size=16, Hkv=2, d=128)
    f.update(patch)
    return A._Pages(*[f[n] for n, _ in A._Pages._fields_])


def _rot(**patch):
    f = dict(turns=BASE, plane=None, rot_dim=64, interleaved=0, planes=1, scale=1.0)
    f.update(patch)
    return A._Rotary(*[f[n] for n, _ in A._Rotary._fields_])


BAD_PAGES = [(dict(k=None), I), (dict(v=None), I), (dict(k=BASE + 8), I), (dict(dtype=7), U), (dict(n_pages=0), I),
             (dict(n_pages=1 << 28), U), (dict(page_size=20), U), (dict(Hkv=0), I), (dict(Hkv=300), U), (dict(d=96), U)]
BAD_ROT = [(dict(turns=None), I), (dict(turns=BASE + 4), I), (dict(plane=BASE + 2), I), (dict(rot_dim=0), I),
           (dict(rot_dim=-16), I), (dict(rot_dim=24), U), (dict(rot_dim=144), U), (dict(planes=0), I), (dict(planes=5), U),
           (dict(scale=NAN), I), (dict(scale=INF), I), (dict(planes=2), I)]  # (two planes, stride 0)

NORM = dict(stream=None, rot=None, dtype=A.BF16, d=128, n=8, pos=P, pos_stride=0, qw=None, kw=None, eps=1e-6, q=P, qs=512,
            Hq=4, qo=OTHER, qos=512, k=P, ks=256, Hkv=2, ko=OTHER, kos=256)


@pytest.mark.parametrize("rot, patch, rc", [(r, {}, rc) for r, rc in BAD_ROT] + [
    ({}, dict(dtype=2), U), ({}, dict(d=96), U), (dict(rot_dim=128), dict(d=64), U), ({}, dict(n=-1), I),
    ({}, dict(n=BIG), U), ({}, dict(pos=None), I), ({}, dict(pos=ctypes.c_void_p(BASE + 4)), I),
    (dict(planes=3), dict(pos_stride=7), I), (dict(planes=3), dict(pos_stride=1 << 62), I), ({}, dict(eps=-1e-9), I),
    ({}, dict(eps=NAN), I), ({}, dict(eps=INF), I), ({}, dict(q=None), I), ({}, dict(q=ODD), I), ({}, dict(qs=511), I),
    ({}, dict(qs=516), I), ({}, dict(qs=256), I), ({}, dict(qo=None), I), ({}, dict(qo=ODD), I), ({}, dict(qos=508), I),
    ({}, dict(qo=P, qos=520), I), ({}, dict(k=None), I), ({}, dict(ks=128), I), ({}, dict(ko=None), I),
    ({}, dict(ko=P, kos=264), I), ({}, dict(Hq=-1), I), ({}, dict(Hkv=-1), I), ({}, dict(Hq=257, qs=1 << 16, qos=1 << 16), U),
    ({}, dict(Hkv=300), U), ({}, dict(n=0, q=None, pos=None), A.OK), ({}, dict(Hq=0, Hkv=0, q=None, k=None), A.OK)])
def test_norm_rotary_refusals(rot, patch, rc):
    a = {**NORM, **patch}
    a["rot"] = ctypes.byref(_rot(**rot))
    assert A.lib().avtp_norm_rotary(*a.values()) == rc


STORE = dict(stream=None, pages=None, rot=None, n=8, pos=P, pos_stride=0, qw=None, kw=None, eps=1e-6, q=P, qs=512, Hq=4,
             qo=OTHER, qos=512, k=P, ks=256, v=P, vs=256, slot=P)


@pytest.mark.parametrize("pages, rot, patch, rc", [(p, {}, {}, rc) for p, rc in BAD_PAGES] + [
    ({}, r, {}, rc) for r, rc in BAD_ROT] + [
    (dict(d=64), dict(rot_dim=128), {}, U), ({}, {}, dict(n=-1), I), ({}, {}, dict(pos=None), I), ({}, {}, dict(eps=NAN), I),
    ({}, {}, dict(q=None), I), ({}, {}, dict(qo=None), I), ({}, {}, dict(qo=P, qos=520), I), ({}, {}, dict(Hq=-1), I),
    ({}, {}, dict(Hq=300), U), ({}, {}, dict(k=None), I), ({}, {}, dict(ks=128), I), ({}, {}, dict(v=ODD), I),
    ({}, {}, dict(vs=260), I), ({}, {}, dict(slot=None), I), ({}, {}, dict(n=0, slot=None), A.OK)])
def test_store_rotary_refusals(pages, rot, patch, rc):
    a = {**STORE, **patch}
    a["pages"], a["rot"] = ctypes.byref(_pages(**pages)), ctypes.byref(_rot(**rot))
    assert A.lib().avtp_page_store_rotary(*a.values()) == rc


ATT = dict(stream=None, pages=None, q=P, qs=512, Hq=4, B=2, N_q=6, cu_q=P, kv_len=P, table=P, max_pages=4,
           max_kv=64, window=16, sinks=4, scale=0.1, out=P, os=512, lse=None, status=None, ws=P, ws_bytes=1 << 62)


@pytest.mark.parametrize("pages, patch, rc", [(p, {}, rc) for p, rc in BAD_PAGES] + [
    ({}, dict(window=0), I), ({}, dict(window=-5), I), ({}, dict(sinks=-1), I), ({}, dict(q=None), I), ({}, dict(os=256), I),
    ({}, dict(Hq=3), I), ({}, dict(B=0), I), ({}, dict(B=1 << 20), U), ({}, dict(N_q=-1), I), ({}, dict(N_q=1 << 30), U),
    ({}, dict(cu_q=None), I), ({}, dict(kv_len=None), I), ({}, dict(table=None), I), ({}, dict(max_pages=0), I),
    ({}, dict(max_kv=-1), I), ({}, dict(scale=0.0), I), ({}, dict(scale=NAN), I),
    ({}, dict(max_kv=1 << 20, window=1 << 20, ws=None), W), ({}, dict(max_kv=1 << 20, window=1 << 20, ws_bytes=1), W),
    ({}, dict(N_q=0, q=None, out=None), A.OK)])
def test_window_attention_refusals(pages, patch, rc):
    a = {**ATT, **patch}
    a["pages"] = ctypes.byref(_pages(**pages))
    assert A.lib().avtp_page_attention_window(*a.values()) == rc


def test_window_workspace_size():
    size = lambda Hq, B, N, kv, w, s, **p: A.lib().avtp_page_attention_window_workspace_size(  # noqa: E731
        ctypes.byref(_pages(**p)), Hq, B, N, kv, w, s)
    assert size(4, 2, 6, 1 << 20, 0, 0) == size(4, 2, 6, 1 << 20, 8, -1) == size(3, 1, 1, 64, 8, 0) == 0
    # as for caches of what a row sees
    whole = lambda kv: A.lib().avtp_page_attention_workspace_size(ctypes.byref(_pages()), 4, 1, 1, kv)  # noqa: E731
    assert size(4, 1, 1, 1 << 20, 5000, 120) == whole(5120) > 0
    assert size(4, 1, 1, 2000, 1 << 30, 1 << 30) == whole(2000) > 0
    assert size(4, 1, 1, 1 << 20, 100, 4) == 0
    big = 2 ** 31 - 1
    assert size(256, 1 << 16, big // 256, 2 ** 62, big, big, Hkv=256) >= 0
    assert A.lib().avtp_page_attention_window_workspace_size(None, 4, 2, 6, 64, 8, 0) == 0


FORK = dict(stream=None, B=3, page_size=16, parent=P, fork_len=P, seq_len=P, free_pages=P, n_pages=10, free_count=P, table=P,
            max_pages=4, gone=P, seq_len_out=OTHER, free_count_out=OTHER, src=THIRD, dst=FOURTH, gone_out=FIFTH, status=None)


@pytest.mark.parametrize("patch, rc", [
    (dict(B=0), I), (dict(B=(1 << 16) + 1), U), (dict(page_size=0), I), (dict(page_size=8), U), (dict(n_pages=0), I),
    (dict(max_pages=0), I), (dict(max_pages=1 << 30), U), (dict(n_pages=1 << 28), U), (dict(gone=None), I),
    (dict(gone_out=None), I), (dict(free_count_out=P), I), (dict(src=P), I), (dict(dst=P), I), (dict(gone_out=P), I),
    (dict(seq_len_out=P), I)] + [(dict([(n, None)]), I) for n in (
        "parent", "fork_len", "seq_len", "free_pages", "free_count", "table", "seq_len_out", "free_count_out", "src", "dst")])
def test_fork_refusals(patch, rc):
    assert A.lib().avtp_page_fork(*{**FORK, **patch}.values()) == rc


@pytest.mark.parametrize("pages, patch, rc", [(p, {}, rc) for p, rc in BAD_PAGES] + [
    ({}, dict(src=None), I), ({}, dict(dst=None), I), ({}, dict(n=-1), I), ({}, dict(n=BIG), U), ({}, dict(n=0, src=None), A.OK)])
def test_copy_refusals(pages, patch, rc):
    a = {**dict(stream=None, pages=ctypes.byref(_pages(**pages)), src=P, dst=OTHER, n=4), **patch}
    assert A.lib().avtp_page_copy(*a.values()) == rc


REL = dict(stream=None, B=3, page_size=16, keep_len=P, seq_len=P, table=P, max_pages=4, free_pages=P, n_pages=10, free_count=P,
           window=8, sinks=4, gone=P, seq_len_out=OTHER, free_count_out=OTHER, gone_out=THIRD, status=None, ws=P,
           ws_bytes=1 << 20)


@pytest.mark.parametrize("patch, rc", [
    (dict(B=-1), I), (dict(B=(1 << 16) + 1), U), (dict(page_size=24), U), (dict(max_pages=0), I), (dict(n_pages=-4), I),
    (dict(window=-1), I), (dict(sinks=-1), I), (dict(window=(1 << 30) + 1), U), (dict(sinks=(1 << 30) + 1), U),
    (dict(gone=None), I), (dict(gone_out=None), I), (dict(gone=None, gone_out=None), I), (dict(seq_len_out=P), I),
    (dict(gone_out=P), I), (dict(gone_out=OTHER), I), (dict(free_count_out=P), I), (dict(ws=None), W), (dict(ws=ODD), W),
    (dict(ws_bytes=83), W)] + [(dict([(n, None)]), I) for n in (
        "keep_len", "seq_len", "table", "free_pages", "free_count", "seq_len_out", "free_count_out")])
def test_release_refusals(patch, rc):
    assert A.lib().avtp_page_release(*{**REL, **patch}.values()) == rc


def test_release_workspace_size():
    size = A.lib().avtp_page_release_workspace_size
    assert size(0) == size(-3) == 0
    for n in (1, 10, 1023, 1024, 1025, 100000):        # two counts a page, rounded up to chunks, and a sum a chunk
        assert 8 * n + 4 <= size(n) <= 8 * (n + 1024) + n // 256 + 64
        assert A.lib().avtp_page_release(*{**REL, "n_pages": n, "ws_bytes": size(n) - 1}.values()) == W
    assert size(2 ** 31 - 1) > 2 ** 34


def test_null_pool_and_rotation():
    lib = A.lib()
    rot, pages = ctypes.byref(_rot()), ctypes.byref(_pages())
    assert lib.avtp_norm_rotary(*NORM.values()) == I
    assert lib.avtp_page_store_rotary(*{**STORE, "rot": rot}.values()) == I
    assert lib.avtp_page_store_rotary(*{**STORE, "pages": pages}.values()) == I
    assert lib.avtp_page_attention_window(*ATT.values()) == I
    assert lib.avtp_page_copy(None, None, P, P, 1) == I


def test_binding_refuses_host_tensors():
    i = torch.zeros(4, dtype=torch.int32)
    table = torch.zeros(3, 4, dtype=torch.int32)
    s = ctypes.c_void_p(0)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        A.page_fork(16, i, i, i[:3], i, i, table, stream=s)
    with pytest.raises(ValueError, match="GPU"):
        A.page_release(16, i, i[:3], table, i, i, stream=s)
    with pytest.raises(ValueError, match="block_table"):
        A.page_release(16, i, i, table, i, i, stream=s)
    with pytest.raises(ValueError, match="GPU"):
        A.norm_rotary(Rotary(64, device="cpu"), torch.zeros(1, 3, dtype=torch.int64), x, x, stream=s)
    with pytest.raises(ValueError, match="q or k"):
        A.norm_rotary(Rotary(64, device="cpu"), torch.zeros(1, 3, dtype=torch.int64), None, None, stream=s)


def test_cache_refuses_windows_that_are_none():
    for bad in (dict(window=0), dict(window=-4), dict(sinks=4), dict(window=8, sinks=-1)):
        with pytest.raises(ValueError, match="window"):
            PagedCache(2, 8, 4, 2, 64, device="cpu", **bad)


@pytest.mark.skipif("AVTP_LIBRARY" in os.environ, reason="the sanitized run itself")
def test_refusals_are_clean_under_asan_and_ubsan(tmp_path):
    from test_host_sanitizers import ROOT, _asan_runtime
    rt = _asan_runtime()
    if rt is None or shutil.which("/opt/rocm/bin/hipcc") is None:
        pytest.skip("clang ASan runtime or hipcc not available")
    from paper_2608_26806_amd import build as B
    lib = B.build_host_sanitized(str(tmp_path / "libavtp_san.so"))
    env = dict(os.environ)
    pre = env.get("LD_PRELOAD", "")
    env.update(LD_PRELOAD=rt + (":" + pre if pre else ""), AVTP_LIBRARY=lib,
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-s", "-p",
                        "no:cacheprovider"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert r.returncode == 0 and " passed" in out, out[-4000:]
