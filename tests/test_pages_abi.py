"""The calls on the paged cache reject bad arguments on the host, before
anything is launched (no GPU here: the pointers are host memory that no call
dereferences), also with the host layer under the address and
undefined-behaviour sanitizers."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest
import torch

from paper_2608_26806_amd import avtp as A

BUF = torch.zeros(4096 + 256, dtype=torch.uint8)
P = ctypes.c_void_p((BUF.data_ptr() + 255) // 256 * 256)
ODD = ctypes.c_void_p(P.value + 8)
I = A.ERR_INVALID_ARG
U = A.ERR_UNSUPPORTED
BIG = 1 << 40


def _pages(**patch):
    f = dict(k=P.value, v=P.value, dtype=A.BF16, n_pages=10, page_size=16, Hkv=2, d=128)
    f.update(patch)
    return A._Pages(*[f[n] for n, _ in A._Pages._fields_])


OTHER = ctypes.c_void_p(P.value + 64)
TABLES = dict(stream=None, B=3, page_size=16, cu_new=P, seq_len=P, free_pages=P, n_pages=10, free_count=P,
              block_table=P, max_pages=4, slot_map=P, n_new=5, seq_len_out=OTHER, free_count_out=OTHER, status=None)


@pytest.mark.parametrize("patch, rc", [
    (dict(B=0), I), (dict(B=(1 << 16) + 1), U), (dict(page_size=0), I),
    (dict(page_size=8), U), (dict(page_size=48), U), (dict(page_size=2048), U), (dict(n_pages=0), I),
    (dict(max_pages=0), I), (dict(max_pages=1 << 30), U), (dict(n_pages=1 << 28), U), (dict(cu_new=None), I),
    (dict(seq_len=None), I), (dict(free_pages=None), I), (dict(free_count=None), I), (dict(block_table=None), I),
    (dict(slot_map=None), I), (dict(n_new=-1), I), (dict(n_new=BIG), U), (dict(seq_len_out=None), I),
    (dict(free_count_out=None), I), (dict(seq_len_out=P), I), (dict(free_count_out=P), I)])
def test_tables_refusals(patch, rc):
    assert A.lib().avtp_page_tables(*{**TABLES, **patch}.values()) == rc


TRIM = dict(stream=None, B=3, page_size=16, keep_len=P, seq_len=P, block_table=P, max_pages=4, free_pages=P,
            n_pages=10, free_count=P, seq_len_out=OTHER, free_count_out=OTHER, status=None)


@pytest.mark.parametrize("patch, rc", [
    (dict(B=-1), I), (dict(B=(1 << 16) + 1), U), (dict(page_size=24), U), (dict(max_pages=0), I),
    (dict(keep_len=None), I), (dict(seq_len=None), I), (dict(block_table=None), I), (dict(free_pages=None), I),
    (dict(n_pages=-4), I), (dict(free_count=None), I), (dict(seq_len_out=None), I), (dict(free_count_out=None), I),
    (dict(seq_len_out=P), I), (dict(free_count_out=P), I)])
def test_trim_refusals(patch, rc):
    assert A.lib().avtp_page_trim(*{**TRIM, **patch}.values()) == rc


BAD_PAGES = [(dict(k=None), I), (dict(v=None), I), (dict(k=P.value + 8), I), (dict(v=P.value + 2), I),
             (dict(dtype=7), U), (dict(n_pages=0), I), (dict(n_pages=1 << 28), U), (dict(page_size=20), U),
             (dict(page_size=0), I), (dict(Hkv=0), I), (dict(Hkv=300), U), (dict(d=96), U)]
STORE = dict(stream=None, pages=None, k=P, ks=256, v=P, vs=256, n_src=8, slot_map=P, keep_idx=None, n=8)


@pytest.mark.parametrize("pages, patch, rc", [(p, {}, rc) for p, rc in BAD_PAGES] + [
    ({}, dict(k=None), I), ({}, dict(v=None), I), ({}, dict(k=ODD), I), ({}, dict(v=ODD), I), ({}, dict(ks=255), I),
    ({}, dict(vs=128), I), ({}, dict(ks=260), I), ({}, dict(ks=1 << 62), I), ({}, dict(ks=-256), I),
    ({}, dict(n_src=-1), I), ({}, dict(n=9), I), ({}, dict(n=-1), I), ({}, dict(slot_map=None), I),
    ({}, dict(n=BIG, n_src=BIG), U), ({}, dict(n=0), A.OK), ({}, dict(n_src=0, keep_idx=P), A.OK)])
def test_store_refusals(pages, patch, rc):
    a = {**STORE, **patch}
    a["pages"] = ctypes.byref(_pages(**pages))
    assert A.lib().avtp_page_store(*a.values()) == rc


ATT = dict(stream=None, pages=None, q=P, qs=512, Hq=4, B=2, N_q=6, cu_q=P, kv_len=P, table=P, max_pages=4,
           max_kv=64, scale=0.1, out=P, os=512, lse=None, status=None, ws=P, ws_bytes=1 << 62)


@pytest.mark.parametrize("pages, patch, rc", [(p, {}, rc) for p, rc in BAD_PAGES] + [
    ({}, dict(q=None), I), ({}, dict(out=None), I), ({}, dict(q=ODD), I), ({}, dict(out=ODD), I),
    ({}, dict(qs=511), I), ({}, dict(os=256), I), ({}, dict(qs=516), I), ({}, dict(Hq=3), I), ({}, dict(Hq=0), I),
    ({}, dict(Hq=512), U), ({}, dict(B=0), I), ({}, dict(B=1 << 20), U), ({}, dict(N_q=-1), I),
    ({}, dict(N_q=1 << 30), U), ({}, dict(cu_q=None), I), ({}, dict(kv_len=None), I), ({}, dict(table=None), I),
    ({}, dict(max_pages=0), I), ({}, dict(max_kv=-1), I), ({}, dict(scale=0.0), I), ({}, dict(scale=-1.0), I),
    ({}, dict(scale=float("nan")), I), ({}, dict(scale=float("inf")), I),
    ({}, dict(max_kv=1 << 20, ws=None), A.ERR_WORKSPACE), ({}, dict(max_kv=1 << 20, ws=ODD), A.ERR_WORKSPACE),
    ({}, dict(max_kv=1 << 20, ws_bytes=1), A.ERR_WORKSPACE), ({}, dict(N_q=0, q=None, out=None), A.OK)])
def test_attention_refusals(pages, patch, rc):
    a = {**ATT, **patch}
    a["pages"] = ctypes.byref(_pages(**pages))
    assert A.lib().avtp_page_attention(*a.values()) == rc


def test_attention_refuses_more_blocks_than_a_launch_has():
    # 2^16 sequences of 256 key heads: half of the blocks for the rows, half for tiles' ends
    for N_q in (1 << 22, (1 << 31) // 256 - 1):
        a = {**ATT, "pages": ctypes.byref(_pages(Hkv=256)), "Hq": 256, "B": 1 << 16, "N_q": N_q, "qs": 1 << 15,
             "os": 1 << 15}
        assert A.lib().avtp_page_attention(*a.values()) == U
        assert A.lib().avtp_page_attention_workspace_size(a["pages"], 256, 1 << 16, N_q, 64) == 0


def test_null_pool():
    lib = A.lib()
    assert lib.avtp_page_store(*{**STORE, "pages": None}.values()) == I
    assert lib.avtp_page_attention(*{**ATT, "pages": None}.values()) == I
    assert lib.avtp_page_attention_workspace_size(None, 4, 2, 6, 64) == 0


def test_workspace_size():
    size = lambda Hq, B, N, kv, **p: A.lib().avtp_page_attention_workspace_size(  # noqa: E731
        ctypes.byref(_pages(**p)), Hq, B, N, kv)
    assert size(4, 2, 0, 1 << 20) == 0
    assert size(4, 2, 6, 64) == 0                                    # few rows and keys: nothing is cut
    one = size(4, 1, 1, 2000)
    assert one >= 2 * 16 * (128 + 1) * 4                             # the parts of one cut tile
    assert one <= size(4, 1, 1, 1 << 20) == size(4, 1, 2, 1 << 20)   # as many workers as the chip holds
    assert size(4, 1, 1, 64, dtype=A.FP32) > 0
    assert size(4, 1, 9000, 1 << 20) == 0                            # chunks that fill the chip uncut
    assert size(4, 1, 100, 1 << 20) >= 2 * 128 * (128 + 1) * 4       # and one that does not
    assert size(3, 1, 1, 64) == 0 and size(4, 0, 1, 64) == 0 and size(4, 1, 1, -1) == 0
    # bounds at the edge of what is allowed: no overflow (the sanitizer build runs this too)
    assert size(256, 1 << 16, (2 ** 31 - 1) // 256, 2 ** 62, Hkv=256) >= 0
    assert size(1, 1, 1, 2 ** 63 - 1, Hkv=1) > 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        A.Pages(k, k)
    with pytest.raises(ValueError, match="n_pages"):
        A.Pages(k, k[:3])
    with pytest.raises(ValueError, match="n_pages"):
        A.Pages(k[0], k[0])
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        A.page_tables(16, i, i[:3], i, i, torch.zeros(3, 4, dtype=torch.int32), 4, stream=ctypes.c_void_p(0))
    with pytest.raises(ValueError, match="block_table"):
        A.page_trim(16, i, i, torch.zeros(3, 4, dtype=torch.int32), i, i, stream=ctypes.c_void_p(0))


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
