"""Outputs of forks and releases that share memory with each other or with what
other blocks still read are refused on the host (no GPU here: the pointers are host
memory that no call dereferences)."""
import ctypes

import pytest
import torch

from paper_2608_26806_amd import avtp as A

BUF = torch.zeros(4096, dtype=torch.uint8)
BASE = (BUF.data_ptr() + 255) // 256 * 256
at = lambda x: ctypes.c_void_p(BASE + 4 * x)  # noqa: E731  (element x)
B = 3
FORK = dict(stream=None, B=B, page_size=16, parent=at(0), fork_len=at(3), seq_len=at(6), free_pages=at(9), n_pages=10,
            free_count=at(19), table=at(20), max_pages=4, gone=at(32), seq_len_out=at(64), free_count_out=at(67), src=at(68),
            dst=at(71), gone_out=at(74), status=None)
REL = dict(stream=None, B=B, page_size=16, keep_len=at(0), seq_len=at(3), table=at(6), max_pages=4, free_pages=at(20),
           n_pages=10, free_count=at(30), window=8, sinks=4, gone=at(31), seq_len_out=at(64), free_count_out=at(67),
           gone_out=at(68), status=None, ws=at(128), ws_bytes=1 << 20)


def shared(outs, ins):
    """Patches that lay one buffer of (name, length) onto another, whole or by an element."""
    for i, (a, n) in enumerate(outs):
        for b, m in outs[i + 1:] + ins:
            for shift in sorted({0, m - 1, 1 - n}):
                yield a, b, shift


def place(call, name):
    return (call[name].value - BASE) // 4


FORK_OUTS = [("seq_len_out", B), ("src", B), ("dst", B), ("gone_out", B), ("free_count_out", 1)]
FORK_INS = [("parent", B), ("fork_len", B), ("seq_len", B), ("gone", B), ("free_count", 1), ("free_pages", 10), ("table", 12)]


@pytest.mark.parametrize("a, b, shift", shared(FORK_OUTS, FORK_INS))
def test_fork(a, b, shift):
    x = max(0, place(FORK, b) + shift)
    assert A.lib().avtp_page_fork(*{**FORK, a: at(x)}.values()) == A.ERR_INVALID_ARG


REL_OUTS = [("seq_len_out", B), ("gone_out", B), ("free_count_out", 1)]
REL_INS = [("keep_len", B), ("seq_len", B), ("gone", B), ("free_count", 1), ("table", 12), ("free_pages", 10)]


@pytest.mark.parametrize("a, b, shift", shared(REL_OUTS, REL_INS))
def test_release(a, b, shift):
    x = max(0, place(REL, b) + shift)
    assert A.lib().avtp_page_release(*{**REL, a: at(x)}.values()) == A.ERR_INVALID_ARG
