"""Steps on the paged cache that go wrong: refused rows, requests without pages."""
import numpy as np
import pytest
import torch

from gpu_util import need_gpu, say
from paper_2608_26806_amd import avtp as A
from paper_2608_26806_amd.paged import PagedCache
from paper_2608_26806_amd.progressive import ProgressivePruner
from paper_2608_26806_amd.workloads import build_layout

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    need_gpu()
    A.lib()


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def _normal(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)


def _state(cache):
    """Lengths, tables' pages in use and free pages (the stack's order aside)."""
    lens = cache.seq_len.tolist()
    held = [cache.block_table[b, :-(-n // cache.page_size)].tolist() for b, n in enumerate(lens)]
    return lens, held, sorted(cache.free_pages[:int(cache.free_count)].tolist())


def test_a_pruning_step_that_refuses_its_rows_leaves_the_cache_as_it_was():
    dl = A.DeviceLayout(build_layout([[40, 20], [30]], 3, 12, 50))
    rnd = _normal(4)
    cur, k = rnd(dl.N_tok, 64), rnd(dl.N_tok, 2, 64)
    pruner = ProgressivePruner(dl, rnd(dl.N_tok, 64))
    cache = PagedCache(dl.B, n_pages=20, max_pages=10, Hkv=2, d=64, page_size=16)
    cache.reserve(ints([0, 5, 22]), 22)
    before = _state(cache)
    say("[paged steps] refused rows")
    for bad, match in ((rnd(2, dl.N_tok, 64).transpose(0, 1), "contiguous"),
                       (rnd(dl.N_tok, 132)[:, :128].unflatten(1, (2, 64)), "aligned"), (k.cpu(), "GPU")):
        for kv in (dict(k=bad, v=k), dict(k=k, v=bad)):
            with pytest.raises(ValueError, match=match):
                pruner.step(cur, cache=cache, **kv)
            assert _state(cache) == before and pruner.dl is dl
    h, *_ = pruner.step(cur, cache=cache, k=k, v=k)
    assert sum(_state(cache)[0]) == 22 + h.shape[0]
