"""What lies around the paged cache on a pool whose elements and bytes pass 32 bits: rows in its last pages."""
import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp
from tests.gpu_util import ensure_built
from tests.test_gpu_cache_window import Windowed
from tests.test_gpu_rope import close, make, plain

pytestmark = pytest.mark.gpu
PAGES, PAGE, HKV, D = 33000, 64, 8, 128  # 2.2e9 elements, 4.3 GB, of K and of V


@pytest.fixture(scope="module")
def cache():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    ensure_built()
    yield avtp.PagedCache.new(PAGES, PAGE, HKV, D)
    torch.cuda.empty_cache()


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def status(call):
    return avtp.read_device_status(call.workspace)


def test_rows_rotated_into_the_last_pages(cache):
    x = make(100, 4, HKV, D, D, seed=1)
    slots = (PAGES * PAGE - 1 - torch.arange(100)).int()
    call = avtp.RopeCall(x["pos"].cuda(), x["inv"].cuda(), q=x["q"].cuda(), k=x["k"].cuda(), v=x["v"].cuda(), cache=cache,
                         slot_map=slots.cuda()).run()
    assert status(call) == avtp.OK
    at = slots.long().cuda()
    close(cache.k[at // PAGE, at % PAGE], plain(x["k"], x["pos"], x["inv"], "half", None, 1.0, None))
    assert torch.equal(cache.v[at // PAGE, at % PAGE].cpu(), x["v"])


def test_copies_and_compactions_in_the_last_pages(cache):
    g = torch.Generator().manual_seed(2)
    table = np.asarray([[PAGES - 1, 3, PAGES - 2, PAGES - 5]])
    rows = torch.randn(4, PAGE, HKV, D, generator=g).bfloat16()
    for t in (cache.k, cache.v):
        t[torch.from_numpy(table[0]).cuda()] = rows.cuda()
    call = avtp.CacheCopyCall(cache, i32([PAGES - 1, 3]), i32([PAGES - 7, PAGES - 8])).run()
    assert status(call) == avtp.OK
    for t in (cache.k, cache.v):
        assert torch.equal(t[[PAGES - 7, PAGES - 8]].cpu(), rows[:2])
    flat = rows.reshape(-1, HKV, D)
    keep = np.arange(3, 250, 2)
    to = [[PAGES - 9, PAGES - 10]]
    for dst in (to, None):
        call = avtp.CacheCompactCall(cache, i32([0, len(keep)]), i32(keep), i32([250]), i32(table),
                                     dst_table=i32(dst) if dst else None).run()
        assert status(call) == avtp.OK
        j = np.arange(len(keep))
        pages = np.asarray(dst[0] if dst else table[0])[j // PAGE]
        at = torch.from_numpy(pages).cuda(), torch.from_numpy(j % PAGE).cuda()
        for t in (cache.k, cache.v):
            assert torch.equal(t[at].cpu(), flat[keep])


@pytest.mark.parametrize("new", [1, 70])
def test_windows_over_the_last_pages(cache, new):
    b = Windowed([(500, new), (300, 1)], 16, HKV, D, PAGE, 100, 5)
    # the batch's pages at the end of the large pool
    n = b.cache.n_pages
    cache.k[PAGES - n:] = b.cache.k
    cache.v[PAGES - n:] = b.cache.v
    b.cache = cache
    b.dev["table"] = torch.where(b.table >= 0, b.table + PAGES - n, b.table).cuda()
    c = b.call().run()
    assert status(c) == avtp.OK
    b.check(c.o, c.lse)
