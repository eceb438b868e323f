"""Attention in a window, the host side without a GPU: argument checks (every refusal returns before the first CUDA
call) and the struct."""
import ctypes

import pytest

from paper_2608_26806_gb300 import avtp
from tests.gpu_util import ensure_built

FAKE = 0x7f0000000000  # a 256-aligned address that is never dereferenced on these paths
BIG = 1 << 34
I, U, G, W = avtp.ERR_INVALID_ARG, avtp.ERR_UNSUPPORTED, avtp.ERR_RANGE, avtp.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return ensure_built()


def _cache(page=64):
    s = (page * 8 * 128, 8 * 128, 128)
    return avtp._Cache(FAKE, FAKE, 100, page, 8, 128, *s, *s)


def _attn(T=100, max_new=70, max_pages=1000):
    return avtp._CacheAttnArgs(4, T, max_new, 32, FAKE, 4096, FAKE, FAKE, FAKE, max_pages, max_pages, 128 ** -0.5, FAKE, 4096,
                               FAKE, T)


def both(lib, c, a, w, code):
    size = ctypes.c_size_t()
    refs = [ctypes.byref(x) if x is not None else None for x in (c, a, w)]
    assert lib.avtp_cache_window_attention_workspace_size(*refs, ctypes.byref(size)) == code
    if code != avtp.OK:
        assert lib.avtp_cache_window_attention(*refs, FAKE, BIG, None) == code
    return size.value


@pytest.mark.parametrize("window,sinks,code", [(0, 0, I), (-3, 0, I), (5, -1, I), (1, 0, avtp.OK),
                                               ((1 << 31) - 1, (1 << 31) - 1, avtp.OK)])
def test_windows(lib, window, sinks, code):
    both(lib, _cache(), _attn(), avtp._CacheWindow(window, sinks), code)


def test_what_the_attention_refuses_is_refused(lib):
    w = avtp._CacheWindow(10, 2)
    both(lib, None, _attn(), w, I)
    both(lib, _cache(), None, w, I)
    both(lib, _cache(), _attn(), None, I)
    both(lib, _cache(page=24), _attn(), w, U)
    a = _attn()
    a.softmax_scale = 0.0
    both(lib, _cache(), a, w, I)
    c, a = _cache(), _attn()
    need = both(lib, c, a, w, avtp.OK)
    size = ctypes.c_size_t()
    assert lib.avtp_cache_attention_workspace_size(ctypes.byref(c), ctypes.byref(a), ctypes.byref(size)) == avtp.OK
    assert size.value == need
    args = (ctypes.byref(c), ctypes.byref(a), ctypes.byref(w))
    assert lib.avtp_cache_window_attention_workspace_size(*args, None) == I
    for ws, n in ((None, BIG), (FAKE + 16, BIG), (FAKE, need - 1)):
        assert lib.avtp_cache_window_attention(*args, ws, n, None) == W


def test_a_line_of_work_too_long_to_count_is_refused(lib):
    """Blocks of rows (new tokens / 64 and a few) times the blocks of 128 keys that each sees, times 8 KV heads, of 2^27 keys
    a request: refused from 2^31 on, but for calls without chunks or without a window to speak of."""
    c = _cache(page=1 << 14)
    for T, window, code in ((4096, 1 << 20, avtp.OK), (1 << 24, 1 << 10, avtp.OK), (1 << 24, 1 << 20, G),
                            (1 << 24, 1 << 30, avtp.OK)):
        a = _attn(T=T, max_pages=1 << 13)
        both(lib, c, a, avtp._CacheWindow(window, 4), code)
    a = _attn(T=1 << 24, max_new=8, max_pages=1 << 13)
    both(lib, c, a, avtp._CacheWindow(1 << 20, 4), avtp.OK)
    a = _attn(T=1 << 24, max_pages=1 << 13)
    both(lib, c, a, avtp._CacheWindow(1 << 10, 1 << 26), G)


def test_the_struct_matches_the_header():
    assert ctypes.sizeof(avtp._CacheWindow) == 8 and avtp._CacheWindow.n_sinks.offset == 4
