"""The paged cache's host side, without a GPU: argument checks of the C entry points (every refusal
returns before the first CUDA call), the binding's structs and its refusals."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp
from tests.cache_util import slots_plain
from tests.gpu_util import ensure_built

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7f0000000000  # a 256-aligned address that is never dereferenced on these paths
BIG = 1 << 34


@pytest.fixture(scope="module")
def lib():
    return ensure_built()


def _cache(pages=100, page=64, h=8, d=128):
    s = (page * h * d, h * d, d)
    return avtp._Cache(FAKE, FAKE, pages, page, h, d, *s, *s)


def _slots(R=4, n=100):
    return avtp._CacheSlotsArgs(R, n, 64, 100, 10, 10, FAKE, FAKE, FAKE, 50, FAKE, FAKE, FAKE, FAKE, FAKE)


def _write(n=10, h=8, d=128):
    return avtp._CacheWriteArgs(FAKE, FAKE, h * d, h * d, 20, FAKE, FAKE, n)


def _attn(R=4, T=100, hq=32, d=128):
    return avtp._CacheAttnArgs(R, T, 7, hq, FAKE, hq * d, FAKE, FAKE, FAKE, 10, 10, d ** -0.5, FAKE, hq * d, FAKE, T)


def _with(struct, **fields):
    for k, v in fields.items():
        setattr(struct, k, v)
    return struct


I, U, G, W = avtp.ERR_INVALID_ARG, avtp.ERR_UNSUPPORTED, avtp.ERR_RANGE, avtp.ERR_WORKSPACE


@pytest.mark.parametrize("field,value,code", [
    ("n_requests", 0, I), ("n_tokens", -1, I), ("n_tokens", 1 << 31, G), ("page_size", 0, I), ("n_pages", 0, I),
    ("n_pages", 1 << 26, G), ("max_pages", 0, I), ("table_stride", 9, I), ("cu_new", None, I), ("free_pages", None, I),
    ("n_free", -1, I), ("n_free", 1 << 31, G), ("block_table", None, I), ("seq_len", None, I), ("slot_map", None, I)])
def test_slots_arguments(lib, field, value, code):
    a = _with(_slots(), **{field: value})
    assert lib.avtp_cache_slots(ctypes.byref(a), FAKE, BIG, None) == code
    size = ctypes.c_size_t()
    assert lib.avtp_cache_slots_workspace_size(ctypes.byref(a), ctypes.byref(size)) == code


@pytest.mark.parametrize("R,code", [((1 << 31) - 1, G), ((1 << 31) - 1024, G), ((1 << 31) - 1025, avtp.OK)])
def test_slots_refuse_more_requests_than_their_loops_count(lib, R, code):
    a, size = _with(_slots(), n_requests=R), ctypes.c_size_t()
    assert lib.avtp_cache_slots_workspace_size(ctypes.byref(a), ctypes.byref(size)) == code
    if code != avtp.OK:
        assert lib.avtp_cache_slots(ctypes.byref(a), FAKE, BIG, None) == code


def test_workspaces_are_checked(lib):
    c, s, w, a = _cache(), _slots(), _write(), _attn()
    size = ctypes.c_size_t()
    assert lib.avtp_cache_slots_workspace_size(ctypes.byref(s), ctypes.byref(size)) == avtp.OK
    assert lib.avtp_cache_slots(ctypes.byref(s), FAKE, size.value - 1, None) == W
    assert lib.avtp_cache_attention_workspace_size(ctypes.byref(c), ctypes.byref(a), ctypes.byref(size)) == avtp.OK
    assert lib.avtp_cache_attention(ctypes.byref(c), ctypes.byref(a), FAKE, size.value - 1, None) == W
    for ws in (None, FAKE + 16):
        assert lib.avtp_cache_slots(ctypes.byref(s), ws, BIG, None) == W
        assert lib.avtp_cache_write(ctypes.byref(c), ctypes.byref(w), ws, BIG, None) == W
        assert lib.avtp_cache_attention(ctypes.byref(c), ctypes.byref(a), ws, BIG, None) == W
    assert lib.avtp_cache_write(ctypes.byref(c), ctypes.byref(w), FAKE, 8, None) == W
    assert lib.avtp_cache_slots(None, FAKE, BIG, None) == I
    assert lib.avtp_cache_write(None, ctypes.byref(w), FAKE, BIG, None) == I
    assert lib.avtp_cache_write(ctypes.byref(c), None, FAKE, BIG, None) == I
    assert lib.avtp_cache_attention(ctypes.byref(c), None, FAKE, BIG, None) == I
    assert lib.avtp_cache_slots_workspace_size(ctypes.byref(s), None) == I
    assert lib.avtp_cache_attention_workspace_size(ctypes.byref(c), ctypes.byref(a), None) == I


@pytest.mark.parametrize("field,value,code", [
    ("k", None, I), ("v", None, I), ("k", FAKE + 8, U), ("v", FAKE + 8, U), ("n_pages", 0, I), ("page_size", 0, I),
    ("n_pages", 1 << 26, G), ("n_kv_heads", 0, I), ("n_kv_heads", 1 << 17, G), ("head_dim", 96, U),
    ("k_page_stride", 64 * 1024 + 4, U), ("k_page_stride", 0, I), ("v_token_stride", 1028, U), ("v_head_stride", 0, I),
    ("k_head_stride", 1 << 20, U), ("v_token_stride", 1 << 20, U), ("v_page_stride", 1 << 39, G)])
def test_cache_arguments(lib, field, value, code):
    c = _with(_cache(), **{field: value})
    assert lib.avtp_cache_write(ctypes.byref(c), ctypes.byref(_write()), FAKE, BIG, None) == code
    assert lib.avtp_cache_attention(ctypes.byref(c), ctypes.byref(_attn()), FAKE, BIG, None) == code


@pytest.mark.parametrize("field,value,code", [
    ("n", -1, I), ("n", 1 << 31, G), ("n_rows", -1, I), ("n_rows", 1 << 31, G), ("k", None, I), ("v", None, I),
    ("slot_map", None, I), ("k_stride", 1016, I), ("v_stride", 1016, I), ("k_stride", 1028, U), ("v_stride", 1028, U),
    ("k", FAKE + 8, U), ("v", FAKE + 2, U)])
def test_write_arguments(lib, field, value, code):
    a = _with(_write(), **{field: value})
    assert lib.avtp_cache_write(ctypes.byref(_cache()), ctypes.byref(a), FAKE, BIG, None) == code


@pytest.mark.parametrize("field,value,code", [
    ("n_requests", 0, I), ("n_tokens", -1, I), ("n_tokens", 1 << 31, G), ("max_new", -1, I), ("n_q_heads", 0, I),
    ("n_q_heads", 30, U), ("n_q_heads", 8 * 129, U), ("max_new", 1 << 30, G), ("q", None, I), ("o", None, I),
    ("q", FAKE + 8, U), ("o", FAKE + 8, U), ("q_stride", 4088, I), ("o_stride", 4088, I), ("q_stride", 4100, U),
    ("o_stride", 4100, U), ("cu_new", None, I), ("seq_len", None, I), ("block_table", None, I), ("max_pages", 0, I),
    ("table_stride", 9, I), ("lse_stride", 99, I), ("softmax_scale", 0.0, I), ("softmax_scale", float("nan"), I),
    ("softmax_scale", float("inf"), I), ("softmax_scale", -1.0, I)])
def test_attention_arguments(lib, field, value, code):
    a = _with(_attn(), **{field: value})
    assert lib.avtp_cache_attention(ctypes.byref(_cache()), ctypes.byref(a), FAKE, BIG, None) == code


def test_attention_refuses_more_rows_than_its_line_of_work_counts(lib):
    """2^27 blocks of rows over all KV heads, from the requests or from the new tokens."""
    size = ctypes.c_size_t()
    for fields, code in (({"n_requests": 1 << 27}, G), ({"n_requests": 1 << 24}, G),
                         ({"n_requests": (1 << 24) - 1}, avtp.OK),
                         ({"n_tokens": (1 << 31) - 1, "lse_stride": 1 << 31, "n_q_heads": 8 * 128, "q_stride": 1 << 17,
                           "o_stride": 1 << 17}, G)):
        a = _with(_attn(), **fields)
        assert lib.avtp_cache_attention_workspace_size(ctypes.byref(_cache()), ctypes.byref(a), ctypes.byref(size)) == code
        if code != avtp.OK:
            assert lib.avtp_cache_attention(ctypes.byref(_cache()), ctypes.byref(a), FAKE, BIG, None) == code


@pytest.mark.parametrize("page", [1, 8, 24, 40])
def test_attention_wants_pages_of_whole_sixteens(lib, page):
    assert lib.avtp_cache_attention(ctypes.byref(_cache(page=page)), ctypes.byref(_attn()), FAKE, BIG, None) == U


def test_structs_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("needs a host C compiler")
    structs = {"avtp_cache_t": avtp._Cache, "avtp_cache_slots_args_t": avtp._CacheSlotsArgs,
               "avtp_cache_write_args_t": avtp._CacheWriteArgs, "avtp_cache_attn_args_t": avtp._CacheAttnArgs}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "avtp.h"', "int main(void) {"]
    for c_name, py in structs.items():
        lines.append(f'  printf("%zu\\n", sizeof({c_name}));')
        lines += [f'  printf("%zu\\n", offsetof({c_name}, {f}));' for f, _ in py._fields_]
    src = tmp_path / "abi.c"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "abi")],
                   check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "abi")], capture_output=True, text=True,
                                          check=True).stdout.split()]
    want = []
    for py in structs.values():
        want += [ctypes.sizeof(py)] + [getattr(py, f).offset for f, _ in py._fields_]
    assert got == want


def test_the_binding_refuses_tensors_off_the_gpu():
    t = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        avtp.PagedCache(torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16), torch.zeros(2, 16, 1, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        avtp.PagedCache(torch.zeros(2, 16, 1, 64), torch.zeros(2, 16, 1, 64))
    with pytest.raises(ValueError):
        avtp.cache_slots(t, 4, page_size=16, n_pages=4, block_table=torch.zeros(2, 4, dtype=torch.int32), free_pages=t)
    with pytest.raises(ValueError):
        avtp.cache_slots(t.long(), 4, page_size=16, n_pages=4, block_table=torch.zeros(2, 4, dtype=torch.int32),
                         free_pages=t)
    with pytest.raises(ValueError):
        avtp.cache_slots(t, 4, page_size=16, n_pages=4, block_table=torch.zeros(3, 4, dtype=torch.int32), free_pages=t)


def test_the_plain_slots_follow_their_formula():
    """slots_plain (a token at a time) against the closed form of the operator."""
    rng = np.random.default_rng(2)
    for page in (1, 7, 16):
        past, new = rng.integers(0, 50, 6), rng.integers(0, 40, 6)
        cu = np.concatenate([[0], np.cumsum(new)])
        have, need = -(-past // page), -(-(past + new) // page)
        table = np.full((6, int(need.max())), -1)
        for r in range(6):
            table[r, :have[r]] = 1000 * r + np.arange(have[r])
        free = 100000 + np.arange(int((need - have).sum()))
        got, slots, seq, head = slots_plain(cu, past, table, free, 0, page, int(cu[-1]) + 3)
        assert head == len(free) and np.array_equal(seq, past + new) and np.all(slots[cu[-1]:] == -1)
        first = np.cumsum(need - have) - (need - have)
        for r in range(6):
            assert np.array_equal(got[r, have[r]:need[r]], free[first[r]:first[r] + need[r] - have[r]])
            p = past[r] + np.arange(new[r])
            assert np.array_equal(slots[cu[r]:cu[r + 1]], got[r, p // page] * page + p % page)
