"""The upkeep of the cache's pages without a GPU: argument checks of the C entry points, the binding's structs and
refusals, and the plain forms that the GPU tests compare with."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp
from tests.gpu_util import ensure_built
from tests.pages_util import compact_plain, fork_plain, free_plain, holds

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7f0000000000  # a 256-aligned address that is never dereferenced on these paths
BIG = 1 << 34
I, U, G, W = avtp.ERR_INVALID_ARG, avtp.ERR_UNSUPPORTED, avtp.ERR_RANGE, avtp.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return ensure_built()


def _cache(h=8, d=128, page=64):
    s = (page * h * d, h * d, d)
    return avtp._Cache(FAKE, FAKE, 100, page, h, d, *s, *s)


def _compact():
    return avtp._CacheCompactArgs(4, 100, FAKE, FAKE, FAKE, FAKE, FAKE, 10, 10, FAKE, 10, 10, FAKE, 64, 4, FAKE, FAKE + 256)


def _fork():
    return avtp._CacheForkArgs(8, 4, 64, 100, 10, 10, FAKE, FAKE, FAKE, FAKE, 50, FAKE, FAKE, FAKE, FAKE, 64, 4, FAKE, FAKE,
                               FAKE, FAKE)


def _free():
    return avtp._CacheFreeArgs(8, 64, 100, 10, 10, FAKE, FAKE, FAKE, FAKE, 50, FAKE, FAKE, 64, 4, FAKE, FAKE, FAKE, FAKE)


def _with(struct, field, value):
    setattr(struct, field, value)
    return struct


@pytest.mark.parametrize("field,value,code", [
    ("n_requests", 0, I), ("n_requests", (1 << 31) - 1024, G), ("n_kept", -1, I), ("n_kept", 1 << 31, G),
    ("keep_cu", None, I), ("keep_idx", None, I), ("seq_len", None, I), ("block_table", None, I), ("max_pages", 0, I),
    ("table_stride", 9, I), ("dst_max_pages", 0, I), ("dst_stride", 9, I), ("window", -1, I), ("n_sinks", -1, I),
    ("held_len", None, I), ("len_out", FAKE, I)])
def test_compact_arguments(lib, field, value, code):
    a = _with(_compact(), field, value)
    assert lib.avtp_cache_compact(ctypes.byref(_cache()), ctypes.byref(a), FAKE, BIG, None) == code


@pytest.mark.parametrize("field,value,code", [
    ("n_requests", 0, I), ("n_requests", (1 << 31) - 1, G), ("n_children", -1, I), ("n_children", (1 << 31) - 1, G),
    ("page_size", 0, I), ("n_pages", 0, I), ("n_pages", 1 << 26, G), ("max_pages", 0, I), ("table_stride", 9, I),
    ("parent", None, I), ("child", None, I), ("free_pages", None, I), ("n_free", -1, I), ("n_free", 1 << 31, G),
    ("block_table", None, I), ("seq_len", None, I), ("shared", None, I), ("window", -1, I), ("n_sinks", -1, I),
    ("held_len", None, I), ("copy_src", None, I), ("copy_dst", None, I)])
def test_fork_arguments(lib, field, value, code):
    a = _with(_fork(), field, value)
    assert lib.avtp_cache_fork(ctypes.byref(a), FAKE, BIG, None) == code
    size = ctypes.c_size_t()
    assert lib.avtp_cache_fork_workspace_size(ctypes.byref(a), ctypes.byref(size)) == code


@pytest.mark.parametrize("field,value,code", [
    ("n_requests", 0, I), ("n_requests", (1 << 31) - 1, G), ("page_size", 0, I), ("n_pages", 0, I), ("n_pages", 1 << 26, G),
    ("max_pages", 0, I), ("table_stride", 9, I), ("seq_len", None, I), ("new_len", None, I), ("block_table", None, I),
    ("free_pages", None, I), ("n_free", -1, I), ("n_free", 1 << 31, G), ("free_head", None, I), ("window", -1, I),
    ("n_sinks", -1, I), ("held_len", None, I), ("seq_len_out", None, I), ("held_len_out", None, I),
    ("free_head_out", None, I)])
def test_free_arguments(lib, field, value, code):
    a = _with(_free(), field, value)
    assert lib.avtp_cache_free(ctypes.byref(a), FAKE, BIG, None) == code
    size = ctypes.c_size_t()
    assert lib.avtp_cache_free_workspace_size(ctypes.byref(a), ctypes.byref(size)) == code


def test_copy_arguments_and_workspaces(lib):
    c, size = _cache(), ctypes.c_size_t()
    for src, dst, n, code in ((None, FAKE, 3, I), (FAKE, None, 3, I), (FAKE, FAKE, -1, I), (FAKE, FAKE, 1 << 31, G)):
        assert lib.avtp_cache_copy(ctypes.byref(c), src, dst, n, FAKE, BIG, None) == code
    bad = _with(_cache(), "k_page_stride", 8)
    assert lib.avtp_cache_copy(ctypes.byref(bad), FAKE, FAKE, 3, FAKE, BIG, None) == I
    assert lib.avtp_cache_compact(ctypes.byref(bad), ctypes.byref(_compact()), FAKE, BIG, None) == I
    assert lib.avtp_cache_compact(ctypes.byref(c), None, FAKE, BIG, None) == I
    assert lib.avtp_cache_fork(None, FAKE, BIG, None) == I and lib.avtp_cache_free(None, FAKE, BIG, None) == I
    for ws, n in ((None, BIG), (FAKE + 16, BIG), (FAKE, 8)):
        assert lib.avtp_cache_copy(ctypes.byref(c), FAKE, FAKE, 3, ws, n, None) == W
        assert lib.avtp_cache_compact(ctypes.byref(c), ctypes.byref(_compact()), ws, n, None) == W
    f, g = _fork(), _free()
    assert lib.avtp_cache_fork_workspace_size(ctypes.byref(f), None) == I
    assert lib.avtp_cache_fork_workspace_size(ctypes.byref(f), ctypes.byref(size)) == avtp.OK
    assert lib.avtp_cache_fork(ctypes.byref(f), FAKE, size.value - 1, None) == W
    assert lib.avtp_cache_free_workspace_size(ctypes.byref(g), None) == I
    assert lib.avtp_cache_free_workspace_size(ctypes.byref(g), ctypes.byref(size)) == avtp.OK
    assert lib.avtp_cache_free(ctypes.byref(g), FAKE, size.value - 1, None) == W
    with_counts = size.value
    assert lib.avtp_cache_free_workspace_size(ctypes.byref(_with(_free(), "shared", None)), ctypes.byref(size)) == avtp.OK
    assert size.value < with_counts


def test_structs_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("needs a host C compiler")
    structs = {"avtp_cache_compact_args_t": avtp._CacheCompactArgs, "avtp_cache_fork_args_t": avtp._CacheForkArgs,
               "avtp_cache_free_args_t": avtp._CacheFreeArgs}
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
    t, table = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int32)
    one = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        avtp.cache_free(t, t, table, page_size=16, n_pages=4, free_pages=t, free_head=one)
    with pytest.raises(ValueError):
        avtp.cache_fork(one, one, t, table, page_size=16, n_pages=4, free_pages=t, shared=torch.zeros(4, dtype=torch.int32))


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 5), (9, 0)])
@pytest.mark.parametrize("page", [1, 7, 16])
def test_the_plain_forms_keep_every_page_accounted_for(page, window, sinks):
    """A random run of new tokens, forks, cuts and ends: a page's holders are the rows that hold it, and pages without
    holders, and no others, are in the free list."""
    rng = np.random.default_rng(page + window)
    R, columns, n_pages = 6, -(-260 // page) + 1, 6 * (-(-260 // page) + 1)
    table, seq, held = np.full((R, columns), -1, np.int64), np.zeros(R, np.int64), np.zeros(R, np.int64)
    free, head, shared = rng.permutation(n_pages), 0, np.zeros(n_pages, np.int64)
    for step in range(60):
        for r in range(R):  # new tokens
            n = int(rng.integers(0, 30))
            if seq[r] + n > 250:
                continue
            for j in range(-(-int(seq[r]) // page), -(-(int(seq[r]) + n) // page)):
                table[r, j], head = free[head], head + 1
            seq[r] += n
        parents = [r for r in range(R) if seq[r] > 0]
        empty = [r for r in range(R) if seq[r] == 0]
        if parents and empty:
            p = [int(rng.choice(parents)) for _ in empty]
            table, seq, head, shared, _, _, held = fork_plain(p, empty, seq, table, free, head, page, shared, None, window,
                                                              sinks, held)
        new = np.where(rng.random(R) < 0.2, 0, seq)
        free, head, shared = free_plain(seq, new, table, free, head, page, shared, window, sinks, held)
        seq, held = new, new.copy()
        holders = np.zeros(n_pages, np.int64)
        for r in range(R):
            for j in range(-(-int(seq[r]) // page)):
                if holds(j, seq[r], held[r], page, window, sinks):
                    holders[table[r, j]] += 1
        assert np.array_equal(np.maximum(holders - 1, 0), shared)
        assert sorted(free[head:]) == sorted(np.flatnonzero(holders == 0))


def test_compaction_in_place_reads_every_row_before_it_is_written_over():
    rng = np.random.default_rng(3)
    page, n = 8, 50
    table = rng.permutation(7)[None]
    pool = rng.random((7, page, 2))
    keep = np.flatnonzero(rng.random(n) < 0.5)
    want = [pool[table[0, p // page], p % page] for p in keep]
    got = compact_plain(pool, [0, len(keep)], keep, table, table, page)
    for j, row in enumerate(want):
        assert np.array_equal(got[table[0, j // page], j % page], row)
