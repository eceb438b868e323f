"""Rotary positions' host side, without a GPU: argument checks of avtp_rope (every refusal returns before the
first CUDA call), the binding's structs and its refusals, and the frequencies."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp
from tests.gpu_util import ensure_built

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


def _rope(T=100, hq=32, hkv=8, d=128, rot=128):
    return avtp._RopeArgs(T, hq, hkv, d, FAKE, hq * d, FAKE, hq * d, FAKE, hkv * d, FAKE, hkv * d, FAKE, hkv * d, FAKE, rot,
                          avtp.ROPE_HALF, FAKE, FAKE, T, 3, FAKE, 1.0, FAKE, FAKE, 1e-6)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("field,value,code", [
    ("n_tokens", -1, I), ("n_tokens", 1 << 31, G), ("n_q_heads", -1, I), ("n_kv_heads", -1, I), ("n_q_heads", 1 << 17, G),
    ("n_kv_heads", 1 << 17, G), ("n_kv_heads", 4, I), ("head_dim", 96, U), ("head_dim", 64, I), ("q", None, I),
    ("q", FAKE + 8, U), ("q_stride", 4088, I), ("q_stride", 4100, U), ("q_out", None, I), ("q_out", FAKE + 2, U),
    ("q_out_stride", 4088, I), ("k", None, I), ("k", FAKE + 8, U), ("k_stride", 1020, I), ("k_out", FAKE + 8, U),
    ("k_out_stride", 1028, U), ("v", None, I), ("v", FAKE + 8, U), ("v_stride", 1028, U), ("slot_map", None, I),
    ("rot_dim", -8, I), ("rot_dim", 136, I), ("rot_dim", 20, U), ("style", 2, I), ("style", -1, I), ("inv_freq", None, I),
    ("pos", None, I), ("pos_stride", 99, I), ("n_planes", 0, I), ("attn_factor", NAN, I), ("attn_factor", INF, I),
    ("eps", -1.0, I), ("eps", NAN, I), ("q_norm", FAKE + 8, U), ("k_norm", FAKE + 2, U)])
def test_rope_arguments(lib, field, value, code):
    a = _rope()
    setattr(a, field, value)
    assert lib.avtp_rope(ctypes.byref(a), ctypes.byref(_cache()), FAKE, BIG, None) == code


def test_rope_without_a_cache_wants_rows_for_the_keys(lib):
    a = _rope()
    a.k_out = None
    assert lib.avtp_rope(ctypes.byref(a), None, FAKE, BIG, None) == I
    assert lib.avtp_rope(None, None, FAKE, BIG, None) == I
    bad = _cache()
    bad.v = None
    assert lib.avtp_rope(ctypes.byref(_rope()), ctypes.byref(bad), FAKE, BIG, None) == I
    for ws, size in ((None, BIG), (FAKE + 16, BIG), (FAKE, 8)):
        assert lib.avtp_rope(ctypes.byref(_rope()), ctypes.byref(_cache()), ws, size, None) == W


def test_structs_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("needs a host C compiler")
    structs = {"avtp_rope_args_t": avtp._RopeArgs, "avtp_rope_freq_args_t": avtp._RopeFreqArgs}
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


# ---------------------------------------------------------------- frequencies
# pow and the few operations around it in 64 bits, then one rounding to fp32: half a step, 2^-24 relative
@pytest.mark.parametrize("rot,base", [(2, 1e4), (24, 1e4), (64, 5e5), (128, 5e6)])
def test_frequencies(lib, rot, base):
    th = base ** (-np.arange(0, rot, 2) / rot)
    tol = 2.0 ** -24 * (1 + 1e-6)

    def close(got, want):
        assert np.all(np.abs(got[0] - want) <= tol * want)

    plain = avtp.rope_frequencies(rot, base)
    close(plain, th)
    assert plain[1] == 1.0 and plain[0].dtype == np.float32
    close(avtp.rope_frequencies(rot, base, "linear", factor=8), th / 8)
    if rot >= 4:
        ntk = avtp.rope_frequencies(rot, base, "ntk", factor=8)
        close(ntk, (base * 8.0 ** (rot / (rot - 2))) ** (-np.arange(0, rot, 2) / rot))
        assert ntk[0][0] == 1.0 and abs(ntk[0][-1] * 8 / th[-1] - 1) < 1e-6  # ends: kept, and as interpolated
    turns = 4096 * th / (2 * math.pi)
    g = np.clip((turns - 1) / 31, 0, 1)
    yarn = avtp.rope_frequencies(rot, base, "yarn", factor=16, original_len=4096)
    close(yarn, (1 - g) * th / 16 + g * th)
    assert abs(yarn[1] - (0.1 * math.log(16) + 1)) <= 2.0 ** -23


@pytest.mark.parametrize("fields", [
    dict(rot_dim=0), dict(rot_dim=7), dict(base=1.0), dict(base=INF), dict(scaling="linear", factor=0.5),
    dict(scaling="ntk", factor=NAN), dict(rot_dim=2, scaling="ntk", factor=2), dict(scaling="yarn", factor=2),
    dict(scaling="yarn", factor=2, original_len=10, slow=3, fast=3),
    dict(scaling="yarn", factor=2, original_len=10, slow=-1, fast=3)])
def test_frequencies_refuse(lib, fields):
    with pytest.raises(avtp.AVTPError):
        avtp.rope_frequencies(**{"rot_dim": 64, **fields})
    with pytest.raises(ValueError):
        avtp.rope_frequencies(64, scaling="other")


def test_the_binding_refuses_tensors_off_the_gpu():
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    pos, inv = torch.zeros(3, dtype=torch.int32), torch.zeros(32)
    with pytest.raises(ValueError):
        avtp.rope(pos, inv, q=q)
    with pytest.raises(ValueError):
        avtp.rope(pos, inv)
    with pytest.raises(ValueError):
        avtp.rope(pos, inv, q=q, slot_map=pos)
