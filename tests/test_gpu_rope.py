"""Rotary positions on the GPU against a plain 64-bit form: styles, parts of a head, planes, norms, the cache as
destination, and the calls that could go wrong."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2608_26806_gb300 import avtp
from tests.cache_util import pool
from tests.gpu_util import ensure_built

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    ensure_built()


def status(call):
    return avtp.read_device_status(call.workspace)


def plain(x, pos, inv_freq, style, plane, factor, norm):
    """64 bits: (values, how far bf16 outputs of 32-bit work may be off).

    Off: the output's rounding, 2^-8 of the value, and of the pair's |y_a| + |y_b| times the factor
    - the norm: a sum of squares of 16 terms a lane and four more steps (10 roundings of the sum count half), rsqrt to
      2 units in the last place, three products: below 2^-20;
    - sine and cosine: half a turn in 24 bits (2^-25 of a half turn, 2^-23.3 rad), two units of sincospif (2^-23), the
      factor's product and the rotation's three (2^-22): below 2^-20 together;
    - the angle: 2^-61 pos (1 + f) for its fraction of a turn, 2^-32 of a turn for the bits that are left, and what
      64 bits leave here, 2^-53 of it: below pos f 2^-52 + 2^-29.
    """
    d = x.shape[-1]
    y = x.double()
    if norm is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS) * norm.double()
    rot = 2 * len(inv_freq)
    p = pos if pos.dim() == 2 else pos[None]
    which = plane if plane is not None else torch.zeros(rot // 2, dtype=torch.int64)
    angle = p.double()[which].t() * inv_freq.double()  # [T, rot / 2]
    cos, sin = (torch.cos(angle) * factor)[:, None], (torch.sin(angle) * factor)[:, None]
    i = torch.arange(rot // 2)
    a, b = (i, i + rot // 2) if style == "half" else (2 * i, 2 * i + 1)
    want, size = y.clone(), y.abs()
    off = torch.zeros_like(y)
    want[..., a], want[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
    both = (y[..., a].abs() + y[..., b].abs()) * abs(factor)
    size[..., a] = size[..., b] = both
    off[..., a] = off[..., b] = both * (angle.abs() * 2.0 ** -52 + 2.0 ** -29)[:, None]
    assert d == x.shape[-1]
    return want, want.abs() * 2.0 ** -8 * (1 + 2.0 ** -7) + off + size * (2.0 ** -19)


def close(got, want_tol):
    want, tol = want_tol
    diff = (got.cpu().double() - want).abs() - tol
    assert torch.isfinite(got).all() and diff.max() <= 0, f"off by {float((got.cpu().double() - want).abs().max())}"


def make(T, Hq, Hkv, d, rot, planes=1, norm=True, seed=0, far=5000, base=1e4):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = dict(q=r(T, Hq, d).mul(3).bfloat16(), k=r(T, Hkv, d).bfloat16(), v=r(T, Hkv, d).bfloat16())
    x["pos"] = torch.randint(0, far, (planes, T) if planes > 1 else (T,), generator=g, dtype=torch.int64).int()
    x["inv"] = torch.from_numpy(avtp.rope_frequencies(rot, base)[0]) if rot else torch.zeros(0)
    x["plane"] = torch.randint(0, planes, (rot // 2,), generator=g).int() if planes > 1 else None
    x["qn"] = (1 + 0.3 * r(d)).bfloat16() if norm else None
    x["kn"] = (1 + 0.3 * r(d)).bfloat16() if norm else None
    return x


def cuda(t):
    return None if t is None else t.cuda()


CASES = {
    # T, Hq, Hkv, d, rot, style, planes, norm, factor
    "one_token": (1, 32, 8, 128, 128, "half", 1, True, 1.0),
    "one_head": (3, 1, 1, 64, 64, "half", 1, True, 1.0),
    "planes": (77, 32, 8, 128, 128, "half", 3, True, 1.0),
    "interleaved": (77, 28, 4, 128, 128, "interleaved", 3, True, 1.2),
    "part": (130, 16, 16, 64, 32, "half", 1, False, 1.0),
    "part_interleaved": (130, 16, 16, 64, 32, "interleaved", 2, False, 1.3),
    "odd_half": (50, 5, 3, 128, 24, "half", 1, True, 1.0),
    "odd_half_small": (50, 9, 1, 64, 40, "half", 2, True, 0.7),
    "eight": (50, 9, 1, 64, 8, "half", 1, True, 1.0),
    "eight_interleaved": (50, 3, 1, 128, 8, "interleaved", 1, False, 1.0),
    "twenty_four": (50, 3, 2, 64, 24, "interleaved", 1, True, 1.0),
    "fifty_six": (20, 6, 2, 64, 56, "half", 4, False, 1.0),
    "one_twenty": (20, 6, 2, 128, 120, "half", 1, True, 1.0),
    "norm_alone": (61, 12, 2, 128, 0, "half", 1, True, 1.0),
    "many": (3001, 28, 4, 128, 128, "half", 3, True, 1.0),
    "many_small": (5003, 4, 2, 64, 64, "interleaved", 1, True, 1.0),
}


@pytest.mark.parametrize("name", CASES)
def test_rows(name):
    T, Hq, Hkv, d, rot, style, planes, norm, factor = CASES[name]
    x = make(T, Hq, Hkv, d, rot, planes, norm, seed=len(name))
    call = avtp.RopeCall(cuda(x["pos"]), cuda(x["inv"]) if rot else None, q=x["q"].cuda(), k=x["k"].cuda(), style=style,
                         pair_plane=cuda(x["plane"]), attn_factor=factor, q_norm=cuda(x["qn"]), k_norm=cuda(x["kn"]),
                         eps=EPS).run()
    assert status(call) == avtp.OK
    plane = None if x["plane"] is None else x["plane"].long()
    close(call.q_out, plain(x["q"], x["pos"], x["inv"], style, plane, factor, x["qn"]))
    close(call.k_out, plain(x["k"], x["pos"], x["inv"], style, plane, factor, x["kn"]))


@pytest.mark.parametrize("order", ["token", "head", "mixed", "padded", "shared"])
@pytest.mark.parametrize("T,page", [(1, 16), (9, 7), (700, 64)])
def test_into_the_cache(order, T, page):
    Hq, Hkv, d = 8, 4, 128
    x = make(T, Hq, Hkv, d, d, 3, True, seed=T)
    n_pages = -(-T // page) + 2
    k, v = pool(n_pages, page, Hkv, d, order)
    cache = avtp.PagedCache(k, v)
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(1))[:T].int()
    if T > 4:
        slots[2] = -1
    rows = torch.full((T, Hkv, d), 9.0, dtype=torch.bfloat16, device="cuda") if T == 9 else None
    call = avtp.RopeCall(x["pos"].cuda(), x["inv"].cuda(), q=x["q"].cuda(), k=x["k"].cuda(), v=x["v"].cuda(), k_out=rows,
                         pair_plane=x["plane"].cuda(), q_norm=x["qn"].cuda(), k_norm=x["kn"].cuda(), cache=cache,
                         slot_map=slots.cuda()).run()
    assert status(call) == avtp.OK
    want, tol = plain(x["k"], x["pos"], x["inv"], "half", x["plane"].long(), 1.0, x["kn"])
    used = slots >= 0
    at = slots[used].long()
    close(k.cpu()[at // page, at % page], (want[used], tol[used]))
    assert torch.equal(v.cpu()[at // page, at % page], x["v"][used])
    untouched = torch.ones(n_pages * page, dtype=torch.bool)
    untouched[at] = False
    for t in (k, v):
        assert torch.isnan(t.cpu().reshape(n_pages * page, Hkv, d)[untouched]).all()
    if rows is not None:
        close(rows, (want, tol))
    else:
        assert call.k_out is None
    close(call.q_out, plain(x["q"], x["pos"], x["inv"], "half", x["plane"].long(), 1.0, x["qn"]))


@pytest.mark.parametrize("style,rot", [("half", 128), ("half", 24), ("interleaved", 64)])
def test_over_the_inputs_of_a_joint_projection(style, rot):
    """q, k and v side by side in one tensor, rotated where they lie; the values and what follows them stay."""
    T, Hq, Hkv, d = 300, 6, 2, 128
    x = make(T, Hq, Hkv, d, rot, seed=4)
    joint = torch.full((T + 2, Hq + 2 * Hkv + 1, d), 7.0, dtype=torch.bfloat16)
    joint[:T, :Hq], joint[:T, Hq:Hq + Hkv], joint[:T, Hq + Hkv:Hq + 2 * Hkv] = x["q"], x["k"], x["v"]
    dev = joint.cuda()
    q, k = dev[:T, :Hq], dev[:T, Hq:Hq + Hkv]
    avtp.rope(x["pos"].cuda(), x["inv"].cuda(), q=q, k=k, q_out=q, k_out=k, style=style, q_norm=x["qn"].cuda(),
              k_norm=x["kn"].cuda())
    close(q, plain(x["q"], x["pos"], x["inv"], style, None, 1.0, x["qn"]))
    close(k, plain(x["k"], x["pos"], x["inv"], style, None, 1.0, x["kn"]))
    rest = dev.cpu()
    assert torch.equal(rest[:, Hq + Hkv:], joint[:, Hq + Hkv:]) and torch.equal(rest[T:], joint[T:])


def test_queries_or_keys_alone():
    x = make(40, 4, 2, 64, 64, seed=6)
    pos, inv = x["pos"].cuda(), x["inv"].cuda()
    q, none = avtp.rope(pos, inv, q=x["q"].cuda())
    assert none is None
    close(q, plain(x["q"], x["pos"], x["inv"], "half", None, 1.0, None))
    none, k = avtp.rope(pos, inv, k=x["k"].cuda(), k_norm=x["kn"].cuda())
    assert none is None
    close(k, plain(x["k"], x["pos"], x["inv"], "half", None, 1.0, x["kn"]))


@pytest.mark.parametrize("first", [(1 << 31) - 40, 1 << 24, -40, -(1 << 31)])
def test_far_and_negative_positions(first):
    x = make(40, 2, 1, 64, 64, norm=False, seed=7)
    pos = (first + torch.arange(40, dtype=torch.int64)).int()
    for style in ("half", "interleaved"):
        q, _ = avtp.rope(pos.cuda(), x["inv"].cuda(), q=x["q"].cuda(), style=style)
        close(q, plain(x["q"], pos, x["inv"], style, None, 1.0, None))


def test_frequencies_of_any_size_and_sign():
    """Negative ones turn the other way, ones above a turn a position wrap, zero leaves its pair."""
    x = make(64, 2, 1, 64, 64, norm=False, seed=8)
    inv = torch.linspace(-9.0, 9.0, 32)
    inv[5] = 0.0
    q, _ = avtp.rope(x["pos"].cuda(), inv.cuda(), q=x["q"].cuda())
    close(q, plain(x["q"], x["pos"], inv, "half", None, 1.0, None))
    assert torch.equal(q[..., [5, 37]].cpu(), x["q"][..., [5, 37]])


@pytest.mark.parametrize("style,rot", [("half", 32), ("half", 24), ("interleaved", 24)])
def test_elements_behind_the_rotated_ones_pass_whatever_they_hold(style, rot):
    x = make(33, 3, 1, 64, rot, norm=False, seed=9)
    q = x["q"].clone()
    q[..., rot:] = torch.tensor([float("inf"), float("nan"), -0.0, -float("inf")], dtype=torch.bfloat16).repeat((64 - rot) // 4)
    got, _ = avtp.rope(x["pos"].cuda(), x["inv"].cuda(), q=q.cuda(), style=style)
    assert torch.equal(got.cpu()[..., rot:].view(torch.int16), q[..., rot:].view(torch.int16))
    clean = x["q"][..., :rot]
    want, tol = plain(clean, x["pos"], x["inv"], style, None, 1.0, None)
    close(got[..., :rot], (want, tol))


def test_a_plain_copy_keeps_every_bit():
    bits = torch.randint(-32768, 32767, (29, 3, 128), generator=torch.Generator().manual_seed(2)).short()
    q = bits.view(torch.bfloat16)
    got, _ = avtp.rope(None, None, q=q.cuda())
    assert torch.equal(got.cpu().view(torch.int16), bits)


def test_large_and_tiny_rows():
    """Rows whose squares leave fp32's range give what the formula does in 32 bits: zeros, and eps alone."""
    x = make(4, 1, 1, 64, 64, seed=3)
    q = x["q"].clone()
    q[0] = 1e30   # the sum overflows: x * 0
    q[1] = 1e-30  # the sum underflows: x / sqrt(eps)
    q[2] = 0.0
    got, _ = avtp.rope(torch.zeros(4, dtype=torch.int32).cuda(), x["inv"].cuda(), q=q.cuda(), q_norm=x["qn"].cuda(), eps=EPS)
    got = got.cpu().double()
    assert torch.equal(got[0], torch.zeros(1, 64).double()) and torch.equal(got[2], torch.zeros(1, 64).double())
    want = 1e-30 / EPS ** 0.5 * x["qn"].double()
    assert ((got[1] - want).abs() <= want.abs() * 2.0 ** -7).all()


# ---------------------------------------------------------------- refusals by the device
def test_bad_slots_are_skipped_and_recorded():
    T, page, Hkv, d = 20, 16, 2, 64
    x = make(T, 4, Hkv, d, d, seed=5)
    k, v = pool(3, page, Hkv, d)
    slots = torch.arange(T).int()
    slots[3], slots[7], slots[9] = 3 * page, -2, -1
    call = avtp.RopeCall(x["pos"].cuda(), x["inv"].cuda(), q=x["q"].cuda(), k=x["k"].cuda(), v=x["v"].cuda(),
                         cache=avtp.PagedCache(k, v), slot_map=slots.cuda()).run()
    assert status(call) == avtp.ERR_DEVICE_INPUT
    good = [t for t in range(T) if t not in (3, 7, 9)]
    want, tol = plain(x["k"], x["pos"], x["inv"], "half", None, 1.0, None)
    got = k.cpu().reshape(3 * page, Hkv, d)
    close(got[good], (want[good], tol[good]))
    assert torch.isnan(got[[3, 7, 9]]).all() and torch.isnan(got[T:]).all()
    close(call.q_out, plain(x["q"], x["pos"], x["inv"], "half", None, 1.0, None))


@pytest.mark.parametrize("what", ["nan", "inf", "plane", "minus"])
def test_bad_tables_write_nothing(what):
    T, page, Hkv, d = 300, 16, 2, 64
    x = make(T, 4, Hkv, d, d, planes=2, seed=5)
    inv, plane = x["inv"].clone(), x["plane"].clone()
    if what in ("nan", "inf"):
        inv[31] = float(what)
    else:
        plane[17] = 2 if what == "plane" else -1
    k, v = pool(20, page, Hkv, d)
    q_out = torch.full((T, 4, d), 5.0, dtype=torch.bfloat16, device="cuda")
    call = avtp.RopeCall(x["pos"].cuda(), inv.cuda(), q=x["q"].cuda(), k=x["k"].cuda(), v=x["v"].cuda(), q_out=q_out,
                         pair_plane=plane.cuda(), cache=avtp.PagedCache(k, v), slot_map=torch.arange(T).int().cuda()).run()
    assert status(call) == avtp.ERR_DEVICE_INPUT
    assert (q_out == 5.0).all() and torch.isnan(k).all() and torch.isnan(v).all()


@pytest.mark.parametrize("T", [4096, 4097, 9000])
def test_what_many_tokens_have_wrong_is_recorded(T):
    """By one CTA up to 4096 tokens, by those that rotate beyond."""
    page, Hkv, d = 16, 1, 64
    x = make(T, 2, Hkv, d, d, planes=2, seed=T)
    dev = {n: x[n].cuda() for n in ("pos", "inv", "q", "k", "v", "plane")}
    n_pages = T // page + 2
    slots = torch.arange(T).int()

    def call(slots, **tables):
        k, v = pool(n_pages, page, Hkv, d)
        t = {**dev, **tables}
        c = avtp.RopeCall(t["pos"], t["inv"], q=t["q"], k=t["k"], v=t["v"], pair_plane=t["plane"],
                          cache=avtp.PagedCache(k, v), slot_map=slots.cuda(),
                          q_out=torch.full((T, 2, d), 5.0, dtype=torch.bfloat16, device="cuda"))
        return c.run(), k, v

    c, k, v = call(slots)
    assert status(c) == avtp.OK
    want, tol = plain(x["k"], x["pos"], x["inv"], "half", x["plane"].long(), 1.0, None)
    close(k.reshape(-1, Hkv, d)[:T], (want, tol))
    bad = slots.clone()
    bad[T - 1], bad[7] = n_pages * page, -2
    c, k, v = call(bad)
    assert status(c) == avtp.ERR_DEVICE_INPUT
    good = torch.ones(n_pages * page, dtype=torch.bool)
    good[[7, T - 1]] = False
    good[T:] = False
    at = torch.nonzero(good)[:, 0]
    close(k.cpu().reshape(-1, Hkv, d)[at], (want[at], tol[at]))
    assert torch.isnan(k.cpu().reshape(-1, Hkv, d)[~good]).all() and torch.isnan(v.cpu().reshape(-1, Hkv, d)[~good]).all()
    inv = x["inv"].clone()
    inv[30] = float("nan")
    c, k, v = call(slots, inv=inv.cuda())
    assert status(c) == avtp.ERR_DEVICE_INPUT
    assert (c.q_out == 5.0).all() and torch.isnan(k).all() and torch.isnan(v).all()


# ---------------------------------------------------------------- how programs call it
def test_no_tokens():
    e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    call = avtp.RopeCall(torch.empty(0, dtype=torch.int32, device="cuda"), torch.ones(32, device="cuda"), q=e(0, 4, 64),
                         k=e(0, 2, 64)).run()
    assert status(call) == avtp.OK and call.q_out.shape == (0, 4, 64)


def test_no_tokens_and_no_tables():
    """A call without tokens reads nothing, the frequencies among it."""
    ws = avtp.new_workspace(256)
    a = avtp._RopeArgs(0, 4, 2, 64, None, 256, None, 256, None, 128, None, 128, None, 128, None, 64, avtp.ROPE_HALF, None,
                       None, 0, 1, None, 1.0, None, None, 1e-6)
    assert avtp.load().avtp_rope(ctypes.byref(a), None, ws.data_ptr(), 256, None) == avtp.OK
    assert avtp.read_device_status(ws) == avtp.OK


def test_no_heads():
    a = avtp._RopeArgs(5, 0, 0, 64, None, 0, None, 0, None, 0, None, 0, None, 0, None, 0, avtp.ROPE_HALF, None, None, 0, 1,
                       None, 1.0, None, None, 1e-6)
    ws = avtp.new_workspace(256)
    assert avtp.load().avtp_rope(ctypes.byref(a), None, ws.data_ptr(), 256, None) == avtp.OK
    assert avtp.read_device_status(ws) == avtp.OK


def test_a_captured_call_replays_on_new_positions():
    x = make(64, 8, 2, 128, 128, 3, seed=12)
    pos, q = x["pos"].cuda(), x["q"].cuda()
    call = avtp.RopeCall(pos, x["inv"].cuda(), q=q, pair_plane=x["plane"].cuda(), q_norm=x["qn"].cuda(), eps=EPS)
    call.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    new = make(64, 8, 2, 128, 128, 3, seed=13)
    pos.copy_(new["pos"])
    q.copy_(new["q"])
    graph.replay()
    torch.cuda.synchronize()
    close(call.q_out, plain(new["q"], new["pos"], x["inv"], "half", x["plane"].long(), 1.0, x["qn"]))


def test_on_another_stream():
    x = make(512, 8, 2, 128, 128, seed=14)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    dev = [x[n].cuda() for n in ("pos", "inv", "q")]
    torch.cuda.synchronize()
    q, _ = avtp.rope(dev[0], dev[1], q=dev[2], stream=s)
    s.synchronize()
    close(q, plain(x["q"], x["pos"], x["inv"], "half", None, 1.0, None))


def test_results_do_not_change_from_run_to_run():
    x = make(2000, 28, 4, 128, 128, 3, seed=15)
    call = avtp.RopeCall(x["pos"].cuda(), x["inv"].cuda(), q=x["q"].cuda(), k=x["k"].cuda(), pair_plane=x["plane"].cuda(),
                         q_norm=x["qn"].cuda(), k_norm=x["kn"].cuda())
    first = [t.clone() for t in (call.run().q_out, call.k_out)]
    for _ in range(3):
        call.run()
        assert torch.equal(first[0], call.q_out) and torch.equal(first[1], call.k_out)


def test_the_binding_refuses():
    x = make(10, 4, 2, 64, 64)
    pos, inv, q, k = (x[n].cuda() for n in ("pos", "inv", "q", "k"))
    for kw in (dict(q=q.float()), dict(q=q, k=k[:5]), dict(q=q, pair_plane=pos), dict(q=q, q_norm=inv),
               dict(q=q, q_out=k), dict(q=q[..., ::2]), dict(q=q.transpose(0, 1)), dict(q=q, k_out=k)):
        with pytest.raises(ValueError):
            avtp.rope(pos, inv, **kw)
    for p, i in ((pos.long(), inv), (pos[:5], inv), (pos, inv.double()), (None, inv), (pos, inv[::2])):
        with pytest.raises(ValueError):
            avtp.rope(p, i, q=q)
    with pytest.raises(KeyError):
        avtp.rope(pos, inv, q=q, style="other")
    with pytest.raises(avtp.AVTPError):
        avtp.rope(pos, torch.ones(33, device="cuda"), q=q)  # more than the head


def test_it_shares_the_frequencies_of_rope_frequencies():
    inv, factor = avtp.rope_frequencies(64, 1e4, "yarn", factor=4, original_len=2048)
    x = make(16, 2, 1, 64, 64, norm=False, far=8192, seed=1)
    q, _ = avtp.rope(x["pos"].cuda(), torch.from_numpy(inv).cuda(), q=x["q"].cuda(), attn_factor=factor)
    close(q, plain(x["q"], x["pos"], torch.from_numpy(inv), "half", None, float(np.float32(factor)), None))
