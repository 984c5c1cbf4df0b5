"""Argument checks of positioning and of contexts in 4 bits, and their header (CPU: refused before any GPU call)."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_2502_01960_amd as mpic

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20          # addresses that nothing is read from
INVALID, UNSUPPORTED = -1, -2


@pytest.fixture(params=["bf16", "f32"])
def ctx(request):
    return mpic.Context(8, 2, 128, mpic.MPIC_BF16 if request.param == "bf16" else mpic.MPIC_F32, 1e4)


def _lib():
    return mpic.load_library()


def test_header_is_plain_c_and_every_entry_point_is_exported(tmp_path):
    header = os.path.join(ROOT, "include", "mpic_q4.h")
    r = subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Wextra", "-Werror", "-fsyntax-only", "-x", "c", header],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    names = set(re.findall(r"^int (mpic_\w+)\(", open(header).read(), re.M))
    assert names == {"mpic_position_rows", "mpic_q4_bytes", "mpic_q4_write", "mpic_q4_read", "mpic_q4_attn_workspace", "mpic_q4_attn"}
    lib = C.CDLL(mpic.lib_path())
    for n in names:
        assert hasattr(lib, n) and hasattr(mpic, n)


def _position(ctx, **kw):
    a = dict(q=A, q_stride=1024, k=A, k_stride=256, n=4, pos=A, n_axes=1, axis=None, wq=None, wk=None, eps=1e-6, qo=2 * A,
             qo_stride=1024, ko=2 * A, ko_stride=256)
    a.update(kw)
    return _lib().mpic_position_rows(ctx.handle, *a.values(), None)


def test_position_rows_refuses(ctx):
    bad = (C.c_int32 * 64)(*([0] * 63 + [1]))
    for kw in (dict(n=-1), dict(n=2 ** 31), dict(n_axes=0), dict(n_axes=5), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(eps=-1.0, wq=A), dict(eps=-1.0, wk=A), dict(axis=bad), dict(q_stride=1023), dict(q_stride=1025), dict(k_stride=0),
               dict(qo_stride=1016), dict(ko_stride=-256), dict(q=None), dict(k=None), dict(pos=None), dict(qo=None), dict(ko=None),
               dict(q=A + 8), dict(ko=A + 2), dict(wq=A + 4), dict(qo=A, qo_stride=2048), dict(ko=A, ko_stride=512)):
        assert _position(ctx, **kw) == INVALID, kw
    assert "position_rows" in mpic.binding.mpic_last_error(ctx.handle)
    assert _lib().mpic_position_rows(*([None, A, 1024, A, 256, 4, A, 1, None, None, None, 0.0, A, 1024, A, 256, None])) == INVALID
    assert _position(ctx, n=0, q=None, k=None, pos=None, qo=None, ko=None) == 0
    assert _position(ctx, n=2 ** 31 - 2) == UNSUPPORTED


def _write(ctx, read=False, **kw):
    a = dict(k=A, k_stride=256, v=A, v_stride=256, n=4, slots=A, cache=A, size=1 << 40, n_slots=64)
    a.update(kw)
    if read:
        return _lib().mpic_q4_read(ctx.handle, a["cache"], a["size"], a["n_slots"], a["slots"], a["n"], a["k"], a["k_stride"], a["v"], a["v_stride"], None)
    return _lib().mpic_q4_write(ctx.handle, *a.values(), None)


@pytest.mark.parametrize("read", [False, True])
def test_rows_refuse(ctx, read):
    for kw in (dict(n=-1), dict(n=2 ** 31), dict(n_slots=-1), dict(n_slots=2 ** 31), dict(k_stride=255), dict(k_stride=257),
               dict(v_stride=128), dict(slots=None, n=65), dict(k=None), dict(v=None), dict(cache=None), dict(k=A + 8), dict(v=A + 2),
               dict(cache=A + 4), dict(size=64 * 2 * 144 - 1), dict(size=0)):
        assert _write(ctx, read, **kw) == INVALID, kw
    assert ("q4_read" if read else "q4_write") in mpic.binding.mpic_last_error(ctx.handle)
    assert _write(ctx, read, n=0, k=None, v=None) == 0
    assert _write(ctx, read, n_slots=0, cache=None, size=0) == 0          # no row has a slot
    assert _write(ctx, read, n=2 ** 31 - 2, n_slots=2 ** 31 - 2) == UNSUPPORTED


def test_bytes():
    for d, dt, per in ((128, mpic.MPIC_BF16, 144), (128, mpic.MPIC_F32, 160), (64, mpic.MPIC_F32, 80)):
        ctx = mpic.Context(6, 3, d, dt, 1e4)
        for n in (0, 1, 16, 17, 2 ** 31 - 2):
            assert mpic.mpic_q4_bytes(ctx.handle, n) == -(-n // 16) * 16 * 3 * per
        for n in (-1, 2 ** 31 - 1):
            with pytest.raises(mpic.MpicError):
                mpic.mpic_q4_bytes(ctx.handle, n)
    assert _lib().mpic_q4_bytes(None, 1, C.byref(C.c_int64())) == INVALID


def _attn(ctx, **kw):
    a = dict(q=A, q_stride=1024, n_rows=3, q_off=None, max_q=1, cache=A, size=1 << 40, n_slots=64, table=A, width=4, page=16, lens=A, n_requests=3,
             max_len=64, scale=0.1, out=A, lse=None, ws=None, ws_bytes=0)
    a.update(kw)
    return _lib().mpic_q4_attn(ctx.handle, *a.values(), None)


def test_attention_refuses(ctx):
    for kw in (dict(n_rows=-1), dict(n_rows=4), dict(max_q=0), dict(max_q=2), dict(n_requests=-1), dict(max_len=-1), dict(max_len=65),
               dict(max_len=2 ** 31), dict(page=0), dict(page=8), dict(page=24), dict(page=-16), dict(width=-1), dict(width=2 ** 40),
               dict(n_slots=-1), dict(n_slots=2 ** 31), dict(n_slots=0), dict(size=64 * 2 * 144 - 1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(q_stride=1023), dict(q_stride=1025), dict(q=None), dict(cache=None), dict(table=None),
               dict(lens=None), dict(out=None), dict(q=A + 8), dict(cache=A + 8), dict(out=A + 2), dict(ws=A + 4),
               dict(max_len=1 << 20, width=1 << 16), dict(max_len=1 << 20, width=1 << 16, ws=A, ws_bytes=100),
               dict(q_off=A, max_q=2 ** 31 - 1)):
        assert _attn(ctx, **kw) == INVALID, kw
    assert "q4_attn" in mpic.binding.mpic_last_error(ctx.handle)
    assert _attn(ctx, n_rows=0, n_requests=0) == 0
    assert _attn(ctx, n_rows=0, q_off=A, q=None, out=None) == 0
    assert _attn(ctx, q_off=A, max_q=1 << 21) == UNSUPPORTED
    assert _attn(ctx, n_rows=70000, n_requests=70000) == UNSUPPORTED


def test_workspace(ctx):
    need = lambda *a: mpic.mpic_q4_attn_workspace(ctx.handle, *a)
    assert need(0, 0, 1, 1 << 20) == 0 and need(1, 1, 1, 0) == 0 and need(1, 1, 1, 100) == 0
    assert need(1, 1, 1, 1 << 20) > 0 and need(1, 1, 1, 1 << 20) % 4 == 0
    assert need(1, 0, 1, 1 << 20) == 0
    wide = mpic.Context(1 << 10, 1, 128, mpic.MPIC_BF16, 1e4)
    with pytest.raises(mpic.MpicError):
        mpic.mpic_q4_attn_workspace(wide.handle, 1, 2 ** 31 - 2, 1, 1 << 20)
    assert mpic.mpic_q4_attn_workspace(wide.handle, 1, 1 << 20, 1, 1 << 30) > 1 << 40
    for a, status in (((-1, 1, 1, 1), INVALID), ((1, -1, 1, 1), INVALID), ((1, 1, 0, 1), INVALID), ((1, 1, 1, -1), INVALID),
                      ((1, 1, 1, 2 ** 31), INVALID), ((65536, 65536, 1, 100), UNSUPPORTED), ((1, 1, 1 << 24, 100), UNSUPPORTED)):
        with pytest.raises(mpic.MpicError) as e:
            need(*a)
        assert e.value.status == status


def test_binding_refuses_tensors_that_do_not_fit():
    ctx = mpic.Context(4, 2, 128, mpic.MPIC_BF16, 1e4)
    t = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    cache = torch.zeros(mpic.mpic_q4_bytes(ctx.handle, 32), dtype=torch.uint8)
    with pytest.raises(mpic.MpicError):
        mpic.mpic_q4_write(ctx.handle, t(3, 2, 128), t(3, 2, 128), i(3), cache, 33, 0)
    for call in (lambda: mpic.mpic_q4_write(ctx.handle, t(3, 2, 128), t(2, 2, 128), i(3), cache, 32),
                 lambda: mpic.mpic_q4_write(ctx.handle, t(3, 2, 128), t(3, 2, 128), i(2), cache, 32),
                 lambda: mpic.mpic_q4_write(ctx.handle, t(3, 128, 2).transpose(1, 2), t(3, 2, 128), i(3), cache, 32),
                 lambda: mpic.mpic_q4_read(ctx.handle, cache, 32, i(3).long(), t(3, 2, 128), t(3, 2, 128)),
                 lambda: mpic.mpic_position_rows(ctx.handle, t(3, 4, 128), t(3, 2, 128), i(1, 2), t(3, 4, 128), t(3, 2, 128)),
                 lambda: mpic.mpic_position_rows(ctx.handle, t(3, 4, 128), t(3, 2, 128), i(1, 3), t(3, 4, 128), t(3, 2, 128), pair_axis=[0] * 63),
                 lambda: mpic.mpic_position_rows(ctx.handle, t(3, 4, 128), t(3, 2, 128), i(1, 3), t(3, 4, 128), t(3, 2, 128), eps=-1.0),
                 lambda: mpic.mpic_q4_attn(ctx.handle, t(3, 4, 128), cache, 32, i(3, 2), 16, i(2), 0.1, t(3, 4, 128)),
                 lambda: mpic.mpic_q4_attn(ctx.handle, t(3, 4, 128), cache, 32, i(3, 2), 16, i(3), 0.1, t(3, 4, 128), q_off=i(3)),
                 lambda: mpic.mpic_q4_attn(ctx.handle, t(3, 4, 128), cache, 32, i(3, 2), 16, i(3), 0.1, t(3, 4, 128), lse=t(3, 4)),
                 lambda: mpic.mpic_q4_read(ctx.handle, cache[::2], 2, i(3), t(3, 2, 128), t(3, 2, 128))):
        with pytest.raises(ValueError):
            call()
