"""What the binding takes and refuses in front of the calls on positions and contexts in 4 bits (CPU: nothing reaches the GPU)."""
import pytest
import torch

import paper_2502_01960_amd as mpic
from paper_2502_01960_amd import binding

HQ, HKV, D, SLOTS, PAGE = 4, 2, 128, 32, 16


class _Taken:
    """Stands for the library: every call that gets there is noted and does nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def taken(monkeypatch):
    lib = mpic.load_library()
    t = _Taken()
    t.mpic_destroy = lib.mpic_destroy
    monkeypatch.setattr(binding, "_lib", t)
    yield t
    monkeypatch.setattr(binding, "_lib", lib)


@pytest.fixture(params=[mpic.MPIC_BF16, mpic.MPIC_F32], ids=["bf16", "f32"])
def ctx(request):
    c = mpic.Context(HQ, HKV, D, request.param, 1e4)
    c.cache_bytes = mpic.mpic_q4_bytes(c.handle, SLOTS)
    c.torch_dtype = torch.float32 if request.param == mpic.MPIC_F32 else torch.bfloat16
    return c


def _i(*s):
    return torch.zeros(s, dtype=torch.int32)


def _args(ctx, call, n=3, **kw):
    """(function, arguments) of a call that is right but for what kw replaces."""
    t = lambda h: torch.zeros((n, h, D), dtype=ctx.torch_dtype)
    cache = torch.zeros(ctx.cache_bytes, dtype=torch.uint8)
    a = {"position": lambda: dict(q=t(HQ), k=t(HKV), pos=_i(1, n), q_out=t(HQ), k_out=t(HKV), stream=0),
         "write": lambda: dict(k=t(HKV), v=t(HKV), slots=_i(n), cache=cache, n_slots=SLOTS, stream=0),
         "read": lambda: dict(cache=cache, n_slots=SLOTS, slots=_i(n), k=t(HKV), v=t(HKV), stream=0),
         "attn": lambda: dict(q=t(HQ), cache=cache, n_slots=SLOTS, page_table=_i(n, 2), page_size=PAGE, lens=_i(n), softmax_scale=0.1,
                              out=t(HQ), stream=0)}[call]()
    a.update(kw)
    return {"position": mpic.mpic_position_rows, "write": mpic.mpic_q4_write, "read": mpic.mpic_q4_read, "attn": mpic.mpic_q4_attn}[call], a


def _refused(ctx, taken, call, **kw):
    f, a = _args(ctx, call, **kw)
    with pytest.raises(ValueError):
        f(ctx.handle, **a)
    assert not taken.calls, kw


@pytest.mark.parametrize("call", ["position", "write", "read", "attn"])
def test_calls_that_are_right_arrive(ctx, taken, call):
    for n in (0, 1, 3):
        f, a = _args(ctx, call, n=n)
        f(ctx.handle, **a)
    assert len(taken.calls) == 3


@pytest.mark.parametrize("dtype", [torch.float32, torch.uint32, torch.int64, torch.int16])
@pytest.mark.parametrize("call,names", [("position", ["pos"]), ("write", ["slots"]), ("read", ["slots"]), ("attn", ["page_table", "lens", "q_off"])])
def test_what_is_not_int32_is_refused(ctx, taken, call, names, dtype):
    """A float32 length of 64 would be read as 1115684864."""
    _, right = _args(ctx, call)
    for name in names:
        _refused(ctx, taken, call, **{name: (_i(4) if name == "q_off" else right[name]).to(dtype)})


@pytest.fixture
def one_head():
    return mpic.Context(1, 1, D, mpic.MPIC_BF16, 1e4)


def test_one_head_may_have_any_stride(one_head, taken):
    """A contiguous [n][1][D] tensor that was [1][n][D] before: the stride of its only head is that of all rows."""
    ctx = one_head
    x = lambda: torch.zeros((1, 5, D), dtype=torch.bfloat16).transpose(0, 1)
    assert x().is_contiguous() and x().stride(1) == 5 * D
    cache = torch.zeros(SLOTS * 144, dtype=torch.uint8)
    mpic.mpic_position_rows(ctx.handle, x(), x(), _i(5), x(), x(), stream=0)
    mpic.mpic_q4_write(ctx.handle, x(), x(), _i(5), cache, SLOTS, 0)
    mpic.mpic_q4_read(ctx.handle, cache, SLOTS, _i(5), x(), x(), 0)
    mpic.mpic_q4_attn(ctx.handle, x(), cache, SLOTS, _i(5, 2), PAGE, _i(5), 0.1, x(), stream=0)
    assert [name for name, _ in taken.calls] == ["mpic_position_rows", "mpic_q4_write", "mpic_q4_read", "mpic_q4_attn"]
    strides = [a[i] for (_, a), where in zip(taken.calls, ((2, 4, 13, 15), (2, 4), (7, 9), (2,))) for i in where]
    assert strides == [D] * len(strides)


def _rows_of(call):
    return {"position": (("q", HQ), ("k", HKV), ("q_out", HQ), ("k_out", HKV)), "write": (("k", HKV), ("v", HKV)),
            "read": (("k", HKV), ("v", HKV)), "attn": (("q", HQ), ("out", HQ))}[call]


@pytest.mark.parametrize("call", ["position", "write", "read", "attn"])
def test_rows_of_another_type_or_form_are_refused(ctx, taken, call):
    """A bf16 output of an f32 context would be written to twice its size; rows of a projection with fewer heads than the
    context's take the next part of the row along."""
    other = torch.float32 if ctx.torch_dtype == torch.bfloat16 else torch.bfloat16
    for name, heads in _rows_of(call):
        t = lambda h=heads, n=3, d=D, dt=ctx.torch_dtype: torch.zeros((n, h, d), dtype=dt)
        wide = torch.zeros((3, 8, D), dtype=ctx.torch_dtype)
        bad = [t(dt=other), t(dt=torch.float16), t(h=heads - 1), t(h=heads + 1), t(d=D // 2), t(d=2 * D)]
        if name != "out":
            bad += [wide[:, :heads - 1], wide[:, :heads + 1]]
        if name not in ("q", "k") or (call, name) == ("position", "k"):
            bad += [t(n=2), t(n=4)]
        for x in bad:
            _refused(ctx, taken, call, **{name: x})
    if call == "attn":           # q and out alike, and unlike the context
        for h in (2, 8):
            x = torch.zeros((3, h, D), dtype=ctx.torch_dtype)
            _refused(ctx, taken, call, q=x, out=x.clone())
        for lse in (torch.zeros((3, HQ), dtype=torch.int32), torch.zeros((3, HQ), dtype=torch.float64), torch.zeros((3, HQ + 1))):
            _refused(ctx, taken, call, lse=lse)
        f, a = _args(ctx, call, lse=torch.zeros((3, HQ)))
        f(ctx.handle, **a)


def test_a_handle_that_was_made_elsewhere_serves_as_before(ctx, taken):
    """Its form is not known, so rows only have to agree among themselves."""
    import ctypes
    for call in ("position", "write", "read", "attn"):
        f, a = _args(ctx, call)
        f(ctypes.c_void_p(ctx.handle.value), **a)
        f(ctx.handle.value, **a)
        name, heads = _rows_of(call)[-1]
        f, a = _args(ctx, call, **{name: torch.zeros((3, heads + 1, D + 1), dtype=ctx.torch_dtype)})
        with pytest.raises(ValueError):
            f(ctx.handle.value, **a)
    assert len(taken.calls) == 8


def test_weights_of_another_type_or_length_are_refused(ctx, taken):
    """f32 weights of a bf16 context would be read as bf16, short ones past their end, strided ones between their values."""
    other = torch.float32 if ctx.torch_dtype == torch.bfloat16 else torch.bfloat16
    w = torch.zeros(D, dtype=ctx.torch_dtype)
    for bad in (w.to(other), w[:D // 2], w[:D - 1], torch.zeros(D + 1, dtype=ctx.torch_dtype), torch.zeros(2 * D, dtype=ctx.torch_dtype)[::2]):
        for name in ("q_weight", "k_weight"):
            _refused(ctx, taken, "position", eps=1e-6, **{name: bad})
    for kw in (dict(q_weight=w, k_weight=w), dict(q_weight=w), dict(k_weight=w[None]), {}):
        f, a = _args(ctx, "position", eps=1e-6, **kw)
        f(ctx.handle, **a)
    assert len(taken.calls) == 4
