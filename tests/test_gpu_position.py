"""mpic_position_rows against the float64 oracle (needs an MI355X)."""
import numpy as np
import pytest
import torch

import paper_2502_01960_amd as mpic
from oracle import position_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _run(rows, hq, hkv, d, bf16, *, norm=True, weights=True, interleaved=False, axes=1, far=20000, fused=False, in_place=False,
         seed=0):
    dt = torch.bfloat16 if bf16 else torch.float32
    gen = torch.Generator().manual_seed(seed + rows)
    rng = np.random.default_rng(seed + rows)
    theta = 1e6 if bf16 else 1e4
    normal = lambda *s: torch.randn(s, generator=gen).to(dt)
    if fused:
        both = normal(rows, hq + 2 * hkv, d)
        held = both.to(DEV)
        q, k = held[:, :hq], held[:, hq:hq + hkv]
    else:
        q, k = normal(rows, hq, d).to(DEV), normal(rows, hkv, d).to(DEV)
        held = None
    qh, kh = q.double().cpu().numpy(), k.double().cpu().numpy()
    pos = rng.integers(-far, far, (axes, rows), endpoint=True)
    pos[:, 0] = 0
    pair_axis = None if axes == 1 else [int(a) for a in rng.integers(0, axes, d // 2)]
    wq, wk = ((1 + 0.2 * normal(d).float()).to(dt), (1 + 0.2 * normal(d).float()).to(dt)) if norm and weights else (None, None)
    eps = 1e-6 if norm else None
    ctx = mpic.Context(hq, hkv, d, mpic.MPIC_BF16 if bf16 else mpic.MPIC_F32, theta, int(interleaved))
    if in_place:
        qo, ko = q, k
    else:
        qo, ko = (torch.full(x.shape, float("nan"), dtype=dt, device=DEV) for x in (q, k))
    dev = lambda t: None if t is None else t.to(DEV)
    mpic.mpic_position_rows(ctx.handle, q, k, torch.from_numpy(pos).to(torch.int32).to(DEV), qo, ko, dev(wq), dev(wk), eps, pair_axis)
    torch.cuda.synchronize()
    for x, w, got in ((qh, wq, qo), (kh, wk, ko)):
        ref = position_rows(x, pos, theta, interleaved, pair_axis, None if w is None else w.double().numpy(), eps)
        got = got.double().cpu().numpy()
        # what the two values of a pair amount to before the rotation bounds what rounding in fp32 does to it: some 32
        # roundings of 2^-24 (sum of squares, root, weight, sine and cosine, products), and the last one to the type
        plain = np.abs(position_rows(x, np.zeros_like(pos), theta, interleaved, pair_axis, None if w is None else w.double().numpy(), eps))
        half = d // 2
        other = np.concatenate([plain[..., half:], plain[..., :half]], -1) if not interleaved else \
            plain.reshape(plain.shape[:-1] + (half, 2))[..., ::-1].reshape(plain.shape)
        tol = 32 * 2.0 ** -24 * (plain + other) + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(ref)
        err = np.abs(got - ref)
        assert (err <= tol).all(), float((err - tol).max())
    if fused and in_place:    # the values of the projection next to them are left alone
        assert torch.equal(held[:, hq + hkv:].cpu(), both[:, hq + hkv:])


@pytest.mark.parametrize("rows", [1, 2, 5, 64, 257, 4099])
@pytest.mark.parametrize("heads", [(28, 4), (3, 1), (32, 32), (72, 8)])
def test_bf16(rows, heads):
    if rows * sum(heads) < 200000:
        _run(rows, *heads, 128, True, axes=1 + rows % 4, interleaved=rows % 2 == 0, fused=rows % 3 == 0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 7, 130, 4100])
@pytest.mark.parametrize("interleaved", [False, True])
def test_f32(d, rows, interleaved):
    _run(rows, 4, 2, d, False, axes=1 + rows % 3, interleaved=interleaved, norm=rows != 7, fused=rows == 130)


@pytest.mark.parametrize("norm,weights", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("fused", [False, True])
def test_forms(norm, weights, in_place, fused):
    _run(37, 14, 2, 128, True, norm=norm, weights=weights, in_place=in_place, fused=fused, axes=3)
    _run(37, 6, 2, 64, False, norm=norm, weights=weights, in_place=in_place, fused=fused, axes=2)


def test_far_positions():
    _run(300, 4, 2, 128, True, far=2 ** 31 - 1, axes=4)
    _run(300, 4, 2, 128, False, far=2 ** 24)


def test_positions_past_an_fp32_product():
    """A whole number of turns of the first pair apart as nearly as whole numbers come: the rows agree to 1e-6, which
    angles formed in fp32 miss by 0.5."""
    ctx = mpic.Context(1, 1, 64, mpic.MPIC_F32, 1e4)
    x = torch.zeros((2, 1, 64), device=DEV)
    x[..., 0] = 1
    out = torch.empty_like(x)
    pos = torch.tensor([[0, 710 * 3 * 10 ** 5]], dtype=torch.int32, device=DEV)
    mpic.mpic_position_rows(ctx.handle, x, x.clone(), pos, out, torch.empty_like(x))
    want = position_rows(x.double().cpu().numpy(), pos.cpu().numpy(), 1e4)
    assert np.abs(out.double().cpu().numpy() - want).max() < 1e-6


def test_equals_the_rotation_of_the_linker():
    """Rows positioned here and linked equal rows that a fresh_pre_rope context positions itself, up to a rounding."""
    n, hq, hkv, d = 33, 4, 2, 128
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((n, h, d), generator=gen).to(torch.bfloat16).to(DEV) for h in (hq, hkv, hkv))
    got = []
    for pre in (0, 1):
        ctx = mpic.Context(hq, hkv, d, mpic.MPIC_BF16, 1e6, 0, 0, pre)
        plan = mpic.Plan(ctx, [[("text", n)]], 0)
        kr, qr = k.clone(), q.clone()
        if not pre:
            mpic.mpic_position_rows(ctx.handle, qr, kr, torch.arange(n, dtype=torch.int32, device=DEV), qr, kr)
        kc, vc = (torch.zeros((n, hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        mpic.mpic_assemble_kv(ctx.handle, plan.handle, None, kr, v, kc, vc)
        torch.cuda.synchronize()
        got.append(kc.double().cpu())
    assert (got[0] - got[1]).abs().max() <= 2.0 ** -7 * got[0].abs().max()


def test_rows_that_are_zero_or_not_finite_stay_their_own():
    ctx = mpic.Context(2, 1, 128, mpic.MPIC_BF16, 1e4)
    q = torch.ones((4, 2, 128), dtype=torch.bfloat16, device=DEV)
    k = torch.ones((4, 1, 128), dtype=torch.bfloat16, device=DEV)
    q[1, 0] = 0
    q[2, 1, 5] = float("nan")
    k[3] = float("inf")
    pos = torch.arange(4, dtype=torch.int32, device=DEV)
    mpic.mpic_position_rows(ctx.handle, q, k, pos, q, k, eps=1e-6)
    torch.cuda.synchronize()
    assert (q[1, 0] == 0).all() and torch.isnan(q[2, 1].float()).all() and torch.isnan(k[3].float()).all()
    assert torch.isfinite(q[[0, 3]].float()).all() and torch.isfinite(q[2, 0].float()).all() and torch.isfinite(k[:3].float()).all()


@pytest.mark.parametrize("bf16", [True, False])
def test_zeros_stay_zeros_for_any_eps(bf16):
    ctx = mpic.Context(2, 1, 128, mpic.MPIC_BF16 if bf16 else mpic.MPIC_F32, 1e4)
    for eps in (1e-300, 1e-40, 1e300):
        q, k = (torch.zeros((3, h, 128), dtype=torch.bfloat16 if bf16 else torch.float32, device=DEV) for h in (2, 1))
        mpic.mpic_position_rows(ctx.handle, q, k, torch.arange(3, dtype=torch.int32, device=DEV), q, k, eps=eps)
        torch.cuda.synchronize()
        assert (q == 0).all() and (k == 0).all(), eps


def test_no_rows():
    ctx = mpic.Context(2, 1, 128, mpic.MPIC_BF16, 1e4)
    e = lambda h: torch.empty((0, h, 128), dtype=torch.bfloat16, device=DEV)
    mpic.mpic_position_rows(ctx.handle, e(2), e(1), torch.empty((1, 0), dtype=torch.int32, device=DEV), e(2), e(1))
