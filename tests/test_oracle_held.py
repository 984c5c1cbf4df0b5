"""Pins of the oracle for positioned rows and contexts held in 4 bits (CPU)."""
import numpy as np
import pytest
import torch

from oracle import attend, build_plan, position_rows, q4_attend, q4_hold, rotate
from oracle.held import GROUP, round_bf16


def test_bf16_rounding_is_torch_s():
    x = np.random.default_rng(1).standard_normal(20000) * 10.0 ** np.random.default_rng(2).integers(-30, 30, 20000)
    x[:4] = [1.00390625, 1.01171875, 0.0, -1.00390625]       # halves between neighbours
    want = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).double().numpy()
    assert np.array_equal(round_bf16(x), want)


@pytest.mark.parametrize("interleaved", [False, True])
def test_one_axis_is_rotate_and_axes_are_independent(interleaved):
    rng = np.random.default_rng(3)
    x, pos = rng.standard_normal((5, 3, 64)), np.array([0, 1, 17, -4, 90001])
    got = position_rows(x, pos, 1e4, interleaved)
    for r in range(5):
        assert np.allclose(got[r], rotate(x[r], float(pos[r]), 1e4, interleaved), rtol=0, atol=1e-9)
    other = rng.integers(0, 1000, 5)
    axis = [i % 2 for i in range(32)]
    both = position_rows(x, [pos, other], 1e4, interleaved, axis)
    alone = [position_rows(x, p, 1e4, interleaved) for p in (pos, other)]
    for i in range(32):
        for e in ((2 * i, 2 * i + 1) if interleaved else (i, i + 32)):
            assert np.array_equal(both[..., e], alone[axis[i]][..., e])


def test_norm_has_unit_mean_square_and_keeps_zero_rows():
    x = np.random.default_rng(4).standard_normal((2, 2, 64)) * 100
    x[1, 1] = 0
    y = position_rows(x, np.zeros(2), 1e4, eps=1e-6)
    assert np.allclose((y[0] ** 2).mean(-1), 1, atol=1e-6) and (y[1, 1] == 0).all()
    assert np.allclose(position_rows(x, np.zeros(2), 1e4, weight=np.full(64, 3.0), eps=1e-6), 3 * y)


def test_a_group_by_hand():
    x = np.zeros((1, 1, 64))
    x[..., 0], x[..., 1], x[..., 2], x[..., 3], x[..., 4] = 15.0, 7.0, 2.5, 2.4, -0.0
    value, code, scale, low = q4_hold(x, True)
    assert scale.item() == 1.0 and low.item() == 0.0
    assert code[0, 0, :6].tolist() == [15, 7, 3, 2, 0, 0]      # the half goes up
    assert np.array_equal(value, code)


@pytest.mark.parametrize("bf16", [True, False])
def test_codes_name_the_nearest_value_and_the_least_is_kept(bf16):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((40, 2, 128)) * 10.0 ** rng.integers(-6, 6, (40, 2, 1)) + rng.standard_normal((40, 2, 1))
    x = round_bf16(x) if bf16 else x.astype(np.float32).astype(np.float64)
    value, code, scale, low = q4_hold(x, bf16)
    g, v = x.reshape(40, 2, 2, GROUP), value.reshape(40, 2, 2, GROUP)
    levels = low[..., None, None] + scale[..., None, None] * np.arange(16)
    best = np.abs(g[..., None] - levels).min(-1)
    assert (np.abs(g - v) <= best * (1 + 1e-6) + 1e-7 * np.abs(g)).all()
    assert (v.min(-1) == g.min(-1)).all()
    # half a scale, and at the upper end what 15 roundings of the scale may add
    assert (np.abs(g - v) <= scale[..., None] * (0.5 + 15 * (2.0 ** -8 if bf16 else 2.0 ** -23)) + 2.0 ** -23 * np.abs(g)).all()


def test_groups_that_are_flat_tiny_or_not_finite():
    x = np.zeros((5, 1, 64))
    x[0] = 3.0
    x[1, 0, 5] = 2.0 ** -99                       # a scale below 2^-100
    x[2, 0, 7], x[3, 0, 7] = np.nan, -np.inf
    x[4, 0, 0], x[4, 0, 1] = 3e38, -3e38          # a range beyond float32
    value, code, scale, low = q4_hold(x, False)
    assert (value[0] == 3.0).all() and (value[1] == 0.0).all() and np.isnan(value[2:]).all() and (code == 0).all()


def test_attention_is_attend_on_the_held_values():
    rng = np.random.default_rng(6)
    reqs, k = [[("text", 3), ("chunk", 0, 9, 0), ("text", 2)]], 0
    plan = build_plan(reqs, k, 0, None)
    kv = [q4_hold(rng.standard_normal((14, 2, 64)), False)[0] for _ in range(2)]
    q = rng.standard_normal((5, 4, 64))
    want, want_lse = attend(q, kv[0], kv[1], plan, 0.2)
    got, lse = q4_attend(q[3:], [kv[0]], [kv[1]], [14], [2], 0.2)
    assert np.allclose(got, want[3:], atol=1e-12) and np.allclose(lse, want_lse[3:], atol=1e-12)
    none, lse = q4_attend(q[:2], [kv[0][:1], kv[0][:0]], [kv[1][:1], kv[1][:0]], [1, 0], [2, 0], 0.2)
    assert (none[0] == 0).all() and (lse[0] == -np.inf).all() and np.isfinite(lse[1]).all()
