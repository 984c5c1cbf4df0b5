"""The bound of closeness.py rejects what faulty kernels would return and takes what the stated roundings give (CPU: every
mistake is planted in the oracle)."""
import math

import numpy as np
import pytest

from closeness import allowed, hold, worst
from oracle.held import round_bf16, round_f32


def _problem(n, new, hq, hkv, d, bf16, seed, spread=1.0):
    rng = np.random.default_rng(seed)
    last = round_bf16 if bf16 else round_f32
    k = last(rng.standard_normal((n, hkv, d)) + 2 * rng.standard_normal((1, hkv, d)))
    v = last(rng.standard_normal((n, hkv, d)))
    q = last(spread * rng.standard_normal((new, hq, d)))
    return q, hold([k], bf16), hold([v], bf16), [n], [new], 1 / math.sqrt(d)


def _computed(q, held_k, held_v, n, new, scale, bf16, mid_bits=16, keep=None):
    """What a kernel with the stated roundings returns; keep: tokens whose V takes part (a planted mistake otherwise)."""
    (k, _, _, _), (_, code, v_scale, v_low) = held_k[0], held_v[0]
    last = round_bf16 if bf16 else round_f32
    out = np.zeros(q.shape)
    for i in range(new):
        seen = n - new + i + 1
        for h in range(q.shape[1]):
            kv = h // (q.shape[1] // k.shape[1])
            s = scale * (k[:seen, kv] @ q[i, h])
            p = np.exp(s - s.max())
            z = p.sum()
            if keep is not None:
                p = np.where(keep[:seen], p, 0.0)
            for g in range(k.shape[2] // 64):
                sc, lo = v_scale[:seen, kv, g], v_low[:seen, kv, g]
                w = last(p * sc)
                m = p if mid_bits == 16 or not bf16 else round_bf16(p)
                cols = slice(64 * g, 64 * g + 64)
                out[i, h, cols] = (w @ (code[:seen, kv, cols] - 8.0) + m @ (lo + 8 * sc)) / z
    return last(out)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n,new,spread", [(1, 1, 1.0), (40, 3, 1.0), (1000, 1, 1.0), (9000, 1, 0.0), (4097, 1, 8.0)])
def test_the_stated_roundings_pass(bf16, n, new, spread):
    p = _problem(n, new, 4, 2, 128, bf16, n, spread)
    ref, bound = allowed(*p, bf16)
    assert worst(_computed(*p[:3], n, new, p[5], bf16), ref, bound) <= 0.8
    assert worst((round_bf16 if bf16 else round_f32)(ref), ref, bound) <= 0.8


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("n", [1000, 9000, 30000])
def test_values_that_are_left_out_are_rejected(bf16, n):
    """One split of 256 tokens, one unit of 32, in f32 a single token: of V only, so that the log-sum-exp says nothing."""
    p = _problem(n, 1, 4, 2, 128, bf16, 1)
    ref, bound = allowed(*p, bf16)
    for first, last in ((256, 512), (320, 352)) + (() if bf16 else ((n // 2, n // 2 + 1),)):
        keep = np.ones(n, bool)
        keep[first:last] = False
        assert worst(_computed(*p[:3], n, 1, p[5], bf16, keep=keep), ref, bound) > 1.5, (first, last)
    assert worst(ref * 1.03, ref, bound) > 1.5


def test_rows_that_see_nothing_have_to_be_zeros():
    p = _problem(3, 5, 4, 2, 128, True, 2)
    ref, bound = allowed(*p, True)
    assert (bound[:2] == 0).all() and worst(ref, ref, bound) == 0.0
    ref2 = ref.copy()
    ref2[0, 0, 0] = 1e-30
    assert worst(ref2, ref, bound) == math.inf


def opposite(n, new, hq, hkv, c=64.0):
    """One token of weight 1 with values near c, three of weight near 1/3 with values near -c, the rest far off: an output of
    nearly nothing, in which the weights that meet the minima show as they were rounded."""
    rng = np.random.default_rng(n + new)
    k, v, q = np.zeros((n, hkv, 128)), rng.standard_normal((n, hkv, 128)), np.zeros((new, hq, 128))
    k[..., 0] = -60.0
    k[5, :, 0] = 1.875
    v[5] = c
    for j in (10, 20, 30):
        k[j, :, 0] = 0.0
        v[j] = -c
    v[[5, 10, 20, 30]] += 0.5 * rng.integers(0, 2, (4, hkv, 128))
    q[..., 0] = 6.625
    return q, round_bf16(k), round_bf16(v)


def test_minima_met_by_weights_of_eight_bits_are_rejected():
    q, k, v = opposite(100, 4, 8, 2)
    p = (q, hold([k], True), hold([v], True))
    ref, bound = allowed(*p, [100], [4], 1 / math.sqrt(128), True)
    assert worst(_computed(*p, 100, 4, 1 / math.sqrt(128), True), ref, bound) <= 0.8
    assert worst(_computed(*p, 100, 4, 1 / math.sqrt(128), True, mid_bits=8), ref, bound) > 2
