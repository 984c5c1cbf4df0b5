"""Attention over contexts in 4 bits, row by row as near to the oracle as its roundings allow (needs an MI355X)."""
import math

import numpy as np
import pytest
import torch

import paper_2502_01960_amd as mpic
from closeness import allowed, hold, worst
from test_closeness_host import opposite
from test_gpu_q4 import BOUND, DEV, Held, _attend, _dt, _i32

pytestmark = pytest.mark.gpu

# (query heads, kv heads, head dim, bf16), new tokens of a request: 8, 16 and 32 rows a workgroup, f32 of both head dims
FORMS = {"8_rows": ((8, 2, 128, True), 1), "16_rows": ((8, 2, 128, True), 4), "32_rows": ((8, 2, 128, True), 40),
         "f32_128": ((4, 2, 128, False), 2), "f32_64": ((4, 2, 64, False), 3)}


def _close(p, out, lens=None, scale=None):
    held = [hold([x.double().numpy() for x in side], p.bf16) for side in (p.k, p.v)]
    ref, bound = allowed(p.q.double().numpy(), *held, p.lens if lens is None else lens, p.news, scale or 1 / math.sqrt(p.d), p.bf16)
    share = worst(out, ref, bound)
    print(f"error norm {share:.3f} of what is allowed")
    assert share <= 1.0


@pytest.mark.parametrize("form", [f for f in FORMS if FORMS[f][0][3]])
def test_values_far_from_zero_that_cancel(form):
    """Minima of 64 and -64 in an output of nearly nothing: the weights that meet them have 16 bits in every form."""
    model, new = FORMS[form]
    p = Held([100], [new], *model)
    q, k, v = opposite(100, new, *model[:2])
    p.q, p.k, p.v = torch.from_numpy(q).to(_dt(True)), [torch.from_numpy(k).to(_dt(True))], [torch.from_numpy(v).to(_dt(True))]
    j = np.arange(100)
    mpic.mpic_q4_write(p.ctx.handle, p.k[0].to(DEV), p.v[0].to(DEV), _i32(p.table[0, j // 16] * 16 + j % 16), p.cache, p.n_slots)
    _close(p, p.run(max_len=BOUND if new == 40 else None)[0])


@pytest.mark.parametrize("form", FORMS)
def test_the_least_scale_weighs_all_tokens_alike(form):
    """Some of which are not seen."""
    model, new = FORMS[form]
    p = Held([90, 33], [new, 2], *model)
    out = torch.full(p.q.shape, 77.0, dtype=_dt(p.bf16), device=DEV)
    bound = BOUND if new == 40 else p.table.shape[1] * p.page
    table = np.pad(p.table, ((0, 0), (0, bound // p.page - p.table.shape[1])), constant_values=-1)
    _attend(p.ctx, p.q.to(DEV), p.cache, p.n_slots, _i32(table), p.page, _i32(p.lens), out, None, _i32(p.q_off), max(p.news), bound,
            2.0 ** -126)
    _close(p, out.double().cpu().numpy(), scale=2.0 ** -126)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("n", [2000, 4000, 9000])
def test_splits_and_their_merge(form, n):
    """Up to 8 splits, up to 16, more: the merge has a shape for each."""
    model, new = FORMS[form]
    p = Held([n, n // 2 + 1, 2], [new, new, 1], *model, page=64)
    for max_len in (None, 3 * n):
        _close(p, p.run(max_len=max_len)[0])
    if new == 40:
        _close(p, p.run(max_len=BOUND)[0])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("n", [1, 2, 16, 33, 130, 500])
def test_short_contexts(form, n):
    model, new = FORMS[form]
    p = Held([n, 3], [new, 1], *model, page=16)
    _close(p, p.run()[0])
    _close(p, p.run(max_len=BOUND)[0])


@pytest.mark.parametrize("form", [f for f in FORMS if f != "32_rows"])
def test_pages_are_looked_up_again_behind_32_units_of_a_wavefront(form):
    """A launch of so many requests that a split has 53 units for every wavefront; one request has keys for two and a half of
    them, in shuffled pages."""
    model, new = FORMS[form]
    lens, news = [14000] + [0, 1, 40, 0, 0, 2, 0] * 146 + [300], [new] + [1] * 1023
    p = Held(lens, news, *model, page=64)
    _close(p, p.run(max_len=20000)[0])


def test_requests_that_are_shifted_or_cut_by_their_offsets():
    """Rows of no request are left as they were, the others are right: offsets that leave rows in front and behind, that are
    cut to the rows there are, that run backwards (a request without queries)."""
    p = Held([64, 64, 33], [2, 2, 1], 4, 2, 128, True)
    every = p.q
    for off, rows in (([2, 5, 5, 5], {0: (2, 3)}), ([1, 1, 3, 3], {1: (1, 2)}), ([0, 9, 1, 0], {0: (0, 5)}),
                      ([-9, 1, 2 ** 31 - 1, 7], {0: (0, 1), 1: (1, 4)}), ([4, 1, 0, 0], {}), ([3, 2, 5, 4], {1: (2, 3)})):
        p.q, p.q_off = every, np.array(off)
        out, lse = p.run(max_q=5)
        told = np.zeros(len(every), bool)
        for b, (first, n) in rows.items():
            told[first:first + n] = True
            one = Held([1], [1], 4, 2, 128, True)
            one.k, one.v, one.q, one.lens, one.news = [p.k[b]], [p.v[b]], every[first:first + n], [p.lens[b]], [n]
            _close(one, out[first:first + n])
        assert (out[~told] == 77).all() and (lse[~told] == 77).all(), off
