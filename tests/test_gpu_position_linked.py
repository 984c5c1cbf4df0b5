"""Rows positioned on several axes and stored chunks linked behind each other (needs an MI355X)."""
import numpy as np
import pytest
import torch

import paper_2502_01960_amd as mpic
from oracle import position_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("origin", [37, 5, 4000])
def test_a_chunk_of_several_axes_is_moved_to_its_token_index_on_all_of_them(bf16, interleaved, origin):
    """Text, an image positioned on (time, height, width) from its own origin, text: the image's first token stands at its
    token index, 37, on every axis.  Where it belongs elsewhere, its keys are turned by the difference first."""
    hq, hkv, d, theta = 4, 2, 128, 1e6
    dt = torch.bfloat16 if bf16 else torch.float32
    first, h, w = 37, 9, 13
    n = h * w
    grid = np.stack([np.zeros(n), np.repeat(np.arange(h), w), np.tile(np.arange(w), h)]).astype(np.int64)
    pair_axis = [0] * 16 + [1] * 24 + [2] * 24
    gen = torch.Generator().manual_seed(4)
    rand = lambda m: torch.randn((m, hkv, d), generator=gen).to(dt)
    raw_k, v, text_k, text_v = rand(n), rand(n), rand(first + 20), rand(first + 20)
    ctx = mpic.Context(hq, hkv, d, mpic.MPIC_BF16 if bf16 else mpic.MPIC_F32, theta, interleaved)
    pos = lambda p: torch.from_numpy(p).to(torch.int32).to(DEV)

    def positioned(x, p, axes):
        out = torch.empty_like(x, device=DEV)
        q = torch.zeros((x.shape[0], hq, d), dtype=dt, device=DEV)
        mpic.mpic_position_rows(ctx.handle, q, x.to(DEV), pos(p), q, out, pair_axis=axes)
        return out

    stored = positioned(raw_k, grid, pair_axis)
    text_pos = np.concatenate([np.arange(first), first + n + np.arange(20)])
    if origin != first:
        stored = positioned(stored.cpu(), np.full((1, n), origin - first), None)
    fresh = positioned(text_k, np.stack([text_pos] * 3), pair_axis)
    total = first + n + 20
    plan = mpic.Plan(ctx, [[("text", first), ("chunk", 0, n, None), ("text", 20)]], 0)
    k_ctx, v_ctx = (torch.full((total, hkv, d), float("nan"), dtype=dt, device=DEV) for _ in range(2))
    mpic.mpic_assemble_kv(ctx.handle, plan.handle, [(stored, v.to(DEV))], fresh, text_v.to(DEV), k_ctx, v_ctx)
    torch.cuda.synchronize()
    everything = np.concatenate([np.stack([np.arange(first)] * 3), grid + origin, first + n + np.stack([np.arange(20)] * 3)], axis=1)
    x = torch.cat([text_k[:first], raw_k, text_k[first:]]).double().numpy()
    want = position_rows(x, everything, theta, bool(interleaved), pair_axis)
    # two rotations (three), each with its own rounding to the type, of which the earlier ones are turned along with the pair; a
    # pair's amplitude bounds its values.  f32: some 32 roundings of 2^-24 in a rotation, as many in the linker's tables and shift
    half = d // 2
    a, b = (x[..., ::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    size = np.hypot(a, b)
    size = np.stack([size, size], -1).reshape(x.shape) if interleaved else np.concatenate([size, size], -1)
    turns = 1 if origin == first else 2       # in front of the last
    tol = ((2.0 ** -8 * (1 + turns * np.sqrt(2)) if bf16 else 0) + 32 * (turns + 1) * 2.0 ** -24) * size
    err = np.abs(k_ctx.double().cpu().numpy() - want)
    assert (err <= tol).all(), float((err / tol).max())
    assert torch.equal(v_ctx.cpu(), torch.cat([text_v[:first], v, text_v[first:]]))
