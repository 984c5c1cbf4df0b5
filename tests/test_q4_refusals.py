"""What the entry points for positions and contexts in 4 bits refuse at the ends of their ranges (CPU: nothing reaches the GPU)."""
import os
import shutil
import subprocess

import pytest

import paper_2502_01960_amd as mpic
from test_q4_host import A, INVALID, ROOT, UNSUPPORTED, _attn, _lib, _position, ctx    # noqa: F401


def test_scales_that_are_no_positive_fp32_number_are_refused(ctx):
    """1e-60 is zero in fp32, and zero times the -infinity of a token that is not seen is no number."""
    for scale in (1e-60, 1e-300, 5e-324, 2.0 ** -127, 2.0 ** 124, 1e38, 1e300):
        assert _attn(ctx, scale=scale) == INVALID, scale
        assert "softmax_scale" in mpic.binding.mpic_last_error(ctx.handle)
    for scale in (2.0 ** -126, 2.0 ** 123):
        assert _attn(ctx, scale=scale, n_rows=0, q_off=A, q=None, out=None) == 0, scale


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_refusals_without_host_memory_throw_nothing(tmp_path):
    exe = str(tmp_path / "q4_no_memory")
    lib = mpic.lib_path()
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "native", "q4_no_memory.cpp"),
                    lib, "-Wl,-rpath," + os.path.dirname(lib), "-o", exe], check=True, capture_output=True, text=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "refused without memory" in r.stdout, r.stdout + r.stderr


@pytest.mark.parametrize("dtype,heads", [(mpic.MPIC_BF16, 8 * 65535), (mpic.MPIC_F32, 4 * 65535)])
def test_more_heads_than_a_launch_holds_are_refused(dtype, heads):
    """Few rows spread their heads over the grid's second dimension, 65535 workgroups of 8 heads (f32: 4)."""
    wide = mpic.Context(heads, 1, 128, dtype, 1e4)      # (and one of k)
    row = heads * 128
    assert _position(wide, q_stride=row, qo_stride=row) == UNSUPPORTED
    assert "position_rows" in mpic.binding.mpic_last_error(wide.handle)
    assert _position(wide, q_stride=row, qo_stride=row, n=0) == 0


@pytest.mark.parametrize("heads", [1 << 24, 1 << 25, 1 << 26, 1 << 28, 2 ** 31 - 1])
def test_sizes_of_a_cache_do_not_pass_64_bits(heads):
    """2^27 blocks of 2304 bytes for 2^28 heads are 9 * 2^63 bytes."""
    wide = mpic.Context(heads, heads, 128, mpic.MPIC_BF16, 1e4)
    exact = (1 << 27) * heads * 2304
    if exact < 1 << 63:
        assert mpic.mpic_q4_bytes(wide.handle, 2 ** 31 - 2) == exact
    else:
        with pytest.raises(mpic.MpicError) as e:
            mpic.mpic_q4_bytes(wide.handle, 2 ** 31 - 2)
        assert e.value.status == UNSUPPORTED
    assert mpic.mpic_q4_bytes(wide.handle, 16) == heads * 2304
    # and no buffer is taken to hold such a cache
    assert _lib().mpic_q4_write(wide.handle, A, heads * 128, A, heads * 128, 1, A, A, 2 ** 63 - 1, 2 ** 31 - 2, None) in (INVALID, UNSUPPORTED)
    assert _lib().mpic_q4_attn(wide.handle, A, heads * 128, 1, None, 1, A, 2 ** 63 - 1, 2 ** 31 - 2, A, 4, 16, A, 1, 64, 0.1, A, None, None, 0,
                               None) in (INVALID, UNSUPPORTED)
