"""GPU: explicit softmax scales over the 4-bit cache, subnormal ones among them,
where units are run once and where they are run again with their rows' maxima.
The bars are those of the default scale."""
import numpy as np
import pytest

from test_gpu_kv4 import DIFF, VER, Attn, _lib, check  # noqa: F401
from test_gpu_kv4_ranges import set_scores, size_of

pytestmark = pytest.mark.gpu
HEADS = [((8, 2, 64), 1), ((16, 2, 128), 2), ((16, 2, 64), 7), ((40, 8, 128), 13), ((20, 1, 128), 8)]


def with_scale(c, scale):
    c.params.softmax_scale = scale
    c.scale = float(np.float32(scale))
    return c


@pytest.mark.parametrize("heads,bl", HEADS)
@pytest.mark.parametrize("scale", [1e-39, 3e-39, 1.2e-38, 1e-30, 1e-3, 0.07, 0.5])
def test_scales(orc, heads, bl, scale):
    c = with_scale(Attn(900 + bl, heads, 16, [300, 0, 1], bl), scale)
    for mode in (DIFF, VER):
        out, lse = c.run(mode)
        check(out, lse, *c.oracle(orc, mode), size=size_of(c))
    # a table: units that begin inside the block take their rows' maxima first
    mask = np.array([(0xFFFFFFFF << (i % bl)) & ((1 << bl) - 1) for i in range(bl)], np.uint32)
    out, lse = c.run(mask=mask)
    check(out, lse, *c.oracle(orc, mask=mask), size=size_of(c))


@pytest.mark.parametrize("heads,bl", HEADS[2:])
@pytest.mark.parametrize("profile", ["ramp", "late_peak", "first_high"])
@pytest.mark.parametrize("factor", [0.3, 1.9])
def test_scales_out_of_range_of_the_first_reference(orc, heads, bl, profile, factor):
    """Score levels of up to 285, with rows that disagree about them."""
    c = Attn(950 + bl, heads, 16, [900, 40], bl)
    set_scores(c, np.random.default_rng(bl), profile, (1.0, -1.0, 0.01, 0.5))
    with_scale(c, factor / np.sqrt(c.D))
    for mode in (DIFF, VER):
        out, lse = c.run(mode)
        check(out, lse, *c.oracle(orc, mode), size=size_of(c))
