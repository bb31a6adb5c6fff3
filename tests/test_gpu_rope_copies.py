"""GPU: what an append copies, it copies bit for bit: V, and the channels of q
and K that are not rotated, every bf16 bit pattern among them."""
import numpy as np
import pytest
import torch

from paper_2607_05722_gb300 import nld
from test_gpu_kv4 import Append, _lib, i32  # noqa: F401

pytestmark = pytest.mark.gpu


def bits_of(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


@pytest.mark.parametrize("heads,new,rot,style", [
    ((2, 1, 64), [300, 300], 0, "half"), ((4, 2, 128), [70, 60], 64, "half"), ((4, 2, 128), [70, 60], 32, "interleaved"),
    ((2, 1, 128), [2000, 600], 16, "half"),  # rows in great number: a warp each
])
@pytest.mark.parametrize("kv4", [False, True])
def test_copies_keep_their_bits(heads, new, rot, style, kv4):
    c = Append(12, heads, 16, [5, 0], new, rot, style)
    T, H = sum(new), c.Hq + 2 * c.Hkv
    bits = np.resize(np.random.default_rng(0).permutation(1 << 16), T * H * c.D).astype(np.uint16).reshape(T, H, c.D)
    x = torch.from_numpy(bits.view(np.int16)).cuda().view(torch.bfloat16)
    q, k, v = x[:, :c.Hq], x[:, c.Hq:c.Hq + c.Hkv], x[:, c.Hq + c.Hkv:]
    q_out = torch.zeros(T, c.Hq, c.D, dtype=torch.bfloat16, device="cuda")
    pages = [torch.zeros(c.num_pages, c.Hkv, 16, c.D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    if kv4:
        pages = [torch.zeros(nld.kv4_pages_shape(c.params), dtype=torch.uint8, device="cuda")]
    call = nld.nld_rope_append_kv4 if kv4 else nld.nld_rope_append
    call(c.params, q, k, v, c.rope_dev(), i32(c.table), i32(c.lens), *pages, q_out=q_out, **c.args())
    assert np.array_equal(bits_of(q_out)[..., rot:], bits[:, :c.Hq, rot:])
    if kv4:  # it holds no infinities or NaN, and says so
        assert nld.nld_device_error(clear=True) == nld.NLD_DEVERR_NONFINITE
        return
    page, slot = c.table[c.b, c.at // 16], c.at % 16
    assert np.array_equal(bits_of(pages[0])[page, :, slot][..., rot:], bits[:, c.Hq:c.Hq + c.Hkv, rot:])
    assert np.array_equal(bits_of(pages[1])[page, :, slot], bits[:, c.Hq + c.Hkv:])
