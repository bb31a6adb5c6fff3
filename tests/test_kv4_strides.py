"""The row strides that the appends' binding accepts (no GPU: a stand-in says it
is a CUDA tensor, and the entry is never reached)."""
import pytest
import torch

from paper_2607_05722_gb300 import nld

T, H, D = 6, 4, 64


class OnGpu:
    """A CPU tensor that calls itself a CUDA one."""

    def __init__(self, t):
        self.t, self.is_cuda = t, True

    def __getattr__(self, name):
        return getattr(self.t, name)


def bf16(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def refuse(*args):
    raise AssertionError("the entry point was called")


@pytest.mark.parametrize("which", ["q", "k_new", "v_new"])
@pytest.mark.parametrize("rows", [
    bf16(1, H, D).expand(T, H, D),                        # one row for all
    bf16(H * D + 8 * T).as_strided((T, H, D), (8, D, 1)),  # rows that start inside the one before
])
def test_rows_that_share_storage_are_refused(which, rows):
    t = dict.fromkeys(("q", "k_new", "v_new"), OnGpu(bf16(T, H, D)))
    t[which] = OnGpu(rows)
    params = nld.make_params(2, H, H, D, 16, 4, 2)
    i32 = lambda *s: OnGpu(torch.zeros(*s, dtype=torch.int32))  # noqa: E731
    with pytest.raises(ValueError, match=f"^{which}: rows overlap"):
        nld._append(refuse, params, t["q"], t["k_new"], t["v_new"], None, i32(2, 2), i32(2), (), OnGpu(bf16(T, H, D)), None,
                    None, nld.NLD_ROPE_HALF, None, None)


@pytest.mark.parametrize("rows,stride", [
    (bf16(T, H, D), H * D),
    (bf16(T, 3 * H, D)[:, H:2 * H], 3 * H * D),   # a slice of a projection
    (bf16(1, 3 * H, D)[:, :H], H * D),            # a single row has no stride
    (bf16(1, H, D).expand(1, H, D), H * D),
    (bf16(0, 3 * H, D)[:, :H], H * D),
])
def test_row_strides(rows, stride):
    assert nld._rows(OnGpu(rows), tuple(rows.shape), "k_new") == stride
