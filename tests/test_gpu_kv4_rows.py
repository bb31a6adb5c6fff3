"""GPU: row offsets (cu_tokens) that leave rows to nobody, or claim rows twice:
every entry point that takes them flags them, and touches nothing of the rows
that belong to no sequence."""
import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2607_05722_gb300 import nld
from test_gpu_kv4 import Append, _lib, i32  # noqa: F401

pytestmark = pytest.mark.gpu
FLAG = nld.NLD_DEVERR_PREFIX_RANGE
ENTRIES = ["append", "append without queries", "append_kv4", "append_kv4 without queries", "read"]


def call(entry, c, cu):
    """One call over the rows of c with the offsets cu; the error word, and the
    rows that the read-back wrote."""
    queries = "without" not in entry
    q_out = torch.zeros(len(c.b), c.Hq, c.D, dtype=torch.bfloat16, device="cuda")
    head = (c.params, c.q if queries else None, c.k, c.v, None, i32(c.table), i32(c.lens))
    tail = dict(q_out=q_out if queries else None, cu_tokens=i32(cu))
    pool = torch.from_numpy(ref.random_pool(np.random.default_rng(3), nld.kv4_pages_shape(c.params))).cuda()
    written = None
    if entry == "read":
        out = [torch.full((len(c.b), c.Hkv, c.D), 333.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        nld.nld_kv4_read(c.params, pool, i32(c.table), i32(c.lens), *out, cu_tokens=i32(cu))
        written = (out[0] != 333.0).any(-1).any(-1).tolist()
    elif entry.startswith("append_kv4"):
        nld.nld_rope_append_kv4(*head, pool, **tail)
    else:
        pages = [torch.zeros(c.num_pages, c.Hkv, c.P, c.D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        nld.nld_rope_append(*head, *pages, **tail)
    return nld.nld_device_error(clear=True), written


@pytest.mark.parametrize("entry", ENTRIES)
@pytest.mark.parametrize("cu,rows", [
    ((0, 2, 5), [0, 1, 2, 3, 4]), ((0, 0, 5), [0, 1, 2, 3, 4]), ((0, 5, 5), [0, 1, 2, 3, 4]),
    ((1, 2, 5), [1, 2, 3, 4]),       # row 0 belongs to nobody
    ((0, 2, 4), [0, 1, 2, 3]),       # row 4
    ((0, 0, 0), []),                 # none does
    ((-1, 2, 5), [0, 1, 2, 3, 4]),
    ((0, 6, 5), [0, 1, 2, 3, 4]),    # past the end, then back
    ((0, 2, 6), [0, 1, 2, 3, 4]),
])
def test_uncovered_rows_are_flagged(entry, cu, rows):
    c = Append(9, (4, 1, 64), 16, [4, 20], [3, 2], 0, "half")
    c.table = np.full((2, 3), 0, np.int32) + np.arange(6, dtype=np.int32).reshape(2, 3)  # room for 5 rows each
    c.num_pages, c.max_pages = 6, 3
    c.params = nld.make_params(2, 4, 1, 64, 16, 6, 3)
    err, written = call(entry, c, cu)
    assert err == (0 if cu[0] == 0 and cu[2] == 5 and cu[1] <= 5 else FLAG)
    if written is not None:
        assert [r for r in range(5) if written[r]] == rows


@pytest.mark.parametrize("entry", ENTRIES)
@pytest.mark.parametrize("at", [0, 1, 137, 699, 700])
def test_one_wrong_offset_among_many(entry, at):
    """700 sequences of 4 rows, one offset past its neighbour."""
    c = Append(10, (4, 1, 64), 16, [0] * 700, [4] * 700, 0, "half")
    assert call(entry, c, c.cu)[0] == 0
    cu = c.cu.copy()
    cu[at] += 5 if at < 700 else -1
    assert call(entry, c, cu)[0] == FLAG
