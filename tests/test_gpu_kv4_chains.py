"""GPU: calls back to back on one stream read what the calls before them wrote.

Every kernel may start while its predecessor is still running and has to wait
before its first load of data that an earlier kernel may produce. Here the
predecessors are long (an append of many rows) and their last products small
(the lengths, advanced in place), so that a load made too early sees old values.
"""
import pytest
import torch

from paper_2607_05722_gb300 import nld
from test_gpu_kv4 import VER, Append, _lib, i32  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,bl", [((8, 2, 64), 1), ((16, 2, 128), 8), ((32, 8, 128), 1), ((40, 8, 128), 16)])
def test_calls_see_their_predecessors(heads, bl):
    new = [3000, 1, 2500, 800]
    c = Append(81, heads, 16, [5, 0, 40, 700], [n + 3 * bl for n in new], 64, "half")
    B, Hq, Hkv, D = 4, *heads
    x = torch.randn(sum(new), Hq + 2 * Hkv, D, generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    y = torch.randn(3, B * bl, Hq + 2 * Hkv, D, generator=torch.Generator("cuda").manual_seed(2), device="cuda").bfloat16()
    cu = i32([0, 3000, 3001, 5501, 6301])
    table, rope = i32(c.table), c.rope_dev()
    parts = lambda t: (t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:])  # noqa: E731

    def run(wait):
        lens = i32(c.lens)
        pool = torch.zeros(nld.kv4_pages_shape(c.params), dtype=torch.uint8, device="cuda")
        pages = [torch.zeros(c.num_pages, Hkv, 16, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        q_all = torch.empty(sum(new), Hq, D, dtype=torch.bfloat16, device="cuda")
        q = [torch.empty(B * bl, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        rows = [torch.empty(B * bl, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(6)]
        out = [torch.empty(B, bl, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(6)]
        ws = torch.empty(max(16, nld.nld_block_attn_kv4_workspace_size(c.params, bl)), dtype=torch.uint8, device="cuda")
        work = nld.alloc_workspace(c.params, bl)
        torch.cuda.synchronize()

        def done():
            if wait:
                torch.cuda.synchronize()

        _, k, v = parts(x)
        nld.nld_rope_append(c.params, None, k, v, rope, table, lens, *pages, cu_tokens=cu)
        done()
        nld.nld_rope_append_kv4(c.params, x[:, :Hq], k, v, rope, table, lens, pool, q_all, cu_tokens=cu, new_lens=lens)
        done()
        for i in range(3):
            qi, ki, vi = parts(y[i])
            nld.nld_rope_append_kv4(c.params, qi, ki, vi, rope, table, lens, pool, q[i])
            done()
            nld.nld_block_attn_kv4(c.params, q[i].view(out[i].shape), pool, table, lens, bl, VER, out[i], None, ws)
            done()
            nld.nld_kv4_read(c.params, pool, table, lens, rows[2 * i], rows[2 * i + 1])
            done()
            # the rows read back go into the bf16 cache, which then advances with the other
            nld.nld_rope_append(c.params, None, rows[2 * i], rows[2 * i + 1], None, table, lens, *pages)
            done()
            nld.nld_block_attn(c.params, q[i].view(out[i].shape), *pages, table, lens, bl, VER, out[3 + i], None, work)
            done()
            nld.nld_rope_append(c.params, None, rows[2 * i], rows[2 * i + 1], None, table, lens, *pages, new_lens=lens)
            done()
        torch.cuda.synchronize()
        return [lens, pool, *pages, q_all, *q, *rows, *out]

    want = run(True)
    assert want[0].tolist() == [5 + 3000 + 3 * bl, 1 + 3 * bl, 40 + 2500 + 3 * bl, 700 + 800 + 3 * bl]
    for _ in range(5):
        for a, b in zip(run(False), want):
            assert torch.equal(a, b)
