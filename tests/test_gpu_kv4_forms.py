"""GPU: documented forms of the 4-bit cache's operators: explicit positions into
the cache, the prefix-ready flag, and capture in a graph."""
import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2607_05722_gb300 import nld
from test_gpu_kv4 import DIFF, VER, Append, Attn, _lib, bits_to_bf16, f32_of, i32, ref_append  # noqa: F401

pytestmark = pytest.mark.gpu


SHORT, MANY = ([5, 0, 77], [13, 1, 40]), ([0, 3], [1300, 1400])  # many: a warp per row


@pytest.mark.parametrize("heads,rot,style,rows", [
    ((4, 1, 64), 64, "half", SHORT), ((16, 2, 64), 32, "interleaved", SHORT), ((12, 4, 128), 64, "half", SHORT),
    ((12, 4, 128), 128, "interleaved", SHORT), ((32, 8, 128), 128, "half", SHORT), ((12, 4, 128), 16, "half", SHORT),
    ((4, 1, 64), 32, "interleaved", MANY), ((5, 1, 128), 128, "half", MANY),
])
def test_positions_into_the_4bit_cache(heads, rot, style, rows):
    """Rows at positions of their own: q and K against the exact rotation (K as
    the bf16 append leaves it, whose bar is the rotation's), codes bit for bit."""
    lens, new = rows
    c = Append(71, heads, 32, lens, new, rot, style, positions=True)
    assert not np.array_equal(c.pos, c.at)
    q_out = torch.empty(sum(new), c.Hq, c.D, dtype=torch.bfloat16, device="cuda")
    pool = torch.zeros(nld.kv4_pages_shape(c.params), dtype=torch.uint8, device="cuda")
    nld.nld_rope_append_kv4(c.params, c.q, c.k, c.v, c.rope_dev(), i32(c.table), i32(lens), pool, q_out, **c.args())
    want, bar = c.rotated(0, c.Hq)
    assert np.all(np.abs(q_out.float().cpu().numpy() - want) <= bar)
    pages = [torch.zeros(c.num_pages, c.Hkv, 32, c.D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    nld.nld_rope_append(c.params, None, c.k, c.v, c.rope_dev(), i32(c.table), i32(lens), *pages, **c.args())
    k = pages[0].float().cpu().numpy()[c.table[c.b, c.at // 32], :, c.at % 32]
    want, bar = c.rotated(c.Hq, c.Hq + c.Hkv)
    assert np.all(np.abs(k - want) <= bar)
    want = ref_append(c, np.zeros(tuple(pool.shape), np.uint8), k, f32_of(c.bits[:, c.Hq + c.Hkv:]))
    assert np.array_equal(pool.cpu().numpy(), want)


@pytest.mark.parametrize("heads,bl", [((8, 2, 64), 1), ((16, 2, 128), 2), ((32, 8, 128), 16), ((40, 8, 128), 31)])
def test_prefix_ready_changes_nothing(heads, bl):
    c = Attn(72, heads, 16, [700, 0, 33], bl)
    for mode in (DIFF, VER):
        c.params.flags = 0
        a = c.run(mode)
        c.params.flags = nld.NLD_ATTN_PREFIX_READY
        b = c.run(mode)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("heads,bl", [((8, 2, 64), 1), ((16, 2, 128), 8), ((40, 8, 128), 16)])
def test_graph_replays(heads, bl):
    """A step of appends, read-back and attention captured once: every replay
    takes the rows and lengths that lie there by then."""
    B, steps = 3, 4
    c = Append(73, heads, 16, [40, 0, 100], [bl * steps] * B, 64, "half")
    T = B * bl
    table, rope = i32(c.table), c.rope_dev()
    rng = np.random.default_rng(5)
    start = ref.random_pool(rng, nld.kv4_pages_shape(c.params))
    rows = [torch.randn(T, c.Hq + 2 * c.Hkv, c.D, generator=torch.Generator("cuda").manual_seed(s), device="cuda").bfloat16()
            for s in range(steps)]

    def new_state():
        kv16 = (c.num_pages, c.Hkv, 16, c.D)
        s = dict(pool=torch.from_numpy(start).cuda(), lens=i32(c.lens), x=rows[0].clone(),
                 q=torch.empty(T, c.Hq, c.D, dtype=torch.bfloat16, device="cuda"),
                 k=[torch.empty(T, c.Hkv, c.D, dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                 pages=[torch.zeros(kv16, dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                 out=torch.empty(B, bl, c.Hq, c.D, dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty(B, c.Hq, bl, device="cuda"))
        n = nld.nld_block_attn_kv4_workspace_size(c.params, bl)
        s["ws"] = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")
        return s

    def step(s):
        q, k, v = s["x"][:, :c.Hq], s["x"][:, c.Hq:c.Hq + c.Hkv], s["x"][:, c.Hq + c.Hkv:]
        nld.nld_rope_append_kv4(c.params, q, k, v, rope, table, s["lens"], s["pool"], s["q"])
        nld.nld_kv4_read(c.params, s["pool"], table, s["lens"], *s["k"])
        nld.nld_rope_append(c.params, None, *s["k"], None, table, s["lens"], *s["pages"])
        nld.nld_block_attn_kv4(c.params, s["q"].view(s["out"].shape), s["pool"], table, s["lens"], bl, VER, s["out"], s["lse"], s["ws"])
        nld.nld_rope_append_kv4(c.params, None, k, v, rope, table, s["lens"], s["pool"], new_lens=s["lens"])  # advances

    def trace(s, once):
        got = []
        for x in rows:
            s["x"].copy_(x)
            once()
            got.append([t.clone() for t in (s["out"], s["lse"], s["lens"], s["pool"], *s["k"], *s["pages"])])
        return got

    eager = new_state()
    want = trace(eager, lambda: step(eager))
    s = new_state()
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()  # the state comes from the default stream
    with torch.cuda.stream(stream):
        step(s)  # (loads the kernels; undone below)
    torch.cuda.synchronize()
    fresh = new_state()
    for key in ("pool", "lens"):
        s[key].copy_(fresh[key])
    for t in s["pages"]:
        t.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(s)
    for a, b in zip(trace(s, graph.replay), want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert s["lens"].tolist() == [40 + bl * steps, bl * steps, 100 + bl * steps]
