"""GPU: rows of the tcgen05 kernel over the 4-bit cache whose terms lie far below
their group's reference, over so many tokens that small terms add up.

Two million tokens, made of a few pages that the table repeats. A token has K =
c and V = v in every channel; rows with weights 1 and -1 see it at the scores c
sqrt(D) and -c sqrt(D). Expected values come from the counts of equal tokens.

Bars. lse: a lane adds 2^14 equal terms one by one in fp32, at most 2^-24 of
the sum each: 2^-10, and 2^-14 for the scores themselves. Outputs: the value
product adds 2^17 equal parts, each at most 2^-23 of the sum: 2^-6, and three
roundings to bf16 (a term, an output, a scale): below 2^-5 of the output.
"""
import numpy as np
import pytest
import torch

import kv4_ref as ref
from paper_2607_05722_gb300 import nld
from test_gpu_kv4 import VER, _lib, f32_of, i32  # noqa: F401

pytestmark = pytest.mark.gpu
D, P, PAGES = 64, 256, 8192
HEADS = 20                       # one KV head: 20 rows, more than the register kernel takes


def page_of(tokens):
    """A page's records for its 256 tokens (c, v)."""
    page = np.zeros((P // 16, 20 * D), np.uint8)
    c = ref.to_bf16_bits(np.array([t[0] for t in tokens])).reshape(-1, 16)
    v = ref.to_bf16_bits(np.array([t[1] for t in tokens])).reshape(-1, 16)
    for r in range(P // 16):
        ks = np.zeros((16, D // 32, 2), np.uint16)
        ks[:, :, 1] = c[r][:, None]
        vs = np.zeros((D // 32, 2, 16), np.uint16)
        vs[:, 1] = v[r]
        page[r, 16 * D:18 * D] = ks.view(np.uint8).ravel()
        page[r, 18 * D:] = vs.view(np.uint8).ravel()
    return page


def run(pages, order, batch):
    pool = torch.from_numpy(np.stack([page_of(p) for p in pages])[:, None]).cuda()
    params = nld.make_params(batch, HEADS, 1, D, P, len(pages), PAGES)
    table = i32(np.tile(np.asarray(order, np.int32), (batch, 1)))
    w = np.where(np.arange(HEADS) % 2 == 0, 1.0, -1.0)
    q = torch.from_numpy(w).cuda().to(torch.bfloat16)[None, None, :, None].expand(batch, 1, HEADS, D).contiguous()
    out, lse = torch.empty_like(q), torch.empty(batch, HEADS, 1, device="cuda")
    ws = torch.empty(max(16, nld.nld_block_attn_kv4_workspace_size(params, 1)), dtype=torch.uint8, device="cuda")
    nld.nld_block_attn_kv4(params, q, pool, table, i32([PAGES * P - 1] * batch), 1, VER, out, lse, ws)

    kinds, counts = np.unique(np.asarray(order), return_counts=True)
    c, v, n = [], [], []
    for kind, count in zip(kinds, counts):
        for token in sorted(set(pages[kind])):
            c.append(token[0])
            v.append(token[1])
            n.append(count * pages[kind].count(token))
    c, v, n = (np.asarray(x, np.float64) for x in (c, v, n))
    c = f32_of(ref.to_bf16_bits(c)).astype(np.float64)
    s = w[:, None] * c * np.sqrt(D)
    top = s.max(-1, keepdims=True)
    p = n * np.exp(s - top)
    want_lse, want = top[:, 0] + np.log(p.sum(-1)), (p * v).sum(-1) / p.sum(-1)
    got = out.double().cpu().numpy()[:, 0]
    assert np.all(np.abs(got - want[None, :, None]) <= 2.0 ** -5 * np.abs(want)[None, :, None] + 1e-9)
    assert np.all(np.abs(lse.double().cpu().numpy()[:, :, 0] - want_lse) <= 2.0 ** -10 + 2.0 ** -14)


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def test_small_terms_of_a_far_row():
    """A whole unit per CTA: for the rows of weight -1 all tokens but one are 2^127
    below the group's reference and that one 2^99; together they weigh 0.9% of it."""
    plain, loud = (3.5625, 1.0), (1.1484375, 0.0)
    pages = [[plain] * P, [plain] * 7 + [loud] + [plain] * (P - 8)]
    run(pages, [0] * 4000 + [1] + [0] * (PAGES - 4001), sms())


def test_far_part_of_a_cut_row():
    """Two CTAs to a unit, whose references lie 2^127 apart: for the rows of weight
    -1 the first half's tokens reach 2 to the reference, the second half's one loud
    token is 2^99 below its own; the first half weighs 0.7% of it."""
    near, far = (-3.96875, 1.0), (11.0625, 0.0)
    pages = [[near] * P, [(0.0, 1.0)] + [near] * (P - 1), [(0.0, 0.0)] * P,
             [far, (-6.3125, 0.0)] + [(0.0, 0.0)] * (P - 2)]
    half = PAGES // 2
    run(pages, [1] + [0] * (half - 1) + [3] + [2] * (half - 1), sms() // 2)
