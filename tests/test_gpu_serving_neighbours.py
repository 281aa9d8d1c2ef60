"""Attention where every wave of a workgroup walks along a key head of its own: many long contexts, slots first.  Sequences
share the pages of a small pool, so that the inputs stay small."""
import math

import pytest
import torch

from serving_reference import attend, check, seen_mask
from test_gpu_serving import BF, F32, _offsets

pytestmark = pytest.mark.gpu


def _turns_of_a_part(rows, cached, heads, kv_heads, D, dtype, window):
    """Turns of a part as the kernel for few rows deals them out; from 8 on, and with a multiple of four key heads, waves have heads
    of their own."""
    group, block = heads // kv_heads, 32 if dtype == BF else 16
    pairs = max(rows) * group
    tiles = 1 if pairs <= 16 else 2
    assert pairs <= 32 and (dtype == F32 or pairs <= 16 or D <= 128)      # (the kernel for few rows)
    if D > 128 and dtype == F32:
        tiles = 1
    columns, target = min(pairs, 16 * tiles), 2048 // tiles
    total = 0
    for r, c in zip(rows, cached):
        begin = (c - window + 1) // 32 * 32 if window and c >= window else 0
        total += -(-r * group // columns) * -(-(r + c - begin) // block)
    return math.ceil(total * kv_heads / (4 * target))


CASES = [
    # sequences, rows at most, cached at most, heads, kv_heads, D, page, dtype, causal, window, holes
    (70, 1, 4600, 8, 8, 128, 16, BF, True, 0, False),
    (70, 1, 4600, 32, 8, 128, 64, BF, True, 0, True),
    (70, 3, 4600, 32, 4, 128, 16, BF, True, 0, False),       # 24 columns
    (70, 3, 4600, 32, 4, 128, 24, BF, False, 0, True),       # and keys looked up one by one
    (66, 2, 4900, 8, 8, 72, 16, BF, True, 0, False),         # heads shorter than the kernel's
    (66, 2, 4900, 16, 8, 80, 24, BF, True, 0, True),
    (66, 2, 9000, 8, 8, 64, 16, BF, True, 4700, False),      # a long window
    (66, 2, 9000, 8, 8, 24, 40, BF, False, 4700, True),
    (66, 1, 4900, 8, 8, 256, 32, BF, True, 0, True),
    (40, 2, 4200, 8, 8, 128, 16, F32, True, 0, True),
    (40, 2, 4200, 8, 8, 64, 24, F32, False, 0, False),
    (40, 5, 4200, 16, 4, 64, 16, F32, True, 0, False),       # 20 columns
    (40, 2, 7500, 8, 8, 200, 16, F32, True, 4000, False),
]


@pytest.mark.parametrize("bad", [False, True])
@pytest.mark.parametrize("B,most,context,heads,kv_heads,D,page,dtype,causal,window,holes", CASES)
def test_waves_with_heads_of_their_own(B, most, context, heads, kv_heads, D, page, dtype, causal, window, holes, bad):
    """`bad`: an infinite and a NaN value that only later rows of a sequence see, and one behind its end."""
    import paper_2605_07355_amd as ttf
    g = torch.Generator().manual_seed(B + D + page)
    rows = [most if b % 9 == 0 else 1 + b % most for b in range(B)]
    cached = [context - 13 * b for b in range(B)]
    assert kv_heads % 4 == 0 and _turns_of_a_part(rows, cached, heads, kv_heads, D, dtype, window) >= 8
    pool, width = 120, -(-(context + most) // page) + 1
    k, v = torch.randn((pool, page, kv_heads, D), generator=g).to(dtype), (torch.randn((pool, page, kv_heads, D), generator=g) + 0.3).to(dtype)
    table = torch.randint(2, pool, (B, width), generator=g).int()
    table[0, -2:] = torch.tensor([0, 1])                     # the last pages of sequence 0 are its own
    if holes:
        table[:, 5:width - 2:11], table[3, :width - 3] = -1, pool
    if bad:
        last = cached[0] + rows[0] - 1
        for u, value in ((last, math.nan), (last - 1, math.inf), (last + 1, math.nan)):
            if u > cached[0] or u == last + 1:
                v[int(table[0, u // page]), u % page, :, 5] = value
    q = (2 * torch.randn((sum(rows), heads, D), generator=g)).to(dtype)
    out, lse = torch.full_like(q, 5.0, device="cuda"), torch.full((sum(rows), heads), 5.0, device="cuda")
    ttf.ttf_paged_attention(q.cuda(), ttf.TTFKVCache(k.cuda(), v.cuda(), table.cuda()), _offsets(rows).cuda(),
                            torch.tensor(cached).int().cuda(), max_rows=most, causal=causal, window=window, out=out, lse=lse)
    out, lse, at = out.cpu(), lse.cpu(), _offsets(rows).tolist()
    for b in (0, 1, 3, B // 2, B - 1):
        n, r = rows[b] + cached[b], slice(at[b], at[b + 1])
        u = torch.arange(n)
        pages = table[b].long()[u // page]
        there = (pages >= 0) & (pages < pool)
        ks, vs = (t[pages.clamp(0, pool - 1), u % page] for t in (k, v))
        seen = seen_mask(rows[b], cached[b], n, causal, window, there)
        want, want_lse, slack, lse_slack = attend(q[r], ks, vs, seen, D ** -0.5)
        if bad and b == 0 and most > 1 and causal:           # the first row sees neither, the last both
            assert bool(torch.isfinite(want[0]).all()) and not bool(torch.isfinite(want[-1, :, 5]).any())
        check(out[r], want, slack, dtype, f"sequence {b}")
        check(lse[r], want_lse, lse_slack, F32, f"lse of sequence {b}")
    if not bad:
        assert bool(torch.isfinite(out).all())
