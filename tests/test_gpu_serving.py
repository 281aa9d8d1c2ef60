"""GPU parity of the operators behind the compressed rows (norm and rotation of queries and keys, cache append,
attention over a paged cache) against the formulas in 64 bits, where they can go wrong."""
import math

import pytest
import torch

from serving_reference import attend, check, norm_rotate, seen_mask

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _offsets(rows):
    return torch.tensor([0] + list(rows)).cumsum(0).int()


# ------------------------------------------------------------------------------ norm and rotation
ROPE = [
    # rows, heads, kv_heads, D, rotary_dim, axes, layout, dtype, norm
    (1, 4, 2, 128, 128, 1, "half", BF, True),
    (37, 32, 8, 128, 128, 3, "half", BF, True),
    (3, 1, 1, 8, 8, 1, "interleaved", F32, True),
    (5, 6, 2, 80, 32, 1, "half", F32, False),
    (5, 6, 2, 80, 32, 4, "interleaved", BF, True),
    (9, 3, 3, 72, 72, 3, "half", BF, False),          # units of 4 entries
    (9, 3, 1, 72, 24, 3, "interleaved", BF, True),
    (7, 2, 2, 256, 256, 2, "half", F32, True),
    (7, 2, 2, 256, 250, 1, "half", BF, True),         # single entries, two units a lane
    (6, 5, 1, 40, 10, 1, "interleaved", BF, True),
    (6, 5, 1, 40, 6, 1, "half", F32, True),
    (4, 7, 1, 64, 0, 1, "half", BF, True),            # the norm alone
    (2100, 3, 1, 64, 64, 1, "half", BF, True),        # more waves than the chip holds: one a row
]


@pytest.mark.parametrize("rows,heads,kv_heads,D,rot,axes,layout,dtype,norm", ROPE)
def test_norm_and_rotation(rows, heads, kv_heads, D, rot, axes, layout, dtype, norm):
    import paper_2605_07355_amd as ttf
    g = _gen(rows + D)
    qkv = (torch.randn((rows, heads + kv_heads, D), generator=g) * 3).to(dtype)
    pos = torch.randint(0, 1 << 20, (axes, rows), generator=g).int()
    if rows > 2:
        pos[:, 1] = 0
        pos[:, 2] = -5
    axis = (torch.arange(max(rot // 2, 1)) % axes).int()[:rot // 2] if axes > 1 else None
    freq = 10000.0 ** (-2.0 * torch.arange(rot // 2).double() / max(rot, 1))
    factor = 1.1 if rot else 1.0
    wq, wk = ((1 + 0.3 * torch.randn(D, generator=g)).to(dtype) if norm else None for _ in range(2))
    x = qkv.cuda()
    rope = ttf.TTFRope(freq.cuda(), None if axis is None else axis.cuda(), layout, factor) if rot else None
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    q, k = ttf.ttf_qk_norm_rope(x[:, :heads], x[:, heads:], pos.cuda(), rope, q_weight=cu(wq), k_weight=cu(wk), eps=1e-5)
    for got, part, w in ((q, qkv[:, :heads], wq), (k, qkv[:, heads:], wk)):
        want, slack = norm_rotate(part, w, 1e-5, pos, freq if rot else None, axis, layout, factor)
        check(got, want, slack, dtype)
    # in place, and one operand alone
    y = x.clone()
    ttf.ttf_qk_norm_rope(y[:, :heads], None, pos.cuda(), rope, q_weight=cu(wq), eps=1e-5, q_out=y[:, :heads])
    assert torch.equal(y[:, :heads], q) and torch.equal(y[:, heads:], x[:, heads:])
    ttf.ttf_qk_norm_rope(None, y[:, heads:], pos.cuda(), rope, k_weight=cu(wk), eps=1e-5, k_out=y[:, heads:])
    assert torch.equal(y[:, heads:], k)


def test_rotation_stays_inside_its_rows():
    """Rows outside row_offsets and everything between the heads stay as they were."""
    import paper_2605_07355_amd as ttf
    g = _gen(3)
    x = torch.randn((12, 6, 64), generator=g).to(BF).cuda()
    out = torch.full((12, 9, 64), 7.0, dtype=BF, device="cuda")
    rope = ttf.ttf_rope_table(64, 1e4)
    pos = torch.arange(12).int().cuda()
    offsets = torch.tensor([2, 5, 5, 9]).int().cuda()
    ttf.ttf_qk_norm_rope(x[:, :4], None, pos, rope, row_offsets=offsets, q_out=out[:, 2:6])
    whole, _ = ttf.ttf_qk_norm_rope(x[:, :4], None, pos, rope)
    assert torch.equal(out[2:9, 2:6], whole[2:9])
    out[2:9, 2:6] = 7.0
    assert bool((out == 7.0).all())


def test_zero_and_infinite_heads():
    import paper_2605_07355_amd as ttf
    x = torch.ones((3, 2, 64), dtype=F32)
    x[0, 0] = 0.0
    x[1, 1, 5] = math.inf
    x[2, 0, 5] = math.nan
    w = torch.ones(64)
    q, _ = ttf.ttf_qk_norm_rope(x.cuda(), None, torch.arange(3).int().cuda(), ttf.ttf_rope_table(64), q_weight=w.cuda(), eps=1e-6)
    q = q.cpu()
    assert bool((q[0, 0] == 0).all())
    assert bool(torch.isfinite(q[0, 1]).all()) and bool(torch.isfinite(q[1, 0]).all()) and bool(torch.isfinite(q[2, 1]).all())
    assert bool(torch.isnan(q[2, 0]).all())


# ------------------------------------------------------------------------------ the cache
def _cache(pages, page, kv_heads, D, dtype, heads_first, fill=math.nan):
    shape = (pages, kv_heads, page, D) if heads_first else (pages, page, kv_heads, D)
    k = torch.full(shape, fill, dtype=dtype)
    v = torch.full(shape, fill, dtype=dtype)
    return (k.transpose(1, 2), v.transpose(1, 2)) if heads_first else (k, v)


def _table(rows, cached, page, g, spare=2, extra=1):
    used = [-(-(r + max(c, 0)) // page) for r, c in zip(rows, cached)]
    width = max(used + [1]) + extra
    order = torch.randperm(sum(used) + spare, generator=g).int()
    table = torch.full((len(rows), width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(used) + spare


APPEND = [
    # rows of the sequences, cached, heads, kv_heads, D, rot, page, heads first, dtype, layout
    ([1], [0], 4, 1, 64, 64, 16, False, BF, "half"),
    ([1, 1, 1], [0, 31, 100], 32, 8, 128, 128, 16, False, BF, "half"),
    ([0, 5, 0, 17, 1], [3, 0, 9, 30, 47], 6, 2, 80, 32, 24, True, F32, "interleaved"),
    ([33, 1], [1, 7], 2, 2, 72, 24, 7, False, BF, "half"),
    ([1] * 70, list(range(70)), 2, 1, 64, 64, 8, True, BF, "half"),          # more sequences than lanes
    ([0] * 130 + [3], [0] * 131, 2, 1, 64, 10, 1, False, F32, "half"),       # one slot a page
]


@pytest.mark.parametrize("rows,cached,heads,kv_heads,D,rot,page,heads_first,dtype,layout", APPEND)
def test_append(rows, cached, heads, kv_heads, D, rot, page, heads_first, dtype, layout):
    import paper_2605_07355_amd as ttf
    g = _gen(len(rows) * D + page)
    n = sum(rows) + 3
    x = torch.randn((n, heads + 2 * kv_heads, D), generator=g).to(dtype)
    pos = torch.randint(0, 5000, (1, n), generator=g).int()
    wk = (1 + 0.3 * torch.randn(D, generator=g)).to(dtype)
    freq = 10000.0 ** (-2.0 * torch.arange(rot // 2).double() / rot)
    table, pages = _table(rows, cached, page, g)
    k0, v0 = _cache(pages, page, kv_heads, D, dtype, heads_first, fill=9.0)
    k1, v1 = k0.cuda(), v0.cuda()
    cache = ttf.TTFKVCache(k1, v1, table.cuda())
    xg = x.cuda()
    q_out = torch.full((n, heads, D), 9.0, dtype=dtype, device="cuda")
    ttf.ttf_cache_append(cache, xg[:, heads:heads + kv_heads], xg[:, heads + kv_heads:], _offsets(rows).cuda(),
                         torch.tensor(cached).int().cuda(), pos=pos.cuda(), rope=ttf.TTFRope(freq.cuda(), layout=layout),
                         k_weight=wk.cuda(), q=xg[:, :heads], q_out=q_out)
    want_q, slack = norm_rotate(x[:, :heads], None, 0, pos, freq, None, layout, 1.0)
    total = sum(rows)
    check(q_out[:total], want_q[:total], slack[:total], dtype, "q")
    assert bool((q_out[total:] == 9.0).all())
    want_k, slack = norm_rotate(x[:, heads:heads + kv_heads], wk, 1e-6, pos, freq, None, layout, 1.0)
    wk_all, wk_slack, wv_all = k0.double(), torch.zeros(k0.shape, dtype=torch.float64), v0.clone()
    i = 0
    for b, r in enumerate(rows):
        for j in range(r):
            t = cached[b] + j
            p = int(table[b, t // page])
            wk_all[p, t % page], wk_slack[p, t % page], wv_all[p, t % page] = want_k[i], slack[i], x[i, heads + kv_heads:]
            i += 1
    check(k1, wk_all, wk_slack, dtype, "k")
    assert torch.equal(v1.cpu(), wv_all)


def test_append_leaves_out_what_has_no_slot():
    """Pages that are not there, entries beyond the table, a negative length: nothing is written for them."""
    import paper_2605_07355_amd as ttf
    k, v = (t.cuda() for t in _cache(4, 16, 1, 64, BF, False, fill=9.0))
    table = torch.tensor([[0, -1], [4, 1], [2, 99], [-2147483648, 2147483647]]).int().cuda()
    rows, cached = [20, 20, 40, 33], [0, 0, 10, -1]
    x = torch.ones((sum(rows), 1, 64), dtype=BF, device="cuda")
    q = torch.ones((sum(rows), 2, 64), dtype=BF, device="cuda")
    q_out = torch.zeros_like(q)
    ttf.ttf_cache_append(ttf.TTFKVCache(k, v, table), x, x, _offsets(rows).cuda(), torch.tensor(cached).int().cuda(), q=q, q_out=q_out)
    want = torch.full((4, 16), 9.0)
    want[0, :] = 1.0                   # sequence 0: its first page only
    want[1, 0:4] = 1.0                 # sequence 1: entries 16..19
    want[2, 10:16] = 1.0               # sequence 2: entries 10..15
    assert torch.equal(k[:, :, 0, 0].float().cpu(), want) and torch.equal(v[:, :, 0, 63].float().cpu(), want)
    assert bool((q_out == 1).all())    # queries do not depend on the cache


# ------------------------------------------------------------------------------ attention
def _problem(rows, cached, heads, kv_heads, D, page, dtype, heads_first=False, seed=0, peak=2.0, slack_rows=0):
    """Queries, a cache whose slots hold NaN wherever no entry was put, and the entries by sequence."""
    g = _gen(seed + D + page)
    total = sum(rows)
    table, pages = _table(rows, cached, page, g)
    k, v = _cache(pages, page, kv_heads, D, dtype, heads_first)
    ks, vs = [], []
    for b, (r, c) in enumerate(zip(rows, cached)):
        n = r + c
        kb, vb = torch.randn((n, kv_heads, D), generator=g).to(dtype), (torch.randn((n, kv_heads, D), generator=g) + 0.3).to(dtype)
        t = torch.arange(n)
        p = table[b].long()[t // page] if n else t
        k[p, t % page], v[p, t % page] = kb, vb
        ks.append(kb)
        vs.append(vb)
    q = (peak * torch.randn((total + slack_rows, heads, D), generator=g)).to(dtype)
    return q, k, v, table, ks, vs


def _run_attention(q, k, v, table, rows, cached, causal=True, window=0, max_rows=None, scale=None, stream=None):
    import paper_2605_07355_amd as ttf
    out = torch.full_like(q, 5.0, device="cuda")
    lse = torch.full(q.shape[:2], 5.0, dtype=torch.float32, device="cuda")
    cache = ttf.TTFKVCache(k.cuda(), v.cuda(), table.cuda())
    ttf.ttf_paged_attention(q.cuda(), cache, _offsets(rows).cuda(), torch.tensor(cached).int().cuda(), max_rows=max_rows,
                            scale=scale, causal=causal, window=window, out=out, lse=lse)
    return out.cpu(), lse.cpu()


def _check_attention(out, lse, q, ks, vs, rows, cached, causal, window, dtype, scale=None, there=None):
    first = 0
    scale = q.shape[2] ** -0.5 if scale is None else scale
    for b, (r, c) in enumerate(zip(rows, cached)):
        n = r + c
        ok = torch.ones(n, dtype=torch.bool) if there is None else there[b]
        want, want_lse, slack, lse_slack = attend(q[first:first + r], ks[b], vs[b], seen_mask(r, c, n, causal, window, ok), scale)
        check(out[first:first + r], want, slack, dtype, f"sequence {b}")
        check(lse[first:first + r], want_lse, lse_slack, torch.float32, f"lse of sequence {b}")
        empty = want_lse == -math.inf
        assert torch.equal(lse[first:first + r] == -math.inf, empty) and bool((out[first:first + r][empty] == 0).all())
        first += r
    assert bool((out[first:] == 5.0).all()) and bool((lse[first:] == 5.0).all())     # rows behind the last sequence


ATTENTION = [
    # rows, cached, heads, kv_heads, D, page, dtype, causal, window, heads first
    ([1], [0], 4, 1, 64, 16, BF, True, 0, False),                        # one key
    ([1], [400], 32, 8, 128, 16, BF, True, 0, False),
    ([1, 1, 1, 0, 1], [0, 31, 32, 5, 700], 8, 2, 128, 64, BF, True, 0, False),
    ([3, 1, 2], [127, 128, 129], 8, 1, 128, 16, BF, True, 0, True),      # 24 columns
    ([1, 2], [100, 515], 7, 7, 72, 8, BF, True, 0, False),               # page of 8: keys looked up one by one
    ([5, 2], [63, 200], 6, 2, 80, 24, F32, False, 0, True),
    ([1, 4], [1, 90], 3, 3, 256, 7, F32, True, 0, False),
    ([2, 1], [90, 300], 8, 1, 256, 32, BF, True, 0, False),
    ([70, 9], [0, 200], 4, 2, 128, 16, BF, True, 0, False),              # several tiles
    ([130, 1, 33], [0, 65, 31], 8, 2, 64, 16, BF, True, 0, False),
    ([65, 40], [10, 0], 2, 2, 40, 48, F32, True, 0, False),
    ([20, 50], [0, 64], 5, 5, 200, 16, BF, False, 0, False),
    ([1, 3], [300, 257], 8, 2, 64, 16, BF, True, 40, False),             # windows
    ([90, 20], [11, 300], 4, 2, 128, 32, BF, True, 33, False),
    ([64, 2], [0, 100], 4, 4, 64, 16, F32, True, 1, False),              # only itself
    ([40, 9], [3, 70], 4, 1, 96, 16, BF, False, 17, False),
    ([1], [5000], 4, 1, 128, 16, BF, True, 0, False),                    # cut into many parts
    ([2, 1, 1], [3000, 1, 40], 2, 1, 64, 16, F32, True, 0, False),
]


@pytest.mark.parametrize("rows,cached,heads,kv_heads,D,page,dtype,causal,window,heads_first", ATTENTION)
def test_attention(rows, cached, heads, kv_heads, D, page, dtype, causal, window, heads_first):
    q, k, v, table, ks, vs = _problem(rows, cached, heads, kv_heads, D, page, dtype, heads_first, slack_rows=2)
    out, lse = _run_attention(q, k, v, table, rows, cached, causal, window, max_rows=max(rows))
    _check_attention(out, lse, q, ks, vs, rows, cached, causal, window, dtype)


@pytest.mark.parametrize("rows,cached,heads,D", [
    ([33, 0, 35, 40], [5000, 3, 5900, 6200], 64, 64),        # two rounds of parts
    ([34, 36, 33], [6100, 5500, 5800], 32, 256),
    ([34] + 69 * [1], [3000] + 69 * [20], 4, 128),           # more sequences than lanes
])
def test_attention_of_rows_in_many_parts(rows, cached, heads, D):
    q, k, v, table, ks, vs = _problem(rows, cached, heads, heads, D, 16, BF, slack_rows=1)
    out, lse = _run_attention(q, k, v, table, rows, cached, max_rows=max(rows))
    _check_attention(out, lse, q, ks, vs, rows, cached, True, 0, BF)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("max_rows", [1, 4, 8, 100, 1 << 20])
def test_attention_does_not_rely_on_max_rows(dtype, max_rows):
    rows, cached = [37, 1, 0, 12], [50, 300, 7, 0]
    q, k, v, table, ks, vs = _problem(rows, cached, 8, 2, 128, 16, dtype)
    out, lse = _run_attention(q, k, v, table, rows, cached, max_rows=max_rows)
    _check_attention(out, lse, q, ks, vs, rows, cached, True, 0, dtype)


@pytest.mark.parametrize("page", [16, 10])
@pytest.mark.parametrize("rows", [[1, 2], [50, 70]])
def test_attention_without_some_pages(rows, page):
    """Pages that are not there leave their keys out; rows that see none of the others get 0 and -inf."""
    cached = [100, 64]
    q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, 64, page, BF)
    table[0, 2], table[0, 3], table[1, :table.shape[1] - 1] = -7, k.shape[0], 1 << 30
    there = []
    for b, (r, c) in enumerate(zip(rows, cached)):
        p = table[b].long()[torch.arange(r + c) // page]
        there.append((p >= 0) & (p < k.shape[0]))
    out, lse = _run_attention(q, k, v, table, rows, cached, max_rows=max(rows))
    _check_attention(out, lse, q, ks, vs, rows, cached, True, 0, BF, there=there)
    assert bool((lse[rows[0]:] == -math.inf).all())


@pytest.mark.parametrize("heads,rows,max_rows", [(4, 40, 1), (4, 8, 8), (32, 60, 60)])
def test_offsets_that_decrease_stay_inside_the_buffers(heads, rows, max_rows):
    """More work than the grid holds, and notes of every kind in the workspace: the rows past `rows` and the guards stay."""
    import paper_2605_07355_amd as ttf
    batch, D, length = 40, 64, 4000
    g = _gen(3)
    table, pages = _table([rows], [length], 16, g)
    k, v = _cache(pages, 16, 4, D, BF, False, fill=0.5)
    table = table.repeat(batch, 1)
    offsets = torch.tensor([0 if b % 2 == 0 else rows for b in range(batch + 1)]).int()
    cached = torch.full((batch,), 10).int()
    cached[batch - 2:] = length
    cache = ttf.TTFKVCache(k.cuda(), v.cuda(), table.cuda())
    need = ttf.ttf_attention_workspace_size(rows, batch, heads, 4, D, max_rows=max_rows)
    for fill in (0, 1, 0x7f, 0x80, 0xff):
        buffer = torch.full((rows + 64, heads, D), 5.0, dtype=BF, device="cuda")
        lse = torch.full((rows + 64, heads), 5.0, device="cuda")
        ttf.ttf_paged_attention(torch.ones((rows, heads, D), dtype=BF, device="cuda"), cache, offsets.cuda(), cached.cuda(),
                                max_rows=max_rows, out=buffer[32:32 + rows], lse=lse[32:32 + rows],
                                workspace=torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        for x in (buffer, lse):
            assert bool((x[:32] == 5.0).all()) and bool((x[32 + rows:] == 5.0).all())


def test_attention_of_short_tables_and_odd_lengths():
    """Entries beyond the table are not there; a negative length sees nothing."""
    rows, cached = [2, 3, 1], [40, 20, 0]
    q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, 64, 16, BF)
    there = [torch.arange(r + c) < 32 for r, c in zip(rows, cached)]
    out, lse = _run_attention(q, k, v, table[:, :2].contiguous(), rows, cached)
    _check_attention(out, lse, q, ks, vs, rows, cached, True, 0, BF, there=there)
    out, lse = _run_attention(q, k, v, table, rows, [40, -1, -2147483648])
    assert bool((out[2:] == 0).all()) and bool((lse[2:] == -math.inf).all())
    _check_attention(out[:2], lse[:2], q[:2], ks[:1], vs[:1], [2], [40], True, 0, BF)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,heads", [([70, 6], 4), ([9, 6], 2), ([300, 6], 4)])
def test_what_a_row_does_not_see_does_not_reach_it(rows, heads, dtype):
    """NaN and infinities in keys and values ahead of a row and behind its window; weights of 0 times them are no 0."""
    cached = [40, 33]
    for window in (0, 24):
        q, k, v, table, ks, vs = _problem(rows, cached, heads, 2, 128, 16, dtype, seed=5)
        bad = 40 + rows[0] // 2                            # seen from the middle of the chunk on
        for s, (value, key) in ((bad, (math.inf, None)), (bad + 1, (math.nan, None)), (bad + 2, (-math.inf, math.nan)), (3, (math.nan, None))):
            if s == 3 and not window:
                continue
            p = int(table[0, s // 16])
            v[p, s % 16, :, 7] = value
            vs[0][s, :, 7] = value
            if key is not None:
                k[p, s % 16] = key
                ks[0][s] = key
        out, lse = _run_attention(q, k, v, table, rows, cached, window=window, max_rows=max(rows))
        first = 0
        for b, (r, c) in enumerate(zip(rows, cached)):
            seen = seen_mask(r, c, r + c, True, window, torch.ones(r + c, dtype=torch.bool))
            taints = torch.zeros(r, dtype=torch.bool) if b else seen[:, [s for s in (bad, bad + 1, bad + 2) if s < r + c] + [3] * bool(window)].any(1)
            clean = ~taints
            want, want_lse, slack, lse_slack = attend(q[first:first + r][clean], ks[b], vs[b], seen[clean], 128 ** -0.5)
            check(out[first:first + r][clean], want, slack, dtype, f"sequence {b}")
            check(lse[first:first + r][clean], want_lse, lse_slack, F32, f"lse {b}")
            if b == 0:
                assert bool(clean.any()) and bool(taints.any())
                assert not bool(torch.isfinite(out[:r][taints][:, :, 7]).any())
            first += r


def test_attention_large_and_small_scores():
    """Scores far apart, all alike, and so large that only a maximum taken off first keeps them finite."""
    rows, cached = [3, 40], [300, 10]
    for peak, scale in ((40.0, None), (1e-4, None), (3.0, -0.2), (3.0, 0.0)):
        q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, 64, 16, BF, peak=peak)
        out, lse = _run_attention(q, k, v, table, rows, cached, scale=scale, max_rows=40)
        _check_attention(out, lse, q, ks, vs, rows, cached, True, 0, BF, scale=scale)


def test_attention_repeats_bit_for_bit_and_in_place():
    import paper_2605_07355_amd as ttf
    rows, cached = [1, 1, 5], [2000, 30, 700]
    q, k, v, table, _, _ = _problem(rows, cached, 8, 2, 128, 16, BF)
    first = _run_attention(q, k, v, table, rows, cached)
    for _ in range(3):
        again = _run_attention(q, k, v, table, rows, cached)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    qg = q.cuda()
    ttf.ttf_paged_attention(qg, ttf.TTFKVCache(k.cuda(), v.cuda(), table.cuda()), _offsets(rows).cuda(),
                            torch.tensor(cached).int().cuda(), out=qg)
    assert torch.equal(qg.cpu(), first[0])
