"""The operators behind the compressed rows at the edges of what they accept."""
import math

import pytest
import torch

from serving_reference import attend, check, norm_rotate, seen_mask
from test_gpu_serving import BF, F32, _cache, _check_attention, _offsets, _problem, _run_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,heads_first", [(16, False), (16, True), (7, False)])
@pytest.mark.parametrize("D,dtype", [(8, BF), (16, BF), (24, BF), (8, F32), (24, F32)])
@pytest.mark.parametrize("rows", [[1, 2], [3, 40]])
def test_attention_of_short_heads(rows, D, dtype, page, heads_first):
    """Heads shorter than the 64 bytes that four lanes read side by side."""
    cached = [60, 11]
    q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, D, page, dtype, heads_first)
    out, lse = _run_attention(q, k, v, table, rows, cached, max_rows=max(rows))
    _check_attention(out, lse, q, ks, vs, rows, cached, True, 0, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [[3], [100, 1]])
@pytest.mark.parametrize("page", [1, 16])
def test_windows_behind_the_end_of_the_table(rows, page, dtype):
    """`cached` of up to 2^31 - 1, and windows that begin where the table has long ended: no entry is seen."""
    import paper_2605_07355_amd as ttf
    k, v = (t.cuda() for t in _cache(9, page, 2, 64, dtype, False, fill=1.0))
    table = torch.zeros((len(rows), 100), dtype=torch.int32, device="cuda")
    q = torch.ones((sum(rows), 4, 64), dtype=dtype, device="cuda")
    for cached in (2 ** 31 - 1, 2 ** 31 - 40, 10 ** 6):
        for window in (1, 33):
            lse = torch.zeros((sum(rows), 4), device="cuda")
            have = torch.full((len(rows),), cached, dtype=torch.int32, device="cuda")
            out = ttf.ttf_paged_attention(q, ttf.TTFKVCache(k, v, table), _offsets(rows).cuda(), have, window=window, lse=lse)
            assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_a_cache_whose_page_table_grows():
    """The table is replaced by a wider one between calls; the old one's memory holds other numbers by then."""
    import paper_2605_07355_amd as ttf
    rows, cached = [2, 1], [200, 77]
    q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, 64, 16, BF)
    cache = ttf.TTFKVCache(k.cuda(), v.cuda(), table[:, :1].contiguous().cuda())
    new = torch.randn((3, 2, 64), generator=torch.Generator().manual_seed(2)).to(BF)
    old, cache.page_table = cache.page_table, table.cuda()
    old.fill_(-1)
    have, offsets = torch.tensor(cached).int().cuda(), _offsets(rows).cuda()
    ttf.ttf_cache_append(cache, new.cuda(), new.cuda(), offsets, have)
    first = 0
    for b, (r, c) in enumerate(zip(rows, cached)):
        ks[b][c:] = vs[b][c:] = new[first:first + r]
        first += r
    out, lse = torch.full_like(q, 5.0, device="cuda"), torch.full((3, 4), 5.0, device="cuda")
    ttf.ttf_paged_attention(q.cuda(), cache, offsets, have, out=out, lse=lse)
    _check_attention(out.cpu(), lse.cpu(), q, ks, vs, rows, cached, True, 0, BF)


@pytest.mark.parametrize("heads,kv_heads,D,dtype", [(32, 8, 128, BF), (16, 4, 256, BF), (8, 4, 64, F32)])
def test_one_workspace_for_a_large_chunk_and_then_small_ones(heads, kv_heads, D, dtype):
    import paper_2605_07355_amd as ttf
    work = torch.zeros(ttf.ttf_attention_workspace_size(600, 3, heads, kv_heads, D, dtype, max_rows=400), dtype=torch.uint8, device="cuda")
    for rows, cached in (([400, 3, 197], [100, 3000, 20]), ([1, 1, 2], [900, 3000, 20]), ([1], [2500]), ([8, 5], [300, 1])):
        q, k, v, table, ks, vs = _problem(rows, cached, heads, kv_heads, D, 16, dtype)
        cache, have = ttf.TTFKVCache(k.cuda(), v.cuda(), table.cuda()), torch.tensor(cached).int().cuda()
        out = ttf.ttf_paged_attention(q.cuda(), cache, _offsets(rows).cuda(), have, max_rows=max(rows), workspace=work)
        own = ttf.ttf_paged_attention(q.cuda(), cache, _offsets(rows).cuda(), have, max_rows=max(rows))
        assert torch.equal(out, own) and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("rows,cached,low,bad", [
    ([1], [300], range(200), 40),              # not cut: waves join
    ([1], [6000], range(5000), 70),            # cut into parts
    ([20], [30], range(45), 40),               # seen from the middle of the chunk on
    ([20], [30], range(36, 50), 40),
    ([60, 1], [5000, 9], range(4000), 70),
    ([200], [100], range(200), 150),
    ([200], [100], range(101, 300), 150),
])
def test_a_value_of_tiny_weight_is_not_lost(rows, cached, low, bad, value, dtype):
    """Weights of e^-512 are 0 in 32 bits; an infinite or NaN value that a row sees reaches it all the same."""
    q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, 64, 16, dtype, peak=0.05)
    q[:, :, 0] = 16.0
    for b, n in enumerate(r + c for r, c in zip(rows, cached)):
        t = torch.arange(n)
        ks[b][:, :, 0] = torch.where((t >= low.start) & (t < low.stop), -16.0, 16.0)[:, None].to(dtype)
        if b == 0:
            vs[b][bad, :, 7] = value
        page = table[b].long()[t // 16]
        k[page, t % 16], v[page, t % 16] = ks[b], vs[b]
    out, lse = _run_attention(q, k, v, table, rows, cached, max_rows=max(rows), scale=1.0)
    first = 0
    for b, (r, c) in enumerate(zip(rows, cached)):
        seen = seen_mask(r, c, r + c, True, 0, torch.ones(r + c, dtype=torch.bool))
        for x in (range(r) if r < 30 else (0, 1, bad - c - 1, bad - c, r // 2, r - 1)):
            if not 0 <= x < r:
                continue
            want, want_lse, slack, lse_slack = attend(q[first + x:first + x + 1], ks[b], vs[b], seen[x:x + 1], 1.0)
            assert bool(torch.isfinite(want[..., 7]).all()) != bool(b == 0 and seen[x, bad])
            check(out[first + x:first + x + 1], want, slack, dtype, f"row {x}")
            check(lse[first + x:first + x + 1], want_lse, lse_slack, F32, "lse")
        first += r


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("factor", [1.0, 1.25])
def test_sines_and_cosines_are_rounded_once(layout, factor):
    """Pairs (1, 0) turn into (c, s): within half a step of fp32, and the error that the angle has in 64 bits."""
    import paper_2605_07355_amd as ttf
    rows, R = 4000, 128
    g = torch.Generator().manual_seed(9)
    pos = torch.randint(-(1 << 20), 1 << 20, (1, rows), generator=g).int()
    freq = 10000.0 ** (-2.0 * torch.arange(R // 2).double() / R)
    x = torch.zeros((rows, 1, R))
    first, second = (slice(0, R // 2), slice(R // 2, R)) if layout == "half" else (slice(0, R, 2), slice(1, R, 2))
    x[..., first] = 1.0
    out, _ = ttf.ttf_qk_norm_rope(x.cuda(), None, pos.cuda(), ttf.TTFRope(freq.cuda(), layout=layout, attention_factor=factor))
    out = out.cpu().double()
    theta = pos[0].double()[:, None] * freq
    # 64 bits: 1 / 2 pi, its product with the frequency, that with the position, each rounded, and sine and cosine themselves; here the product
    slack = factor * 2.0 ** -53 * (4 * theta.abs() + 4)
    for got, want in ((out[:, 0, first], factor * torch.cos(theta)), (out[:, 0, second], factor * torch.sin(theta))):
        past = ((got - want).abs() - 2.0 ** -24 * (want.abs() + slack) - slack).max().item()
        assert past <= 0


@pytest.mark.parametrize("D,rot,layout", [(128, 128, "half"), (80, 32, "interleaved"), (72, 10, "half")])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_norms_of_heads_whose_squares_leave_the_range(D, rot, layout, dtype):
    """Squares that overflow, or that all underflow where eps does not cover them, beside ordinary heads."""
    import paper_2605_07355_amd as ttf
    g = torch.Generator().manual_seed(D)
    sizes = torch.tensor([1.0, 1e25, 1e-30, 3e36, 1e-37, 1e19, 1e-18, 1e18, 1e-20])
    x = torch.randn((9, 3, D), generator=g) * sizes[:, None, None]
    x[:, 1] = torch.randn((9, D), generator=g)              # the ordinary neighbour in each row
    x[1, 2, 1:] = torch.randn(D - 1, generator=g)           # one large entry alone
    x = x.to(dtype)
    w = (1 + 0.3 * torch.randn(D, generator=g)).to(dtype)
    pos = torch.arange(9).int()[None]
    freq = 10000.0 ** (-2.0 * torch.arange(rot // 2).double() / rot)
    rope = ttf.TTFRope(freq.cuda(), layout=layout)
    for eps in (0.0, 1e-35, 1e-6):
        got, _ = ttf.ttf_qk_norm_rope(x.cuda(), None, pos.cuda(), rope, q_weight=w.cuda(), eps=eps)
        eps = float(torch.tensor(eps))                      # (fp32, as the call takes it)
        want, slack = norm_rotate(x, w, eps, pos, freq, None, layout, 1.0)
        # results below the normal numbers of the type are off by up to half of its least step besides
        check(got, want, slack + 2.0 ** -134, dtype, f"eps {eps}")


@pytest.mark.parametrize("rows,cached,heads,kv_heads,D,page", [
    ([1], [900], 32, 8, 128, 16),
    ([1, 2, 1], [3000, 41, 700], 8, 2, 64, 16),
    ([3, 1], [700, 2000], 8, 1, 128, 16),        # 24 columns
    ([2, 1], [600, 90], 6, 2, 72, 16),
    ([1, 1], [600, 1500], 4, 4, 80, 24),
    ([2], [1100], 8, 2, 200, 16),
    ([1], [1100], 4, 2, 256, 10),
])
def test_few_rows_round_their_output_alone(rows, cached, heads, kv_heads, D, page):
    """bf16: a weight goes into the second product as two bf16 values, half a step of the second off, 2^-16 of it at most; sums are in
    32 bits, and the output is rounded once."""
    q, k, v, table, ks, vs = _problem(rows, cached, heads, kv_heads, D, page, BF)
    out, _ = _run_attention(q, k, v, table, rows, cached, max_rows=max(rows))
    first = 0
    for b, (r, c) in enumerate(zip(rows, cached)):
        seen, part = seen_mask(r, c, r + c, True, 0, torch.ones(r + c, dtype=torch.bool)), q[first:first + r].float()
        want, _, slack, _ = attend(part, ks[b].float(), vs[b].float(), seen, D ** -0.5)
        size, _, _, _ = attend(part, ks[b].float(), vs[b].float().abs(), seen, D ** -0.5)
        check(out[first:first + r], want, slack + 2.0 ** -16 * (1 + 2.0 ** -8) * size, BF, f"sequence {b}")
        first += r


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cached,bad", [([1], [300], 40), ([1, 2], [3000, 20], 700), ([4], [90], 92), ([100], [300], 70), ([100], [300], 350)])
def test_an_infinite_value_stays_infinite(rows, cached, bad, dtype):
    """Values of inf and -inf, each in an entry of its own, with weights that do not underflow: the output is infinite likewise."""
    q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, 64, 16, dtype, peak=0.3)
    for entry, value in ((7, math.inf), (20, -math.inf)):
        vs[0][bad, :, entry] = v[int(table[0, bad // 16]), bad % 16, :, entry] = value
    out, lse = _run_attention(q, k, v, table, rows, cached, max_rows=max(rows))
    sees = cached[0] + torch.arange(rows[0]) >= bad
    assert bool(sees.any()) and bool((out[:rows[0]][sees][..., 7] == math.inf).all()) and bool((out[:rows[0]][sees][..., 20] == -math.inf).all())
    assert not bool(torch.isnan(out).any()) and bool(torch.isfinite(lse).all())
    out[:rows[0]][..., [7, 20]] = 0.0
    for b in range(len(vs)):
        vs[b][..., [7, 20]] = 0.0
    assert bool(torch.isfinite(out[:rows[0]]).all())
    for x in {0, rows[0] // 2, rows[0] - 1}:
        want, _, slack, _ = attend(q[x:x + 1], ks[0], vs[0], seen_mask(rows[0], cached[0], len(ks[0]), True, 0, torch.ones(len(ks[0]), dtype=torch.bool))[x:x + 1], 0.125)
        check(out[x:x + 1], want, slack, dtype, f"row {x}")
