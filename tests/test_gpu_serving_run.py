"""The operators behind the compressed rows as they are used together: a compressed batch goes into the cache and
is attended to, then token by token; on other streams, in captured graphs, and far into a large cache."""
import math

import pytest
import torch

from serving_reference import attend, check, norm_rotate, seen_mask
from test_gpu_serving import BF, F32, _check_attention, _gen, _offsets, _problem

pytestmark = pytest.mark.gpu


def _gather(t, table, b, n, page):
    u = torch.arange(n)
    return t.cpu()[table[b].long()[u // page], u % page]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_compressed_clips_into_attention(dtype):
    """ttf_compress -> projections -> append -> attention of the whole ragged batch -> two single tokens each."""
    import paper_2605_07355_amd as ttf
    B, F, H, W, C, heads, kv_heads, D, page = 3, 4, 6, 5, 64, 4, 2, 64, 16
    g = _gen(11)
    base = torch.randn((B, 1, H, W, C), generator=g)
    x = (base + 0.5 * torch.rand((B, F, H, W, 1), generator=g) * torch.randn((B, F, H, W, C), generator=g)).to(dtype).cuda()
    out = ttf.ttf_compress(x, r=1, t=0.9)
    offsets, cap = out.buffers.row_offsets, B * F * H * W
    total = out.total_rows
    kept = [int(n) for n in out.buffers.kept_count.cpu()]
    assert H * W * B < total < cap                        # some fused, some kept
    rows = out.buffers.tokens_out.float()
    rows[total:] = 0
    wq, wk, wv = ((torch.randn((C, n * D), generator=g) / math.sqrt(C)).cuda() for n in (heads, kv_heads, kv_heads))
    project = lambda z: [(z @ w).to(dtype).view(z.shape[0], -1, D) for w in (wq, wk, wv)]  # noqa: E731
    q, k, v = project(rows)
    norm_q, norm_k = ((1 + 0.2 * torch.randn(D, generator=g)).to(dtype).cuda() for _ in range(2))
    rope = ttf.ttf_rope_table(D, 1e4, sections=(12, 10, 10), take_turns=True)
    steps = 2
    width = -(-(cap // B + steps) // page)
    table = torch.randperm(B * width + 1, generator=g).int()[:B * width].view(B, width).contiguous()
    kc, vc = (torch.full((B * width + 1, page, kv_heads, D), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    cache = ttf.TTFKVCache(kc, vc, table.cuda())
    cached = torch.zeros(B, dtype=torch.int32, device="cuda")
    # the pass's own offsets and positions go straight in
    q_rot = ttf.ttf_cache_append(cache, k, v, offsets, cached, pos=out.buffers.pos_ids, rope=rope, q=q, q_weight=norm_q, k_weight=norm_k)
    lse = torch.zeros((cap, heads), dtype=torch.float32, device="cuda")
    got = ttf.ttf_paged_attention(q_rot, cache, offsets, cached, lse=lse)
    also, _ = ttf.ttf_qk_norm_rope(q, None, out.buffers.pos_ids, rope, q_weight=norm_q, row_offsets=offsets)
    assert torch.equal(also[:total], q_rot[:total])
    pos = out.buffers.pos_ids.cpu()
    want, slack = norm_rotate(q[:total].cpu(), norm_q.cpu(), 1e-6, pos[:, :total], rope.inv_freq.cpu(), rope.axis.cpu(), "half", 1.0)
    check(q_rot[:total], want, slack, dtype, "q")
    want, slack = norm_rotate(k[:total].cpu(), norm_k.cpu(), 1e-6, pos[:, :total], rope.inv_freq.cpu(), rope.axis.cpu(), "half", 1.0)
    at = offsets.cpu().tolist()
    ks = [_gather(kc, table, b, kept[b], page) for b in range(B)]
    vs = [_gather(vc, table, b, kept[b], page) for b in range(B)]
    for b in range(B):
        check(ks[b], want[at[b]:at[b + 1]], slack[at[b]:at[b + 1]], dtype, "k")
        assert torch.equal(vs[b], v[at[b]:at[b + 1]].cpu())
        o, l, so, sl = attend(q_rot[at[b]:at[b + 1]].cpu(), ks[b], vs[b], seen_mask(kept[b], 0, kept[b], True, 0, torch.ones(kept[b], dtype=torch.bool)), D ** -0.5)
        check(got[at[b]:at[b + 1]], o, so, dtype, "prefill")
        check(lse[at[b]:at[b + 1]], l, sl, F32, "lse")
    # decoding: position and length by the library's own bookkeeping
    ones = torch.arange(B + 1).int().cuda()
    for step in range(steps):
        place = [ttf.ttf_decode_alignment(kept[b], 0, step) for b in range(B)]
        cached = torch.tensor([p for _, p, _ in place]).int().cuda()
        q, k, v = project(torch.randn((B, C), generator=g).cuda())
        where = cached[None].expand(3, B).contiguous()
        q_rot = ttf.ttf_cache_append(cache, k, v, ones, cached, pos=where, rope=rope, q=q, q_weight=norm_q, k_weight=norm_k)
        got = ttf.ttf_paged_attention(q_rot, cache, ones, cached, max_rows=1)
        for b in range(B):
            n = place[b][2]                               # mask length
            o, _, so, _ = attend(q_rot[b:b + 1].cpu(), _gather(kc, table, b, n, page), _gather(vc, table, b, n, page),
                                 torch.ones((1, n), dtype=torch.bool), D ** -0.5)
            check(got[b:b + 1], o, so, dtype, "token")


def test_parts_of_a_context_join_by_their_lse():
    """A row over all entries = its results over two shares of the pages, joined by their lse."""
    import paper_2605_07355_amd as ttf
    rows, cached = [2], [150]
    q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, 64, 16, F32)
    offsets, have = _offsets(rows).cuda(), torch.tensor(cached).int().cuda()
    even = torch.arange(table.shape[1]) % 2 == 0
    parts = []
    for keep in (even, ~even):
        lse = torch.zeros((2, 4), device="cuda")
        o = ttf.ttf_paged_attention(q.cuda(), ttf.TTFKVCache(k.cuda(), v.cuda(), torch.where(keep, table, -1).cuda()), offsets, have, lse=lse)
        parts.append((o, lse))
    lse = torch.logaddexp(parts[0][1], parts[1][1])
    joined = sum(o * torch.exp(l - lse)[..., None] for o, l in parts)
    want, want_lse, slack, lse_slack = attend(q, ks[0], vs[0], seen_mask(2, 150, 152, True, 0, torch.ones(152, dtype=torch.bool)), 64 ** -0.5)
    check(joined, want, 4 * slack + 8 * lse_slack[..., None] * want.abs(), F32)
    check(lse, want_lse, 4 * lse_slack, F32)


def test_another_stream_and_two_at_once():
    """Calls on two streams at a time, each with the memory the binding takes for it."""
    import paper_2605_07355_amd as ttf
    rows, cached = [1, 1], [1500, 3000]
    q, k, v, table, ks, vs = _problem(rows, cached, 8, 2, 128, 16, BF)
    cache, offsets, have, qg = ttf.TTFKVCache(k.cuda(), v.cuda(), table.cuda()), _offsets(rows).cuda(), torch.tensor(cached).int().cuda(), q.cuda()
    want = ttf.ttf_paged_attention(qg, cache, offsets, have)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for i in range(20):
        outs.append(ttf.ttf_paged_attention(qg, cache, offsets, have, stream=streams[i % 2]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    o, _, slack, _ = attend(q[:1], ks[0], vs[0], torch.ones((1, 1501), dtype=torch.bool), 128 ** -0.5)
    check(want[:1], o, slack, BF)


@pytest.mark.parametrize("chunk", [1, 40])
def test_captured_steps(chunk):
    """Append and attention captured once and replayed while lengths, rows and pages change; two graphs share a workspace."""
    import paper_2605_07355_amd as ttf
    B, heads, kv_heads, D, page, width = 2, 4, 2, 64, 16, 40
    g = _gen(4)
    n = B * chunk
    kc, vc = (torch.full((B * width, page, kv_heads, D), math.nan, dtype=BF, device="cuda") for _ in range(2))
    table = torch.randperm(B * width, generator=g).int().view(B, width).cuda()
    cache = ttf.TTFKVCache(kc, vc, table)
    ref = ttf.TTFKVCache(kc.clone(), vc.clone(), table)
    offsets = (torch.arange(B + 1) * chunk).int().cuda()
    cached, pos = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((1, n), dtype=torch.int32, device="cuda")
    x = torch.zeros((n, heads + 2 * kv_heads, D), dtype=BF, device="cuda")
    rope = ttf.ttf_rope_table(D)
    work = torch.empty(ttf.ttf_attention_workspace_size(n, B, heads, kv_heads, D, BF, max_rows=chunk) + 256, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros((n, heads, D), dtype=BF, device="cuda") for _ in range(2)]
    q_rot = torch.zeros((n, heads, D), dtype=BF, device="cuda")

    def step(c, out, window):
        ttf.ttf_cache_append(c, x[:, heads:heads + kv_heads], x[:, heads + kv_heads:], offsets, cached, pos=pos, rope=rope, q=x[:, :heads], q_out=q_rot)
        ttf.ttf_paged_attention(q_rot, c, offsets, cached, max_rows=chunk, window=window, out=out, workspace=work)

    step(cache, outs[0], 0)
    step(cache, outs[1], 30)
    torch.cuda.synchronize()
    graphs = []
    for out, window in zip(outs, (0, 30)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(cache, out, window)
        graphs.append(graph)
    length = 0
    for i in range(6):
        x.copy_(torch.randn(x.shape, generator=g))
        cached.fill_(length)
        pos.copy_((length + torch.arange(chunk).repeat(B))[None])
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for got, window in zip(outs, (0, 30)):
            want = torch.zeros_like(got)
            step(ref, want, window)
            torch.cuda.synchronize()
            assert torch.equal(got, want) and bool(torch.isfinite(want).all()), (i, window)
        length += chunk


@pytest.mark.parametrize("dtype", [BF, F32])
def test_far_into_a_large_cache(dtype):
    """Slots whose offsets pass 2^32 bytes and 2^31 elements."""
    import paper_2605_07355_amd as ttf
    kv_heads, D, page = 8, 128, 64
    pages = (1 << 31) // (page * kv_heads * D) + 40
    kc, vc = (torch.empty((pages, page, kv_heads, D), dtype=dtype, device="cuda") for _ in range(2))
    rows, cached = [1, 70], [0, 100]
    q, k, v, table, ks, vs = _problem(rows, cached, 8, kv_heads, D, page, dtype)
    far = pages - 1 - table
    used = table >= 0
    for b in range(2):
        for p in table[b][used[b]].tolist():
            kc[pages - 1 - p], vc[pages - 1 - p] = k[p].cuda(), v[p].cuda()
    table = torch.where(used, far, -1)
    cache = ttf.TTFKVCache(kc, vc, table.cuda())
    new = torch.randn((71, 8, D), generator=_gen(1)).to(dtype)
    offsets, have = _offsets(rows).cuda(), torch.tensor(cached).int().cuda()
    ttf.ttf_cache_append(cache, new.cuda(), new.cuda(), offsets, have)
    ks[0][0:1] = vs[0][0:1] = new[:1]
    ks[1][100:] = vs[1][100:] = new[1:]
    out = torch.full_like(q, 5.0, device="cuda")
    lse = torch.full((71, 8), 5.0, device="cuda")
    ttf.ttf_paged_attention(q.cuda(), cache, offsets, have, out=out, lse=lse)
    _check_attention(out.cpu(), lse.cpu(), q, ks, vs, rows, cached, True, 0, dtype)


@pytest.mark.parametrize("max_rows", [1, 64])
def test_shared_pages_and_many_sequences(max_rows):
    """The same page in several tables (a shared beginning), and more sequences than a wave has lanes."""
    import paper_2605_07355_amd as ttf
    B, D, page = 150, 64, 16
    rows, cached = [b % 3 for b in range(B)], [16 + b % 20 for b in range(B)]
    q, k, v, table, ks, vs = _problem(rows, cached, 4, 2, D, page, BF)
    table[:, 0] = table[0, 0]
    for b in range(B):
        n = min(16, len(ks[b]))
        ks[b][:n], vs[b][:n] = k[table[0, 0], :n], v[table[0, 0], :n]
    out, lse = torch.full_like(q, 5.0, device="cuda"), torch.full((sum(rows), 4), 5.0, device="cuda")
    ttf.ttf_paged_attention(q.cuda(), ttf.TTFKVCache(k.cuda(), v.cuda(), table.cuda()), _offsets(rows).cuda(), torch.tensor(cached).int().cuda(),
                            max_rows=max_rows, out=out, lse=lse)
    _check_attention(out.cpu(), lse.cpu(), q, ks, vs, rows, cached, True, 0, BF)


@pytest.mark.parametrize("dtype,heads,kv_heads,rows,cached", [
    (BF, 8, 8, [1, 1, 0, 1, 1], [90001, 1, 400, 70000, 73333]),
    (BF, 8, 4, [2, 1, 1], [230000, 240000, 17]),
    (F32, 4, 4, [1, 2], [150000, 100000]),
])
def test_long_contexts_side_by_side(dtype, heads, kv_heads, rows, cached):
    """Contexts so long that workgroups walk along four heads of a slot at once; and the same entries with heads first."""
    import paper_2605_07355_amd as ttf
    D, page = 64, 64
    q, k, v, table, ks, vs = _problem(rows, cached, heads, kv_heads, D, page, dtype)
    offsets, have = _offsets(rows).cuda(), torch.tensor(cached).int().cuda()
    for first in (False, True):
        kg, vg = (t.cuda().transpose(1, 2).contiguous().transpose(1, 2) if first else t.cuda() for t in (k, v))
        out, lse = torch.full_like(q, 5.0, device="cuda"), torch.full((sum(rows), heads), 5.0, device="cuda")
        ttf.ttf_paged_attention(q.cuda(), ttf.TTFKVCache(kg, vg, table.cuda()), offsets, have, max_rows=max(rows), out=out, lse=lse)
        _check_attention(out.cpu(), lse.cpu(), q, ks, vs, rows, cached, True, 0, dtype)
