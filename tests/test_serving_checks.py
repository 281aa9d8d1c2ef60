"""CPU-only checks of the entry points behind the compressed rows: refusals before any HIP call, workspace
sizes, structure layouts, and the frequencies of a rotation against the formulas."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import paper_2605_07355_amd as ttf
from paper_2605_07355_amd import serving

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, SMALL = 1, 2, 3
A = 1 << 20                    # an address that is never followed: the checks come first


def _qk(**change):
    p = dict(dtype=0, head_dim=64, heads=4, kv_heads=2, rows=8, batch=2, row_offsets=A, cached=A, q=A, k=A, v=A, q_row=256,
             q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, q_out=A, k_out=A, qo_row=256, qo_head=64, ko_row=128,
             ko_head=64, q_weight=A, k_weight=None, eps=1e-6, rotary_dim=64, layout=0, axes=1, inv_freq=A, axis=None, pos=A,
             pos_stride=8, attention_factor=1.0)
    p.update(change)
    return serving._QKParams(**p)


def _cache(**change):
    c = dict(k=A, v=A, page_table=A, page_stride=16 * 128, slot_stride=128, head_stride=64, table_stride=4, pages=9, page_size=16,
             table_width=4)
    c.update(change)
    return serving._KVCache(**c)


def _attention(**change):
    p = dict(dtype=0, head_dim=64, heads=4, kv_heads=2, rows=8, batch=2, max_rows=4, causal=1, window=0, scale=0.125, row_offsets=A,
             cached=A, q=A, out=A, lse=None, q_row=256, q_head=64, o_row=256, o_head=64)
    p.update(change)
    return serving._AttentionParams(**p)


QK_BAD = [
    (INVALID, dict(rows=0)), (INVALID, dict(rows=(1 << 24) + 1)), (INVALID, dict(batch=0)), (INVALID, dict(batch=(1 << 20) + 1)),
    (INVALID, dict(heads=-1)), (INVALID, dict(heads=0, kv_heads=0)), (INVALID, dict(rows=1 << 24, heads=16)),
    (INVALID, dict(q=None)), (INVALID, dict(q_out=None)), (INVALID, dict(k=None)), (INVALID, dict(q_row=32)), (INVALID, dict(k_head=8)),
    (INVALID, dict(q_row=-256)), (INVALID, dict(head_dim=0)), (INVALID, dict(rotary_dim=7)), (INVALID, dict(rotary_dim=66)),
    (INVALID, dict(rotary_dim=-2)), (INVALID, dict(layout=2)), (INVALID, dict(axes=0)), (INVALID, dict(axes=5)),
    (INVALID, dict(pos=None)), (INVALID, dict(inv_freq=None)), (INVALID, dict(axes=2, pos_stride=7)),
    (INVALID, dict(attention_factor=math.inf)), (INVALID, dict(eps=-1.0)), (INVALID, dict(eps=math.nan)),
    (UNSUPPORTED, dict(dtype=2)), (UNSUPPORTED, dict(head_dim=264, rotary_dim=0)), (UNSUPPORTED, dict(head_dim=60, rotary_dim=60)),
    (UNSUPPORTED, dict(q=A + 8)), (UNSUPPORTED, dict(q_row=260)), (UNSUPPORTED, dict(k_head=68)), (UNSUPPORTED, dict(q_weight=A + 2)),
]


@pytest.mark.parametrize("status,change", QK_BAD + [(INVALID, dict(k_out=None))])
def test_norm_and_rotation_refuses(status, change):
    assert ttf.load_library() and serving._library().ttf_qk_norm_rope(ctypes.byref(_qk(**change)), None) == status


@pytest.mark.parametrize("status,change", QK_BAD + [(INVALID, dict(row_offsets=None)), (INVALID, dict(cached=None)), (INVALID, dict(v=None)),
                                                    (INVALID, dict(kv_heads=0)), (UNSUPPORTED, dict(v_row=132))])
def test_append_refuses(status, change):
    assert serving._library().ttf_cache_append(ctypes.byref(_qk(**change)), ctypes.byref(_cache()), None) == status


CACHE_BAD = [(INVALID, dict(k=None)), (INVALID, dict(v=None)), (INVALID, dict(page_table=None)), (INVALID, dict(pages=0)),
             (INVALID, dict(page_size=0)), (INVALID, dict(page_size=(1 << 20) + 1)), (INVALID, dict(table_width=0)),
             (INVALID, dict(table_stride=3)), (INVALID, dict(page_stride=-8)), (INVALID, dict(page_stride=56)),
             (INVALID, dict(slot_stride=0)), (INVALID, dict(head_stride=32)), (UNSUPPORTED, dict(k=A + 4)), (UNSUPPORTED, dict(slot_stride=132))]


@pytest.mark.parametrize("status,change", CACHE_BAD)
def test_cache_is_checked(status, change):
    lib = serving._library()
    assert lib.ttf_cache_append(ctypes.byref(_qk()), ctypes.byref(_cache(**change)), None) == status
    assert lib.ttf_paged_attention(ctypes.byref(_attention()), ctypes.byref(_cache(**change)), A, 1 << 40, None) == status


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(rows=0)), (INVALID, dict(heads=5)), (INVALID, dict(kv_heads=0)), (INVALID, dict(max_rows=0)), (INVALID, dict(causal=2)),
    (INVALID, dict(window=-1)), (INVALID, dict(scale=math.nan)), (INVALID, dict(row_offsets=None)), (INVALID, dict(cached=None)),
    (INVALID, dict(q=None)), (INVALID, dict(out=None)), (INVALID, dict(o_row=8)), (UNSUPPORTED, dict(dtype=5)),
    (UNSUPPORTED, dict(head_dim=20)), (UNSUPPORTED, dict(out=A + 8)), (INVALID, dict(batch=1 << 20, heads=8, kv_heads=8)),
])
def test_attention_refuses(status, change):
    assert serving._library().ttf_paged_attention(ctypes.byref(_attention(**change)), ctypes.byref(_cache()), A, 1 << 40, None) == status


def test_null_structures_and_workspace():
    lib = serving._library()
    assert lib.ttf_qk_norm_rope(None, None) == INVALID
    assert lib.ttf_cache_append(ctypes.byref(_qk()), None, None) == INVALID
    assert lib.ttf_paged_attention(None, ctypes.byref(_cache()), A, 1 << 40, None) == INVALID
    p, c, n = _attention(), _cache(), ctypes.c_size_t(0)
    assert lib.ttf_attention_workspace_size(None, ctypes.byref(n)) == INVALID
    assert lib.ttf_attention_workspace_size(ctypes.byref(p), None) == INVALID
    assert lib.ttf_attention_workspace_size(ctypes.byref(p), ctypes.byref(n)) == 0
    assert 0 < n.value <= 512 << 20
    assert lib.ttf_paged_attention(ctypes.byref(p), ctypes.byref(c), None, n.value, None) == INVALID
    assert lib.ttf_paged_attention(ctypes.byref(p), ctypes.byref(c), A + 128, n.value, None) == UNSUPPORTED
    assert lib.ttf_paged_attention(ctypes.byref(p), ctypes.byref(c), A, n.value - 1, None) == SMALL
    for dtype in (torch.bfloat16, torch.float32):
        for D in (8, 64, 128, 136, 256):
            for rows in (1, 7, 5000, 1 << 24):                # does not grow with the rows or the context
                assert ttf.ttf_attention_workspace_size(rows, 1, 8, 2, D, dtype) <= 512 << 20


@pytest.mark.parametrize("change", [dict(qo_row=512), dict(qo_head=256, qo_row=64), dict(ko_row=256)])
def test_outputs_over_their_inputs_keep_the_strides(change):
    assert serving._library().ttf_qk_norm_rope(ctypes.byref(_qk(**change)), None) == INVALID
    if "ko_row" not in change:                               # (an append writes no k_out)
        assert serving._library().ttf_cache_append(ctypes.byref(_qk(**change)), ctypes.byref(_cache()), None) == INVALID


@pytest.mark.parametrize("change", [dict(o_row=512), dict(o_head=256, o_row=64)])
def test_attention_over_its_queries_keeps_the_strides(change):
    p = _attention(**change)
    assert serving._library().ttf_paged_attention(ctypes.byref(p), ctypes.byref(_cache()), A, 1 << 40, None) == INVALID


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,batch", [(1 << 24, 1), (1 << 24, 1000), (100, 2)])
def test_max_rows_below_the_mean_counts_as_the_mean(rows, batch, dtype):
    mean = -(-rows // batch)
    size = [ttf.ttf_attention_workspace_size(rows, batch, 4, 4, 64, dtype, max_rows=n) for n in (1, mean)]
    assert size[0] == size[1]


def test_binding_refuses():
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):                       # no CPU path
        ttf.ttf_qk_norm_rope(x, x)
    with pytest.raises(TypeError):
        ttf.ttf_qk_norm_rope(x.half(), x.half())
    for q, k in ((x.transpose(1, 2), x), (x, x[:3]), (x[0], x), (x, x.float()), (None, None)):
        with pytest.raises((ValueError, TypeError)):
            ttf.ttf_qk_norm_rope(q, k)
    k = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16)
    table = torch.zeros((2, 4), dtype=torch.int32)
    for bad in ((k, k[:2], table), (k, k.transpose(1, 2), table), (k[0], k[0], table), (k, k, table.long()), (k, k, table[0]), (k, k, table.t())):
        with pytest.raises(ValueError):
            ttf.TTFKVCache(*bad)
    cache, offsets, cached = ttf.TTFKVCache(k, k.clone(), table), torch.tensor([0, 2, 4]).int(), torch.tensor([0, 0]).int()
    for kw in (dict(q=x.float()), dict(row_offsets=offsets[:2]), dict(row_offsets=offsets.long()), dict(cached=cached[:1]), dict(out=x[:3]),
               dict(lse=torch.zeros(4, 2, dtype=torch.bfloat16)), dict(q=torch.zeros((4, 2, 32), dtype=torch.bfloat16)), dict()):
        args = dict(q=x, row_offsets=offsets, cached=cached) | kw
        with pytest.raises(ValueError):
            ttf.ttf_paged_attention(args.pop("q"), cache, args.pop("row_offsets"), args.pop("cached"), **args)
    with pytest.raises(ValueError):
        ttf.ttf_cache_append(cache, x[:, :1], x[:, :1], offsets, cached)
    assert ttf.ttf_paged_attention(x[:0], cache, offsets, cached).shape == (0, 2, 64)        # nothing to do


def test_structures_match_the_header(tmp_path):
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ttf.h"\n'
                   'int main(void) { printf("%zu %zu %zu %zu %zu %zu\\n", sizeof(ttf_qk_params), sizeof(ttf_kv_cache),\n'
                   '  sizeof(ttf_attention_params), offsetof(ttf_qk_params, attention_factor), offsetof(ttf_qk_params, eps),\n'
                   '  offsetof(ttf_attention_params, o_head)); return 0; }\n')
    exe = str(tmp_path / "sz")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", str(src), "-I", os.path.join(ROOT, "include"), "-o", exe], check=True)
    out = [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    q, c, a = serving._QKParams, serving._KVCache, serving._AttentionParams
    assert out == [ctypes.sizeof(q), ctypes.sizeof(c), ctypes.sizeof(a), q.attention_factor.offset, q.eps.offset, a.o_head.offset]


# ------------------------------------------------------------------------------ frequencies
def _close(got, want):
    assert torch.allclose(got, torch.tensor(want, dtype=torch.float64), rtol=1e-13, atol=0)


def test_plain_and_stretched_frequencies():
    R, base = 12, 10000.0
    f = [base ** (-2 * j / R) for j in range(R // 2)]
    table = lambda **kw: ttf.ttf_rope_table(R, base, device="cpu", **kw)  # noqa: E731
    assert table().axis is None and table().attention_factor == 1.0 and table().inv_freq.dtype == torch.float64
    _close(table().inv_freq, f)
    _close(table(scaling="linear", factor=4.0).inv_freq, [x / 4 for x in f])
    b = table(scaling="base", factor=4.0).inv_freq
    _close(b[:1], f[:1])
    _close(b[-1:], [f[-1] / 4])
    _close(ttf.ttf_rope_table(2, base, scaling="base", factor=4.0, device="cpu").inv_freq, [1.0])


def test_frequencies_divided_in_part():
    R, base, L, s, fast, slow = 128, 10000.0, 4096, 16.0, 32.0, 1.0
    f = [base ** (-2 * j / R) for j in range(R // 2)]
    turns = [L * x / (2 * math.pi) for x in f]
    t = ttf.ttf_rope_table(R, base, scaling="parts", factor=s, original_length=L, fast=fast, slow=slow, device="cpu")
    assert t.attention_factor == pytest.approx(0.1 * math.log(s) + 1, rel=1e-6)
    low, high = max(j for j in range(64) if turns[j] >= fast), min(j for j in range(64) if turns[j] <= slow)
    g = [min(max((j - low) / (high - low), 0.0), 1.0) for j in range(64)]
    _close(t.inv_freq, [x * (1 - y) + x / s * y for x, y in zip(f, g)])
    t = ttf.ttf_rope_table(R, base, scaling="turns", factor=s, original_length=L, fast=4.0, slow=1.0, device="cpu")
    g = [min(max((4.0 - n) / 3.0, 0.0), 1.0) for n in turns]
    assert t.attention_factor == 1.0 and 0 < sum(0 < y < 1 for y in g)
    _close(t.inv_freq, [x * (1 - y) + x / s * y for x, y in zip(f, g)])
    # a context so short that no pair turns once: all are divided but the first
    t = ttf.ttf_rope_table(8, 100.0, scaling="parts", factor=2.0, original_length=2, device="cpu")
    _close(t.inv_freq, [100.0 ** (-2 * j / 8) / (2 if j else 1) for j in range(4)])


def test_planes_of_the_pairs():
    table = lambda **kw: ttf.ttf_rope_table(16, device="cpu", **kw).axis.tolist()  # noqa: E731
    assert table(sections=(4, 2, 2)) == [0, 0, 0, 0, 1, 1, 2, 2]
    assert table(sections=(0, 8)) == [1] * 8
    assert table(sections=(4, 2, 2), take_turns=True) == [0, 1, 2, 0, 1, 2, 0, 0]
    assert table(sections=(8, 0), take_turns=True) == [0] * 8
    assert table(sections=(8,)) == [0] * 8


@pytest.mark.parametrize("kw", [dict(rotary_dim=7), dict(rotary_dim=0), dict(base=1.0), dict(base=math.inf), dict(scaling="linear", factor=0.5),
                                dict(scaling="parts", factor=2.0), dict(scaling="turns", factor=2.0, original_length=100, fast=1.0, slow=1.0),
                                dict(sections=(4, 3)), dict(sections=(-1, 9)), dict(sections=(2, 2, 2, 1, 1)),
                                dict(sections=(1, 7), take_turns=True)])
def test_table_refuses(kw):
    args = dict(rotary_dim=16, base=1e4, device="cpu") | kw
    with pytest.raises(ttf.TTFError) as e:
        ttf.ttf_rope_table(args.pop("rotary_dim"), args.pop("base"), **args)
    assert e.value.status == INVALID
