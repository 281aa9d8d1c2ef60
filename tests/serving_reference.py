"""The operators behind the compressed rows in 64 bits on the CPU, written from their formulas, and how far a
right implementation may be off.

Half a step of a type, relative to the value: bf16 2^-8, fp32 2^-24.  ``u`` below is fp32's 2^-24."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24


def rotate(x, pos, inv_freq, axis, layout, factor):
    """x [rows, heads, D] float64; pos [axes, rows]."""
    half = inv_freq.numel()
    y = x.clone()
    for j in range(half):
        a = 0 if axis is None else int(axis[j])
        theta = pos[a].double() * inv_freq[j]
        c, s = factor * torch.cos(theta)[:, None], factor * torch.sin(theta)[:, None]
        i0, i1 = (j, j + half) if layout == "half" else (2 * j, 2 * j + 1)
        y[..., i0] = x[..., i0] * c - x[..., i1] * s
        y[..., i1] = x[..., i1] * c + x[..., i0] * s
    return y


def norm_rotate(x, weight, eps, pos, inv_freq, axis, layout, factor):
    """([rows, heads, D] in 64 bits, bound on the fp32 error before the last rounding)."""
    D = x.shape[-1]
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.double()
    y = rotate(x, pos, inv_freq, axis, layout, factor) if inv_freq is not None else x.clone()
    # the norm's sum of D squares (all of one sign: (D/2 + 1) u at most after halving by the root), square root, division and two products, then two
    # products and a sum with sine and cosine good to 4 u: (D/2 + 16) u of the pair's length
    size = x.abs()
    if inv_freq is not None:
        half = inv_freq.numel()
        if layout == "half":
            pair = torch.sqrt(x[..., :half] ** 2 + x[..., half:2 * half] ** 2)
            size[..., :half] = size[..., half:2 * half] = pair
        else:
            pair = torch.sqrt(x[..., 0:2 * half:2] ** 2 + x[..., 1:2 * half:2] ** 2)
            size[..., 0:2 * half:2] = size[..., 1:2 * half:2] = pair
        size = size * max(1.0, abs(factor))
    return y, (D / 2 + 16) * U * size


def check(got, want, slack, dtype, what=""):
    """got within half a step of its type of want, and `slack` more; where want is not finite, got is not either."""
    got = got.double().cpu()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine), f"{what}: finite in other places"
    err = (got - want).abs()[fine]
    most = (HALF_STEP[dtype] * (want.abs() + slack) + slack)[fine]
    worst = (err - most).max().item() if err.numel() else -1.0
    assert worst <= 0, f"{what}: {worst:.3g} past the bound, error {err.max().item():.3g}"


def attend(q, k, v, seen, scale):
    """One sequence: q [r, H, D], k and v [n, Hk, D], seen [r, n].  Returns out, lse and the bounds on their fp32 (and
    weight) errors; rows that see nothing: 0 and -inf."""
    r, H, D = q.shape
    n, Hk = k.shape[:2]
    dtype = q.dtype
    q, k, v = q.double(), k.double(), v.double()
    out, lse = torch.zeros((r, H, D), dtype=torch.float64), torch.full((r, H), -math.inf, dtype=torch.float64)
    out_slack, lse_slack = torch.zeros_like(out), torch.zeros((r, H), dtype=torch.float64)
    for h in range(H):
        g = h // (H // Hk)
        for i in range(r):
            at = seen[i].nonzero()[:, 0]
            if not at.numel():
                continue
            s = scale * (k[at, g] @ q[i, h])
            lse[i, h] = torch.logsumexp(s, 0)
            w = torch.exp(s - lse[i, h])
            out[i, h] = w @ v[at, g]
            # a score: D products and sums, the factor, the difference to the maximum and the power of 2 (2 u, and
            # its argument's rounding): at most (D + 8) u of sum |q k| scale, and 8 u
            d = (D + 8) * U * float((abs(scale) * (k[at, g].abs() @ q[i, h].abs())).max()) + 8 * U
            # sums over the keys, the moves of the maximum and the join: (n + 64) u of the sum of absolute terms
            d_sum = (at.numel() + 64) * U
            lse_slack[i, h] = d + d_sum + 4 * U * abs(float(lse[i, h]))
            weight = HALF_STEP[dtype] if dtype == torch.bfloat16 else 0.0      # weights rounded to bf16 for the product
            out_slack[i, h] = (2 * d + 2 * d_sum + weight * (1 + 2 * d)) * (w @ v[at, g].abs())
    return out, lse, out_slack, lse_slack


def seen_mask(rows, cached, length, causal, window, there):
    """[rows, length]; `there` [length] truth values of the slots."""
    t = cached + torch.arange(rows)[:, None]
    u = torch.arange(length)[None]
    seen = there[None].expand(rows, length).clone()
    if causal:
        seen &= u <= t
    if window:
        seen &= u > t - window
    return seen
