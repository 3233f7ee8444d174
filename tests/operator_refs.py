"""Plain 64-bit forms of the operators around the decode step, and the bounds their tests use.

bf16 has 8 significant bits: rounding to it is off by at most 2^-8 of the value (HALF_ULP), by less
than 2^-9 on average.  An attention output is a mean of values with weights that are rounded to bf16
independently of one another; with A = sum p |v| / sum p, each rounding of the weights and that of
their sum is taken as 2^-9 A, the output's own as 2^-9 of itself (for a single visible key, whose weight
is 1, what is left of the sum covers a whole HALF_ULP).  Scores are off by a few 1e-4 (fp32 sums of a few
hundred products around 1, 136 times larger before a 4-bit code's offset cancels), and so, relatively,
are weights: 1e-3 A covers them.
"""
import math

import torch

HALF_ULP = 2.0 ** -8


def held(x):
    """What the 4-bit cache holds of bf16 x [...][d]: per 32 channels s = bf16(max |x| / 7) and the
    whole numbers nearest to x / s, halves away from zero."""
    y = x.double().unflatten(-1, (-1, 32))
    largest = y.abs().amax(-1, keepdim=True)
    s = (largest / 7).bfloat16().double()
    bad = ~torch.isfinite(largest)
    zero = s < 2.0 ** -126
    ratio = y / torch.where(zero | bad, torch.ones_like(s), s)
    q = torch.sign(ratio) * torch.floor(ratio.abs() + 0.5)
    v = torch.where(zero, torch.zeros_like(y), q * s)
    return torch.where(bad, torch.full_like(y, math.nan), v).flatten(-2)


def visible(L, window, sinks, t=None):
    """Positions u that a query at position t (default the last of L) sees."""
    u = torch.arange(L, device="cuda")
    t = L - 1 if t is None else t
    keep = u <= t
    return keep if window == 0 else keep & ((u < sinks) | (u > t - window))


def attend(q, k, v, see):
    """(softmax(q k^T / sqrt(d)) v, A) for q [h][n][d], k and v [g][L][d] (64-bit), see [n][L]: only
    seen positions are touched."""
    h, n, d = q.shape
    G = h // k.shape[0]
    some = see.any(0)
    k, v, see = k[:, some], v[:, some], see[:, some]
    k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
    s = (q @ k.transpose(1, 2) / math.sqrt(d)).masked_fill(~see, -math.inf)
    p = torch.softmax(s, -1)
    v0 = torch.nan_to_num(v)
    return p @ v0, p @ v0.abs()


def assert_attention(got, want, spread, roundings, floor=0.0):
    """got bf16 against want; spread = A; floor: an absolute part (same shape or a number)."""
    bound = ((roundings + 1) * HALF_ULP / 2 + 1e-3) * spread + HALF_ULP / 2 * want.abs() + floor + 1e-30
    err = (got.double() - want).abs()
    assert torch.isfinite(got.float()).all()
    worst = float((err / bound).max())
    assert worst <= 1.0, worst
