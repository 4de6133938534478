"""Quantised rows from their definition, in float64 and on the CPU, and how far attention that is
joined from two parts may be from float64.

A block is 32 neighbouring dims: value = code * 2^(s - 127).  s is the least in [10, 254] for which the
block's largest size is at most 464 (e4m3) or 7 (e2m1) times 2^(s - 127); every value becomes the nearest
of the format's numbers, the one with the even code in the middle."""
import math

import torch

import serve_harness as S
from paper_2608_07001_amd import gracekv as gk

BITS = {gk.E4M3: 8, gk.E2M1: 4}
LARGEST = {gk.E4M3: 448.0, gk.E2M1: 6.0}
LIMIT = {gk.E4M3: 464.0, gk.E2M1: 7.0}


def numbers(fmt):
    """What the positive codes stand for, ascending (e4m3 without its NaN)."""
    if fmt == gk.E2M1:
        return torch.tensor([(1 + (c & 1) / 2) * 2.0 ** ((c >> 1) - 1) if c > 1 else c / 2 for c in range(8)], dtype=torch.float64)
    return torch.tensor([(1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) if c > 7 else c / 8 * 2.0 ** -6 for c in range(127)], dtype=torch.float64)


def quantise(x, fmt):
    """x [..., d] float64: codes [..., d] (one a place), scales [..., d / 32], uint8; a code's sign is x's."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    s = torch.full(top.shape, 10, dtype=torch.int64)
    for _ in range(245):
        s += top > LIMIT[fmt] * torch.exp2((s - 127).double())
    none = ~(top < 2.0 ** 127)
    a = torch.where(none[..., None], 0.0, x.abs() * torch.exp2((127 - s).double())[..., None]).clamp(max=LARGEST[fmt])
    v = numbers(fmt)
    hi = torch.searchsorted(v, a.contiguous()).clamp(max=len(v) - 1)
    lo = (hi - 1).clamp(min=0)
    middle = (v[hi] + v[lo]) / 2
    code = torch.where((a > middle) | ((a == middle) & (hi % 2 == 0)), hi, lo)
    sign = torch.where(none[..., None], False, torch.signbit(x)).long() << (BITS[fmt] - 1)
    return (code + sign).flatten(-2).to(torch.uint8), torch.where(none, 255, s).to(torch.uint8)


def packed(codes, fmt):
    return codes if fmt == gk.E4M3 else codes[..., 0::2] | codes[..., 1::2] << 4


def values(codes, scales, fmt):
    """What packed codes stand for, float64."""
    if fmt == gk.E2M1:
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    n = 1 << (BITS[fmt] - 1)
    v = numbers(fmt)
    v = torch.cat([v, torch.full((n - len(v),), math.nan, dtype=torch.float64)])
    x = v[(codes % n).long()] * torch.where(codes >= n, -1.0, 1.0).double()
    s = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))
    return x * s.repeat_interleave(32, -1)


def rotated32(x, cos, sin):
    """Products and sums in fp32, each rounded (CPU)."""
    h = x.shape[-1] // 2
    a, e, c, s = x[..., :h].float(), x[..., h:].float(), cos[:, None], sin[:, None]
    return torch.cat([a * c - e * s, e * c + a * s], -1)


def check_joined(got, got_lse, ref, n, d, bf16, what):
    """Rows joined from two attentions, `ref` over all entries.  A part's mean is off by what serve_harness
    bounds, and its weight by its lse's error (w / 2 + sums + 4 u |lse|) and the exponential of a difference of
    two lse (8 u |lse|): twice the one bound and 32 u of the largest |lse| cover both parts, whose logits
    are the whole row's."""
    out, lse, A, X = ref
    tol, tol_lse = S.bounds(out, lse, A, X, n, d, bf16)
    L = torch.where(lse > -math.inf, lse, 0.0).abs() + X + math.log(max(n, 1))       # |lse| of either part, at most
    tol, tol_lse = 2 * tol + 32 * S.U * (A * L[:, None]), 2 * tol_lse + 32 * S.U * L
    got, got_lse = got.double(), got_lse.double()
    assert torch.isfinite(got).all(), what
    d_out = ((got - out).abs() - tol).max()
    assert d_out <= 0, (what, "out", float(d_out))
    none = lse == -math.inf
    assert torch.equal(none, got_lse == -math.inf), (what, "rows with no key")
    assert (torch.where(none, -1.0, (got_lse - lse).abs() - tol_lse) <= 0).all(), (what, "lse")
