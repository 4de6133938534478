"""Plain float64 forms of the operators around the compressed cache, and how far fp32
or bf16 arithmetic may be from them.

The bounds count roundings, u = 2^-24 (fp32, half a step), b = 2^-8 (bf16).  With x the
logits of a row, X = max sum_i |q_i k_i| / sqrt(d) over its keys and A = sum_j p_j |v_j|:
  * a logit's product sum of d terms and its scaling: off by (d + 3) u X;
  * the exponential of (x - max): argument rounded (at most 4 X u), the hardware's 2 u;
    weights are off by w = 2 ((d + 3) X + 4 X + 4) u of themselves (numerator and sum);
  * sums of n weights and of n products, and n / 16 rescalings of them: 2 (n + n / 16 + 8) u;
  * bf16: weights rounded for the second product, b / (1 + b); the output rounded, b.
So |out - ref| <= A (w + 2 (n + n / 16 + 8) u [+ b]) + |ref| (u [or b]), and
|lse - ref| <= w / 2 + (n + n / 16 + 8) u + 4 u |ref|."""
import math
import random

import torch

U, B16 = 2.0 ** -24, 2.0 ** -8


def attend64(q, k, v, bias=None, seen=None):
    """q [n, d], k, v [m, d], bias [m], seen [n, m] (float64, CPU): out, lse, A, X of every row.
    Keys that are not seen, or have no weight, take part in nothing, whatever they hold."""
    n, m = q.shape[0], k.shape[0]
    if m == 0:
        z = torch.zeros(n, q.shape[1], dtype=torch.float64)
        return z, torch.full((n,), -math.inf, dtype=torch.float64), z, torch.zeros(n, dtype=torch.float64)
    x = q @ k.T / math.sqrt(q.shape[1]) + (0 if bias is None else bias)
    on = torch.ones(n, m, dtype=torch.bool) if seen is None else seen
    if bias is not None:
        on = on & (bias > -math.inf)
    x = torch.where(on, x, -math.inf)
    lse = torch.logsumexp(x, -1)
    p = torch.where(on, (x - torch.where(lse > -math.inf, lse, 0.0)[:, None]).exp(), 0.0)
    fin = torch.isfinite(v)
    vf = torch.where(fin, v, 0.0)
    out, A = p @ vf, p @ vf.abs()
    if not fin.all():                    # what is not finite, for the rows that see it
        for j in (~fin).any(1).nonzero()[:, 0].tolist():
            hit = on[:, j]
            out[hit] += torch.where(fin[j], 0.0, v[j])
    X = torch.where(on, q.abs() @ k.abs().T / math.sqrt(q.shape[1]), 0.0).amax(-1)
    return out, lse, A, X


def bounds(out, lse, A, X, n, d, bf16):
    w = 2 * ((d + 3) * X + 4 * X + 4) * U
    sums = (n + n / 16 + 8) * U
    tol = A * (w + 2 * sums + (B16 if bf16 else 0))[:, None] + out.abs().nan_to_num(0, 0, 0) * (B16 if bf16 else U)
    return tol, w / 2 + sums + 4 * U * torch.where(lse > -math.inf, lse, 0.0).abs()


def check_rows(got, got_lse, ref, n, d, bf16, what):
    out, lse, A, X = ref
    tol, tol_lse = bounds(out, lse, A, X, n, d, bf16)
    got, got_lse = got.double(), got_lse.double()
    fin = torch.isfinite(out)
    assert torch.equal(fin, torch.isfinite(got)), (what, "finite places")
    assert torch.equal(torch.isnan(out), torch.isnan(got)) and torch.equal(out[torch.isinf(out)], got[torch.isinf(out)]), what
    d_out = torch.where(fin, (got - out).abs() - tol, -1.0)
    assert (d_out <= 0).all(), (what, "out", float((got - out).abs()[fin].max()), float(d_out.max()))
    none = lse == -math.inf
    assert torch.equal(none, got_lse == -math.inf), (what, "rows with no key")
    d_lse = torch.where(none, -1.0, (got_lse - lse).abs() - tol_lse)
    assert (d_lse <= 0).all(), (what, "lse", float(d_lse.max()))


def laid(x, layout):
    """[n][heads][d] with the memory of `layout`: token-major, head-major, or rows in a wider buffer."""
    if layout == "token":
        return x.contiguous()
    if layout == "head":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.full((x.shape[0], x.shape[1] + 2, x.shape[2] + 16), float("nan"), dtype=x.dtype, device=x.device)
    wide[:, 1:-1, 8:-8] = x
    return wide[:, 1:-1, 8:-8]


def prompt64(q, k, v, lq, lk, check):
    """check(rows, head, reference, keys) for every sequence and head (CPU float64 inputs)."""
    a = b = 0
    per = q.shape[1] // k.shape[1]
    for n, m in zip(lq, lk):
        seen = torch.arange(m)[None] <= torch.arange(n)[:, None] + (m - n)
        for h in range(q.shape[1]):
            if n:
                check(slice(a, a + n), h, attend64(q[a:a + n, h], k[b:b + m, h // per], v[b:b + m, h // per], seen=seen), m)
        a, b = a + n, b + m


def rotate64(x, cos, sin):
    """x [n][heads][d], cos, sin [n][d/2], in float64."""
    h = x.shape[-1] // 2
    a, e = x[..., :h], x[..., h:]
    c, s = cos[:, None], sin[:, None]
    return torch.cat([a * c - e * s, e * c + a * s], -1)


def paged_shapes():
    """Shapes that take paged attention down its rarer ways, name: (G, H, lens, page, counts of packed
    entries or None).  `searched`: more units than a wave looks at in one round (64), rows of several
    chunks among them, first, last and between; `long`: rows of more chunks than the join takes at once (d / 2)."""
    r = random.Random(7)
    ragged = [0 if i % 5 == 0 else r.randint(20, 60) for i in range(130)]
    ragged[0], ragged[64], ragged[129] = 9000, 3001, 5003
    few = [r.randint(0, 40) for _ in range(24)]
    packed = [r.randint(0, 3000) if r.random() < 0.7 else r.choice([0, 1, 64]) for _ in range(24 * 8)]
    packed[0], packed[63], packed[64], packed[191] = 3000, 2999, 0, 2800
    return {"searched pages": (2, 4, ragged, 16, None), "searched entries": (8, 16, few, 16, packed),
            "long pages": (1, 4, [131072], 64, None), "long entries": (1, 4, [100], 64, [131073])}
