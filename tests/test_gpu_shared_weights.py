"""Weights of shared entries in bf16 are held in two bf16 parts, whichever kernel a call takes: for the product with
the values each is off by at most 2^-15 of itself (rounded to one part, by up to 2^-8)."""
import pytest
import torch

import serve_harness as S
import shared_harness as P
from paper_2608_07001_amd import gracekv as gk
from test_gpu_quant import Shared
from test_gpu_shared_large import Large

pytestmark = pytest.mark.gpu


def _check(c):
    part, per, a = c.call(), c.H // c.G, 0
    o = part.o.cpu().double()
    for s, m in enumerate(c.groups):
        for g in range(c.G if m else 0):
            k, v, lm = c.entries(s, g)
            h = slice(g * per, (g + 1) * per)
            ref = S.attend64(c.q[a:a + m, h].reshape(m * per, -1).double(), k, v, bias=lm)
            # a part's mean is fp32: of bf16 roundings only the weights' are left
            tol = S.bounds(*ref, max(len(k), 1), c.d, False)[0] + ref[2] * 2.0 ** -15
            over = ((o[a:a + m, h].reshape(m * per, -1) - ref[0]).abs() - tol).max()
            assert over <= 0, (s, g, float(over))
        a += m


@pytest.mark.parametrize("kind", [k for k in P.KINDS if k[0] == "bf16"])
def test_weights_of_large_tiles(kind):
    # few entries with weights of about the same size, whose roundings are not lost in a sum; and many
    for i, (G, H, groups) in enumerate(P.one_group(kind)):
        for n in (2, 3, 9, 300):
            _check(Large(kind, G, H, groups, [n, n + 1][:G], seed=30 + i))
    _check(Large(kind, *P.several_groups(kind), seed=33))
    _check(Large(kind, *P.deep(kind), seed=34))


@pytest.mark.parametrize("d", [64, 128])
def test_weights_of_small_tiles(d):
    for rows, waves in ((1, 4), (16, 4), (40, 8 if d == 128 else 4)):
        for n in (2, 3, 9, 300, 1500 if waves == 4 else 1700):
            _check(Shared("bf16", d, 1, 2, [rows], [n], seed=35 + rows))


def test_weights_do_not_depend_on_other_rows_of_the_arrays():
    # the same call on arrays of its own and on those that hold other entries as well: another kernel, the same precision
    a = Shared("bf16", 128, 1, 4, [20], [20], seed=36)
    b = Large(("bf16", 128, 8), 1, 4, [20], [20], seed=36)
    assert P.kernel("bf16", 128, 1, 4, 20, 1, a.pre["K"].shape[0])[0] == "few"
    x, y = a.call().o.cpu().double(), b.call().o.cpu().double()
    ref = [S.attend64(a.q[:, h].double(), *a.entries(0, 0)[:2], bias=a.entries(0, 0)[2]) for h in range(4)]
    for h, (out, lse, A, X) in enumerate(ref):
        tol = 2 * (S.bounds(out, lse, A, X, 20, 128, False)[0] + A * 2.0 ** -15)
        assert ((x[:, h] - y[:, h]).abs() <= tol).all()
