"""Entries that groups of sequences share, on the kernels of large row tiles and the launch that joins their states
(every call asserts which kernel it takes), against float64; tolerances count roundings (serve_harness).  The shared
calls of test_gpu_quant.py, however many rows they have, take the kernel of small tiles, but for a few of long entries."""
import math

import pytest
import torch

import serve_harness as S
import shared_harness as P
from paper_2608_07001_amd import gracekv as gk
from test_gpu_quant import Cache, Shared, _joined

pytestmark = pytest.mark.gpu


class Large(Shared):
    """Groups whose packed arrays hold, before and behind the entries in use, as many others as make the work look
    large; all of those are NaN.  `kind`: (type, d, waves) of the kernel that it has to take."""

    def __init__(self, kind, G, Hq, groups, counts, behind=0, seed=0):
        super().__init__(kind[0], kind[1], G, Hq, groups, counts, behind=behind, seed=seed)
        self.kind, self.kernel = kind, ("many", kind[2])

    def packed(self):
        n = self.pre["K"].shape[0]
        rows = n + P.PAD * self.G * len(self.groups)
        assert P.kernel(self.kind[0], self.d, self.G, self.H, self.n, len(self.groups), rows) == self.kernel
        far, out = (rows - n) // 2, dict(start=self.pre["start"].cuda() + (rows - n) // 2, count=self.pre["count"].cuda())
        for k in ("K", "V", "logm"):
            x = torch.full((rows,) + self.pre[k].shape[1:], math.nan, dtype=self.pre[k].dtype, device="cuda")
            x[far:far + n] = self.pre[k].cuda()
            out[k] = x
        return gk.Prefix(**out)

    def check(self, part=None, wide=0.0):
        """`wide`: the largest |log m| where it adds to the size of the logits' sums."""
        part, per, a = part or self.call(), self.H // self.G, 0
        o, lse = part.o.cpu(), part.lse.cpu()
        for s, m in enumerate(self.groups):
            for g in range(self.G if m else 0):
                k, v, lm = self.entries(s, g)
                h = slice(g * per, (g + 1) * per)
                out, ref_lse, A, X = S.attend64(self.q[a:a + m, h].reshape(m * per, -1).double(), k, v, bias=lm)
                S.check_rows(o[a:a + m, h].reshape(m * per, -1), lse[a:a + m, h].reshape(-1), (out, ref_lse, A, X + wide), max(len(k), 1), self.d,
                             self.dtype == "bf16", (self.kind, self.G, self.H, s, g))
            a += m
        assert (o[a:] == 7).all() and (lse[a:] == 7).all()      # behind the last group

    def call(self, ws=None, prefix=None):
        q = self.q.cuda()
        cfg = gk.shared_config(q, self.G, len(self.groups))
        ws = torch.full((gk.shared_ws_bytes(cfg),), 255, dtype=torch.uint8, device="cuda") if ws is None else ws
        part = gk.Part(torch.full((self.n, self.H, self.d), 7.0, device="cuda"), torch.full((self.n, self.H), 7.0, device="cuda"))
        gk.shared_attention(cfg, q, self.cu.cuda(), self.packed() if prefix is None else prefix, part, ws)
        torch.cuda.synchronize()
        return part


def _shapes(kind):
    """name, shape with entries"""
    for i, (G, H, groups) in enumerate(P.one_group(kind)):
        yield f"one {i}", (G, H, groups, [[300], [129, 1], [700]][i])
    yield "several", P.several_groups(kind)
    yield "deep", P.deep(kind)


def _all(kind, names=("one 0", "one 1", "one 2", "several", "deep")):
    for seed, (name, shape) in enumerate(_shapes(kind)):
        if name in names:
            yield name, Large(kind, *shape, behind=2 if len(shape[2]) > 1 else 0, seed=90 + seed)


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_groups(kind):
    for _, c in _all(kind):
        c.pre["V"] += torch.linspace(0, 4, c.pre["V"].shape[0])[:, None].to(c.pre["V"].dtype)      # a chunk lost or taken twice shows
        c.check()


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_every_number_of_entries(kind):
    for i, (G, H, groups) in enumerate(P.one_group(kind)):
        for n in (0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257):
            Large(kind, G, H, groups, [n, 257 - n][:G], seed=n).check()


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_long_rows(kind):
    # chunks of several key tiles of one group, and more chunks than the join takes at once
    G, H, groups = P.one_group(kind)[1]
    c = Large(kind, G, H, groups, [40001, 30000], seed=60)
    c.pre["V"] += torch.linspace(0, 4, c.pre["V"].shape[0])[:, None].to(c.pre["V"].dtype)
    c.check()


@pytest.mark.parametrize("kind", P.KINDS)
@pytest.mark.parametrize("what", ["some", "first", "tile", "all"])
def test_large_masked_entries(kind, what):
    # log m = -inf of some entries, of the first, of whole key tiles and of all; what is masked or behind the entries
    # holds NaN and infinities
    for _, c in _all(kind, ("one 0", "one 1", "several", "deep")):
        lm = c.pre["logm"]
        i = torch.arange(len(lm))
        mask = {"some": i % 3 == 0, "first": i < 303, "tile": i % 600 >= 250, "all": i >= 0}[what]
        mask[-3:] = True
        lm[mask] = -math.inf
        c.pre["V"][mask & (i % 7 == 0)] = math.nan
        c.pre["V"][mask & (i % 7 == 3)] = math.inf
        c.pre["K"][mask, ::2] = math.inf
        c.pre["K"][mask & (i % 2 == 0)] = math.nan
        c.check()


def _lowest(c, n, place, low):
    """Entries of the lowest value, -inf among them, in one unit; then one other entry."""
    lm, bf16 = c.pre["logm"], c.dtype == "bf16"
    lm[:n] = low
    lm[5:n:7] = -math.inf
    c.pre["V"][5:n:7] = math.inf
    part = c.call()
    _, v, _ = c.entries(0, 0)
    seen = lm[:n] == low
    m, per = c.groups[0], c.H // c.G
    mean, tol = v[seen].mean(0), (S.B16 * 2 if bf16 else 1e-5) * v[seen].abs().mean(0) + 1e-6
    assert ((part.o[:m, :per].cpu().double() - mean).abs() <= tol).all()
    assert torch.isfinite(part.lse[:m, :per]).all() and (part.lse[:m, :per] <= low * 0.999).all()
    lm[place] = 0.5
    c.pre["V"][place] = 1.0
    c.check()


@pytest.mark.parametrize("kind", P.KINDS)
@pytest.mark.parametrize("low", [torch.finfo(torch.float32).min, torch.finfo(torch.bfloat16).min, -1e37])
def test_large_lowest_log_m(kind, low):
    # the lowest value as a mask: no weight beside other entries, equal weights among themselves; whole tiles
    # and chunks of them before and behind others
    for i, (G, H, groups) in enumerate(P.one_group(kind)[:2]):
        for n, place in ((40, 3), (700, 3), (700, 650), (300, 200)):
            c = Large(kind, G, H, groups, [n, 50][:G], seed=7 + i)
            c.q[:] = 0.0
            _lowest(c, n, place, low)
    G, H, groups, counts = P.deep(kind)
    for place in (3, 480):
        c = Large(kind, G, H, groups, counts, seed=9)
        c.q[:] = 0.0
        _lowest(c, counts[0], place, low)


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_different_lowest_values(kind):
    # of entries that are all below what counts the largest log m decide, in whichever tile they lie
    for n, place in ((300, 7), (300, 290), (900, 500)):
        G, H, groups = P.one_group(kind)[0]
        c = Large(kind, G, H, groups, [n], seed=12)
        c.pre["logm"][:n] = torch.linspace(-3e38, -2e37, n)[torch.randperm(n, generator=torch.Generator().manual_seed(n))]
        c.pre["logm"][place] = -1e37
        part = c.call()
        v = c.pre["V"][place].float()                              # its weight is 1, in two bf16 parts off by at most 2^-15
        assert ((part.o.cpu() - v).abs() <= v.abs() * 2.0 ** -15).all() and (part.lse.cpu() == torch.tensor(-1e37)).all()


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_infinite_values_stay_in_their_dimension(kind):
    for name, c in _all(kind, ("one 0", "one 1", "deep")):
        c.pre["V"][77, 5], c.pre["V"][128, c.d - 1] = math.inf, -math.inf
        c.check()


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_logits(kind):
    for _, c in _all(kind):
        c.q *= 16
        c.check()


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_logits_along_the_entries(kind):
    # what is subtracted rises from tile to tile, or falls by far: weights that vanish and sums that are rescaled
    for up in (1, -1):
        G, H, groups, counts = P.deep(kind)
        c = Large(kind, G, H, groups, counts, seed=13)
        c.pre["logm"] = up * torch.arange(len(c.pre["logm"]), dtype=torch.float32) % 1000 * 0.1
        c.check(wide=100.0)                                        # log m is summed up with the products


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_many_units(kind):
    c = Large(kind, *P.many_units(kind), behind=2, seed=14)
    c.check()
    c.pre["logm"][::2] = -math.inf
    c.pre["V"][::2] = math.nan
    c.check()


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_malformed_inputs_stay_inside(kind):
    G, H, groups, counts = P.several_groups(kind)
    c = Large(kind, G, H, groups, counts, seed=15)
    pre = c.packed()
    n = pre.K.shape[0]
    pre.start[0], pre.count[1], pre.count[6], pre.start[4] = -4, -3, -(1 << 40), 1 << 40
    part = c.call(prefix=pre)
    far = int(pre.start[2]) - int(c.pre["start"][2])
    want = c.pre
    want["start"], want["count"] = pre.start.cpu(), pre.count.cpu()
    # unit 0 begins at the arrays' first row, which is NaN; the others are held to nothing
    a = groups[0]
    assert torch.isnan(part.o[:a, :2]).all() and torch.isnan(part.lse[:a, :2]).all()
    for u in (1, 4, 6):
        want["start"][u], want["count"][u] = far, 0
    want["start"] -= far
    o, lse = part.o.clone(), part.lse.clone()
    want["start"][0], want["count"][0] = 0, 0
    o[:a, :2], lse[:a, :2] = 0.0, -math.inf
    c.check(gk.Part(o, lse))
    long = c.packed()
    long.start[0], long.count[0] = n - 5, 1 << 40                  # held to the arrays' end
    assert torch.isnan(c.call(prefix=long).o[:a, :2]).all()
    B = c.n
    for cu in ([B + 9, 3, 7, 0], [0, B + 9, 0, B + 9], [-5, 2 ** 31 - 1, -2 ** 31, 7], [9, 9, 9, 9], [0, 0, 0, 0]):
        c.cu = torch.tensor((cu * 3)[:len(groups) + 1], dtype=torch.int32)
        need = gk.shared_ws_bytes(gk.shared_config(c.q, G, len(groups)))
        ws = torch.full((2 * need + (64 << 20),), 85, dtype=torch.uint8, device="cuda")
        c.call(ws=ws[:need])                                        # (what the rows hold is not specified)
        assert (ws[need:] == 85).all()


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_descending_groups_stay_inside(kind):
    # every second group has all sequences: many more chunks than places, none of them written behind the workspace
    for G, H, groups in P.descending(kind):
        n = len(groups)
        c = Large(kind, G, H, groups, [300] * (G * n), seed=10)
        c.cu = torch.tensor([groups[0] * (j % 2) for j in range(n + 1)], dtype=torch.int32)
        need = gk.shared_ws_bytes(gk.shared_config(c.q, G, n))
        ws = torch.full((4 * need + (64 << 20),), 85, dtype=torch.uint8, device="cuda")
        c.call(ws=ws[:need])                                        # (what the rows hold is not specified)
        assert (ws[need:] == 85).all()


@pytest.mark.parametrize("fill", [0, 1, 127, 255])
def test_large_workspace_needs_no_clearing(fill):
    # one workspace for all kernels in turn: what one leaves in it is nothing to the next, and the bits are the same again
    cases = [Large(kind, *f(kind), seed=20) for kind in P.KINDS for f in (P.several_groups, P.deep)]
    cases[2:2] = [Shared("bf16", 128, 2, 8, [20, 1], [4001, 3, 0, 900], seed=20), Shared("f32", 64, 1, 20, [3] * 40, [60] * 39 + [3000], seed=21)]
    ws = torch.full((256 << 20,), fill, dtype=torch.uint8, device="cuda")
    first = {}
    for c in cases + cases[::-1]:
        part = c.call(ws=ws)
        if id(c) not in first:
            c.check(part)
        was = first.setdefault(id(c), part)
        assert torch.equal(was.o, part.o) and torch.equal(was.lse, part.lse)


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_joined_to_quantised_pages(kind):
    dtype, d, _ = kind
    fmt = gk.E4M3 if d == 128 else gk.E2M1
    G, H, groups, counts = P.several_groups(kind)
    sh = Large(kind, G, H, groups, counts, seed=71)
    lens = torch.randint(0, 60, (sh.n,), generator=torch.Generator().manual_seed(5)).tolist()
    lens[1] = 2000
    c = Cache(dtype, d, fmt, G, H, lens, 16, seed=70)
    sh.q = c.q
    out, lse = c.call(part=sh.call())
    _joined(c, sh, out, lse, c.entries, 3, dtype, d)


class Captured:
    """A call of one kernel on tensors that stay where they are."""

    def __init__(self, c, ws):
        self.c, self.pre, self.q, self.cu = c, c.packed(), c.q.cuda(), c.cu.cuda()
        self.cfg = gk.shared_config(self.q, c.G, len(c.groups))
        self.ws = torch.empty(gk.shared_ws_bytes(self.cfg), dtype=torch.uint8, device="cuda") if ws is None else ws
        self.part = gk.Part(torch.full((c.n, c.H, c.d), 7.0, device="cuda"), torch.full((c.n, c.H), 7.0, device="cuda"))

    def run(self, stream=None):
        gk.shared_attention(self.cfg, self.q, self.cu, self.pre, self.part, self.ws, stream=stream)

    def capture(self, side):
        side.wait_stream(torch.cuda.current_stream())
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph, stream=side):
            self.run()


@pytest.mark.parametrize("kind", P.KINDS)
def test_large_captured_and_replayed(kind):
    c = Large(kind, *P.several_groups(kind), seed=80)
    a, side = Captured(c, None), torch.cuda.Stream()
    a.capture(side)
    n, S_ = c.n, len(c.groups)
    r = torch.Generator().manual_seed(3)
    for i in range(5):
        cut = sorted(torch.randint(0, n + 1, (S_ - 1,), generator=r).tolist())
        c.cu = torch.tensor([0] + cut + [n], dtype=torch.int32)
        c.groups = [int(y - x) for x, y in zip(c.cu[:-1], c.cu[1:])]
        c.q = torch.randn(c.q.shape, generator=r).to(c.q.dtype)
        a.q.copy_(c.q)
        a.cu.copy_(c.cu)
        a.part.o.fill_(7.0)
        a.part.lse.fill_(7.0)
        torch.cuda.synchronize()
        a.graph.replay()
        torch.cuda.synchronize()
        got = a.part.o.clone(), a.part.lse.clone()
        c.check(gk.Part(*got))
        a.run(side)                                                # eager, on the side stream
        side.synchronize()
        assert torch.equal(got[0], a.part.o) and torch.equal(got[1], a.part.lse)


def test_large_graphs_in_turn_on_one_workspace():
    ws, side = torch.full((256 << 20,), 255, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    calls = [Captured(Large(kind, *P.several_groups(kind), seed=81), ws) for kind in P.KINDS]
    want = []
    for x in calls:
        x.run()
        torch.cuda.synchronize()
        want.append((x.part.o.clone(), x.part.lse.clone()))
        x.capture(side)
    for _ in range(3):
        for x in calls:
            x.part.o.fill_(7.0)
            x.graph.replay()
        torch.cuda.synchronize()
        for x, (o, lse) in zip(calls, want):
            assert torch.equal(x.part.o, o) and torch.equal(x.part.lse, lse)


def test_large_calls_at_once_on_two_streams():
    for kind in P.KINDS:
        c = Large(kind, *P.several_groups(kind), seed=82)
        a, b, w = Captured(c, None), Captured(c, None), Captured(c, None)
        w.run()
        sides = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        for _ in range(10):
            for x, stream in zip((a, b), sides):
                x.run(stream)
        torch.cuda.synchronize()
        for x in (a, b):
            assert torch.equal(x.part.o, w.part.o) and torch.equal(x.part.lse, w.part.lse)


def test_one_layer_of_several_in_the_arrays():
    # the arrays' slice of one layer, which begins on no boundary of log m, and the whole of them: another kernel each, and
    # rows of other layers that are NaN
    for kind in P.KINDS:
        G, H, groups = P.one_group(kind)[1]
        c = Large(kind, G, H, groups, [300, 129], seed=40)
        whole = c.packed()
        a = int(whole.start[0]) - 1
        n = int(c.pre["count"].sum()) + 2
        one = gk.Prefix(whole.start - a, whole.count, whole.K[a:a + n], whole.V[a:a + n], whole.logm[a:a + n])
        assert P.kernel(c.dtype, c.d, G, H, c.n, 1, n)[0] == "few" and whole.logm[a:].data_ptr() % 16
        c.check(c.call(prefix=one))
        c.check(c.call(prefix=whole))
