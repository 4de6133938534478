"""Attention over prompts, appending to pages and attention over pages on the GPU,
against plain float64 forms; tolerances count roundings (serve_harness)."""
import itertools
import math

import pytest
import torch

import gpu_harness as H
import serve_harness as S
from paper_2608_07001_amd import gracekv as gk
from synth.workloads import make_case, small_shape

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HEADS = [(2, 8), (1, 1), (3, 15), (2, 34), (1, 7)]
TYPES = [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)]


def _rand(gen, *shape, dtype="bf16", scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(DT[dtype])


def _cu(lens):
    return torch.tensor([0] + list(lens), dtype=torch.int32).cumsum(0).to(torch.int32)


# ---------------------------------------------------------------------------
# prompts


def _prompt(q, k, v, cu_q, cu_k, layout="token", poison=True):
    """The call on copies of CPU tensors; workspace and outputs start as NaN or 7."""
    qd, kd, vd = (S.laid(x.cuda(), layout) for x in (q, k, v))
    out = S.laid(torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), layout)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    cfg = gk.prompt_config(qd, kd, vd, out, cu_q.numel() - 1)
    n = gk.prompt_ws_bytes(cfg)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None
    gk.prompt_attention(cfg, qd, kd, vd, cu_q.cuda(), cu_k.cuda(), out, ws, lse=lse)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu(), n > 0


def _check_prompt(dtype, d, G, Hq, lq, lk, layout="token", behind=0, seed=0, edit=None, scale=1.5):
    gen = torch.Generator().manual_seed(seed)
    q = _rand(gen, sum(lq) + behind, Hq, d, dtype=dtype, scale=scale)
    k, v = (_rand(gen, sum(lk) + behind, G, d, dtype=dtype) for _ in range(2))
    if edit:
        edit(q, k, v)
    out, lse, split = _prompt(q, k, v, _cu(lq), _cu(lk), layout)

    def check(rows, h, ref, m):
        S.check_rows(out[rows, h], lse[rows, h], ref, max(m, 1), d, dtype == "bf16", (dtype, d, G, Hq, rows, h))
    S.prompt64(q.double(), k.double(), v.double(), lq, lk, check)
    assert (out[sum(lq):] == 7).all() and (lse[sum(lq):] == 7).all()       # behind the last sequence
    return split


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("G,Hq", HEADS)
def test_prompt_packed(dtype, d, G, Hq):
    _check_prompt(dtype, d, G, Hq, [1, 0, 31, 33, 64, 2, 127], [1, 0, 31, 33, 64, 2, 127], behind=3, seed=Hq)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("layout", ["token", "head", "wide"])
def test_prompt_layouts(dtype, d, layout):
    _check_prompt(dtype, d, 2, 6, [65, 17, 130], [65, 17, 130], layout, behind=2, seed=3)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_every_length(dtype, d):
    for n in (1, 2, 15, 16, 17, 32, 63, 65, 95, 96, 128, 129, 191, 257):
        _check_prompt(dtype, d, 1, 2, [n], [n], seed=n)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_later_pieces_and_rows_with_no_key(dtype, d):
    # a question's window, a chunk, no cached key at all, more queries than keys, no query
    _check_prompt(dtype, d, 2, 8, [7, 40, 9, 50, 0, 1], [300, 41, 0, 21, 64, 130], behind=1, seed=5)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_split_over_the_keys(dtype, d):
    split = _check_prompt(dtype, d, 2, 8, [5], [3001], seed=6)
    split &= _check_prompt(dtype, d, 1, 4, [3, 0, 2], [1500, 10, 700], behind=2, seed=7)
    split &= _check_prompt(dtype, d, 1, 1, [600], [600], seed=8)
    assert split


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_long(dtype, d):
    split = _check_prompt(dtype, d, 1, 1, [1999], [1999], seed=9)
    assert split
    assert not _check_prompt(dtype, d, 8, 32, [1030, 1030], [1030, 1030], seed=10) or dtype == "f32"


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_piece_over_the_longest_contexts(dtype, d):
    # a few queries over 128K keys, alone and beside short ones; values that rise along the keys
    def edit(q, k, v):
        v += torch.linspace(0, 4, v.shape[0])[:, None, None].to(v.dtype)
    assert _check_prompt(dtype, d, 1, 4, [5], [131072 + 5], seed=25, edit=edit)
    assert _check_prompt(dtype, d, 2, 4, [3, 1, 9], [40, 131072, 9], "head", seed=26, edit=edit)


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_whole_context(d):
    # a prefill of 128K tokens: rows from all over it against float64
    n = 131072 + 33
    gen = torch.Generator().manual_seed(27)
    q, k, v = _rand(gen, n, 2, d, scale=1.5), _rand(gen, n, 1, d), _rand(gen, n, 1, d)
    v += torch.linspace(0, 4, n)[:, None, None].to(v.dtype)
    out, lse, _ = _prompt(q, k, v, _cu([n]), _cu([n]))
    rows = torch.cat([torch.tensor([0, 1, 63, 64, 4095, 65535, 65536, n - 33, n - 1]), torch.randint(0, n, (40,), generator=gen)])
    k64, v64 = k[:, 0].double(), v[:, 0].double()
    for i in rows.tolist():
        S.check_rows(out[i], lse[i], S.attend64(q[i].double(), k64[:i + 1], v64[:i + 1]), i + 1, d, True, i)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,Hq,lq,lk", [(1, 32, 259, 259), (1, 2, 259, 259), (1, 2, 6, 259)])
def test_prompt_far_rows(dtype, G, Hq, lq, lk):
    """Rows 2^24 elements apart, the longest distance of keys and values: the last lie past 32 bits of elements,
    in pairs (bf16, 32 heads), single waves and parts (fp32); then heads 2^32 elements apart.  Appending likewise."""
    d, far = 128, 1 << 24
    gen = torch.Generator().manual_seed(28)
    q, k, v = (_rand(gen, n, x, d, dtype=dtype) for n, x in ((lq, Hq), (lk, G), (lk, G)))
    pool = torch.empty((lk + 1) * far, dtype=DT[dtype], device="cuda")

    def place(x, at):                                          # rows of all heads, `far` apart
        y = pool[at:].as_strided(x.shape, (far, d, 1))
        return y.copy_(x)
    room = 32 * d + 8
    qd, kd, vd, out = place(q, 0), place(k, room), place(v, 2 * room), place(torch.full_like(q, 7), 3 * room)
    lse = torch.empty(lq, Hq, device="cuda")

    def run(qd, kd, vd, out):
        cfg = gk.prompt_config(qd, kd, vd, out, 1)
        ws = torch.full((max(gk.prompt_ws_bytes(cfg), 1),), 255, dtype=torch.uint8, device="cuda")
        gk.prompt_attention(cfg, qd, kd, vd, _cu([lq]).cuda(), _cu([lk]).cuda(), out, ws, lse=lse)
        got, got_lse = out.cpu(), lse.cpu()
        S.prompt64(q.double(), k.double(), v.double(), [lq], [lk],
                   lambda rows, h, ref, m: S.check_rows(got[rows, h], got_lse[rows, h], ref, m, d, dtype == "bf16", (dtype, Hq, h)))
    run(qd, kd, vd, out)
    table = torch.arange(17, dtype=torch.int32, device="cuda")[None]
    K = torch.zeros(17, G, 16, d, dtype=DT[dtype], device="cuda")
    V = torch.zeros_like(K)
    gk.cache_append(gk.page_config(K, Hq, table), kd, vd, K, V, table, torch.zeros(1, dtype=torch.int32, device="cuda"), _cu([lk]).cuda())
    for got, want in ((K, k), (V, v)):
        assert torch.equal(got.transpose(1, 2).reshape(-1, G, d)[:lk].cpu(), want)
    if Hq == 2:                                                # the second head past 32 bits
        two = lambda x, at: pool[at:].as_strided(x.shape, (d, 1 << 32, 1)).copy_(x)      # noqa: E731
        run(two(q, 0), place(k, room << 4), place(v, room << 5), two(torch.full_like(q, 7), 1 << 20))


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_broadcast_rows_and_heads(dtype, d):
    # strides of 0: one query, key or value for all tokens, or for all heads
    gen = torch.Generator().manual_seed(29)
    for G, Hq, lq, lk in ((2, 8, [70, 1, 33], [70, 40, 33]), (8, 32, [600], [600]), (2, 4, [3], [2500])):
        n, m = sum(lq), sum(lk)
        for which in range(3):
            q = _rand(gen, n if which else 1, Hq, d, dtype=dtype).expand(n, Hq, d)
            k = _rand(gen, m, 1 if which else G, d, dtype=dtype).expand(m, G, d)
            v = _rand(gen, 1 if which == 2 else m, G, d, dtype=dtype).expand(m, G, d)
            if which == 0:
                k = k[:1].expand(m, G, d)
            out, lse = torch.full((n, Hq, d), 7.0, dtype=DT[dtype], device="cuda"), torch.full((n, Hq), 7.0, device="cuda")
            dev = [x.cuda() if 0 not in x.stride() else x[:1 if x.stride(0) == 0 else None, :1 if x.stride(1) == 0 else None].cuda().expand(x.shape)
                   for x in (q, k, v)]
            assert [x.stride() for x in dev] != [x.contiguous().stride() for x in dev]
            cfg = gk.prompt_config(*dev, out, len(lq))
            ws = torch.full((max(gk.prompt_ws_bytes(cfg), 1),), 255, dtype=torch.uint8, device="cuda")
            gk.prompt_attention(cfg, *dev, _cu(lq).cuda(), _cu(lk).cuda(), out, ws, lse=lse)
            got, got_lse = out.cpu(), lse.cpu()
            S.prompt64(q.double(), k.double(), v.double(), lq, lk,
                       lambda rows, h, ref, mm: S.check_rows(got[rows, h], got_lse[rows, h], ref, mm, d, dtype == "bf16", (which, h)))


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_waves_in_pairs(d):
    # few short prompts of many heads: two waves to the same rows; odd ends, a row with no key, infinities
    assert not _check_prompt("bf16", d, 8, 32, [700, 0, 3, 321, 1], [700, 0, 3, 321, 1], behind=2, seed=20)
    assert not _check_prompt("bf16", d, 8, 40, [33, 500, 330], [1, 530, 330], "head", seed=21)

    def edit(q, k, v):
        v[417, 3, 5], v[40, 0, 1], v[-1, 7] = math.inf, math.nan, -math.inf
    assert not _check_prompt("bf16", d, 8, 32, [418, 607], [418, 607], seed=22, edit=edit)


@pytest.mark.parametrize("d", [64, 128])
def test_prompt_between_pairs_and_parts(d):
    # lengths and head counts on both sides of every rule that chooses the kernel and the parts
    for i, (G, Hq, lq, lk) in enumerate([(8, 32, [127], None), (8, 32, [256], None), (8, 32, [511, 2], None), (4, 16, [700], None),
                                         (4, 16, [200], [1000]), (4, 32, [256], [1400]), (8, 32, [3, 60, 0, 300, 20], None),
                                         (1, 8, [1000, 900, 700], None), (2, 16, [5, 700], [2100, 705])]):
        _check_prompt("bf16", d, G, Hq, lq, lk or lq, seed=40 + i)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_prompt_masked_places_reach_nothing(dtype, d, bad):
    # a value (and a key) that is not finite: the queries before it do not see it, those
    # from it on do; rows behind the last sequence and between tiles likewise
    for at in (0, 40, 70, 99):
        def edit(q, k, v):
            v[at, 0, 3] = bad
            v[100:, :, :] = bad            # the second sequence has its own, and rows behind it
            v[100:160] = 1.0
            k[160:] = bad
        _check_prompt(dtype, d, 1, 3, [100, 60], [100, 60], behind=9, seed=11, edit=edit)

    def late(q, k, v):                     # the last key: its own query alone sees it
        v[-1, :, -1] = bad
    _check_prompt(dtype, d, 2, 4, [333], [333], seed=12, edit=late)
    if not math.isnan(bad):                # a key that gives the queries after it no number, and the ones before their own
        gen = torch.Generator().manual_seed(13)
        q, k, v = _rand(gen, 90, 2, d, dtype=dtype), _rand(gen, 90, 1, d, dtype=dtype), _rand(gen, 90, 1, d, dtype=dtype)
        k[50] = math.nan
        out, lse, _ = _prompt(q, k, v, _cu([90]), _cu([90]))
        assert torch.isnan(out[50:]).all() and torch.isnan(lse[50:]).all() and torch.isfinite(out[:50]).all()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_large_logits(dtype, d):
    # logits in the hundreds, rising and falling along the keys: the maximum moves all the way
    def edit(q, k, v):
        q[:] = 1.0
        k[:] = (torch.arange(k.shape[0]).float() - 150)[:, None, None] / 8
    _check_prompt(dtype, d, 1, 2, [300], [300], seed=14, edit=edit)

    def fall(q, k, v):
        q[:] = -1.0
        k[:] = (torch.arange(k.shape[0]).float() - 150)[:, None, None] / 8
    _check_prompt(dtype, d, 1, 2, [300], [300], seed=15, edit=fall)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_large_values_stay_finite(dtype, d):
    """Values of 5e34 at keys whose logits rise and fall by 5 from block to block: averages of up to 2000
    of them at weights up to 1 stay below 1.1e38, so no sum on the way passes fp32's range (weights of
    e^5 beside a first block of weight 1 would, from 64 keys on).  One part, pairs, several parts."""
    def edit(q, k, v):
        q[:] = 1.0
        k[:] = ((torch.arange(k.shape[0]) // 64 % 2) * 5.0 / math.sqrt(d))[:, None, None]
        v.abs_().add_(0.5).mul_(5e34)
    _check_prompt(dtype, d, 1, 1, [200], [200], seed=18, edit=edit)
    _check_prompt(dtype, d, 8, 32, [1024], [1024], seed=19, edit=edit)
    assert _check_prompt(dtype, d, 2, 4, [5], [4000], seed=20, edit=edit)


def test_prompt_malformed_starts_stay_inside():
    # starts outside the rows, and descending: held inside, the call ends, rows before stay right
    gen = torch.Generator().manual_seed(1)
    q, k, v = _rand(gen, 70, 2, 64), _rand(gen, 70, 1, 64), _rand(gen, 70, 1, 64)
    for cu in ([0, 30, 1000], [-9, 30, 70], [0, 30, 20], [0, 80, 90]):
        c = torch.tensor(cu, dtype=torch.int32)
        out, lse, _ = _prompt(q, k, v, c, c)
        n = min(cu[1], 70)
        want = S.attend64(q[:n, 0].double(), k[:n, 0].double(), v[:n, 0].double(), seen=torch.ones(n, n).tril().bool())
        S.check_rows(out[:n, 0], lse[:n, 0], want, n, 64, True, cu)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_descending_starts_stay_inside(dtype, d):
    """A descending pair between sequences of several tiles, alone and among more sequences than one
    look of the search: the call ends and writes to rows of its sequences only."""
    gen = torch.Generator().manual_seed(16)
    for lead in (0, 100):
        cu = torch.tensor([10] * lead + [10, 500, 200, 900], dtype=torch.int32)
        q, k, v = _rand(gen, 1000, 2, d, dtype=dtype), _rand(gen, 1000, 1, d, dtype=dtype), _rand(gen, 1000, 1, d, dtype=dtype)
        wide = torch.full((1000, 4, d + 16), 7.0, dtype=DT[dtype], device="cuda")
        out, lse = wide[:, 1:3, 8:-8], torch.full((1000, 2), 7.0, device="cuda")
        cfg = gk.prompt_config(q, k, v, out, cu.numel() - 1)
        ws = torch.full((max(gk.prompt_ws_bytes(cfg), 1),), 0, dtype=torch.uint8, device="cuda")
        gk.prompt_attention(cfg, q.cuda(), k.cuda(), v.cuda(), cu.cuda(), cu.cuda(), out, ws, lse=lse)
        torch.cuda.synchronize()
        out[10:900], lse[10:900] = 7.0, 7.0
        assert (wide == 7).all() and (lse == 7).all()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_prompt_many_sequences(dtype, d):
    # more sequences than one look of the search (64), and than two (64 * 64), empty ones among them
    for B, most, seed in ((65, 40, 1), (200, 9, 2), (4200, 3, 3)):
        lens = torch.randint(0, most, (B,), generator=torch.Generator().manual_seed(seed)).tolist()
        lens[-1] = 150
        gen = torch.Generator().manual_seed(seed)
        n = sum(lens) + 2
        q, k, v = _rand(gen, n, 2, d, dtype=dtype, scale=1.5), _rand(gen, n, 1, d, dtype=dtype), _rand(gen, n, 1, d, dtype=dtype)
        out, lse, _ = _prompt(q, k, v, _cu(lens), _cu(lens))
        looked = set(range(B)) if B < 300 else set(range(0, B, 97)) | {B - 2, B - 1}
        a = 0
        for b, m in enumerate(lens):
            if b in looked and m:
                for h in range(2):
                    ref = S.attend64(q[a:a + m, h].double(), k[a:a + m, 0].double(), v[a:a + m, 0].double(), seen=torch.ones(m, m).tril().bool())
                    S.check_rows(out[a:a + m, h], lse[a:a + m, h], ref, m, d, dtype == "bf16", (B, b, h))
            a += m
        assert torch.isfinite(lse).all() and (out[a:] == 7).all() and (lse[a:] == 7).all()
        assert not (lse[:a] == 7).any()


def test_prompt_nothing_to_do():
    q, k = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    cu = torch.zeros(4, dtype=torch.int32, device="cuda")
    cfg = gk.prompt_config(q, k, k, q, 3)
    gk.prompt_attention(cfg, q, k, k, cu, cu, q)
    x = torch.ones(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(x, 7), torch.full((3, 4), 7.0, device="cuda")
    cfg = gk.prompt_config(x, k, k, out, 3)                    # queries without a single key
    gk.prompt_attention(cfg, x, k, k, torch.tensor([0, 1, 1, 2], dtype=torch.int32, device="cuda"), cu, out, lse=lse)
    assert (out[:2] == 0).all() and (lse[:2] == -math.inf).all() and (out[2] == 7).all() and (lse[2] == 7).all()


# ---------------------------------------------------------------------------
# append


def _tables(gen, need, page, extra=2):
    """Page ids in no order, -1 where a row of the table has no page, and the number of pages."""
    n = [-(-x // page) for x in need]
    total, width = sum(n) + extra, max(max(n), 1)
    ids = torch.randperm(total, generator=gen).to(torch.int32)
    table = torch.full((len(need), width), -1, dtype=torch.int32)
    at = 0
    for b, x in enumerate(n):
        table[b, :x] = ids[at:at + x]
        at += x
    return table, total


def _rope(rows, d):
    ang = torch.arange(rows, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    return ang.cos().float(), ang.sin().float()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("G,Hq", [(2, 8), (1, 1), (3, 15)])
@pytest.mark.parametrize("page,layout", [(16, "token"), (32, "head"), (256, "wide")])
def test_append(dtype, d, G, Hq, page, layout):
    gen = torch.Generator().manual_seed(page + Hq)
    start, new = [0, 15, 16, 33, 250, 5], [1, 2, 40, 0, 17, 1]
    n = sum(new) + 2                                           # two rows behind the last sequence
    table, n_pages = _tables(gen, [a + b for a, b in zip(start, new)], page)
    k, v, q = (_rand(gen, n, x, d, dtype=dtype) for x in (G, G, Hq))
    pos = torch.randint(0, 400, (n,), generator=gen).to(torch.int32)
    cos, sin = _rope(400, d)
    pool = torch.randn(n_pages, 3, G, page, d, generator=gen).to(DT[dtype])     # the middle layer of a pool of three
    K, V = pool.clone(), pool.clone() + 1
    Kd, Vd, q_out = K.cuda(), V.cuda(), S.laid(torch.full((n, Hq, d), 7.0, dtype=DT[dtype], device="cuda"), layout)
    cfg = gk.page_config(Kd[:, 1], Hq, table)
    gk.cache_append(cfg, S.laid(k.cuda(), layout), S.laid(v.cuda(), layout), Kd[:, 1], Vd[:, 1], table.cuda(),
                    torch.tensor(start, dtype=torch.int32).cuda(), _cu(new).cuda(), pos.cuda(), cos.cuda(), sin.cuda(),
                    S.laid(q.cuda(), layout), q_out)
    torch.cuda.synchronize()
    kr, qr = (S.rotate64(x.double(), cos[pos.long()].double(), sin[pos.long()].double()) for x in (k, q))
    eps = S.B16 if dtype == "bf16" else S.U
    # two products and a sum in fp32, rounded to the type: 3 u of |x c| + |y s|, then half a step of the value
    ks, qs = k.double().abs().amax() * 6 * S.U + eps * kr.abs(), q.double().abs().amax() * 6 * S.U + eps * qr.abs()
    want_K, want_V, tol = K.double(), V.clone(), torch.zeros_like(K, dtype=torch.float64)
    i = 0
    for b, (a, m) in enumerate(zip(start, new)):
        for j in range(m):
            p, at = int(table[b, (a + j) // page]), (a + j) % page
            want_K[p, 1, :, at], tol[p, 1, :, at], want_V[p, 1, :, at] = kr[i], ks[i], v[i]
            i += 1
    assert ((Kd.cpu().double() - want_K).abs() <= tol).all()   # exact where nothing was written
    assert torch.equal(Vd.cpu(), want_V)
    got = q_out.cpu().double()
    assert ((got[:i] - qr[:i]).abs() <= qs[:i]).all() and (got[i:] == 7).all()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_append_without_rotation_or_queries(dtype, d):
    gen = torch.Generator().manual_seed(2)
    table, n_pages = _tables(gen, [20, 40], 16)
    k, v = _rand(gen, 23, 2, d, dtype=dtype), _rand(gen, 23, 2, d, dtype=dtype)
    k[0, 0, 0], k[1, 1, 1], v[2, 0, 2] = math.nan, math.inf, -math.inf
    K = torch.zeros(n_pages, 2, 16, d, dtype=DT[dtype], device="cuda")
    V = torch.zeros_like(K)
    gk.cache_append(gk.page_config(K, 4, table), k.cuda(), v.cuda(), K, V, table.cuda(), torch.tensor([10, 27], dtype=torch.int32).cuda(),
                    _cu([10, 13]).cuda())
    rows = torch.cat([torch.stack([table[0, (10 + torch.arange(10)) // 16], (10 + torch.arange(10)) % 16], 1),
                      torch.stack([table[1, (27 + torch.arange(13)) // 16], (27 + torch.arange(13)) % 16], 1)]).long()
    for got, want in ((K, k), (V, v)):
        assert torch.equal(got.cpu()[rows[:, 0], :, rows[:, 1]].view(torch.int16), want.view(torch.int16))     # bit for bit
        assert int((got.view(torch.int32) != 0).any(-1).sum()) <= 23 * 2


def test_append_in_place_and_left_out_tokens():
    # q_out = q; tokens whose place has no page, or whose position has no row, change nothing
    gen = torch.Generator().manual_seed(3)
    d, page = 64, 16
    table = torch.tensor([[0, -1, 9], [2, 1, 3]], dtype=torch.int32)           # nine pages: id 9 is none
    start, new = [14, 44], [22, 9]                                           # places 14..35 and 44..52 (48 on: past the table)
    n = sum(new)
    k, v, q = (_rand(gen, n, x, d) for x in (1, 1, 2))
    pos = torch.arange(n, dtype=torch.int32)
    pos[1], pos[24], pos[25] = -1, 100, 2 ** 31 - 1
    cos, sin = _rope(100, d)
    K = torch.full((9, 1, page, d), 5.0, dtype=torch.bfloat16, device="cuda")
    V, qd = K.clone(), q.cuda()
    gk.cache_append(gk.page_config(K, 2, table), k.cuda(), v.cuda(), K, V, table.cuda(), torch.tensor(start, dtype=torch.int32).cuda(),
                    _cu(new).cuda(), pos.cuda(), cos.cuda(), sin.cuda(), qd, qd)
    kept = [i for i in range(n) if i not in (1, 24, 25) and ((i < 22 and 14 + i < 16) or (i >= 22 and i - 22 + 44 < 48))]
    assert kept == [0, 22, 23]
    want_V = torch.full((9, 1, page, d), 5.0, dtype=torch.bfloat16)
    for i in kept:
        place = 14 + i if i < 22 else i - 22 + 44
        want_V[table[0 if i < 22 else 1, place // page], :, place % page] = v[i]
    assert torch.equal(V.cpu(), want_V)
    assert torch.equal((K.cpu() != 5).any(-1).any(1), (want_V != 5).any(-1).any(1))
    qr = S.rotate64(q.double(), cos[pos.long() % 100].double(), sin[pos.long() % 100].double())
    for i in range(n):
        if i in kept:
            assert ((qd[i].cpu().double() - qr[i]).abs() <= S.B16 * qr[i].abs() + 1e-6 * 6).all()
        else:
            assert torch.equal(qd[i].cpu(), q[i])


def test_append_many_sequences():
    # more sequences than a wave looks at in one step, empty ones among them
    gen = torch.Generator().manual_seed(4)
    B, d, page = 5000, 64, 16
    new = torch.randint(0, 3, (B,), generator=gen)
    start = torch.randint(0, 30, (B,), generator=gen).to(torch.int32)
    table = torch.randperm(2 * B, generator=gen).to(torch.int32).view(B, 2)
    n = int(new.sum())
    k = _rand(gen, n, 1, d)
    K = torch.zeros(2 * B, 1, page, d, dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    gk.cache_append(gk.page_config(K, 1, table), k.cuda(), k.cuda(), K, V, table.cuda(), start.cuda(), _cu(new.tolist()).cuda())
    b = torch.repeat_interleave(torch.arange(B), new)
    place = start.long()[b] + torch.arange(n) - (new.cumsum(0) - new)[b]
    want = torch.zeros(2 * B, 1, page, d, dtype=torch.bfloat16)
    on = place < 2 * page
    want[table.long()[b[on], place[on] // page], 0, place[on] % page] = k[on, 0]
    assert torch.equal(K.cpu(), want) and torch.equal(V.cpu(), want)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_append_nothing(dtype, d):
    # a step in which no sequence has a new token, with and without queries and rotation
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    K = torch.full((4, 2, 16, d), 5.0, dtype=DT[dtype], device="cuda")
    V, start, cu = K.clone(), torch.tensor([3, 20], dtype=torch.int32, device="cuda"), _cu([0, 0]).cuda()
    cfg = gk.page_config(K, 4, table)
    cos, sin = (x.cuda() for x in _rope(50, d))
    k, q = torch.ones(0, 2, d, dtype=DT[dtype], device="cuda"), torch.ones(0, 4, d, dtype=DT[dtype], device="cuda")
    pos = torch.zeros(0, dtype=torch.int32, device="cuda")
    gk.cache_append(cfg, k, k, K, V, table, start, cu, pos, cos, sin, q, q.clone())
    gk.cache_append(cfg, k, k, K, V, table, start, cu, pos, cos, sin)
    gk.cache_append(cfg, k, k, K, V, table, start, cu)
    assert (K == 5).all() and (V == 5).all()


def test_append_descending_starts_stay_inside():
    # a token lands in its own place of a sequence that could hold it, or nowhere
    gen = torch.Generator().manual_seed(17)
    d, page, n = 64, 16, 70
    cu = [0, 40, 20, 60]                                       # the middle sequence is none, the others overlap
    table = torch.randperm(9, generator=gen).to(torch.int32).view(3, 3)
    k = _rand(gen, n, 1, d)
    K = torch.full((12, 1, page, d), 5.0, dtype=torch.bfloat16, device="cuda")
    V = K.clone()
    gk.cache_append(gk.page_config(K, 1, table), k.cuda(), k.cuda(), K, V, table.cuda(), torch.zeros(3, dtype=torch.int32).cuda(),
                    torch.tensor(cu, dtype=torch.int32).cuda())
    assert torch.equal(K, V)
    K = K.cpu()
    for b in range(3):
        for place in range(3 * page):
            row, t = K[table[b, place // page], 0, place % page], cu[b] + place
            assert (row == 5).all() or (b != 1 and place < 40 and torch.equal(row, k[t, 0])), (b, place)
    assert (K[9:] == 5).all()


# ---------------------------------------------------------------------------
# pages


class Cache:
    """A paged cache with ragged lengths and, if asked, packed entries in front, on the CPU."""

    def __init__(self, dtype, d, G, Hq, lens, page, counts=None, seed=0, share=False):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.d, self.G, self.H, self.lens, self.page = dtype, d, G, Hq, list(lens), page
        self.table, n_pages = _tables(gen, lens, page)
        self.K, self.V = (_rand(gen, n_pages, G, page, d, dtype=dtype) for _ in range(2))
        self.q = _rand(gen, len(lens), Hq, d, dtype=dtype, scale=1.5)
        self.len = torch.tensor(lens, dtype=torch.int32)
        self.pre = None
        if counts is not None:
            c = torch.tensor(counts, dtype=torch.int64)
            n = int(c.sum()) + 3
            start = torch.zeros_like(c) if share else c.cumsum(0) - c
            self.pre = dict(start=start, count=c, K=_rand(gen, n, d, dtype=dtype), V=_rand(gen, n, d, dtype=dtype),
                            logm=torch.rand(n, generator=gen) * 4)

    def call(self, out=None, ws=None):
        g = lambda x: x.cuda()                                   # noqa: E731
        table = g(self.table)
        K, V = g(self.K), g(self.V)
        cfg = gk.page_config(K, self.H, table)
        out = torch.full(self.q.shape, 7.0, dtype=DT[self.dtype], device="cuda") if out is None else out
        lse = torch.full(self.q.shape[:2], 7.0, device="cuda")
        ws = torch.full((gk.paged_ws_bytes(cfg),), 255, dtype=torch.uint8, device="cuda") if ws is None else ws
        pre = None if self.pre is None else gk.Prefix(**{k: g(x) for k, x in self.pre.items()})
        q = S.laid(g(self.q), "token")
        wide = torch.full((q.shape[0], self.H + 3, self.d), float("nan"), dtype=q.dtype, device="cuda")
        wide[:, :self.H] = q
        gk.paged_attention(cfg, wide[:, :self.H], K, V, table, g(self.len), out, ws, lse=lse, prefix=pre)
        torch.cuda.synchronize()
        return out.cpu(), lse.cpu()

    def entries(self, b, g):
        """Keys, values and log m of (b, g), in order (float64)."""
        n = max(0, min(int(self.len[b]), self.table.shape[1] * self.page))
        ids = self.table[b].long()
        k, v = (torch.cat([x[i, g] if 0 <= i < x.shape[0] else torch.zeros(self.page, self.d) for i in ids.tolist()])[:n].double()
                for x in (self.K, self.V))
        ok = torch.tensor([0 <= int(ids[t // self.page]) < self.K.shape[0] for t in range(n)], dtype=torch.bool)
        lm = torch.zeros(n, dtype=torch.float64)
        lm[~ok] = -math.inf
        if self.pre is not None:
            a = int(self.pre["start"][b * self.G + g])
            e = a + int(self.pre["count"][b * self.G + g])
            k, v = torch.cat([self.pre["K"][a:e].double(), k]), torch.cat([self.pre["V"][a:e].double(), v])
            lm = torch.cat([self.pre["logm"][a:e].double(), lm])
        return k, v, lm

    def check(self, got=None):
        out, lse = got or self.call()
        per = self.H // self.G
        for b, g in itertools.product(range(len(self.lens)), range(self.G)):
            k, v, lm = self.entries(b, g)
            h = slice(g * per, (g + 1) * per)
            S.check_rows(out[b, h], lse[b, h], S.attend64(self.q[b, h].double(), k, v, bias=lm), max(len(k), 1), self.d,
                         self.dtype == "bf16", (self.dtype, self.d, self.G, self.H, b, g))


LENS = [0, 1, 15, 16, 17, 31, 32, 33, 100, 257]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("G,Hq", HEADS)
@pytest.mark.parametrize("page", [16, 64])
def test_paged(dtype, d, G, Hq, page):
    Cache(dtype, d, G, Hq, LENS, page, seed=Hq).check()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("G,Hq", [(2, 8), (3, 15)])
@pytest.mark.parametrize("page", [32, 128, 256])
def test_paged_with_packed_entries(dtype, d, G, Hq, page):
    gen = torch.Generator().manual_seed(1)
    counts = torch.randint(0, 70, (len(LENS) * G,), generator=gen).tolist()
    counts[0], counts[1], counts[5] = 0, 1, 600
    Cache(dtype, d, G, Hq, LENS, page, counts, seed=Hq).check()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_paged_long_and_split(dtype, d):
    # rows of many chunks beside rows of one; the sum of all is past what one chunk takes
    c = Cache(dtype, d, 2, 8, [4001, 3, 0, 9000, 64], 16, [5, 3000, 0, 0, 1, 2, 700, 0, 0, 33], seed=4)
    c.check()
    one = Cache(dtype, d, 1, 4, [20000], 64, seed=5)
    one.check()
    # lengths on the device decide: the same buffers and shapes with short rows
    one.len[0] = 70
    one.check()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_paged_masked_entries(dtype, d):
    # log m = -inf, alone and for whole rows; what is masked, past the end or in a missing page holds NaN and infinities
    for what in ("some", "head", "all"):
        c = Cache(dtype, d, 2, 6, [40, 0, 5], 16, [50, 3, 20, 33, 0, 64], seed=6)
        lm = c.pre["logm"]
        mask = torch.zeros_like(lm, dtype=torch.bool)
        mask[{"some": slice(0, None, 3), "head": slice(0, 53), "all": slice(0, None)}[what]] = True
        lm[mask] = -math.inf
        c.pre["V"][mask] = math.nan
        c.pre["K"][mask, ::2] = math.inf
        c.table[0, 1] = -1                                     # places 16 .. 31 of the first sequence have no page
        used = torch.zeros(c.K.shape[0], dtype=torch.bool)
        used[c.table[c.table >= 0].long()] = True
        c.K[~used], c.V[~used] = math.nan, math.inf
        c.K[c.table[0, 2].long(), :, 8:] = math.nan            # past place 40
        c.V[c.table[0, 2].long(), :, 8:] = -math.inf
        c.V[c.table[2, 0].long(), :, 5:] = math.nan
        c.check()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_paged_lowest_log_m(dtype, d):
    # the type's lowest value as a mask: no weight beside other entries, equal weights among themselves
    c = Cache(dtype, d, 1, 3, [9, 0], 16, [40, 37], seed=7)
    c.q[:] = 0.0
    c.pre["logm"][:] = torch.finfo(torch.float32).min
    c.pre["logm"][3] = 0.5
    out, lse = c.call()
    per = slice(0, 3)
    k, v, lm = c.entries(0, 0)
    S.check_rows(out[0, per], lse[0, per], S.attend64(c.q[0, per].double(), k, v, bias=lm), 49, d, dtype == "bf16", "beside others")
    k, v, _ = c.entries(1, 0)
    tol = (S.B16 * 2 if dtype == "bf16" else 1e-5) * v.abs().mean(0) + 1e-6
    assert ((out[1, per].double() - v.mean(0)).abs() <= tol).all()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf])
def test_paged_infinite_values_stay_in_their_dimension(dtype, d, bad):
    c = Cache(dtype, d, 2, 8, [70, 1, 33], 16, [40, 2, 0, 0, 5, 31], seed=8)
    c.V[c.table[0, 1].long(), 0, 3, 5] = bad
    c.V[c.table[2, 2].long(), 1, 0, d - 1] = bad
    c.pre["V"][41, 7] = bad
    c.check()


@pytest.mark.parametrize("dtype,d", TYPES)
def test_paged_infinite_values_at_the_smallest_weights(dtype, d):
    # infinities at weights from 1 down to e^-84, among them some that bf16 holds exactly
    c = Cache(dtype, d, 1, 4, [20], 16, [60], seed=25)
    c.q[:] = 0.0
    c.pre["logm"][:] = 0.0
    for i, (dim, lm) in enumerate([(1, 0.0), (2, -math.log(2.0)), (3, -1.0), (4, -20.0), (5, -60.0), (6, -78.0), (7, -80.0), (8, -84.0)]):
        c.pre["logm"][3 * i + 1] = lm
        c.pre["V"][3 * i + 1, dim] = math.inf if i % 2 else -math.inf
    c.check()


@pytest.mark.parametrize("d", [64, 128])
def test_paged_weights_keep_more_than_bf16(d):
    """Values that nearly cancel under weights that bf16 does not hold: the output is far below the
    weighted values, and so are the weights' errors, 2^-15 of themselves (two bf16 parts), where weights
    rounded to bf16 would leave up to 2^-8."""
    gen = torch.Generator().manual_seed(26)
    for lens, counts in (([700], None), ([0], [900]), ([3000], [40])):
        c = Cache("bf16", d, 1, 16, lens, 16, counts, seed=27)
        amp = (torch.rand(d, generator=gen) + 0.5).bfloat16()
        c.q[:] = torch.linspace(0.05, 0.3, 16)[None, :, None].bfloat16()
        for K, V in [(c.K, c.V)] + ([] if counts is None else [(c.pre["K"], c.pre["V"])]):
            odd = torch.arange(K.shape[-2]) % 2 == 1
            K[:] = 0.0
            K[..., odd, :] = -1.0 / math.sqrt(d)
            V[:] = amp
            V[..., odd, :] = -amp
        if counts is not None:
            c.pre["logm"][:] = 0.0
        out, lse = c.call()
        k, v, lm = c.entries(0, 0)
        ref, ref_lse, A, X = S.attend64(c.q[0].double(), k, v, bias=lm)
        n = len(k)
        w = 2 * ((d + 3) * X + 4 * X + 4) * S.U + 2.0 ** -15
        tol = A * (w + 2 * (n + n / 16 + 8) * S.U)[:, None] + ref.abs() * S.B16
        assert ((out[0].double() - ref).abs() <= tol).all(), (d, lens, float(((out[0].double() - ref).abs() / tol).max()))


def test_paged_malformed_inputs_stay_inside():
    # lengths past the table, negative ones, pages that are none, packed rows outside the arrays
    c = Cache("bf16", 64, 2, 4, [40, 20, 33], 16, [10, 20, 5, 6, 7, 8], seed=9)
    c.table[1, 0], c.table[2, 1] = c.K.shape[0], 2 ** 31 - 1
    c.len[:] = torch.tensor([2 ** 31 - 1, -5, 33], dtype=torch.int32)
    c.pre["start"][0], c.pre["count"][1], c.pre["count"][2], c.pre["start"][3] = -4, 1 << 40, -3, 1 << 40
    out, lse = c.call()
    n = c.pre["K"].shape[0]
    c.pre["start"].clamp_(0, n)
    c.pre["count"].clamp_(min=0)
    c.pre["count"] = torch.minimum(c.pre["count"], n - c.pre["start"])
    c.check((out, lse))


@pytest.mark.parametrize("fill", [0, 1, 127, 255])
def test_paged_workspace_needs_no_clearing(fill):
    # whatever a workspace holds, also what calls of other shapes left in it; the same twice
    a = Cache("bf16", 128, 2, 8, [4001, 3, 0, 900], 16, seed=20)
    b = Cache("f32", 64, 1, 20, [60] * 40 + [3000], 16, [5] * 41, seed=21)
    ws = torch.full((8 << 20,), fill, dtype=torch.uint8, device="cuda")
    for c in (a, b, a, a, b):
        c.check(c.call(ws=ws))


@pytest.mark.parametrize("word", [0x7fffffffffff0000, 0x7fffffffffff1000, 0x7fffffffffffffff, -1, -2 ** 63, 1, 0x7fffffff7fffffff])
def test_paged_workspace_words_around_a_count(word):
    # any word that is not between the first and the last number of a count; the same workspace again afterwards
    c = Cache("bf16", 64, 2, 8, [4001, 3, 900], 16, seed=23)
    ws = torch.full((1 << 19,), word, dtype=torch.int64, device="cuda")
    for _ in range(2):
        c.check(c.call(ws=ws))


def test_paged_every_batch_size():
    for B in (1, 2, 63, 64, 65, 257, 700):
        gen = torch.Generator().manual_seed(B)
        lens = torch.randint(0, 60, (B,), generator=gen).tolist()
        c = Cache("bf16", 64, 1, 2, lens, 16, torch.randint(0, 40, (B,), generator=gen).tolist() if B % 2 else None, seed=B)
        c.check()


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("name", list(S.paged_shapes()))
def test_paged_rarer_ways(dtype, d, name):
    # rows of several chunks among more units than one round of the search; rows of more chunks than the
    # join takes at once (values that rise along the row: a part that is lost or taken twice shows)
    G, Hq, lens, page, counts = S.paged_shapes()[name]
    c = Cache(dtype, d, G, Hq, lens, page, counts, seed=24)
    if name == "long pages":
        c.V[c.table[0].long()] += torch.linspace(0, 4, lens[0]).view(-1, 1, page, 1).to(c.V.dtype)
    if name == "long entries":
        c.pre["V"][:counts[0]] += torch.linspace(0, 4, counts[0])[:, None].to(c.V.dtype)
    c.check()


def test_paged_prefix_of_no_rows():
    c = Cache("bf16", 64, 2, 6, [70, 0], 16, [0] * 4, seed=22)
    for name in ("K", "V", "logm"):
        c.pre[name] = c.pre[name][:0]
    c.check()


def test_paged_shared_pages_and_packed_rows():
    # sequences that share their first pages, and a compressed context that all of them share
    c = Cache("bf16", 128, 2, 8, [48, 48, 48], 16, [30] * 6, seed=10, share=True)
    c.table[1:, :2] = c.table[0, :2]
    c.check()


def test_paged_far_pages():
    # pages past 32 bits of elements and bytes: the last page of a pool of 4.3 G elements
    page, d = 256, 128
    stride = 1 << 26
    pool = torch.empty(65 * stride, dtype=torch.bfloat16, device="cuda")
    K = pool.as_strided((65, 1, page, d), (stride, page * d, d, 1))
    gen = torch.Generator().manual_seed(11)
    k, v, q = _rand(gen, 2 * page, 1, d), _rand(gen, 2 * page, 1, d), _rand(gen, 1, 4, d)
    table = torch.tensor([[64, 0]], dtype=torch.int32, device="cuda")
    V = pool[page * d:].as_strided((65, 1, page, d), (stride, page * d, d, 1))
    cfg = gk.page_config(K, 4, table)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    gk.cache_append(cfg, k.cuda(), v.cuda(), K, V, table, zero, _cu([2 * page]).cuda())
    assert torch.equal(K[64, 0].cpu(), k[:page, 0]) and torch.equal(V[0, 0].cpu(), v[page:, 0])
    out, lse = torch.empty(1, 4, d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 4, device="cuda")
    ws = torch.empty(gk.paged_ws_bytes(cfg), dtype=torch.uint8, device="cuda")
    gk.paged_attention(cfg, q.cuda(), K, V, table, zero + 2 * page, out, ws, lse=lse)
    S.check_rows(out[0].cpu(), lse[0].cpu(), S.attend64(q[0].double(), k[:, 0].double(), v[:, 0].double()), 512, d, True, "far")


# ---------------------------------------------------------------------------
# together


def test_compressed_context_then_generated_tokens():
    """A prompt's attention, its cache compressed, the window and new tokens appended, and
    every new token's attention over packed entries and pages, as a serving program runs them."""
    sh = small_shape("serve", L=2, G=2, H=8, d=128, N_ctx=600, W=24, x=6.0, n_segments=6, dtype="bf16")
    case = H.to_dev(make_case(sh, 5, with_hidden=True))
    K, V, Q = case["K"], case["V"], case["Q"]
    # the question's window over the context, in the library's own layouts
    for l in range(sh.L):
        q, k, v = Q[l].transpose(0, 1), K[l].transpose(0, 1), V[l].transpose(0, 1)
        out, lse = torch.empty_like(q), torch.empty(sh.W, sh.H, device="cuda")
        cfg = gk.prompt_config(q, k, v, out, 1)
        ws = torch.empty(gk.prompt_ws_bytes(cfg), dtype=torch.uint8, device="cuda")
        gk.prompt_attention(cfg, q, k, v, _cu([sh.W]).cuda(), _cu([sh.T]).cuda(), out, ws, lse=lse)
        S.prompt64(q.cpu().double(), k.cpu().double(), v.cpu().double(), [sh.W], [sh.T],
                   lambda rows, h, ref, m: S.check_rows(out[rows, h].cpu(), lse[rows, h].cpu(), ref, m, sh.d, True, (l, h)))
    ccfg = H.make_cfg(sh)
    buf = gk.allocate(ccfg)
    gk.compress(buf, K, V, Q, case["rope_cos"], case["rope_sin"], case["hidden"], case["surprisal"], case["omega_raw"])
    gk.check(ccfg, buf.trees)
    # a pool of pages for both layers: the window's rows as they are, then tokens one by one
    page, steps = 16, 11
    n_pages = -(-(sh.W + steps) // page) + 1
    pool = [torch.zeros(n_pages, sh.L, sh.G, page, sh.d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1))[None, :n_pages - 1].to(torch.int32).cuda().contiguous()
    cfg = gk.page_config(pool[0][:, 0], sh.H, table)
    ws = torch.empty(gk.paged_ws_bytes(cfg), dtype=torch.uint8, device="cuda")
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")         # noqa: E731
    gen = torch.Generator().manual_seed(2)
    cos, sin = (x.cuda() for x in _rope(sh.T + steps, sh.d))
    kept = {}
    for l in range(sh.L):
        win = [x[l, :, sh.N_ctx:].transpose(0, 1) for x in (K, V)]
        gk.cache_append(cfg, *win, pool[0][:, l], pool[1][:, l], table, i32(0), _cu([sh.W]).cuda())
        kept[l] = [x.cpu().double() for x in win]
    for step in range(steps):
        at = sh.W + step
        for l in range(sh.L):
            k, v, q = (_rand(gen, 1, x, sh.d).cuda() for x in (sh.G, sh.G, sh.H))
            qr = torch.empty_like(q)
            gk.cache_append(cfg, k, v, pool[0][:, l], pool[1][:, l], table, i32(at), _cu([1]).cuda(), i32(sh.N_ctx + at), cos, sin, q, qr)
            out, lse = torch.empty(1, sh.H, sh.d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, sh.H, device="cuda")
            rows = slice(l * sh.G, (l + 1) * sh.G)
            pre = gk.Prefix(buf.offsets[rows], buf.counts[rows], buf.K_out, buf.V_out, buf.logm_out)
            gk.paged_attention(cfg, qr, pool[0][:, l], pool[1][:, l], table, i32(at + 1), out, ws, lse=lse, prefix=pre)
            turned = S.rotate64(k.cpu().double(), cos[sh.N_ctx + at:][:1].cpu().double(), sin[sh.N_ctx + at:][:1].cpu().double())
            stored = pool[0][int(table[0, at // page]), l, :, at % page].cpu().double()[None]
            assert ((stored - turned).abs() <= S.B16 * turned.abs() + 1e-5).all()
            kept[l] = [torch.cat([kept[l][0], stored]), torch.cat([kept[l][1], v.cpu().double()])]
            off = buf.offsets.cpu()
            for g in range(sh.G):
                a, e = int(off[l * sh.G + g]), int(off[l * sh.G + g + 1])
                kk = torch.cat([buf.K_out[a:e].cpu().double(), kept[l][0][:, g]])
                vv = torch.cat([buf.V_out[a:e].cpu().double(), kept[l][1][:, g]])
                lm = torch.cat([buf.logm_out[a:e].cpu().double(), torch.zeros(at + 1, dtype=torch.float64)])
                h = slice(g * 4, g * 4 + 4)
                S.check_rows(out[0, h].cpu(), lse[0, h].cpu(), S.attend64(qr[0, h].cpu().double(), kk, vv, bias=lm), len(kk), sh.d, True, (step, l, g))


def test_step_captured_and_replayed_on_a_stream():
    """Append and attention of a batch captured once on a side stream and replayed while
    lengths, tables and tokens change in place; every replay against the eager calls."""
    gen = torch.Generator().manual_seed(3)
    c = Cache("bf16", 128, 2, 8, [90, 3, 500, 17], 16, [100, 0, 33, 64, 1, 2, 300, 5], seed=12)
    dev = {n: getattr(c, n).cuda() for n in ("K", "V", "table", "len", "q")}
    pre = gk.Prefix(**{n: x.cuda() for n, x in c.pre.items()})
    cfg = gk.page_config(dev["K"], c.H, dev["table"])
    k, v = (_rand(gen, 4, 2, 128).cuda() for _ in range(2))
    pos, cu, (cos, sin) = torch.arange(4, dtype=torch.int32).cuda(), _cu([1] * 4).cuda(), (x.cuda() for x in _rope(600, 128))
    start = (dev["len"] - 1).contiguous()
    ws, qr = torch.empty(gk.paged_ws_bytes(cfg), dtype=torch.uint8, device="cuda"), torch.empty_like(dev["q"])
    out, lse = torch.empty_like(dev["q"]), torch.empty(4, 8, device="cuda")

    def step(K, V, stream=None):
        gk.cache_append(cfg, k, v, K, V, dev["table"], start, cu, pos, cos, sin, dev["q"], qr, stream=stream)
        gk.paged_attention(cfg, qr, K, V, dev["table"], dev["len"], out, ws, lse=lse, prefix=pre, stream=stream)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(dev["K"], dev["V"])
    for i in range(5):
        k.copy_(_rand(gen, 4, 2, 128))
        dev["q"].copy_(_rand(gen, 4, 8, 128))
        dev["len"].copy_(torch.tensor([90 - 7 * i, 3, 500 - 100 * i, 17 - i], dtype=torch.int32))
        start.copy_(dev["len"] - 1)
        pos.add_(i)
        K2, V2 = dev["K"].clone(), dev["V"].clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), qr.clone()
        with torch.cuda.stream(side):                            # eager, on the side stream
            step(K2, V2)
        side.synchronize()
        assert torch.equal(K2, dev["K"]) and torch.equal(V2, dev["V"])
        assert torch.equal(got[0], out) and torch.equal(got[1], lse) and torch.equal(got[2], qr)


def test_two_graphs_in_turn_on_one_workspace():
    """Two captured batches of different shapes and types, one workspace, replayed one after the other."""
    a = Cache("bf16", 128, 2, 8, [4001, 3, 0, 900], 16, [5] * 8, seed=31)
    b = Cache("f32", 64, 1, 20, [60] * 20 + [3000], 16, seed=32)
    size = max(gk.paged_ws_bytes(gk.page_config(c.K, c.H, c.table)) for c in (a, b))
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    side, runs = torch.cuda.Stream(), []
    for c in (a, b):
        dev = {n: getattr(c, n).cuda() for n in ("K", "V", "table", "len", "q")}
        pre = None if c.pre is None else gk.Prefix(**{n: x.cuda() for n, x in c.pre.items()})
        out, lse = torch.empty_like(dev["q"]), torch.empty(c.q.shape[:2], device="cuda")
        graph = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            gk.paged_attention(gk.page_config(dev["K"], c.H, dev["table"]), dev["q"], dev["K"], dev["V"], dev["table"], dev["len"], out, ws,
                               lse=lse, prefix=pre)
        runs.append((c, graph, out, lse, dev, pre))
    for _ in range(4):
        for c, graph, out, lse, _, _ in runs:
            out.fill_(7.0)
            graph.replay()
        torch.cuda.synchronize()
        for c, _, out, lse, _, _ in runs:
            c.check((out.cpu(), lse.cpu()))


def test_prompt_captured_and_replayed():
    gen = torch.Generator().manual_seed(4)
    q, k, v = _rand(gen, 40, 8, 128).cuda(), _rand(gen, 2000, 2, 128).cuda(), _rand(gen, 2000, 2, 128).cuda()
    out, lse = torch.empty_like(q), torch.empty(40, 8, device="cuda")
    cfg = gk.prompt_config(q, k, v, out, 2)
    ws = torch.empty(gk.prompt_ws_bytes(cfg), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    cu_q, cu_k = _cu([30, 10]).cuda(), _cu([1500, 500]).cuda()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        gk.prompt_attention(cfg, q, k, v, cu_q, cu_k, out, ws, lse=lse)
    for i in range(4):
        q.copy_(_rand(gen, 40, 8, 128))
        cu_q.copy_(_cu([5 + 8 * i, 35 - 8 * i]))
        cu_k.copy_(_cu([1500 - 300 * i, 500 + 300 * i]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        out.zero_()
        gk.prompt_attention(cfg, q, k, v, cu_q, cu_k, out, ws, lse=lse)
        assert torch.equal(got[0], out) and torch.equal(got[1], lse)


def test_calls_at_once_on_two_streams():
    """Prompts and a batch's next tokens on two streams at the same time, a workspace each:
    bit for bit what one after the other gives."""
    gen = torch.Generator().manual_seed(5)
    c = Cache("bf16", 128, 2, 16, [9000, 40, 3000, 0, 1, 700], 64, seed=30)
    dev = {n: getattr(c, n).cuda() for n in ("K", "V", "table", "len", "q")}
    page = gk.page_config(dev["K"], c.H, dev["table"])
    q, k, v = _rand(gen, 100, 16, 128).cuda(), _rand(gen, 4000, 2, 128).cuda(), _rand(gen, 4000, 2, 128).cuda()
    cu_q, cu_k = _cu([100]).cuda(), _cu([4000]).cuda()
    prompt = gk.prompt_config(q, k, v, q, 1)
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in sides + [None]:
        got.append(dict(po=torch.zeros_like(q), pl=torch.zeros(100, 16, device="cuda"), do=torch.zeros_like(dev["q"]),
                        dl=torch.zeros(6, 16, device="cuda"), pw=torch.empty(gk.prompt_ws_bytes(prompt), dtype=torch.uint8, device="cuda"),
                        dw=torch.empty(gk.paged_ws_bytes(page), dtype=torch.uint8, device="cuda")))

    def run(b, stream):
        gk.prompt_attention(prompt, q, k, v, cu_q, cu_k, b["po"], b["pw"], lse=b["pl"], stream=stream)
        gk.paged_attention(page, dev["q"], dev["K"], dev["V"], dev["table"], dev["len"], b["do"], b["dw"], lse=b["dl"], stream=stream)
    run(got[2], None)
    torch.cuda.synchronize()
    for _ in range(20):
        for b, stream in zip(got, sides):
            run(b, stream)
    torch.cuda.synchronize()
    for b in got[:2]:
        for name in ("po", "pl", "do", "dl"):
            assert torch.equal(b[name], got[2][name]), name
    c.check((got[2]["do"].cpu(), got[2]["dl"].cpu()))
