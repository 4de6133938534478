"""Performance cases of the operators that serve a batch from quantised pages and from
a context that its sequences share, for one layer.

  write    new tokens' keys and values quantised into a paged cache as they are written
           (keys and queries rotated on the way), and rows read back from it: those just
           written, or the sequences so far, for the attention of a chunk
  read     whole quantised sequences back as rows, for a compression
  attend   attention of one new token of every sequence over its quantised pages
  shared   groups of sequences that begin with the same packed entries (one compressed
           context, many questions), which are gone through once for the group, and each
           sequence's own pages behind them

Quantised rows have blocks of 32 neighbouring dims with one power of two each, as
``_quantise`` has it.  Head layouts: the 8B shape (8 KV heads, 32 query heads of 128), a
share of the 70B shape (8 query heads per KV head), a 64-wide one, one head per KV head,
and the small fp32 one.  ``own`` chooses between the plain forms here and the library's calls.
"""
import functools
import math
import random

import torch

own = False
DEV = "cuda"

H8B, H70B, NARROW, MHA, SMALL = (8, 32, 128), (8, 64, 128), (8, 32, 64), (4, 4, 128), (2, 4, 64)
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BITS = {"e4m3": 8, "e2m1": 4}


def _text(lens):
    return ",".join(str(int(n)) for n in lens)


def _lens(text):
    return [int(n) for n in text.split(",")]


def _named(name, **case):
    return dict(case, name=name) if name else case


def _write(name, heads, start, new, page, fmt, back="new", dtype="bf16", layout="token"):
    return _named(name, op="write", G=heads[0], H=heads[1], d=heads[2], start=_text(start), new=_text(new), page=page, format=fmt,
                  back=back, dtype=dtype, layout=layout)


def _read(name, heads, lens, page, fmt, dtype="bf16", layout="head"):
    return _named(name, op="read", G=heads[0], H=heads[1], d=heads[2], lens=_text(lens), page=page, format=fmt, dtype=dtype, layout=layout)


def _attention(name, heads, lens, page, fmt, dtype="bf16"):
    return _named(name, op="attend", G=heads[0], H=heads[1], d=heads[2], lens=_text(lens), page=page, format=fmt, dtype=dtype)


def _shared(name, heads, groups, entries, lens, page, fmt="plain", dtype="bf16"):
    return _named(name, op="shared", G=heads[0], H=heads[1], d=heads[2], groups=_text(groups), entries=entries, lens=_text(lens),
                  page=page, format=fmt, dtype=dtype)


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _spread(count, lo, hi, seed):
    r = random.Random(seed)
    return [_logint(r, lo, hi) for _ in range(count)]


def listed():
    return [
        # one generated token of a batch of 64: every step of every layer pays this
        _write("write-step-64-e4m3", H8B, _spread(64, 1, 8192, 1), [1] * 64, 16, "e4m3"),
        # the pages of a whole prefill
        _write("write-prefill-8k-e2m1", H8B, [0, 17], [8192, 2047], 64, "e2m1"),
        # chunks of prompts: the sequences so far come back for the chunks' attention
        _write("write-chunks-back-e4m3", H70B, [8192, 1, 2999, 0], [512, 77, 1, 300], 32, "e4m3", back="all"),
        # a long context back as rows, to be compressed
        _read("read-32k-e4m3", H8B, [32768 + 64], 64, "e4m3"),
        # ragged sequences, fp32 rows
        _read("read-ragged-e2m1-f32", (3, 15, 64), _spread(16, 1, 4096, 4), 16, "e2m1", "f32", "token"),
        # one conversation: latency
        _attention("attend-one-8k-e4m3", H8B, [8192 + 9], 16, "e4m3"),
        # a server's batch of 64 sequences of very different lengths
        _attention("attend-batch-64-e4m3", H8B, _spread(64, 1, 8192, 2), 16, "e4m3"),
        # long caches, eight query heads per KV head
        _attention("attend-70b-128k-e2m1", H70B, [131072, 131072 - 31, 98765, 131072], 64, "e2m1"),
        # fp32 rows, an odd head layout
        _attention("attend-f32-odd-e4m3", (3, 15, 64), [1, 700, 5003], 16, "e4m3", "f32"),
        # 16 questions on one context of 32K tokens compressed 16x, and what was generated for each
        _shared("shared-16-x2k", H8B, [16], 2048, _spread(16, 1, 1024, 3), 16),
        # the largest: 64 sequences behind one long prefix, their own tokens quantised
        _shared("shared-64-x16k-e4m3", H8B, [64], 16384, _spread(64, 1, 2048, 5), 64, "e4m3"),
        # several contexts with few sequences each, one with none, fp32
        _shared("shared-groups-f32", SMALL, [1, 5, 0, 2], 300, _spread(8, 1, 200, 6), 16, "plain", "f32"),
    ]


def draw(rng):
    op = rng.choice(["write", "write", "read", "attend", "attend", "shared", "shared", "shared"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    heads = rng.choice([H8B, H70B, NARROW, MHA, SMALL])
    if rng.random() < 0.25:
        G = rng.randint(1, 6)
        heads = (G, G * rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]), rng.choice([64, 128]))
    layout = rng.choice(["token", "head"])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    fmt = rng.choice(["e4m3", "e2m1"])
    B = _logint(rng, 1, 64)
    if op == "write":
        new = [1] * B if rng.random() < 0.5 else _spread(B, 1, max(1, 16384 // B), rng.random())
        return _write(None, heads, _spread(B, 1, 4096, rng.random()), new, page, fmt, rng.choice(["new", "all"]), dtype, layout)
    if op == "read":
        return _read(None, heads, _spread(B, 1, 65536 // B, rng.random()), page, fmt, dtype, layout)
    if op == "attend":
        return _attention(None, heads, _spread(B, 1, min(131072, (1 << 18) // B), rng.random()), page, fmt, dtype)
    groups = [B] if rng.random() < 0.5 else _spread(rng.randint(2, 8), 1, max(1, B // 2), rng.random())
    n, most = sum(groups), max(groups)
    # the plain form pads to the largest group and row; fp32's products are slower
    room = (1 << 30) // (len(groups) * most * heads[1] * heads[2] // 32 * (8 if dtype == "f32" else 1))
    return _shared(None, heads, groups, _logint(rng, 1, max(64, min(16384, room))), _spread(n, 1, min(4096, (1 << 17) // n), rng.random()),
                   page, rng.choice(["plain", fmt]), dtype)


# ---------------------------------------------------------------------------
# blocks of 32 dims with one power of two: s = the least at which no value is off by more than half a step
# of the largest ones; a block with a value that is no finite number stands for NaN

_HALVES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


@functools.lru_cache(maxsize=None)
def _table(device):
    """The numbers of the 16 e2m1 codes."""
    return torch.tensor(_HALVES + tuple(-h for h in _HALVES), device=device)


def _quantise(x, fmt):
    """x [..., d] fp32: codes uint8 [..., d * bits / 8], scales uint8 [..., d / 32] (2^(s - 127); 255: NaN)."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    # largest values 448 = 1.75 * 2^8 and 6 = 1.5 * 2^2; up to 464 and 7 they are the nearest
    lift, emax = (0x17ffff, 8) if fmt == "e4m3" else (0x1fffff, 2)
    s = (((top.view(torch.int32) + lift) >> 23) - emax).clamp(10, 254)
    none = ~(top < 2.0 ** 127)
    y = x * torch.where(none, 0, (254 - s) << 23).view(torch.float32)[..., None]
    y = torch.where(none[..., None], 0.0, y)
    if fmt == "e4m3":
        codes = y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    else:
        a = y.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        a = (torch.round(a / step) * step).clamp(max=6)
        c = torch.bucketize(a, _table(x.device)[:8]) + 8 * torch.signbit(y)
        c = c.to(torch.uint8).flatten(-2)
        codes = c[..., 0::2] | c[..., 1::2] << 4
    return codes, torch.where(none, 255, s).to(torch.uint8)


def _values(codes, scales, fmt):
    """What codes and scales stand for, fp32."""
    if fmt == "e4m3":
        x = codes.view(torch.float8_e4m3fn).float()
    else:
        x = _table(codes.device)[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()]
    s = torch.where(scales == 255, 0x7fc00000, scales.int() << 23).view(torch.float32)
    return (x.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


# ---------------------------------------------------------------------------
# inputs


def _rows(gen, n, heads, d, dtype, layout, topics, aim=0.0, scale=1.0):
    """[n][heads][d] values that walk from topic to topic (``aim``: how strongly a row points at a random one)."""
    x = torch.randn(n, heads, d, generator=gen, device=DEV)
    which = torch.arange(n, device=DEV) // 128 % topics.shape[0]
    if aim:
        which = torch.randint(0, topics.shape[0], (n,), generator=gen, device=DEV)
    t = topics[which].repeat_interleave(heads // topics.shape[1], 1)
    part = aim or 0.8
    x = ((1 - part * part) ** 0.5 * x + part * t) * scale
    return _laid(x.to(dtype), layout)


def _laid(x, layout):
    """The same [n][heads][d] tensor, its memory token-major or head-major."""
    return x.contiguous() if layout == "token" else x.transpose(0, 1).contiguous().transpose(0, 1)


def _cu(lens):
    return torch.tensor([0] + lens, device=DEV).cumsum(0).to(torch.int32)


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _tables(gen, lens, page):
    """Page ids in no order, and how many pages there are; unused places of a row hold -1."""
    need = [-(-n // page) for n in lens]
    width, total = max(need), sum(need) + 3
    ids = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    used = torch.arange(width, device=DEV)[None] < torch.tensor(need, device=DEV)[:, None]
    table[used] = ids[:sum(need)]
    return table, total


def _pools(s, gen, n_pages, case, topics):
    """Pages of keys and values, plain or quantised."""
    G, page, d, fmt = case["G"], case["page"], case["d"], case["format"]
    for name in ("K", "V"):
        plain = fmt == "plain"
        x = _rows(gen, n_pages * page, G, d, DTYPES[case["dtype"]] if plain else torch.float32, "token", topics)
        x = x.view(n_pages, page, G, d).transpose(1, 2).contiguous()
        if plain:
            s[name] = x
            continue
        parts = [_quantise(y, fmt) for y in x.split(max(1, (1 << 26) // (G * page * d)))]
        s[name], s[name + "s"] = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])


@functools.lru_cache(maxsize=64)
def _counts(text, G, average):
    """Entries of every (group, KV head): a compression spreads them unevenly."""
    r = random.Random("%s %d" % (text, average))
    return [int(average * r.uniform(0.5, 1.5)) for _ in range(len(_lens(text)) * G)]


def _rope(rows, d):
    ang = torch.arange(rows, device=DEV, dtype=torch.float64)[:, None] * 5.0e5 ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)
    return ang.cos().float().contiguous(), ang.sin().float().contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    op, G, H, d, dtype = case["op"], case["G"], case["H"], case["d"], DTYPES[case["dtype"]]
    topics, s = torch.randn(64, G, d, generator=gen, device=DEV), dict(case=case)
    if op in ("write", "read"):
        start, new = (_lens(case["start"]), _lens(case["new"])) if op == "write" else ([0], [0])
        upto = [a + b for a, b in zip(start, new)] if op == "write" else _lens(case["lens"])
        s["table"], n_pages = _tables(gen, upto, case["page"])
        _pools(s, gen, n_pages, case, topics)
        if op == "write":
            n = sum(new)
            s.update(k=_rows(gen, n, G, d, dtype, case["layout"], topics), v=_rows(gen, n, G, d, dtype, case["layout"], topics),
                     q=_rows(gen, n, H, d, dtype, case["layout"], topics, 0.3, 2.0), cu=_cu(new), start=_int(start))
            # the rotation goes by the position in the text, which a compressed context puts ahead of the place in the cache
            s["pos"] = torch.cat([torch.arange(n, device=DEV, dtype=torch.int32) + a + 100 for a, n in zip(start, new)])
            s["cos"], s["sin"] = _rope(max(upto) + 100, d)
            s["q_out"] = torch.zeros(n, H, d, dtype=dtype, device=DEV)
        first = start if op == "write" and case["back"] == "new" else [0] * len(upto)
        back = [b - a for a, b in zip(first, upto)]
        s.update(first=_int(first), cu_back=_cu(back))
        s["k_back"], s["v_back"] = (_laid(torch.zeros(sum(back), G, d, dtype=dtype, device=DEV), case["layout"]) for _ in range(2))
        return s
    lens = _lens(case["lens"])
    s["table"], n_pages = _tables(gen, lens, case["page"])
    _pools(s, gen, n_pages, case, topics)
    s.update(len=_int(lens), q=_rows(gen, len(lens), H, d, dtype, "token", topics, 0.3, 2.0),
             out=torch.zeros(len(lens), H, d, dtype=dtype, device=DEV), lse=torch.zeros(len(lens), H, device=DEV))
    if op == "shared":
        counts, groups = _counts(case["groups"], G, case["entries"]), _lens(case["groups"])
        count = torch.tensor(counts, device=DEV)
        n = sum(counts) + 5
        entries = lambda: _rows(gen, n, 1, d, dtype, "token", topics[:, :1]).view(n, d)      # noqa: E731
        s.update(groups=groups, cu_group=_cu(groups), p_count=count, p_start=count.cumsum(0) - count, p_most=max(counts), p_K=entries(),
                 p_V=entries(), p_logm=torch.log1p(torch.rand(n, generator=gen, device=DEV) * 20))
    return s


# ---------------------------------------------------------------------------
# plain forms


def _places(s, cu, first, n):
    """Page and place in it of rows that begin at `first` of their sequences."""
    page = s["case"]["page"]
    cu, i = cu.long(), torch.arange(n, device=DEV)
    b = torch.searchsorted(cu, i, right=True) - 1
    place = first.long()[b] + i - cu[b]
    return s["table"].long()[b, place // page], place % page


def _rotate(x, cos, sin):
    """Products and their difference in fp32, each rounded."""
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_back(s):
    at, place = _places(s, s["cu_back"], s["first"], s["k_back"].shape[0])
    for name, to in (("K", "k_back"), ("V", "v_back")):
        s[to].copy_(_values(s[name][at, :, place], s[name + "s"][at, :, place], s["case"]["format"]))
    return {"k": s["k_back"], "v": s["v_back"]}


def _plain_write(s):
    at, place = _places(s, s["cu"], s["start"], s["k"].shape[0])
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    for name, x in (("K", _rotate(s["k"], cos, sin)), ("V", s["v"].float())):
        s[name][at, :, place], s[name + "s"][at, :, place] = _quantise(x, s["case"]["format"])
    s["q_out"].copy_(_rotate(s["q"], cos, sin))
    return dict(_plain_back(s), q=s["q_out"])


def _attend(q, k, v, bias, seen):
    """q [B, G, n, d], k and v [B, G, m, d], bias [B, G, 1, m] or None, seen broadcast over [B, G, n, m]: mean and lse, fp32."""
    B, G, n, d = q.shape
    x = torch.bmm(q.reshape(B * G, n, d) * d ** -0.5, k.reshape(B * G, -1, d).transpose(1, 2).contiguous()).view(B, G, n, -1)
    if bias is not None:
        x += bias
    x.masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.bmm(x.view(B * G, n, -1), v.reshape(B * G, -1, d)).view(B, G, n, d)
    return torch.where(z > 0, o / z, 0.0), (m + z.log())[..., 0]


def _over_pages(s):
    """Mean [B, H, d] and lse [B, H] over each sequence's pages."""
    q, table = s["q"], s["table"].long().clamp(min=0)
    (B, H, d), G, fmt = q.shape, s["case"]["G"], s["case"]["format"]

    def pages(name):
        x = s[name][table].float() if fmt == "plain" else _values(s[name][table], s[name + "s"][table], fmt)
        return x.transpose(1, 2).reshape(B, G, -1, d)
    k, v = pages("K"), pages("V")
    seen = (torch.arange(k.shape[2], device=DEV) < s["len"][:, None])[:, None, None]
    o, lse = _attend(q.float().view(B, G, H // G, d), k, v, None, seen)
    return o.view(B, H, d), lse.view(B, H)


def _given(s, o, lse):
    s["out"].copy_(o)
    s["lse"].copy_(lse)
    return {"out": s["out"], "lse": s["lse"]}


def _plain_shared(s):
    q, cu = s["q"], s["cu_group"].long()
    (B, H, d), G, S = q.shape, s["case"]["G"], cu.numel() - 1
    n, most = cu.diff(), max(s["groups"])
    # a group's sequences side by side, and its entries
    i, j = torch.arange(most, device=DEV), torch.arange(s["p_most"], device=DEV)
    on = i < n[:, None]
    at_q = (cu[:-1, None] + i) * on
    qp = q[at_q].float().view(S, most, G, H // G, d).transpose(1, 2).reshape(S, G, -1, d)
    has = j < s["p_count"][:, None]
    at = (s["p_start"][:, None] + j) * has
    o, lse = _attend(qp, s["p_K"][at].float().view(S, G, -1, d), s["p_V"][at].float().view(S, G, -1, d),
                     s["p_logm"][at].view(S, G, 1, -1), has.view(S, G, 1, -1))
    o = o.view(S, G, most, H // G, d).transpose(1, 2).reshape(S, most, H, d)[on]
    lse = lse.view(S, G, most, H // G).transpose(1, 2).reshape(S, most, H)[on]
    # and each sequence's own pages
    o2, lse2 = _over_pages(s)
    both = torch.logaddexp(lse, lse2)
    return _given(s, o * (lse - both).exp()[..., None] + o2 * (lse2 - both).exp()[..., None], both)


_PLAIN = {"write": _plain_write, "read": _plain_back, "attend": lambda s: _given(s, *_over_pages(s)), "shared": _plain_shared}


# ---------------------------------------------------------------------------
# the library's calls


def _own_pages(s):
    """The handle of the quantised pages and the shapes that a program keeps."""
    from paper_2608_07001_amd import gracekv as gk
    if "cfg" not in s:
        c = s["case"]
        s["pages"] = gk.QuantPages(gk.E4M3 if c["format"] == "e4m3" else gk.E2M1, s["K"], s["V"], s["Ks"], s["Vs"])
        s["cfg"] = gk.quant_config(s["pages"], DTYPES[c["dtype"]], c["H"], s["table"])
    return gk


def _own_back(s):
    gk = _own_pages(s)
    gk.quant_read(s["cfg"], s["pages"], s["table"], s["first"], s["cu_back"], s["k_back"], s["v_back"])
    return {"k": s["k_back"], "v": s["v_back"]}


def _own_write(s):
    gk = _own_pages(s)
    gk.quant_append(s["cfg"], s["pages"], s["k"], s["v"], s["table"], s["start"], s["cu"], pos=s["pos"], rope_cos=s["cos"],
                    rope_sin=s["sin"], q=s["q"], q_out=s["q_out"])
    return dict(_own_back(s), q=s["q_out"])


def _own_attend(s, part=None):
    gk = _own_pages(s)
    if "ws" not in s:
        s["ws"] = torch.empty(gk.paged_ws_bytes(s["cfg"]), dtype=torch.uint8, device=DEV)
    gk.quant_attention(s["cfg"], s["pages"], s["q"], s["table"], s["len"], s["out"], s["ws"], lse=s["lse"], part=part)
    return {"out": s["out"], "lse": s["lse"]}


def _own_shared(s):
    from paper_2608_07001_amd import gracekv as gk
    if "part" not in s:
        c, (B, H, d) = s["case"], s["q"].shape
        s["scfg"] = gk.shared_config(s["q"], c["G"], len(s["groups"]))
        s["sws"] = torch.empty(gk.shared_ws_bytes(s["scfg"]), dtype=torch.uint8, device=DEV)
        s["prefix"] = gk.Prefix(s["p_start"], s["p_count"], s["p_K"], s["p_V"], s["p_logm"])
        s["part"] = gk.Part(torch.empty(B, H, d, device=DEV), torch.empty(B, H, device=DEV))
        if c["format"] == "plain":
            s["cfg"] = gk.page_config(s["K"], H, s["table"])
            s["ws"] = torch.empty(gk.paged_ws_bytes(s["cfg"]), dtype=torch.uint8, device=DEV)
    gk.shared_attention(s["scfg"], s["q"], s["cu_group"], s["prefix"], s["part"], s["sws"])
    if s["case"]["format"] != "plain":
        return _own_attend(s, s["part"])
    gk.paged_attention(s["cfg"], s["q"], s["K"], s["V"], s["table"], s["len"], s["out"], s["ws"], lse=s["lse"], part=s["part"])
    return {"out": s["out"], "lse": s["lse"]}


_OWN = {"write": _own_write, "read": _own_back, "attend": _own_attend, "shared": _own_shared}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


# ---------------------------------------------------------------------------


def work(case):
    G, H, d, e = case["G"], case["H"], case["d"], 2 if case["dtype"] == "bf16" else 4
    c = e * d if case["format"] == "plain" else d * BITS[case["format"]] // 8 + d // 32      # bytes of a row in the pages
    if case["op"] in ("write", "read"):
        start, new = (_lens(case["start"]), _lens(case["new"])) if case["op"] == "write" else ([0], [0])
        n = sum(new)
        m = sum(_lens(case["lens"])) if case["op"] == "read" else n + (sum(start) if case["back"] == "all" else 0)
        return {"bytes": n * (2 * e * d * (G + H) + 4 * d + 2 * G * c) + 2 * m * G * (c + e * d), "flops": n * d * (5 * G + 3 * H) + 2 * m * G * d}
    lens, per = _lens(case["lens"]), H // G
    pairs, moved = G * sum(lens), 2 * c * G * sum(lens) + len(lens) * H * (2 * e * d + 4)
    if case["op"] == "shared":
        counts = _counts(case["groups"], G, case["entries"])
        moved += sum(counts) * (2 * e * d + 4)
        pairs += sum(n * sum(counts[i * G:i * G + G]) for i, n in enumerate(_lens(case["groups"])))
    return {"bytes": moved, "flops": 4 * d * per * pairs}


# ---------------------------------------------------------------------------
# from the definitions, in 64 bits


def _exact_values(codes, scales, fmt):
    """The numbers that codes stand for, by the fields of their bits."""
    c = codes.long()
    if fmt == "e2m1":
        c = torch.stack([c % 16, c // 16], -1).flatten(-2)
    m, bias = (3, 7) if fmt == "e4m3" else (1, 1)
    sign, e, f = c >> (BITS[fmt] - 1), (c >> m) & ((1 << (BITS[fmt] - 1 - m)) - 1), (c & ((1 << m) - 1)).double() / (1 << m)
    x = torch.where(e > 0, (1 + f) * torch.exp2((e - bias).double()), f * 2.0 ** (1 - bias)) * (1 - 2 * sign)
    s = torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))
    return x * s.repeat_interleave(32, -1)


def _exact_round(x, fmt):
    """Rows x [..., d] (float64) as the blocks hold them: nearest multiples of the step, ties to the even one."""
    y = x.unflatten(-1, (-1, 32))
    largest, limit, bits, least = (448.0, 464.0, 3, -6) if fmt == "e4m3" else (6.0, 7.0, 1, 0)
    top = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1e-300) / limit)) - 1       # and from there upwards, exactly
    e = e + (top > limit * torch.exp2(e))
    scale = torch.exp2((e + (top > limit * torch.exp2(e))).clamp(min=-117))
    a = (y / scale).abs()
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** least))) - bits)
    a = (torch.round(a / step) * step).clamp(max=largest) * scale
    return torch.where(top < 2.0 ** 127, torch.where(y < 0, -a, a), math.nan).flatten(-2)


def _exact_rows(s, case):
    G, d, page, fmt = case["G"], case["d"], case["page"], case["format"]
    written = {}
    res = {}
    if case["op"] == "write":
        c, z = s["cos"].double()[s["pos"].long()][:, None], s["sin"].double()[s["pos"].long()][:, None]

        def turned(x, step):
            lo, hi = x.double()[..., :d // 2], x.double()[..., d // 2:]
            return torch.cat([step(step(lo * c) - step(hi * z)), step(step(hi * c) + step(lo * z))], -1)
        res["q"] = turned(s["q"], lambda x: x)
        # keys are quantised from products and sums that the definition has in fp32
        written = {"K": _exact_round(turned(s["k"], lambda x: x.float().double()), fmt), "V": _exact_round(s["v"].double(), fmt)}
    for name, to in (("K", "k"), ("V", "v")):
        rows, i = [], 0
        lens = _lens(case["lens"]) if case["op"] == "read" else [a + b for a, b in zip(_lens(case["start"]), _lens(case["new"]))]
        for b, n in enumerate(lens):
            n_new = _lens(case["new"])[b] if written else 0
            held = n - n_new
            if held and not (written and case["back"] == "new"):
                ids = s["table"][b, :-(-held // page)].long()
                x = _exact_values(s[name][ids], s[name + "s"][ids], fmt)
                rows.append(x.transpose(1, 2).reshape(-1, G, d)[:held])
            if n_new:
                rows.append(written[name][i:i + n_new])
                i += n_new
        res[to] = torch.cat(rows)
    return res


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("write", "read"):
        return _exact_rows(s, case)
    G, H, d, page, fmt = case["G"], case["H"], case["d"], case["page"], case["format"]
    per = H // G
    out, lse = s["out"].double(), s["lse"].double()
    group = [i for i, n in enumerate(_lens(case["groups"])) for _ in range(n)] if case["op"] == "shared" else None
    for b, n in enumerate(_lens(case["lens"])):
        ids = s["table"][b, :-(-n // page)].long()
        for g in range(G):
            k, v = (s[x][ids, g].double() if fmt == "plain" else _exact_values(s[x][ids, g], s[x + "s"][ids, g], fmt) for x in ("K", "V"))
            k, v = k.reshape(-1, d)[:n], v.reshape(-1, d)[:n]
            bias = torch.zeros(n, dtype=torch.float64, device=DEV)
            if group:
                at = int(s["p_start"][group[b] * G + g])
                to = at + int(s["p_count"][group[b] * G + g])
                k, v, bias = torch.cat([s["p_K"][at:to].double(), k]), torch.cat([s["p_V"][at:to].double(), v]), torch.cat([s["p_logm"][at:to].double(), bias])
            h = slice(g * per, (g + 1) * per)
            x = s["q"][b, h].double() @ k.T / math.sqrt(d) + bias
            lse[b, h] = torch.logsumexp(x, -1)
            out[b, h] = (x - lse[b, h, None]).exp() @ v
    return {"out": out, "lse": lse}
