"""Quantised pages and shared entries on the host: structures and argument checks (no GPU call is
made), and how groups' rows and entries are cut, compiled for the CPU."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

from paper_2608_07001_amd import gracekv as gk
from test_serve_host import _page

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(1 << 20)               # aligned, never dereferenced on these paths
ODD = ctypes.c_void_p((1 << 20) + 4)
SCALES = 8 * 16 * 4                           # bytes of a page's scales


def test_struct_layouts_match_the_header(tmp_path):
    pairs = [("gracekv_part", gk.PartArrays), ("gracekv_quant_pages", gk.QuantArrays), ("gracekv_read_config", gk.ReadConfig),
             ("gracekv_shared_config", gk.SharedConfig)]
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "gracekv.h"', "int main(void){"]
    want = []
    for name, cls in pairs:
        src.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
        for f, _ in cls._fields_:
            src.append(f'printf("%zu\\n", offsetof({name}, {f}));')
            want.append(getattr(cls, f).offset)
    src.append('printf("%d\\n%d\\n", GRACEKV_E4M3, GRACEKV_E2M1);')
    (tmp_path / "l.c").write_text("\n".join(src + ["return 0;}"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == want + [gk.E4M3, gk.E2M1]


def _quant(**kw):
    c = dict(format=gk.E4M3, reserved=0, scale_stride=SCALES, K=FAKE, V=FAKE, K_scale=FAKE, V_scale=FAKE)
    c.update(kw)
    return gk.QuantArrays(**c)


def _append(c, p, row=None, n_new=3, **kw):
    names = ["k", "v", "q", "table", "start", "cu", "pos", "cos", "sin", "q_out"]
    r = gk.AppendConfig(n_new, 16, 1024, 128, 1024, 128, 4096, 128, 4096, 128)
    for k, x in (row or {}).items():
        setattr(r, k, x)
    return gk.lib().gracekv_quant_append(ctypes.byref(c), ctypes.byref(r), None if p is None else ctypes.byref(p), *[kw.get(n, FAKE) for n in names], None)


def _read(c, p, row=None, n_rows=3, table=FAKE, start=FAKE, cu=FAKE, k=FAKE, v=FAKE):
    r = gk.ReadConfig(n_rows, 1024, 128, 1024, 128)
    for n, x in (row or {}).items():
        setattr(r, n, x)
    return gk.lib().gracekv_quant_read(ctypes.byref(c), ctypes.byref(r), None if p is None else ctypes.byref(p), table, start, cu, k, v, None)


def _attend(c, p, q=FAKE, q_tok=4096, table=FAKE, lens=FAKE, part=None, out=FAKE, ws=FAKE, n=0):
    return gk.lib().gracekv_quant_attention(ctypes.byref(c), None if p is None else ctypes.byref(p), q, q_tok, table, lens,
                                            None if part is None else ctypes.byref(part), out, None, ws, n, None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), -1), (dict(G=0), -1), (dict(H=31), -1), (dict(n_seq=0), -1), (dict(reserved=1), -1), (dict(page_size=8), -2),
    (dict(page_size=48), -2), (dict(table_width=0), -1), (dict(n_pages=0), -1), (dict(page_stride=8 * 16 * 128 - 16), -1),
    (dict(page_stride=8 * 16 * 128 + 8), -1), (dict(d=96), -2), (dict(n_pages=1 << 50), -1), (dict(n_seq=8193), -2)])
def test_pages_refuse_configurations(bad, code):
    c, p = _page(**bad), _quant()
    assert _append(c, p) == code and _read(c, p) == code and _attend(c, p) == code


@pytest.mark.parametrize("bad", [
    dict(format=2), dict(format=-1), dict(reserved=1), dict(scale_stride=SCALES - 16), dict(scale_stride=SCALES + 8), dict(K=None),
    dict(V=None), dict(K_scale=None), dict(V_scale=None), dict(K=ODD), dict(V=ODD), dict(K_scale=ODD), dict(V_scale=ODD)])
def test_pages_refuse_pools(bad):
    c, p = _page(), _quant(**bad)
    assert _append(c, p) == -1 and _read(c, p) == -1 and _attend(c, p) == -1
    assert _append(c, None) == -1 and _read(c, None) == -1 and _attend(c, None) == -1


def test_four_bits_need_pages_of_whole_pieces():
    # a multiple of 16 bytes of codes: 16 of e4m3, 32 of e2m1
    c = _page(page_stride=8 * 16 * 128 + 16)
    assert _attend(c, _quant()) == -4 and _attend(c, _quant(format=gk.E2M1)) == -1
    assert _attend(_page(page_stride=8 * 16 * 128 + 32), _quant(format=gk.E2M1)) == -4


def test_append_refuses_pointers_and_strides():
    c, p = _page(), _quant()
    names = ["k", "v", "q", "table", "start", "cu", "pos", "cos", "sin", "q_out"]
    for name in names:                        # one of a pair or triple missing is an error too
        assert _append(c, p, **{name: None}) == -1, name
    for name in ("k", "v", "q", "cos", "sin", "q_out"):
        assert _append(c, p, **{name: ODD}) == -1, name
    for bad in (dict(k_tok=4), dict(v_head=-8), dict(q_tok=12), dict(qout_tok=0), dict(qout_head=0), dict(rope_rows=-1)):
        assert _append(c, p, row=bad) == -1, bad
    assert _append(c, p, n_new=-1) == -1 and _append(c, p, n_new=1 << 24) == -2
    assert _append(c, p, n_new=0) == 0 and _append(c, p, n_new=0, k=None, v=None, q=None, pos=None, q_out=None) == 0


def test_read_refuses_pointers_and_strides():
    c, p = _page(), _quant()
    for name in ("table", "start", "cu"):
        assert _read(c, p, **{name: None}) == -1, name
    for name in ("k", "v"):
        assert _read(c, p, **{name: ODD}) == -1, name
    for bad in (dict(k_tok=4), dict(v_head=-8), dict(k_tok=0), dict(v_head=0)):      # rows on rows
        assert _read(c, p, row=bad) == -1, bad
    assert _read(c, p, n_rows=-1) == -1 and _read(c, p, n_rows=1 << 24) == -2
    assert _read(c, p, n_rows=0) == 0 and _read(c, p, k=None, v=None) == 0
    assert _read(c, p, n_rows=0, row=dict(k_tok=0, v_tok=0)) == 0


def _part(**kw):
    return gk.PartArrays(**dict(dict(o=FAKE, lse=FAKE), **kw))


def test_attention_refuses_pointers_and_workspaces():
    c, p = _page(), _quant()
    for name in ("q", "table", "lens", "out", "ws"):
        assert _attend(c, p, **{name: None}) == -1, name
    for name in ("q", "out", "ws"):
        assert _attend(c, p, **{name: ODD}) == -1, name
    assert _attend(c, p, q_tok=4) == -1 and _attend(c, p, q_tok=-4096) == -1
    assert _attend(c, p, n=gk.paged_ws_bytes(c) - 1) == -4
    f = gk.lib().gracekv_paged_attention_part
    for bad in (_part(o=None), _part(lse=None), _part(o=ODD)):
        assert _attend(c, p, part=bad) == -1
        assert f(ctypes.byref(c), FAKE, 4096, FAKE, FAKE, FAKE, FAKE, None, ctypes.byref(bad), FAKE, None, FAKE, 0, None) == -1
    assert _attend(c, p, part=_part()) == -4
    assert f(ctypes.byref(c), FAKE, 4096, FAKE, FAKE, FAKE, FAKE, None, ctypes.byref(_part()), FAKE, None, FAKE, 0, None) == -4


def _sc(**kw):
    c = dict(dtype=gk.BF16, G=8, H=32, d=128, n_seq=16, n_group=2, q_tok=4096)
    c.update(kw)
    return gk.SharedConfig(*[c[n] for n, _ in gk.SharedConfig._fields_])


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), -1), (dict(G=0), -1), (dict(H=31), -1), (dict(n_seq=0), -1), (dict(n_group=0), -1), (dict(q_tok=4), -1),
    (dict(q_tok=-8), -1), (dict(d=96), -2), (dict(n_group=8193), -2), (dict(H=1 << 17), -2), (dict(n_seq=(1 << 21) + 1), -2),
    (dict(n_seq=1 << 26, G=1, H=2), -2)])
def test_shared_refuses_configurations(bad, code):
    n, c = ctypes.c_size_t(0), _sc(**bad)
    assert gk.lib().gracekv_shared_ws_bytes(ctypes.byref(c), ctypes.byref(n)) == code
    pre = gk.PrefixArrays(FAKE, FAKE, FAKE, FAKE, FAKE, 10)
    assert gk.lib().gracekv_shared_attention(ctypes.byref(c), FAKE, FAKE, ctypes.byref(pre), ctypes.byref(_part()), FAKE, 1 << 40, None) == code


def test_shared_refuses_pointers_and_workspaces():
    c = _sc()
    good = dict(start=FAKE, count=FAKE, K=FAKE, V=FAKE, logm=FAKE, rows=10)

    def call(q=FAKE, cu=FAKE, pre=gk.PrefixArrays(**good), part=_part(), ws=FAKE, n=0):
        return gk.lib().gracekv_shared_attention(ctypes.byref(c), q, cu, None if pre is None else ctypes.byref(pre),
                                                 None if part is None else ctypes.byref(part), ws, n, None)
    for name in ("q", "cu", "pre", "part", "ws"):
        assert call(**{name: None}) == -1, name
    for name in ("q", "ws"):
        assert call(**{name: ODD}) == -1, name
    for name in ("start", "count", "K", "V", "logm"):
        assert call(pre=gk.PrefixArrays(**dict(good, **{name: None}))) == -1, name
    for bad in (dict(K=ODD), dict(V=ODD), dict(rows=-1)):
        assert call(pre=gk.PrefixArrays(**dict(good, **bad))) == -1, bad
    for bad in (_part(o=None), _part(lse=None), _part(o=ODD)):
        assert call(part=bad) == -1
    assert call(n=gk.shared_ws_bytes(c) - 1) == -4
    assert call(pre=gk.PrefixArrays(**dict(good, K=None, V=None, logm=None, rows=0))) == -4
    assert gk.lib().gracekv_shared_ws_bytes(ctypes.byref(c), None) == -1


GROUPS = r"""
#include <stdio.h>
#include <vector>
#include "groups.h"
using namespace gkv;
// a key tile's keys, a chunk's fewest tiles and a row's chunks as the kernels have them
static int keys_of(const SharedPlan& p, bool bf, int d) { return p.few ? (bf || d == 64 ? 32 : 16) * (p.waves / 4) : (bf ? 128 : 32); }
static int chunks(const SharedPlan& p, int n, int size, int d) { return p.few ? chunks_of(n, size, 0.6f * (d / 64) / (p.waves / 4)) : (n + size - 1) / size; }
int main() {
  int bf, G, per, d, B, S;
  while (scanf("%d %d %d %d %d %d", &bf, &G, &per, &d, &B, &S) == 6) {
    SharedDims sd{bf, G, G * per, d, per, B, S, 0};
    std::vector<int32_t> cu(S + 1);
    std::vector<long> count(S * G);
    for (auto& x : cu) if (scanf("%d", &x) != 1) return 1;
    for (auto& x : count) if (scanf("%ld", &x) != 1) return 1;
    long rows = 0;
    for (long x : count) rows += x;
    const SharedPlan p = shared_plan(sd, rows);
    int bad = 0;
    // row tiles: each group's own, in order, inside the table
    int64_t last = -1;
    unsigned long long total = 0;
    const int keys = keys_of(p, bf, d);
    std::vector<std::pair<int, long>> unit;
    for (int b = 0; b < S; ++b) {
      const Span sp = span_of(cu.data(), b, B);
      const int mt = tiles_of_group(sd, sp.n, p.rows);
      const int64_t a = first_tile(sd, (int)sp.a, b, p.rows);
      if (mt && a <= last) ++bad;
      if (mt) last = a + mt - 1;
      if (mt && (last + 1) * G > p.tiles) ++bad;
      for (int g = 0; g < G; ++g) {
        long n = (count[b * G + g] + keys - 1) / keys;
        if (n == 0) n = 1;
        unit.push_back({mt, n});
        total += (unsigned long long)mt * n;
      }
    }
    const int room = (int)(p.places - p.tiles);
    if (room < 1 || p.places % 8) ++bad;
    const int size = shared_chunk(total, room, p.few ? PA_MIN : 1);
    long long all = 0;
    for (auto& u : unit) all += (long long)u.first * chunks(p, (int)u.second, size, d);
    if (all > p.places) ++bad;                  // every chunk has a place
    printf("%d %d %d %lld\n", bad, p.few, p.waves, all);
  }
  return 0;
}
"""


def test_groups_are_cut_into_what_the_grid_holds(tmp_path):
    (tmp_path / "g.cpp").write_text(GROUPS)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2608_07001_amd", "csrc"),
                    str(tmp_path / "g.cpp"), "-o", str(tmp_path / "g")], check=True)
    r, text = random.Random(1), []
    for i in range(2000):
        S, G, per = int(2 ** r.uniform(0, 7)), r.choice([1, 2, 3, 8]), r.choice([1, 3, 4, 8, 20])
        groups = [r.choice([0, 1, r.randint(0, 9), r.randint(0, 200)]) for _ in range(S)]
        B = max(sum(groups), 1)
        cu = [sum(groups[:j]) for j in range(S + 1)]
        top = int(2 ** r.uniform(0, 17))
        counts = [r.randint(0, top) if r.random() < 0.8 else 0 for _ in range(S * G)]
        text.append(" ".join(map(str, [i % 2, G, per, r.choice([64, 128]), B, S] + cu + counts)))
    out = subprocess.run([str(tmp_path / "g")], input="\n".join(text), capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(text)
    for line, case in zip(out, text):
        assert line.split()[0] == "0", (line, case[:200])
    assert {tuple(line.split()[1:3]) for line in out} == {("1", "4"), ("1", "8"), ("0", "4"), ("0", "8")}       # every kernel among them


DESCENDING = r"""
#include <stdio.h>
#include <vector>
#include "groups.h"
using namespace gkv;
int main() {
  int G, per, B, S, n;
  while (scanf("%d %d %d %d %d", &G, &per, &B, &S, &n) == 5) {
    SharedDims sd{1, G, G * per, 128, per, B, S, 0};
    std::vector<int32_t> cu(S + 1);
    for (auto& x : cu) if (scanf("%d", &x) != 1) return 1;
    const SharedPlan p = shared_plan(sd, (int64_t)n * S * G);
    const int keys = p.few ? 8 * p.waves : 128, tiles = (n + keys - 1) / keys;
    int bad = 0, seen = 0;
    long long all = 0;
    unsigned long long total = 0;
    for (int b = 0; b < S; ++b) {
      const Span sp = span_of(cu.data(), b, B);
      const int mt = tiles_of_group(sd, sp.n, p.rows);
      total += (unsigned long long)G * mt * tiles;
      all += (long long)G * mt;
      if (mt && (int64_t)(first_tile(sd, (int)sp.a, b, p.rows) + mt) * G > p.tiles) ++bad;        // a ticket of every row tile
    }
    const int size = shared_chunk(total, (int)(p.places - p.tiles), p.few ? PA_MIN : 1);
    all *= p.few ? chunks_of(tiles, size, 4.8f / p.waves) : (tiles + size - 1) / size;
    std::vector<char> taken(p.places);
    for (int bid = 0; bid < p.places; ++bid) {
      const int id = item_of(bid, (int)all, p.places);
      if (id < -1 || id >= p.places || (id >= 0 && taken[id])) ++bad;
      else if (id >= 0) { taken[id] = 1; ++seen; }
    }
    if (seen != (all < p.places ? all : p.places)) ++bad;
    printf("%d %d\n", bad, all > p.places);
  }
  return 0;
}
"""


def test_descending_groups_stay_inside_the_workspace(tmp_path):
    # bounds that go up and down give rows to several groups: more items than the grid has places
    (tmp_path / "g.cpp").write_text(DESCENDING)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2608_07001_amd", "csrc"),
                    str(tmp_path / "g.cpp"), "-o", str(tmp_path / "g")], check=True)
    r, text = random.Random(2), []
    for _ in range(1000):
        G, S, B = r.choice([1, 2, 3]), r.randint(1, 64), int(2 ** r.uniform(0, 13))
        cu = r.choice([[B * (j % 2) for j in range(S + 1)], [r.randint(-3, B + 3) for _ in range(S + 1)]])
        text.append(" ".join(map(str, [G, r.choice([1, 4, 8, 20]), B, S, int(2 ** r.uniform(0, 15))] + cu)))
    out = subprocess.run([str(tmp_path / "g")], input="\n".join(text), capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(text)
    for line, case in zip(out, text):
        assert line.split()[0] == "0", (line, case[:200])
    assert sum(line.split()[1] == "1" for line in out) > 50


def test_binding_refuses_other_tensors(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)           # noqa: E731
    table = torch.zeros(1, 3, dtype=torch.int32)
    pages = gk.QuantPages(gk.E2M1, u8(3, 2, 16, 32), u8(3, 2, 16, 32), u8(3, 2, 16, 2), u8(3, 2, 16, 2))
    cfg = gk.quant_config(pages, torch.float32, 4, table)
    assert (cfg.d, cfg.G, cfg.H, cfg.page_size, cfg.page_stride) == (64, 2, 4, 16, 2048)
    with pytest.raises(ValueError, match="format"):
        gk.QuantPages(7, *[pages.K] * 4)
    with pytest.raises(ValueError, match="page_size"):
        gk.QuantPages(gk.E4M3, *[u8(3, 2, 64)] * 4)
    for name, x in (("K", u8(3, 2, 16, 64)), ("V", u8(2, 2, 16, 32)), ("K_scale", u8(3, 2, 16, 4)),
                    ("V_scale", torch.zeros(3, 2, 16, 2, dtype=torch.int8)), ("V", u8(6, 2, 16, 32)[::2]),
                    ("V_scale", u8(6, 2, 16, 2)[::2]), ("K_scale", u8(3, 2, 2, 16).transpose(2, 3))):
        with pytest.raises(ValueError, match="K_scale|V" if name == "K" else name):
            gk.QuantPages(**{f: x if f == name else getattr(pages, f) for f in ("format", "K", "V", "K_scale", "V_scale")})
    with pytest.raises(AttributeError):                          # the tensors are looked over once
        pages.K = u8(3, 2, 16, 32)
    with pytest.raises(ValueError, match="float16"):
        gk.quant_config(pages, torch.float16, 4, table)
    with pytest.raises(ValueError, match="table_width"):
        gk.quant_config(pages, torch.float32, 4, table[0])
    q, kv, i = torch.zeros(1, 4, 64), torch.zeros(1, 2, 64), torch.zeros(1, dtype=torch.int32)
    cu = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="on cpu"):              # no copies behind the caller's back
        gk.quant_append(cfg, pages, kv, kv, table, i, cu)
    with pytest.raises(ValueError, match="on cpu"):
        gk.quant_read(cfg, pages, table, i, cu, kv, kv)
    with pytest.raises(ValueError, match="on cpu"):
        gk.quant_attention(cfg, pages, q, table, i, q, None)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    with pytest.raises(ValueError, match="on device -1"):
        gk.quant_attention(cfg, pages, q, table, i, q, None)
    four = gk.QuantPages(gk.E2M1, *[torch.cat([x, x[:1]]) for x in (pages.K, pages.V, pages.K_scale, pages.V_scale)])
    with pytest.raises(ValueError, match="n_pages"):             # another cache's shapes
        gk.quant_attention(cfg, four, q, table, i, q, None)
    pages = gk.QuantPages(gk.E2M1, pages.K, pages.V, pages.K_scale, pages.V_scale)
    with pytest.raises(ValueError, match="part.lse"):
        gk.Part(torch.zeros(1, 4, 64), torch.zeros(1, 3))
    with pytest.raises(ValueError, match="part.o"):
        gk.Part(torch.zeros(1, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 4))
    with pytest.raises(ValueError, match="part.o"):
        gk.Part(torch.zeros(1, 64), torch.zeros(1))
    with pytest.raises(ValueError, match="part: got"):
        gk.quant_attention(cfg, pages, q, table, i, q, None, part=gk.Part(torch.zeros(2, 4, 64), torch.zeros(2, 4)))
    part = gk.Part(torch.zeros(1, 4, 64), torch.zeros(1, 4))
    sc = gk.shared_config(q, 2, 1)
    pre = gk.Prefix(torch.zeros(2, dtype=torch.int64), torch.zeros(2, dtype=torch.int64), torch.zeros(5, 64), torch.zeros(5, 64), torch.zeros(5))
    with pytest.raises(ValueError, match="cu_group"):
        gk.shared_attention(sc, q, torch.zeros(3, dtype=torch.int32), pre, part, None)
    with pytest.raises(ValueError, match="prefix.start"):
        gk.shared_attention(sc, q, cu, gk.Prefix(**dict(pre.__dict__, start=torch.zeros(4, dtype=torch.int64))), part, None)
