"""The operators around the compressed cache on the host: their structures and argument
checks (no GPU call is made), and the index arithmetic of the pages, compiled for the CPU."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

import serve_harness as S
from paper_2608_07001_amd import gracekv as gk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = ctypes.c_void_p(1 << 20)               # aligned, never dereferenced on these paths
ODD = ctypes.c_void_p((1 << 20) + 4)


def test_struct_layouts_match_the_header(tmp_path):
    pairs = [("gracekv_prompt_config", gk.PromptConfig), ("gracekv_page_config", gk.PageConfig),
             ("gracekv_append_config", gk.AppendConfig), ("gracekv_prefix", gk.PrefixArrays)]
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "gracekv.h"', "int main(void){"]
    want = []
    for name, cls in pairs:
        src.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
        for f, _ in cls._fields_:
            src.append(f'printf("%zu\\n", offsetof({name}, {f}));')
            want.append(getattr(cls, f).offset)
    (tmp_path / "l.c").write_text("\n".join(src + ["return 0;}"]))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    out = subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == want


PAGES = r"""
#include <stdio.h>
#include "pages.h"
using namespace gkv;
int main() {
  int bad = 0;
  for (int shift = 4; shift <= 8; ++shift)
    for (int G = 1; G <= 3; ++G) {
      PageDims p{1, G, G, 64, 1, 2, shift, 5, 7, (int64_t)G * 64 * (1 << shift) + 128};
      // every row of every page lies inside the pool and no two meet
      int64_t last = -1;
      for (int64_t id = 0; id < p.n_pages; ++id)
        for (int g = 0; g < G; ++g)
          for (int at = 0; at < (1 << shift); ++at) {
            const int64_t r = page_row(p, id, g, at);
            if (r <= last || r % 64 || r + 64 > p.n_pages * p.page_stride) ++bad;
            last = r + 63;
          }
      // no page: nothing
      const int64_t none[] = {-1, -7, 7, 8, 2147483647, -2147483648LL};
      for (int64_t id : none) if (page_row(p, id, 0, 0) != -1) ++bad;
      // lengths are held to what the table can name
      const int64_t most = 5LL << shift;
      if (held_len(p, -1) != 0 || held_len(p, 0) != 0 || held_len(p, most) != most || held_len(p, most + 1) != most ||
          held_len(p, 2147483647) != most) ++bad;
    }
  // pages far apart: elements past 32 bits
  PageDims far{1, 8, 8, 128, 1, 1, 8, 4, 1 << 20, 1 << 18};
  if (page_row(far, (1 << 20) - 1, 7, 255) != ((1LL << 20) - 1) * (1 << 18) + (7 * 256 + 255) * 128LL) ++bad;
  // spans: inside, past the end, descending, negative
  const int32_t cu[] = {0, 3, 3, 9, 4, 100, -5, 2};
  const int64_t want[][2] = {{0, 3}, {3, 0}, {3, 6}, {9, 0}, {4, 6}, {10, 0}, {0, 2}};
  for (int b = 0; b < 7; ++b) {
    const Span s = span_of(cu, b, 10);
    if (s.a != want[b][0] || s.n != want[b][1]) ++bad;
  }
  printf("%d\n", bad);
  return 0;
}
"""


def test_page_arithmetic(tmp_path):
    (tmp_path / "p.cpp").write_text(PAGES)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2608_07001_amd", "csrc"),
                    str(tmp_path / "p.cpp"), "-o", str(tmp_path / "p")], check=True)
    assert subprocess.run([str(tmp_path / "p")], capture_output=True, text=True, check=True).stdout.strip() == "0"


CHUNKS = r"""
#include <stdio.h>
#include <algorithm>
#include <vector>
#include "pages.h"
using namespace gkv;
// how a call's rows are cut: what launch_paged and find_chunk work out, printed for every shape read
template <int TILE> void replay(const PageDims& p, int64_t px_rows, const std::vector<long>& len, const std::vector<long>& count) {
  const int R = p.n_seq * p.G, units = px_rows ? R : p.n_seq, mult = px_rows ? 1 : p.G;
  const int room = (int)chunk_room(p, px_rows, TILE);
  std::vector<int> n;
  uint64_t total = 0;
  for (int u = 0; u < units; ++u) {
    n.push_back(tiles_of<TILE>(held_len(p, len[px_rows ? u / p.G : u]), px_rows ? count[u] : 0));
    total += (uint64_t)n[u] * mult;
  }
  const int size = chunk_tiles(total, room);
  int64_t sum = 0;
  int most = 0;
  for (int x : n) {
    const int c = chunks_of(x, size, join_cost(p.hpg, p.d));
    sum += (int64_t)c * mult;
    most = std::max(most, c);
    if (c < 1 || (int64_t)(c - 1) * size >= x) most = 1 << 30;          // no chunk is empty
  }
  printf("%d %d %d %d %llu %lld %d\n", units, room, size, *std::max_element(n.begin(), n.end()), (unsigned long long)total,
         (long long)sum, most);
}
int main() {
  int bf, G, H, d, B, shift, width;
  long px;
  while (scanf("%d %d %d %d %d %d %d %ld", &bf, &G, &H, &d, &B, &shift, &width, &px) == 8) {
    PageDims p{bf, G, H, d, H / G, B, shift, width, 1, 1};
    std::vector<long> len(B), count(px ? B * G : 0);
    for (long& x : len) if (scanf("%ld", &x) != 1) return 1;
    for (long& x : count) if (scanf("%ld", &x) != 1) return 1;
    if (!bf && d == 128) replay<16>(p, px, len, count); else replay<32>(p, px, len, count);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def chunks(tmp_path_factory):
    """chunks(shapes): for each (dtype, d, G, H, lens, page, counts, rows) the units looked through, places beside
    one a row, tiles of a chunk, of the longest row and of all, chunks of all and of the row with the most."""
    at = tmp_path_factory.mktemp("chunks")
    (at / "c.cpp").write_text(CHUNKS)
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2608_07001_amd", "csrc"),
                    str(at / "c.cpp"), "-o", str(at / "c")], check=True)

    def run(shapes):
        text = []
        for dtype, d, G, Hq, lens, page, counts, rows in shapes:
            width = max(max(-(-n // page) for n in lens), 1)
            text.append(" ".join(map(str, [int(dtype == "bf16"), G, Hq, d, len(lens), page.bit_length() - 1, width, rows] + lens
                                     + (counts or []))))
        out = subprocess.run([str(at / "c")], input="\n".join(text), capture_output=True, text=True, check=True).stdout
        return [[int(x) for x in line.split()] for line in out.splitlines()]
    return run


def test_chunks_fit_the_grid(chunks):
    """Every row's chunks have a place whatever the lengths are, none is empty, and the grid is as large
    as rows with entries of their own could use."""
    r = random.Random(1)
    shapes = []
    for i in range(3000):
        G = r.choice([1, 2, 3, 8])
        B = int(2 ** r.uniform(0, 9))
        page = r.choice([16, 64, 256])
        top = int(2 ** r.uniform(0, 17))
        lens = [r.randint(0, top) if r.random() < 0.8 else r.choice([0, 1, 15, 33]) for _ in range(B)]
        counts, rows = None, 0
        if i % 2:                                              # entries of their own, or shared
            few = int(2 ** r.uniform(0, 15))
            counts = [r.randint(0, few) for _ in range(B * G)]
            rows = sum(counts) + 1 if i % 4 == 1 else few
        shapes.append((r.choice(["bf16", "f32"]), r.choice([64, 128]), G, G * r.choice([1, 4, 8, 20]), lens, page, counts, rows))
    for shape, (units, room, size, longest, total, all_chunks, most) in zip(shapes, chunks(shapes)):
        R = len(shape[4]) * shape[2]
        assert most < 1 << 30 and all_chunks <= R + room, shape
        target = 768 if R < 256 else 1536
        if not shape[7] or shape[7] > sum(shape[6]):
            assert room >= min(max(target - R // 2, target // 4), -(-total // 4) - R), shape


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
def test_shapes_of_the_rarer_ways_take_them(chunks, dtype, d):
    """The shapes that tests/test_gpu_serve.py runs for the search past its first round and for the join's
    second block do reach them."""
    shapes = S.paged_shapes()
    cut = chunks([(dtype, d, G, Hq, lens, page, counts, sum(counts) + 3 if counts else 0)
                  for G, Hq, lens, page, counts in shapes.values()])
    for name, (units, room, size, longest, total, all_chunks, most) in zip(shapes, cut):
        if name.startswith("searched"):
            assert units > 64 and longest > size and most > 1, name
        else:
            assert most > d // 2, name


def _prompt(**kw):
    c = dict(dtype=gk.BF16, G=8, H=32, d=128, n_seq=2, reserved=0, n_q=64, n_k=128, q_tok=4096, q_head=128, k_tok=1024, k_head=128,
             v_tok=1024, v_head=128, out_tok=4096, out_head=128)
    c.update(kw)
    return gk.PromptConfig(*[c[n] for n, _ in gk.PromptConfig._fields_])


def _page(**kw):
    c = dict(dtype=gk.BF16, G=8, H=32, d=128, n_seq=4, page_size=16, table_width=9, reserved=0, n_pages=40, page_stride=8 * 16 * 128)
    c.update(kw)
    return gk.PageConfig(*[c[n] for n, _ in gk.PageConfig._fields_])


def _status(f, *a):
    return f(*[ctypes.byref(x) if isinstance(x, ctypes.Structure) else x for x in a])


def _prompt_call(cfg, drop=None, odd=None, ws=FAKE, ws_bytes=1 << 40):
    ptr = [FAKE] * 6                          # Q K V cu_q cu_k out
    if drop is not None:
        ptr[drop] = None
    if odd is not None:
        ptr[odd] = ODD
    return _status(gk.lib().gracekv_prompt_attention, cfg, *ptr, None, ws, ws_bytes, None)


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), -1), (dict(G=0), -1), (dict(H=30), -1), (dict(n_seq=0), -1), (dict(reserved=1), -1), (dict(n_q=-1), -1),
    (dict(n_k=-1), -1), (dict(n_q=1 << 31), -1), (dict(d=96), -2), (dict(q_tok=4), -1), (dict(k_head=-128), -1), (dict(v_tok=12), -1),
    (dict(out_tok=0), -1), (dict(out_head=0), -1), (dict(out_head=4), -1), (dict(k_tok=(1 << 24) + 8), -2),
    (dict(n_seq=1 << 24), -2), (dict(n_seq=(1 << 31) - 1), -2), (dict(n_seq=1 << 22), -2), (dict(n_q=1 << 26), -2),
    (dict(n_q=1 << 30, G=1, H=1, dtype=gk.F32), -2), (dict(n_q=1 << 24, H=128), -2)])
def test_prompt_refuses_configurations(bad, code):
    n = ctypes.c_size_t(0)
    assert _status(gk.lib().gracekv_prompt_ws_bytes, _prompt(**bad), ctypes.byref(n)) == code
    assert _prompt_call(_prompt(**bad)) == code


def test_prompt_refuses_pointers_and_workspaces():
    c = _prompt(n_k=4096)
    for i in range(6):
        assert _prompt_call(c, drop=i) == -1
    for i in (0, 1, 2, 5):
        assert _prompt_call(c, odd=i) == -1
    need = gk.prompt_ws_bytes(c)              # 64 tokens x 4 heads are few rows: the keys are split
    assert need > 0
    assert _prompt_call(c, ws=None) == -1 and _prompt_call(c, ws=ODD) == -1
    assert _prompt_call(c, ws_bytes=need - 1) == -4
    assert gk.prompt_ws_bytes(_prompt(n_q=65536, n_k=65536)) == 0
    assert _status(gk.lib().gracekv_prompt_ws_bytes, c, None) == -1
    assert gk.lib().gracekv_prompt_attention(None, *[FAKE] * 6, None, FAKE, 1 << 40, None) == -1


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), -1), (dict(G=0), -1), (dict(H=31), -1), (dict(n_seq=0), -1), (dict(reserved=1), -1), (dict(page_size=8), -2),
    (dict(page_size=48), -2), (dict(page_size=512, page_stride=1 << 22), -2), (dict(table_width=0), -1), (dict(n_pages=0), -1),
    (dict(page_stride=8 * 16 * 128 - 8), -1), (dict(page_stride=8 * 16 * 128 + 4), -1), (dict(d=80), -2),
    (dict(n_pages=1 << 50), -1), (dict(table_width=(1 << 21) + 1), -2), (dict(n_seq=8193), -2),
    (dict(n_seq=65536, G=1, H=65536), -2)])
def test_pages_refuse_configurations(bad, code):
    n, c = ctypes.c_size_t(0), _page(**bad)
    rows = gk.AppendConfig(1, 16, 1024, 128, 1024, 128, 4096, 128, 4096, 128)
    assert _status(gk.lib().gracekv_paged_ws_bytes, c, ctypes.byref(n)) == code
    assert _status(gk.lib().gracekv_paged_attention, c, FAKE, 4096, FAKE, FAKE, FAKE, FAKE, None, FAKE, None, FAKE, 1 << 40, None) == code
    assert _status(gk.lib().gracekv_cache_append, c, rows, *[FAKE] * 12, None) == code


def test_paged_refuses_pointers_and_workspaces():
    c = _page()
    f = gk.lib().gracekv_paged_attention

    def call(q=FAKE, q_tok=4096, k=FAKE, v=FAKE, table=FAKE, lens=FAKE, prefix=None, out=FAKE, ws=FAKE, n=1 << 40):
        return f(ctypes.byref(c), q, q_tok, k, v, table, lens, None if prefix is None else ctypes.byref(prefix), out, None, ws, n, None)
    for name in ("q", "k", "v", "table", "lens", "out", "ws"):
        assert call(**{name: None}) == -1, name
    for name in ("q", "k", "v", "out", "ws"):
        assert call(**{name: ODD}) == -1, name
    assert call(q_tok=4) == -1 and call(q_tok=-4096) == -1
    assert call(n=gk.paged_ws_bytes(c) - 1) == -4
    good = dict(start=FAKE, count=FAKE, K=FAKE, V=FAKE, logm=FAKE, rows=10)
    for name in ("start", "count", "K", "V", "logm"):
        assert call(prefix=gk.PrefixArrays(**dict(good, **{name: None})), n=0) == -1, name
    assert call(prefix=gk.PrefixArrays(**dict(good, K=ODD)), n=0) == -1
    assert call(prefix=gk.PrefixArrays(**dict(good, rows=-1)), n=0) == -1
    assert call(prefix=gk.PrefixArrays(**good), n=0) == -4
    none = dict(good, K=None, V=None, logm=None, rows=0)
    assert call(prefix=gk.PrefixArrays(**none), n=0) == -4
    assert call(prefix=gk.PrefixArrays(**dict(none, start=None)), n=0) == -1


def test_append_refuses_pointers_and_strides():
    c = _page()
    names = ["k", "v", "q", "table", "start", "cu", "pos", "cos", "sin", "K", "V", "q_out"]

    def call(row=None, n_new=3, **kw):
        r = gk.AppendConfig(n_new, 16, 1024, 128, 1024, 128, 4096, 128, 4096, 128)
        for k, x in (row or {}).items():
            setattr(r, k, x)
        return gk.lib().gracekv_cache_append(ctypes.byref(c), ctypes.byref(r), *[kw.get(n, FAKE) for n in names], None)
    for name in names:                        # one of a pair or triple missing is an error too
        assert call(**{name: None}) == -1, name
    for name in ("k", "v", "q", "cos", "sin", "K", "V", "q_out"):
        assert call(**{name: ODD}) == -1, name
    for bad in (dict(k_tok=4), dict(v_head=-8), dict(q_tok=12), dict(qout_tok=0), dict(qout_head=0), dict(rope_rows=-1)):
        assert call(row=bad) == -1, bad
    assert call(n_new=-1) == -1 and call(n_new=1 << 24) == -2 and call(n_new=1 << 31) == -2
    assert gk.lib().gracekv_cache_append(ctypes.byref(c), None, *[FAKE] * 12, None) == -1


def test_nothing_to_append_is_no_error():
    # a call of no tokens: tensors without elements have no address, tables and pools do
    c = _page()
    names = ["k", "v", "q", "table", "start", "cu", "pos", "cos", "sin", "K", "V", "q_out"]

    def call(n_new=0, rope_rows=16, **kw):
        r = gk.AppendConfig(n_new, rope_rows, 1024, 128, 1024, 128, 4096, 128, 4096, 128)
        return gk.lib().gracekv_cache_append(ctypes.byref(c), ctypes.byref(r), *[kw.get(n, FAKE) for n in names], None)
    assert call() == 0
    assert call(k=None, v=None, q=None, q_out=None, pos=None) == 0
    assert call(k=None, v=None, q=None, pos=None) == 0         # the output's buffer may be there all the same
    assert call(rope_rows=0, cos=None, sin=None) == 0 and call(pos=None, cos=None, sin=None) == 0
    for name in ("table", "start", "cu", "K", "V"):
        assert call(**{name: None}) == -1, name
    for name in ("k", "cos", "K", "q_out"):
        assert call(**{name: ODD}) == -1, name
    for kw in (dict(pos=None), dict(q=None), dict(cos=None), dict(cos=None, sin=None, rope_rows=0), dict(k=None)):
        assert call(n_new=3, **kw) == -1, kw


def test_binding_refuses_other_tensors(monkeypatch):
    q, k = torch.zeros(4, 8, 64), torch.zeros(4, 2, 64)
    with pytest.raises(ValueError, match="k: got 32"):
        gk.prompt_config(q, torch.zeros(4, 2, 32), k, q, 1)
    with pytest.raises(ValueError, match="v"):
        gk.prompt_config(q, k, torch.zeros(5, 2, 64), q, 1)
    with pytest.raises(ValueError, match="out"):
        gk.prompt_config(q, k, k, torch.zeros(3, 8, 64), 1)
    with pytest.raises(ValueError, match="contiguous heads"):
        gk.prompt_config(torch.zeros(4, 8, 128)[..., ::2], k, k, q, 1)
    with pytest.raises(ValueError, match="float16"):
        gk.prompt_config(q.half(), k.half(), k.half(), q.half(), 1)
    with pytest.raises(ValueError, match="strides"):
        gk.page_config(torch.zeros(3, 2, 32, 64)[:, :, ::2], 2, torch.zeros(1, 3, dtype=torch.int32))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    cfg, cu = gk.prompt_config(q, k, k, q, 1), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="on cpu"):          # no copies behind the caller's back
        gk.prompt_attention(cfg, q, k, k, cu, cu, q)
    with pytest.raises(ValueError, match="float32"):
        gk.prompt_attention(cfg, q.bfloat16(), k, k, cu, cu, q)
    with pytest.raises(ValueError, match="strides"):
        gk.prompt_attention(cfg, q.transpose(0, 1).contiguous().transpose(0, 1), k, k, cu, cu, q)
    class Other:
        device_index, cuda_stream = 1, 1 << 20
    with pytest.raises(ValueError, match="device 1"):
        gk._raw(Other(), 0)
    # a length of one has no stride that matters
    one = torch.zeros(1, 8, 64).as_strided((1, 8, 64), (3, 64, 1))
    assert gk.prompt_config(one, k, k, one, 1).q_tok == 0
