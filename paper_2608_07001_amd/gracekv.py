"""Python binding of libgracekv (ctypes).  Argument marshalling only: every
step of the path runs in the HIP kernels of the library; torch supplies device
memory and the stream.  The functions carry the names of the C ABI
(include/gracekv.h) without the ``gracekv_`` prefix.  A missing library raises
instead of falling back to anything else."""
from __future__ import annotations

import ctypes
import dataclasses
import os
from typing import Dict, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgracekv.so")

F32, BF16 = 0, 1
E4M3, E2M1 = 0, 1        # formats of quantised pages
ABI_VERSION = 13         # GRACEKV_ABI_VERSION this binding is written for
_STATUS = {0: "ok", -1: "invalid argument", -2: "unsupported configuration", -3: "budget",
           -4: "workspace too small", -5: "HIP error", -6: "numeric fault on the device",
           -7: "the tree buffer holds no build", -8: "malformed slot partition on the device",
           -9: "packed cache over its capacity on the device"}


class GraceKVError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {_STATUS.get(status, status)} ({status})")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [("L", ctypes.c_int32), ("G", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32),
                ("n_seg", ctypes.c_int32), ("D_hidden", ctypes.c_int32), ("W", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("N_ctx", ctypes.c_int64), ("x", ctypes.c_double),
                ("r_default", ctypes.c_int32), ("r_min", ctypes.c_int32),
                ("lam_stab", ctypes.c_float), ("lam_s", ctypes.c_float), ("eps_seg", ctypes.c_float),
                ("mad_factor", ctypes.c_float), ("win", ctypes.c_int32 * 3),
                ("n_min", ctypes.c_int32), ("n_max", ctypes.c_int32), ("n0", ctypes.c_int32),
                ("lam_d", ctypes.c_float), ("lam_n", ctypes.c_float), ("c_cut", ctypes.c_float),
                ("lam_Z", ctypes.c_float), ("lam_M", ctypes.c_float), ("k_curv", ctypes.c_int32),
                ("lam_kappa", ctypes.c_float), ("beta_frac", ctypes.c_float), ("eps", ctypes.c_float),
                ("lambda_graph", ctypes.c_float), ("alpha_floor", ctypes.c_double), ("flags", ctypes.c_int32)]

FLAG_PRUNE = 1
FLAG_DP_SERIAL = 2
FLAG_UNIFORM_SLOTS = 4
FLAG_PAIR_QUOTAS = 8
FLAG_STATS_READY = 16
FLAG_STAGE_TIMES = 32
# stage ids of the stage clock (GRACEKV_STAGE_*), in order
STAGES = ["segment", "rowstats", "token_relevance", "root", "root_split", "refine", "pack", "floor_candidates",
          "floor_realise"]


_OFFS = ["off_node_a", "off_node_n", "off_node_child", "off_node_parent", "off_node_nch", "off_node_kind",
         "off_node_cut", "off_node_D", "off_node_R", "off_sp_U", "off_sp_E", "off_sp_cost", "off_sp_exec",
         "off_unit_nn", "off_unit_Ddrop", "off_add_U", "off_add_E", "off_add_exec", "off_tok_R",
         "off_tok_A", "off_row_stats", "off_probe_m", "off_probe_ZC", "off_lg_S", "off_omega", "off_status", "off_slots",
         "off_nslots", "off_partial", "off_theta", "off_selstate", "off_work", "off_wctr", "off_proto",
         "off_proto_logm", "off_floor"]


class Plan(ctypes.Structure):
    _fields_ = ([("T", ctypes.c_int64), ("N_c", ctypes.c_int64), ("B_total", ctypes.c_int64),
                 ("B_free", ctypes.c_int64), ("r", ctypes.c_int32), ("J_cap", ctypes.c_int32),
                 ("unit_cap", ctypes.c_int64), ("node_cap", ctypes.c_int64),
                 ("seg_ws_bytes", ctypes.c_size_t), ("tree_bytes", ctypes.c_size_t),
                 ("sel_ws_bytes", ctypes.c_size_t), ("pack_ws_bytes", ctypes.c_size_t)]
                + [(n, ctypes.c_size_t) for n in _OFFS] + [("build_lds_bytes", ctypes.c_int32),
                                                            ("build_ws_bytes", ctypes.c_size_t)])


class PromptConfig(ctypes.Structure):
    """gracekv_prompt_config."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "G", "H", "d", "n_seq", "reserved")]
                + [(n, ctypes.c_int64) for n in ("n_q", "n_k", "q_tok", "q_head", "k_tok", "k_head", "v_tok", "v_head",
                                                 "out_tok", "out_head")])


class PageConfig(ctypes.Structure):
    """gracekv_page_config."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "G", "H", "d", "n_seq", "page_size", "table_width", "reserved")]
                + [(n, ctypes.c_int64) for n in ("n_pages", "page_stride")])


class AppendConfig(ctypes.Structure):
    """gracekv_append_config."""
    _fields_ = [(n, ctypes.c_int64) for n in ("n_new", "rope_rows", "k_tok", "k_head", "v_tok", "v_head", "q_tok", "q_head",
                                              "qout_tok", "qout_head")]


class PrefixArrays(ctypes.Structure):
    """gracekv_prefix."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("start", "count", "K", "V", "logm")] + [("rows", ctypes.c_int64)]


class PartArrays(ctypes.Structure):
    """gracekv_part."""
    _fields_ = [("o", ctypes.c_void_p), ("lse", ctypes.c_void_p)]


class QuantArrays(ctypes.Structure):
    """gracekv_quant_pages."""
    _fields_ = ([("format", ctypes.c_int32), ("reserved", ctypes.c_int32), ("scale_stride", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("K", "V", "K_scale", "V_scale")])


class ReadConfig(ctypes.Structure):
    """gracekv_read_config."""
    _fields_ = [(n, ctypes.c_int64) for n in ("n_rows", "k_tok", "k_head", "v_tok", "v_head")]


class SharedConfig(ctypes.Structure):
    """gracekv_shared_config."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "G", "H", "d", "n_seq", "n_group")] + [("q_tok", ctypes.c_int64)])


SYMBOLS = ["gracekv_abi_version", "gracekv_default_config", "gracekv_plan_sizes", "gracekv_status_string", "gracekv_check",
           "gracekv_segment", "gracekv_build_trees", "gracekv_score", "gracekv_select", "gracekv_pack",
           "gracekv_selftest_mfma", "gracekv_decode_ws_bytes", "gracekv_decode_attention", "gracekv_relevance_stats",
           "gracekv_decode_attention_noalloc", "gracekv_stage_times", "gracekv_prompt_ws_bytes", "gracekv_prompt_attention",
           "gracekv_cache_append", "gracekv_paged_ws_bytes", "gracekv_paged_attention", "gracekv_paged_attention_part",
           "gracekv_quant_append", "gracekv_quant_read", "gracekv_quant_attention", "gracekv_shared_ws_bytes",
           "gracekv_shared_attention"]

_lib = None


def lib() -> ctypes.CDLL:
    """Loads libgracekv.so from the package directory (raises if not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build()")
    L = ctypes.CDLL(LIB_PATH)
    # argument lists and structures differ across interface versions: refuse a stale library
    if not hasattr(L, "gracekv_abi_version"):
        raise RuntimeError(f"{LIB_PATH} predates the versioned interface; rebuild it")
    L.gracekv_abi_version.argtypes = []
    L.gracekv_abi_version.restype = ctypes.c_int32
    if L.gracekv_abi_version() != ABI_VERSION:
        raise RuntimeError(f"{LIB_PATH} has interface version {L.gracekv_abi_version()}, "
                           f"this binding needs {ABI_VERSION}; rebuild it")
    P = ctypes.c_void_p
    S = ctypes.c_size_t
    sig = {
        "gracekv_default_config": [ctypes.POINTER(Config)],
        "gracekv_plan_sizes": [ctypes.POINTER(Config), ctypes.POINTER(Plan)],
        "gracekv_check": [ctypes.POINTER(Config), P, P],
        "gracekv_segment": [ctypes.POINTER(Config), P, P, P, P, P, P, P, S, P],
        "gracekv_build_trees": [ctypes.POINTER(Config), P, P, P, P, P, P, P, P, P, P, P, P, S, P],
        "gracekv_score": [ctypes.POINTER(Config), P, P, P],
        "gracekv_select": [ctypes.POINTER(Config), P, P, P, S, P],
        "gracekv_pack": [ctypes.POINTER(Config), P, P, P, P, P, P, P, P, P, P, P, P, S, P],
        "gracekv_selftest_mfma": [ctypes.c_int32, P, P],
        "gracekv_decode_ws_bytes": [ctypes.POINTER(Config), ctypes.POINTER(S)],
        "gracekv_relevance_stats": [ctypes.POINTER(Config), P, P, P, P],
        "gracekv_decode_attention": [ctypes.POINTER(Config), P, P, P, P, P, P, P, P, P, S, P],
        "gracekv_decode_attention_noalloc": [ctypes.POINTER(Config), P, P, P, P, P, P, P, P, P],
        "gracekv_stage_times": [P, P],
        "gracekv_prompt_ws_bytes": [ctypes.POINTER(PromptConfig), ctypes.POINTER(S)],
        "gracekv_prompt_attention": [ctypes.POINTER(PromptConfig), P, P, P, P, P, P, P, P, S, P],
        "gracekv_cache_append": [ctypes.POINTER(PageConfig), ctypes.POINTER(AppendConfig), P, P, P, P, P, P, P, P, P, P, P, P, P],
        "gracekv_paged_ws_bytes": [ctypes.POINTER(PageConfig), ctypes.POINTER(S)],
        "gracekv_paged_attention": [ctypes.POINTER(PageConfig), P, ctypes.c_int64, P, P, P, P, ctypes.POINTER(PrefixArrays),
                                    P, P, P, S, P],
        "gracekv_paged_attention_part": [ctypes.POINTER(PageConfig), P, ctypes.c_int64, P, P, P, P, ctypes.POINTER(PrefixArrays),
                                         ctypes.POINTER(PartArrays), P, P, P, S, P],
        "gracekv_quant_append": [ctypes.POINTER(PageConfig), ctypes.POINTER(AppendConfig), ctypes.POINTER(QuantArrays),
                                 P, P, P, P, P, P, P, P, P, P, P],
        "gracekv_quant_read": [ctypes.POINTER(PageConfig), ctypes.POINTER(ReadConfig), ctypes.POINTER(QuantArrays), P, P, P, P, P, P],
        "gracekv_quant_attention": [ctypes.POINTER(PageConfig), ctypes.POINTER(QuantArrays), P, ctypes.c_int64, P, P,
                                    ctypes.POINTER(PartArrays), P, P, P, S, P],
        "gracekv_shared_ws_bytes": [ctypes.POINTER(SharedConfig), ctypes.POINTER(S)],
        "gracekv_shared_attention": [ctypes.POINTER(SharedConfig), P, P, ctypes.POINTER(PrefixArrays), ctypes.POINTER(PartArrays), P, S, P],
    }
    for name, args in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = ctypes.c_int
    L.gracekv_status_string.argtypes = [ctypes.c_int]
    L.gracekv_status_string.restype = ctypes.c_char_p
    _lib = L
    return L


def _ok(status: int, where: str):
    if status != 0:
        raise GraceKVError(status, where)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libgracekv must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:                     # the raw handle: a Stream object costs 3 us a call
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return ctypes.c_void_p(stream.cuda_stream)


def default_config(**shape) -> Config:
    c = Config()
    _ok(lib().gracekv_default_config(ctypes.byref(c)), "default_config")
    for k, v in shape.items():
        setattr(c, k, v)
    return c


def plan_sizes(cfg: Config) -> Plan:
    p = Plan()
    _ok(lib().gracekv_plan_sizes(ctypes.byref(cfg), ctypes.byref(p)), "plan_sizes")
    return p


def check(cfg: Config, trees: torch.Tensor, stream=None):
    _ok(lib().gracekv_check(ctypes.byref(cfg), _ptr(trees), _stream(stream)), "check")


def stage_times() -> Dict[str, Tuple[float, int]]:
    """{stage: (summed ms, event pairs)} of the calls made with FLAG_STAGE_TIMES
    since the previous read (waits for their events)."""
    n = len(STAGES)
    ms = (ctypes.c_float * n)()
    cnt = (ctypes.c_int32 * n)()
    _ok(lib().gracekv_stage_times(ms, cnt), "stage_times")
    return {s: (float(ms[i]), int(cnt[i])) for i, s in enumerate(STAGES)}


def segment(cfg, hidden, surprisal, kappa, bscore, slot_starts, n_slots, ws, stream=None):
    _ok(lib().gracekv_segment(ctypes.byref(cfg), _ptr(hidden), _ptr(surprisal), _ptr(kappa), _ptr(bscore),
                              _ptr(slot_starts), _ptr(n_slots), _ptr(ws), ws.numel() * ws.element_size(),
                              _stream(stream)), "segment")


def build_trees(cfg, K, V, Q, rope_cos, rope_sin, slot_starts, n_slots, kappa, trees, stream=None, omega_raw=None,
                Q_graph=None, ws=None):
    """``Q_graph`` and ``ws`` (plan.build_ws_bytes) are read when cfg.lambda_graph > 0."""
    _ok(lib().gracekv_build_trees(ctypes.byref(cfg), _ptr(K), _ptr(V), _ptr(Q), _ptr(Q_graph), _ptr(rope_cos),
                                  _ptr(rope_sin), _ptr(slot_starts), _ptr(n_slots), _ptr(kappa), _ptr(omega_raw),
                                  _ptr(trees), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                                  _stream(stream)), "build_trees")


def relevance_stats(cfg, K, Q, trees, stream=None):
    """Relevance row statistics into the tree buffer (see GRACEKV_FLAG_STATS_READY)."""
    _ok(lib().gracekv_relevance_stats(ctypes.byref(cfg), _ptr(K), _ptr(Q), _ptr(trees), _stream(stream)),
        "relevance_stats")


def score(cfg, omega_raw, trees, stream=None):
    _ok(lib().gracekv_score(ctypes.byref(cfg), _ptr(omega_raw), _ptr(trees), _stream(stream)), "score")


def select(cfg, trees, b_used, ws, stream=None):
    _ok(lib().gracekv_select(ctypes.byref(cfg), _ptr(trees), _ptr(b_used), _ptr(ws),
                             ws.numel() * ws.element_size(), _stream(stream)), "select")


def pack(cfg, K, V, rope_cos, rope_sin, trees, offsets, counts, K_out, V_out, pos_out, logm_out, ws, stream=None):
    _ok(lib().gracekv_pack(ctypes.byref(cfg), _ptr(K), _ptr(V), _ptr(rope_cos), _ptr(rope_sin), _ptr(trees),
                           _ptr(offsets), _ptr(counts), _ptr(K_out), _ptr(V_out), _ptr(pos_out), _ptr(logm_out),
                           _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)), "pack")


def decode_ws_bytes(cfg: Config) -> int:
    n = ctypes.c_size_t(0)
    _ok(lib().gracekv_decode_ws_bytes(ctypes.byref(cfg), ctypes.byref(n)), "decode_ws_bytes")
    return int(n.value)


def decode_attention(cfg, q, offsets, K_out, V_out, logm_out, K, V, out, ws, stream=None):
    """Attention of q [L][H][d] over the packed cache plus the window rows of K, V
    (eq:app_decode_logit); out [L][H][d] fp32; ``ws``: decode_ws_bytes(cfg) bytes."""
    _ok(lib().gracekv_decode_attention(ctypes.byref(cfg), _ptr(q), _ptr(offsets), _ptr(K_out), _ptr(V_out),
                                       _ptr(logm_out), _ptr(K), _ptr(V), _ptr(out), _ptr(ws),
                                       ctypes.c_size_t(ws.numel() * ws.element_size()), _stream(stream)),
        "decode_attention")


DECODE_SCRATCH_BYTES = 64 << 20     # GRACEKV_DECODE_SCRATCH_BYTES


def decode_attention_noalloc(cfg, q, offsets, K_out, V_out, logm_out, K, V, out, stream=None):
    """decode_attention without a workspace: the partial states go to the
    library's fixed device scratch (for callers that cannot allocate); calls
    that overlap on one GPU race."""
    _ok(lib().gracekv_decode_attention_noalloc(ctypes.byref(cfg), _ptr(q), _ptr(offsets), _ptr(K_out), _ptr(V_out),
                                               _ptr(logm_out), _ptr(K), _ptr(V), _ptr(out), _stream(stream)),
        "decode_attention_noalloc")


# ---------------------------------------------------------------------------
# Around the compression, one layer at a time: prompts, pages and the next token.

_DTYPE = {torch.float32: F32, torch.bfloat16: BF16}
_TORCH = {v: k for k, v in _DTYPE.items()}


def _same(what: str, got, want):
    if got != want:
        raise ValueError(f"{what}: got {got}, need {want}")


# These checks run in front of every generated token, so a good call costs one
# comparison each and the words are found only for a bad one.

def _refuse(name: str, t: torch.Tensor, dtype, shape, dev: int, strides=None):
    raise ValueError(f"{name}: got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}, need {dtype} {tuple(shape)} "
                     f"{'contiguous' if strides is None else f'with strides {strides}'} on the current device cuda:{dev}")


def _tensor(name: str, t: torch.Tensor, dtype: torch.dtype, shape, dev: int) -> int:
    """Address of a contiguous tensor of that type and shape on device ``dev``."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _refuse(name, t, dtype, shape, dev)
    return t.data_ptr()


def _rows(name: str, t: torch.Tensor, dtype: torch.dtype, shape, dev: int):
    """Address and strides of [rows][heads][d] rows on device ``dev``: 0 for a length of one,
    whatever the tensor says."""
    tok, head, one = t.stride()
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or one != 1:
        _refuse(name, t, dtype, shape, dev, "(any, any, 1)")
    return t.data_ptr(), tok if shape[0] > 1 else 0, head if shape[1] > 1 else 0


def _strided(name: str, t: torch.Tensor, dtype: torch.dtype, shape, tok: int, head: int, dev: int) -> int:
    """Address of [rows][heads][d] rows that have these strides."""
    p, a, b = _rows(name, t, dtype, shape, dev)
    if a != tok or b != head:
        _refuse(name, t, dtype, shape, dev, (tok, head, 1))
    return p


def _heads(name: str, t: torch.Tensor):
    if t.dim() != 3 or t.stride(2) != 1:
        raise ValueError(f"{name}: need [rows][heads][d] with contiguous heads, got {tuple(t.shape)}, strides {t.stride()}")
    return t.shape


def _dtype_of(name: str, t: torch.Tensor) -> int:
    if t.dtype not in _DTYPE:
        raise ValueError(f"{name}: got {t.dtype}, need one of {list(_DTYPE)}")
    return _DTYPE[t.dtype]


def _strides(t: torch.Tensor):
    """Strides of rows and heads; 0 where there is one, whatever the tensor says."""
    (n, h, _), (tok, head, _) = t.shape, t.stride()
    return tok if n > 1 else 0, head if h > 1 else 0


def prompt_config(q, k, v, out, n_seq: int) -> PromptConfig:
    """The shapes and strides of these tensors (q, out [n_q][H][d], k, v [n_k][G][d], any
    strides of rows and heads) for prompt_attention."""
    (n_q, H, d), (n_k, G, _) = _heads("q", q), _heads("k", k)
    _same("k", k.shape[2], d)
    _same("v", tuple(_heads("v", v)), (n_k, G, d))
    _same("out", tuple(_heads("out", out)), (n_q, H, d))
    return PromptConfig(_dtype_of("q", q), G, H, d, n_seq, 0, n_q, n_k, *_strides(q), *_strides(k), *_strides(v), *_strides(out))


def prompt_ws_bytes(cfg: PromptConfig) -> int:
    n = ctypes.c_size_t(0)
    _ok(lib().gracekv_prompt_ws_bytes(ctypes.byref(cfg), ctypes.byref(n)), "prompt_ws_bytes")
    return int(n.value)


def prompt_attention(cfg: PromptConfig, q, k, v, cu_q, cu_k, out, ws=None, lse=None, stream=None):
    """Causal attention over packed prompts (gracekv_prompt_attention): ``cfg`` from
    prompt_config; cu_q, cu_k [n_seq + 1] int32; lse [n_q][H] fp32; ws: prompt_ws_bytes(cfg) bytes."""
    dev, t, n, G, H, d, n_q, n_k = torch.cuda.current_device(), _TORCH[cfg.dtype], (cfg.n_seq + 1,), cfg.G, cfg.H, cfg.d, cfg.n_q, cfg.n_k
    _ok(lib().gracekv_prompt_attention(
        ctypes.byref(cfg), _strided("q", q, t, (n_q, H, d), cfg.q_tok, cfg.q_head, dev),
        _strided("k", k, t, (n_k, G, d), cfg.k_tok, cfg.k_head, dev), _strided("v", v, t, (n_k, G, d), cfg.v_tok, cfg.v_head, dev),
        _tensor("cu_q", cu_q, torch.int32, n, dev), _tensor("cu_k", cu_k, torch.int32, n, dev),
        _strided("out", out, t, (n_q, H, d), cfg.out_tok, cfg.out_head, dev),
        None if lse is None else _tensor("lse", lse, torch.float32, (n_q, H), dev), *_workspace(ws, dev), _raw(stream, dev)),
        "prompt_attention")


def _workspace(ws, dev: int):
    if ws is None:
        return None, 0
    if not ws.is_contiguous() or ws.get_device() != dev:
        _refuse("ws", ws, ws.dtype, ws.shape, dev)
    return ws.data_ptr(), ws.nbytes


def page_config(K_pages, H: int, block_table) -> PageConfig:
    """The shapes of a paged cache: K_pages [n_pages][G][page_size][d] (pages any distance
    apart, each contiguous), block_table [n_seq][table_width] int32, H query heads."""
    if K_pages.dim() != 4 or block_table.dim() != 2:
        raise ValueError(f"need [n_pages][G][page_size][d] and [n_seq][table_width], got {tuple(K_pages.shape)}, {tuple(block_table.shape)}")
    n, G, page, d = K_pages.shape
    far = K_pages.stride(0) if n > 1 else G * page * d
    cfg = PageConfig(_dtype_of("K_pages", K_pages), G, H, d, block_table.shape[0], page, block_table.shape[1], 0, n, far)
    _page_strides("K_pages", cfg, K_pages)
    return cfg


def _page_strides(name: str, cfg: PageConfig, t: torch.Tensor):
    want = (cfg.page_stride, cfg.page_size * cfg.d, cfg.d, 1)
    if any(n > 1 and a != b for n, a, b in zip(t.shape, t.stride(), want)):
        raise ValueError(f"{name}: strides {t.stride()}, need {want}")


def _pages(cfg: PageConfig, K_pages, V_pages, dev: int):
    """Addresses of both pools of a cache."""
    t, G, page, d = _TORCH[cfg.dtype], cfg.G, cfg.page_size, cfg.d
    shape, far = (cfg.n_pages, G, page, d), (cfg.page_stride, page * d, d, 1)
    for name, x in (("K_pages", K_pages), ("V_pages", V_pages)):
        if x.dtype is not t or x.shape != shape or x.get_device() != dev:
            _refuse(name, x, t, shape, dev, far)
        if x.stride() != far:
            _page_strides(name, cfg, x)
    return K_pages.data_ptr(), V_pages.data_ptr()


def _raw(stream, dev: int) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        raise ValueError(f"stream: got one of device {stream.device_index}, need the current device cuda:{dev}")
    return stream.cuda_stream


def cache_append(cfg: PageConfig, k, v, K_pages, V_pages, block_table, start, cu_new, pos=None, rope_cos=None, rope_sin=None,
                 q=None, q_out=None, stream=None):
    """New tokens into the pages (gracekv_cache_append): k, v [n_new][G][d] and q, q_out
    [n_new][H][d] with any strides of rows and heads; start [n_seq], cu_new [n_seq + 1],
    pos [n_new] int32; rope_cos, rope_sin [rope_rows][d/2] fp32."""
    dev, t, i32 = torch.cuda.current_device(), _TORCH[cfg.dtype], torch.int32
    n, n_seq, G, d = k.shape[0], cfg.n_seq, cfg.G, cfg.d
    kp, k_tok, k_head = _rows("k", k, t, (n, G, d), dev)
    vp, v_tok, v_head = _rows("v", v, t, (n, G, d), dev)
    qp, q_tok, q_head = (None, 0, 0) if q is None else _rows("q", q, t, (n, cfg.H, d), dev)
    op, o_tok, o_head = (None, 0, 0) if q_out is None else _rows("q_out", q_out, t, (n, cfg.H, d), dev)
    r = 0 if rope_cos is None else rope_cos.shape[0]
    _ok(lib().gracekv_cache_append(
        ctypes.byref(cfg), ctypes.byref(AppendConfig(n, r, k_tok, k_head, v_tok, v_head, q_tok, q_head, o_tok, o_head)), kp, vp, qp,
        _tensor("block_table", block_table, i32, (n_seq, cfg.table_width), dev), _tensor("start", start, i32, (n_seq,), dev),
        _tensor("cu_new", cu_new, i32, (n_seq + 1,), dev), None if pos is None else _tensor("pos", pos, i32, (n,), dev),
        None if rope_cos is None else _tensor("rope_cos", rope_cos, torch.float32, (r, d // 2), dev),
        None if rope_sin is None else _tensor("rope_sin", rope_sin, torch.float32, (r, d // 2), dev),
        *_pages(cfg, K_pages, V_pages, dev), op, _raw(stream, dev)), "cache_append")


def paged_ws_bytes(cfg: PageConfig) -> int:
    n = ctypes.c_size_t(0)
    _ok(lib().gracekv_paged_ws_bytes(ctypes.byref(cfg), ctypes.byref(n)), "paged_ws_bytes")
    return int(n.value)


@dataclasses.dataclass
class Prefix:
    """Packed entries in front of the pages (gracekv_prefix): start, count [n_seq * G]
    int64; K, V [rows][d]; logm [rows] fp32.  For one sequence these are slices of pack's
    outputs: layer l takes offsets[l * G:l * G + G] and counts[l * G:l * G + G]."""
    start: torch.Tensor
    count: torch.Tensor
    K: torch.Tensor
    V: torch.Tensor
    logm: torch.Tensor


@dataclasses.dataclass(frozen=True, eq=False)
class Part:
    """An attention of the same queries over other entries (gracekv_part), as shared_attention
    writes it: o [n_seq][H][d] and lse [n_seq][H], fp32.  Looked over once, when it is made; it
    holds both tensors, which stay where they are."""
    o: torch.Tensor
    lse: torch.Tensor

    def __post_init__(self):
        f32, dev = torch.float32, self.o.get_device()
        if self.o.dim() != 3:
            raise ValueError(f"part.o: need [n_seq][H][d], got {tuple(self.o.shape)}")
        arrays = PartArrays(_tensor("part.o", self.o, f32, self.o.shape, dev), _tensor("part.lse", self.lse, f32, self.o.shape[:2], dev))
        held = object.__setattr__
        held(self, "device", dev)
        held(self, "shape", tuple(self.o.shape))
        held(self, "arrays", arrays)


def _part(part: Optional[Part], n: int, H: int, d: int, dev: int):
    if part is None:
        return None
    if part.device != dev or part.shape != (n, H, d):
        raise ValueError(f"part: got {part.shape} on device {part.device}, need {(n, H, d)} on the current device cuda:{dev}")
    return ctypes.byref(part.arrays)


def _packed(prefix: Prefix, n: int, dtype: torch.dtype, d: int, dev: int):
    """The packed entries of n rows (sequences or groups, KV heads)."""
    rows = prefix.K.shape[0]
    return ctypes.byref(PrefixArrays(
        _tensor("prefix.start", prefix.start, torch.int64, (n,), dev), _tensor("prefix.count", prefix.count, torch.int64, (n,), dev),
        _tensor("prefix.K", prefix.K, dtype, (rows, d), dev), _tensor("prefix.V", prefix.V, dtype, (rows, d), dev),
        _tensor("prefix.logm", prefix.logm, torch.float32, (rows,), dev), rows))


def _tokens(q, dtype: torch.dtype, n: int, H: int, d: int, dev: int):
    """Address of one token's query of every sequence, and the distance of two."""
    qp, far, head = _rows("q", q, dtype, (n, H, d), dev)
    if head != (d if H > 1 else 0):
        _refuse("q", q, dtype, (n, H, d), dev, (far, d, 1))
    return qp, far


def paged_attention(cfg: PageConfig, q, K_pages, V_pages, block_table, seq_len, out, ws, lse=None, prefix: Optional[Prefix] = None,
                    part: Optional[Part] = None, stream=None):
    """Attention of one token of every sequence over its pages and packed entries
    (gracekv_paged_attention): q [n_seq][H][d] (rows any distance apart), seq_len [n_seq]
    int32, out [n_seq][H][d], lse [n_seq][H] fp32, ws: paged_ws_bytes(cfg) bytes.  ``part``:
    joined to it (gracekv_paged_attention_part)."""
    dev, t, n, G, H, d = torch.cuda.current_device(), _TORCH[cfg.dtype], cfg.n_seq, cfg.G, cfg.H, cfg.d
    qp, far = _tokens(q, t, n, H, d, dev)
    px = None if prefix is None else _packed(prefix, n * G, t, d, dev)
    _ok(lib().gracekv_paged_attention_part(
        ctypes.byref(cfg), qp, far, *_pages(cfg, K_pages, V_pages, dev), _tensor("block_table", block_table, torch.int32, (n, cfg.table_width), dev),
        _tensor("seq_len", seq_len, torch.int32, (n,), dev), px, _part(part, n, H, d, dev), _tensor("out", out, t, (n, H, d), dev),
        None if lse is None else _tensor("lse", lse, torch.float32, (n, H), dev), *_workspace(ws, dev), _raw(stream, dev)),
        "paged_attention")


@dataclasses.dataclass(frozen=True, eq=False)
class QuantPages:
    """Quantised pages of one layer (gracekv_quant_pages): codes K, V uint8 [n_pages][G][page_size][d]
    (E4M3) or [..][d / 2] (E2M1), scales K_scale, V_scale uint8 [n_pages][G][page_size][d / 32]; pages
    any distance apart, the same for K and V, each contiguous.  Looked over once, when it is
    made; it holds the four tensors, which stay where they are."""
    format: int
    K: torch.Tensor
    V: torch.Tensor
    K_scale: torch.Tensor
    V_scale: torch.Tensor

    def __post_init__(self):
        if self.format not in (E4M3, E2M1):
            raise ValueError(f"format: got {self.format}, need E4M3 or E2M1")
        if self.K.dim() != 4 or self.K_scale.dim() != 4:
            raise ValueError(f"need [n_pages][G][page_size][bytes], got {tuple(self.K.shape)}, {tuple(self.K_scale.shape)}")
        each, dev, u8 = (1 if self.format == E4M3 else 2), self.K.get_device(), torch.uint8
        n, G, page, row = self.K.shape
        d = row * each
        far, scale_far = (self.K.stride(0), self.K_scale.stride(0)) if n > 1 else (G * page * row, G * page * (d // 32))
        for names, width, apart in ((("K", "V"), row, far), (("K_scale", "V_scale"), d // 32, scale_far)):
            shape, strides = (n, G, page, width), (apart, page * width, width, 1)
            for name in names:
                x = getattr(self, name)
                if x.dtype is not u8 or x.shape != shape or x.get_device() != dev:
                    _refuse(name, x, u8, shape, dev, strides)
                if any(k > 1 and a != b for k, a, b in zip(shape, x.stride(), strides)):
                    raise ValueError(f"{name}: strides {x.stride()}, need {strides}")
        held = object.__setattr__
        held(self, "device", dev)
        held(self, "shape", (n, G, page, d, far * each))
        held(self, "arrays", QuantArrays(self.format, 0, scale_far, *(x.data_ptr() for x in (self.K, self.V, self.K_scale, self.V_scale))))


def quant_config(pages: QuantPages, dtype: torch.dtype, H: int, block_table) -> PageConfig:
    """The shapes of a quantised paged cache with rows of ``dtype`` around it (torch.bfloat16 or
    torch.float32), block_table [n_seq][table_width] int32, H query heads."""
    if block_table.dim() != 2:
        raise ValueError(f"block_table: need [n_seq][table_width], got {tuple(block_table.shape)}")
    if dtype not in _DTYPE:
        raise ValueError(f"dtype: got {dtype}, need one of {list(_DTYPE)}")
    n, G, page, d, far = pages.shape
    return PageConfig(_DTYPE[dtype], G, H, d, block_table.shape[0], page, block_table.shape[1], 0, n, far)


def _quantised(cfg: PageConfig, p: QuantPages, dev: int):
    """The pools of a quantised cache of these shapes on device ``dev``."""
    if p.device != dev or p.shape != (cfg.n_pages, cfg.G, cfg.page_size, cfg.d, cfg.page_stride):
        raise ValueError(f"pages: got (n_pages, G, page_size, d, page_stride) {p.shape} on device {p.device}, need "
                         f"{(cfg.n_pages, cfg.G, cfg.page_size, cfg.d, cfg.page_stride)} on the current device cuda:{dev}")
    return ctypes.byref(p.arrays)


def quant_append(cfg: PageConfig, pages: QuantPages, k, v, block_table, start, cu_new, pos=None, rope_cos=None, rope_sin=None,
                 q=None, q_out=None, stream=None):
    """New tokens quantised into the pages (gracekv_quant_append); ``cfg`` from quant_config,
    the other arguments as cache_append's."""
    dev, t, i32 = torch.cuda.current_device(), _TORCH[cfg.dtype], torch.int32
    n, n_seq, G, d = k.shape[0], cfg.n_seq, cfg.G, cfg.d
    kp, k_tok, k_head = _rows("k", k, t, (n, G, d), dev)
    vp, v_tok, v_head = _rows("v", v, t, (n, G, d), dev)
    qp, q_tok, q_head = (None, 0, 0) if q is None else _rows("q", q, t, (n, cfg.H, d), dev)
    op, o_tok, o_head = (None, 0, 0) if q_out is None else _rows("q_out", q_out, t, (n, cfg.H, d), dev)
    r = 0 if rope_cos is None else rope_cos.shape[0]
    _ok(lib().gracekv_quant_append(
        ctypes.byref(cfg), ctypes.byref(AppendConfig(n, r, k_tok, k_head, v_tok, v_head, q_tok, q_head, o_tok, o_head)),
        _quantised(cfg, pages, dev), kp, vp, qp,
        _tensor("block_table", block_table, i32, (n_seq, cfg.table_width), dev), _tensor("start", start, i32, (n_seq,), dev),
        _tensor("cu_new", cu_new, i32, (n_seq + 1,), dev), None if pos is None else _tensor("pos", pos, i32, (n,), dev),
        None if rope_cos is None else _tensor("rope_cos", rope_cos, torch.float32, (r, d // 2), dev),
        None if rope_sin is None else _tensor("rope_sin", rope_sin, torch.float32, (r, d // 2), dev),
        op, _raw(stream, dev)), "quant_append")


def quant_read(cfg: PageConfig, pages: QuantPages, block_table, start, cu_rows, k=None, v=None, stream=None):
    """Rows back from quantised pages (gracekv_quant_read): row cu_rows[b] + i of k and v
    [n_rows][G][d] (any strides of rows and heads; either may be None) becomes what place
    start[b] + i of sequence b stands for."""
    dev, t, n_seq, G, d = torch.cuda.current_device(), _TORCH[cfg.dtype], cfg.n_seq, cfg.G, cfg.d
    n = k.shape[0] if k is not None else (v.shape[0] if v is not None else 0)
    kp, k_tok, k_head = (None, 0, 0) if k is None else _rows("k", k, t, (n, G, d), dev)
    vp, v_tok, v_head = (None, 0, 0) if v is None else _rows("v", v, t, (n, G, d), dev)
    _ok(lib().gracekv_quant_read(
        ctypes.byref(cfg), ctypes.byref(ReadConfig(n, k_tok, k_head, v_tok, v_head)), _quantised(cfg, pages, dev),
        _tensor("block_table", block_table, torch.int32, (n_seq, cfg.table_width), dev),
        _tensor("start", start, torch.int32, (n_seq,), dev), _tensor("cu_rows", cu_rows, torch.int32, (n_seq + 1,), dev),
        kp, vp, _raw(stream, dev)), "quant_read")


def quant_attention(cfg: PageConfig, pages: QuantPages, q, block_table, seq_len, out, ws, lse=None, part: Optional[Part] = None,
                    stream=None):
    """Attention of one token of every sequence over its quantised pages, joined to ``part``
    (gracekv_quant_attention); ``cfg`` from quant_config, the other arguments as paged_attention's."""
    dev, t, n, H, d = torch.cuda.current_device(), _TORCH[cfg.dtype], cfg.n_seq, cfg.H, cfg.d
    qp, far = _tokens(q, t, n, H, d, dev)
    _ok(lib().gracekv_quant_attention(
        ctypes.byref(cfg), _quantised(cfg, pages, dev), qp, far, _tensor("block_table", block_table, torch.int32, (n, cfg.table_width), dev),
        _tensor("seq_len", seq_len, torch.int32, (n,), dev), _part(part, n, H, d, dev), _tensor("out", out, t, (n, H, d), dev),
        None if lse is None else _tensor("lse", lse, torch.float32, (n, H), dev), *_workspace(ws, dev), _raw(stream, dev)),
        "quant_attention")


def shared_config(q, G: int, n_group: int) -> SharedConfig:
    """The shapes of n_group groups of the sequences whose queries these are (q [n_seq][H][d], rows
    any distance apart), with G KV heads, for shared_attention."""
    n, H, d = _heads("q", q)
    return SharedConfig(_dtype_of("q", q), G, H, d, n, n_group, q.stride(0) if n > 1 else 0)


def shared_ws_bytes(cfg: SharedConfig) -> int:
    n = ctypes.c_size_t(0)
    _ok(lib().gracekv_shared_ws_bytes(ctypes.byref(cfg), ctypes.byref(n)), "shared_ws_bytes")
    return int(n.value)


def shared_attention(cfg: SharedConfig, q, cu_group, prefix: Prefix, part: Part, ws, stream=None):
    """Attention of one token of every sequence over packed entries that its group shares
    (gracekv_shared_attention), written to ``part``: cu_group [n_group + 1] int32, prefix.start and
    .count [n_group * G], ws: shared_ws_bytes(cfg) bytes.  Of arrays of several layers pass one layer's
    rows (K[a:b], V[a:b], logm[a:b], start - a): the kernel is chosen by how many there are."""
    dev, t, n, H, d = torch.cuda.current_device(), _TORCH[cfg.dtype], cfg.n_seq, cfg.H, cfg.d
    qp, far = _tokens(q, t, n, H, d, dev)
    if far != cfg.q_tok:
        _refuse("q", q, t, (n, H, d), dev, (cfg.q_tok, d, 1))
    _ok(lib().gracekv_shared_attention(
        ctypes.byref(cfg), qp, _tensor("cu_group", cu_group, torch.int32, (cfg.n_group + 1,), dev),
        _packed(prefix, cfg.n_group * cfg.G, t, d, dev), _part(part, n, H, d, dev), *_workspace(ws, dev), _raw(stream, dev)),
        "shared_attention")


def selftest_mfma(which: int, stream=None) -> torch.Tensor:
    out = torch.zeros(256, dtype=torch.float32, device="cuda")
    _ok(lib().gracekv_selftest_mfma(which, _ptr(out), _stream(stream)), "selftest_mfma")
    return out.view(16, 16).cpu()


# ---------------------------------------------------------------------------
def tree_arrays(plan: Plan, trees: torch.Tensor) -> Dict[str, torch.Tensor]:
    """Typed views of the tree buffer (layout from plan_sizes)."""
    NC, UC = plan.node_cap, plan.unit_cap

    def v(off, n, dt):
        nbytes = n * torch.tensor([], dtype=dt).element_size()
        return trees[off:off + nbytes].view(dt)
    return dict(
        node_a=v(plan.off_node_a, NC, torch.int32), node_n=v(plan.off_node_n, NC, torch.int32),
        node_child=v(plan.off_node_child, NC, torch.int32), node_parent=v(plan.off_node_parent, NC, torch.int32),
        node_nch=v(plan.off_node_nch, NC, torch.uint8), node_kind=v(plan.off_node_kind, NC, torch.uint8),
        node_cut=v(plan.off_node_cut, NC, torch.int32), node_D=v(plan.off_node_D, NC, torch.float32),
        node_R=v(plan.off_node_R, NC, torch.float32), sp_U=v(plan.off_sp_U, NC, torch.float32),
        sp_E=v(plan.off_sp_E, NC, torch.int64), sp_cost=v(plan.off_sp_cost, NC, torch.uint8),
        sp_exec=v(plan.off_sp_exec, NC, torch.uint8), unit_nn=v(plan.off_unit_nn, UC, torch.int32),
        unit_Ddrop=v(plan.off_unit_Ddrop, UC, torch.float32), add_U=v(plan.off_add_U, UC, torch.float32),
        add_E=v(plan.off_add_E, UC, torch.int64), add_exec=v(plan.off_add_exec, UC, torch.uint8),
        status=v(plan.off_status, 2, torch.int32), nslots=v(plan.off_nslots, 1, torch.int32),
        slots=v(plan.off_slots, plan.J_cap + 1, torch.int32),
    )


def floor_arrays(plan: Plan, trees: torch.Tensor) -> Dict[str, torch.Tensor]:
    """Typed views of the singleton floor's region (alpha_floor > 0): state (B_floor,
    cap, total cost of the initial lists, lists reduced, ...), initial and kept list
    lengths, the lists, the candidate flags and the ops the floor executed."""
    LG = plan.unit_cap // plan.J_cap
    N = plan.N_c
    al = lambda x: (x + 255) & ~255
    o = plan.off_floor
    out = {}
    for name, n, dt in (("state", 8, torch.int64), ("cnt", LG, torch.int32), ("keep", LG, torch.int32),
                        ("list", LG * N, torch.int32), ("flag", LG * N, torch.uint8),
                        ("pre_add", plan.unit_cap, torch.uint8), ("pre_sp", plan.node_cap, torch.uint8)):
        nbytes = n * torch.tensor([], dtype=dt).element_size()
        out[name] = trees[o:o + nbytes].view(dt)
        o += al(nbytes)
    return out


@dataclasses.dataclass
class Buffers:
    cfg: Config
    plan: Plan
    kappa: torch.Tensor
    bscore: torch.Tensor
    slot_starts: torch.Tensor
    n_slots: torch.Tensor
    seg_ws: torch.Tensor
    trees: torch.Tensor
    sel_ws: torch.Tensor
    pack_ws: torch.Tensor
    b_used: torch.Tensor
    offsets: torch.Tensor
    counts: torch.Tensor
    K_out: torch.Tensor
    V_out: torch.Tensor
    pos_out: torch.Tensor
    logm_out: torch.Tensor
    build_ws: Optional[torch.Tensor] = None   # multi-hop scratch (lambda_graph > 0)


def config_for(L, G, H, d, W, N_ctx, x, dtype, n_seg, D_hidden, **hyper) -> Config:
    return default_config(L=L, G=G, H=H, d=d, W=W, N_ctx=N_ctx, x=float(x), dtype=dtype, n_seg=n_seg,
                          D_hidden=D_hidden, **hyper)


def allocate(cfg: Config, device="cuda") -> Buffers:
    """Device buffers of one compression (sizes from plan_sizes)."""
    p = plan_sizes(cfg)
    kvdt = torch.bfloat16 if cfg.dtype == BF16 else torch.float32
    u8 = dict(dtype=torch.uint8, device=device)
    trees = torch.empty(max(p.tree_bytes, 16), **u8)
    trees[p.off_status:p.off_status + 16].zero_()     # no build yet: check() reports it
    return Buffers(
        cfg=cfg, plan=p,
        kappa=torch.empty(p.T, dtype=torch.float32, device=device),
        bscore=torch.empty(p.T, dtype=torch.float32, device=device),
        slot_starts=torch.zeros(p.J_cap + 1, dtype=torch.int32, device=device),
        n_slots=torch.zeros(1, dtype=torch.int32, device=device),
        seg_ws=torch.empty(max(p.seg_ws_bytes, 16), **u8),
        trees=trees,
        sel_ws=torch.empty(max(p.sel_ws_bytes, 16), **u8),
        pack_ws=torch.empty(max(p.pack_ws_bytes, 16), **u8),
        b_used=torch.zeros(1, dtype=torch.int64, device=device),
        offsets=torch.zeros(cfg.L * cfg.G + 1, dtype=torch.int64, device=device),
        counts=torch.zeros(cfg.L * cfg.G, dtype=torch.int64, device=device),
        K_out=torch.empty(max(p.B_total, 1), cfg.d, dtype=kvdt, device=device),
        V_out=torch.empty(max(p.B_total, 1), cfg.d, dtype=kvdt, device=device),
        pos_out=torch.empty(max(p.B_total, 1), dtype=torch.int32, device=device),
        logm_out=torch.empty(max(p.B_total, 1), dtype=torch.float32, device=device),
        build_ws=torch.empty(p.build_ws_bytes, **u8) if p.build_ws_bytes else None,
    )


def compress(buf: Buffers, K, V, Q, rope_cos, rope_sin, hidden, surprisal, omega_raw, stream=None,
             kappa: Optional[torch.Tensor] = None, slot_starts: Optional[torch.Tensor] = None,
             n_slots: Optional[torch.Tensor] = None, Q_graph: Optional[torch.Tensor] = None):
    """The five calls in order.  ``kappa``/``slot_starts``/``n_slots`` may be
    given to skip segmentation (then ``hidden`` may be None); ``Q_graph`` is
    read when cfg.lambda_graph > 0."""
    cfg = buf.cfg
    if slot_starts is None:
        segment(cfg, hidden, surprisal, buf.kappa, buf.bscore, buf.slot_starts, buf.n_slots, buf.seg_ws, stream)
        kappa, slot_starts, n_slots = buf.kappa, buf.slot_starts, buf.n_slots
    build_trees(cfg, K, V, Q, rope_cos, rope_sin, slot_starts, n_slots, kappa, buf.trees, stream, omega_raw=omega_raw,
                Q_graph=Q_graph, ws=buf.build_ws)
    score(cfg, omega_raw, buf.trees, stream)
    select(cfg, buf.trees, buf.b_used, buf.sel_ws, stream)
    pack(cfg, K, V, rope_cos, rope_sin, buf.trees, buf.offsets, buf.counts, buf.K_out, buf.V_out, buf.pos_out,
         buf.logm_out, buf.pack_ws, stream)
