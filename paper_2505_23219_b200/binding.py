"""ctypes binding of ``libghd.so``: same names as the C-ABI, torch tensors in.

Only argument marshalling happens here.  Device buffers are torch tensors (the
library borrows them), the stream is torch's current stream at context creation.
"""
from __future__ import annotations

import ctypes as C
from pathlib import Path

import numpy as np
import torch
from torch._C import _cuda_getCurrentRawStream as _raw_stream

from . import build as _build

__all__ = [
    "GhdError", "ModelCfg", "LayerWeights", "ModelWeights", "KvLayer", "Tree", "Ctx", "load_library",
    "ghd_create", "ghd_destroy", "ghd_set_option", "ghd_tree_build", "ghd_tree_from_mask", "ghd_verify_layer",
    "ghd_verify_step", "ghd_accept", "ghd_linear", "ghd_rmsnorm", "ghd_tree_attention", "ghd_argmax",
    "ghd_sync_status", "ghd_launch_count", "pack_mask", "ghd_copy_hidden", "ghd_gate_up", "ghd_tree_attention_static", "ghd_path_count", "ghd_kv_commit", "ghd_medusa_draft", "ghd_tree_fill_tokens",
    "Kv4Cache", "Kv4Rows", "ghd_kv4_pool_bytes", "ghd_kv4_pool", "ghd_kv4_append", "ghd_kv4_attention", "ghd_kv4_read", "ghd_kv4_commit", "GHD_MAX_SEQS",
    "Mx4", "ghd_mx4", "ghd_mx4_quantize", "ghd_mx4_read", "ghd_mx4_linear", "ghd_mx4_gate_up", "ghd_mx4_code_bytes", "ghd_mx4_scale_bytes",
    "SampledRows", "ghd_draft_sample", "ghd_accept_sampled",
    "ghd_kv_len_set", "ghd_kv_len_get", "KV_LEN_DEVICE", "MedusaWeights", "GHD_MAX_TOPK",
    "PATH_GEMM_TILE", "PATH_GEMM_SIMT", "PATH_ATTN_TC", "PATH_ATTN_SIMT", "PATH_ATTN_COO", "PATH_GEMM_PAIR", "PATH_KV4_ROWS", "PATH_KV4_TC", "OPT_GEMM_PAIR", "OPT_ATTN_ROWS", "OPT_GEMM_SKEW", "OPT_ATTN_SMALL",
    "GHD_F32", "GHD_F16", "GHD_MAX_NODES", "OPT_GEMM_PATH", "OPT_ATTN_SPLITS", "OPT_ATTN_PATH", "OPT_GRAPH",
    "OPT_GEMM_CTAS", "OPT_GEMM_BURST", "OPT_NO_PDL", "OPT_GEMM_STAGES", "OPT_GEMM_EPI", "OPT_ATTN_SPARSE", "OPT_CHAIN_CALLS", "OPT_FUSED_NORM", "EXPORTS",
]

GHD_F32, GHD_F16 = 0, 1
GHD_MAX_NODES = 256
GHD_MAX_TOPK = 16
GHD_MAX_SEQS = 1024
KV_LEN_DEVICE = -1      # "take the cache length from the context's device word"
OPT_GEMM_PATH, OPT_ATTN_SPLITS, OPT_ATTN_PATH, OPT_GRAPH, OPT_GEMM_CTAS, OPT_GEMM_BURST, OPT_NO_PDL = 0, 1, 2, 3, 4, 5, 6
OPT_GEMM_STAGES, OPT_GEMM_EPI, OPT_ATTN_SPARSE, OPT_CHAIN_CALLS, OPT_FUSED_NORM = 7, 8, 9, 10, 11
PATH_GEMM_TILE, PATH_GEMM_SIMT, PATH_ATTN_TC, PATH_ATTN_SIMT, PATH_ATTN_COO, PATH_GEMM_PAIR = 0, 1, 2, 3, 4, 5
PATH_KV4_ROWS, PATH_KV4_TC = 6, 7
OPT_GEMM_PAIR, OPT_ATTN_ROWS, OPT_GEMM_SKEW, OPT_ATTN_SMALL = 12, 13, 14, 15
_STATUS = ["GHD_OK", "GHD_EINVAL", "GHD_ESHAPE", "GHD_ETREE", "GHD_ENOSPACE", "GHD_ECUDA", "GHD_ETIMEOUT",
           "GHD_EUNSUPPORTED"]

# every symbol include/ghd.h declares
EXPORTS = [
    "ghd_create", "ghd_destroy", "ghd_workspace_bytes", "ghd_set_workspace", "ghd_set_option", "ghd_tree_build",
    "ghd_tree_from_mask", "ghd_verify_layer", "ghd_verify_step", "ghd_accept", "ghd_linear", "ghd_rmsnorm",
    "ghd_tree_attention", "ghd_argmax", "ghd_sync_status", "ghd_status_str", "ghd_last_error", "ghd_launch_count",
    "ghd_tree_attention_static", "ghd_path_count", "ghd_kv_commit", "ghd_kv_len_set", "ghd_kv_len_get",
    "ghd_medusa_draft", "ghd_tree_fill_tokens", "ghd_copy_hidden", "ghd_gate_up",
    "ghd_kv4_pool_bytes", "ghd_kv4_append", "ghd_kv4_attention", "ghd_kv4_read", "ghd_kv4_commit",
    "ghd_mx4_code_bytes", "ghd_mx4_scale_bytes", "ghd_mx4_quantize", "ghd_mx4_read", "ghd_mx4_linear", "ghd_mx4_gate_up",
    "ghd_draft_sample", "ghd_accept_sampled",
]


class GhdError(RuntimeError):
    def __init__(self, status: int, detail: str = ""):
        self.status = status
        self.name = _STATUS[status] if 0 <= status < len(_STATUS) else str(status)
        super().__init__(f"{self.name}: {detail}" if detail else self.name)


class _Cfg(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("d_model", "n_heads", "n_kv_heads", "d_head", "d_ffn", "vocab", "n_layers",
                                          "max_kv_len", "max_nodes", "dtype")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float)]


class _LayerW(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("wqkv", "wo", "w_gate_up", "w_down", "rms1", "rms2")]


class _ModelW(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("layers", C.POINTER(_LayerW)), ("rms_final", C.c_void_p),
                ("lm_head", C.c_void_p)]


class _MedusaW(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("w1", C.c_void_p), ("w2", C.c_void_p)]


class _Kv(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("len", C.c_int32)]


class _Tree(C.Structure):
    _fields_ = [("n", C.c_int32), ("kv_len", C.c_int32), ("n_words", C.c_int32), ("has_parent", C.c_int32),
                ("mask", C.c_void_p), ("parent", C.c_void_p), ("depth", C.c_void_p), ("pos", C.c_void_p),
                ("rope", C.c_void_p), ("coo_ptr", C.c_void_p), ("coo_col", C.c_void_p), ("nnz", C.c_int32)]


class _Kv4(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("n_seqs", "n_pages", "page_rows", "max_pages", "n_kv_heads")] + \
               [("page_table", C.c_void_p), ("kv_len", C.c_void_p)]


class _Kv4Rows(C.Structure):
    _fields_ = [("n_rows", C.c_int32), ("mask_words", C.c_int32), ("row_start", C.c_void_p), ("pos", C.c_void_p), ("mask", C.c_void_p)]


class _Mx4(C.Structure):
    _fields_ = [("m", C.c_int32), ("k", C.c_int32), ("codes", C.c_void_p), ("scales", C.c_void_p)]


class _Sampled(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("n_rows", C.c_int32)] + \
               [(k, C.c_void_p) for k in ("row_start", "parent", "tokens", "logits", "uniforms", "draft_row", "draft_logits")] + \
               [("n_draft", C.c_int32), ("temperature", C.c_float), ("draft_temperature", C.c_float)]


_LIB = None


def load_library(path: str | Path | None = None):
    """Loads libghd.so (built by ``build.build()``); raises if it is not there."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    p = Path(path) if path else _build.LIB
    if not p.exists():
        raise RuntimeError(f"{p} is missing: build the CUDA library first "
                           "(python -m paper_2505_23219_b200.build); there is no fallback path")
    lib = C.CDLL(str(p))
    vp, i32 = C.c_void_p, C.c_int32
    sig = {
        "ghd_create": ([C.POINTER(_Cfg), vp, C.POINTER(vp)], C.c_int),
        "ghd_destroy": ([vp], None),
        "ghd_workspace_bytes": ([vp], C.c_size_t),
        "ghd_set_workspace": ([vp, vp, C.c_size_t], C.c_int),
        "ghd_set_option": ([vp, i32, i32], C.c_int),
        "ghd_path_count": ([vp, i32], C.c_int64),
        "ghd_tree_build": ([vp, vp, i32, i32, C.POINTER(_Tree)], C.c_int),
        "ghd_tree_from_mask": ([vp, vp, vp, vp, i32, i32, C.POINTER(_Tree)], C.c_int),
        "ghd_verify_layer": ([vp, C.POINTER(_LayerW), C.POINTER(_Kv), C.POINTER(_Tree), vp, vp], C.c_int),
        "ghd_verify_step": ([vp, C.POINTER(_ModelW), C.POINTER(_Kv), C.POINTER(_Tree), vp, vp, vp], C.c_int),
        "ghd_accept": ([vp, C.POINTER(_Tree), vp, vp, vp], C.c_int),
        "ghd_copy_hidden": ([vp, i32, vp], C.c_int),
        "ghd_kv_commit": ([vp, C.POINTER(_Kv), i32, i32, vp], C.c_int),
        "ghd_kv_len_set": ([vp, i32], C.c_int),
        "ghd_kv_len_get": ([vp, C.POINTER(i32)], C.c_int),
        "ghd_medusa_draft": ([vp, C.POINTER(_MedusaW), vp, vp, vp, vp], C.c_int),
        "ghd_tree_fill_tokens": ([vp, vp, vp, vp, vp, i32, vp], C.c_int),
        "ghd_linear": ([vp, vp, vp, i32, i32, i32, vp], C.c_int),
        "ghd_rmsnorm": ([vp, vp, vp, i32, vp], C.c_int),
        "ghd_gate_up": ([vp, vp, vp, i32, vp], C.c_int),
        "ghd_tree_attention": ([vp, vp, C.POINTER(_Kv), C.POINTER(_Tree), vp], C.c_int),
        "ghd_argmax": ([vp, vp, i32, i32, vp], C.c_int),
        "ghd_kv4_pool_bytes": ([vp, C.POINTER(_Kv4)], C.c_size_t),
        "ghd_kv4_append": ([vp, C.POINTER(_Kv4), C.POINTER(_Kv4Rows), vp, vp, C.c_int64, vp, vp, C.c_int64, vp], C.c_int),
        "ghd_kv4_attention": ([vp, C.POINTER(_Kv4), C.POINTER(_Kv4Rows), vp, vp, vp], C.c_int),
        "ghd_kv4_read": ([vp, C.POINTER(_Kv4), C.POINTER(_Kv4Rows), vp, vp, vp, vp], C.c_int),
        "ghd_kv4_commit": ([vp, C.POINTER(_Kv4), C.POINTER(_Kv4Rows), vp, i32, vp], C.c_int),
        "ghd_mx4_code_bytes": ([i32, i32], C.c_size_t),
        "ghd_mx4_scale_bytes": ([i32, i32], C.c_size_t),
        "ghd_mx4_quantize": ([vp, vp, C.c_int64, C.POINTER(_Mx4)], C.c_int),
        "ghd_mx4_read": ([vp, C.POINTER(_Mx4), vp, C.c_int64], C.c_int),
        "ghd_mx4_linear": ([vp, vp, C.c_int64, C.POINTER(_Mx4), i32, vp], C.c_int),
        "ghd_mx4_gate_up": ([vp, vp, C.c_int64, C.POINTER(_Mx4), C.POINTER(_Mx4), i32, vp], C.c_int),
        "ghd_draft_sample": ([vp, vp, i32, C.c_float, i32, vp, vp], C.c_int),
        "ghd_accept_sampled": ([vp, C.POINTER(_Sampled), vp], C.c_int),
        "ghd_sync_status": ([vp], C.c_int),
        "ghd_status_str": ([C.c_int], C.c_char_p),
        "ghd_last_error": ([vp], C.c_char_p),
        "ghd_launch_count": ([vp], C.c_int64),
        "ghd_tree_attention_static": ([vp, i32, i32, i32, i32, vp, vp, vp, vp, i32, i32, vp, C.c_char_p, C.c_size_t],
                                      C.c_int),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, res
    if path is None:
        _LIB = lib
    return lib


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


class ModelCfg:
    def __init__(self, d_model, n_heads, d_head, d_ffn, vocab, n_layers, max_kv_len, max_nodes, dtype,
                 rms_eps=1e-6, rope_theta=10000.0, n_kv_heads=None):
        self.c = _Cfg(d_model, n_heads, n_heads if n_kv_heads is None else n_kv_heads, d_head, d_ffn, vocab,
                      n_layers, max_kv_len, max_nodes, GHD_F32 if dtype in ("f32", GHD_F32) else GHD_F16,
                      rms_eps, rope_theta)

    @property
    def torch_dtype(self):
        return torch.float32 if self.c.dtype == GHD_F32 else torch.float16


class LayerWeights:
    """Device tensors of one layer (kept alive here)."""
    FIELDS = ("wqkv", "wo", "w_gate_up", "w_down", "rms1", "rms2")

    def __init__(self, **tensors):
        self.t = {k: tensors[k] for k in self.FIELDS}
        self.c = _LayerW(*[_ptr(self.t[k]) for k in self.FIELDS])


class ModelWeights:
    def __init__(self, embed, layers, rms_final, lm_head):
        self.embed, self.layers, self.rms_final, self.lm_head = embed, list(layers), rms_final, lm_head
        self._arr = (_LayerW * max(len(self.layers), 1))(*[l.c for l in self.layers])
        self.c = _ModelW(_ptr(embed), self._arr, _ptr(rms_final), _ptr(lm_head))


class MedusaWeights:
    """Drafting heads: w1 [n_heads][d_model][d_model], w2 [n_heads][vocab][d_model] (device tensors)."""

    def __init__(self, w1, w2):
        self.w1, self.w2 = w1, w2
        self.c = _MedusaW(int(w1.shape[0]), _ptr(w1), _ptr(w2))


class KvLayer:
    def __init__(self, k, v, length: int):
        self.k, self.v, self.len = k, v, int(length)

    @property
    def c(self):
        return _Kv(_ptr(self.k), _ptr(self.v), self.len)


def _need(t, dtype, what: str, numel: int, dev: int | None = None):
    """A contiguous device tensor of `dtype` with at least `numel` elements (its pointer), on device `dev` if that is given;
    raises otherwise."""
    if (not t.is_cuda if dev is None else t.get_device() != dev) or t.dtype is not dtype or t.numel() < numel or not t.is_contiguous():
        raise GhdError(1, f"{what}: want a contiguous {dtype} device tensor of at least {numel} elements"
                          f"{'' if dev is None else f' on cuda:{dev}'}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


_INT = 0x80000000      # numbers outside [-_INT, _INT) are refused: ctypes would cut them off, and sizes be checked against others


class _Description:
    """Holds tensors beside the struct with their pointers, and does not change: an attribute that was set to another tensor would
    free the one that the struct still points to.  (The constructors write to __dict__.)"""

    def __setattr__(self, name, value):
        raise AttributeError(f"{type(self).__name__}.{name} is fixed: write into its tensors, or make another {type(self).__name__}")

    def __delattr__(self, name):
        raise AttributeError(f"{type(self).__name__}.{name} is fixed")


class Kv4Cache(_Description):
    """Paging of a 4-bit cache: page_table int32 [n_seqs][max_pages], kv_len int32 [n_seqs] (device tensors; the pools of
    the layers come with each call).  The kernels run on the context's stream, whichever is the current one: tensors have to be
    ready there, and to stay alive until the kernels have run.  Their contents may change, the description may not."""

    def __init__(self, page_table, kv_len, page_rows: int, n_kv_heads: int, n_pages: int):
        if page_table.dim() != 2:
            raise GhdError(1, "kv4: page_table is not [n_seqs][max_pages]")
        n_seqs, max_pages = page_table.shape
        if not (-_INT <= page_rows < _INT and -_INT <= n_kv_heads < _INT and -_INT <= n_pages < _INT):
            raise GhdError(1, f"kv4: page_rows {page_rows}, n_kv_heads {n_kv_heads} or n_pages {n_pages} is outside 32 bits")
        table, dev = _need(page_table, torch.int32, "page_table", 0), page_table.get_device()
        c = _Kv4(n_seqs, n_pages, page_rows, max_pages, n_kv_heads, table, _need(kv_len, torch.int32, "kv_len", n_seqs, dev))
        own = self.__dict__
        own["page_table"], own["kv_len"], own["dev"], own["n_seqs"], own["n_kv_heads"] = page_table, kv_len, dev, n_seqs, n_kv_heads
        own["n_rows"], own["c"], own["ref"] = n_pages * n_kv_heads * page_rows, c, C.byref(c)


class Kv4Rows(_Description):
    """The new rows of a call: row_start int32 [n_seqs + 1]; optional pos int32 [n_rows]; optional mask int64
    [n_rows][words], bit j of row i = the sequence's new row j is visible to it (device tensors)."""

    def __init__(self, row_start, n_rows: int, pos=None, mask=None):
        n_rows = int(n_rows)
        if not -_INT <= n_rows < _INT:
            raise GhdError(1, f"kv4: n_rows {n_rows} is outside 32 bits")
        start, dev = _need(row_start, torch.int32, "row_start", 2), row_start.get_device()
        words = 0 if mask is None else int(mask.shape[-1])
        c = _Kv4Rows(n_rows, words, start, None if pos is None else _need(pos, torch.int32, "pos", n_rows, dev),
                     None if mask is None else _need(mask, torch.int64, "mask", n_rows * words, dev))
        own = self.__dict__
        own["row_start"], own["n_rows"], own["pos"], own["mask"] = row_start, n_rows, pos, mask
        own["n_starts"], own["dev"], own["c"], own["ref"] = row_start.numel(), dev, c, C.byref(c)


class Mx4(_Description):
    """A matrix [m][k] in microscaled 4-bit floating point: uint8 device tensors with its codes and scales (any shape with the bytes that
    ghd_mx4_code_bytes and ghd_mx4_scale_bytes give; ghd_mx4 makes them)."""

    def __init__(self, codes, scales, m: int, k: int):
        if not (0 < m < _INT and 0 < k < _INT):
            raise GhdError(1, f"mx4: m {m} or k {k} is outside [1, 2^31)")
        lib = load_library()
        nc, ns = lib.ghd_mx4_code_bytes(m, k), lib.ghd_mx4_scale_bytes(m, k)
        if not nc:
            raise GhdError(2, f"mx4: a matrix of {m} x {k}")
        c = _Mx4(m, k, _need(codes, torch.uint8, "codes", nc), _need(scales, torch.uint8, "scales", ns, codes.get_device()))
        own = self.__dict__
        own["codes"], own["scales"], own["m"], own["k"], own["dev"], own["c"], own["ref"] = codes, scales, m, k, codes.get_device(), c, C.byref(c)


class SampledRows(_Description):
    """The drafted trees of n_seqs sequences with their target logits: parent, tokens int32 [n_rows], logits float [n_rows][vocab], uniforms
    float [n_rows]; row_start int32 [n_seqs + 1] (None: one sequence); where candidates were drawn, draft_row int32 [n_rows] and
    draft_logits float [n_draft][vocab] (device tensors, whose contents may change)."""

    def __init__(self, parent, tokens, logits, uniforms, row_start=None, temperature: float = 1.0, draft_row=None, draft_logits=None,
                 draft_temperature: float = 1.0):
        if parent.dim() != 1 or logits.dim() != 2 or logits.shape[0] < parent.shape[0]:
            raise GhdError(1, "sampled: parent is not [n_rows], or logits not [n_rows][vocab]")
        n, (_, vocab) = parent.shape[0], logits.shape
        at = _need(parent, torch.int32, "parent", 0)
        dev = parent.get_device()
        if (draft_row is None) != (draft_logits is None):
            raise GhdError(1, "sampled: give both draft_row and draft_logits or neither")
        n_draft = 0
        if draft_row is not None:
            if draft_logits.dim() != 2 or draft_logits.shape[1] != vocab:
                raise GhdError(1, "sampled: draft_logits is not [n_draft][vocab]")
            n_draft = draft_logits.shape[0]
        n_seqs = 1 if row_start is None else row_start.numel() - 1
        if not (n < _INT and n_seqs < _INT and n_draft < _INT):
            raise GhdError(1, "sampled: more than 2^31 rows")
        c = _Sampled(n_seqs, n, None if row_start is None else _need(row_start, torch.int32, "row_start", 2, dev), at,
                     _need(tokens, torch.int32, "tokens", n, dev), _need(logits, torch.float32, "logits", n * vocab, dev),
                     _need(uniforms, torch.float32, "uniforms", n, dev),
                     None if draft_row is None else _need(draft_row, torch.int32, "draft_row", n, dev),
                     None if draft_row is None else _need(draft_logits, torch.float32, "draft_logits", n_draft * vocab, dev),
                     n_draft, temperature, draft_temperature)
        own = self.__dict__
        own["tensors"] = (parent, tokens, logits, uniforms, row_start, draft_row, draft_logits)
        own["n_seqs"], own["vocab"], own["dev"], own["c"], own["ref"] = n_seqs, vocab, dev, c, C.byref(c)


class Tree:
    """Device buffers of a built tree plus the struct that describes them."""

    def __init__(self, ctx: "Ctx"):
        n, dev = ctx.cfg.c.max_nodes, ctx.device
        self.mask = torch.zeros(n * 4, dtype=torch.int64, device=dev)
        self.parent = torch.zeros(n, dtype=torch.int32, device=dev)
        self.depth = torch.zeros(n, dtype=torch.int32, device=dev)
        self.pos = torch.zeros(n, dtype=torch.int32, device=dev)
        self.rope = torch.zeros(n * ctx.cfg.c.d_head, dtype=torch.float32, device=dev)
        self.coo_ptr = torch.zeros(n + 1, dtype=torch.int32, device=dev)
        self.coo_col = torch.zeros(n * (n + 1) // 2, dtype=torch.int32, device=dev)
        self.c = _Tree(0, 0, 0, 0, _ptr(self.mask), _ptr(self.parent), _ptr(self.depth), _ptr(self.pos),
                       _ptr(self.rope), _ptr(self.coo_ptr), _ptr(self.coo_col), 0)

    @property
    def n(self):
        return self.c.n

    def coo(self):
        """-> (row pointers int32 [n + 1], visible node ids int32 [nnz]) on the host."""
        n = self.c.n
        ptr = self.coo_ptr[: n + 1].cpu().numpy()
        return ptr, self.coo_col[: int(ptr[n])].cpu().numpy()

    def mask_words(self) -> np.ndarray:
        """mask as uint64 [n][n_words] on the host."""
        n, w = self.c.n, self.c.n_words
        return self.mask[: n * w].cpu().numpy().view(np.uint64).reshape(n, w)


class Ctx:
    def __init__(self, cfg: ModelCfg, device="cuda:0"):
        self.lib = load_library()
        self.cfg = cfg
        self.dtype, self.d_head, self.n_heads = cfg.torch_dtype, cfg.c.d_head, cfg.c.n_heads
        self.kv4_row = self.d_head + 4 * self.dtype.itemsize      # bytes of a row of one head in the 4-bit cache
        self.device = torch.device(device)
        self.handle = C.c_void_p()
        with torch.cuda.device(self.device):
            self.dev = torch.cuda.current_device()
            self.stream = torch.cuda.current_stream(self.device)
            self.raw_stream = self.stream.cuda_stream
            st = self.lib.ghd_create(C.byref(cfg.c), C.c_void_p(self.stream.cuda_stream), C.byref(self.handle))
            if st != 0:
                raise GhdError(st, "ghd_create")
            nbytes = self.lib.ghd_workspace_bytes(self.handle)
            self.blank = torch.empty(0, dtype=self.dtype, device=self.device)      # outputs are made like it
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            self._check(self.lib.ghd_set_workspace(self.handle, self.workspace.data_ptr(), nbytes))

    def _check(self, st: int):
        if st != 0:
            raise GhdError(st, self.lib.ghd_last_error(self.handle).decode())

    def close(self):
        if self.handle:
            self.lib.ghd_destroy(self.handle)
            self.handle = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def pack_mask(visible) -> np.ndarray:
    """bool [n][n] visibility matrix -> uint64 [n][ceil(n/64)] words, bit j of row i LSB first."""
    vis = np.asarray(visible, dtype=bool)
    n = vis.shape[0]
    w = (n + 63) // 64
    out = np.zeros((n, w), dtype=np.uint64)
    for i in range(n):
        for j in np.nonzero(vis[i])[0]:
            out[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return out


# ---------------------------------------------------------------- same names as the C-ABI
def ghd_create(cfg: ModelCfg, device="cuda:0") -> Ctx:
    return Ctx(cfg, device)


def ghd_destroy(ctx: Ctx):
    ctx.close()


def ghd_set_option(ctx: Ctx, option: int, value: int):
    ctx._check(ctx.lib.ghd_set_option(ctx.handle, option, value))


def ghd_path_count(ctx: Ctx, path: int) -> int:
    """Launches so far that went to kernel family `path` (PATH_*)."""
    return int(ctx.lib.ghd_path_count(ctx.handle, path))


def ghd_tree_build(ctx: Ctx, parent, kv_len: int, tree: Tree | None = None) -> Tree:
    tree = tree or Tree(ctx)
    parent = np.ascontiguousarray(parent, dtype=np.int32)
    ctx._check(ctx.lib.ghd_tree_build(ctx.handle, parent.ctypes.data if parent.size else None, parent.size, kv_len,
                                      C.byref(tree.c)))
    return tree


def ghd_tree_from_mask(ctx: Ctx, mask_words, kv_len: int, depth=None, parent=None, tree: Tree | None = None) -> Tree:
    tree = tree or Tree(ctx)
    mask_words = np.ascontiguousarray(mask_words, dtype=np.uint64)
    n = mask_words.shape[0]
    depth = None if depth is None else np.ascontiguousarray(depth, dtype=np.int32)
    parent = None if parent is None else np.ascontiguousarray(parent, dtype=np.int32)
    ctx._check(ctx.lib.ghd_tree_from_mask(ctx.handle, mask_words.ctypes.data,
                                          None if depth is None else depth.ctypes.data,
                                          None if parent is None else parent.ctypes.data, n, kv_len, C.byref(tree.c)))
    return tree


def ghd_verify_layer(ctx: Ctx, w: LayerWeights, kv: KvLayer, tree: Tree, x_in, x_out=None):
    x_out = torch.empty_like(x_in) if x_out is None else x_out
    kvc = kv.c
    ctx._check(ctx.lib.ghd_verify_layer(ctx.handle, C.byref(w.c), C.byref(kvc), C.byref(tree.c), x_in.data_ptr(),
                                        x_out.data_ptr()))
    return x_out


def ghd_verify_step(ctx: Ctx, w: ModelWeights, kvs, tree: Tree, tokens, logits=None, argmax=None):
    """-> (logits or None, argmax).  Pass ``logits=False`` to keep the logits in the workspace only."""
    n = tree.c.n
    if logits is None:
        logits = torch.empty((n, ctx.cfg.c.vocab), dtype=torch.float32, device=ctx.device)
    elif logits is False:
        logits = None
    if argmax is None:
        argmax = torch.empty(n, dtype=torch.int32, device=ctx.device)
    arr = (_Kv * max(len(kvs), 1))(*[kv.c for kv in kvs])
    ctx._check(ctx.lib.ghd_verify_step(ctx.handle, C.byref(w.c), arr, C.byref(tree.c), tokens.data_ptr(),
                                       _ptr(logits), argmax.data_ptr()))
    return logits, argmax


def ghd_copy_hidden(ctx: Ctx, n: int, out=None):
    """-> float32 device tensor [n][d_model]: the last layer's output of the last ghd_verify_step (before the final norm)."""
    if out is None:
        out = torch.empty((n, ctx.cfg.c.d_model), dtype=torch.float32, device=ctx.device)
    ctx._check(ctx.lib.ghd_copy_hidden(ctx.handle, n, out.data_ptr()))
    return out


def ghd_accept(ctx: Ctx, tree: Tree, tokens, argmax, out=None):
    """-> int32 device tensor laid out as ghd_accept_result: [n_matched, n_emitted, nodes[256], tokens[256]]."""
    if out is None:
        out = torch.zeros(2 + 2 * GHD_MAX_NODES, dtype=torch.int32, device=ctx.device)
    ctx._check(ctx.lib.ghd_accept(ctx.handle, C.byref(tree.c), tokens.data_ptr(), argmax.data_ptr(), out.data_ptr()))
    return out


def ghd_kv_commit(ctx: Ctx, kvs, kv_len: int, result):
    """Moves the cache rows of the accepted path (device struct `result` from ghd_accept) to slots
    kv_len .. kv_len + n_matched in every layer of `kvs`.  The layers' `len` fields are left alone."""
    arr = (_Kv * len(kvs))(*[kv.c for kv in kvs])
    ctx._check(ctx.lib.ghd_kv_commit(ctx.handle, arr, len(kvs), kv_len, result.data_ptr()))


def ghd_kv_len_set(ctx: Ctx, kv_len: int):
    """Writes the context's device word with the cache length (read by calls given KV_LEN_DEVICE)."""
    ctx._check(ctx.lib.ghd_kv_len_set(ctx.handle, int(kv_len)))


def ghd_kv_len_get(ctx: Ctx) -> int:
    """Waits for the stream and reads the device word back."""
    out = C.c_int32(0)
    ctx._check(ctx.lib.ghd_kv_len_get(ctx.handle, C.byref(out)))
    return int(out.value)


def ghd_medusa_draft(ctx: Ctx, w: MedusaWeights, result, topk, want_logits: bool = False):
    """Candidates of the drafting heads at the last accepted node of `result` (device struct of ghd_accept).
    -> int32 device tensor [n_heads][GHD_MAX_TOPK] (best first, -1 past a head's top-k) (+ float logits [n_heads][vocab])."""
    topk = np.ascontiguousarray(topk, dtype=np.int32)
    k = w.c.n_heads
    cand = torch.empty((k, GHD_MAX_TOPK), dtype=torch.int32, device=ctx.device)
    logits = torch.empty((k, ctx.cfg.c.vocab), dtype=torch.float32, device=ctx.device) if want_logits else None
    ctx._check(ctx.lib.ghd_medusa_draft(ctx.handle, C.byref(w.c), result.data_ptr(), topk.ctypes.data, cand.data_ptr(),
                                        logits.data_ptr() if want_logits else None))
    return (cand, logits) if want_logits else cand


def ghd_tree_fill_tokens(ctx: Ctx, cand, result, level, rank, tokens=None):
    """tokens[0] = bonus token of `result`; tokens[i] = cand[level[i] - 1][rank[i]] (level, rank: int32 device tensors)."""
    n = int(level.numel())
    if tokens is None:
        tokens = torch.empty(n, dtype=torch.int32, device=ctx.device)
    ctx._check(ctx.lib.ghd_tree_fill_tokens(ctx.handle, cand.data_ptr(), result.data_ptr(), level.data_ptr(), rank.data_ptr(), n,
                                            tokens.data_ptr()))
    return tokens


def _kv4_here(ctx: Ctx) -> bool:
    """Whether the current stream is the context's.  The tensors that a call makes for its results are made on the context's, where
    the kernels write them: made on another, their fill (or what still runs there on the memory that they get) could come after."""
    return _raw_stream(ctx.dev) == ctx.raw_stream


def _kv4_there(ctx: Ctx, make, *args, **kw):
    """make(...) under the context's stream, for use on the current one."""
    with torch.cuda.stream(ctx.stream):
        t = make(*args, **kw)
    t.record_stream(torch.cuda.current_stream(ctx.device))
    return t


def ghd_kv4_pool_bytes(ctx: Ctx, kv: Kv4Cache) -> int:
    return int(ctx.lib.ghd_kv4_pool_bytes(ctx.handle, C.byref(kv.c)))


def ghd_kv4_pool(ctx: Ctx, kv: Kv4Cache, n_layers: int = 1):
    """A zeroed pool per layer, uint8 [n_layers][bytes]."""
    shape = (n_layers, ghd_kv4_pool_bytes(ctx, kv))
    if _kv4_here(ctx):
        return torch.zeros(shape, dtype=torch.uint8, device=ctx.device)
    return _kv4_there(ctx, torch.zeros, shape, dtype=torch.uint8, device=ctx.device)


def _kv4_match(ctx: Ctx, kv: Kv4Cache, rows: Kv4Rows):
    """Refuses descriptions that do not belong together or to the context's device."""
    if rows.n_starts <= kv.n_seqs:
        raise GhdError(1, "kv4: row_start has fewer than n_seqs + 1 entries")
    if kv.dev != ctx.dev or rows.dev != ctx.dev:
        raise GhdError(1, f"kv4: page table on cuda:{kv.dev}, rows on cuda:{rows.dev}, context on cuda:{ctx.dev}")


def _kv4_pool(ctx: Ctx, kv: Kv4Cache, pool):
    return _need(pool, torch.uint8, "pool", kv.n_rows * ctx.kv4_row, ctx.dev)


def _kv4_strided(ctx: Ctx, t, n: int, width: int, what: str):
    """Rows of `width` elements, contiguous inside a row and apart from one another -> (pointer, row stride; 0 for a single row,
    whose stride says nothing)."""
    if t.dim() != 2 or t.shape[0] < n or t.shape[1] != width or t.stride(1) != 1 or t.dtype != ctx.dtype or t.get_device() != ctx.dev:
        raise GhdError(1, f"{what}: want {ctx.dtype} [{n}][{width}] with contiguous rows on cuda:{ctx.dev}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    if n > 1 and t.stride(0) < width:       # a broadcast row has stride 0, which the call takes for rows one behind the other
        raise GhdError(1, f"{what}: rows of {width} elements overlap (row stride {t.stride(0)})")
    return t.data_ptr(), t.stride(0) if n > 1 else 0


def ghd_kv4_append(ctx: Ctx, kv: Kv4Cache, rows: Kv4Rows, pool, q, k, v, q_out=None):
    """Rotates q and k, quantises k and v into the pool behind each sequence's cache rows.  q, k, v: [n_rows][heads * d_head], rows may
    be strided (column blocks of one projection); q None: keys and values only.  -> rotated queries (q_out)."""
    n, width = rows.n_rows, kv.n_kv_heads * ctx.d_head
    _kv4_match(ctx, kv, rows)
    at = _kv4_pool(ctx, kv, pool)
    kp, kld = _kv4_strided(ctx, k, n, width, "k")
    vp, vld = _kv4_strided(ctx, v, n, width, "v")
    if kld != vld:
        raise GhdError(1, "kv4_append: k and v have different row strides")
    qp, qld, op = None, 0, None
    if q is not None:
        width = ctx.n_heads * ctx.d_head
        qp, qld = _kv4_strided(ctx, q, n, width, "q")
        if q_out is None:
            q_out = ctx.blank.new_empty((n, width)) if _kv4_here(ctx) else _kv4_there(ctx, ctx.blank.new_empty, (n, width))
        op = _need(q_out, ctx.dtype, "q_out", n * width, ctx.dev)
    ctx._check(ctx.lib.ghd_kv4_append(ctx.handle, kv.ref, rows.ref, at, qp, qld, kp, vp, kld, op))
    return q_out


def ghd_kv4_attention(ctx: Ctx, kv: Kv4Cache, rows: Kv4Rows, pool, q, out=None):
    """Attention of the new rows (rotated queries q [n_rows][n_heads * d_head]) over the paged 4-bit cache."""
    numel = rows.n_rows * ctx.n_heads * ctx.d_head
    _kv4_match(ctx, kv, rows)
    at = _kv4_pool(ctx, kv, pool)
    qp = _need(q, ctx.dtype, "q", numel, ctx.dev)
    if out is None:
        out = torch.zeros_like(q) if _kv4_here(ctx) else _kv4_there(ctx, torch.zeros_like, q)
    ctx._check(ctx.lib.ghd_kv4_attention(ctx.handle, kv.ref, rows.ref, at, qp, _need(out, ctx.dtype, "out", numel, ctx.dev)))
    return out


def ghd_kv4_read(ctx: Ctx, kv: Kv4Cache, pool, row_start, n_rows: int, first=None, k_out=None, v_out=None, keys: bool = True, values: bool = True):
    """Cache rows first[s] + i (first None: the new rows' places) in the storage type -> (k, v) [n_rows][n_kv_heads * d_head], None for
    the one that is not asked for."""
    rows = Kv4Rows(row_start, n_rows)
    _kv4_match(ctx, kv, rows)
    at = _kv4_pool(ctx, kv, pool)
    n, width = rows.n_rows, kv.n_kv_heads * ctx.d_head
    if n < 0:
        raise GhdError(1, "kv4_read: negative n_rows")
    shape = (n, width)
    kp = vp = None
    here = _raw_stream(ctx.dev) == ctx.raw_stream
    if k_out is not None:
        kp = _need(k_out, ctx.dtype, "k_out", n * width, ctx.dev)
    elif keys:
        k_out = ctx.blank.new_empty(shape) if here else _kv4_there(ctx, ctx.blank.new_empty, shape)
        kp = k_out.data_ptr()
    if v_out is not None:
        vp = _need(v_out, ctx.dtype, "v_out", n * width, ctx.dev)
    elif values:
        if here:
            v_out = torch.empty_like(k_out) if kp and k_out.shape == shape else ctx.blank.new_empty(shape)      # (the like of a tensor is made sooner)
        else:
            v_out = _kv4_there(ctx, ctx.blank.new_empty, shape)
        vp = v_out.data_ptr()
    if (kp and not keys) or (vp and not values):
        raise GhdError(1, "kv4_read: an output for what is not asked for")
    st = ctx.lib.ghd_kv4_read(ctx.handle, kv.ref, rows.ref, at, None if first is None else _need(first, torch.int32, "first", kv.n_seqs, ctx.dev), kp, vp)
    if st:
        ctx._check(st)
    return k_out, v_out


def ghd_kv4_commit(ctx: Ctx, kv: Kv4Cache, rows: Kv4Rows, pools, results=None):
    """Keeps the accepted rows of every sequence in all pools (a list, or one tensor [n_layers][...]) and advances kv.kv_len.
    results: int32 [n_seqs][514] as ghd_accept writes them; None keeps every new row (pools are not touched)."""
    _kv4_match(ctx, kv, rows)
    ptrs = [] if results is None else [_kv4_pool(ctx, kv, p) for p in pools]
    arr = (C.c_void_p * max(len(ptrs), 1))(*ptrs)
    ctx._check(ctx.lib.ghd_kv4_commit(ctx.handle, kv.ref, rows.ref, arr, len(ptrs),
                                      None if results is None else _need(results, torch.int32, "results", kv.n_seqs * (2 + 2 * GHD_MAX_NODES), ctx.dev)))


def _make(ctx: Ctx, shape, dtype):
    """An empty tensor for a result, made on the context's stream."""
    if _kv4_here(ctx):
        return torch.empty(shape, dtype=dtype, device=ctx.device)
    return _kv4_there(ctx, torch.empty, shape, dtype=dtype, device=ctx.device)


def ghd_mx4_code_bytes(m: int, k: int) -> int:
    return int(load_library().ghd_mx4_code_bytes(m, k))


def ghd_mx4_scale_bytes(m: int, k: int) -> int:
    return int(load_library().ghd_mx4_scale_bytes(m, k))


def ghd_mx4(ctx: Ctx, m: int, k: int) -> Mx4:
    """Room for a matrix [m][k] (its contents are anything until ghd_mx4_quantize has run)."""
    nc = ghd_mx4_code_bytes(m, k)
    if not nc:
        raise GhdError(2, f"mx4: a matrix of {m} x {k}")
    return Mx4(_make(ctx, (nc,), torch.uint8), _make(ctx, (ghd_mx4_scale_bytes(m, k),), torch.uint8), m, k)


def _mx4_here(ctx: Ctx, w: Mx4):
    if w.dev != ctx.dev:
        raise GhdError(1, f"mx4: a matrix on cuda:{w.dev}, the context is on cuda:{ctx.dev}")


def _mx4_rows(ctx: Ctx, t, n: int, k: int, what: str):
    """Rows of k elements, contiguous inside a row and apart from one another -> (pointer, row stride)."""
    if t.dim() != 2 or t.shape[0] != n or t.shape[1] != k or (k > 1 and t.stride(1) != 1) or t.dtype != ctx.dtype or t.get_device() != ctx.dev:
        raise GhdError(1, f"{what}: want {ctx.dtype} [{n}][{k}] with contiguous rows on cuda:{ctx.dev}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    if n > 1 and t.stride(0) < k:
        raise GhdError(1, f"{what}: rows of {k} elements overlap (row stride {t.stride(0)})")
    return t.data_ptr(), t.stride(0) if n > 1 else 0


def ghd_mx4_quantize(ctx: Ctx, x, w: Mx4 | None = None) -> Mx4:
    """x [m][k] (rows may be strided) in 4 bits, into w or a new one."""
    if x.dim() != 2:
        raise GhdError(1, "mx4_quantize: x is not [m][k]")
    if w is None:
        w = ghd_mx4(ctx, *x.shape)
    _mx4_here(ctx, w)
    at, ld = _mx4_rows(ctx, x, w.m, w.k, "x")
    ctx._check(ctx.lib.ghd_mx4_quantize(ctx.handle, at, ld, w.ref))
    return w


def ghd_mx4_read(ctx: Ctx, w: Mx4, out=None):
    """-> the values that w stands for, [m][k] (out's rows may be strided)."""
    _mx4_here(ctx, w)
    if out is None:
        out = _make(ctx, (w.m, w.k), ctx.dtype)
    at, ld = _mx4_rows(ctx, out, w.m, w.k, "out")
    ctx._check(ctx.lib.ghd_mx4_read(ctx.handle, w.ref, at, ld))
    return out


def ghd_mx4_linear(ctx: Ctx, x, w: Mx4, y=None):
    """y float [n][m] = x [n][k] (rows may be strided) w^T."""
    _mx4_here(ctx, w)
    n = x.shape[0]
    at, ld = _mx4_rows(ctx, x, n, w.k, "x")
    if y is None:
        y = _make(ctx, (n, w.m), torch.float32)
    ctx._check(ctx.lib.ghd_mx4_linear(ctx.handle, at, ld, w.ref, n, _need(y, torch.float32, "y", n * w.m, ctx.dev)))
    return y


def ghd_mx4_gate_up(ctx: Ctx, h, w_gate: Mx4, w_up: Mx4, u=None):
    """u [n][m] = SiLU(h w_gate^T) * (h w_up^T) (h's rows may be strided)."""
    _mx4_here(ctx, w_gate)
    _mx4_here(ctx, w_up)
    n = h.shape[0]
    at, ld = _mx4_rows(ctx, h, n, w_gate.k, "h")
    if u is None:
        u = _make(ctx, (n, w_gate.m), ctx.dtype)
    ctx._check(ctx.lib.ghd_mx4_gate_up(ctx.handle, at, ld, w_gate.ref, w_up.ref, n, _need(u, ctx.dtype, "u", n * w_gate.m, ctx.dev)))
    return u


def ghd_draft_sample(ctx: Ctx, logits, uniforms, n_draws: int, temperature: float = 1.0, cand=None):
    """Tokens drawn without replacement from each row of logits float [n_rows][vocab] with uniforms float [n_rows][GHD_MAX_TOPK]
    -> int32 [n_rows][GHD_MAX_TOPK], -1 from n_draws on."""
    if logits.dim() != 2 or logits.shape[1] != ctx.cfg.c.vocab:
        raise GhdError(1, f"draft_sample: logits are not [n_rows][{ctx.cfg.c.vocab}]")
    n = logits.shape[0]
    if not (n < _INT and -_INT <= n_draws < _INT):
        raise GhdError(1, "draft_sample: n_rows or n_draws is outside 32 bits")
    if cand is None:
        cand = _make(ctx, (n, GHD_MAX_TOPK), torch.int32)
    ctx._check(ctx.lib.ghd_draft_sample(ctx.handle, _need(logits, torch.float32, "logits", 0, ctx.dev), n, temperature, n_draws,
                                        _need(uniforms, torch.float32, "uniforms", n * GHD_MAX_TOPK, ctx.dev),
                                        _need(cand, torch.int32, "cand", n * GHD_MAX_TOPK, ctx.dev)))
    return cand


def ghd_accept_sampled(ctx: Ctx, rows: SampledRows, out=None):
    """-> int32 [n_seqs][514], a ghd_accept_result for every sequence: [n_matched, n_emitted, nodes[256], tokens[256]]."""
    if rows.dev != ctx.dev or rows.vocab != ctx.cfg.c.vocab:
        raise GhdError(1, f"accept_sampled: {rows.vocab} logits a row on cuda:{rows.dev}, the context has {ctx.cfg.c.vocab} on cuda:{ctx.dev}")
    if out is None:
        out = _make(ctx, (rows.n_seqs, 2 + 2 * GHD_MAX_NODES), torch.int32)
    ctx._check(ctx.lib.ghd_accept_sampled(ctx.handle, rows.ref, _need(out, torch.int32, "out", rows.n_seqs * (2 + 2 * GHD_MAX_NODES), ctx.dev)))
    return out


def ghd_linear(ctx: Ctx, x, w, y=None):
    n, k = x.shape
    m = w.shape[0]
    if y is None:
        y = torch.empty((n, m), dtype=torch.float32, device=ctx.device)
    ctx._check(ctx.lib.ghd_linear(ctx.handle, x.data_ptr(), w.data_ptr(), n, k, m, y.data_ptr()))
    return y


def ghd_gate_up(ctx: Ctx, h, w_gate_up, u=None):
    """u [n][d_ffn] = SiLU(h Wg^T) * (h Wu^T) with the layer's own kernel (gate rows first in w_gate_up)."""
    n = h.shape[0]
    if u is None:
        u = torch.empty((n, ctx.cfg.c.d_ffn), dtype=ctx.cfg.torch_dtype, device=ctx.device)
    ctx._check(ctx.lib.ghd_gate_up(ctx.handle, h.data_ptr(), w_gate_up.data_ptr(), n, u.data_ptr()))
    return u


def ghd_rmsnorm(ctx: Ctx, x, g, out=None):
    if out is None:
        out = torch.empty(x.shape, dtype=ctx.cfg.torch_dtype, device=ctx.device)
    ctx._check(ctx.lib.ghd_rmsnorm(ctx.handle, x.data_ptr(), g.data_ptr(), x.shape[0], out.data_ptr()))
    return out


def ghd_tree_attention(ctx: Ctx, q, kv: KvLayer, tree: Tree, out=None):
    out = torch.empty_like(q) if out is None else out
    kvc = kv.c
    ctx._check(ctx.lib.ghd_tree_attention(ctx.handle, q.data_ptr(), C.byref(kvc), C.byref(tree.c), out.data_ptr()))
    return out


def ghd_tree_attention_static(q, k_cache, v_cache, mask_dev, n_heads: int, d_head: int, kv_len: int, out=None):
    """Tree attention without a context or workspace, for callers that may not allocate device
    memory: the split partials live in an array inside the library (limits: 64 nodes,
    n_heads * d_head <= 4096).  Runs on torch's current stream; ``out`` is the caller's."""
    lib = load_library()
    n = q.shape[0]
    out = torch.empty_like(q) if out is None else out
    err = C.create_string_buffer(256)
    st = lib.ghd_tree_attention_static(C.c_void_p(torch.cuda.current_stream().cuda_stream),
                                       GHD_F32 if q.dtype == torch.float32 else GHD_F16, n_heads, d_head,
                                       k_cache.shape[1], q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
                                       mask_dev.data_ptr(), n, kv_len, out.data_ptr(), err, 256)
    if st != 0:
        raise GhdError(st, err.value.decode())
    return out


def ghd_argmax(ctx: Ctx, logits, out=None):
    n, v = logits.shape
    if out is None:
        out = torch.empty(n, dtype=torch.int32, device=ctx.device)
    ctx._check(ctx.lib.ghd_argmax(ctx.handle, logits.data_ptr(), n, v, out.data_ptr()))
    return out


def ghd_sync_status(ctx: Ctx):
    ctx._check(ctx.lib.ghd_sync_status(ctx.handle))


def ghd_launch_count(ctx: Ctx) -> int:
    return int(ctx.lib.ghd_launch_count(ctx.handle))
