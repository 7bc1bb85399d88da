"""ctypes binding of ``librheo.so`` (include/rheo.h): argument marshalling only.

Every step of the path runs in the library's CUDA kernels.  PyTorch provides
device memory and the current stream.  There is no CPU fallback: importing
works anywhere, but the first call raises if the library has not been built.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librheo.so")

RHEO_F32, RHEO_BF16 = 0, 1
RHEO_OK, RHEO_EINVAL, RHEO_ELAUNCH, RHEO_ETOOLARGE = 0, -1, -2, -3
VERIFY_RHEO, VERIFY_RRSW, VERIFY_ONEHOT = 0, 1, 2
STATUS_BAD_LOGIT, STATUS_EMPTY_ROW, STATUS_BAD_TEMPERATURE, STATUS_INTERNAL = 1, 2, 4, 8
STATUS_BAD_LENGTH, STATUS_NO_PAGES, STATUS_BAD_INDEX, STATUS_BAD_VALUE = 16, 32, 64, 128
SLOT_ROOT, SLOT_LEAD, SLOT_SAMPLED, SLOT_FILL = 0, 1, 2, 3

EXPORTS = ("rheo_sizes", "rheo_workspace_init", "rheo_expand", "rheo_prune", "rheo_verify", "rheo_verify_static",
           "rheo_tree_attention", "rheo_verify_variant", "rheo_verify_full",
           "rheo_get_status", "rheo_cache_sizes", "rheo_scratch_init", "rheo_scratch_status", "rheo_cache_reserve",
           "rheo_qk_norm_rope", "rheo_tree_attend", "rheo_cache_commit", "rheo_logprob_sizes", "rheo_token_logprobs",
           "rheo_window_attend", "rheo_packed_sizes", "rheo_cache_pack", "rheo_cache_unpack", "rheo_packed_attend")


class RheoError(RuntimeError):
    pass


class _Config(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("vocab", ctypes.c_int32), ("K", ctypes.c_int32),
                ("m", ctypes.c_int32), ("support", ctypes.c_int32), ("depth", ctypes.c_int32),
                ("budget", ctypes.c_int32), ("eps", ctypes.c_float), ("dtype", ctypes.c_int32)]


_VP = ctypes.c_void_p


class _Tree(ctypes.Structure):
    _fields_ = [(n, _VP) for n in ("token", "parent", "log_proxy", "score", "qtilde", "slot", "frontier",
                                   "tail_ids", "tail_q", "lse1", "lse_tail")]


class _Pruned(ctypes.Structure):
    _fields_ = [(n, _VP) for n in ("gen_id", "token", "parent", "depth", "first_child", "n_child",
                                   "sampled_child")]


class _VerifyOut(ctypes.Structure):
    _fields_ = [(n, _VP) for n in ("accepted_len", "accepted_tokens", "accepted_nodes", "bonus_token",
                                   "row_lse")]


class _TreeAttn(ctypes.Structure):
    _fields_ = [(n, _VP) for n in ("mask", "position", "retrieve", "n_leaves")]


class _CacheConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "tokens", "pages", "page_size", "max_pages", "q_heads",
                                              "kv_heads", "head_dim", "dtype")]


class _Pages(ctypes.Structure):
    _fields_ = [(n, _VP) for n in ("block_table", "n_pages", "free_list", "n_free")]


class _KV(ctypes.Structure):
    _fields_ = [("key", _VP), ("value", _VP)] + [(n, ctypes.c_int64) for n in (
        "key_page", "key_head", "key_token", "value_page", "value_head", "value_token")]


class _QKV(ctypes.Structure):
    _fields_ = [(n, _VP) for n in "qkv"] + [(f"{n}_{d}", ctypes.c_int64) for n in "qkv"
                                            for d in ("batch", "token", "head")]


class _AttendIO(ctypes.Structure):
    _fields_ = [(n, _VP) for n in ("q", "out", "lse")] + [(f"{n}_{d}", ctypes.c_int64) for n in ("q", "out")
                                                          for d in ("batch", "token", "head")]


class _LogprobConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "vocab", "top", "dtype", "rows_per_temperature")]


class _Logprobs(ctypes.Structure):
    _fields_ = [(n, _VP) for n in ("logprob", "rank", "entropy", "top_ids", "top_logprobs")]


class _Window(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("sinks", ctypes.c_int32), ("depth", _VP)]


class _Packed(ctypes.Structure):
    _fields_ = [("data", _VP), ("page", ctypes.c_int64), ("head", ctypes.c_int64)]


_lib = None


def library_path() -> str:
    return _LIB_PATH


def lib():
    """Load librheo.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RheoError(f"{_LIB_PATH} not found: build it with paper_2609_21827_gb300.build.build()")
        L = ctypes.CDLL(_LIB_PATH)
        C = ctypes.POINTER(_Config)
        L.rheo_sizes.argtypes = [C, ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64),
                                 ctypes.POINTER(ctypes.c_size_t)]
        L.rheo_workspace_init.argtypes = [C, _VP, ctypes.c_size_t, _VP]
        L.rheo_expand.argtypes = [C, ctypes.c_int32, _VP, ctypes.c_int64, _VP, _VP, _VP, ctypes.POINTER(_Tree),
                                  _VP, _VP]
        L.rheo_prune.argtypes = [C, ctypes.POINTER(_Tree), ctypes.POINTER(_Pruned), _VP, _VP]
        L.rheo_verify.argtypes = [C, _VP, ctypes.c_int64, _VP, _VP, _VP, ctypes.POINTER(_Tree),
                                  ctypes.POINTER(_Pruned), ctypes.POINTER(_VerifyOut), _VP, _VP]
        L.rheo_verify_static.argtypes = [C, _VP, ctypes.c_int64, _VP, _VP, _VP, ctypes.POINTER(_Tree),
                                         ctypes.POINTER(_Pruned), ctypes.POINTER(_VerifyOut), _VP, _VP]
        L.rheo_get_status.argtypes = [C, _VP, _VP, ctypes.POINTER(ctypes.c_int32)]
        L.rheo_verify_variant.argtypes = [C, ctypes.c_int32, _VP, ctypes.c_int64, _VP, _VP, _VP,
                                          ctypes.POINTER(_Tree), ctypes.POINTER(_Pruned), ctypes.POINTER(_VerifyOut),
                                          _VP, _VP]
        L.rheo_verify_full.argtypes = [C, _VP, ctypes.c_int64, _VP, ctypes.c_int64, _VP, _VP, _VP,
                                       ctypes.POINTER(_Tree), ctypes.POINTER(_Pruned), ctypes.POINTER(_VerifyOut),
                                       _VP, _VP]
        L.rheo_tree_attention.argtypes = [C, ctypes.POINTER(_Pruned), ctypes.POINTER(_TreeAttn), _VP, _VP]
        K, i32, i64, f32 = ctypes.POINTER(_CacheConfig), ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        KV, PG = ctypes.POINTER(_KV), ctypes.POINTER(_Pages)
        L.rheo_cache_sizes.argtypes = [K, ctypes.POINTER(ctypes.c_size_t)]
        L.rheo_scratch_init.argtypes = [_VP, ctypes.c_size_t, _VP]
        L.rheo_scratch_status.argtypes = [_VP, _VP, ctypes.POINTER(i32)]
        L.rheo_cache_reserve.argtypes = [K, _VP, _VP, _VP, PG, PG, _VP, _VP, _VP, _VP]
        L.rheo_qk_norm_rope.argtypes = [K, ctypes.POINTER(_QKV), _VP, _VP, f32, _VP, i32, i32, i32, _VP, _VP, KV, _VP,
                                        i64, i64, i64, _VP, _VP]
        L.rheo_tree_attend.argtypes = [K, ctypes.POINTER(_AttendIO), KV, _VP, _VP, _VP, _VP, f32, _VP, _VP]
        L.rheo_cache_commit.argtypes = [K, i32, KV, i64, i64, _VP, _VP, _VP, _VP, i32, _VP, _VP, _VP]
        L.rheo_logprob_sizes.argtypes = [ctypes.POINTER(_LogprobConfig), ctypes.POINTER(ctypes.c_size_t)]
        L.rheo_token_logprobs.argtypes = [ctypes.POINTER(_LogprobConfig), _VP, i64, i64, _VP, _VP, _VP,
                                          ctypes.POINTER(_Logprobs), _VP, _VP]
        W, P4 = ctypes.POINTER(_Window), ctypes.POINTER(_Packed)
        L.rheo_window_attend.argtypes = [K, ctypes.POINTER(_AttendIO), KV, _VP, _VP, _VP, _VP, W, f32, _VP, _VP]
        L.rheo_packed_sizes.argtypes = [K, ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_size_t)]
        L.rheo_cache_pack.argtypes = [K, K, i32, KV, i64, i64, P4, i64, i32, PG, PG, _VP, PG, PG, _VP, _VP, _VP]
        L.rheo_cache_unpack.argtypes = [K, K, i32, P4, i64, KV, i64, i64, i32, _VP, _VP, _VP, _VP]
        L.rheo_packed_attend.argtypes = [K, K, ctypes.POINTER(_AttendIO), KV, _VP, _VP, _VP, P4, _VP, _VP, _VP, W, f32, _VP,
                                         _VP]
        for name in EXPORTS:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


# The current stream's handle without a Stream object (3 us less a call), where this build of torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(_device())
    return torch.cuda.current_stream().cuda_stream


def _check(rc: int, what: str):
    if rc != RHEO_OK:
        raise RheoError(f"{what} failed with code {rc}")


@dataclass
class Config:
    batch: int
    vocab: int
    K: int
    depth: int
    budget: int
    m: int = 1
    support: int | None = None
    eps: float = 1e-6
    dtype: str = "bf16"

    def __post_init__(self):
        if self.support is None:
            self.support = min(128, self.vocab)

    @property
    def dtype_code(self) -> int:
        return RHEO_BF16 if self.dtype == "bf16" else RHEO_F32

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    def c(self) -> _Config:
        return _Config(self.batch, self.vocab, self.K, self.m, self.support, self.depth, self.budget,
                       self.eps, self.dtype_code)

    def sizes(self):
        g1, e, ws = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_size_t()
        _check(lib().rheo_sizes(ctypes.byref(self.c()), ctypes.byref(g1), ctypes.byref(e), ctypes.byref(ws)),
               "rheo_sizes")
        return g1.value, e.value, ws.value

    def rows_at(self, d: int) -> int:
        return 1 if d == 1 else self.K


class Tree:
    """Device buffers of the unpruned tree (include/rheo.h rheo_tree)."""

    def __init__(self, cfg: Config, device="cuda"):
        G1, E, _ = cfg.sizes()
        B, TL = cfg.batch, (0 if cfg.support == 0 else cfg.support - cfg.m)
        i32, f32 = torch.int32, torch.float32
        self.token = torch.full((B, G1), -1, dtype=i32, device=device)
        self.parent = torch.full((B, G1), -1, dtype=i32, device=device)
        self.log_proxy = torch.zeros((B, G1), dtype=f32, device=device)
        self.score = torch.zeros((B, G1), dtype=f32, device=device)
        self.qtilde = torch.zeros((B, G1), dtype=f32, device=device)
        self.slot = torch.zeros((B, G1), dtype=torch.uint8, device=device)
        self.frontier = torch.zeros((B, max(cfg.K, 1)), dtype=i32, device=device)
        self.tail_ids = torch.zeros((B, E, TL), dtype=i32, device=device)
        self.tail_q = torch.zeros((B, E, TL), dtype=f32, device=device)
        self.lse1 = torch.zeros((B, E), dtype=f32, device=device)
        self.lse_tail = torch.zeros((B, E), dtype=f32, device=device)

    def c(self) -> _Tree:
        return _Tree(*[getattr(self, n).data_ptr() for n, _ in _Tree._fields_])


class Pruned:
    def __init__(self, cfg: Config, device="cuda"):
        shape = (cfg.batch, cfg.budget + 1)
        for n, _ in _Pruned._fields_:
            setattr(self, n, torch.zeros(shape, dtype=torch.int32, device=device))

    def c(self) -> _Pruned:
        return _Pruned(*[getattr(self, n).data_ptr() for n, _ in _Pruned._fields_])


class VerifyOut:
    def __init__(self, cfg: Config, device="cuda", row_lse: bool = True):
        B, D = cfg.batch, cfg.depth
        self.accepted_len = torch.zeros(B, dtype=torch.int32, device=device)
        self.accepted_tokens = torch.zeros((B, D), dtype=torch.int32, device=device)
        self.accepted_nodes = torch.zeros((B, D), dtype=torch.int32, device=device)
        self.bonus_token = torch.zeros(B, dtype=torch.int32, device=device)
        self.row_lse = torch.zeros((B, cfg.budget + 1), dtype=torch.float32, device=device) if row_lse else None

    def c(self) -> _VerifyOut:
        return _VerifyOut(self.accepted_len.data_ptr(), self.accepted_tokens.data_ptr(),
                          self.accepted_nodes.data_ptr(), self.bonus_token.data_ptr(),
                          self.row_lse.data_ptr() if self.row_lse is not None else None)


class Workspace:
    def __init__(self, cfg: Config, device="cuda", stream=None):
        _, _, nbytes = cfg.sizes()
        self.nbytes = nbytes
        self.buf = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
        self.init(cfg, stream)

    def init(self, cfg: Config, stream=None):
        _check(lib().rheo_workspace_init(ctypes.byref(cfg.c()), self.buf.data_ptr(), self.nbytes, _stream(stream)),
               "rheo_workspace_init")

    def ptr(self) -> int:
        return self.buf.data_ptr()


def _rows(cfg: Config, logits: torch.Tensor, n_rows: int):
    """Validate a [.., V] logits tensor whose rows are uniformly strided; returns the row stride."""
    if logits.dtype != cfg.torch_dtype:
        raise RheoError(f"logits dtype {logits.dtype} does not match config dtype {cfg.dtype}")
    if not logits.is_cuda:
        raise RheoError("logits must be a CUDA tensor")
    if logits.shape[-1] != cfg.vocab or logits.stride(-1) != 1:
        raise RheoError("the last dimension must be the vocabulary, unit stride")
    rows = logits.reshape(-1, cfg.vocab) if logits.dim() != 2 else logits
    if rows.shape[0] != n_rows:
        raise RheoError(f"expected {n_rows} rows, got {rows.shape[0]}")
    if rows.data_ptr() != logits.data_ptr():
        raise RheoError("rows must be addressable with a single row stride")
    return rows.stride(0)


def _i64(x: torch.Tensor) -> torch.Tensor:
    if x.dtype not in (torch.int64, torch.uint64) or not x.is_cuda or not x.is_contiguous():
        raise RheoError("seed/offset must be contiguous 64-bit CUDA tensors")
    return x


def _f32(x: torch.Tensor) -> torch.Tensor:
    if x.dtype != torch.float32 or not x.is_cuda or not x.is_contiguous():
        raise RheoError("temperature must be a contiguous float32 CUDA tensor")
    return x


def expand(cfg: Config, d: int, logits: torch.Tensor, temperature: torch.Tensor, seed: torch.Tensor,
           offset: torch.Tensor, tree: Tree, ws: Workspace, stream=None) -> None:
    """rheo_expand: logits [B, F_d, V] (or [B*F_d, V]) of the frontier rows in frontier order."""
    stride = _rows(cfg, logits, cfg.batch * cfg.rows_at(d))
    _check(lib().rheo_expand(ctypes.byref(cfg.c()), d, logits.data_ptr(), stride, _f32(temperature).data_ptr(),
                             _i64(seed).data_ptr(), _i64(offset).data_ptr(), ctypes.byref(tree.c()), ws.ptr(),
                             _stream(stream)), "rheo_expand")


def prune(cfg: Config, tree: Tree, pruned: Pruned, ws: Workspace, stream=None) -> None:
    _check(lib().rheo_prune(ctypes.byref(cfg.c()), ctypes.byref(tree.c()), ctypes.byref(pruned.c()), ws.ptr(),
                            _stream(stream)), "rheo_prune")


class TreeAttn:
    """Outputs of rheo_tree_attention (ancestor mask, positions, root-to-leaf paths)."""

    def __init__(self, cfg: Config, device="cuda"):
        B, NP, W = cfg.batch, cfg.budget + 1, cfg.depth + 1
        self.mask = torch.zeros((B, NP, NP), dtype=torch.uint8, device=device)
        self.position = torch.zeros((B, NP), dtype=torch.int32, device=device)
        self.retrieve = torch.zeros((B, NP, W), dtype=torch.int32, device=device)
        self.n_leaves = torch.zeros((B,), dtype=torch.int32, device=device)

    def c(self) -> _TreeAttn:
        return _TreeAttn(*[getattr(self, n).data_ptr() for n, _ in _TreeAttn._fields_])


def tree_attention(cfg: Config, pruned: Pruned, out: TreeAttn, ws: Workspace, stream=None) -> None:
    _check(lib().rheo_tree_attention(ctypes.byref(cfg.c()), ctypes.byref(pruned.c()), ctypes.byref(out.c()),
                                     ws.ptr(), _stream(stream)), "rheo_tree_attention")


def verify(cfg: Config, logits: torch.Tensor, temperature: torch.Tensor, seed: torch.Tensor,
           offset: torch.Tensor, tree: Tree, pruned: Pruned, out: VerifyOut, ws: Workspace, stream=None) -> None:
    """rheo_verify: logits [B, N+1, V] of the pruned nodes in pruned order."""
    stride = _rows(cfg, logits, cfg.batch * (cfg.budget + 1))
    _check(lib().rheo_verify(ctypes.byref(cfg.c()), logits.data_ptr(), stride, _f32(temperature).data_ptr(),
                             _i64(seed).data_ptr(), _i64(offset).data_ptr(), ctypes.byref(tree.c()),
                             ctypes.byref(pruned.c()), ctypes.byref(out.c()), ws.ptr(), _stream(stream)),
           "rheo_verify")


def verify_variant(cfg: Config, variant: int, logits: torch.Tensor, temperature: torch.Tensor, seed: torch.Tensor,
                   offset: torch.Tensor, tree: Tree, pruned: Pruned, out: VerifyOut, ws: Workspace,
                   stream=None) -> None:
    """rheo_verify_variant: VERIFY_RHEO (Algorithm 1), VERIFY_RRSW or VERIFY_ONEHOT."""
    stride = _rows(cfg, logits, cfg.batch * (cfg.budget + 1))
    _check(lib().rheo_verify_variant(ctypes.byref(cfg.c()), int(variant), logits.data_ptr(), stride,
                                     _f32(temperature).data_ptr(), _i64(seed).data_ptr(), _i64(offset).data_ptr(),
                                     ctypes.byref(tree.c()), ctypes.byref(pruned.c()), ctypes.byref(out.c()),
                                     ws.ptr(), _stream(stream)),
           "rheo_verify_variant")


def verify_full(cfg: Config, logits: torch.Tensor, draft_rows: list, temperature: torch.Tensor, seed: torch.Tensor,
                offset: torch.Tensor, tree: Tree, pruned: Pruned, out: VerifyOut, ws: Workspace, stream=None) -> None:
    """rheo_verify_full: draft_rows[d-1] = the [B, F_d, V] rows given to expand at depth d."""
    stride = _rows(cfg, logits, cfg.batch * (cfg.budget + 1))
    dstride = None
    ptrs = (ctypes.c_void_p * cfg.depth)()
    for d, x in enumerate(draft_rows):
        st = _rows(cfg, x, x.shape[0] * x.shape[1])
        if dstride is None:
            dstride = st
        elif st != dstride:
            raise RheoError("draft rows of every depth need the same row stride")
        ptrs[d] = x.data_ptr()
    _check(lib().rheo_verify_full(ctypes.byref(cfg.c()), logits.data_ptr(), stride, ptrs, dstride,
                                  _f32(temperature).data_ptr(), _i64(seed).data_ptr(), _i64(offset).data_ptr(),
                                  ctypes.byref(tree.c()), ctypes.byref(pruned.c()), ctypes.byref(out.c()), ws.ptr(),
                                  _stream(stream)),
           "rheo_verify_full")


def verify_static(cfg: Config, logits: torch.Tensor, temperature: torch.Tensor, seed: torch.Tensor,
                  offset: torch.Tensor, tree: Tree, pruned: Pruned, out: VerifyOut,
                  status: torch.Tensor = None, stream=None) -> None:
    """rheo_verify_static: rheo_verify without a workspace, for callers that may
    not allocate device memory when they verify.  Its scratch is a fixed static
    array inside the library (calls must not overlap on the GPU); configurations
    that need more than it holds raise RheoError with code RHEO_ETOOLARGE.
    status: optional int32 device tensor of one element that receives the
    call's status word."""
    stride = _rows(cfg, logits, cfg.batch * (cfg.budget + 1))
    st = 0
    if status is not None:
        if status.dtype != torch.int32 or status.numel() < 1 or not status.is_cuda:
            raise RheoError("status must be an int32 device tensor")
        st = status.data_ptr()
    _check(lib().rheo_verify_static(ctypes.byref(cfg.c()), logits.data_ptr(), stride, _f32(temperature).data_ptr(),
                                    _i64(seed).data_ptr(), _i64(offset).data_ptr(), ctypes.byref(tree.c()),
                                    ctypes.byref(pruned.c()), ctypes.byref(out.c()), st,
                                    _stream(stream)),
           "rheo_verify_static")


def status(cfg: Config, ws: Workspace, stream=None) -> int:
    """Synchronise the stream, return and clear the device status word."""
    st = ctypes.c_int32()
    _check(lib().rheo_get_status(ctypes.byref(cfg.c()), ws.ptr(), _stream(stream), ctypes.byref(st)),
           "rheo_get_status")
    return st.value


# ---------------------------------------------------------------------------
# The target forward over the pruned tree, with a paged key/value cache, and the
# log probabilities of given tokens (include/rheo.h has the definitions).
# ---------------------------------------------------------------------------

_CODES = {"bf16": (RHEO_BF16, torch.bfloat16), "f32": (RHEO_F32, torch.float32)}


def _dtype_of(name: str):
    if name not in _CODES:
        raise RheoError(f"dtype {name!r}: 'bf16' or 'f32' is wanted")
    return _CODES[name]


@dataclass(frozen=True)
class CacheConfig:
    """Sizes of the cache functions (include/rheo.h rheo_cache_config): up to `tokens` new tokens
    (a pruned tree: budget + 1) of each of `batch` requests, over `pages` pages of `page_size`."""

    batch: int
    tokens: int
    pages: int
    page_size: int
    max_pages: int
    q_heads: int
    kv_heads: int
    head_dim: int
    dtype: str = "bf16"

    def __post_init__(self):
        code, torch_dtype = _dtype_of(self.dtype)
        c = _CacheConfig(self.batch, self.tokens, self.pages, self.page_size, self.max_pages, self.q_heads,
                         self.kv_heads, self.head_dim, code)
        B, T, H, D = self.batch, self.tokens, self.kv_heads, self.head_dim
        for name, value in (("torch_dtype", torch_dtype), ("_c", c), ("_ref", ctypes.byref(c)), ("_bytes", None), ("_bytes4", None),
                            ("_one", (B,)), ("_each", (B, T)), ("_table", (B, self.max_pages)),
                            ("_free", (self.pages,)), ("_q", (B, T, self.q_heads, D)), ("_k", (B, T, H, D)),
                            ("_lse", (B, T, self.q_heads)), ("_mask", (B, T, T)), ("_pool", (self.pages, H, self.page_size, D))):
            object.__setattr__(self, name, value)

    def scratch_bytes(self) -> int:
        if self._bytes is None:
            n = ctypes.c_size_t()
            _check(lib().rheo_cache_sizes(self._ref, ctypes.byref(n)), "rheo_cache_sizes")
            object.__setattr__(self, "_bytes", n.value)
        return self._bytes

    def packed_scratch_bytes(self) -> int:
        if self._bytes4 is None:
            n = ctypes.c_size_t()
            _check(lib().rheo_packed_sizes(self._ref, None, ctypes.byref(n)), "rheo_packed_sizes")
            object.__setattr__(self, "_bytes4", n.value)
        return self._bytes4


@dataclass(frozen=True)
class LogprobConfig:
    """Sizes of token_logprobs (include/rheo.h rheo_logprob_config)."""

    rows: int
    vocab: int
    top: int = 0
    dtype: str = "bf16"
    rows_per_temperature: int = 1

    def __post_init__(self):
        code, torch_dtype = _dtype_of(self.dtype)
        c = _LogprobConfig(self.rows, self.vocab, self.top, code, self.rows_per_temperature)
        for name, value in (("torch_dtype", torch_dtype), ("_c", c), ("_ref", ctypes.byref(c)), ("_bytes", None),
                            ("_rows", (self.rows,)), ("_top", (self.rows, self.top)),
                            ("_groups", (-(-self.rows // max(self.rows_per_temperature, 1)),))):
            object.__setattr__(self, name, value)

    def scratch_bytes(self) -> int:
        if self._bytes is None:
            n = ctypes.c_size_t()
            _check(lib().rheo_logprob_sizes(self._ref, ctypes.byref(n)), "rheo_logprob_sizes")
            object.__setattr__(self, "_bytes", n.value)
        return self._bytes


class _Scratch:
    """A scratch buffer, zeroed when made; one for each stream whose calls may overlap."""

    def __init__(self, cfg, device="cuda", stream=None):
        self.nbytes = self._size(cfg)
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        self._ptr = self.buf.data_ptr()
        self.init(stream)

    @staticmethod
    def _size(cfg) -> int:
        return cfg.scratch_bytes()

    def of(self, cfg) -> int:
        """The buffer's pointer, if it is large enough for cfg."""
        if self.nbytes < (cfg._bytes or cfg.scratch_bytes()):
            raise RheoError(f"the workspace holds {self.nbytes} bytes, {cfg.scratch_bytes()} are wanted")
        return self._ptr

    def init(self, stream=None):
        _check(lib().rheo_scratch_init(self._ptr, self.nbytes, _stream(stream)), "rheo_scratch_init")

    def ptr(self) -> int:
        return self._ptr


class CacheWorkspace(_Scratch):
    """For the functions over packed pages too, which only bf16 caches have and which ask for more, some four times as much, up
    to 32 query rows (tokens * q_heads / kv_heads) of a key/value head: a workspace of a few more rows is refused there."""

    @staticmethod
    def _size(cfg) -> int:
        return cfg.packed_scratch_bytes() if cfg.dtype == "bf16" else cfg.scratch_bytes()

    def of_packed(self, cfg) -> int:
        """The buffer's pointer, if it is large enough for the functions over packed pages."""
        wanted = cfg._bytes4 or cfg.packed_scratch_bytes()
        if self.nbytes < wanted:
            raise RheoError(f"the workspace holds {self.nbytes} bytes, {wanted} are wanted for packed pages")
        return self._ptr


class LogprobWorkspace(_Scratch):
    pass


def scratch_status(ws: _Scratch, stream=None) -> int:
    """Synchronise the stream, return and clear the status word of a cache or log-probability workspace."""
    st = ctypes.c_int32()
    _check(lib().rheo_scratch_status(ws.ptr(), _stream(stream), ctypes.byref(st)), "rheo_scratch_status")
    return st.value


def _want(x: torch.Tensor, name: str, dtype, shape) -> int:
    """The pointer of a contiguous CUDA tensor of this type and shape."""
    if x.dtype is not dtype or not x.is_cuda or x.shape != shape or not x.is_contiguous():
        raise RheoError(f"{name}: a contiguous CUDA tensor of {dtype} and shape {list(shape)} is wanted, "
                        f"got {x.dtype} {list(x.shape)} on {x.device}")
    return x.data_ptr()


def _want_opt(x, name: str, dtype, shape) -> int:
    return 0 if x is None else _want(x, name, dtype, shape)


def _want_strided(x: torch.Tensor, name: str, dtype, shape) -> tuple:
    """The pointer and the strides of a CUDA tensor whose last dimension is contiguous."""
    if x.dtype is not dtype or not x.is_cuda or x.shape != shape:
        raise RheoError(f"{name}: a CUDA tensor of {dtype} and shape {list(shape)} is wanted, "
                        f"got {x.dtype} {list(x.shape)} on {x.device}")
    st = x.stride()
    if st[-1] != 1:
        raise RheoError(f"{name}: the last dimension has to be contiguous")
    return x.data_ptr(), st


class Pages:
    """Pages of the requests and the stack of free ones.  Without arguments every page is free
    (page 0 on top); given tensors are used as they are."""

    def __init__(self, cfg: CacheConfig, device="cuda", block_table=None, n_pages=None, free_list=None, n_free=None):
        i32 = torch.int32
        if block_table is None:
            block_table = torch.full((cfg.batch, cfg.max_pages), -1, dtype=i32, device=device)
        if n_pages is None:
            n_pages = torch.zeros(cfg.batch, dtype=i32, device=device)
        if free_list is None:
            free_list = torch.arange(cfg.pages - 1, -1, -1, dtype=i32, device=device)
        if n_free is None:
            n_free = torch.full((1,), cfg.pages, dtype=i32, device=device)
        self.block_table, self.n_pages, self.free_list, self.n_free = block_table, n_pages, free_list, n_free

    def table(self, cfg: CacheConfig) -> int:
        return _want(self.block_table, "block_table", torch.int32, cfg._table)

    def c(self, cfg: CacheConfig) -> _Pages:
        i32 = torch.int32
        return _Pages(self.table(cfg), _want(self.n_pages, "n_pages", i32, cfg._one),
                      _want(self.free_list, "free_list", i32, cfg._free), _want(self.n_free, "n_free", i32, (1,)))


class CachePlan:
    """Slots [B, T] (int64) and positions [B, T] (int32) of a call's new tokens."""

    def __init__(self, cfg: CacheConfig, device="cuda", slot=None, position=None):
        shape = (cfg.batch, cfg.tokens)
        self.slot = torch.full(shape, -1, dtype=torch.int64, device=device) if slot is None else slot
        self.position = torch.full(shape, -1, dtype=torch.int32, device=device) if position is None else position

    def ptrs(self, cfg: CacheConfig) -> tuple:
        return (_want(self.slot, "slot", torch.int64, cfg._each),
                _want(self.position, "position", torch.int32, cfg._each))


def make_cache(cfg: CacheConfig, layers: int = 1, device="cuda"):
    """Zeroed key and value pools [layers, pages, kv_heads, page_size, head_dim]."""
    shape = (layers, cfg.pages, cfg.kv_heads, cfg.page_size, cfg.head_dim)
    return (torch.zeros(shape, dtype=cfg.torch_dtype, device=device),
            torch.zeros(shape, dtype=cfg.torch_dtype, device=device))


def _kv(cfg: CacheConfig, key: torch.Tensor, value: torch.Tensor) -> _KV:
    kp, (kb, kh, kt, _) = _want_strided(key, "key cache", cfg.torch_dtype, cfg._pool)
    vp, (vb, vh, vt, _) = _want_strided(value, "value cache", cfg.torch_dtype, cfg._pool)
    return _KV(kp, vp, kb, kh, kt, vb, vh, vt)


def cache_reserve(cfg: CacheConfig, ctx_len: torch.Tensor, pages: Pages, plan: CachePlan, ws: CacheWorkspace,
                  new_len: torch.Tensor = None, depth: torch.Tensor = None, out: Pages = None, stream=None) -> None:
    """rheo_cache_reserve: pages for ctx_len + new_len tokens a request, slots and positions of the new ones.
    `pages` is updated in place, or stays as it is and `out` receives the new state."""
    i32 = torch.int32
    before = pages.c(cfg)
    after = before if out is None else out.c(cfg)
    slot, position = plan.ptrs(cfg)
    _check(lib().rheo_cache_reserve(
        cfg._ref, _want(ctx_len, "ctx_len", i32, cfg._one), _want_opt(new_len, "new_len", i32, cfg._one),
        _want_opt(depth, "depth", i32, cfg._each), before, after, slot, position, ws.of(cfg), _stream(stream)),
        "rheo_cache_reserve")


def qk_norm_rope(cfg: CacheConfig, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_weight, k_weight, cos_sin,
                 plan: CachePlan, key_cache: torch.Tensor, value_cache: torch.Tensor, q_out: torch.Tensor,
                 ws: CacheWorkspace, eps: float = 1e-6, interleaved: bool = False, stream=None) -> None:
    """rheo_qk_norm_rope: q [B, T, q_heads, D], k and v [B, T, kv_heads, D] of one layer; weights [D] or None (no
    norm); cos_sin [positions, rot] fp32 (cosines, then sines) or None (no rotation).  Queries go to q_out (may be
    q), keys and values to the caches [pages, kv_heads, page_size, D] at plan.slot."""
    dt, one = cfg.torch_dtype, (cfg.head_dim,)
    qp, qs = _want_strided(q, "q", dt, cfg._q)
    kp, ks = _want_strided(k, "k", dt, cfg._k)
    vp, vs = _want_strided(v, "v", dt, cfg._k)
    op, os_ = (qp, qs) if q_out is q else _want_strided(q_out, "q_out", dt, cfg._q)
    if op == qp and os_ != qs:
        raise RheoError("q_out on q's memory needs q's strides")
    most = rot = table = 0
    if cos_sin is not None:
        if cos_sin.dim() != 2:
            raise RheoError("cos_sin: [positions, rot] is wanted")
        most, rot = cos_sin.shape
        table = _want(cos_sin, "cos_sin", torch.float32, (most, rot))
    kv = _kv(cfg, key_cache, value_cache)
    x = _QKV(qp, kp, vp, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2], vs[0], vs[1], vs[2])
    slot, position = plan.ptrs(cfg)
    _check(lib().rheo_qk_norm_rope(
        cfg._ref, x, _want_opt(q_weight, "q_weight", dt, one), _want_opt(k_weight, "k_weight", dt, one), eps, table, most,
        rot, 1 if interleaved else 0, slot, position, kv, op, os_[0], os_[1], os_[2], ws.of(cfg), _stream(stream)),
        "rheo_qk_norm_rope")


def tree_attend(cfg: CacheConfig, q: torch.Tensor, key_cache: torch.Tensor, value_cache: torch.Tensor, pages: Pages,
                ctx_len: torch.Tensor, out: torch.Tensor, ws: CacheWorkspace, new_len: torch.Tensor = None,
                mask: torch.Tensor = None, lse: torch.Tensor = None, scale: float = None, stream=None) -> None:
    """rheo_tree_attend: attention of the new tokens q [B, T, q_heads, D] over the cache, their own keys and values
    included; mask [B, T, T] uint8 as tree_attention writes it (None: every earlier token); scale: 1/sqrt(D)."""
    dt, i32 = cfg.torch_dtype, torch.int32
    qp, qs = _want_strided(q, "q", dt, cfg._q)
    op, os_ = _want_strided(out, "out", dt, cfg._q)
    io = _AttendIO(qp, op, _want_opt(lse, "lse", torch.float32, cfg._lse), qs[0], qs[1], qs[2], os_[0], os_[1], os_[2])
    kv = _kv(cfg, key_cache, value_cache)
    _check(lib().rheo_tree_attend(
        cfg._ref, io, kv, pages.table(cfg), _want(ctx_len, "ctx_len", i32, cfg._one),
        _want_opt(new_len, "new_len", i32, cfg._one), _want_opt(mask, "mask", torch.uint8, cfg._mask),
        cfg.head_dim ** -0.5 if scale is None else scale, ws.of(cfg), _stream(stream)), "rheo_tree_attend")


def cache_commit(cfg: CacheConfig, key_cache: torch.Tensor, value_cache: torch.Tensor, pages: Pages,
                 ctx_len: torch.Tensor, accepted_len: torch.Tensor, accepted_nodes: torch.Tensor,
                 next_len: torch.Tensor, ws: CacheWorkspace, stream=None) -> None:
    """rheo_cache_commit: the accepted path's lines move behind the root in caches [layers, pages, kv_heads,
    page_size, D]; next_len = ctx_len + 1 + accepted_len (a tensor apart from the other ones)."""
    i32 = torch.int32
    if key_cache.dim() != 5 or accepted_nodes.dim() != 2:
        raise RheoError("caches [layers, pages, kv_heads, page_size, D] and accepted_nodes [B, depth] are wanted")
    layers, depth = key_cache.shape[0], accepted_nodes.shape[1]
    shape = (layers,) + cfg._pool
    kp, ks = _want_strided(key_cache, "key cache", cfg.torch_dtype, shape)
    vp, vs = _want_strided(value_cache, "value cache", cfg.torch_dtype, shape)
    _check(lib().rheo_cache_commit(
        cfg._ref, layers, _KV(kp, vp, ks[1], ks[2], ks[3], vs[1], vs[2], vs[3]), ks[0], vs[0], pages.table(cfg),
        _want(ctx_len, "ctx_len", i32, cfg._one), _want(accepted_len, "accepted_len", i32, cfg._one),
        _want(accepted_nodes, "accepted_nodes", i32, (cfg.batch, depth)), depth,
        _want(next_len, "next_len", i32, cfg._one), ws.of(cfg), _stream(stream)), "rheo_cache_commit")


class Logprobs:
    """Outputs of token_logprobs."""

    def __init__(self, cfg: LogprobConfig, device="cuda"):
        R, k = cfg.rows, cfg.top
        self.logprob = torch.zeros(R, dtype=torch.float32, device=device)
        self.rank = torch.zeros(R, dtype=torch.int32, device=device)
        self.entropy = torch.zeros(R, dtype=torch.float32, device=device)
        self.top_ids = torch.zeros((R, k), dtype=torch.int32, device=device)
        self.top_logprobs = torch.zeros((R, k), dtype=torch.float32, device=device)

    def c(self, cfg: LogprobConfig) -> _Logprobs:
        f32, i32, rows, top = torch.float32, torch.int32, cfg._rows, cfg._top
        return _Logprobs(_want(self.logprob, "logprob", f32, rows), _want(self.rank, "rank", i32, rows),
                         _want(self.entropy, "entropy", f32, rows), _want(self.top_ids, "top_ids", i32, top),
                         _want(self.top_logprobs, "top_logprobs", f32, top))


def token_logprobs(cfg: LogprobConfig, logits: torch.Tensor, tokens: torch.Tensor, out: Logprobs,
                   ws: LogprobWorkspace, temperature: torch.Tensor = None, rows: torch.Tensor = None,
                   stream=None) -> None:
    """rheo_token_logprobs: row i reads row rows[i] (None: i) of logits [..., V] and token tokens[i]; -1 leaves a
    row or a token out; temperature [ceil(R / rows_per_temperature)] fp32 or None (1)."""
    R, V, i32 = cfg.rows, cfg.vocab, torch.int32
    if logits.dtype is not cfg.torch_dtype or not logits.is_cuda or logits.shape[-1] != V:
        raise RheoError(f"logits: a CUDA tensor of {cfg.torch_dtype} and {V} columns is wanted")
    flat = logits if logits.dim() == 2 else logits.reshape(-1, V)
    st, p = flat.stride(), flat.data_ptr()
    if (st[1] != 1 and V > 1) or (flat is not logits and p != logits.data_ptr()):
        raise RheoError("logits rows must be contiguous and addressable with a single row stride")
    n = flat.shape[0]
    if rows is None and n < R:
        raise RheoError(f"{R} rows are asked for, logits have {n}")
    _check(lib().rheo_token_logprobs(
        cfg._ref, p, max(st[0], V) if n == 1 else st[0], n, _want_opt(rows, "rows", i32, cfg._rows),
        _want(tokens, "tokens", i32, cfg._rows), _want_opt(temperature, "temperature", torch.float32, cfg._groups),
        out.c(cfg), ws.of(cfg), _stream(stream)), "rheo_token_logprobs")


# ---------------------------------------------------------------------------
# Long contexts: attention limited to a window, and caches held in 4 bits (include/rheo.h
# has the definitions).  A packed pool has a CacheConfig of its own, the cache's but for
# pages and max_pages, and Pages like any other.
# ---------------------------------------------------------------------------

def packed_page_bytes(packed_cfg: CacheConfig) -> int:
    """Bytes of a packed page of one head."""
    n = ctypes.c_int64()
    _check(lib().rheo_packed_sizes(packed_cfg._ref, ctypes.byref(n), None), "rheo_packed_sizes")
    return n.value


def make_packed(packed_cfg: CacheConfig, layers: int = 1, device="cuda") -> torch.Tensor:
    """Packed pages [layers, pages, kv_heads, bytes] (uint8), unwritten ones zero."""
    return torch.zeros((layers, packed_cfg.pages, packed_cfg.kv_heads, packed_page_bytes(packed_cfg)), dtype=torch.uint8,
                       device=device)


def _packed_shape(packed_cfg: CacheConfig) -> tuple:
    shape = getattr(packed_cfg, "_packed", None)
    if shape is None:
        shape = (packed_cfg.pages, packed_cfg.kv_heads, packed_page_bytes(packed_cfg))
        object.__setattr__(packed_cfg, "_packed", shape)
    return shape


def _count(x: int, name: str) -> int:
    """A number of positions, which the library holds in 32 bits."""
    if not 0 <= x < 1 << 31:
        raise RheoError(f"{name}: 0 .. 2^31 - 1 is wanted, got {x}")
    return x


def _window(cfg: CacheConfig, window: int, sinks: int, depth) -> _Window:
    _count(window, "window"), _count(sinks, "sinks")
    return _Window(window, sinks, _want_opt(depth, "depth", torch.int32, cfg._each))


def _attend_io(cfg: CacheConfig, q: torch.Tensor, out: torch.Tensor, lse) -> _AttendIO:
    qp, qs = _want_strided(q, "q", cfg.torch_dtype, cfg._q)
    op, os_ = _want_strided(out, "out", cfg.torch_dtype, cfg._q)
    return _AttendIO(qp, op, _want_opt(lse, "lse", torch.float32, cfg._lse), qs[0], qs[1], qs[2], os_[0], os_[1], os_[2])


def window_attend(cfg: CacheConfig, q: torch.Tensor, key_cache: torch.Tensor, value_cache: torch.Tensor, pages: Pages,
                  ctx_len: torch.Tensor, out: torch.Tensor, ws: CacheWorkspace, window: int, sinks: int = 0,
                  depth: torch.Tensor = None, new_len: torch.Tensor = None, mask: torch.Tensor = None,
                  lse: torch.Tensor = None, scale: float = None, stream=None) -> None:
    """rheo_window_attend: tree_attend in which a token sees the last `window` positions (its own among them; 0: all) and
    the first `sinks`; depth [B, T] int32, the new tokens' depths as tree_attention writes them (None: 0, 1, ...)."""
    i32 = torch.int32
    _check(lib().rheo_window_attend(
        cfg._ref, _attend_io(cfg, q, out, lse), _kv(cfg, key_cache, value_cache), pages.table(cfg),
        _want(ctx_len, "ctx_len", i32, cfg._one), _want_opt(new_len, "new_len", i32, cfg._one),
        _want_opt(mask, "mask", torch.uint8, cfg._mask), _window(cfg, window, sinks, depth),
        cfg.head_dim ** -0.5 if scale is None else scale, ws.of(cfg), _stream(stream)), "rheo_window_attend")


def packed_attend(cfg: CacheConfig, packed_cfg: CacheConfig, q: torch.Tensor, key_cache: torch.Tensor,
                  value_cache: torch.Tensor, pages: Pages, ctx_len: torch.Tensor, packed: torch.Tensor, packed_pages: Pages,
                  out: torch.Tensor, ws: CacheWorkspace, window: int = 0, sinks: int = 0, depth: torch.Tensor = None,
                  new_len: torch.Tensor = None, mask: torch.Tensor = None, lse: torch.Tensor = None, scale: float = None,
                  stream=None) -> None:
    """rheo_packed_attend: attention over packed_pages.n_pages packed pages a request (packed [pages, kv_heads, bytes], one
    layer) and the ctx_len tokens in 16 bits behind them; the window as in window_attend (0: none)."""
    i32 = torch.int32
    pp, ps = _want_strided(packed, "packed", torch.uint8, _packed_shape(packed_cfg))
    _check(lib().rheo_packed_attend(
        cfg._ref, packed_cfg._ref, _attend_io(cfg, q, out, lse), _kv(cfg, key_cache, value_cache), pages.table(cfg),
        _want(ctx_len, "ctx_len", i32, cfg._one), _want_opt(new_len, "new_len", i32, cfg._one), _Packed(pp, ps[0], ps[1]),
        packed_pages.table(packed_cfg), _want(packed_pages.n_pages, "n_pages", i32, packed_cfg._one),
        _want_opt(mask, "mask", torch.uint8, cfg._mask), _window(cfg, window, sinks, depth),
        cfg.head_dim ** -0.5 if scale is None else scale, ws.of_packed(cfg), _stream(stream)), "rheo_packed_attend")


def _layers(cfg: CacheConfig, packed_cfg: CacheConfig, key_cache, value_cache, packed) -> tuple:
    """Layers, key and value caches [layers, pages, kv_heads, page_size, D] and packed pages with their layers' strides."""
    if key_cache.dim() != 5 or packed.dim() != 4:
        raise RheoError("caches [layers, pages, kv_heads, page_size, D] and packed pages [layers, pages, kv_heads, bytes] "
                        "are wanted")
    n = key_cache.shape[0]
    kp, ks = _want_strided(key_cache, "key cache", cfg.torch_dtype, (n,) + cfg._pool)
    vp, vs = _want_strided(value_cache, "value cache", cfg.torch_dtype, (n,) + cfg._pool)
    pp, ps = _want_strided(packed, "packed", torch.uint8, (n,) + _packed_shape(packed_cfg))
    return n, _KV(kp, vp, ks[1], ks[2], ks[3], vs[1], vs[2], vs[3]), ks[0], vs[0], _Packed(pp, ps[1], ps[2]), ps[0]


def cache_pack(cfg: CacheConfig, packed_cfg: CacheConfig, key_cache: torch.Tensor, value_cache: torch.Tensor,
               packed: torch.Tensor, pages: Pages, packed_pages: Pages, ctx_len: torch.Tensor, ws: CacheWorkspace,
               keep: int = 0, out: tuple = None, stream=None) -> None:
    """rheo_cache_pack: whole pages of the caches [layers, pages, kv_heads, page_size, D] go into 4 bits, all but the last
    `keep` tokens of a request.  pages, packed_pages and ctx_len are updated in place, or stay as they are and
    out = (Pages, Pages, ctx_len) receives the new state."""
    _count(keep, "keep")
    n, kv, kl, vl, p4, pl = _layers(cfg, packed_cfg, key_cache, value_cache, packed)
    before, before4, ctx = pages.c(cfg), packed_pages.c(packed_cfg), _want(ctx_len, "ctx_len", torch.int32, cfg._one)
    after, after4, ctx_out = (before, before4, ctx) if out is None else (
        out[0].c(cfg), out[1].c(packed_cfg), _want(out[2], "ctx_len of out", torch.int32, cfg._one))
    _check(lib().rheo_cache_pack(cfg._ref, packed_cfg._ref, n, kv, kl, vl, p4, pl, keep, before, before4, ctx, after, after4,
                                 ctx_out, ws.of_packed(cfg), _stream(stream)), "rheo_cache_pack")


def cache_unpack(cfg: CacheConfig, packed_cfg: CacheConfig, packed: torch.Tensor, key_cache: torch.Tensor,
                 value_cache: torch.Tensor, src: torch.Tensor, dst: torch.Tensor, ws: CacheWorkspace, stream=None) -> None:
    """rheo_cache_unpack: packed pages src [n] int32 back to pages dst [n] of the caches, in every layer; -1 leaves an
    entry out."""
    n, kv, kl, vl, p4, pl = _layers(cfg, packed_cfg, key_cache, value_cache, packed)
    if src.dim() != 1:
        raise RheoError("src: [n] is wanted")
    shape = tuple(src.shape)
    _check(lib().rheo_cache_unpack(cfg._ref, packed_cfg._ref, n, p4, pl, kv, kl, vl, shape[0],
                                   _want(src, "src", torch.int32, shape), _want(dst, "dst", torch.int32, shape), ws.of_packed(cfg),
                                   _stream(stream)), "rheo_cache_unpack")
