"""Thin Python binding of libmcsd.so: argument marshalling only.

Every step of the verification runs inside the CUDA library; this module turns
torch tensors into raw pointers, fills the descriptor and raises on a non-zero
return code.  It fails loudly when the library is missing: there is no CPU or
eager fallback.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmcsd.so")
DEBUG_LIB_PATH = os.path.join(_HERE, "libmcsd_debug.so")      # the checked build (see mcsd_debug_bounds_hits)

MCSD_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
STATUS_DEGENERATE, STATUS_BAD_TOKEN, STATUS_NO_MASS, STATUS_TIMEOUT, STATUS_NO_PAGES, STATUS_BAD_MASK = 1, 2, 4, 8, 16, 32
MAX_NODES, MAX_CHILDREN, MAX_VOCAB, MAX_SEQUENCES, MAX_GROUP, MAX_TOP = 512, 32, 65536, 4096, 128, 32

EXPORTS = ("mcsd_verify", "mcsd_verify_nodes", "mcsd_verify_walk", "mcsd_verify_host", "mcsd_verify_static", "mcsd_verify_path", "mcsd_sample_candidates", "mcsd_tree_attention_layout",
           "mcsd_gather_accepted_kv",
           "mcsd_workspace_bytes", "mcsd_tree_depth", "mcsd_last_launch_count", "mcsd_status_string",
           "mcsd_version", "mcsd_set_option", "mcsd_get_option", "mcsd_release_host_staging",
           "mcsd_shard_columns", "mcsd_shard_workspace_bytes", "mcsd_shard_rounds", "mcsd_shard_partials",
           "mcsd_shard_decide", "mcsd_shard_endpoint", "mcsd_shard_finish", "mcsd_shard_commit", "mcsd_debug_bounds_hits", "mcsd_last_kernel_times",
           "mcsd_apply_logit_rules", "mcsd_build_page_tables", "mcsd_kv_block_bytes", "mcsd_append_kv", "mcsd_read_kv",
           "mcsd_tree_attention", "mcsd_tree_attention_workspace_bytes", "mcsd_gather_accepted_pages",
           "mcsd_chunk_attention", "mcsd_chunk_attention_workspace_bytes", "mcsd_accumulate_weights", "mcsd_evict_rows", "mcsd_token_logprobs")
OPT_CLUSTER, OPT_EPT, OPT_DIRECT, OPT_SAMPLE_AHEAD, OPT_WAIT_POLLS, OPT_TEST_EXTRA_TX, OPT_PDL, OPT_TEST_SHRINK_RANGES, OPT_SPLIT, OPT_TIME_KERNELS, OPT_TRACE, OPT_WALK_CLUSTER = range(12)


class McsdDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_nodes", ctypes.c_int32), ("n_internal", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("ld_target", ctypes.c_int64), ("ld_draft", ctypes.c_int64),
                ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t),
                ("node_accept", ctypes.c_void_p), ("node_bonus", ctypes.c_void_p),
                ("node_ratio", ctypes.c_void_p), ("out_status", ctypes.c_void_p),
                ("out_path_nodes", ctypes.c_void_p), ("node_residual", ctypes.c_void_p)]


class McsdShardDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_nodes", ctypes.c_int32), ("n_internal", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("n_shards", ctypes.c_int32), ("shard", ctypes.c_int32),
                ("ld_target", ctypes.c_int64), ("ld_draft", ctypes.c_int64),
                ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("node_ratio", ctypes.c_void_p), ("node_accept", ctypes.c_void_p)]


class McsdLogitRules(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("history_len", ctypes.c_void_p), ("prompt_len", ctypes.c_void_p),
                ("ld_history", ctypes.c_int64), ("repetition", ctypes.c_void_p), ("frequency", ctypes.c_void_p),
                ("presence", ctypes.c_void_p), ("bias_ids", ctypes.c_void_p), ("bias_values", ctypes.c_void_p),
                ("masks", ctypes.c_void_p), ("mask_index", ctypes.c_void_p), ("n_masks", ctypes.c_int64),
                ("ld_mask", ctypes.c_int64), ("n_history", ctypes.c_int32), ("n_bias", ctypes.c_int32)]


class McsdPageDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("new_tokens", ctypes.c_int32), ("ring_capacity", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("ld_table", ctypes.c_int64), ("n_slots", ctypes.c_int64), ("start", ctypes.c_void_p),
                ("count", ctypes.c_void_p), ("page_table", ctypes.c_void_p), ("held", ctypes.c_void_p),
                ("held_out", ctypes.c_void_p), ("ring", ctypes.c_void_p), ("ring_state", ctypes.c_void_p),
                ("ring_state_out", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("cu_tokens", ctypes.c_void_p),
                ("status", ctypes.c_void_p), ("stream", ctypes.c_void_p)]


class McsdKvCache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("n_pages", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32)]


class McsdAttentionDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_nodes", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("ld_table", ctypes.c_int64), ("q_seq_stride", ctypes.c_int64), ("q_node_stride", ctypes.c_int64),
                ("q_head_stride", ctypes.c_int64), ("out_seq_stride", ctypes.c_int64),
                ("out_node_stride", ctypes.c_int64), ("out_head_stride", ctypes.c_int64), ("scale", ctypes.c_float),
                ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class McsdChunkDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_heads", ctypes.c_int32), ("dtype", ctypes.c_int32), ("max_pages", ctypes.c_int32),
                ("max_new", ctypes.c_int32), ("reserved", ctypes.c_int32), ("n_tokens", ctypes.c_int64), ("ld_table", ctypes.c_int64),
                ("q_token_stride", ctypes.c_int64), ("q_head_stride", ctypes.c_int64), ("out_token_stride", ctypes.c_int64),
                ("out_head_stride", ctypes.c_int64), ("scale", ctypes.c_float), ("stream", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class McsdEvictDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("keep", ctypes.c_int32), ("sink", ctypes.c_int32),
                ("recent", ctypes.c_int32), ("reserved", ctypes.c_int32), ("n_layers", ctypes.c_int64), ("layer_stride", ctypes.c_int64),
                ("weight_stride", ctypes.c_int64), ("ld_table", ctypes.c_int64), ("page_table", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("keep_len", ctypes.c_void_p), ("weights", ctypes.c_void_p), ("len_out", ctypes.c_void_p), ("stream", ctypes.c_void_p)]


class McsdLogprobDesc(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32), ("n_given", ctypes.c_int32), ("n_top", ctypes.c_int32),
                ("path_len", ctypes.c_int32), ("nodes_per_tree", ctypes.c_int32), ("n_logits", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("n_out", ctypes.c_int64), ("logits", ctypes.c_void_p), ("row_index", ctypes.c_void_p), ("path_nodes", ctypes.c_void_p),
                ("tokens", ctypes.c_void_p), ("logprobs", ctypes.c_void_p), ("entropy", ctypes.c_void_p), ("top_ids", ctypes.c_void_p),
                ("top_logprobs", ctypes.c_void_p), ("temperature", ctypes.c_float), ("reserved", ctypes.c_int32), ("stream", ctypes.c_void_p)]


class McsdError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"libmcsd error {code}: {text}")
        self.code = code


_lib = None


def load_library(path: Optional[str] = None):
    """dlopen libmcsd.so and declare its signatures.  Raises if it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it with `python -m paper_2401_06706_b200.build` "
                           "(there is no fallback path)")
    lib = ctypes.CDLL(p)
    vp, i32, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
    dp = ctypes.POINTER(McsdDesc)
    lib.mcsd_verify.argtypes = [dp, vp, vp, vp, vp, vp, f32, ctypes.c_int, vp, vp, vp]
    lib.mcsd_verify.restype = ctypes.c_int
    lib.mcsd_verify_path.argtypes = [dp, vp, vp, vp, vp, vp, f32, ctypes.c_int, vp, vp, vp]
    lib.mcsd_verify_path.restype = ctypes.c_int
    lib.mcsd_sample_candidates.argtypes = [dp, vp, vp, vp, f32, ctypes.c_int, i32, i32, vp]
    lib.mcsd_sample_candidates.restype = ctypes.c_int
    lib.mcsd_tree_attention_layout.argtypes = [vp, i32, i32, vp, vp, vp]
    lib.mcsd_tree_attention_layout.restype = ctypes.c_int
    i64 = ctypes.c_int64
    lib.mcsd_gather_accepted_kv.argtypes = [vp, i64, i64, i32, i64, i64, i64, i64, vp, vp, vp, i32, vp]
    lib.mcsd_gather_accepted_kv.restype = ctypes.c_int
    lib.mcsd_verify_static.argtypes = [dp, vp, vp, vp, vp, vp, f32, ctypes.c_int, vp, vp, vp]
    lib.mcsd_verify_static.restype = ctypes.c_int
    lib.mcsd_verify_nodes.argtypes = [dp, vp, vp, vp, vp, vp, f32, ctypes.c_int]
    lib.mcsd_verify_nodes.restype = ctypes.c_int
    lib.mcsd_verify_walk.argtypes = [dp, vp, vp, vp, vp, vp, f32, vp, vp, vp]
    lib.mcsd_verify_walk.restype = ctypes.c_int
    lib.mcsd_verify_host.argtypes = [dp, vp, vp, vp, vp, vp, f32, ctypes.c_int, vp, vp, vp, vp]
    lib.mcsd_verify_host.restype = ctypes.c_int
    lib.mcsd_workspace_bytes.argtypes = [dp]
    lib.mcsd_workspace_bytes.restype = ctypes.c_size_t
    lib.mcsd_tree_depth.argtypes = [vp, i32]
    lib.mcsd_tree_depth.restype = ctypes.c_int
    lib.mcsd_last_launch_count.argtypes = []
    lib.mcsd_last_launch_count.restype = ctypes.c_int
    lib.mcsd_status_string.argtypes = [ctypes.c_int]
    lib.mcsd_status_string.restype = ctypes.c_char_p
    lib.mcsd_version.argtypes = []
    lib.mcsd_version.restype = ctypes.c_int
    lib.mcsd_set_option.argtypes = [ctypes.c_int, ctypes.c_int]
    lib.mcsd_set_option.restype = ctypes.c_int
    lib.mcsd_get_option.argtypes = [ctypes.c_int]
    lib.mcsd_get_option.restype = ctypes.c_int
    lib.mcsd_release_host_staging.argtypes = []
    lib.mcsd_release_host_staging.restype = ctypes.c_int
    sp = ctypes.POINTER(McsdShardDesc)
    lib.mcsd_shard_columns.argtypes = [i32, i32, i32, i32, vp, vp, vp]
    lib.mcsd_shard_columns.restype = ctypes.c_int
    lib.mcsd_shard_workspace_bytes.argtypes = [sp]
    lib.mcsd_shard_workspace_bytes.restype = ctypes.c_size_t
    lib.mcsd_shard_rounds.argtypes = [vp, i32]
    lib.mcsd_shard_rounds.restype = ctypes.c_int
    lib.mcsd_shard_partials.argtypes = [sp, vp, vp, vp, vp, f32, i32, vp, vp]
    lib.mcsd_shard_partials.restype = ctypes.c_int
    lib.mcsd_shard_decide.argtypes = [sp, vp, vp, vp, f32, ctypes.c_int, i32, vp, vp]
    lib.mcsd_shard_decide.restype = ctypes.c_int
    lib.mcsd_shard_endpoint.argtypes = [sp, vp, vp, vp, f32, i32, vp, vp, vp]
    lib.mcsd_shard_endpoint.restype = ctypes.c_int
    lib.mcsd_shard_finish.argtypes = [sp, vp, vp, vp, vp, vp, f32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.mcsd_shard_finish.restype = ctypes.c_int
    lib.mcsd_shard_commit.argtypes = [sp, vp, vp, vp, vp]
    lib.mcsd_shard_commit.restype = ctypes.c_int
    lib.mcsd_last_kernel_times.argtypes = [vp, i32]
    lib.mcsd_last_kernel_times.restype = ctypes.c_int
    lib.mcsd_debug_bounds_hits.argtypes = [ctypes.c_int]
    lib.mcsd_debug_bounds_hits.restype = ctypes.c_longlong
    cp = ctypes.POINTER(McsdKvCache)
    lib.mcsd_apply_logit_rules.argtypes = [dp, ctypes.POINTER(McsdLogitRules), vp, vp, vp, i64, vp, i64, i32, i32, i32]
    lib.mcsd_apply_logit_rules.restype = ctypes.c_int
    lib.mcsd_build_page_tables.argtypes = [ctypes.POINTER(McsdPageDesc)]
    lib.mcsd_build_page_tables.restype = ctypes.c_int
    lib.mcsd_kv_block_bytes.argtypes = [i32, i32]
    lib.mcsd_kv_block_bytes.restype = ctypes.c_size_t
    lib.mcsd_append_kv.argtypes = [cp, vp, i64, i64, vp, i64, i64, i32, i64, vp, vp]
    lib.mcsd_append_kv.restype = ctypes.c_int
    lib.mcsd_read_kv.argtypes = [cp, vp, i64, i64, vp, i64, i64, i32, i64, vp, vp]
    lib.mcsd_read_kv.restype = ctypes.c_int
    ap = ctypes.POINTER(McsdAttentionDesc)
    lib.mcsd_tree_attention_workspace_bytes.argtypes = [ap, cp]
    lib.mcsd_tree_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.mcsd_tree_attention.argtypes = [ap, cp, vp, vp, vp, vp, vp, vp]
    lib.mcsd_tree_attention.restype = ctypes.c_int
    lib.mcsd_gather_accepted_pages.argtypes = [cp, i64, i64, vp, i64, i32, i32, vp, vp, vp, i32, vp]
    lib.mcsd_gather_accepted_pages.restype = ctypes.c_int
    kp = ctypes.POINTER(McsdChunkDesc)
    lib.mcsd_chunk_attention_workspace_bytes.argtypes = [kp, cp]
    lib.mcsd_chunk_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.mcsd_chunk_attention.argtypes = [kp, cp, vp, vp, vp, vp, vp, vp]
    lib.mcsd_chunk_attention.restype = ctypes.c_int
    lib.mcsd_accumulate_weights.argtypes = [kp, cp, vp, vp, vp, vp, vp, vp, f32, i32]
    lib.mcsd_accumulate_weights.restype = ctypes.c_int
    lib.mcsd_evict_rows.argtypes = [ctypes.POINTER(McsdEvictDesc), cp]
    lib.mcsd_evict_rows.restype = ctypes.c_int
    lib.mcsd_token_logprobs.argtypes = [ctypes.POINTER(McsdLogprobDesc)]
    lib.mcsd_token_logprobs.restype = ctypes.c_int
    if path is None:
        _lib = lib
    return lib


def status_string(code: int) -> str:
    return load_library().mcsd_status_string(int(code)).decode()


def _check(code: int):
    if code != 0:
        raise McsdError(code, status_string(code))


def mcsd_version() -> int:
    return int(load_library().mcsd_version())


def mcsd_tree_depth(parent) -> int:
    parent = np.ascontiguousarray(parent, dtype=np.int32)
    rc = load_library().mcsd_tree_depth(parent.ctypes.data, parent.shape[0])
    _check(rc if rc < 0 else 0)
    return rc


def mcsd_last_launch_count() -> int:
    return int(load_library().mcsd_last_launch_count())


def mcsd_set_option(option: int, value: int) -> None:
    _check(load_library().mcsd_set_option(int(option), int(value)))


def mcsd_get_option(option: int) -> int:
    rc = load_library().mcsd_get_option(int(option))
    _check(rc if rc < 0 else 0)
    return rc


def mcsd_last_kernel_times():
    """[cluster / argmax / naive, streaming statistics, single test, walk] kernel milliseconds of the last call
    (needs MCSD_OPT_TIME_KERNELS); None where no such kernel ran."""
    ms = (ctypes.c_float * 4)()
    rc = load_library().mcsd_last_kernel_times(ctypes.addressof(ms), 4)
    _check(rc if rc < 0 else 0)
    return [None if x < 0 else float(x) for x in ms]


def mcsd_debug_bounds_hits(reset: bool = False) -> int:
    return int(load_library().mcsd_debug_bounds_hits(1 if reset else 0))


def mcsd_release_host_staging() -> None:
    _check(load_library().mcsd_release_host_staging())


def _n_internal(parent: np.ndarray) -> int:
    has = np.zeros(parent.shape[0], dtype=bool)
    if parent.shape[0] > 1:
        has[parent[1:][parent[1:] >= 0]] = True
    return int(has.sum())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _row_stride(t: torch.Tensor) -> int:
    """Elements between consecutive rows of a [B, rows, V] tensor whose rows are contiguous and
    whose leading dimensions collapse to one stride."""
    assert t.dim() == 3 and (t.shape[2] == 1 or t.stride(2) == 1), "vocabulary axis must be contiguous"
    ld = t.stride(1) if t.shape[1] > 1 else max(t.shape[2], t.stride(1))
    if t.shape[0] > 1:
        assert t.stride(0) == ld * t.shape[1], "batch stride must equal rows * row stride"
    return int(ld)


@dataclass
class VerifyOutput:
    accept_len: torch.Tensor            # [B] int32
    tokens: torch.Tensor                # [B, gamma+1] int32
    residual: Optional[torch.Tensor]    # [B, V] float32
    status: torch.Tensor                # [B] int32
    node_accept: Optional[torch.Tensor] = None
    node_bonus: Optional[torch.Tensor] = None
    node_ratio: Optional[torch.Tensor] = None
    path_nodes: Optional[torch.Tensor] = None  # [B, gamma+1] tree nodes of the accepted tokens, -1 padded
    node_residual: Optional[torch.Tensor] = None  # [B, n_nodes, V] float32; rows of nodes that cannot end a walk are NaN


class Verifier:
    """Holds the descriptor and device buffers for one (batch, tree, vocab, dtype) shape so that
    repeated calls allocate nothing."""

    def __init__(self, batch: int, parent, vocab: int, dtype: torch.dtype, device="cuda", *,
                 want_residual: bool = True, node_outputs: bool = False, ld_target: Optional[int] = None,
                 ld_draft: Optional[int] = None, node_residual: bool = False):
        self.lib = load_library()
        self.parent = np.ascontiguousarray(parent, dtype=np.int32)
        self.device = torch.device(device)
        self.batch, self.vocab, self.dtype = int(batch), int(vocab), dtype
        self.n_nodes = int(self.parent.shape[0])
        self.n_internal = _n_internal(self.parent)
        gamma = self.lib.mcsd_tree_depth(self.parent.ctypes.data, self.n_nodes)
        _check(gamma if gamma < 0 else 0)
        self.gamma = gamma
        self.desc = McsdDesc()
        d = self.desc
        d.batch, d.n_nodes, d.n_internal, d.vocab = self.batch, self.n_nodes, self.n_internal, self.vocab
        d.dtype = MCSD_DTYPE[dtype]
        d.ld_target = int(ld_target if ld_target is not None else vocab)
        d.ld_draft = int(ld_draft if ld_draft is not None else vocab)
        ws = int(self.lib.mcsd_workspace_bytes(ctypes.byref(d)))
        if ws == 0:
            _check(-2)
        self.workspace = torch.empty(ws + 256, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        d.workspace = (base + 255) // 256 * 256
        d.workspace_bytes = ws
        i32 = dict(dtype=torch.int32, device=self.device)
        self.accept_len = torch.empty(self.batch, **i32)
        self.tokens = torch.empty((self.batch, self.gamma + 1), **i32)
        self.residual = (torch.empty((self.batch, self.vocab), dtype=torch.float32, device=self.device)
                         if want_residual else None)
        self.status = torch.zeros(self.batch, **i32)
        d.out_status = self.status.data_ptr()
        self.path_nodes = torch.empty((self.batch, self.gamma + 1), **i32)
        d.out_path_nodes = self.path_nodes.data_ptr()
        self.node_accept = self.node_bonus = self.node_ratio = None
        if node_outputs:
            self.node_accept = torch.empty((self.batch, self.n_nodes), **i32)
            self.node_bonus = torch.empty((self.batch, self.n_nodes), **i32)
            self.node_ratio = torch.full((self.batch, self.n_nodes), float("nan"), dtype=torch.float32,
                                         device=self.device)
            d.node_accept = self.node_accept.data_ptr()
            d.node_bonus = self.node_bonus.data_ptr()
            d.node_ratio = self.node_ratio.data_ptr()
        self.node_residual = None
        if node_residual:   # a debugging output: B * n_nodes * V floats
            self.node_residual = torch.full((self.batch, self.n_nodes, self.vocab), float("nan"), dtype=torch.float32,
                                            device=self.device)
            d.node_residual = self.node_residual.data_ptr()

    def _bind(self, target, draft):
        assert target.dtype == self.dtype and target.shape == (self.batch, self.n_nodes, self.vocab)
        self.desc.ld_target = _row_stride(target)
        if draft is not None:
            assert draft.dtype == self.dtype and draft.shape == (self.batch, self.n_internal, self.vocab)
            self.desc.ld_draft = _row_stride(draft) if self.n_internal else self.vocab
        self.desc.stream = torch.cuda.current_stream(self.device).cuda_stream

    def _out(self) -> VerifyOutput:
        return VerifyOutput(self.accept_len, self.tokens, self.residual, self.status, self.node_accept,
                            self.node_bonus, self.node_ratio, self.path_nodes, self.node_residual)

    def mcsd_verify(self, target, draft, cand, unif, temperature: float, mode: int) -> VerifyOutput:
        self._bind(target, draft)
        if self.node_ratio is not None:
            self.node_ratio.fill_(float("nan"))
        _check(self.lib.mcsd_verify(ctypes.byref(self.desc), _ptr(target), _ptr(draft), self.parent.ctypes.data,
                                    _ptr(cand), _ptr(unif), float(temperature), int(mode),
                                    _ptr(self.accept_len), _ptr(self.tokens), _ptr(self.residual)))
        return self._out()

    def mcsd_verify_path(self, target, draft, cand, unif, temperature: float, mode: int) -> VerifyOutput:
        """Level-by-level form: only the nodes the walks visit are evaluated (see mcsd.h)."""
        self._bind(target, draft)
        if self.node_ratio is not None:
            self.node_ratio.fill_(float("nan"))
        _check(self.lib.mcsd_verify_path(ctypes.byref(self.desc), _ptr(target), _ptr(draft),
                                         self.parent.ctypes.data, _ptr(cand), _ptr(unif), float(temperature),
                                         int(mode), _ptr(self.accept_len), _ptr(self.tokens), _ptr(self.residual)))
        return self._out()

    def mcsd_verify_static(self, target, draft, cand, unif, temperature: float, mode: int) -> VerifyOutput:
        """The same call with the library's built-in scratch array instead of this object's
        workspace (for callers that may not allocate device memory); see mcsd.h for its limit."""
        self._bind(target, draft)
        if self.node_ratio is not None:
            self.node_ratio.fill_(float("nan"))
        _check(self.lib.mcsd_verify_static(ctypes.byref(self.desc), _ptr(target), _ptr(draft),
                                           self.parent.ctypes.data, _ptr(cand), _ptr(unif), float(temperature),
                                           int(mode), _ptr(self.accept_len), _ptr(self.tokens),
                                           _ptr(self.residual)))
        return self._out()

    def mcsd_verify_nodes(self, target, draft, cand, unif, temperature: float, mode: int) -> None:
        self._bind(target, draft)
        _check(self.lib.mcsd_verify_nodes(ctypes.byref(self.desc), _ptr(target), _ptr(draft),
                                          self.parent.ctypes.data, _ptr(cand), _ptr(unif), float(temperature),
                                          int(mode)))

    def mcsd_verify_walk(self, target, draft, cand, unif, temperature: float) -> VerifyOutput:
        self._bind(target, draft)
        _check(self.lib.mcsd_verify_walk(ctypes.byref(self.desc), _ptr(target), _ptr(draft),
                                         self.parent.ctypes.data, _ptr(cand), _ptr(unif), float(temperature),
                                         _ptr(self.accept_len), _ptr(self.tokens), _ptr(self.residual)))
        return self._out()


def mcsd_verify(target, draft, parent, cand, unif, temperature: float, mode: int, *,
                want_residual: bool = True, node_outputs: bool = False) -> VerifyOutput:
    """One-shot convenience wrapper: device tensors in, device tensors out."""
    B, _, V = target.shape
    v = Verifier(B, parent, V, target.dtype, target.device, want_residual=want_residual,
                 node_outputs=node_outputs)
    return v.mcsd_verify(target, draft, cand, unif, temperature, mode)


def mcsd_tree_attention_layout(parent, prefix_len: int, device="cuda"):
    """Ancestor-only attention mask [n, n] (uint8) and position ids [n] (int32) of the flattened tree."""
    lib = load_library()
    parent = np.ascontiguousarray(parent, dtype=np.int32)
    n = int(parent.shape[0])
    mask = torch.empty((n, n), dtype=torch.uint8, device=device)
    pos = torch.empty(n, dtype=torch.int32, device=device)
    _check(lib.mcsd_tree_attention_layout(parent.ctypes.data, n, int(prefix_len), _ptr(mask), _ptr(pos),
                                          torch.cuda.current_stream(torch.device(device)).cuda_stream))
    return mask, pos


def mcsd_gather_accepted_kv(cache: torch.Tensor, prefix_len: torch.Tensor, path_nodes: torch.Tensor,
                            accept_len: torch.Tensor) -> torch.Tensor:
    """Moves, in place, the cache rows of the accepted path to their committed positions (see mcsd.h).
    cache: device tensor [slabs, batch, positions, ...] whose trailing dimensions form one contiguous row;
    prefix_len, accept_len: int32 [batch]; path_nodes: int32 [batch, gamma + 1].  Returns cache."""
    lib = load_library()
    assert cache.dim() >= 4 and cache.is_cuda
    S, B, L = cache.shape[:3]
    row = cache[0, 0, 0]
    assert row.is_contiguous(), "the trailing dimensions must form one contiguous row"
    es = cache.element_size()
    assert path_nodes.dtype == torch.int32 and path_nodes.is_contiguous() and path_nodes.shape[0] == B
    assert prefix_len.dtype == torch.int32 and accept_len.dtype == torch.int32
    gamma = int(path_nodes.shape[1]) - 1
    _check(lib.mcsd_gather_accepted_kv(cache.data_ptr(), S, cache.stride(0) * es, B, cache.stride(1) * es,
                                       cache.stride(2) * es, row.numel() * es, L, _ptr(prefix_len),
                                       _ptr(path_nodes), _ptr(accept_len), gamma,
                                       torch.cuda.current_stream(cache.device).cuda_stream))
    return cache


def mcsd_sample_candidates(draft, parent, unif_draw, temperature: float, mode: int, *, node_begin: int = 0,
                           node_end: Optional[int] = None, cand: Optional[torch.Tensor] = None,
                           status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Candidate tokens of the children of nodes [node_begin, node_end): device tensors in, the
    [B, n_nodes] int32 token tensor out (entries outside the range keep their value, -1 if new)."""
    lib = load_library()
    parent = np.ascontiguousarray(parent, dtype=np.int32)
    B, n_internal, V = draft.shape
    n_nodes = int(parent.shape[0])
    d = McsdDesc()
    d.batch, d.n_nodes, d.n_internal, d.vocab = B, n_nodes, n_internal, V
    d.dtype = MCSD_DTYPE[draft.dtype]
    d.ld_target = V
    d.ld_draft = _row_stride(draft) if n_internal else V
    d.stream = torch.cuda.current_stream(draft.device).cuda_stream
    d.out_status = _ptr(status)
    if cand is None:
        cand = torch.full((B, n_nodes), -1, dtype=torch.int32, device=draft.device)
    _check(lib.mcsd_sample_candidates(ctypes.byref(d), _ptr(draft), parent.ctypes.data, _ptr(unif_draw),
                                      float(temperature), int(mode), int(node_begin),
                                      int(n_internal if node_end is None else node_end), _ptr(cand)))
    return cand


def mcsd_verify_host(target, draft, parent, cand, unif, temperature: float, mode: int, *,
                     want_residual: bool = True, out: Optional[dict] = None) -> VerifyOutput:
    """Host tensors (CPU, ideally pinned) in, host tensors out; all copies happen inside the library."""
    lib = load_library()
    parent = np.ascontiguousarray(parent, dtype=np.int32)
    B, n_nodes, V = target.shape
    assert not target.is_cuda and target.is_contiguous()
    d = McsdDesc()
    d.batch, d.n_nodes, d.n_internal, d.vocab = B, n_nodes, _n_internal(parent), V
    d.dtype = MCSD_DTYPE[target.dtype]
    d.ld_target = V
    d.ld_draft = V
    gamma = lib.mcsd_tree_depth(parent.ctypes.data, n_nodes)
    _check(gamma if gamma < 0 else 0)
    if out is None:
        out = {}
    pin = torch.cuda.is_available()
    accept_len = out.get("accept_len", torch.empty(B, dtype=torch.int32, pin_memory=pin))
    tokens = out.get("tokens", torch.empty((B, gamma + 1), dtype=torch.int32, pin_memory=pin))
    residual = out.get("residual", torch.empty((B, V), dtype=torch.float32, pin_memory=pin)) if want_residual else None
    status = out.get("status", torch.zeros(B, dtype=torch.int32, pin_memory=pin))
    _check(lib.mcsd_verify_host(ctypes.byref(d), _ptr(target), _ptr(draft), parent.ctypes.data, _ptr(cand),
                                _ptr(unif), float(temperature), int(mode), _ptr(accept_len), _ptr(tokens),
                                _ptr(residual), _ptr(status)))
    return VerifyOutput(accept_len, tokens, residual, status)


# ---------------------------------------------------------------- the steps around the verification
class _on_device:
    """Makes the device of a tensor current for a call (the library works on the current device); gives the raw
    handle of the device's current stream."""

    __slots__ = ("index", "guard")

    def __init__(self, device: torch.device):
        self.index, self.guard = device.index, None

    def __enter__(self):
        current = torch._C._cuda_getDevice()
        if self.index is not None and self.index != current:
            self.guard, current = torch.cuda.device(self.index), self.index
            self.guard.__enter__()
        return torch._C._cuda_getCurrentRawStream(current)

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _device_tensor(t: Optional[torch.Tensor], dtype, shape, device, name: str, contiguous: bool = True):
    """The tensor (or None), once its device, type, shape and layout are what a call needs."""
    if t is None:
        return None
    assert t.device == device, f"{name} must be on {device}"
    assert t.dtype is dtype, f"{name} must be {dtype}"
    assert shape is None or t.shape == shape, f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}"
    assert not contiguous or t.is_contiguous(), f"{name} must be contiguous"
    return t


def _settle(device: torch.device) -> None:
    """Waits until what was enqueued for new buffers (their fill, and what used their memory before) is done, so that
    the first call that uses them may be on any stream.  (In a capture they belong to its graph: nothing to wait for.)"""
    if not torch.cuda.is_current_stream_capturing():
        torch.cuda.current_stream(device).synchronize()


class LogitRules:
    """The rules of mcsd_apply_logit_rules (see mcsd.h); every argument is a device tensor or None.
    history [B, H] int32 with unit stride along a row; history_len, prompt_len [B] int32; repetition, frequency,
    presence [B] float32; bias_ids [B, K] int32 with bias_values [B, K] float32; masks [M, words] int32 with unit
    stride along a row; mask_index [B, n_nodes] int32.  The tensors are kept and may change between calls."""

    def __init__(self, *, history=None, history_len=None, prompt_len=None, repetition=None, frequency=None, presence=None,
                 bias_ids=None, bias_values=None, masks=None, mask_index=None):
        given = [t for t in (history, repetition, frequency, presence, bias_ids, masks) if t is not None]
        self.tensors = (history, history_len, prompt_len, repetition, frequency, presence, bias_ids, bias_values, masks, mask_index)
        self.device = given[0].device if given else None
        self.batch = next((t.shape[0] for t in (history, repetition, frequency, presence, bias_ids) if t is not None), None)
        r = self.desc = McsdLogitRules()
        B, dev = self.batch, self.device
        if history is not None:
            assert history.dim() == 2 and (history.shape[1] <= 1 or history.stride(1) == 1), "history rows must be contiguous"
            assert history_len is not None, "history needs history_len"
            _device_tensor(history, torch.int32, None, dev, "history", contiguous=False)
            r.history = history.data_ptr()
            r.n_history = int(history.shape[1])
            r.ld_history = int(history.stride(0)) if history.shape[0] > 1 else r.n_history
        r.history_len = _ptr(_device_tensor(history_len, torch.int32, (B,), dev, "history_len"))
        r.prompt_len = _ptr(_device_tensor(prompt_len, torch.int32, (B,), dev, "prompt_len"))
        r.repetition = _ptr(_device_tensor(repetition, torch.float32, (B,), dev, "repetition"))
        r.frequency = _ptr(_device_tensor(frequency, torch.float32, (B,), dev, "frequency"))
        r.presence = _ptr(_device_tensor(presence, torch.float32, (B,), dev, "presence"))
        if bias_ids is not None:
            assert bias_values is not None and bias_ids.shape == bias_values.shape
            r.n_bias = int(bias_ids.shape[1])
            if r.n_bias:
                r.bias_ids = _ptr(_device_tensor(bias_ids, torch.int32, (B, r.n_bias), dev, "bias_ids"))
                r.bias_values = _ptr(_device_tensor(bias_values, torch.float32, (B, r.n_bias), dev, "bias_values"))
        self.mask_index = mask_index
        if masks is not None:
            assert masks.dim() == 2 and (masks.shape[1] <= 1 or masks.stride(1) == 1), "mask rows must be contiguous"
            _device_tensor(masks, torch.int32, None, dev, "masks", contiguous=False)
            r.masks, r.n_masks = masks.data_ptr(), int(masks.shape[0])
            r.ld_mask = int(masks.stride(0)) if masks.shape[0] > 1 else int(masks.shape[1])
            self.mask_words = int(masks.shape[1])
            if mask_index is not None:
                _device_tensor(mask_index, torch.int32, None, dev, "mask_index")
                r.mask_index = mask_index.data_ptr()


def mcsd_apply_logit_rules(logits: torch.Tensor, parent, cand: Optional[torch.Tensor], rules: LogitRules, *,
                           out: Optional[torch.Tensor] = None, node_begin: int = 0, node_end: Optional[int] = None,
                           status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Applies the rules to rows [node_begin, node_end) of logits [B, rows, V] (rows: n_nodes for target logits, n_internal
    for draft logits).  out=None works in place; returns the tensor written."""
    lib = load_library()
    parent = np.ascontiguousarray(parent, dtype=np.int32)
    assert logits.is_cuda and logits.dim() == 3
    (B, rows, V), device = logits.shape, logits.device
    n_nodes = int(parent.shape[0])
    out = logits if out is None else out
    assert out is logits or (out.shape == logits.shape and out.dtype is logits.dtype and out.device == device)
    assert rules.device is None or rules.device == device
    assert rules.batch is None or rules.batch == B, "the rules are for another batch size"
    if rules.mask_index is not None:
        assert tuple(rules.mask_index.shape) == (B, n_nodes)
    elif rules.desc.masks:
        assert rules.desc.n_masks >= B * n_nodes, "masks without mask_index hold a row per node"
    assert not rules.desc.masks or rules.mask_words >= (V + 31) // 32, "mask rows are too short for the vocabulary"
    _device_tensor(cand, torch.int32, (B, n_nodes), device, "cand")
    _device_tensor(status, torch.int32, (B,), device, "status")
    d = McsdDesc()
    d.batch, d.n_nodes, d.vocab, d.dtype, d.out_status = B, n_nodes, V, MCSD_DTYPE[logits.dtype], _ptr(status)
    with _on_device(logits.device) as stream:
        d.stream = stream
        rc = lib.mcsd_apply_logit_rules(d, rules.desc, parent.ctypes.data, _ptr(cand), logits.data_ptr(),
                                        _row_stride(logits) if rows else V, out.data_ptr(), _row_stride(out) if rows else V,
                                        rows, node_begin, rows if node_end is None else node_end)
    _check(rc)
    return out


class PageTables:
    """Page tables of a batch and the ring of free pages behind them (see mcsd.h): holds the descriptor, so that a
    step allocates nothing.  table [B, max_pages] int32, held [B] int32, ring [capacity] int32, ring_state [4] int32
    (head, free pages, 0, 0).  Without held_out and ring_state_out the state is advanced in place."""

    def __init__(self, table, held, ring, ring_state, page_size: int, *, held_out=None, ring_state_out=None):
        self.lib = load_library()
        dev, (B, W) = table.device, table.shape
        assert table.is_cuda and table.dtype == torch.int32 and (W <= 1 or table.stride(1) == 1)
        _device_tensor(held, torch.int32, (B,), dev, "held")
        _device_tensor(ring, torch.int32, None, dev, "ring")
        _device_tensor(ring_state, torch.int32, (4,), dev, "ring_state")
        _device_tensor(held_out, torch.int32, (B,), dev, "held_out")
        _device_tensor(ring_state_out, torch.int32, (4,), dev, "ring_state_out")
        self.device, self.batch, self.page_size = dev, B, int(page_size)
        self.table, self.held, self.ring, self.ring_state = table, held, ring, ring_state
        self.held_out = held if held_out is None else held_out
        self.ring_state_out = ring_state if ring_state_out is None else ring_state_out
        self.cu_tokens = torch.empty(B + 1, dtype=torch.int32, device=dev)
        self.status = torch.empty(B, dtype=torch.int32, device=dev)
        d = self.desc = McsdPageDesc()
        d.batch, d.page_size, d.max_pages, d.ring_capacity = B, self.page_size, W, int(ring.shape[0])
        d.ld_table = int(table.stride(0)) if B > 1 else W
        d.page_table, d.held, d.ring, d.ring_state = table.data_ptr(), held.data_ptr(), ring.data_ptr(), ring_state.data_ptr()
        d.held_out, d.ring_state_out = _ptr(held_out), _ptr(ring_state_out)
        d.cu_tokens, d.status = self.cu_tokens.data_ptr(), self.status.data_ptr()

    @classmethod
    def empty(cls, batch: int, max_pages: int, n_pages: int, page_size: int, device="cuda"):
        """Tables of a batch that holds nothing yet, over a pool of n_pages free pages."""
        i32 = dict(dtype=torch.int32, device=device)
        plan = cls(torch.full((batch, max_pages), -1, **i32), torch.zeros(batch, **i32), torch.arange(n_pages, **i32),
                   torch.tensor([0, n_pages, 0, 0], **i32), page_size)
        _settle(plan.device)
        return plan

    def mcsd_build_page_tables(self, start: torch.Tensor, count, *, slots: Optional[torch.Tensor] = None):
        """start [B] int32; count: tokens per sequence, an int for all or [B] int32; slots: [n] int64, filled in packed
        order (or None).  Returns slots."""
        d = self.desc
        d.start = _ptr(_device_tensor(start, torch.int32, (self.batch,), self.device, "start"))
        if isinstance(count, torch.Tensor):
            d.count, d.new_tokens = _ptr(_device_tensor(count, torch.int32, (self.batch,), self.device, "count")), 0
        else:
            d.count, d.new_tokens = None, int(count)
        _device_tensor(slots, torch.int64, None, self.device, "slots")
        d.slots, d.n_slots = _ptr(slots), 0 if slots is None else int(slots.numel())
        with _on_device(self.device) as stream:
            d.stream = stream
            rc = self.lib.mcsd_build_page_tables(d)
        _check(rc)
        return slots


def mcsd_kv_block_bytes(head_dim: int, page_size: int) -> int:
    """Bytes of one head of one page of the 4-bit cache (0: a size that is not supported)."""
    return int(load_library().mcsd_kv_block_bytes(int(head_dim), int(page_size)))


class KvCache:
    """The paged 4-bit key/value cache of one layer, pages [n_pages, heads, block] uint8, or of several layers,
    [layers, n_pages, heads, block] (see mcsd.h for a block's layout); block = mcsd_kv_block_bytes(head_dim, page_size).
    `layer(i)` is the cache of one of several layers."""

    def __init__(self, pages: torch.Tensor, head_dim: int, page_size: int):
        self.lib = load_library()
        block = mcsd_kv_block_bytes(head_dim, page_size)
        if block == 0:
            _check(-10)
        assert pages.is_cuda and pages.dtype == torch.uint8 and pages.dim() in (3, 4) and pages.shape[-1] == block
        assert pages.stride(-1) == 1 and (pages.shape[-2] == 1 or pages.stride(-2) == block), "the heads of a page follow each other"
        self.pages, self.device, self.head_dim, self.page_size = pages, pages.device, int(head_dim), int(page_size)
        self.n_pages, self.n_heads = int(pages.shape[-3]), int(pages.shape[-2])
        self.n_layers = int(pages.shape[0]) if pages.dim() == 4 else 1
        self.layer_stride = int(pages.stride(0)) if pages.dim() == 4 else 0
        c = self.desc = McsdKvCache()
        c.pages, c.n_pages, c.n_heads = pages.data_ptr(), self.n_pages, self.n_heads
        c.page_stride = int(pages.stride(-3)) if self.n_pages > 1 else self.n_heads * block
        c.head_dim, c.page_size = self.head_dim, self.page_size

    @classmethod
    def empty(cls, n_pages: int, n_heads: int, head_dim: int, page_size: int, device="cuda", n_layers: Optional[int] = None):
        lead = (n_pages,) if n_layers is None else (n_layers, n_pages)
        block = mcsd_kv_block_bytes(head_dim, page_size)
        if block == 0:
            _check(-10)
        cache = cls(torch.zeros(lead + (n_heads, block), dtype=torch.uint8, device=device), head_dim, page_size)
        _settle(cache.device)
        return cache

    def layer(self, i: int) -> "KvCache":
        assert self.pages.dim() == 4
        return KvCache(self.pages[i], self.head_dim, self.page_size)


def _rows_args(cache: KvCache, t: Optional[torch.Tensor], n: int, name: str):
    if t is None:
        return None, 0, 0
    token, head, one = t.stride()
    assert t.device == cache.device and t.shape == (n, cache.n_heads, cache.head_dim) and one == 1, \
        f"{name} must be [tokens, heads, head_dim] with contiguous rows on the cache's device"
    return t.data_ptr(), (token if n > 1 else cache.n_heads * cache.head_dim), (head if cache.n_heads > 1 else cache.head_dim)


def mcsd_append_kv(cache: KvCache, keys: torch.Tensor, values: torch.Tensor, slots: torch.Tensor) -> None:
    """Quantises keys and values [tokens, heads, head_dim] and stores them at slots [tokens] int64 (-1: skipped)."""
    assert cache.pages.dim() == 3, "one layer at a time: cache.layer(i)"
    n = int(slots.shape[0])
    _device_tensor(slots, torch.int64, (n,), cache.device, "slots")
    assert keys.dtype == values.dtype
    k, v = _rows_args(cache, keys, n, "keys"), _rows_args(cache, values, n, "values")
    with _on_device(cache.device) as stream:
        rc = cache.lib.mcsd_append_kv(cache.desc, *k, *v, MCSD_DTYPE[keys.dtype], n, slots.data_ptr(), stream)
    _check(rc)


def mcsd_read_kv(cache: KvCache, slots: torch.Tensor, dtype: Optional[torch.dtype] = None, *, keys: Optional[torch.Tensor] = None,
                 values: Optional[torch.Tensor] = None):
    """(keys, values) [tokens, heads, head_dim] of the rows at slots; rows of slots outside the cache keep what the
    outputs hold (zeros if made here).  With neither output given both are made, in dtype."""
    assert cache.pages.dim() == 3, "one layer at a time: cache.layer(i)"
    n = int(slots.shape[0])
    _device_tensor(slots, torch.int64, (n,), cache.device, "slots")
    if keys is None and values is None:
        keys = torch.zeros((n, cache.n_heads, cache.head_dim), dtype=dtype or torch.float32, device=cache.device)
        values = torch.zeros_like(keys)
    given = (keys if keys is not None else values).dtype
    assert all(t is None or t.dtype == given for t in (keys, values))
    k, v = _rows_args(cache, keys, n, "keys"), _rows_args(cache, values, n, "values")
    with _on_device(cache.device) as stream:
        rc = cache.lib.mcsd_read_kv(cache.desc, *k, *v, MCSD_DTYPE[given], n, slots.data_ptr(), stream)
    _check(rc)
    return keys, values


@dataclass
class AttentionOutput:
    out: torch.Tensor                   # [B, n_nodes, n_heads, head_dim]
    lse: Optional[torch.Tensor]         # [B, n_nodes, n_heads] float32


class TreeAttention:
    """Attention of a draft tree over a paged 4-bit cache: holds the descriptor, the outputs and the workspace of one
    (batch, tree, heads, dtype, cache geometry) shape, so that repeated calls allocate nothing (see mcsd.h). One call at a
    time: calls that may overlap, from other threads or on other streams or in captured graphs, take an object each."""

    def __init__(self, batch: int, parent, n_heads: int, dtype: torch.dtype, cache: KvCache, max_pages: int, *, want_lse: bool = True):
        self.lib = load_library()
        self.parent = np.ascontiguousarray(parent, dtype=np.int32)
        self.device, self.dtype = cache.device, dtype
        self.batch, self.n_nodes, self.n_heads = int(batch), int(self.parent.shape[0]), int(n_heads)
        self.head_dim, self.max_pages = cache.head_dim, int(max_pages)
        self.geometry = (cache.n_heads, cache.head_dim, cache.page_size)
        rc = self.lib.mcsd_tree_depth(self.parent.ctypes.data, self.n_nodes)
        _check(rc if rc < 0 else 0)
        self.parent_ptr = self.parent.ctypes.data
        self.out = torch.zeros((self.batch, self.n_nodes, self.n_heads, self.head_dim), dtype=dtype, device=self.device)
        self.lse = torch.zeros((self.batch, self.n_nodes, self.n_heads), dtype=torch.float32, device=self.device) if want_lse else None
        d = self.desc = McsdAttentionDesc()
        d.batch, d.n_nodes, d.n_heads, d.dtype = self.batch, self.n_nodes, self.n_heads, MCSD_DTYPE[dtype]
        d.max_pages, d.ld_table = self.max_pages, self.max_pages
        d.q_seq_stride, d.q_node_stride, d.q_head_stride = self.out.stride()[:3]
        d.out_seq_stride, d.out_node_stride, d.out_head_stride = self.out.stride()[:3]
        with _on_device(self.device):                # (the size goes by the device that the calls will run on)
            ws = int(self.lib.mcsd_tree_attention_workspace_bytes(ctypes.byref(d), ctypes.byref(cache.desc)))
        if ws == 0:
            _check(self.lib.mcsd_tree_attention(ctypes.byref(d), ctypes.byref(cache.desc), None, None, self.parent.ctypes.data,
                                                None, None, None))
            _check(-2)
        self.workspace = torch.empty(ws + 256, dtype=torch.uint8, device=self.device)
        d.workspace = (self.workspace.data_ptr() + 255) // 256 * 256
        d.workspace_bytes = ws
        _settle(self.device)

    def mcsd_tree_attention(self, q: torch.Tensor, cache: KvCache, page_table: torch.Tensor, prefix_len: torch.Tensor, *,
                            scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> AttentionOutput:
        """q [B, n_nodes, n_heads, head_dim] with contiguous rows; page_table [B, max_pages] int32; prefix_len [B] int32;
        scale: 1 / sqrt(head_dim) if None.  out: a tensor like q to write to instead of this object's."""
        d, shape = self.desc, (self.batch, self.n_nodes, self.n_heads, self.head_dim)
        out = self.out if out is None else out
        assert cache.pages.dim() == 3, "one layer at a time: cache.layer(i)"
        assert cache.device == self.device and self.geometry == (cache.n_heads, cache.head_dim, cache.page_size)
        qs, os_ = q.stride(), out.stride()
        assert q.device == self.device and q.dtype is self.dtype and q.shape == shape and qs[3] == 1
        assert out is self.out or (out.device == self.device and out.dtype is self.dtype and out.shape == shape and os_[3] == 1)
        _device_tensor(page_table, torch.int32, (self.batch, self.max_pages), self.device, "page_table", contiguous=False)
        assert self.max_pages <= 1 or page_table.stride(1) == 1
        _device_tensor(prefix_len, torch.int32, (self.batch,), self.device, "prefix_len")
        d.ld_table = int(page_table.stride(0)) if self.batch > 1 else self.max_pages
        d.q_seq_stride, d.q_node_stride, d.q_head_stride, _ = qs
        d.out_seq_stride, d.out_node_stride, d.out_head_stride, _ = os_
        d.scale = float(scale) if scale is not None else self.head_dim ** -0.5
        with _on_device(self.device) as stream:
            d.stream = stream
            rc = self.lib.mcsd_tree_attention(d, cache.desc, page_table.data_ptr(), prefix_len.data_ptr(), self.parent_ptr,
                                              q.data_ptr(), out.data_ptr(), _ptr(self.lse))
        _check(rc)
        return AttentionOutput(out, self.lse)


def mcsd_gather_accepted_pages(cache: KvCache, page_table: torch.Tensor, prefix_len: torch.Tensor, path_nodes: torch.Tensor,
                               accept_len: torch.Tensor) -> torch.Tensor:
    """mcsd_gather_accepted_kv for the paged cache, all its layers in one launch; in place, returns cache.pages.
    page_table [B, max_pages], path_nodes [B, gamma + 1], prefix_len and accept_len [B], all int32."""
    B, W = page_table.shape
    _device_tensor(page_table, torch.int32, None, cache.device, "page_table", contiguous=False)
    assert W <= 1 or page_table.stride(1) == 1
    _device_tensor(prefix_len, torch.int32, (B,), cache.device, "prefix_len")
    _device_tensor(accept_len, torch.int32, (B,), cache.device, "accept_len")
    _device_tensor(path_nodes, torch.int32, (B, path_nodes.shape[1]), cache.device, "path_nodes")
    with _on_device(cache.device) as stream:
        rc = cache.lib.mcsd_gather_accepted_pages(
            cache.desc, cache.n_layers, cache.layer_stride, page_table.data_ptr(), page_table.stride(0) if B > 1 else W, W, B,
            prefix_len.data_ptr(), path_nodes.data_ptr(), accept_len.data_ptr(), path_nodes.shape[1] - 1, stream)
    _check(rc)
    return cache.pages


# ---------------------------------------------------------------- prompts and long conversations
class ChunkAttention:
    """Attention of a chunk of new tokens of every sequence over a paged 4-bit cache, and the weight that the cached rows
    gather of it (see mcsd.h): holds the descriptor, the outputs and the workspace of one (batch, heads, dtype, cache geometry) shape and
    up to max_tokens tokens, so that repeated calls allocate nothing. max_new: tokens that a sequence has at most (max_tokens if
    None); the fewer, the better the kernels fit. One call at a time: calls that may overlap, from other threads or on other streams or
    in captured graphs, take an object each."""

    def __init__(self, batch: int, max_tokens: int, n_heads: int, dtype: torch.dtype, cache: KvCache, max_pages: int, *,
                 max_new: Optional[int] = None, want_lse: bool = True):
        self.lib = load_library()
        self.device, self.dtype = cache.device, dtype
        self.batch, self.max_tokens, self.n_heads = int(batch), int(max_tokens), int(n_heads)
        self.max_new = self.max_tokens if max_new is None else int(max_new)
        self.head_dim, self.max_pages = cache.head_dim, int(max_pages)
        self.geometry = (cache.n_heads, cache.head_dim, cache.page_size)
        self.out = torch.zeros((self.max_tokens, self.n_heads, self.head_dim), dtype=dtype, device=self.device)
        self.lse = torch.zeros((self.max_tokens, self.n_heads), dtype=torch.float32, device=self.device) if want_lse else None
        d = self.desc = McsdChunkDesc()
        d.batch, d.n_heads, d.dtype, d.max_pages, d.max_new = self.batch, self.n_heads, MCSD_DTYPE[dtype], self.max_pages, self.max_new
        d.ld_table, d.n_tokens, d.scale = self.max_pages, self.max_tokens, 1.0
        d.q_token_stride, d.q_head_stride = d.out_token_stride, d.out_head_stride = self.out.stride()[:2]
        with _on_device(self.device):                # (the size goes by the device that the calls will run on)
            ws = int(self.lib.mcsd_chunk_attention_workspace_bytes(d, cache.desc))
        if ws == 0:
            _check(self.lib.mcsd_chunk_attention(d, cache.desc, None, None, None, None, None, None))
            _check(-2)
        self.workspace = torch.empty(ws + 256, dtype=torch.uint8, device=self.device)
        d.workspace = (self.workspace.data_ptr() + 255) // 256 * 256
        d.workspace_bytes = ws
        _settle(self.device)

    def _bind(self, q, cache, page_table, start, cu_tokens, scale):
        """The arguments that both calls share, checked and put into the descriptor; returns it."""
        d = self.desc
        assert cache.pages.dim() == 3, "one layer at a time: cache.layer(i)"
        assert cache.device == self.device and self.geometry == (cache.n_heads, cache.head_dim, cache.page_size)
        T = q.shape[0]
        assert q.device == self.device and q.dtype is self.dtype and T <= self.max_tokens and q.shape[1:] == (self.n_heads, self.head_dim), \
            "q must be [tokens, heads, head_dim] of this object's type and device, with at most max_tokens tokens"
        assert q.stride(2) == 1, "rows of q must be contiguous"
        _device_tensor(page_table, torch.int32, (self.batch, self.max_pages), self.device, "page_table", contiguous=False)
        assert self.max_pages <= 1 or page_table.stride(1) == 1
        _device_tensor(start, torch.int32, (self.batch,), self.device, "start")
        _device_tensor(cu_tokens, torch.int32, (self.batch + 1,), self.device, "cu_tokens")
        d.ld_table = int(page_table.stride(0)) if self.batch > 1 else self.max_pages
        d.n_tokens, d.q_token_stride, d.q_head_stride = T, q.stride(0), q.stride(1)
        d.scale = float(scale) if scale is not None else self.head_dim ** -0.5
        return d

    def mcsd_chunk_attention(self, q: torch.Tensor, cache: KvCache, page_table: torch.Tensor, start: torch.Tensor, cu_tokens: torch.Tensor, *,
                             scale: Optional[float] = None, out: Optional[torch.Tensor] = None) -> AttentionOutput:
        """q [tokens, n_heads, head_dim] with contiguous rows, packed by sequence; page_table [B, max_pages], start [B] and cu_tokens
        [B + 1] int32 (PageTables has them); scale: 1 / sqrt(head_dim) if None. out: a tensor like q to write to instead of
        this object's. Returns out and lse [tokens, n_heads]."""
        d = self._bind(q, cache, page_table, start, cu_tokens, scale)
        T = q.shape[0]
        out = self.out[:T] if out is None else out
        assert out.device == self.device and out.dtype is self.dtype and out.shape == q.shape and out.stride(2) == 1
        lse = None if self.lse is None else self.lse[:T]
        d.out_token_stride, d.out_head_stride = out.stride(0), out.stride(1)
        with _on_device(self.device) as stream:
            d.stream = stream
            rc = self.lib.mcsd_chunk_attention(d, cache.desc, page_table.data_ptr(), start.data_ptr(), cu_tokens.data_ptr(),
                                               q.data_ptr(), out.data_ptr(), _ptr(lse))
        _check(rc)
        return AttentionOutput(out, lse)

    def mcsd_accumulate_weights(self, q: torch.Tensor, lse: torch.Tensor, cache: KvCache, page_table: torch.Tensor, start: torch.Tensor,
                                cu_tokens: torch.Tensor, weights: torch.Tensor, *, scale: Optional[float] = None, decay: float = 1.0,
                                last_tokens: int = 0) -> torch.Tensor:
        """Adds what the last last_tokens new tokens of every sequence (0: all) give to each cached row to weights
        [n_pages, heads, page_size] float32, in place (rows from before are multiplied by decay first); lse [tokens, n_heads] as
        mcsd_chunk_attention returned it, the other arguments as there. No two sequences with new tokens may share a page. Returns weights."""
        d = self._bind(q, cache, page_table, start, cu_tokens, scale)
        _device_tensor(lse, torch.float32, (q.shape[0], self.n_heads), self.device, "lse")
        _device_tensor(weights, torch.float32, (cache.n_pages, cache.n_heads, cache.page_size), self.device, "weights")
        with _on_device(self.device) as stream:
            d.stream = stream
            rc = self.lib.mcsd_accumulate_weights(d, cache.desc, page_table.data_ptr(), start.data_ptr(), cu_tokens.data_ptr(), q.data_ptr(),
                                                  lse.data_ptr(), weights.data_ptr(), float(decay), int(last_tokens))
        _check(rc)
        return weights


def mcsd_evict_rows(cache: KvCache, weights: torch.Tensor, page_table: torch.Tensor, length: torch.Tensor, keep, *, sink: int = 0, recent: int = 0,
                    len_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Cuts sequences of `length` [B] int32 cached rows down to `keep` (an int for all, or [B] int32, negative: left alone): every
    head of every layer keeps its first `sink` rows, its last `recent` ones and the heaviest of the others, moved to the front in
    order, in place. weights float32 [n_pages, heads, page_size], with a leading [layers] where the cache has several. Returns the
    lengths afterwards (len_out if given)."""
    B, W = page_table.shape
    dev, layers = cache.device, cache.pages.dim() == 4
    _device_tensor(page_table, torch.int32, None, dev, "page_table", contiguous=False)
    assert W <= 1 or page_table.stride(1) == 1
    _device_tensor(length, torch.int32, (B,), dev, "length")
    _device_tensor(len_out, torch.int32, (B,), dev, "len_out")
    shape = (cache.n_pages, cache.n_heads, cache.page_size)
    _device_tensor(weights, torch.float32, ((cache.n_layers,) if layers else ()) + shape, dev, "weights")
    len_out = torch.empty_like(length) if len_out is None else len_out
    d = McsdEvictDesc()
    d.batch, d.max_pages, d.sink, d.recent = B, W, int(sink), int(recent)
    if isinstance(keep, torch.Tensor):
        d.keep_len = _device_tensor(keep, torch.int32, (B,), dev, "keep").data_ptr()
    else:
        d.keep = int(keep)
    d.n_layers, d.layer_stride, d.weight_stride = cache.n_layers, cache.layer_stride, shape[0] * shape[1] * shape[2]
    d.ld_table = page_table.stride(0) if B > 1 else W
    d.page_table, d.len, d.weights, d.len_out = page_table.data_ptr(), length.data_ptr(), weights.data_ptr(), len_out.data_ptr()
    with _on_device(dev) as stream:
        d.stream = stream
        rc = cache.lib.mcsd_evict_rows(d, cache.desc)
    _check(rc)
    return len_out


@dataclass
class LogprobOutput:
    logprobs: torch.Tensor                  # like the tokens, float32
    entropy: Optional[torch.Tensor]         # [rows] (or [B, gamma + 1]) float32
    top_ids: torch.Tensor                   # [rows, n_top] int32 (or [B, gamma + 1, n_top])
    top_logprobs: torch.Tensor              # the same, float32


class TokenLogprobs:
    """Log probabilities of given tokens, the entropy and the n_top largest tokens of rows of logits (see mcsd.h): holds the outputs of
    up to max_rows rows, so that repeated calls allocate nothing (one call at a time). Entries that a call does not write keep what
    they hold, 0 at first."""

    def __init__(self, max_rows: int, vocab: int, dtype: torch.dtype, *, n_given: int = 1, n_top: int = 0, want_entropy: bool = True, device="cuda"):
        self.lib = load_library()
        self.max_rows, self.vocab, self.dtype, self.n_given, self.n_top = int(max_rows), int(vocab), dtype, int(n_given), int(n_top)
        f32 = dict(dtype=torch.float32, device=device)
        self.logprobs = torch.zeros((self.max_rows, self.n_given), **f32)
        self.device = self.logprobs.device
        self.entropy = torch.zeros(self.max_rows, **f32) if want_entropy else None
        self.top_ids = torch.zeros((self.max_rows, self.n_top), dtype=torch.int32, device=device)
        self.top_logprobs = torch.zeros((self.max_rows, self.n_top), **f32)
        d = self.desc = McsdLogprobDesc()
        d.vocab, d.dtype, d.n_given, d.n_top = self.vocab, MCSD_DTYPE[dtype], self.n_given, self.n_top
        d.logprobs, d.entropy = self.logprobs.data_ptr(), _ptr(self.entropy)
        d.top_ids, d.top_logprobs = (self.top_ids.data_ptr(), self.top_logprobs.data_ptr()) if self.n_top else (None, None)
        self._views = (None, None)
        _settle(self.device)

    def _call(self, rows, logits, ld, tokens, temperature, lead):
        d, n = self.desc, rows
        assert logits.device == self.device and logits.dtype is self.dtype and logits.shape[-1] == self.vocab
        assert n <= self.max_rows, f"{n} rows, but this object holds {self.max_rows}"
        d.n_out, d.logits, d.tokens, d.temperature = n, logits.data_ptr(), tokens.data_ptr(), float(temperature)
        d.n_logits, d.ld = logits.numel() // self.vocab, ld
        with _on_device(self.device) as stream:
            d.stream = stream
            rc = self.lib.mcsd_token_logprobs(d)
        _check(rc)
        if self._views[0] != (lead, tokens.dim()):   # (views of the outputs, made anew when the shape changes)
            self._views = (lead, tokens.dim()), LogprobOutput(
                self.logprobs[:n].view(tokens.shape), None if self.entropy is None else self.entropy[:n].view(lead),
                self.top_ids[:n].view(lead + (self.n_top,)), self.top_logprobs[:n].view(lead + (self.n_top,)))
        return self._views[1]

    def mcsd_token_logprobs(self, logits: torch.Tensor, tokens: torch.Tensor, *, temperature: float = 1.0,
                            row_index: Optional[torch.Tensor] = None) -> LogprobOutput:
        """logits [R, V] (rows may be strided); tokens int32 [n] or [n, n_given]; row_index [n] int32: the row of the logits each output row
        reads (row i if None; one that is not there leaves its outputs alone)."""
        n = tokens.shape[0]
        assert logits.dim() == 2 and (self.vocab == 1 or logits.stride(1) == 1), "rows of logits must be contiguous"
        _device_tensor(tokens, torch.int32, (n,) if tokens.dim() == 1 and self.n_given == 1 else (n, self.n_given), self.device, "tokens")
        _device_tensor(row_index, torch.int32, (n,), self.device, "row_index")
        self.desc.row_index, self.desc.path_nodes = _ptr(row_index), None
        return self._call(n, logits, logits.stride(0) if logits.shape[0] > 1 else self.vocab, tokens, temperature, (n,))

    def mcsd_path_logprobs(self, logits: torch.Tensor, path_nodes: torch.Tensor, tokens: torch.Tensor, *, temperature: float = 1.0) -> LogprobOutput:
        """The tokens [B, gamma + 1] of verified walks (path_nodes and tokens as mcsd_verify returns them), each against the row of logits
        [B, n_nodes, V] it was drawn from; entries behind the end of a walk are left alone."""
        assert self.n_given == 1 and logits.dim() == 3 and path_nodes.dim() == 2 and path_nodes.shape[0] == logits.shape[0]
        _device_tensor(path_nodes, torch.int32, None, self.device, "path_nodes")
        _device_tensor(tokens, torch.int32, path_nodes.shape, self.device, "tokens")
        d = self.desc
        d.row_index, d.path_nodes, d.path_len, d.nodes_per_tree = None, path_nodes.data_ptr(), path_nodes.shape[1], logits.shape[1]
        return self._call(path_nodes.numel(), logits, _row_stride(logits) if logits.numel() else self.vocab, tokens, temperature, tuple(path_nodes.shape))


# ---------------------------------------------------------------- vocabulary split over several devices
def mcsd_shard_columns(vocab: int, dtype: torch.dtype, n_shards: int, shard: int):
    """(col_begin, n_cols, entries_per_shard) of one shard; host only (see mcsd.h)."""
    a, b, c = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(load_library().mcsd_shard_columns(int(vocab), MCSD_DTYPE[dtype], int(n_shards), int(shard),
                                             ctypes.addressof(a), ctypes.addressof(b), ctypes.addressof(c)))
    return a.value, b.value, c.value


class ShardedVerifier:
    """One shard of the verification with the vocabulary split over several devices: holds the
    descriptor, the workspace and the exchange buffers of its device and exposes the stage calls of
    mcsd.h under their own names (argument marshalling only).  `sharded_verify` runs a step."""

    def __init__(self, batch: int, parent, vocab: int, dtype: torch.dtype, n_shards: int, shard: int, device="cuda"):
        self.lib = load_library()
        self.parent = np.ascontiguousarray(parent, dtype=np.int32)
        self.device = torch.device(device)
        self.batch, self.vocab, self.dtype = int(batch), int(vocab), dtype
        self.n_nodes, self.n_internal = int(self.parent.shape[0]), _n_internal(self.parent)
        self.n_shards, self.shard = int(n_shards), int(shard)
        self.col_begin, self.n_cols, self.eps = mcsd_shard_columns(vocab, dtype, n_shards, shard)
        self.gamma = mcsd_tree_depth(self.parent)
        rounds = self.lib.mcsd_shard_rounds(self.parent.ctypes.data, self.n_nodes)
        _check(rounds if rounds < 0 else 0)
        self.rounds = rounds
        d = self.desc = McsdShardDesc()
        d.batch, d.n_nodes, d.n_internal, d.vocab = self.batch, self.n_nodes, self.n_internal, self.vocab
        d.dtype, d.n_shards, d.shard = MCSD_DTYPE[dtype], self.n_shards, self.shard
        d.ld_target = d.ld_draft = max(self.n_cols, 1)
        ws = int(self.lib.mcsd_shard_workspace_bytes(ctypes.byref(d)))
        if ws == 0:
            _check(-2)
        self.workspace = torch.zeros(ws + 256, dtype=torch.uint8, device=self.device)
        d.workspace = (self.workspace.data_ptr() + 255) // 256 * 256
        d.workspace_bytes = ws
        n_items = self.batch * self.n_nodes
        f32 = dict(dtype=torch.float32, device=self.device)
        i32 = dict(dtype=torch.int32, device=self.device)
        # exchanged buffers: this shard's part, and what the collective gathers from all shards
        self.part = torch.zeros((n_items, self.eps, 4), **f32)
        self.cval = torch.zeros((n_items, 2), **f32)
        self.totals = torch.zeros((self.batch, self.eps), dtype=torch.float64, device=self.device)
        self.stats_all = torch.zeros((self.n_shards, n_items, self.eps, 4), **f32)
        self.part_all = torch.zeros((self.n_shards, n_items, self.eps, 4), **f32)
        self.cval_all = torch.zeros((self.n_shards, n_items, 2), **f32)
        self.totals_all = torch.zeros((self.n_shards, self.batch, self.eps), dtype=torch.float64, device=self.device)
        self.endpoint_part = torch.full((self.batch,), -1, **i32)
        self.accept_len = torch.empty(self.batch, **i32)
        self.tokens = torch.empty((self.batch, self.gamma + 1), **i32)
        self.status = torch.zeros(self.batch, **i32)
        self.path_nodes = torch.empty((self.batch, self.gamma + 1), **i32)
        self.residual = torch.zeros((self.batch, max(self.n_cols, 1)), **f32)
        self.node_accept = torch.full((self.batch, self.n_nodes), -1, **i32)
        d.node_accept = self.node_accept.data_ptr()

    def _bind(self, target, draft):
        if self.n_cols:
            assert target.dtype == self.dtype and target.shape == (self.batch, self.n_nodes, self.n_cols)
            self.desc.ld_target = _row_stride(target)
            if self.n_internal:
                assert draft.shape == (self.batch, self.n_internal, self.n_cols)
                self.desc.ld_draft = _row_stride(draft)
        self.desc.stream = torch.cuda.current_stream(self.device).cuda_stream

    def mcsd_shard_partials(self, target, draft, cand, temperature: float, rnd: int):
        self._bind(target, draft)
        _check(self.lib.mcsd_shard_partials(ctypes.byref(self.desc), _ptr(target), _ptr(draft), self.parent.ctypes.data,
                                            _ptr(cand), float(temperature), int(rnd), _ptr(self.part), _ptr(self.cval)))

    def mcsd_shard_decide(self, cand, unif, temperature: float, mode: int, rnd: int):
        self.desc.stream = torch.cuda.current_stream(self.device).cuda_stream
        gathered = self.stats_all if rnd == 0 else self.part_all
        _check(self.lib.mcsd_shard_decide(ctypes.byref(self.desc), self.parent.ctypes.data, _ptr(cand), _ptr(unif),
                                          float(temperature), int(mode), int(rnd), _ptr(gathered), _ptr(self.cval_all)))

    def mcsd_shard_endpoint(self, target, draft, temperature: float, attempt: int):
        self._bind(target, draft)
        _check(self.lib.mcsd_shard_endpoint(ctypes.byref(self.desc), _ptr(target), _ptr(draft), self.parent.ctypes.data,
                                            float(temperature), int(attempt), _ptr(self.stats_all), _ptr(self.totals),
                                            _ptr(self.residual)))

    def mcsd_shard_finish(self, target, draft, cand, unif, temperature: float, attempt: int):
        self._bind(target, draft)
        _check(self.lib.mcsd_shard_finish(ctypes.byref(self.desc), _ptr(target), _ptr(draft), self.parent.ctypes.data,
                                          _ptr(cand), _ptr(unif), float(temperature), int(attempt), _ptr(self.stats_all),
                                          _ptr(self.totals_all), _ptr(self.accept_len), _ptr(self.tokens),
                                          _ptr(self.status), _ptr(self.path_nodes), _ptr(self.endpoint_part),
                                          _ptr(self.residual)))


    def mcsd_shard_commit(self):
        self.desc.stream = torch.cuda.current_stream(self.device).cuda_stream
        _check(self.lib.mcsd_shard_commit(ctypes.byref(self.desc), self.parent.ctypes.data, _ptr(self.endpoint_part),
                                          _ptr(self.accept_len), _ptr(self.tokens)))


class DistComm:
    """The collectives of a step over torch.distributed (NCCL between GPUs): all-gathers of a few
    floats per node and one maximum of an int32 per sequence.  No logit crosses devices."""

    def __init__(self, group=None):
        import torch.distributed as dist
        self.dist, self.group = dist, group

    def all_gather(self, shards, name_local: str, name_all: str):
        (sh,) = shards
        self.dist.all_gather_into_tensor(getattr(sh, name_all).view(-1), getattr(sh, name_local).contiguous().view(-1),
                                         group=self.group)

    def all_reduce_max(self, shards, name: str):
        (sh,) = shards
        self.dist.all_reduce(getattr(sh, name), op=self.dist.ReduceOp.MAX, group=self.group)


class LocalComm:
    """The same collectives between shard objects that live in one process (several shards on one
    device, for tests): plain copies."""

    def all_gather(self, shards, name_local: str, name_all: str):
        for dst in shards:
            for src in shards:
                getattr(dst, name_all)[src.shard].copy_(getattr(src, name_local))

    def all_reduce_max(self, shards, name: str):
        best = torch.stack([getattr(sh, name) for sh in shards]).max(dim=0).values
        for sh in shards:
            getattr(sh, name).copy_(best)


def sharded_verify(shards, targets, drafts, cand, unif, temperature: float, mode: int, comm) -> VerifyOutput:
    """One verification step over column-split logits, following the call sequence of mcsd.h.
    shards: the ShardedVerifier objects this process drives (one per rank under torch.distributed; all of
    them when several shards are emulated on one device), targets / drafts: their column slices, in the
    same order; cand, unif: replicated inputs.  Returns the outputs of the first shard; its `residual`
    holds that shard's columns of the distribution."""
    T = float(temperature)
    for sh, t, d in zip(shards, targets, drafts):
        sh.mcsd_shard_partials(t, d, cand, T, 0)
    comm.all_gather(shards, "part", "stats_all")
    comm.all_gather(shards, "cval", "cval_all")
    for sh in shards:
        sh.mcsd_shard_decide(cand, unif, T, mode, 0)
    for rnd in range(1, shards[0].rounds + 1):
        for sh, t, d in zip(shards, targets, drafts):
            sh.mcsd_shard_partials(t, d, cand, T, rnd)
        comm.all_gather(shards, "part", "part_all")
        for sh in shards:
            sh.mcsd_shard_decide(cand, unif, T, mode, rnd)
    for attempt in (0, 1):
        for sh, t, d in zip(shards, targets, drafts):
            sh.mcsd_shard_endpoint(t, d, T, attempt)
        comm.all_gather(shards, "totals", "totals_all")
        for sh, t, d in zip(shards, targets, drafts):
            sh.mcsd_shard_finish(t, d, cand, unif, T, attempt)
    comm.all_reduce_max(shards, "endpoint_part")
    for sh in shards:
        sh.mcsd_shard_commit()
    sh = shards[0]
    return VerifyOutput(sh.accept_len, sh.tokens, sh.residual, sh.status, node_accept=sh.node_accept,
                        path_nodes=sh.path_nodes)
