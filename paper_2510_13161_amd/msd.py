"""Python binding of libmsd.so (include/msd.h): argument marshalling only.

Every step of the verification pass runs in the library's HIP kernels; this
module converts torch tensors into pointers and checks status codes. PyTorch
provides device memory and streams. If the library is not built the import
of any entry point raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, List, Optional, Sequence

import torch  # the HIP runtime libmsd.so binds to is the one torch loaded

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmsd.so")

# status codes / enums (msd.h)
MSD_OK = 0
MSD_ERR_INVALID_ARG, MSD_ERR_SHAPE, MSD_ERR_CAPACITY = -1, -2, -3
MSD_ERR_UNSUPPORTED, MSD_ERR_WORKSPACE, MSD_ERR_HIP = -4, -5, -6
MSD_DEV_CAPACITY, MSD_DEV_CANDIDATE, MSD_DEV_TOKEN, MSD_DEV_PAGE = 1, 2, 4, 8
MSD_NORM_RMS, MSD_NORM_LAYER = 0, 1
MSD_ACT_SWIGLU, MSD_ACT_RELU = 0, 1
MSD_POS_ROPE, MSD_POS_LEARNED = 0, 1
MSD_GREEDY, MSD_REJECTION, MSD_MATCH = 0, 1, 2
MODES = {"greedy": MSD_GREEDY, "rejection": MSD_REJECTION, "match": MSD_MATCH}

GLOBAL_SLOTS = ["embed", "pos_embed", "final_norm.g", "final_norm.b", "lm_head"]
LAYER_SLOTS = ["attn_norm.g", "attn_norm.b", "wq", "wk", "wv", "bq", "bk", "bv", "wo", "bo",
               "mlp_norm.g", "mlp_norm.b", "w_gate", "w_up", "b_up", "w_down", "b_down"]

EXPORTED = ["msd_last_error", "msd_model_create", "msd_model_destroy", "msd_workspace_bytes",
            "msd_verify_block", "msd_early_exit_topk", "msd_accept", "msd_kv_commit",
            "msd_reuse_select", "msd_set_profile", "msd_verify_block_static",
            "msd_paged_append", "msd_paged_commit", "msd_paged_attention",
            "msd_paged_attention_workspace_bytes", "msd_sample", "msd_sample_workspace_bytes",
            "msd_verify_block_paged", "msd_verify_paged_workspace_bytes"]
MSD_STATIC_SCRATCH_BYTES = 64 << 20
MSD_ACCEPT_WS_PER_ROW = 1024  # bytes a row of the acceptance workspace (msd.h)
MSD_K_QKV, MSD_K_ATTN, MSD_K_OPROJ, MSD_K_FFN_UP, MSD_K_FFN_DOWN = 0, 1, 2, 3, 4
MSD_NEXT_BRANCH, MSD_NEXT_CONTINUE, MSD_NEXT_FRESH = 0, 1, 2
MSD_MAX_TREE_NODES = 256
MSD_KV_BF16, MSD_KV_FP8 = 0, 1
MSD_KV_SCALE_TOKENS = 16
MSD_ROPE_HALF, MSD_ROPE_INTERLEAVED = 0, 1
ROPE_LAYOUTS = {"half": MSD_ROPE_HALF, "interleaved": MSD_ROPE_INTERLEAVED}


class MsdError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"msd status {status}: {msg}")
        self.status = status


class ModelConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab",
                 "norm", "act", "pos", "has_bias", "tied_head", "max_positions")] + \
               [("rope_theta", ctypes.c_float), ("norm_eps", ctypes.c_float)]


class KVCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("status", ctypes.c_void_p), ("batch_cap", ctypes.c_int32),
                ("capacity", ctypes.c_int32)]


class Block(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("n_slots", ctypes.c_int32),
                ("tokens", ctypes.c_void_p), ("parent", ctypes.POINTER(ctypes.c_int32))]


class EERequest(ctypes.Structure):
    _fields_ = [("layer", ctypes.c_int32), ("kappa", ctypes.c_int32), ("ids", ctypes.c_void_p),
                ("logp", ctypes.c_void_p), ("ready", ctypes.c_void_p)]


class Sampling(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("temperature", ctypes.c_float),
                ("n_cand", ctypes.c_int32), ("cand_ids", ctypes.c_void_p),
                ("cand_q", ctypes.c_void_p), ("u_accept", ctypes.c_void_p),
                ("u_sample", ctypes.c_void_p), ("tol_logit", ctypes.c_float)]


class HypTree(ctypes.Structure):
    _fields_ = [("n_nodes", ctypes.c_int32), ("parent", ctypes.POINTER(ctypes.c_int32)),
                ("tokens", ctypes.c_void_p)]


class ReuseStats(ctypes.Structure):
    """Layout of msd_reuse_stats (40 bytes); keep it in a device tensor."""
    _fields_ = [("trials", ctypes.c_uint64), ("fallbacks", ctypes.c_uint64),
                ("fallbacks_tau1", ctypes.c_uint64), ("omega_trials", ctypes.c_uint64),
                ("omega_sum", ctypes.c_double)]


class PagedKV(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("k", "v", "k_scale", "v_scale", "page_table", "len", "status")] + \
               [(n, ctypes.c_int32) for n in
                ("format", "n_layers", "n_pages", "n_kv_heads", "page_size", "head_dim",
                 "batch_cap", "max_pages")]


class Rope(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("positions", ctypes.c_int32),
                ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32)]


class KVRows(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in
                ("layer_stride", "seq_stride", "row_stride", "head_stride")] + \
               [(n, ctypes.c_int32) for n in ("layer", "n_layers", "batch", "n_rows")] + \
               [("count", ctypes.c_void_p)]


class PagedAttn(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("q_seq", ctypes.c_int64), ("q_row", ctypes.c_int64),
                ("q_head", ctypes.c_int64), ("out", ctypes.c_void_p), ("out_seq", ctypes.c_int64),
                ("out_row", ctypes.c_int64), ("out_head", ctypes.c_int64),
                ("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p), ("new_seq", ctypes.c_int64),
                ("new_row", ctypes.c_int64), ("new_head", ctypes.c_int64),
                ("parent", ctypes.POINTER(ctypes.c_int32)), ("count", ctypes.c_void_p),
                ("rope", ctypes.POINTER(Rope)), ("scale", ctypes.c_float)] + \
               [(n, ctypes.c_int32) for n in ("batch", "n_slots", "n_heads", "window", "sinks")]


class SampleParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("temperature", "top_k", "top_p", "min_p")]


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build(); "
                               "there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        P, i32 = ctypes.c_void_p, ctypes.c_int32
        L.msd_last_error.restype = ctypes.c_char_p
        L.msd_last_error.argtypes = []
        L.msd_model_create.argtypes = [P, P, i32, P]
        L.msd_model_destroy.argtypes = [P]
        L.msd_model_destroy.restype = None
        L.msd_workspace_bytes.argtypes = [P, i32, i32, i32, i32]
        L.msd_workspace_bytes.restype = ctypes.c_size_t
        L.msd_verify_block.argtypes = [P, P, P, P, P, P, P, P, ctypes.c_size_t, P]
        L.msd_verify_block_static.argtypes = [P, P, P, P, P, P, P, P]
        L.msd_early_exit_topk.argtypes = [P, P, i32, i32, P, P, P, ctypes.c_size_t, P]
        L.msd_accept.argtypes = [P, P, P, P, P, P, P, P, P, P, P, ctypes.c_size_t, P]
        L.msd_kv_commit.argtypes = [P, P, P, P, P, P]
        L.msd_set_profile.argtypes = [P, i32, P, P, i32]
        L.msd_reuse_select.argtypes = [P, P, P, P, P, P, P, P, P, i32, P, P, P, P, P]
        L.msd_paged_append.argtypes = [P, P, P, P]
        L.msd_paged_commit.argtypes = [P, P, P, P, P, P]
        L.msd_paged_attention.argtypes = [P, i32, P, P, ctypes.c_size_t, P]
        L.msd_paged_attention_workspace_bytes.argtypes = [P, i32, i32, i32]
        L.msd_paged_attention_workspace_bytes.restype = ctypes.c_size_t
        L.msd_verify_block_paged.argtypes = [P, P, P, P, P, P, i32, i32, P, P, P, P, ctypes.c_size_t, P]
        L.msd_verify_paged_workspace_bytes.argtypes = [P, P, i32, i32, i32]
        L.msd_verify_paged_workspace_bytes.restype = ctypes.c_size_t
        L.msd_sample.argtypes = [P, ctypes.c_int64, i32, i32, P, P, P, P, P, P, ctypes.c_size_t, P]
        L.msd_sample_workspace_bytes.argtypes = [i32, i32]
        L.msd_sample_workspace_bytes.restype = ctypes.c_size_t
        for f in ("msd_model_create", "msd_verify_block", "msd_verify_block_static",
                  "msd_early_exit_topk", "msd_accept",
                  "msd_kv_commit", "msd_reuse_select", "msd_set_profile", "msd_paged_append",
                  "msd_paged_commit", "msd_paged_attention", "msd_sample", "msd_verify_block_paged"):
            getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


def _need(ok: bool, what: str) -> None:
    """A call whose tensors do not fit its arguments: refused before the library sees addresses."""
    if not ok:
        raise MsdError(MSD_ERR_INVALID_ARG, what)


def _typed(t: torch.Tensor, dtype, shape, what: str) -> torch.Tensor:
    _need(isinstance(t, torch.Tensor) and t.dtype == dtype and tuple(t.shape) == tuple(shape) and t.is_cuda and
          t.is_contiguous(), f"{what}: a contiguous device {dtype} tensor of shape {tuple(shape)}")
    return t


def _fits(kv, rows) -> None:
    """Rows of another head layout than the pages', or tensors of another device than the current one."""
    heads, hd = getattr(rows, "_heads", (None, kv.head_dim))
    if heads not in (None, kv.n_kv_heads) or hd != kv.head_dim:
        _need(False, "rows and pages differ in kv heads or head_dim")
    _here(kv, rows)


def _here(*structs) -> None:
    here = torch.cuda.current_device()
    for s in structs:
        if s is not None and getattr(s, "_device", here) != here:
            _need(False, "tensors of another device than the current one")


def _one_device(*tensors) -> int:
    """The device of a call's tensors (None: absent), which has to be one."""
    at = {t.get_device() for t in tensors if t is not None}
    _need(len(at) == 1 and min(at) >= 0, "tensors of several devices, or of the host")
    return at.pop()


def _nbytes(ws: torch.Tensor) -> int:
    _need(ws.get_device() == torch.cuda.current_device() and ws.is_contiguous(),
          "workspace: a contiguous tensor of the current device")
    return ws.numel() * ws.element_size()


def last_error() -> str:
    return lib().msd_last_error().decode()


def _check(status: int):
    if status != MSD_OK:
        raise MsdError(status, last_error())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:  # the raw handle: building a Stream object costs more than the call itself
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


# ---------------------------------------------------------------------------
# entry points (same names as the C ABI)
# ---------------------------------------------------------------------------
def model_create(cfg: ModelConfig, tensor_ptrs: Sequence[int]) -> ctypes.c_void_p:
    arr = (ctypes.c_void_p * len(tensor_ptrs))(*[p or None for p in tensor_ptrs])
    out = ctypes.c_void_p()
    _check(lib().msd_model_create(ctypes.byref(cfg), arr, len(tensor_ptrs), ctypes.byref(out)))
    return out


def model_destroy(handle) -> None:
    lib().msd_model_destroy(handle)


def workspace_bytes(handle, batch: int, n_slots: int, kappa: int, capacity: int) -> int:
    return int(lib().msd_workspace_bytes(handle, batch, n_slots, kappa, capacity))


def verify_block(handle, kv: KVCache, block: Block, ee: Optional[EERequest], logits, argmax, lse,
                 ws: torch.Tensor, stream=None) -> None:
    _check(lib().msd_verify_block(handle, ctypes.byref(kv), ctypes.byref(block),
                                  ctypes.byref(ee) if ee is not None else None, _ptr(logits),
                                  _ptr(argmax), _ptr(lse), _ptr(ws), ws.numel(), _stream(stream)))


def verify_block_static(handle, kv: KVCache, block: Block, ee: Optional[EERequest], logits, argmax,
                        lse, stream=None) -> None:
    """msd_verify_block with the library's static scratch (no workspace)."""
    _check(lib().msd_verify_block_static(handle, ctypes.byref(kv), ctypes.byref(block),
                                         ctypes.byref(ee) if ee is not None else None, _ptr(logits),
                                         _ptr(argmax), _ptr(lse), _stream(stream)))


def early_exit_topk(handle, hidden: torch.Tensor, kappa: int, ids, logp, ws: torch.Tensor,
                    stream=None) -> None:
    _check(lib().msd_early_exit_topk(handle, _ptr(hidden), hidden.shape[0], kappa, _ptr(ids),
                                     _ptr(logp), _ptr(ws), ws.numel(), _stream(stream)))


def accept(handle, block: Block, logits, argmax, sampling: Optional[Sampling], acc_len, next_tok,
           path, status, ws: Optional[torch.Tensor] = None, stream=None, near_tie=None) -> None:
    """near_tie: optional device uint8 [batch] of near-tie flags (msd.h)."""
    _check(lib().msd_accept(handle, ctypes.byref(block), _ptr(logits), _ptr(argmax),
                            ctypes.byref(sampling) if sampling is not None else None,
                            _ptr(acc_len), _ptr(next_tok), _ptr(path), _ptr(near_tie),
                            _ptr(status), _ptr(ws), 0 if ws is None else ws.numel(),
                            _stream(stream)))


def kv_commit(handle, kv: KVCache, block: Block, acc_len, path, stream=None) -> None:
    _check(lib().msd_kv_commit(handle, ctypes.byref(kv), ctypes.byref(block), _ptr(acc_len),
                               _ptr(path), _stream(stream)))


def hyp_tree(parent, tokens) -> "HypTree":
    """msd_hyp_tree over a host parent list (-1 = root) and a device int32
    tensor of tokens [batch][n_nodes]; keeps the host array alive."""
    n = len(parent)
    P = (ctypes.c_int32 * n)(*parent)
    t = HypTree(n, ctypes.cast(P, ctypes.POINTER(ctypes.c_int32)), _ptr(tokens))
    t._keep = (P, tokens)
    return t


def reuse_select(handle, block: Block, acc_len, next_tok, path, tree: HypTree, next_case, next_node,
                 logits=None, lse=None, ee_ids=None, kappa: int = 0, omega=None, stats=None,
                 stream=None) -> None:
    """stats: a device tensor of at least 40 bytes holding msd_reuse_stats."""
    _check(lib().msd_reuse_select(handle, ctypes.byref(block), _ptr(acc_len), _ptr(next_tok),
                                  _ptr(path), ctypes.byref(tree), _ptr(logits), _ptr(lse),
                                  _ptr(ee_ids), int(kappa), _ptr(next_case), _ptr(next_node),
                                  _ptr(omega), _ptr(stats), _stream(stream)))


def read_reuse_stats(stats) -> dict:
    """Copies a device msd_reuse_stats to the host."""
    raw = bytes(stats.detach().cpu().contiguous().view(-1).numpy().tobytes()[:ctypes.sizeof(ReuseStats)])
    r = ReuseStats.from_buffer_copy(raw)
    return {f: getattr(r, f) for f, _ in ReuseStats._fields_}


def set_profile(handle, kclass: int, begin_events, end_events) -> None:
    """begin/end: sequences of raw hipEvent_t handles (ints), one per layer,
    None to skip a layer; [] turns it off."""
    n = len(begin_events)
    B = (ctypes.c_void_p * max(n, 1))(*begin_events)
    E = (ctypes.c_void_p * max(n, 1))(*end_events)
    _check(lib().msd_set_profile(handle, kclass, B if n else None, E if n else None, n))


def paged_append(kv: PagedKV, rows: KVRows, rope: Optional[Rope] = None, stream=None) -> None:
    _fits(kv, rows)
    if rope is not None:
        _here(rope)
    _check(lib().msd_paged_append(ctypes.byref(kv), ctypes.byref(rows),
                                  ctypes.byref(rope) if rope is not None else None,
                                  _stream(stream)))


def paged_commit(kv: PagedKV, rows: KVRows, acc_len, path, rope: Optional[Rope] = None,
                 stream=None) -> None:
    """acc_len: device int32 [batch], path: device int32 [batch][n_rows], as accept wrote them."""
    _fits(kv, rows)
    _here(rope)
    _typed(acc_len, torch.int32, (rows.batch,), "acc_len")
    _typed(path, torch.int32, (rows.batch, rows.n_rows), "path")
    _need(_one_device(acc_len, path) == torch.cuda.current_device(), "tensors of another device than the current one")
    _check(lib().msd_paged_commit(ctypes.byref(kv), ctypes.byref(rows),
                                  ctypes.byref(rope) if rope is not None else None, _ptr(acc_len),
                                  _ptr(path), _stream(stream)))


def paged_attention_workspace_bytes(kv: PagedKV, batch: int, n_slots: int, n_heads: int) -> int:
    return int(lib().msd_paged_attention_workspace_bytes(ctypes.byref(kv), batch, n_slots, n_heads))


def paged_attention(kv: PagedKV, layer: int, attn: PagedAttn, ws: torch.Tensor, stream=None) -> None:
    _fits(kv, attn)
    _check(lib().msd_paged_attention(ctypes.byref(kv), layer, ctypes.byref(attn), _ptr(ws),
                                     _nbytes(ws), _stream(stream)))


def verify_paged_workspace_bytes(handle, kv: PagedKV, batch: int, n_slots: int, kappa: int) -> int:
    return int(lib().msd_verify_paged_workspace_bytes(handle, ctypes.byref(kv), batch, n_slots, kappa))


def verify_block_paged(handle, kv: PagedKV, block: Block, ee: Optional[EERequest], k_rows: torch.Tensor,
                       v_rows: torch.Tensor, logits, argmax, lse, ws: torch.Tensor, window: int = 0, sinks: int = 0,
                       stream=None) -> None:
    """k_rows, v_rows: bf16 [n_layers][batch][kv_heads][n_slots][head_dim], written; block_rows() commits them."""
    shape = (kv.n_layers, block.batch, kv.n_kv_heads, block.n_slots, kv.head_dim)
    _typed(k_rows, torch.bfloat16, shape, "k_rows")
    _typed(v_rows, torch.bfloat16, shape, "v_rows")
    _need(_one_device(k_rows, v_rows, logits, argmax, lse) == torch.cuda.current_device(),
          "tensors of another device than the current one")
    _here(kv)
    _check(lib().msd_verify_block_paged(handle, ctypes.byref(kv), ctypes.byref(block),
                                        ctypes.byref(ee) if ee is not None else None, _ptr(k_rows), _ptr(v_rows),
                                        int(window), int(sinks), _ptr(logits), _ptr(argmax), _ptr(lse), _ptr(ws),
                                        _nbytes(ws), _stream(stream)))


def sample_workspace_bytes(rows: int, vocab: int) -> int:
    return int(lib().msd_sample_workspace_bytes(rows, vocab))


def sample(logits: torch.Tensor, u: torch.Tensor, params: Optional[SampleParams], tok: torch.Tensor,
           ws: torch.Tensor, logp: Optional[torch.Tensor] = None,
           kept: Optional[torch.Tensor] = None, stream=None) -> None:
    """logits: device fp32 [rows][vocab], rows contiguous (any row stride >= vocab)."""
    _need(logits.dim() == 2 and logits.dtype == torch.float32 and logits.is_cuda and
          (logits.stride(1) == 1 or logits.shape[1] == 1), "logits: a device fp32 [rows][vocab] tensor of contiguous rows")
    rows, vocab = logits.shape
    _typed(u, torch.float32, (rows,), "u")
    _typed(tok, torch.int32, (rows,), "tok")
    if logp is not None:
        _typed(logp, torch.float32, (rows,), "logp")
    if kept is not None:
        _typed(kept, torch.int32, (rows,), "kept")
    _need(params is None or getattr(params, "_rows", None) in (None, rows), "params: one value for each row of logits")
    _need(_one_device(logits, u, tok, logp, kept) == torch.cuda.current_device(), "tensors of another device than the current one")
    _here(params)
    _check(lib().msd_sample(logits.data_ptr(), logits.stride(0) if rows > 1 else vocab, rows, vocab,
                            ctypes.byref(params) if params is not None else None, _ptr(u), _ptr(tok),
                            _ptr(logp), _ptr(kept), _ptr(ws), _nbytes(ws), _stream(stream)))


# ---------------------------------------------------------------------------
# conveniences: still marshalling only
# ---------------------------------------------------------------------------
def config_of(shape) -> ModelConfig:
    """ModelConfig from a shape description with the synth.ModelShape fields."""
    return ModelConfig(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads,
                       shape.head_dim, shape.d_ffn, shape.vocab,
                       MSD_NORM_LAYER if shape.norm == "layer" else MSD_NORM_RMS,
                       MSD_ACT_RELU if shape.act == "relu" else MSD_ACT_SWIGLU,
                       MSD_POS_LEARNED if shape.pos == "learned" else MSD_POS_ROPE,
                       int(shape.bias), int(shape.tied_head),
                       int(getattr(shape, "max_positions_rt", 0) or shape.max_positions or 0),
                       float(shape.rope_theta), float(shape.norm_eps))


class Model:
    """Owns a msd_model handle built from named bf16 device tensors."""

    def __init__(self, shape, tensors: Dict[str, torch.Tensor], max_positions: int):
        cfg = config_of(shape)
        if shape.pos != "learned":
            cfg.max_positions = max_positions
        self.shape = shape
        self.cfg = cfg
        self.tensors = tensors  # keep alive
        ptrs: List[Optional[int]] = [None] * (len(GLOBAL_SLOTS) + len(LAYER_SLOTS) * shape.n_layers)
        for i, n in enumerate(GLOBAL_SLOTS):
            if n in tensors:
                ptrs[i] = _ptr(tensors[n])
        for l in range(shape.n_layers):
            for j, n in enumerate(LAYER_SLOTS):
                t = tensors.get(f"l{l}.{n}")
                if t is not None:
                    ptrs[len(GLOBAL_SLOTS) + l * len(LAYER_SLOTS) + j] = _ptr(t)
        self.handle = model_create(cfg, ptrs)

    def close(self):
        if getattr(self, "handle", None):
            model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Cache:
    """KV cache tensors [L][batch_cap][Hkv][capacity][hd] bf16, len, status."""

    def __init__(self, shape, batch_cap: int, capacity: int, device="cuda"):
        dims = (shape.n_layers, batch_cap, shape.n_kv_heads, capacity, shape.head_dim)
        self.k = torch.zeros(dims, dtype=torch.bfloat16, device=device)
        self.v = torch.zeros(dims, dtype=torch.bfloat16, device=device)
        self.len = torch.zeros(batch_cap, dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.c = KVCache(self.k.data_ptr(), self.v.data_ptr(), self.len.data_ptr(),
                         self.status.data_ptr(), batch_cap, capacity)


def make_block(tokens: torch.Tensor, parent=None) -> Block:
    """tokens: device int32 [batch][n_slots]; parent: host sequence or None (chain)."""
    assert tokens.dtype == torch.int32 and tokens.dim() == 2
    b = Block(tokens.shape[0], tokens.shape[1], _ptr(tokens), None)
    b._keep = (tokens,)  # the block holds only the address: keep the tensor alive with it
    if parent is not None:
        arr = (ctypes.c_int32 * len(parent))(*[int(p) for p in parent])
        b.parent = ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32))
        b._keep = (tokens, arr)
    return b


class PagedCache:
    """A paged cache over the caller's device tensors (msd.h):

    k, v        [n_layers][n_pages][n_kv_heads][page_size][head_dim], bf16, or uint8 codes (8-bit pages)
    page_table  int32 [batch_cap][max_pages]; len int32 [batch_cap]; status int32 [1]
    k_scale, v_scale  8-bit pages: uint8 [n_layers][n_pages][n_kv_heads][page_size // 16]
    """

    def __init__(self, k, v, page_table, len, status, k_scale=None, v_scale=None):
        fp8 = k.dtype == torch.uint8
        _need(k.dim() == 5 and (fp8 or k.dtype == torch.bfloat16), "k: bf16 or uint8 pages [layers][pages][heads][page][dim]")
        _typed(k, k.dtype, k.shape, "k")
        _typed(v, k.dtype, k.shape, "v")
        L, pages, heads, page, hd = k.shape
        if fp8:
            shape = (L, pages, heads, page // MSD_KV_SCALE_TOKENS)
            _typed(k_scale, torch.uint8, shape, "k_scale")
            _typed(v_scale, torch.uint8, shape, "v_scale")
        else:
            _need(k_scale is None and v_scale is None, "bf16 pages have no scales")
        _need(page_table.dim() == 2, "page_table: [batch_cap][max_pages]")
        batch_cap, max_pages = page_table.shape
        _typed(page_table, torch.int32, page_table.shape, "page_table")
        _typed(len, torch.int32, (batch_cap,), "len")
        _typed(status, torch.int32, (1,), "status")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.page_table, self.len, self.status = page_table, len, status
        self.c = PagedKV(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), _ptr(page_table), _ptr(len),
                         _ptr(status), MSD_KV_FP8 if fp8 else MSD_KV_BF16, L, pages, heads, page, hd,
                         batch_cap, max_pages)
        self.c._keep = (k, v, k_scale, v_scale, page_table, len, status)
        self.c._device = _one_device(k, v, k_scale, v_scale, page_table, len, status)

    @staticmethod
    def allocate(n_layers: int, n_kv_heads: int, head_dim: int, n_pages: int, page_size: int,
                 batch_cap: int, max_pages: int, fmt: str = "bf16", device="cuda") -> "PagedCache":
        """Zeroed pages, an empty page table (every id -1) and lengths of zero; fmt "bf16" or "fp8"."""
        _need(fmt in ("bf16", "fp8"), "fmt: bf16 or fp8")
        dt = torch.uint8 if fmt == "fp8" else torch.bfloat16
        kv = [torch.zeros((n_layers, n_pages, n_kv_heads, page_size, head_dim), dtype=dt, device=device)
              for _ in range(2)]
        sc = [torch.zeros((n_layers, n_pages, n_kv_heads, page_size // MSD_KV_SCALE_TOKENS),
                          dtype=torch.uint8, device=device) if fmt == "fp8" else None for _ in range(2)]
        table = torch.full((batch_cap, max_pages), -1, dtype=torch.int32, device=device)
        return PagedCache(kv[0], kv[1], table, torch.zeros(batch_cap, dtype=torch.int32, device=device),
                          torch.zeros(1, dtype=torch.int32, device=device), sc[0], sc[1])


def rope(table: torch.Tensor, layout: str = "half") -> Rope:
    """table: device fp32 [positions][rotary_dim // 2][2] of (cos, sin)."""
    _need(layout in ROPE_LAYOUTS, "layout: half or interleaved")
    _need(table.dim() == 3 and table.shape[2] == 2, "table: [positions][rotary_dim // 2][2]")
    _typed(table, torch.float32, table.shape, "table")
    r = Rope(_ptr(table), table.shape[0], 2 * table.shape[1], ROPE_LAYOUTS[layout])
    r._keep = (table,)
    r._device = _one_device(table)
    return r


def _strided(t: torch.Tensor, what: str):
    """Strides of a bf16 tensor whose rows are contiguous; of an axis of one, 0."""
    _need(t.dtype == torch.bfloat16 and t.is_cuda and t.stride(-1) == 1, f"{what}: a device bf16 tensor, last axis contiguous")
    return [s if n > 1 else 0 for s, n in zip(t.stride()[:-1], t.shape[:-1])]


def kv_rows(k: torch.Tensor, v: torch.Tensor, layer: int = 0, count: Optional[torch.Tensor] = None) -> KVRows:
    """k, v: bf16 [layers][batch][rows][kv_heads][head_dim], or without the first axis for one layer; any strides
    that are multiples of 8, the same for both. They go to the cache's layers `layer` and on."""
    if k.dim() == 4:
        k = k[None]
    if v.dim() == 4:
        v = v[None]
    _need(k.dim() == 5 and k.shape == v.shape, "k and v: [layers][batch][rows][kv_heads][head_dim]")
    st = _strided(k, "k")
    _need(st == _strided(v, "v"), "k and v have the same strides")
    if count is not None:
        _typed(count, torch.int32, (k.shape[1],), "count")
    r = KVRows(k.data_ptr(), v.data_ptr(), *st, layer, k.shape[0], k.shape[1], k.shape[2], _ptr(count))
    r._keep = (k, v, count)
    r._heads, r._device = tuple(k.shape[3:]), _one_device(k, v, count)
    return r


def block_rows(k_rows: torch.Tensor, v_rows: torch.Tensor) -> KVRows:
    """The rows that verify_block_paged wrote, as paged_commit takes them."""
    return kv_rows(k_rows.transpose(2, 3), v_rows.transpose(2, 3))


def paged_attn(q: torch.Tensor, out: torch.Tensor, k_new: Optional[torch.Tensor] = None,
               v_new: Optional[torch.Tensor] = None, parent=None, count: Optional[torch.Tensor] = None,
               rope: Optional[Rope] = None, window: int = 0, sinks: int = 0,
               scale: Optional[float] = None) -> PagedAttn:
    """q, out: bf16 [batch][slots][heads][head_dim]; k_new, v_new: bf16 [batch][slots][kv_heads][head_dim] of the
    same strides; parent: host sequence or None (chain). scale: head_dim ** -0.5 unless given."""
    _need(q.dim() == 4 and q.shape == out.shape, "q and out: [batch][slots][heads][head_dim]")
    B, n, H, hd = q.shape
    qs, os_ = _strided(q, "q"), _strided(out, "out")
    _need(all(st > 0 for st, size in zip(out.stride(), out.shape) if size > 1), "out: no row twice")
    _need((k_new is None) == (v_new is None), "k_new and v_new go together")
    ns = [0, 0, 0]
    if k_new is not None:
        _need(k_new.dim() == 4 and k_new.shape == v_new.shape and k_new.shape[:2] == q.shape[:2] and
              k_new.shape[3] == hd, "k_new and v_new: [batch][slots][kv_heads][head_dim]")
        ns = _strided(k_new, "k_new")
        _need(ns == _strided(v_new, "v_new"), "k_new and v_new have the same strides")
    if count is not None:
        _typed(count, torch.int32, (B,), "count")
    arr = None
    if parent is not None:
        _need(len(parent) == n, "parent: one entry for each slot")
        arr = (ctypes.c_int32 * n)(*[int(p) for p in parent])
    a = PagedAttn(q.data_ptr(), *qs, out.data_ptr(), *os_,
                  None if k_new is None else k_new.data_ptr(), None if v_new is None else v_new.data_ptr(), *ns,
                  ctypes.cast(arr, ctypes.POINTER(ctypes.c_int32)) if arr is not None else None, _ptr(count),
                  ctypes.pointer(rope) if rope is not None else None,
                  float(hd) ** -0.5 if scale is None else float(scale), B, n, H, int(window), int(sinks))
    a._keep = (q, out, k_new, v_new, arr, count, rope)
    a._heads, a._device = (None if k_new is None else k_new.shape[2], hd), _one_device(q, out, k_new, v_new, count, *(rope._keep if rope is not None else ()))
    return a


def sample_params(temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
                  top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None) -> SampleParams:
    """Device tensors of one value a row: fp32, top_k int32; None leaves a filter off."""
    rows = None
    for t, dt, what in ((temperature, torch.float32, "temperature"), (top_k, torch.int32, "top_k"),
                        (top_p, torch.float32, "top_p"), (min_p, torch.float32, "min_p")):
        if t is not None:
            rows = t.numel() if rows is None else rows
            _typed(t, dt, (rows,), what)
    p = SampleParams(_ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p))
    p._rows = rows
    if rows is not None:
        p._device = _one_device(temperature, top_k, top_p, min_p)
    p._keep = (temperature, top_k, top_p, min_p)
    return p
