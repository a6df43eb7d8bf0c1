"""ctypes binding of libcc (include/cc.h): argument marshalling only.

Every function here has the name of the C entry point it calls.  Tensors are torch
tensors on the GPU; the binding passes their data pointers, the current HIP stream and
a workspace tensor it allocates through torch.  All arithmetic runs in libcc's HIP
kernels; there is no fallback: if libcc.so is missing or fails to load, importing this
module raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from dataclasses import dataclass, field
from typing import Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcc.so")

(CC_OK, CC_ERR_ARG, CC_ERR_SHAPE, CC_ERR_DTYPE, CC_ERR_WORKSPACE, CC_ERR_UNSUPPORTED, CC_ERR_HIP,
 CC_ERR_SCRATCH) = range(8)
CC_NOALLOC_SCRATCH_BYTES = 32 << 20
CC_F32, CC_BF16 = 0, 1
CC_DIAG_STRICT, CC_DIAG_INCLUSIVE = 0, 1
CC_MODE_LAST_LAYER, CC_MODE_FULL, CC_MODE_LAST_LAYER_H, CC_MODE_LAST_LAYER_FUSED = 0, 1, 2, 3
CC_KV_CONTIGUOUS, CC_KV_PAGED = 0, 1
CC_MASK_CAUSAL, CC_MASK_COUNTER_CAUSAL = 0, 1
CC_LOGPROBS_MAX_TOP = 32

EXPORTED = [
    "cc_status_str", "cc_version", "cc_score_workspace", "cc_score", "cc_attention_workspace",
    "cc_attention_cc", "cc_lmhead_workspace", "cc_lmhead_score", "cc_linear",
    "cc_select_workspace", "cc_select_keep", "cc_compact_workspace", "cc_compact_kv",
    "cc_compact_rows_workspace", "cc_compact_rows", "cc_fuse_wo_lmhead_workspace",
    "cc_fuse_wo_lmhead", "cc_quantize_fp8_workspace", "cc_quantize_fp8",
    "cc_lmhead_fp8_workspace", "cc_lmhead_score_fp8", "cc_pack_lmhead_bytes", "cc_pack_lmhead",
    "cc_lmhead_score_packed", "cc_lmhead_score_noalloc", "cc_append_kv", "cc_append_kv8",
    "cc_compact_kv8", "cc_attention_kv8_workspace", "cc_attention_kv8",
    "cc_lmhead_logprobs_workspace", "cc_lmhead_logprobs", "cc_attention_kv_workspace", "cc_attention_kv",
    "cc_attention_prefix_workspace", "cc_attention_prefix", "cc_attention_weights_workspace",
    "cc_attention_weights", "cc_weight_scores", "cc_compact_weights",
]

_c_void_p = ctypes.c_void_p
_i32 = ctypes.c_int32
_i64 = ctypes.c_int64


class c_kv(ctypes.Structure):
    _fields_ = [("layout", _i32), ("n_layers", _i32), ("k", _c_void_p), ("v", _c_void_p),
                ("seq_stride", _i64), ("layer_stride", _i64), ("head_stride", _i64),
                ("tok_stride", _i64), ("page_stride", _i64), ("block_table", _c_void_p),
                ("page_size", _i32), ("max_pages", _i32)]


class c_problem(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("mode", _i32), ("diag", _i32), ("n_seqs", _i32),
                ("cu_seqlens_h", ctypes.POINTER(_i32)), ("cu_seqlens_d", _c_void_p),
                ("n_heads_q", _i32), ("n_heads_kv", _i32), ("head_dim", _i32),
                ("hidden", _i32), ("vocab", _i32), ("n_layers", _i32), ("ffn", _i32),
                ("softmax_scale", ctypes.c_float), ("rope_theta", ctypes.c_float),
                ("rms_eps", ctypes.c_float), ("n_frozen", _i32), ("lmhead_packed", _i32)]


class c_layer_weights(ctypes.Structure):
    _fields_ = [("attn_norm", _c_void_p), ("wq", _c_void_p), ("wo", _c_void_p),
                ("mlp_norm", _c_void_p), ("w_gate", _c_void_p), ("w_up", _c_void_p),
                ("w_down", _c_void_p)]


class c_inputs(ctypes.Structure):
    _fields_ = [("q", _c_void_p), ("kv", c_kv), ("token_ids", _c_void_p), ("pos_ids", _c_void_p),
                ("w_o", _c_void_p), ("w_lm", _c_void_p), ("embed", _c_void_p),
                ("layers_h", ctypes.POINTER(c_layer_weights)), ("final_norm", _c_void_p),
                ("h_last", _c_void_p), ("w_lm_packed", _c_void_p)]


class c_kv8(ctypes.Structure):
    _fields_ = [("codes", c_kv), ("k_scale", _c_void_p), ("v_scale", _c_void_p),
                ("scale_seq_stride", _i64), ("scale_layer_stride", _i64),
                ("scale_head_stride", _i64), ("scale_page_stride", _i64), ("scale_block", _i32)]


class c_rows(ctypes.Structure):
    _fields_ = [("base", _c_void_p), ("layer_stride", _i64), ("tok_stride", _i64),
                ("head_stride", _i64)]


class c_append(ctypes.Structure):
    _fields_ = [("k", c_rows), ("v", c_rows), ("q", c_rows), ("q_out", _c_void_p),
                ("cached", _c_void_p), ("pos_ids", _c_void_p), ("capacity", _i64),
                ("layer", _i32), ("n_layers", _i32), ("rotate", _i32)]


class c_prefix(ctypes.Structure):
    _fields_ = [("kv", c_kv), ("n_prefixes", _i32), ("max_len", _i32),
                ("first_seq_h", ctypes.POINTER(_i32)), ("first_seq_d", _c_void_p), ("lens", _c_void_p)]


class c_weights(ctypes.Structure):
    _fields_ = [("base", _c_void_p), ("seq_stride", _i64), ("head_stride", _i64), ("entries", _i64)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libcc.so not built at {LIB_PATH}; run __graft_entry__.build()")
    lib = ctypes.CDLL(LIB_PATH)
    st = _i32
    sz = ctypes.POINTER(ctypes.c_size_t)
    P = ctypes.POINTER
    sig = {
        "cc_status_str": (ctypes.c_char_p, [st]),
        "cc_version": (ctypes.c_char_p, []),
        "cc_score_workspace": (st, [P(c_problem), sz]),
        "cc_score": (st, [P(c_problem), P(c_inputs), _c_void_p, _c_void_p, ctypes.c_size_t,
                          _c_void_p]),
        "cc_attention_workspace": (st, [P(c_problem), sz]),
        "cc_attention_cc": (st, [P(c_problem), _c_void_p, P(c_kv), _i32, _c_void_p, _c_void_p,
                                 ctypes.c_size_t, _c_void_p]),
        "cc_lmhead_workspace": (st, [P(c_problem), sz]),
        "cc_lmhead_score": (st, [P(c_problem), _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                                 _c_void_p, _c_void_p, ctypes.c_size_t, _c_void_p]),
        "cc_lmhead_score_noalloc": (st, [P(c_problem), _c_void_p, _c_void_p, _c_void_p,
                                         _c_void_p, _c_void_p, _c_void_p]),
        "cc_linear": (st, [_i32, _c_void_p, _c_void_p, _c_void_p, _i32, _i32, _i32, _c_void_p]),
        "cc_fuse_wo_lmhead_workspace": (st, [_i32, _i32, _i32, sz]),
        "cc_quantize_fp8_workspace": (st, [_i64, sz]),
        "cc_quantize_fp8": (st, [_i32, _c_void_p, _i64, _i32, _i32, _c_void_p, _c_void_p,
                                 _c_void_p, ctypes.c_size_t, _c_void_p]),
        "cc_lmhead_fp8_workspace": (st, [P(c_problem), sz]),
        "cc_lmhead_score_fp8": (st, [P(c_problem), _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                                     _c_void_p, _c_void_p, _c_void_p, ctypes.c_size_t,
                                     _c_void_p]),
        "cc_pack_lmhead_bytes": (st, [_i64, _i32, sz]),
        "cc_pack_lmhead": (st, [_c_void_p, _i64, _i32, _c_void_p, ctypes.c_size_t, _c_void_p]),
        "cc_lmhead_score_packed": (st, [P(c_problem), _c_void_p, _c_void_p, _c_void_p,
                                        _c_void_p, _c_void_p, _c_void_p, ctypes.c_size_t,
                                        _c_void_p]),
        "cc_fuse_wo_lmhead": (st, [_i32, _c_void_p, _c_void_p, _c_void_p, _i32, _i32, _i32,
                                   _c_void_p, ctypes.c_size_t, _c_void_p]),
        "cc_select_workspace": (st, [_i32, sz]),
        "cc_select_keep": (st, [_c_void_p, _i32, P(_i64), P(_i32), P(_i32), _c_void_p, _c_void_p,
                                ctypes.c_size_t, _c_void_p]),
        "cc_compact_workspace": (st, [P(c_problem), _i32, _i32, sz]),
        "cc_compact_kv": (st, [P(c_problem), P(c_kv), _c_void_p, P(_i32), _i32, _c_void_p,
                               _c_void_p, P(c_kv), _c_void_p, ctypes.c_size_t, _c_void_p]),
        "cc_compact_rows_workspace": (st, [P(c_problem), _i32, _i32, sz]),
        "cc_compact_rows": (st, [P(c_problem), _c_void_p, _i32, _c_void_p, P(_i32), _i32,
                                 _c_void_p, _c_void_p, ctypes.c_size_t, _c_void_p]),
        "cc_append_kv": (st, [P(c_problem), P(c_append), P(c_kv), _c_void_p]),
        "cc_append_kv8": (st, [P(c_problem), P(c_append), P(c_kv8), _c_void_p]),
        "cc_compact_kv8": (st, [P(c_problem), P(c_kv8), _c_void_p, P(_i32), _i32, _c_void_p,
                                _c_void_p, P(c_kv8), _c_void_p]),
        "cc_attention_kv8_workspace": (st, [P(c_problem), _i32, _i32, sz]),
        "cc_attention_kv8": (st, [P(c_problem), _c_void_p, P(c_kv8), _i32, _i32, _c_void_p, _i32,
                                  _c_void_p, _c_void_p, ctypes.c_size_t, _c_void_p]),
        "cc_lmhead_logprobs_workspace": (st, [_i32, _i32, _i32, _i32, _i32, sz]),
        "cc_lmhead_logprobs": (st, [_i32, _c_void_p, _c_void_p, _i32, _i32, _i32, _i32, _c_void_p,
                                    _i32, _c_void_p, _c_void_p, _c_void_p, _c_void_p, _c_void_p,
                                    ctypes.c_size_t, _c_void_p]),
        "cc_attention_kv_workspace": (st, [P(c_problem), _i32, sz]),
        "cc_attention_kv": (st, [P(c_problem), _c_void_p, P(c_kv), _i32, _c_void_p, _i32, _c_void_p,
                                 _c_void_p, _c_void_p, ctypes.c_size_t, _c_void_p]),
        "cc_attention_prefix_workspace": (st, [P(c_problem), P(c_prefix), _i32, sz]),
        "cc_attention_prefix": (st, [P(c_problem), _c_void_p, P(c_prefix), P(c_kv), _i32, _c_void_p, _i32,
                                     _c_void_p, _c_void_p, _c_void_p, ctypes.c_size_t, _c_void_p]),
        "cc_attention_weights_workspace": (st, [P(c_problem), _i32, sz]),
        "cc_attention_weights": (st, [P(c_problem), _c_void_p, P(c_kv), _i32, _c_void_p, _i32, _c_void_p,
                                      P(c_weights), _c_void_p, P(c_weights), _c_void_p, ctypes.c_size_t,
                                      _c_void_p]),
        "cc_weight_scores": (st, [P(c_problem), P(c_weights), _i32, _i32, _c_void_p, _c_void_p]),
        "cc_compact_weights": (st, [P(c_problem), P(c_weights), _c_void_p, P(_i32), _i32, P(c_weights),
                                    _c_void_p]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    return lib


_lib = _load()


class CCError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {_lib.cc_status_str(status).decode()}")
        self.status = status


def _check(status: int, where: str) -> None:
    if status != CC_OK:
        raise CCError(status, where)


def cc_status_str(status: int) -> str:
    return _lib.cc_status_str(status).decode()


def cc_version() -> str:
    return _lib.cc_version().decode()


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    """The handle of `stream`, by default of the current one of the current device.  Taken
    without building a torch.cuda.Stream: that object costs 5 to 10 us of host time, half of
    what a call on a short cache takes in all."""
    if stream is None:
        if not torch.cuda.is_initialized():
            torch.cuda.init()
        return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()))
    return ctypes.c_void_p(stream.cuda_stream)


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 1), dtype=torch.uint8, device=device)


_DTYPES = {CC_F32: torch.float32, CC_BF16: torch.bfloat16}


# ---------------------------------------------------------------- descriptors

@dataclass
class Problem:
    """A cc_problem plus the tensors it points at (kept alive with it)."""
    struct: c_problem
    cu_h: torch.Tensor
    cu_d: torch.Tensor
    device: torch.device

    @property
    def n_tokens(self) -> int:
        return int(self.cu_h[-1])

    @functools.cached_property
    def longest(self) -> int:
        """The most of a sequence."""
        return int((self.cu_h[1:] - self.cu_h[:-1]).max()) if len(self.cu_h) > 1 else 0


def problem(*, dtype: str, cu_seqlens: Sequence[int], n_heads_q: int, n_heads_kv: int,
            head_dim: int, hidden: int, vocab: int, device="cuda", mode: str = "last_layer",
            diag: str = "strict", n_layers: int = 0, ffn: int = 0, softmax_scale: float = 0.0,
            rope_theta: float = 0.0, rms_eps: float = 0.0, n_frozen: int = 0,
            lmhead_packed: bool = False, cu_device: Optional[torch.Tensor] = None) -> Problem:
    """cu_device: the int32 values of cu_seqlens already on the device (the default copies
    them there and waits for the copy, so the problem may be used on any stream)."""
    cu_h = torch.as_tensor(list(cu_seqlens), dtype=torch.int32).contiguous()
    if cu_device is None:
        cu_d = cu_h.to(device)
    elif cu_device.dtype != torch.int32 or cu_device.shape != cu_h.shape or not cu_device.is_contiguous():
        raise ValueError("cu_device must hold the values of cu_seqlens as contiguous int32")
    else:
        cu_d = cu_device
    s = c_problem()
    s.dtype = {"f32": CC_F32, "bf16": CC_BF16}[dtype]
    s.mode = {"last_layer": CC_MODE_LAST_LAYER, "full": CC_MODE_FULL,
              "last_layer_h": CC_MODE_LAST_LAYER_H,
              "last_layer_fused": CC_MODE_LAST_LAYER_FUSED}[mode]
    s.diag = {"strict": CC_DIAG_STRICT, "inclusive": CC_DIAG_INCLUSIVE}[diag]
    s.n_seqs = len(cu_h) - 1
    s.cu_seqlens_h = ctypes.cast(cu_h.data_ptr(), ctypes.POINTER(_i32))
    s.cu_seqlens_d = cu_d.data_ptr()
    s.n_heads_q, s.n_heads_kv, s.head_dim = n_heads_q, n_heads_kv, head_dim
    s.hidden, s.vocab, s.n_layers, s.ffn = hidden, vocab, n_layers, ffn
    s.softmax_scale, s.rope_theta, s.rms_eps = softmax_scale, rope_theta, rms_eps
    s.n_frozen = n_frozen
    s.lmhead_packed = int(lmhead_packed)
    return Problem(s, cu_h, cu_d, torch.device(device))


def packed(p: Problem, on: bool = True) -> Problem:
    """The same problem with the packed LM head switched on (or off)."""
    s = c_problem.from_buffer_copy(p.struct)
    s.lmhead_packed = int(on)
    return Problem(s, p.cu_h, p.cu_d, p.device)


class _View:
    """Where the tensors of a cache view lie: as a tensor says it (None: it holds none)."""

    def __post_init__(self):
        where = {t.get_device() for t in self.keep}
        self._device = where.pop() if len(where) == 1 else "different" if where else None

    def get_device(self) -> Optional[int]:
        if self._device == "different":
            raise ValueError("tensors on different devices")
        return self._device


@dataclass
class KV(_View):
    """A cc_kv view plus the tensors it points at."""
    struct: c_kv
    keep: list = field(default_factory=list)


def kv_contiguous(k: torch.Tensor, v: torch.Tensor, *, n_layers: int, layer_stride: int,
                  head_stride: int, tok_stride: int, seq_stride: int = 0) -> KV:
    s = c_kv()
    s.layout = CC_KV_CONTIGUOUS
    s.n_layers = n_layers
    s.k, s.v = k.data_ptr(), v.data_ptr()
    s.seq_stride, s.layer_stride, s.head_stride, s.tok_stride = (seq_stride, layer_stride,
                                                                 head_stride, tok_stride)
    s.page_stride, s.block_table, s.page_size, s.max_pages = 0, None, 0, 0
    return KV(s, [k, v])


def kv_paged(k: torch.Tensor, v: torch.Tensor, block_table: torch.Tensor, *, n_layers: int,
             layer_stride: int, page_stride: int, head_stride: int, tok_stride: int,
             page_size: int) -> KV:
    bt = block_table.to(torch.int32).contiguous()
    s = c_kv()
    s.layout = CC_KV_PAGED
    s.n_layers = n_layers
    s.k, s.v = k.data_ptr(), v.data_ptr()
    s.seq_stride, s.layer_stride, s.head_stride, s.tok_stride = 0, layer_stride, head_stride, tok_stride
    s.page_stride, s.block_table = page_stride, bt.data_ptr()
    s.page_size, s.max_pages = page_size, bt.shape[1]
    return KV(s, [k, v, bt])


@dataclass
class Inputs:
    struct: c_inputs
    keep: list = field(default_factory=list)


def inputs(*, kv: KV, token_ids: torch.Tensor, w_lm: Optional[torch.Tensor] = None,
           q: Optional[torch.Tensor] = None,
           w_o: Optional[torch.Tensor] = None, pos_ids: Optional[torch.Tensor] = None,
           embed: Optional[torch.Tensor] = None, layers: Optional[list] = None,
           final_norm: Optional[torch.Tensor] = None,
           h_last: Optional[torch.Tensor] = None,
           w_lm_packed: Optional[torch.Tensor] = None) -> Inputs:
    s = c_inputs()
    s.q = q.data_ptr() if q is not None else None
    s.kv = kv.struct
    s.token_ids = token_ids.data_ptr()
    s.pos_ids = pos_ids.data_ptr() if pos_ids is not None else None
    s.w_o = w_o.data_ptr() if w_o is not None else None
    s.w_lm = w_lm.data_ptr() if w_lm is not None else None
    s.embed = embed.data_ptr() if embed is not None else None
    s.h_last = h_last.data_ptr() if h_last is not None else None
    s.w_lm_packed = w_lm_packed.data_ptr() if w_lm_packed is not None else None
    keep = [kv, token_ids, w_lm, q, w_o, pos_ids, embed, final_norm, h_last, w_lm_packed]
    if layers:
        arr = (c_layer_weights * len(layers))()
        for i, L in enumerate(layers):
            for name in ("attn_norm", "wq", "wo", "mlp_norm", "w_gate", "w_up", "w_down"):
                setattr(arr[i], name, L[name].data_ptr())
        s.layers_h = ctypes.cast(arr, ctypes.POINTER(c_layer_weights))
        keep += [arr, layers]
    s.final_norm = final_norm.data_ptr() if final_norm is not None else None
    return Inputs(s, keep)


# ---------------------------------------------------------------- entry points

def _query(fn, *args) -> int:
    n = ctypes.c_size_t(0)
    _check(fn(*args, ctypes.byref(n)), fn.__name__)
    return n.value


def cc_score_workspace(p: Problem) -> int:
    return _query(_lib.cc_score_workspace, ctypes.byref(p.struct))


def cc_score(p: Problem, inp: Inputs, scores: torch.Tensor, workspace: Optional[torch.Tensor] = None,
             stream=None) -> torch.Tensor:
    if workspace is None:
        workspace = _workspace(cc_score_workspace(p), p.device)
    _check(_lib.cc_score(ctypes.byref(p.struct), ctypes.byref(inp.struct), _ptr(scores),
                         _ptr(workspace), workspace.numel(), _stream(stream)), "cc_score")
    return scores


def cc_attention_workspace(p: Problem) -> int:
    return _query(_lib.cc_attention_workspace, ctypes.byref(p.struct))


def cc_attention_cc(p: Problem, q: torch.Tensor, kv: KV, layer: int, o: torch.Tensor,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    if workspace is None:
        workspace = _workspace(cc_attention_workspace(p), p.device)
    _check(_lib.cc_attention_cc(ctypes.byref(p.struct), _ptr(q), ctypes.byref(kv.struct), layer,
                                _ptr(o), _ptr(workspace), workspace.numel(), _stream(stream)),
           "cc_attention_cc")
    return o


def cc_lmhead_workspace(p: Problem) -> int:
    return _query(_lib.cc_lmhead_workspace, ctypes.byref(p.struct))


def cc_lmhead_score(p: Problem, u: torch.Tensor, w_lm: torch.Tensor, token_ids: torch.Tensor,
                    scores: torch.Tensor, lse: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    if workspace is None:
        workspace = _workspace(cc_lmhead_workspace(p), p.device)
    _check(_lib.cc_lmhead_score(ctypes.byref(p.struct), _ptr(u), _ptr(w_lm), _ptr(token_ids),
                                _ptr(scores), _ptr(lse), _ptr(workspace), workspace.numel(),
                                _stream(stream)), "cc_lmhead_score")
    return scores


def cc_lmhead_score_noalloc(p: Problem, u: torch.Tensor, w_lm: torch.Tensor,
                            token_ids: torch.Tensor, scores: torch.Tensor,
                            lse: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """cc_lmhead_score with its scratch in the library's static device array (no workspace)."""
    _check(_lib.cc_lmhead_score_noalloc(ctypes.byref(p.struct), _ptr(u), _ptr(w_lm),
                                        _ptr(token_ids), _ptr(scores), _ptr(lse),
                                        _stream(stream)), "cc_lmhead_score_noalloc")
    return scores


def cc_pack_lmhead_bytes(rows: int, cols: int) -> int:
    return _query(_lib.cc_pack_lmhead_bytes, rows, cols)


def cc_pack_lmhead(x: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The packed LM-head layout of a bf16 [rows][cols] matrix (uint8 buffer)."""
    rows, cols = x.shape
    need = cc_pack_lmhead_bytes(rows, cols)
    if out is None:
        out = torch.empty(need, dtype=torch.uint8, device=x.device)
    _check(_lib.cc_pack_lmhead(_ptr(x), rows, cols, _ptr(out), out.numel() * out.element_size(),
                               _stream(stream)), "cc_pack_lmhead")
    return out


def cc_lmhead_score_packed(p: Problem, u: torch.Tensor, w_packed: torch.Tensor,
                           token_ids: torch.Tensor, scores: torch.Tensor,
                           lse: Optional[torch.Tensor] = None, workspace=None, stream=None):
    if workspace is None:
        workspace = _workspace(cc_lmhead_workspace(p), p.device)
    _check(_lib.cc_lmhead_score_packed(ctypes.byref(p.struct), _ptr(u), _ptr(w_packed),
                                       _ptr(token_ids), _ptr(scores), _ptr(lse), _ptr(workspace),
                                       workspace.numel(), _stream(stream)),
           "cc_lmhead_score_packed")
    return scores


def cc_fuse_wo_lmhead_workspace(dtype: str, hidden: int, qdim: int) -> int:
    n = ctypes.c_size_t()
    _check(_lib.cc_fuse_wo_lmhead_workspace({"f32": CC_F32, "bf16": CC_BF16}[dtype], hidden, qdim,
                                            ctypes.byref(n)), "cc_fuse_wo_lmhead_workspace")
    return n.value


def cc_fuse_wo_lmhead(dtype: str, w_lm: torch.Tensor, w_o: torch.Tensor,
                      out: Optional[torch.Tensor] = None, workspace=None, stream=None):
    """The LAST_LAYER_FUSED weight W_lm W_o [V][Hq*d] from w_lm [V][D] and w_o [D][Hq*d]."""
    V, D = w_lm.shape
    D2, Q = w_o.shape
    if D2 != D:
        raise ValueError(f"w_o has {D2} rows, w_lm has {D} columns")
    if out is None:
        out = torch.empty((V, Q), dtype=w_lm.dtype, device=w_lm.device)
    if workspace is None:
        workspace = _workspace(cc_fuse_wo_lmhead_workspace(dtype, D, Q), w_lm.device)
    _check(_lib.cc_fuse_wo_lmhead({"f32": CC_F32, "bf16": CC_BF16}[dtype], _ptr(w_lm), _ptr(w_o),
                                  _ptr(out), V, D, Q, _ptr(workspace), workspace.numel(),
                                  _stream(stream)), "cc_fuse_wo_lmhead")
    return out


def cc_quantize_fp8_workspace(rows: int) -> int:
    n = ctypes.c_size_t()
    _check(_lib.cc_quantize_fp8_workspace(rows, ctypes.byref(n)), "cc_quantize_fp8_workspace")
    return n.value


def cc_quantize_fp8(dtype: str, x: torch.Tensor, per_row: bool, codes=None, scale=None,
                    workspace=None, stream=None):
    """E4M3 codes (uint8, x's shape) and fp32 scales ([rows], or [1] for the matrix)."""
    rows, cols = x.shape
    if codes is None:
        codes = torch.empty((rows, cols), dtype=torch.uint8, device=x.device)
    if scale is None:
        scale = torch.empty(rows if per_row else 1, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = _workspace(cc_quantize_fp8_workspace(rows), x.device)
    _check(_lib.cc_quantize_fp8({"f32": CC_F32, "bf16": CC_BF16}[dtype], _ptr(x), rows, cols,
                                int(per_row), _ptr(codes), _ptr(scale), _ptr(workspace),
                                workspace.numel(), _stream(stream)), "cc_quantize_fp8")
    return codes, scale


def cc_lmhead_fp8_workspace(p: Problem) -> int:
    return _query(_lib.cc_lmhead_fp8_workspace, ctypes.byref(p.struct))


def cc_lmhead_score_fp8(p: Problem, u: torch.Tensor, w_codes: torch.Tensor, w_scale: torch.Tensor,
                        token_ids: torch.Tensor, scores: torch.Tensor,
                        lse: Optional[torch.Tensor] = None, workspace=None, stream=None):
    if workspace is None:
        workspace = _workspace(cc_lmhead_fp8_workspace(p), p.device)
    _check(_lib.cc_lmhead_score_fp8(ctypes.byref(p.struct), _ptr(u), _ptr(w_codes), _ptr(w_scale),
                                    _ptr(token_ids), _ptr(scores), _ptr(lse), _ptr(workspace),
                                    workspace.numel(), _stream(stream)), "cc_lmhead_score_fp8")
    return scores


def cc_linear(dtype: str, x: torch.Tensor, w: torch.Tensor, y: torch.Tensor, stream=None):
    M, K = x.shape
    N = w.shape[0]
    _check(_lib.cc_linear({"f32": CC_F32, "bf16": CC_BF16}[dtype], _ptr(x), _ptr(w), _ptr(y), M, N,
                          K, _stream(stream)), "cc_linear")
    return y


def cc_select_workspace(n_segs: int) -> int:
    return _query(_lib.cc_select_workspace, n_segs)


def _host_array(x, dtype, ctype):
    """x as a C array of integers to pass by pointer, and its length: a plain short list or tuple of
    ints directly, anything else (a scalar, ints that do not fit) through a C-contiguous numpy array
    (no copy if it is one of that type).  Up to 64 ints are quicker as a C array (8: 1 us against 3 to
    5), from 128 on through numpy (1024: 67 us against 38)."""
    if type(x) in (list, tuple) and len(x) <= 64:
        try:
            arr = (ctype * len(x))(*x)
            if arr[:] == list(x):   # ctypes wraps what does not fit
                return arr, len(x)
        except TypeError:
            pass
    a = np.ascontiguousarray(np.asarray(x), dtype=dtype)
    arr = ctypes.cast(a.ctypes.data, ctypes.POINTER(ctype))
    arr._keep = a
    return arr, len(a)


def cc_select_keep(scores: torch.Tensor, seg_start: Sequence[int], seg_len: Sequence[int],
                   k: Sequence[int], keep_idx: torch.Tensor,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """seg_start, seg_len, k: host sequences or numpy arrays (int64, int32, int32 arrays
    are passed without a copy)."""
    st, _ = _host_array(seg_start, np.int64, _i64)
    ln, n = _host_array(seg_len, np.int32, _i32)
    kk, _ = _host_array(k, np.int32, _i32)
    if workspace is None:
        workspace = _workspace(cc_select_workspace(n), scores.device)
    _check(_lib.cc_select_keep(_ptr(scores), n, st, ln, kk, _ptr(keep_idx), _ptr(workspace),
                               workspace.numel(), _stream(stream)), "cc_select_keep")
    return keep_idx


def cc_compact_workspace(p: Problem, cache_layers: int, per_head: int) -> int:
    return _query(_lib.cc_compact_workspace, ctypes.byref(p.struct), cache_layers, per_head)


def cc_compact_kv(p: Problem, kv: KV, keep_idx: torch.Tensor, k: Sequence[int], per_head: int,
                  token_ids: Optional[torch.Tensor] = None, pos_ids: Optional[torch.Tensor] = None,
                  out: Optional[KV] = None, workspace: Optional[torch.Tensor] = None,
                  stream=None) -> None:
    kk = (_i32 * len(k))(*[int(x) for x in k])
    if workspace is None:
        workspace = _workspace(cc_compact_workspace(p, kv.struct.n_layers, per_head), p.device)
    _check(_lib.cc_compact_kv(ctypes.byref(p.struct), ctypes.byref(kv.struct), _ptr(keep_idx), kk,
                              per_head, _ptr(token_ids), _ptr(pos_ids),
                              ctypes.byref(out.struct) if out is not None else None,
                              _ptr(workspace), workspace.numel(), _stream(stream)),
           "cc_compact_kv")


def cc_compact_rows_workspace(p: Problem, row_bytes: int, per_head: int) -> int:
    return _query(_lib.cc_compact_rows_workspace, ctypes.byref(p.struct), row_bytes, per_head)


def cc_compact_rows(p: Problem, rows: torch.Tensor, keep_idx: torch.Tensor, k: Sequence[int],
                    per_head: int, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """rows: [N][...] token-major; every entry row is compacted with its sequence's keep
    list (in place unless `out` is given)."""
    row_bytes = rows[0].numel() * rows.element_size() if rows.shape[0] else 16
    kk = (_i32 * len(k))(*[int(x) for x in k])
    if workspace is None:
        workspace = _workspace(cc_compact_rows_workspace(p, row_bytes, per_head), p.device)
    _check(_lib.cc_compact_rows(ctypes.byref(p.struct), _ptr(rows), row_bytes, _ptr(keep_idx), kk,
                                per_head, _ptr(out), _ptr(workspace), workspace.numel(),
                                _stream(stream)), "cc_compact_rows")


# ---------------------------------------------------------------- cache in 8 bits

@dataclass
class KV8(_View):
    """A cc_kv8 view (E4M3 codes, E8M0 scales) plus the tensors it points at."""
    struct: c_kv8
    keep: list = field(default_factory=list)


def _kv8(codes: KV, k_scale: torch.Tensor, v_scale: torch.Tensor, scale_block: int, seq: int,
         layer: int, head: int, page: int) -> KV8:
    for t in (*codes.keep[:2], k_scale, v_scale):
        if t.element_size() != 1:
            raise ValueError(f"codes and scales are bytes, got {t.dtype}")
    s = c_kv8()
    s.codes = codes.struct
    s.k_scale, s.v_scale = k_scale.data_ptr(), v_scale.data_ptr()
    s.scale_seq_stride, s.scale_layer_stride, s.scale_head_stride, s.scale_page_stride = seq, layer, head, page
    s.scale_block = scale_block
    return KV8(s, [codes, k_scale, v_scale])


def kv8_contiguous(k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor, *,
                   n_layers: int, layer_stride: int, head_stride: int, tok_stride: int, scale_block: int,
                   scale_layer_stride: int, scale_head_stride: int, seq_stride: int = 0,
                   scale_seq_stride: int = 0) -> KV8:
    """k, v: E4M3 codes, one byte an element (uint8 or float8_e4m3fn); scales: exponent bytes."""
    return _kv8(kv_contiguous(k, v, n_layers=n_layers, layer_stride=layer_stride, head_stride=head_stride,
                              tok_stride=tok_stride, seq_stride=seq_stride),
                k_scale, v_scale, scale_block, scale_seq_stride, scale_layer_stride, scale_head_stride, 0)


def kv8_paged(k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
              block_table: torch.Tensor, *, n_layers: int, layer_stride: int, page_stride: int,
              head_stride: int, tok_stride: int, page_size: int, scale_block: int,
              scale_layer_stride: int, scale_page_stride: int, scale_head_stride: int) -> KV8:
    return _kv8(kv_paged(k, v, block_table, n_layers=n_layers, layer_stride=layer_stride,
                         page_stride=page_stride, head_stride=head_stride, tok_stride=tok_stride,
                         page_size=page_size),
                k_scale, v_scale, scale_block, 0, scale_layer_stride, scale_head_stride, scale_page_stride)


def _rows(r: c_rows, t: torch.Tensor, dtype: torch.dtype, what: str, want: tuple) -> None:
    """The view of rows t, of shape `want` ([M][heads][head_dim], or with layers in front), in any strides."""
    if t.dtype != dtype:
        raise ValueError(f"{what} is {t.dtype}, the problem {dtype}")
    if t.shape != want:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {want}")
    st = t.stride()
    if st[-1] != 1:
        raise ValueError(f"rows of {what} must be contiguous")
    r.base = t.data_ptr()
    # (what strides lead over a single element says nothing)
    r.tok_stride = st[-3] if want[-3] > 1 else 0
    r.head_stride = st[-2] if want[-2] > 1 else 0
    r.layer_stride = st[0] if len(st) == 4 and want[0] > 1 else 0


def _empty(shape, dtype: torch.dtype, device, stream=None) -> torch.Tensor:
    """torch.empty for a call on `stream`: the memory is that stream's, so neither what the current stream
    still does with a block it has freed nor what it is given after this one's release can meet the call."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _on_gpu(*tensors) -> None:
    """Kernels run on the current device: tensors (and cache views) elsewhere would be read there by address."""
    found = {t.get_device() for t in tensors if t is not None}   # negative: not on a GPU
    found.discard(None)
    if not found:
        return
    if min(found) < 0:
        raise ValueError("tensors must be on the GPU")
    if len(found) > 1:
        raise ValueError("tensors on different devices")
    here = found.pop()
    if here != torch._C._cuda_getDevice():
        raise ValueError(f"tensors are on cuda:{here}, the current device is cuda:{torch._C._cuda_getDevice()}")


def _codes(kv) -> Optional[torch.Tensor]:
    """The keys of a cache view, which say where it lies."""
    codes = kv.keep[0] if kv.keep else None
    return codes.keep[0] if isinstance(codes, KV) else codes


def _int32(t: Optional[torch.Tensor], n: int, what: str) -> None:
    if t is not None and (t.dtype != torch.int32 or t.numel() != n or not t.is_contiguous()):
        raise ValueError(f"{what} must be {n} contiguous int32 values")


def _append(fn, p: Problem, kv, k, v, cached, capacity, layer, n_layers, pos_ids, q, q_out, rotate, stream):
    s = p.struct
    n_seqs, d, hkv = s.n_seqs, s.head_dim, s.n_heads_kv
    M = s.cu_seqlens_h[n_seqs]
    dtype = _DTYPES[s.dtype]
    _int32(cached, n_seqs, "cached")
    _int32(pos_ids, M, "pos_ids")
    if isinstance(kv, KV) and kv.keep:   # (8-bit views are of bytes already)
        for t in kv.keep[:2]:
            if t.dtype != dtype:
                raise ValueError(f"the cache holds {t.dtype}, the problem {dtype}")
    a = c_append()
    # one layer may come without its dimension
    want = (n_layers, M, hkv, d) if n_layers != 1 or k.dim() == 4 else (M, hkv, d)
    _rows(a.k, k, dtype, "k", want)
    _rows(a.v, v, dtype, "v", want)
    if q is not None:
        hq = s.n_heads_q
        _rows(a.q, q, dtype, "q", (M, hq, d))
        if q_out is None:
            q_out = _empty((M, hq, d), dtype, q.device, stream)
        elif q_out.dtype != dtype or q_out.numel() != M * hq * d or not q_out.is_contiguous():
            raise ValueError("q_out must be contiguous rows of q's type and size")
        a.q_out = q_out.data_ptr()
    _on_gpu(k, v, q, q_out, cached, pos_ids, p.cu_d, kv)
    a.cached = cached.data_ptr()
    if pos_ids is not None:
        a.pos_ids = pos_ids.data_ptr()
    a.capacity, a.layer, a.n_layers, a.rotate = capacity, layer, n_layers, int(rotate)
    _check(fn(ctypes.byref(s), ctypes.byref(a), ctypes.byref(kv.struct), _stream(stream)), fn.__name__)
    return q_out


def cc_append_kv(p: Problem, kv: KV, k: torch.Tensor, v: torch.Tensor, cached: torch.Tensor, *, capacity: int = 0,
                 layer: int = 0, n_layers: int = 1, pos_ids: Optional[torch.Tensor] = None,
                 q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, rotate: bool = True,
                 stream=None) -> Optional[torch.Tensor]:
    """Appends k, v [M][Hkv][d] (with n_layers > 1: [n_layers][M][Hkv][d]; any token and head strides) behind
    cached[b] entries of each sequence; p.cu_seqlens count the new tokens.  Returns the rotated queries
    where q [M][Hq][d] is given."""
    return _append(_lib.cc_append_kv, p, kv, k, v, cached, capacity, layer, n_layers, pos_ids, q, q_out, rotate, stream)


def cc_append_kv8(p: Problem, kv: KV8, k: torch.Tensor, v: torch.Tensor, cached: torch.Tensor, *, capacity: int = 0,
                  layer: int = 0, n_layers: int = 1, pos_ids: Optional[torch.Tensor] = None,
                  q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, rotate: bool = True,
                  stream=None) -> Optional[torch.Tensor]:
    """cc_append_kv into a cache in 8 bits."""
    return _append(_lib.cc_append_kv8, p, kv, k, v, cached, capacity, layer, n_layers, pos_ids, q, q_out, rotate, stream)


def cc_compact_kv8(p: Problem, kv: KV8, keep_idx: torch.Tensor, k: Sequence[int], per_head: int,
                   token_ids: Optional[torch.Tensor] = None, pos_ids: Optional[torch.Tensor] = None,
                   out: Optional[KV8] = None, stream=None) -> None:
    """cc_compact_kv on a cache in 8 bits (in place unless `out` is given)."""
    kk, n = _host_array(k, np.int32, _i32)
    if n != p.struct.n_seqs * (p.struct.n_heads_kv if per_head else 1):
        raise ValueError(f"{n} budgets for {p.struct.n_seqs} sequences")
    if keep_idx is not None and (keep_idx.dtype != torch.int32 or keep_idx.numel() < sum(k) or not keep_idx.is_contiguous()):
        raise ValueError(f"keep_idx must be {sum(k)} contiguous int32 values")
    N = p.struct.cu_seqlens_h[p.struct.n_seqs]
    for what, t in (("token_ids", token_ids), ("pos_ids", pos_ids)):
        if t is not None and (t.dtype != torch.int32 or t.numel() < N or not t.is_contiguous()):
            raise ValueError(f"{what} must be at least {N} contiguous int32 values")
    _on_gpu(keep_idx, token_ids, pos_ids, p.cu_d, kv, out)
    _check(_lib.cc_compact_kv8(ctypes.byref(p.struct), ctypes.byref(kv.struct), _ptr(keep_idx), kk, per_head,
                               _ptr(token_ids), _ptr(pos_ids),
                               ctypes.byref(out.struct) if out is not None else None, _stream(stream)),
           "cc_compact_kv8")


_MASKS = {"causal": CC_MASK_CAUSAL, "counter": CC_MASK_COUNTER_CAUSAL}


def cc_attention_kv8_workspace(p: Problem, mask: str, max_kv_len: int) -> int:
    return _query(_lib.cc_attention_kv8_workspace, ctypes.byref(p.struct), _MASKS[mask], max_kv_len)


def cc_attention_kv8(p: Problem, q: torch.Tensor, kv: KV8, layer: int, kv_lens: torch.Tensor, max_kv_len: int,
                     o: Optional[torch.Tensor] = None, *, mask: str = "causal",
                     workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of the queries q [N][Hq][d] (p.cu_seqlens count them) over a cache in 8 bits that holds
    kv_lens[b] entries of each sequence, the queries' own last; mask "causal" or "counter"."""
    s = p.struct
    n_seqs = s.n_seqs
    _int32(kv_lens, n_seqs, "kv_lens")
    if (q.dtype != torch.bfloat16 or q.numel() != s.cu_seqlens_h[n_seqs] * s.n_heads_q * s.head_dim
            or not q.is_contiguous()):
        raise ValueError("q must be contiguous bf16 rows [N][Hq][head_dim]")
    if o is None:
        o = _empty(q.shape, q.dtype, q.device, stream)
    elif o.dtype != q.dtype or o.numel() != q.numel() or not o.is_contiguous():
        raise ValueError("o must be contiguous and of q's type and size")
    _on_gpu(q, o, kv_lens, workspace, p.cu_d, kv)
    if workspace is None:
        workspace = _empty(max(1, cc_attention_kv8_workspace(p, mask, max_kv_len)), torch.uint8, q.device, stream)
    _check(_lib.cc_attention_kv8(ctypes.byref(s), _ptr(q), ctypes.byref(kv.struct), layer, _MASKS[mask],
                                 _ptr(kv_lens), max_kv_len, _ptr(o), _ptr(workspace), workspace.numel(),
                                 _stream(stream)), "cc_attention_kv8")
    return o

# ---------------------------------------------------------------- attention over a bf16 cache

def cc_attention_kv_workspace(p: Problem, max_kv_len: int) -> int:
    return _query(_lib.cc_attention_kv_workspace, ctypes.byref(p.struct), max_kv_len)


def _queries(p: Problem, q: torch.Tensor, kv: KV, kv_lens: torch.Tensor) -> None:
    s = p.struct
    _int32(kv_lens, s.n_seqs, "kv_lens")
    if (q.dtype != torch.bfloat16 or q.numel() != s.cu_seqlens_h[s.n_seqs] * s.n_heads_q * s.head_dim
            or not q.is_contiguous()):
        raise ValueError("q must be contiguous bf16 rows [N][Hq][head_dim]")
    _bf16_cache(kv)
    _rows_of_pages(kv, s.n_seqs)


def _rows_of_pages(kv: KV, n: int) -> None:
    if len(kv.keep) > 2 and kv.keep[2].shape[0] < n:
        raise ValueError(f"the block table has {kv.keep[2].shape[0]} rows, expected {n}")


def _bf16_cache(kv: KV) -> None:
    if getattr(kv, "_bf16", False):   # (a view's tensors stay what they are)
        return
    for t in kv.keep[:2]:
        if t.dtype != torch.bfloat16:
            raise ValueError(f"the cache holds {t.dtype}, expected bf16")
    kv._bf16 = True


def _lse(p: Problem, lse: Optional[torch.Tensor]) -> None:
    n = p.struct.cu_seqlens_h[p.struct.n_seqs] * p.struct.n_heads_q
    if lse is not None and (lse.dtype != torch.float32 or lse.numel() != n or not lse.is_contiguous()):
        raise ValueError(f"lse must be {n} contiguous float32 values [N][Hq]")


def cc_attention_kv(p: Problem, q: torch.Tensor, kv: KV, layer: int, kv_lens: torch.Tensor, max_kv_len: int,
                    o: Optional[torch.Tensor] = None, *, lse: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Causal attention of the queries q [N][Hq][d] (p.cu_seqlens count them) over a bf16 cache that holds
    kv_lens[b] entries of each sequence, the queries' own last; lse [N][Hq]: filled where given."""
    return _attention_kv(p, q, None, kv, layer, kv_lens, max_kv_len, o, lse, workspace, stream)


def _attention_kv(p, q, pre, kv, layer, kv_lens, max_kv_len, o, lse, workspace, stream):
    s = p.struct
    _queries(p, q, kv, kv_lens)
    _lse(p, lse)
    if o is None:
        o = _empty(q.shape, q.dtype, q.device, stream)
    elif o.dtype != q.dtype or o.numel() != q.numel() or not o.is_contiguous():
        raise ValueError("o must be contiguous and of q's type and size")
    _on_gpu(q, o, lse, kv_lens, workspace, p.cu_d, kv, pre)
    if workspace is None:
        need = cc_attention_kv_workspace(p, max_kv_len) if pre is None else cc_attention_prefix_workspace(p, pre, max_kv_len)
        workspace = _empty(max(1, need), torch.uint8, q.device, stream)
    out = (_ptr(o), _ptr(lse), _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream))
    if pre is None:
        _check(_lib.cc_attention_kv(ctypes.byref(s), _ptr(q), ctypes.byref(kv.struct), layer, _ptr(kv_lens), max_kv_len,
                                    *out), "cc_attention_kv")
    else:
        _check(_lib.cc_attention_prefix(ctypes.byref(s), _ptr(q), ctypes.byref(pre.struct), ctypes.byref(kv.struct), layer,
                                        _ptr(kv_lens), max_kv_len, *out), "cc_attention_prefix")
    return o


@dataclass
class Prefix(_View):
    """A cc_prefix plus the tensors it points at (first_h on the host)."""
    struct: c_prefix
    keep: list = field(default_factory=list)
    first_h: Optional[torch.Tensor] = None


def prefix(kv: KV, first_seq: Sequence[int], lens: torch.Tensor, max_len: int,
           first_device: Optional[torch.Tensor] = None) -> Prefix:
    """Prefixes that runs of sequences share: "sequence" i of the view kv, of lens[i] entries (device, int32), is
    before the sequences first_seq[i] .. first_seq[i + 1] - 1.  first_device: the int32 values of first_seq already
    on the device (the default copies them there and waits for the copy)."""
    n = len(first_seq) - 1
    if n < 1:
        raise ValueError("first_seq holds where each prefix's sequences start, and where the last one's end")
    _int32(lens, n, "lens")
    _bf16_cache(kv)
    _rows_of_pages(kv, n)
    first_h = torch.as_tensor(list(first_seq), dtype=torch.int32).contiguous()
    if first_device is None:
        first_d = first_h.to(lens.device)
    elif (first_device.dtype != torch.int32 or first_device.shape != first_h.shape or not first_device.is_contiguous()):
        raise ValueError("first_device must hold the values of first_seq as contiguous int32")
    else:
        first_d = first_device
    s = c_prefix()
    s.kv, s.n_prefixes, s.max_len = kv.struct, n, max_len
    s.first_seq_h = ctypes.cast(first_h.data_ptr(), ctypes.POINTER(_i32))
    s.first_seq_d, s.lens = first_d.data_ptr(), lens.data_ptr()
    return Prefix(s, [kv, lens, first_d], first_h)


def cc_attention_prefix_workspace(p: Problem, prefix: Prefix, max_kv_len: int) -> int:
    return _query(_lib.cc_attention_prefix_workspace, ctypes.byref(p.struct), ctypes.byref(prefix.struct), max_kv_len)


def cc_attention_prefix(p: Problem, q: torch.Tensor, prefix: Prefix, kv: KV, layer: int, kv_lens: torch.Tensor,
                        max_kv_len: int, o: Optional[torch.Tensor] = None, *, lse: Optional[torch.Tensor] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """cc_attention_kv of sequences behind shared prefixes; kv, kv_lens and max_kv_len are their own entries'."""
    return _attention_kv(p, q, prefix, kv, layer, kv_lens, max_kv_len, o, lse, workspace, stream)


# ---------------------------------------------------------------- eviction by attention weight

def _weights(p: Problem, w: torch.Tensor, what: str, longest: int, written: bool = False) -> c_weights:
    """The view of weights w [n_seqs][Hkv][entries], entries contiguous; where they are written rows may not overlap."""
    s = p.struct
    if w.dtype != torch.float32:
        raise ValueError(f"{what} is {w.dtype}, expected float32")
    shape = w.shape
    if len(shape) != 3 or shape[0] != s.n_seqs or shape[1] != s.n_heads_kv or shape[2] < longest:
        raise ValueError(f"{what} has shape {tuple(shape)}, expected {(s.n_seqs, s.n_heads_kv)} and at least {longest} entries")
    seq, head, entry = w.stride()
    if not w.is_contiguous():
        if shape[2] > 1 and entry != 1:
            raise ValueError(f"entries of {what} must be contiguous")
        at = sorted((st, n) for st, n in zip((seq, head, entry), shape) if n > 1)
        if written and any(up < st * n for (st, n), (up, _) in zip(at, at[1:])):
            raise ValueError(f"{what} overlaps itself (strides {w.stride()})")
    return c_weights(w.data_ptr(), seq if shape[0] > 1 else 0, head if shape[1] > 1 else 0, shape[2])


def cc_attention_weights_workspace(p: Problem, max_kv_len: int) -> int:
    return _query(_lib.cc_attention_weights_workspace, ctypes.byref(p.struct), max_kv_len)


def cc_attention_weights(p: Problem, q: torch.Tensor, kv: KV, layer: int, kv_lens: torch.Tensor, max_kv_len: int,
                         lse: torch.Tensor, out: torch.Tensor, *, prev: Optional[torch.Tensor] = None,
                         prev_lens: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """What each entry receives of the attention of q [N][Hq][d] (lse [N][Hq] as cc_attention_kv filled it), added to
    prev where that is given (of the first prev_lens[b] entries, as far as prev goes; all without): out
    [n_seqs][Hkv][entries], which may be prev."""
    s = p.struct
    _queries(p, q, kv, kv_lens)
    _lse(p, lse)
    _int32(prev_lens, s.n_seqs, "prev_lens")
    if prev is None and prev_lens is not None:
        raise ValueError("prev_lens without prev")
    to = _weights(p, out, "out", max_kv_len, True)
    had = _weights(p, prev, "prev", 0 if prev_lens is not None else max_kv_len) if prev is not None else None
    _on_gpu(q, lse, out, prev, prev_lens, kv_lens, workspace, p.cu_d, kv)
    if workspace is None:
        workspace = _empty(max(1, cc_attention_weights_workspace(p, max_kv_len)), torch.uint8, q.device, stream)
    _check(_lib.cc_attention_weights(ctypes.byref(s), _ptr(q), ctypes.byref(kv.struct), layer, _ptr(kv_lens), max_kv_len,
                                     _ptr(lse), ctypes.byref(had) if had is not None else None, _ptr(prev_lens),
                                     ctypes.byref(to), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(stream)), "cc_attention_weights")
    return out


def cc_weight_scores(p: Problem, w: torch.Tensor, n_recent: int, per_head: int, scores: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """Scores for cc_select_keep from weights w [n_seqs][Hkv][entries] (p.cu_seqlens count the entries): one segment for
    each sequence, or with per_head for each of its KV heads; the first p.n_frozen and the last n_recent are +inf (more of these than a budget: the first
    ones of them are kept)."""
    s = p.struct
    view = _weights(p, w, "w", p.longest)
    n = s.cu_seqlens_h[s.n_seqs] * (s.n_heads_kv if per_head else 1)
    if scores is None:
        scores = _empty((n,), torch.float32, w.device, stream)
    elif scores.dtype != torch.float32 or scores.numel() < n or not scores.is_contiguous():
        raise ValueError(f"scores must be at least {n} contiguous float32 values")
    _on_gpu(w, scores, p.cu_d)
    _check(_lib.cc_weight_scores(ctypes.byref(s), ctypes.byref(view), n_recent, int(per_head), _ptr(scores),
                                 _stream(stream)), "cc_weight_scores")
    return scores


def cc_compact_weights(p: Problem, w: torch.Tensor, keep_idx: torch.Tensor, k: Sequence[int], per_head: int,
                       out: Optional[torch.Tensor] = None, stream=None) -> None:
    """The weights of the kept entries, moved to the front of w [n_seqs][Hkv][entries] (or of out)."""
    s = p.struct
    kk, n = _host_array(k, np.int32, _i32)
    if n != s.n_seqs * (s.n_heads_kv if per_head else 1):
        raise ValueError(f"{n} budgets for {s.n_seqs} sequences")
    if keep_idx is not None and (keep_idx.dtype != torch.int32 or keep_idx.numel() < sum(k) or not keep_idx.is_contiguous()):
        raise ValueError(f"keep_idx must be {sum(k)} contiguous int32 values")
    src = _weights(p, w, "w", p.longest, out is None)
    dst = _weights(p, out, "out", max(k, default=0), True) if out is not None else None
    _on_gpu(w, keep_idx, out, p.cu_d)
    _check(_lib.cc_compact_weights(ctypes.byref(s), ctypes.byref(src), _ptr(keep_idx), kk, int(per_head),
                                   ctypes.byref(dst) if dst is not None else None, _stream(stream)), "cc_compact_weights")


# ---------------------------------------------------------------- log-probabilities

@dataclass
class Logprobs:
    """Outputs of cc_lmhead_logprobs: [n] (None where no ids were given), [n], [n][top], [n][top]."""
    logprob: Optional[torch.Tensor]
    entropy: torch.Tensor
    top_ids: torch.Tensor
    top_logprob: torch.Tensor


def logprobs_out(n: int, top: int, device="cuda", stream=None, ids: bool = True) -> Logprobs:
    """Tensors for a call of n rows; ids: False for one that is given no words."""
    f = lambda *s: _empty(s, torch.float32, device, stream)
    return Logprobs(f(n) if ids else None, f(n), _empty((n, top), torch.int32, device, stream), f(n, top))


def cc_lmhead_logprobs_workspace(dtype: str, n: int, vocab: int, hidden: int, top: int) -> int:
    return _query(_lib.cc_lmhead_logprobs_workspace, {"f32": CC_F32, "bf16": CC_BF16}[dtype], n, vocab, hidden, top)


def cc_lmhead_logprobs(dtype: str, u: torch.Tensor, w_lm: torch.Tensor, vocab: int, ids: Optional[torch.Tensor],
                       top: int, out: Optional[Logprobs] = None, *, packed: bool = False,
                       workspace: Optional[torch.Tensor] = None, stream=None) -> Logprobs:
    """Log-probabilities of ids [n] (None: not taken, the result has none and out.logprob is left as it is),
    entropies and `top` alternatives of each hidden row u [n][hidden] under the LM head w_lm [vocab][hidden]
    (packed: in the layout of cc_pack_lmhead)."""
    n, hidden = u.shape
    _int32(ids, n, "ids")
    if not u.is_contiguous() or not w_lm.is_contiguous():
        raise ValueError("u and w_lm must be contiguous")
    if u.dtype != torch.bfloat16 or (not packed and w_lm.dtype != torch.bfloat16):
        raise ValueError("u and w_lm must be bf16")
    if not packed and tuple(w_lm.shape) != (vocab, hidden):
        raise ValueError(f"w_lm has shape {tuple(w_lm.shape)}, expected {(vocab, hidden)}")
    if packed and w_lm.numel() * w_lm.element_size() < cc_pack_lmhead_bytes(vocab, hidden):
        raise ValueError("w_lm holds less than a packed weight of that size")
    if out is None:
        out = logprobs_out(n, top, u.device, stream, ids is not None)
    elif ids is None:
        out = Logprobs(None, out.entropy, out.top_ids, out.top_logprob)
    if out.top_ids.numel() < n * top or out.top_logprob.numel() < n * top:
        raise ValueError(f"out has no room for {top} alternatives of {n} rows (top_ids, top_logprob)")
    f32 = torch.float32
    for what, t, m, want in (("logprob", out.logprob, n, f32), ("entropy", out.entropy, n, f32),
                             ("top_ids", out.top_ids, n * top, torch.int32),
                             ("top_logprob", out.top_logprob, n * top, f32)):
        if what == "logprob" and ids is None:
            continue
        if t is None or t.dtype != want or t.numel() < m or not t.is_contiguous():
            raise ValueError(f"{what} must be at least {m} contiguous {want} values")
    _on_gpu(u, w_lm, ids, out.logprob, out.entropy, out.top_ids, out.top_logprob, workspace)
    if workspace is None:
        workspace = _empty(max(1, cc_lmhead_logprobs_workspace(dtype, n, vocab, hidden, top)), torch.uint8, u.device, stream)
    _check(_lib.cc_lmhead_logprobs({"f32": CC_F32, "bf16": CC_BF16}[dtype], _ptr(u), _ptr(w_lm), int(packed), n,
                                   vocab, hidden, _ptr(ids), top, _ptr(out.logprob),
                                   _ptr(out.entropy), _ptr(out.top_ids) if top else None,
                                   _ptr(out.top_logprob) if top else None, _ptr(workspace), workspace.numel(),
                                   _stream(stream)), "cc_lmhead_logprobs")
    return out
