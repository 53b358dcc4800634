"""ctypes binding of libadore.so: the same calls as include/adore.h, argument marshalling only.

torch is used for device memory and the stream; every step of the path runs in
the library's HIP kernels.  There is no fallback: if the library is missing or
a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libadore.so")

ADORE_F32, ADORE_BF16 = 0, 1
KERNELS = ["attend", "attend_combine", "ctrl_input", "ctrl_cell", "release", "rebuild_select", "rebuild_gemm",
           "rescore", "fwd_qkv", "fwd_qkv_cur", "fwd_attend", "fwd_oproj", "fwd_oproj_cur", "rope", "h2o_release",
           "h2o_choice", "h2o_place"]
SCORE_STATIC, SCORE_RESCORE, SCORE_H2O = 0, 1, 2

EXPORTS = [
    "adore_workspace_bytes", "adore_create", "adore_destroy", "adore_init_cache", "adore_attend",
    "adore_schedule", "adore_rebuild", "adore_decode_step", "adore_forward_step", "adore_get_state", "adore_set_state",
    "adore_set_input_order", "adore_check_guards", "adore_set_timing", "adore_read_timing", "adore_kernel_name", "adore_strerror", "adore_abi_version",
    "adore_topk_attention_workspace_bytes", "adore_topk_attention", "adore_topk_attention_static",
    "adore_prompt_attention", "adore_prompt_backward_workspace_bytes", "adore_prompt_attention_backward", "adore_prompt_scores",
]

EXPORTS_Q4 = ["adore_q4_cache_bytes", "adore_q4_workspace_bytes", "adore_q4_fill", "adore_q4_step", "adore_q4_read"]


class AdoreConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("layers", "batch", "heads", "head_dim", "hidden", "cache_slots", "rebuild_budget",
                 "max_positions", "ctrl_hidden", "dtype")] + [("pos_scale", ctypes.c_float),
                                                              ("score_mode", ctypes.c_int32),
                                                              ("rope_base", ctypes.c_float)]


_WEIGHT_FIELDS = ["w_kv", "gru_w_ih", "gru_w_hh", "gru_b_ih", "gru_b_hh", "pos_w", "pos_b", "mlp_w1",
                  "mlp_b1", "out_w", "out_b"]


class AdoreWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in _WEIGHT_FIELDS]


class AdoreForwardWeights(ctypes.Structure):
    _fields_ = [("w_q", ctypes.c_void_p), ("w_o", ctypes.c_void_p)]


class AdorePromptConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("batch", "heads", "kv_heads", "head_dim", "q_tokens", "k_tokens", "dtype")] + [("scale", ctypes.c_float)]


class AdoreQ4Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("batch", "heads", "kv_heads", "head_dim", "slots", "recent", "dtype")] + [("scale", ctypes.c_float)]


class AdoreRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in ("seq", "token", "head")]


class AdoreError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"adore error {code}: {msg}")
        self.code = code


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads libadore.so from the package directory.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} not found: build it with `python -m paper_2407_02328_amd.build` "
            "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    lib.adore_workspace_bytes.restype = sz
    lib.adore_workspace_bytes.argtypes = [ctypes.POINTER(AdoreConfig)]
    lib.adore_create.restype = ctypes.c_int
    lib.adore_create.argtypes = [ctypes.POINTER(AdoreConfig), ctypes.POINTER(AdoreWeights), vp, sz, vp,
                                 ctypes.POINTER(vp)]
    lib.adore_destroy.restype = ctypes.c_int
    lib.adore_destroy.argtypes = [vp]
    lib.adore_init_cache.restype = ctypes.c_int
    lib.adore_init_cache.argtypes = [vp, vp, vp, vp, vp, vp, i32]
    lib.adore_attend.restype = ctypes.c_int
    lib.adore_attend.argtypes = [vp, i32, vp, vp, vp, vp]
    lib.adore_schedule.restype = ctypes.c_int
    lib.adore_schedule.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.adore_rebuild.restype = ctypes.c_int
    lib.adore_rebuild.argtypes = [vp, i32, vp]
    lib.adore_decode_step.restype = ctypes.c_int
    lib.adore_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.adore_forward_step.restype = ctypes.c_int
    lib.adore_forward_step.argtypes = [vp, ctypes.POINTER(AdoreForwardWeights), vp, vp, vp, vp, vp, vp, vp]
    lib.adore_get_state.restype = ctypes.c_int
    lib.adore_get_state.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.POINTER(i32)]
    lib.adore_set_state.restype = ctypes.c_int
    lib.adore_set_state.argtypes = [vp, vp, vp, vp, vp, vp, i32]
    lib.adore_set_input_order.restype = ctypes.c_int
    lib.adore_set_input_order.argtypes = [vp, i32]
    lib.adore_set_timing.restype = ctypes.c_int
    lib.adore_set_timing.argtypes = [vp, i32]
    lib.adore_read_timing.restype = ctypes.c_int
    lib.adore_read_timing.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(i32)]
    lib.adore_kernel_name.restype = ctypes.c_char_p
    lib.adore_kernel_name.argtypes = [i32]
    lib.adore_strerror.restype = ctypes.c_char_p
    lib.adore_strerror.argtypes = [ctypes.c_int]
    lib.adore_check_guards.restype = ctypes.c_int
    lib.adore_check_guards.argtypes = [vp, ctypes.POINTER(ctypes.c_int32)]
    lib.adore_abi_version.restype = ctypes.c_int
    lib.adore_abi_version.argtypes = []
    lib.adore_topk_attention_workspace_bytes.restype = sz
    lib.adore_topk_attention_workspace_bytes.argtypes = [i32, i32, i32]
    lib.adore_topk_attention.restype = ctypes.c_int
    lib.adore_topk_attention.argtypes = [vp, vp, vp, vp, vp, sz, i32, i32, i32, i32, vp]
    lib.adore_topk_attention_static.restype = ctypes.c_int
    lib.adore_topk_attention_static.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp]
    cfg, rows = ctypes.POINTER(AdorePromptConfig), ctypes.POINTER(AdoreRows)
    lib.adore_prompt_attention.restype = ctypes.c_int
    lib.adore_prompt_attention.argtypes = [cfg, vp, vp, rows, rows, rows, rows, vp, rows, vp]
    lib.adore_prompt_backward_workspace_bytes.restype = sz
    lib.adore_prompt_backward_workspace_bytes.argtypes = [cfg, i32]
    lib.adore_prompt_attention_backward.restype = ctypes.c_int
    lib.adore_prompt_attention_backward.argtypes = [cfg, vp, vp] + [rows] * 6 + [vp] + [rows] * 3 + [vp, sz, vp]
    lib.adore_prompt_scores.restype = ctypes.c_int
    lib.adore_prompt_scores.argtypes = [cfg, vp, vp, rows, rows, vp, vp, vp]
    q4 = ctypes.POINTER(AdoreQ4Config)
    lib.adore_q4_cache_bytes.restype = lib.adore_q4_workspace_bytes.restype = sz
    lib.adore_q4_cache_bytes.argtypes = lib.adore_q4_workspace_bytes.argtypes = [q4]
    lib.adore_q4_fill.restype = lib.adore_q4_step.restype = lib.adore_q4_read.restype = ctypes.c_int
    lib.adore_q4_fill.argtypes = [q4, vp, i32, rows, rows] + [vp] * 6
    lib.adore_q4_step.argtypes = [q4] + [vp] * 11 + [sz, vp]
    lib.adore_q4_read.argtypes = [q4] + [vp] * 5
    _lib = lib
    return lib


def _check(lib, rc: int):
    if rc != 0:
        raise AdoreError(rc, lib.adore_strerror(rc).decode())


def make_config(*, layers, batch, heads, head_dim, hidden, cache_slots, rebuild_budget, max_positions,
                ctrl_hidden, dtype, pos_scale, score_mode=0, rope_base=0.0) -> AdoreConfig:
    code = {"f32": ADORE_F32, "bf16": ADORE_BF16}[dtype] if isinstance(dtype, str) else int(dtype)
    return AdoreConfig(layers, batch, heads, head_dim, hidden, cache_slots, rebuild_budget, max_positions,
                       ctrl_hidden, code, pos_scale, int(score_mode), float(rope_base))


def topk_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, top_k: int, out: torch.Tensor = None,
                   workspace: torch.Tensor = None) -> torch.Tensor:
    """adore_topk_attention on torch's current stream.  q, k, v: [rows, seq, head_dim] bf16, contiguous, on the GPU;
    out and workspace (uint8) are allocated here unless given."""
    lib = load_library()
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.shape != q.shape or t.dim() != 3:
            raise ValueError(f"{name}: expected a contiguous bf16 GPU tensor [rows, seq, head_dim]")
    rows, seq, d = q.shape
    if out is None:
        out = torch.empty_like(q)
    elif out.dtype != torch.bfloat16 or not out.is_contiguous() or out.shape != q.shape or out.device != q.device:
        raise ValueError("out: expected a contiguous bf16 tensor like q")
    need = lib.adore_topk_attention_workspace_bytes(rows, seq, d)
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=q.device)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != q.device:
        raise ValueError("workspace: expected a contiguous uint8 tensor on q's device")
    stream = torch.cuda.current_stream(q.device).cuda_stream
    _check(lib, lib.adore_topk_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), workspace.data_ptr(),
                                         workspace.numel(), rows, seq, d, int(top_k), stream))
    return out


def topk_attention_static(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, top_k: int, out: torch.Tensor) -> torch.Tensor:
    """adore_topk_attention_static on torch's current stream: no workspace, nothing allocated (out is the caller's)."""
    lib = load_library()
    for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.shape != q.shape or t.dim() != 3:
            raise ValueError(f"{name}: expected a contiguous bf16 GPU tensor [rows, seq, head_dim]")
    rows, seq, d = q.shape
    stream = torch.cuda.current_stream(q.device).cuda_stream
    _check(lib, lib.adore_topk_attention_static(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), rows, seq, d,
                                                int(top_k), stream))
    return out


_CODES = {torch.float32: ADORE_F32, torch.bfloat16: ADORE_BF16}


# torch's current stream of a device as a number (torch.cuda.current_stream makes an object of it, 2 us)
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
# ... and the current device as one (torch.cuda.current_device looks first whether torch is initialised; who has a GPU tensor knows)
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(lib, index: int, function, *args):
    """A call of the library whose kernels go to the current device, which has to be that of its tensors."""
    if _current() == index:
        rc = function(*args)
    else:
        with torch.cuda.device(index):
            rc = function(*args)
    _check(lib, rc)


class _Prompts:
    """The sequences and heads of a call on prompts, read off q and k, and its tensors' descriptions.

    With starts, q is [q tokens, heads, head_dim] and k [k tokens, kv heads, head_dim]; without, [batch, heads, tokens, head_dim].
    The last dimension is dense, the others may have any strides that keep every row on a 16-byte boundary."""

    def __init__(self, q: torch.Tensor, k: torch.Tensor, q_start, k_start, scale):
        # (once or twice a call, rows() up to twelve times: what short prompts take the GPU is not much more)
        if (q_start is None) != (k_start is None):
            raise ValueError("q_start and k_start: both or neither")
        code = _CODES.get(q.dtype)
        index = q.get_device()
        if code is None or index < 0:
            raise ValueError(f"q: expected a bf16 or fp32 GPU tensor, got {q.device} {q.dtype}")
        self.device, self.index, self.dtype = q.device, index, q.dtype
        self.q_shape, self.k_shape = qs, ks = q.shape, k.shape
        self.q_odd, self.k_odd = 1 in qs or 0 in qs, 1 in ks or 0 in ks
        self.packed = packed = q_start is not None
        if len(qs) != (3 if packed else 4) or len(ks) != len(qs):
            raise ValueError("q, k: expected [tokens, heads, head_dim] with starts, [batch, heads, tokens, head_dim] without")
        # (the kernels go by q's sequences and elements; rows() holds v and the gradients to k's shape)
        if ks[-1] != qs[-1] or (not packed and ks[0] != qs[0]):
            raise ValueError(f"k: expected q's {'' if packed else f'{qs[0]} sequences and '}{qs[-1]} elements, got shape {tuple(ks)}")
        if scale is None:
            scale = 0.0
        elif not scale > 0.0:
            raise ValueError("scale: expected a positive number")
        if packed:
            for name, t in (("q_start", q_start), ("k_start", k_start)):
                if t.dtype is not torch.int32 or t.get_device() != index or t.dim() != 1 or not t.is_contiguous() or t.numel() < 2 or \
                        t.numel() != q_start.numel():
                    raise ValueError(f"{name}: expected contiguous int32 [batch + 1] on q's device")
            self.starts = (q_start.data_ptr(), k_start.data_ptr())
            self.batch = q_start.numel() - 1
            self.cfg = AdorePromptConfig(self.batch, qs[1], ks[1], qs[2], qs[0], ks[0], code, scale)
            self.q_rows, self.k_rows = (qs[1], qs[0]), (ks[1], ks[0])      # of one value per row: lse
        else:
            self.starts = (None, None)
            self.batch = qs[0]
            self.cfg = AdorePromptConfig(self.batch, qs[1], ks[1], qs[3], qs[2], ks[2], code, scale)
            self.q_rows, self.k_rows = qs[:3], ks[:3]

    def rows(self, t: torch.Tensor, shape, name: str, written: bool = False):
        # (sizes of 1 and 0, whose strides mean nothing, are looked for once a shape)
        if not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype is not self.dtype or t.get_device() != self.index:
            raise ValueError(f"{name}: expected a {self.dtype} tensor of shape {tuple(shape)} on {self.device}")
        stride = t.stride()
        odd = self.q_odd if shape is self.q_shape else self.k_odd
        if odd or stride[-1] != 1 or 0 in stride:
            if shape[-1] > 1 and stride[-1] != 1:
                raise ValueError(f"{name}: its last dimension has to be dense")
            stride = tuple(0 if n <= 1 else s for n, s in zip(shape, stride))      # of one row: any
            if written and any(n > 1 and s == 0 for n, s in zip(shape, stride)):
                raise ValueError(f"{name}: its rows lie on one another")
        ptr = t.data_ptr() or 16               # (an empty tensor has no address, and no row of it is touched)
        if self.packed:
            return ctypes.byref(AdoreRows(ptr, 0, stride[0], stride[1]))
        return ctypes.byref(AdoreRows(ptr, stride[0], stride[2], stride[1]))

    def fresh(self, t: torch.Tensor):
        """Rows of a tensor that has just been made for a call: dense, and as it should be."""
        shape = t.shape
        if self.packed:
            return ctypes.byref(AdoreRows(t.data_ptr() or 16, 0, shape[1] * shape[2], shape[2]))
        head = shape[2] * shape[3]
        return ctypes.byref(AdoreRows(t.data_ptr() or 16, shape[1] * head, shape[3], head))

    def values(self, t: torch.Tensor, shape, name: str):
        if not isinstance(t, torch.Tensor) or t.shape != shape or t.dtype is not torch.float32 or t.get_device() != self.index or \
                not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous fp32 of shape {tuple(shape)} on {self.device}")
        return t.data_ptr() or 16

    @property
    def stream(self):
        return _stream(self.index)


def prompt_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, q_start: torch.Tensor = None,
                     k_start: torch.Tensor = None, scale: float = None, out: torch.Tensor = None, rest: bool = False):
    """adore_prompt_attention on torch's current stream: causal attention over whole prompts; returns (out, lse), and with rest=True
    (out, lse, rest) for the backward pass (rest is None where out is fp32 and nothing is lost).

    Packed sequences: q [q tokens, heads, head_dim], k and v [k tokens, kv heads, head_dim], q_start and k_start int32
    [batch + 1] on the GPU.  A dense batch: [batch, heads, tokens, head_dim] without starts.  bf16 or fp32, any strides with a
    dense last dimension (q, k and v may be views of one projection).  out is allocated here unless given.

    Where q, k or v require gradients, out has them: torch's backward pass is prompt_attention_backward (once; lse and rest have
    none, and out cannot be given then).  A step that is captured into a graph calls the two itself, under torch.no_grad()."""
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or (isinstance(v, torch.Tensor) and v.requires_grad)):
        if out is not None:
            raise ValueError("out: cannot be given where gradients are required (call under torch.no_grad())")
        got = _PromptAttention.apply(q, k, v, q_start, k_start, scale, rest)
    else:
        got = _attend_prompts(q, k, v, q_start, k_start, scale, out, rest)
    return got if rest else got[:2]


def _attend_prompts(q, k, v, q_start, k_start, scale, out, rest):
    lib = load_library()
    p = _Prompts(q, k, q_start, k_start, scale)
    rows = None
    if out is None:
        out = torch.empty(p.q_shape, dtype=q.dtype, device=p.device)
        rows = p.fresh(out)
    lse = torch.empty(p.q_rows, dtype=torch.float32, device=p.device)
    left = torch.empty(p.q_shape, dtype=q.dtype, device=p.device) if rest and q.dtype == torch.bfloat16 else None
    _call(lib, p.index, lib.adore_prompt_attention, ctypes.byref(p.cfg), *p.starts, p.rows(q, p.q_shape, "q"), p.rows(k, p.k_shape, "k"),
          p.rows(v, p.k_shape, "v"), rows or p.rows(out, p.q_shape, "out", True), lse.data_ptr() or 16, None if left is None else p.fresh(left),
          p.stream)
    return out, lse, left


class _PromptAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_start, k_start, scale, rest):
        out, lse, left = _attend_prompts(q, k, v, q_start, k_start, scale, None, rest)
        ctx.save_for_backward(q, k, v, out, lse, left, q_start, k_start)
        ctx.scale = scale
        ctx.mark_non_differentiable(*(x for x in (lse, left) if x is not None))
        ctx.set_materialize_grads(False)
        return out, lse, left

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_out, *_):
        if d_out is None:
            return (None,) * 7
        q, k, v, out, lse, left, q_start, k_start = ctx.saved_tensors
        # (whatever made d_out chose its layout: of a sum, one element for all)
        if d_out.stride(-1) != 1 or d_out.data_ptr() % 16 or any(s * d_out.element_size() % 16 for s in d_out.stride()[:-1]):
            d_out = d_out.clone(memory_format=torch.contiguous_format)
        grads = prompt_attention_backward(d_out, q, k, v, out, lse, rest=left, q_start=q_start, k_start=k_start, scale=ctx.scale)
        return *(g if want else None for g, want in zip(grads, ctx.needs_input_grad)), None, None, None, None


def prompt_attention_backward(d_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                              lse: torch.Tensor, *, rest: torch.Tensor = None, q_start: torch.Tensor = None,
                              k_start: torch.Tensor = None, scale: float = None, dq: torch.Tensor = None, dk: torch.Tensor = None,
                              dv: torch.Tensor = None):
    """adore_prompt_attention_backward on torch's current stream: (dq, dk, dv) of sum(d_out * out).  out, lse and rest as
    prompt_attention returned them for these q, k, v, starts and scale; dq, dk, dv are allocated here unless given (the places of
    q, k and v in the gradient of one projection, say)."""
    lib = load_library()
    p = _Prompts(q, k, q_start, k_start, scale)
    def gradient(t, shape, name):
        if t is not None:
            return t, p.rows(t, shape, name, True)
        t = torch.empty(shape, dtype=q.dtype, device=p.device)
        return t, p.fresh(t)

    (dq, dq_rows), (dk, dk_rows), (dv, dv_rows) = gradient(dq, p.q_shape, "dq"), gradient(dk, p.k_shape, "dk"), gradient(dv, p.k_shape, "dv")
    need = lib.adore_prompt_backward_workspace_bytes(ctypes.byref(p.cfg), int(p.packed))
    workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=q.device)
    _call(lib, p.index, lib.adore_prompt_attention_backward, ctypes.byref(p.cfg), *p.starts, p.rows(d_out, p.q_shape, "d_out"),
          p.rows(q, p.q_shape, "q"), p.rows(k, p.k_shape, "k"), p.rows(v, p.k_shape, "v"), p.rows(out, p.q_shape, "out"),
          None if rest is None else p.rows(rest, p.q_shape, "rest"), p.values(lse, p.q_rows, "lse"), dq_rows, dk_rows, dv_rows,
          workspace.data_ptr(), need, p.stream)
    return dq, dk, dv


def prompt_scores(q: torch.Tensor, k: torch.Tensor, lse: torch.Tensor, *, q_start: torch.Tensor = None, k_start: torch.Tensor = None,
                  scale: float = None, scores: torch.Tensor = None) -> torch.Tensor:
    """adore_prompt_scores on torch's current stream: the attention every key received from the queries of its group's heads, fp32
    [kv heads, k tokens] (packed) or [batch, kv heads, tokens].  lse as prompt_attention returned it.  They carry no gradients: what
    goes by them is a choice."""
    lib = load_library()
    p = _Prompts(q, k, q_start, k_start, scale)
    if scores is None:
        scores = torch.empty(p.k_rows, dtype=torch.float32, device=q.device)
    _call(lib, p.index, lib.adore_prompt_scores, ctypes.byref(p.cfg), *p.starts, p.rows(q, p.q_shape, "q"), p.rows(k, p.k_shape, "k"),
          p.values(lse, p.q_rows, "lse"), p.values(scores, p.k_rows, "scores"), p.stream)
    return scores


class Q4Cache:
    """A K/V cache held in 4 bits for `batch` sequences, evicted by the attention its rows received (adore_q4_* in include/adore.h):
    its buffers, and the calls on torch's current stream.  fill() loads prompts, step() takes one token of every sequence, read()
    gives the contents.  Buffers that are given are used as they are; others are made here, empty.

      cache     uint8 [batch, kv_heads, ceil(slots / 64), 68 * head_dim]      slot_pos  int32 [batch, kv_heads, slots]
      cursor    int32 [batch, kv_heads, 2]: next slot, next position          score     fp32 [batch, kv_heads, slots]

    One stream at a time: every call works on the same buffers."""

    def __init__(self, *, batch: int, heads: int, kv_heads: int, head_dim: int, slots: int, recent: int, dtype, scale: float = None,
                 cache: torch.Tensor = None, slot_pos: torch.Tensor = None, score: torch.Tensor = None, cursor: torch.Tensor = None,
                 device="cuda:0"):
        self.lib = load_library()
        code = {"f32": ADORE_F32, "bf16": ADORE_BF16}[dtype] if isinstance(dtype, str) else _CODES[dtype]
        if scale is not None and not scale > 0.0:
            raise ValueError("scale: expected a positive number")
        self.cfg = AdoreQ4Config(batch, heads, kv_heads, head_dim, slots, recent, code, float(scale or 0.0))
        self.dtype = torch.bfloat16 if code == ADORE_BF16 else torch.float32
        need = self.lib.adore_q4_cache_bytes(ctypes.byref(self.cfg))
        if need == 0:
            raise AdoreError(-1, "invalid or unsupported configuration")
        self.device = torch.device(device) if cache is None else cache.device
        rows = (batch, kv_heads)
        self.cache = self._buffer(cache, rows + ((slots + 63) // 64, 68 * head_dim), torch.uint8, 0, "cache", 256)
        self.device = self.cache.device        # (with its number)
        self.slot_pos = self._buffer(slot_pos, rows + (slots,), torch.int32, -1, "slot_pos", 16)
        self.score = self._buffer(score, rows + (slots,), torch.float32, 0, "score", 16)
        self.cursor = self._buffer(cursor, rows + (2,), torch.int32, 0, "cursor", 8)
        self.workspace = torch.empty(self.lib.adore_q4_workspace_bytes(ctypes.byref(self.cfg)), dtype=torch.uint8, device=self.device)
        # what every call hands over, made once (a step of few rows takes the host longer than the GPU)
        self._cfg = ctypes.byref(self.cfg)
        self._state = [ctypes.c_void_p(t.data_ptr()) for t in (self.cache, self.slot_pos, self.score, self.cursor)]
        self._space = [ctypes.c_void_p(self.workspace.data_ptr()), ctypes.c_size_t(self.workspace.numel())]
        self._index = self.cache.get_device()
        self._mine, self._rows = (batch, heads, head_dim), rows + (head_dim,)

    def _buffer(self, t, shape, dtype, value, name, align):
        if t is None:
            return torch.full(shape, value, dtype=dtype, device=self.device)
        return self._tensor(t, shape, dtype, name, align)

    def _tensor(self, t, shape, dtype, name, align=16):
        if not isinstance(t, torch.Tensor) or t.device != self.device or not t.is_cuda or t.dtype != dtype or tuple(t.shape) != tuple(shape) or \
                not t.is_contiguous() or t.data_ptr() % align:
            raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device}, {align}-byte aligned")
        return t

    def fill(self, k: torch.Tensor, v: torch.Tensor, scores: torch.Tensor = None, *, k_start: torch.Tensor = None):
        """The prompts' best tokens: k, v [tokens, kv_heads, head_dim] with k_start (int32 [batch + 1]) and scores [kv_heads, tokens], or
        [batch, kv_heads, tokens, head_dim] and [batch, kv_heads, tokens]; scores as prompt_scores gives them, or None."""
        c = self.cfg
        p = _Prompts(k, k, k_start, k_start, None)
        if p.device != self.device or p.dtype != self.dtype or (p.batch, p.cfg.kv_heads, p.cfg.head_dim) != (c.batch, c.kv_heads, c.head_dim):
            raise ValueError(f"k: expected {self.dtype} rows of {c.batch} sequences, {c.kv_heads} heads, {c.head_dim} elements on {self.device}")
        _call(self.lib, self._index, self.lib.adore_q4_fill, self._cfg, p.starts[1], p.cfg.k_tokens, p.rows(k, p.k_shape, "k"),
              p.rows(v, p.k_shape, "v"), None if scores is None else p.values(scores, p.k_rows, "scores"), *self._state, p.stream)

    def step(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, out: torch.Tensor = None, held: bool = False):
        """One token of every sequence: q [batch, heads, head_dim], k and v [batch, kv_heads, head_dim], contiguous.  Returns out
        [batch, heads, head_dim], with held=True also the token's K and V as the cache holds them."""
        if out is None:
            out = torch.empty_like(q)
        mine, rows = self._mine, self._rows
        ptr = (self._ptr(q, mine, "q"), self._ptr(k, rows, "k"), self._ptr(v, rows, "v"), *self._state, self._ptr(out, mine, "out"))
        stream = _stream(self._index)
        if held:
            k_held, v_held = torch.empty_like(k), torch.empty_like(v)
            _call(self.lib, self._index, self.lib.adore_q4_step, self._cfg, *ptr, k_held.data_ptr(), v_held.data_ptr(), *self._space, stream)
            return out, k_held, v_held
        _call(self.lib, self._index, self.lib.adore_q4_step, self._cfg, *ptr, None, None, *self._space, stream)
        return out

    def _ptr(self, t, shape, name):
        # four of these a step: attributes that cost least (2 -> 0.6 us each)
        if t.dtype is not self.dtype or t.shape != shape or t.get_device() != self._index or not t.is_contiguous() or t.data_ptr() % 16:
            self._tensor(t, shape, self.dtype, name)
        return t.data_ptr()

    def read(self, k: torch.Tensor = None, v: torch.Tensor = None):
        """What the cache holds: K and V [batch, kv_heads, slots, head_dim], zeros in free slots."""
        c = self.cfg
        shape = (c.batch, c.kv_heads, c.slots, c.head_dim)
        k, v = (torch.empty(shape, dtype=self.dtype, device=self.device) if t is None else self._tensor(t, shape, self.dtype, n)
                for t, n in ((k, "k"), (v, "v")))
        _call(self.lib, self._index, self.lib.adore_q4_read, self._cfg, self._state[0], self._state[1], k.data_ptr(), v.data_ptr(),
              _stream(self._index))
        return k, v


class Adore:
    """One decode job.  Method names and argument order follow include/adore.h."""

    def __init__(self, cfg: AdoreConfig, weights: Dict[str, torch.Tensor], device="cuda:0"):
        self.lib = load_library()
        self.cfg = cfg
        self.device = torch.device(device)
        self.storage = torch.bfloat16 if cfg.dtype == ADORE_BF16 else torch.float32
        c = cfg
        dp, Hd = c.ctrl_hidden, c.heads * c.head_dim
        shapes = {"w_kv": (c.layers, 2 * Hd, c.hidden), "gru_w_ih": (3 * dp, c.hidden), "gru_w_hh": (3 * dp, dp),
                  "gru_b_ih": (3 * dp,), "gru_b_hh": (3 * dp,), "pos_w": (dp,), "pos_b": (dp,),
                  "mlp_w1": (dp, dp), "mlp_b1": (dp,), "out_w": (dp,), "out_b": (1,)}
        self._weights = {}
        w = AdoreWeights()
        for name in _WEIGHT_FIELDS:
            dt = self.storage if name in ("w_kv", "gru_w_ih", "gru_w_hh") else torch.float32
            setattr(w, name, self._ptr(weights[name], shapes[name], dt, name))
            self._weights[name] = weights[name]          # keep alive
        nbytes = self.lib.adore_workspace_bytes(ctypes.byref(cfg))
        if nbytes == 0:
            raise AdoreError(-1, "invalid configuration")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        self.stream = torch.cuda.current_stream(self.device)
        handle = ctypes.c_void_p()
        _check(self.lib, self.lib.adore_create(ctypes.byref(cfg), ctypes.byref(w), base, nbytes,
                                               self.stream.cuda_stream, ctypes.byref(handle)))
        self.handle = handle

    # -- marshalling ---------------------------------------------------------
    def _ptr(self, t: Optional[torch.Tensor], shape: tuple, dtype: torch.dtype, name: str,
             optional: bool = False):
        if t is None:
            if optional:
                return None
            raise ValueError(f"{name} is required")
        # eight of these a step: attributes that cost least (1.2 -> 0.7 us each)
        if not t.is_cuda or t.dtype != dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name}: expected contiguous cuda {dtype} tensor of shape {tuple(shape)}, got "
                             f"{t.device} {t.dtype} {tuple(t.shape)} contiguous={t.is_contiguous()}")
        ptr = t.data_ptr()
        if ptr % 16:
            raise ValueError(f"{name}: base not 16-byte aligned")
        return ptr

    def close(self):
        if getattr(self, "handle", None):
            self.lib.adore_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the ABI -------------------------------------------------------------
    def init_cache(self, prompt_k, prompt_v, hidden_store, ctrl_input, score_override, S: int):
        c, st = self.cfg, self.storage
        _check(self.lib, self.lib.adore_init_cache(
            self.handle,
            self._ptr(prompt_k, (c.layers, c.batch, c.heads, S, c.head_dim), st, "prompt_k"),
            self._ptr(prompt_v, (c.layers, c.batch, c.heads, S, c.head_dim), st, "prompt_v"),
            self._ptr(hidden_store, (c.layers, c.batch, c.max_positions, c.hidden), st, "hidden_store",
                      optional=True),                    # None: prepare for forward_step
            self._ptr(ctrl_input, (c.batch, S, c.hidden), st, "ctrl_input"),
            self._ptr(score_override, (c.batch, c.heads, S) if c.score_mode == SCORE_H2O else (c.batch, S),
                      torch.float32, "score_override", optional=True), S))

    def attend(self, layer: int, q, k_new, v_new, out):
        c, st = self.cfg, self.storage
        shp = (c.batch, c.heads, c.head_dim)
        _check(self.lib, self.lib.adore_attend(
            self.handle, layer, self._ptr(q, shp, st, "q"), self._ptr(k_new, shp, st, "k_new"),
            self._ptr(v_new, shp, st, "v_new"), self._ptr(out, shp, torch.float32, "out")))

    def schedule(self, x_n, score_override=None, slot_map=None, released_pos=None, rebuilt_pos=None):
        c = self.cfg
        _check(self.lib, self.lib.adore_schedule(
            self.handle, self._ptr(x_n, (c.batch, c.hidden), self.storage, "x_n", optional=c.score_mode == SCORE_H2O),
            self._ptr(score_override, (c.batch,), torch.float32, "score_override", optional=True),
            self._ptr(slot_map, (c.batch, c.heads, c.cache_slots), torch.int32, "slot_map", optional=True),
            self._ptr(released_pos, (c.batch, c.heads, c.rebuild_budget + 1), torch.int32, "released_pos",
                      optional=True),
            self._ptr(rebuilt_pos, (c.batch, max(c.rebuild_budget, 1)), torch.int32, "rebuilt_pos",
                      optional=True)))

    def rebuild(self, layer: int, hidden_store_layer):
        c = self.cfg
        _check(self.lib, self.lib.adore_rebuild(
            self.handle, layer,
            self._ptr(hidden_store_layer, (c.batch, c.max_positions, c.hidden), self.storage, "hidden_store_layer")))

    def decode_step(self, q, k_new, v_new, hidden_store, x_n, score_override, out, slot_map=None):
        c, st = self.cfg, self.storage
        shp = (c.batch, c.heads, c.head_dim)
        _check(self.lib, self.lib.adore_decode_step(
            self.handle, self._ptr(q, shp, st, "q"), self._ptr(k_new, shp, st, "k_new"),
            self._ptr(v_new, shp, st, "v_new"),
            self._ptr(hidden_store, (c.batch, c.max_positions, c.hidden), st, "hidden_store"),
            self._ptr(x_n, (c.batch, c.hidden), st, "x_n", optional=c.score_mode == SCORE_H2O),
            self._ptr(score_override, (c.batch,), torch.float32, "score_override", optional=True),
            self._ptr(out, shp, torch.float32, "out"),
            self._ptr(slot_map, (c.batch, c.heads, c.cache_slots), torch.int32, "slot_map", optional=True)))

    def forward_step(self, w_q, w_o, embed, score_override, rows_out, slot_map=None, released_pos=None,
                     rebuilt_pos=None, layer_rows=None):
        c, st = self.cfg, self.storage
        Hd = c.heads * c.head_dim
        fw = AdoreForwardWeights(self._ptr(w_q, (c.layers, Hd, c.hidden), st, "w_q"),
                                 self._ptr(w_o, (c.layers, c.hidden, Hd), st, "w_o"))
        _check(self.lib, self.lib.adore_forward_step(
            self.handle, ctypes.byref(fw),
            self._ptr(embed, (c.batch, c.max_positions, c.hidden), st, "embed"),
            self._ptr(score_override, (c.batch,), torch.float32, "score_override", optional=True),
            self._ptr(rows_out, (c.batch, c.rebuild_budget + 1, c.hidden), st, "rows_out"),
            self._ptr(layer_rows, (c.layers, c.batch, c.rebuild_budget + 1, c.hidden), st, "layer_rows", optional=True),
            self._ptr(slot_map, (c.batch, c.heads, c.cache_slots), torch.int32, "slot_map", optional=True),
            self._ptr(released_pos, (c.batch, c.heads, c.rebuild_budget + 1), torch.int32, "released_pos",
                      optional=True),
            self._ptr(rebuilt_pos, (c.batch, max(c.rebuild_budget, 1)), torch.int32, "rebuilt_pos",
                      optional=True)))

    def _state_ptrs(self, slot_pos, scores, z, cache_k, cache_v):
        c, st = self.cfg, self.storage
        cs = (c.layers, c.batch, c.heads, c.cache_slots, c.head_dim)
        return (self._ptr(slot_pos, (c.batch, c.heads, c.cache_slots), torch.int32, "slot_pos", optional=True),
                self._ptr(scores, self._score_shape(), torch.float32, "scores", optional=True),
                self._ptr(z, (c.batch, c.ctrl_hidden), torch.float32, "z", optional=True),
                self._ptr(cache_k, cs, st, "cache_k", optional=True),
                self._ptr(cache_v, cs, st, "cache_v", optional=True))

    def _score_shape(self):
        c = self.cfg
        return (c.batch, c.heads, c.max_positions) if c.score_mode == SCORE_H2O else (c.batch, c.max_positions)

    def get_state(self, slot_pos=None, scores=None, z=None, cache_k=None, cache_v=None) -> int:
        step = ctypes.c_int32(-1)
        _check(self.lib, self.lib.adore_get_state(self.handle, *self._state_ptrs(slot_pos, scores, z, cache_k, cache_v),
                                                  ctypes.byref(step)))
        return step.value

    def set_state(self, slot_pos, scores, z, cache_k, cache_v, step: int):
        _check(self.lib, self.lib.adore_set_state(self.handle, *self._state_ptrs(slot_pos, scores, z, cache_k, cache_v),
                                                  step))

    def set_input_order(self, ordered: bool):
        _check(self.lib, self.lib.adore_set_input_order(self.handle, int(ordered)))

    def check_guards(self) -> int:
        """Damaged guard words of the debug layout (ADORE_GUARD_WORDS=1 at create), or -1 if there are none."""
        bad = ctypes.c_int32(0)
        _check(self.lib, self.lib.adore_check_guards(self.handle, ctypes.byref(bad)))
        return int(bad.value)

    def set_timing(self, enable: bool):
        _check(self.lib, self.lib.adore_set_timing(self.handle, int(enable)))

    def read_timing(self):
        ms = (ctypes.c_float * len(KERNELS))()
        cnt = (ctypes.c_int32 * len(KERNELS))()
        _check(self.lib, self.lib.adore_read_timing(self.handle, ms, cnt))
        return {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(KERNELS)}

    # -- convenience (allocation only) ----------------------------------------
    def empty_state(self):
        c, st, dev = self.cfg, self.storage, self.device
        cs = (c.layers, c.batch, c.heads, c.cache_slots, c.head_dim)
        return dict(slot_pos=torch.empty((c.batch, c.heads, c.cache_slots), dtype=torch.int32, device=dev),
                    scores=torch.empty(self._score_shape(), dtype=torch.float32, device=dev),
                    z=torch.empty((c.batch, c.ctrl_hidden), dtype=torch.float32, device=dev),
                    cache_k=torch.empty(cs, dtype=st, device=dev), cache_v=torch.empty(cs, dtype=st, device=dev))
