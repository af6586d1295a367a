"""Operators that make, train and bound the gradients of feed-forward blocks for a ring's workers (``include/evg_nn.h``).

``BlockNorm`` (the norms on both sides of a block, with its gate and residual scale), ``GatedFFN`` (the gated feed-forward
block), both with their backward passes, and ``GradClip`` (clipping by each worker's global gradient norm, into the arena
that ``evg.Ring.step`` takes).  ``Embedding`` (tokens to rows), ``Router`` (which experts a token goes to) and ``ExpertSort`` (tokens in
the experts' order and back), with their backward passes, are what stands around blocks of several experts; ``Orthogonal`` makes the gradients of
matrices orthogonal updates.  Tensors have the worker as their first axis; one model alone is one worker.

Argument marshalling only, as in ``evg``: every operation runs in the library's HIP kernels, there is no fallback.  An
operator is bound to one stream (the current one when it is made, or the one given) and its calls only enqueue work there.
Tensors that another stream made or will read have to be ordered against it by the caller, as with ``Ring``; outputs
that a call allocates belong to the operator's stream.

The operators are no part of torch's automatic differentiation: ``requires_grad`` of what they are given is ignored, their outputs carry
no graph, and gradients come from ``backward`` alone.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import NamedTuple

import torch

from . import evg

RMS, LAYER = 0, 1
SILU, GELU, GELU_TANH, RELU = 0, 1, 2, 3
ACTIVATIONS = dict(silu=SILU, gelu=GELU, gelu_tanh=GELU_TANH, relu=RELU)
NONFINITE_PASS, NONFINITE_ZERO = 0, 1

EXPORTS = ("evg_clip_init", "evg_clip_run", "evg_clip_destroy",
           "evg_blocknorm_init", "evg_blocknorm_forward", "evg_blocknorm_backward", "evg_blocknorm_destroy",
           "evg_ffn_init", "evg_ffn_saved_bytes", "evg_ffn_forward", "evg_ffn_backward", "evg_ffn_destroy",
           "evg_embed_init", "evg_embed_forward", "evg_embed_backward", "evg_embed_destroy",
           "evg_router_init", "evg_router_forward", "evg_router_backward", "evg_router_destroy",
           "evg_experts_init", "evg_experts_slots", "evg_experts_dispatch", "evg_experts_combine", "evg_experts_combine_backward",
           "evg_experts_destroy", "evg_ortho_init", "evg_ortho_update", "evg_ortho_destroy")

_NOTHING = 256     # the address of a tensor without elements: given, but never read
_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


class Mat(C.Structure):
    _fields_ = [("p", C.c_void_p), ("worker", C.c_int64), ("row", C.c_int64)]


class ClipConfig(C.Structure):
    _fields_ = [("P", C.c_uint32), ("L", C.c_uint32), ("layer_numel", C.POINTER(C.c_uint64)), ("grad_type", C.c_uint32),
                ("out_type", C.c_uint32), ("eps", C.c_float), ("nonfinite", C.c_uint32)]


class BlockNormConfig(C.Structure):
    _fields_ = [("workers", C.c_uint32), ("width", C.c_uint32), ("max_rows", C.c_uint32), ("type", C.c_uint32),
                ("kind", C.c_uint32), ("eps", C.c_float), ("residual_scale", C.c_float), ("branch_scale", C.c_float),
                ("forward_only", C.c_uint32)]


_INPUTS = ("residual", "branch", "gate", "post", "post_bias", "pre", "pre_bias")


class BlockNormIn(C.Structure):
    _fields_ = [("rows", C.c_uint32), ("gate_rows", C.c_uint32)] + [(n, Mat) for n in _INPUTS]


class BlockNormGrads(C.Structure):
    _fields_ = [(n, Mat) for n in _INPUTS]


class FFNConfig(C.Structure):
    _fields_ = [("workers", C.c_uint32), ("width", C.c_uint32), ("hidden", C.c_uint32), ("max_rows", C.c_uint32),
                ("type", C.c_uint32), ("activation", C.c_uint32), ("train", C.c_uint32)]


class EmbedConfig(C.Structure):
    _fields_ = [("workers", C.c_uint32), ("vocab", C.c_uint32), ("width", C.c_uint32), ("max_tokens", C.c_uint32),
                ("type", C.c_uint32), ("scale", C.c_float), ("train", C.c_uint32)]


class Ids(C.Structure):
    _fields_ = [("p", C.c_void_p), ("worker", C.c_int64), ("wide", C.c_uint32)]


class RouterConfig(C.Structure):
    _fields_ = [("workers", C.c_uint32), ("experts", C.c_uint32), ("top", C.c_uint32), ("max_tokens", C.c_uint32),
                ("type", C.c_uint32), ("over_chosen", C.c_uint32)]


class ExpertsConfig(C.Structure):
    _fields_ = [("workers", C.c_uint32), ("experts", C.c_uint32), ("top", C.c_uint32), ("width", C.c_uint32),
                ("max_tokens", C.c_uint32), ("capacity", C.c_uint32), ("type", C.c_uint32)]


class ExpertsPlan(C.Structure):
    _fields_ = [("slot", C.c_void_p), ("source", C.c_void_p), ("counts", C.c_void_p)]


class OrthoConfig(C.Structure):
    _fields_ = [("matrices", C.c_uint32), ("rows", C.c_uint32), ("cols", C.c_uint32), ("type", C.c_uint32), ("out_type", C.c_uint32),
                ("steps", C.c_uint32), ("a", C.c_float), ("b", C.c_float), ("c", C.c_float), ("momentum", C.c_float),
                ("nesterov", C.c_uint32), ("eps", C.c_float), ("scale", C.c_float)]


# Arguments that are structures go as packed bytes, which costs a call less than filling ctypes structures: evg_mat,
# evg_blocknorm_in, evg_blocknorm_grads, evg_ids and evg_experts_plan.
_MAT = struct.Struct("3q").pack
_IN = struct.Struct("2I21q").pack
_GRADS = struct.Struct("21q").pack
_IDS = struct.Struct("2qIxxxx").pack
_PLAN = struct.Struct("3q").pack
assert struct.calcsize("3q") == C.sizeof(Mat) and struct.calcsize("2I21q") == C.sizeof(BlockNormIn)
assert struct.calcsize("2qIxxxx") == C.sizeof(Ids) and struct.calcsize("3q") == C.sizeof(ExpertsPlan)
_ABSENT = (0, 0, 0)

_lib = None


def lib():
    global _lib
    if _lib is None:
        l = evg.lib()
        vp, mp, u32 = C.c_void_p, C.c_void_p, C.c_uint32
        l.evg_clip_init.argtypes = [C.POINTER(vp), C.POINTER(ClipConfig), vp]
        l.evg_clip_run.argtypes = [vp, vp, vp, C.c_float, C.c_float, vp]
        l.evg_blocknorm_init.argtypes = [C.POINTER(vp), C.POINTER(BlockNormConfig), vp]
        l.evg_blocknorm_forward.argtypes = [vp, mp, mp, mp]
        l.evg_blocknorm_backward.argtypes = [vp, mp, mp, mp, mp]
        l.evg_ffn_init.argtypes = [C.POINTER(vp), C.POINTER(FFNConfig), vp]
        l.evg_ffn_saved_bytes.argtypes = [vp, u32]
        l.evg_ffn_saved_bytes.restype = C.c_uint64
        l.evg_ffn_forward.argtypes = [vp, u32] + [mp] * 5 + [vp]
        l.evg_ffn_backward.argtypes = [vp, u32] + [mp] * 5 + [vp] + [mp] * 4
        l.evg_embed_init.argtypes = [C.POINTER(vp), C.POINTER(EmbedConfig), vp]
        l.evg_embed_forward.argtypes = [vp, u32, mp, mp, mp]
        l.evg_embed_backward.argtypes = [vp, u32, mp, mp, mp, u32]
        l.evg_router_init.argtypes = [C.POINTER(vp), C.POINTER(RouterConfig), vp]
        l.evg_router_forward.argtypes = [vp, u32, mp, vp, vp]
        l.evg_router_backward.argtypes = [vp, u32, vp, mp, vp, mp]
        l.evg_experts_init.argtypes = [C.POINTER(vp), C.POINTER(ExpertsConfig), vp]
        l.evg_experts_slots.argtypes = [vp, u32]
        l.evg_experts_slots.restype = C.c_uint64
        l.evg_experts_dispatch.argtypes = [vp, u32, mp, vp, mp, mp]
        l.evg_experts_combine.argtypes = [vp, u32, mp, vp, mp, mp]
        l.evg_experts_combine_backward.argtypes = [vp, u32, mp, mp, vp, mp, mp, vp]
        l.evg_ortho_init.argtypes = [C.POINTER(vp), C.POINTER(OrthoConfig), vp]
        l.evg_ortho_update.argtypes = [vp, mp, mp, mp, mp]
        for name in ("clip", "blocknorm", "ffn", "embed", "router", "experts", "ortho"):
            getattr(l, f"evg_{name}_destroy").argtypes = [vp]
        _lib = l
    return _lib


class _Operator:
    """What they have in common: a handle of the library, its stream and the checks of tensors."""

    _destroy = None

    def _open(self, dtype, device, stream):
        lib()
        if not torch.cuda.is_available():
            raise RuntimeError("no GPU visible: the operators only run on the HIP device")
        if dtype not in _TYPES:
            raise ValueError(f"dtype must be one of {list(_TYPES)}")
        self.dtype = dtype
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("device must be a GPU")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self._raw = self.stream.cuda_stream
        self._h = C.c_void_p()

    def _make(self, init, cfg):
        with torch.cuda.device(self.device):
            evg._check(init(C.byref(self._h), C.byref(cfg), C.c_void_p(self._raw)))

    def _empty(self, shape, dtype=None):
        """Memory of the operator's stream."""
        if torch._C._cuda_getCurrentRawStream(self._index) == self._raw:
            return torch.empty(shape, dtype=dtype or self.dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=dtype or self.dtype, device=self.device)

    def _like(self, t):
        if t.is_contiguous() and torch._C._cuda_getCurrentRawStream(self._index) == self._raw:
            return torch.empty_like(t)
        return self._empty(t.shape)

    def _at(self, t, shape, what, dtype=None):
        """Address and strides of a tensor of the given shape, [workers, rows, columns] or [workers, columns]."""
        dtype = dtype or self.dtype
        if t.dtype is not dtype or t.get_device() != self._index:
            raise ValueError(f"{what} must be {dtype} on {self.device}, is {t.dtype} on {t.device}")
        if t.shape != shape:
            raise ValueError(f"{what} must have the shape {tuple(shape)}, has {tuple(t.shape)}")
        stride = t.stride()
        if stride[-1] != 1 and shape[-1] > 1:
            raise ValueError(f"{what}: the last axis must have stride 1")
        return t.data_ptr() or _NOTHING, stride[0], stride[1] if len(stride) == 3 else 0

    def _mat(self, t, shape, what, dtype=None):
        return _MAT(*self._at(t, shape, what, dtype))

    def _array(self, t, shape, what, dtype=torch.int32):
        """The address of a contiguous tensor."""
        if t.dtype is not dtype or t.get_device() != self._index or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device}")
        return t.data_ptr() or _NOTHING

    def _rows(self, t, width, what):
        if t.dim() != 3 or t.shape[0] != self.workers or t.shape[2] != width:
            raise ValueError(f"{what} must have the shape ({self.workers}, rows, {width}), has {tuple(t.shape)}")
        if t.shape[1] > self.max_rows:
            raise ValueError(f"{what} has {t.shape[1]} rows, at most {self.max_rows} were asked for")
        return t.shape[1]

    def close(self):
        if getattr(self, "_h", None):
            getattr(lib(), self._destroy)(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GradClip(_Operator):
    """Clips each worker's gradient by its global norm over all its tensors.

    Gradients lie in arenas as ``Ring``'s (``evg.Layout(layer_numel)``), [workers, padded length], of any of the types;
    ``out_dtype`` is ``dtype`` or float32, as ``Ring.step`` takes it.
    """

    _destroy = "evg_clip_destroy"

    def __init__(self, layer_numel, workers, *, dtype=torch.float32, out_dtype=None, eps=1e-6, nonfinite=NONFINITE_PASS,
                 device="cuda", stream=None):
        self._open(dtype, device, stream)
        self.out_dtype = dtype if out_dtype is None else out_dtype
        if self.out_dtype not in (dtype, torch.float32):
            raise ValueError("out_dtype must be dtype or float32")
        self.workers = int(workers)
        numel, p = evg._u64(layer_numel)
        self.pitch = evg.padded_numel(layer_numel)
        self._make(lib().evg_clip_init, ClipConfig(self.workers, numel.size, p, _TYPES[dtype], _TYPES[self.out_dtype], eps, nonfinite))

    def clip(self, grad, max_norm, *, out=None, norm=None, scale=1.0):
        """``(out, norm)``: the clipped arena and each worker's norm.  ``out`` may be ``grad`` itself."""
        shape = (self.workers, self.pitch)
        if out is None:
            out = self._empty(shape, self.out_dtype)
        if norm is None:
            norm = self._empty(self.workers, torch.float32)
        for t, dtype, size, what in ((grad, self.dtype, shape, "grad"), (out, self.out_dtype, shape, "out"),
                                     (norm, torch.float32, shape[:1], "norm")):
            if t.dtype is not dtype or t.get_device() != self._index or t.shape != size or not t.is_contiguous():
                raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {size} on {self.device}")
        evg._check(lib().evg_clip_run(self._h, grad.data_ptr(), out.data_ptr(), max_norm, scale, norm.data_ptr()))
        return out, norm


class BlockNorm(_Operator):
    """``residual' = residual_scale * residual + branch_scale * gate * N(branch; post)`` and ``normed = N(residual'; pre)``.

    ``kind``: ``RMS`` or ``LAYER``.  ``gate_rows`` tokens share a row of the gate (0: there is none).  Which norms there are
    follows from the weights that a call is given.  Without ``train`` there is no ``backward``, nor the memory for its sums.  [workers, rows, width]: residual, branch; [workers, ceil(rows /
    gate_rows), width]: gate; [workers, width]: weights and biases.
    """

    _destroy = "evg_blocknorm_destroy"

    def __init__(self, width, *, workers=1, max_rows, dtype=torch.bfloat16, kind=RMS, eps=1e-6, residual_scale=1.0,
                 branch_scale=1.0, gate_rows=0, train=True, device="cuda", stream=None):
        self._open(dtype, device, stream)
        self.width, self.workers, self.max_rows, self.gate_rows = int(width), int(workers), int(max_rows), int(gate_rows)
        self._keeps = residual_scale == 1.0
        self._make(lib().evg_blocknorm_init, BlockNormConfig(self.workers, self.width, self.max_rows, _TYPES[dtype], kind, eps,
                                                             residual_scale, branch_scale, not train))

    def _in(self, residual, branch, gate, post, post_bias, pre, pre_bias):
        """The shapes of tokens, the gate and weights, and the inputs as the library takes them."""
        rows = self._rows(residual, self.width, "residual")
        token, vector, gates = residual.shape, (self.workers, self.width), None
        at = self._at
        if gate is not None:
            if not self.gate_rows:
                raise ValueError("a gate is given, but the operator was made without gate_rows")
            gates = (self.workers, -(-rows // self.gate_rows), self.width)
        return token, gates, vector, _IN(
            rows, self.gate_rows, *at(residual, token, "residual"),
            *(_ABSENT if branch is None else at(branch, token, "branch")),
            *(_ABSENT if gate is None else at(gate, gates, "gate")),
            *(_ABSENT if post is None else at(post, vector, "post")),
            *(_ABSENT if post_bias is None else at(post_bias, vector, "post_bias")),
            *(_ABSENT if pre is None else at(pre, vector, "pre")),
            *(_ABSENT if pre_bias is None else at(pre_bias, vector, "pre_bias")))

    def forward(self, residual, branch=None, *, gate=None, post=None, post_bias=None, pre=None, pre_bias=None,
                residual_out=None, normed=None):
        """``(residual', normed)``; ``normed`` is None without ``pre``.  ``residual_out`` may be ``residual`` itself."""
        token, _, _, arg = self._in(residual, branch, gate, post, post_bias, pre, pre_bias)
        same = branch is None and self._keeps and residual_out is None    # residual' is the residual
        if not same and residual_out is None:
            residual_out = self._like(residual)
        if normed is None and pre is not None:
            normed = self._like(residual)
        out = None if same else self._mat(residual_out, token, "residual_out")
        n = None if normed is None else self._mat(normed, token, "normed")
        if out is not None or n is not None:
            evg._check(lib().evg_blocknorm_forward(self._h, arg, out, n))
        return residual if same else residual_out, normed

    def backward(self, d_residual, d_normed, residual, branch=None, *, gate=None, post=None, post_bias=None, pre=None,
                 pre_bias=None, out=None):
        """The gradients ``d_<name>`` of every tensor given, from those of ``residual'`` and ``normed`` (either may be None).

        ``out``: a dict of tensors to write some of them to."""
        token, gates, vector, arg = self._in(residual, branch, gate, post, post_bias, pre, pre_bias)
        grads, result = [], {}
        for name, t, shape in (("d_residual", residual, token), ("d_branch", branch, token), ("d_gate", gate, gates), ("d_post", post, vector),
                               ("d_post_bias", post_bias, vector), ("d_pre", pre, vector), ("d_pre_bias", pre_bias, vector)):
            if t is None:
                grads += _ABSENT
                continue
            d = out.get(name) if out else None
            if d is None:
                d = self._like(t)
            result[name] = d
            grads += self._at(d, shape, name)
        r = None if d_residual is None else self._mat(d_residual, token, "d_residual")
        n = None if d_normed is None else self._mat(d_normed, token, "d_normed")
        evg._check(lib().evg_blocknorm_backward(self._h, arg, r, n, _GRADS(*grads)))
        return result


class GatedFFN(_Operator):
    """``y = (act(x w_gate^T) * (x w_up^T)) w_down^T`` for each worker, and its backward pass (with ``train``).

    x, y: [workers, rows, width]; w_gate, w_up: [workers, hidden, width]; w_down: [workers, width, hidden].
    """

    _destroy = "evg_ffn_destroy"

    def __init__(self, width, hidden, *, workers=1, max_rows, dtype=torch.bfloat16, activation=SILU, train=False, device="cuda",
                 stream=None):
        self._open(dtype, device, stream)
        self.width, self.hidden, self.workers, self.max_rows = int(width), int(hidden), int(workers), int(max_rows)
        self.train = bool(train)
        self._make(lib().evg_ffn_init, FFNConfig(self.workers, self.width, self.hidden, self.max_rows, _TYPES[dtype], activation,
                                                 self.train))

    def _weights(self, w_gate, w_up, w_down):
        up, down = (self.workers, self.hidden, self.width), (self.workers, self.width, self.hidden)
        return self._mat(w_gate, up, "w_gate"), self._mat(w_up, up, "w_up"), self._mat(w_down, down, "w_down")

    def forward(self, x, w_gate, w_up, w_down, *, out=None, save=False):
        """``y``; with ``save``, ``(y, saved)``, the latter for ``backward``."""
        rows = self._rows(x, self.width, "x")
        if out is None:
            out = self._like(x)
        saved = self._empty(lib().evg_ffn_saved_bytes(self._h, rows), torch.uint8) if save else None
        evg._check(lib().evg_ffn_forward(self._h, rows, self._mat(x, x.shape, "x"), *self._weights(w_gate, w_up, w_down),
                                         self._mat(out, x.shape, "out"), saved.data_ptr() if save else None))
        return (out, saved) if save else out

    def backward(self, dy, x, w_gate, w_up, w_down, saved, *, dx=None, dw_gate=None, dw_up=None, dw_down=None,
                 input_gradient=True, weight_gradients=True):
        """``(dx, dw_gate, dw_up, dw_down)``.  Only tensors that are given are filled, and the others None, without ``input_gradient``
        for ``dx`` and without ``weight_gradients`` for the rest; what is not asked for is not computed."""
        rows = self._rows(x, self.width, "x")
        need = lib().evg_ffn_saved_bytes(self._h, rows)
        if saved.numel() * saved.element_size() != need or saved.device != self.device or not saved.is_contiguous():
            raise ValueError(f"saved must be the {need} bytes that forward(save=True) returned")
        weights = self._weights(w_gate, w_up, w_down)
        if dx is None and input_gradient:
            dx = self._like(x)
        grads = [self._like(w) if d is None and weight_gradients else d for d, w in ((dw_gate, w_gate), (dw_up, w_up), (dw_down, w_down))]
        evg._check(lib().evg_ffn_backward(
            self._h, rows, self._mat(dy, x.shape, "dy"), self._mat(x, x.shape, "x"), *weights, saved.data_ptr() or None,
            None if dx is None else self._mat(dx, x.shape, "dx"),
            *(None if d is None else self._mat(d, w.shape, what)
              for d, w, what in zip(grads, (w_gate, w_up, w_down), ("dw_gate", "dw_up", "dw_down")))))
        return (dx, *grads)


class Embedding(_Operator):
    """``y[t] = scale * table[token[t]]`` for each worker, and the table's gradient (with ``train``).

    tokens: [workers, tokens], int32 or int64; a number outside 0 .. vocab-1 is padding: a row of zeros, no part in the gradient.
    table: [workers, vocab, width]; y: [workers, tokens, width].
    """

    _destroy = "evg_embed_destroy"

    def __init__(self, vocab, width, *, workers=1, max_tokens, dtype=torch.bfloat16, scale=1.0, train=False, device="cuda", stream=None):
        self._open(dtype, device, stream)
        self.vocab, self.width, self.workers, self.max_rows = int(vocab), int(width), int(workers), int(max_tokens)
        self._make(lib().evg_embed_init, EmbedConfig(self.workers, self.vocab, self.width, self.max_rows, _TYPES[dtype], scale, bool(train)))

    def _ids(self, tokens):
        if tokens.dtype not in (torch.int32, torch.int64) or tokens.get_device() != self._index:
            raise ValueError(f"tokens must be int32 or int64 on {self.device}, is {tokens.dtype} on {tokens.device}")
        if tokens.dim() != 2 or tokens.shape[0] != self.workers:
            raise ValueError(f"tokens must have the shape ({self.workers}, tokens), has {tuple(tokens.shape)}")
        count = tokens.shape[1]
        if count > self.max_rows:
            raise ValueError(f"tokens has {count} of a worker, at most {self.max_rows} were asked for")
        if count > 1 and tokens.stride(1) != 1:
            raise ValueError("tokens: the last axis must have stride 1")
        return count, _IDS(tokens.data_ptr() or _NOTHING, tokens.stride(0), tokens.dtype is torch.int64)

    def forward(self, tokens, table, *, out=None):
        """``y``."""
        count, ids = self._ids(tokens)
        shape = (self.workers, count, self.width)
        if out is None:
            out = self._empty(shape)
        evg._check(lib().evg_embed_forward(self._h, count, ids, self._mat(table, (self.workers, self.vocab, self.width), "table"),
                                           self._mat(out, shape, "out")))
        return out

    def backward(self, d_out, tokens, *, d_table=None, accumulate=False):
        """``d_table``.  ``accumulate``: added to what ``d_table`` holds, as where a table has a second use or a batch several parts."""
        count, ids = self._ids(tokens)
        shape = (self.workers, self.vocab, self.width)
        if d_table is None:
            if accumulate:
                raise ValueError("accumulate needs the d_table to add to")
            d_table = self._empty(shape)
        evg._check(lib().evg_embed_backward(self._h, count, ids, self._mat(d_out, (self.workers, count, self.width), "d_out"),
                                            self._mat(d_table, shape, "d_table"), bool(accumulate)))
        return d_table


class Router(_Operator):
    """The ``top`` experts of each token's largest logits, and their weights: the softmax over all logits, or with ``over_chosen`` over the
    chosen ones.

    logits: [workers, tokens, experts]; chosen (int32) and weights (float32): [workers, tokens, top], the largest first, equal
    ones in the experts' order.  Experts at minus infinity are never chosen; where too few are left, -1 with weight 0.
    """

    _destroy = "evg_router_destroy"

    def __init__(self, experts, top, *, workers=1, max_tokens, dtype=torch.float32, over_chosen=True, device="cuda", stream=None):
        self._open(dtype, device, stream)
        self.experts, self.top, self.workers, self.max_rows = int(experts), int(top), int(workers), int(max_tokens)
        self._make(lib().evg_router_init, RouterConfig(self.workers, self.experts, self.top, self.max_rows, _TYPES[dtype], bool(over_chosen)))

    def forward(self, logits, *, chosen=None, weights=None):
        """``(chosen, weights)``."""
        count = self._rows(logits, self.experts, "logits")
        shape = (self.workers, count, self.top)
        if chosen is None:
            chosen = self._empty(shape, torch.int32)
        if weights is None:
            weights = self._empty(shape, torch.float32)
        evg._check(lib().evg_router_forward(self._h, count, self._mat(logits, logits.shape, "logits"), self._array(chosen, shape, "chosen"),
                                            self._array(weights, shape, "weights", torch.float32)))
        return chosen, weights

    def backward(self, d_weights, logits, chosen, *, out=None):
        """The logits' gradient from that of the weights and what ``forward`` chose.  ``out`` may be ``logits`` itself."""
        count = self._rows(logits, self.experts, "logits")
        shape = (self.workers, count, self.top)
        if out is None:
            out = self._like(logits)
        evg._check(lib().evg_router_backward(self._h, count, self._array(d_weights, shape, "d_weights", torch.float32),
                                             self._mat(logits, logits.shape, "logits"), self._array(chosen, shape, "chosen"),
                                             self._mat(out, logits.shape, "out")))
        return out


class ExpertPlan(NamedTuple):
    """Where ``ExpertSort.dispatch`` sent a batch's entries, all int32: ``slot`` [workers, tokens, top], -1 where left out; ``source``
    [workers, slots], the entry ``token * top + k`` of a slot or -1; ``counts`` [workers, experts], with those that found no room."""

    slot: torch.Tensor
    source: torch.Tensor
    counts: torch.Tensor


class ExpertSort(_Operator):
    """Tokens in the order of their experts, and back with weights applied.

    x, y: [workers, tokens, width]; chosen: [workers, tokens, top], int32, -1 for none; rows: [workers, slots, width].  Without ``capacity`` a worker has
    tokens * top slots, one expert's after the other's; with it, experts * capacity, of which expert e has those from e * capacity on, so that
    ``rows.view(workers * experts, capacity, width)`` is what a ``GatedFFN`` with as many workers takes; an expert's later entries
    that find no room are left out.  Empty slots hold zeros.
    """

    _destroy = "evg_experts_destroy"

    def __init__(self, experts, top, width, *, workers=1, max_tokens, capacity=0, dtype=torch.bfloat16, device="cuda", stream=None):
        self._open(dtype, device, stream)
        self.experts, self.top, self.width, self.workers = int(experts), int(top), int(width), int(workers)
        self.max_rows, self.capacity = int(max_tokens), int(capacity)
        self._make(lib().evg_experts_init, ExpertsConfig(self.workers, self.experts, self.top, self.width, self.max_rows, self.capacity,
                                                         _TYPES[dtype]))

    def slots(self, tokens):
        """Slots of each worker for so many tokens."""
        return self.experts * self.capacity if self.capacity else tokens * self.top

    def _sizes(self, count):
        slots = self.slots(count)
        return (self.workers, slots, self.width), (self.workers, count, self.top), (self.workers, slots), (self.workers, self.experts)

    def _plan(self, plan, count):
        _, entry, slots, counts = self._sizes(count)
        return _PLAN(self._array(plan.slot, entry, "slot"), self._array(plan.source, slots, "source"), self._array(plan.counts, counts, "counts"))

    def _count(self, plan):
        count = plan.slot.shape[1] if plan.slot.dim() == 3 else -1
        if not 0 <= count <= self.max_rows:
            raise ValueError(f"the plan must be one of this operator's, of at most {self.max_rows} tokens")
        return count

    def dispatch(self, x, chosen, *, rows=None, plan=None):
        """``(rows, plan)``; a plan that is given is written again."""
        count = self._rows(x, self.width, "x")
        row, entry, slots, counts = self._sizes(count)
        if rows is None:
            rows = self._empty(row)
        if plan is None:
            plan = ExpertPlan(self._empty(entry, torch.int32), self._empty(slots, torch.int32), self._empty(counts, torch.int32))
        evg._check(lib().evg_experts_dispatch(self._h, count, self._mat(x, x.shape, "x"), self._array(chosen, entry, "chosen"),
                                              self._mat(rows, row, "rows"), self._plan(plan, count)))
        return rows, plan

    def dispatch_backward(self, d_rows, plan, *, dx=None):
        """``dx[t]``: the sum of the gradients of the rows that token t was sent to."""
        return self.combine(d_rows, None, plan, out=dx)

    def combine(self, rows, weights, plan, *, out=None):
        """``y[t] = sum_k weights[t, k] * rows[slot[t, k]]``; weights: [workers, tokens, top], float32, or None: all 1."""
        count = self._count(plan)
        row, entry, _, _ = self._sizes(count)
        shape = (self.workers, count, self.width)
        if out is None:
            out = self._empty(shape)
        evg._check(lib().evg_experts_combine(self._h, count, self._mat(rows, row, "rows"),
                                             None if weights is None else self._array(weights, entry, "weights", torch.float32),
                                             self._plan(plan, count), self._mat(out, shape, "out")))
        return out

    def combine_backward(self, dy, rows, weights, plan, *, d_rows=None, d_weights=None, row_gradients=True, weight_gradients=True):
        """``(d_rows, d_weights)``.  One that is neither given nor asked for is None and not computed; ``rows`` is read for
        ``d_weights`` only."""
        count = self._count(plan)
        row, entry, _, _ = self._sizes(count)
        if d_rows is None and row_gradients:
            d_rows = self._empty(row)
        if d_weights is None and weight_gradients:
            d_weights = self._empty(entry, torch.float32)
        evg._check(lib().evg_experts_combine_backward(
            self._h, count, self._mat(dy, (self.workers, count, self.width), "dy"), None if d_weights is None else self._mat(rows, row, "rows"),
            self._array(weights, entry, "weights", torch.float32), self._plan(plan, count),
            None if d_rows is None else self._mat(d_rows, row, "d_rows"),
            None if d_weights is None else self._array(d_weights, entry, "d_weights", torch.float32)))
        return d_rows, d_weights


class Orthogonal(_Operator):
    """Orthogonal updates of matrices by Newton-Schulz products, with the momentum ahead of them.

    ``m' = momentum * m + grad``, ``u = grad + momentum * m'`` (``nesterov``) or ``m'``; ``X = u / (|u| + eps)``; ``steps`` times
    ``X <- a X + (b S + c S S) X`` with ``S = X X^T`` and ``polynomial = (a, b, c)``; the update is ``scale * X``.  grad and the update:
    [matrices, rows, cols], the latter of ``out_dtype``, which is ``dtype`` or float32; m: float32.
    With the usual polynomial and five steps, float16 and float32 updates, and bfloat16 ones of matrices with a smaller side of at most 256, are as exact as sums in 32 bits;
    those of larger bfloat16 matrices may be off by about as much as their rounding once more, whatever ``out_dtype``.
    """

    _destroy = "evg_ortho_destroy"

    def __init__(self, rows, cols, *, matrices=1, dtype=torch.float32, out_dtype=None, steps=5, polynomial=(3.4445, -4.7750, 2.0315),
                 momentum=0.95, nesterov=True, eps=1e-7, scale=1.0, device="cuda", stream=None):
        self._open(dtype, device, stream)
        self.out_dtype = dtype if out_dtype is None else out_dtype
        if self.out_dtype not in (dtype, torch.float32):
            raise ValueError("out_dtype must be dtype or float32")
        self.rows, self.cols, self.matrices = int(rows), int(cols), int(matrices)
        self._make(lib().evg_ortho_init, OrthoConfig(self.matrices, self.rows, self.cols, _TYPES[dtype], _TYPES[self.out_dtype], steps,
                                                     *polynomial, momentum, bool(nesterov), eps, scale))

    def update(self, grad, *, momentum=None, momentum_out=None, out=None):
        """The update.  ``momentum``: m, which becomes m', or stays as it is where ``momentum_out`` is given for m'; None: u is the gradient.
        ``out`` may be ``grad`` itself."""
        shape = (self.matrices, self.rows, self.cols)
        if momentum is None and momentum_out is not None:
            raise ValueError("momentum_out is given, but no momentum")
        if out is None:
            out = self._empty(shape, self.out_dtype)
        old = new = None
        if momentum is not None:
            old = self._mat(momentum, shape, "momentum", torch.float32)
            new = old if momentum_out is None else self._mat(momentum_out, shape, "momentum_out", torch.float32)
        evg._check(lib().evg_ortho_update(self._h, self._mat(grad, shape, "grad"), old, new, self._mat(out, shape, "out", self.out_dtype)))
        return out
