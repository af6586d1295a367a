"""Operators that make, train and bound the gradients of feed-forward blocks for a ring's workers (``include/evg_nn.h``).

``BlockNorm`` (the norms on both sides of a block, with its gate and residual scale), ``GatedFFN`` (the gated feed-forward
block), both with their backward passes, and ``GradClip`` (clipping by each worker's global gradient norm, into the arena
that ``evg.Ring.step`` takes).  Tensors have the worker as their first axis; one model alone is one worker.

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

import torch

from . import evg

RMS, LAYER = 0, 1
SILU, GELU, GELU_TANH, RELU = 0, 1, 2, 3
ACTIVATIONS = dict(silu=SILU, gelu=GELU, gelu_tanh=GELU_TANH, relu=RELU)
NONFINITE_PASS, NONFINITE_ZERO = 0, 1

EXPORTS = ("evg_clip_init", "evg_clip_run", "evg_clip_destroy",
           "evg_blocknorm_init", "evg_blocknorm_forward", "evg_blocknorm_backward", "evg_blocknorm_destroy",
           "evg_ffn_init", "evg_ffn_saved_bytes", "evg_ffn_forward", "evg_ffn_backward", "evg_ffn_destroy")

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


# Arguments that are structures go as packed bytes, which costs a call less than filling ctypes structures: evg_mat,
# evg_blocknorm_in and evg_blocknorm_grads.
_MAT = struct.Struct("3q").pack
_IN = struct.Struct("2I21q").pack
_GRADS = struct.Struct("21q").pack
assert struct.calcsize("3q") == C.sizeof(Mat) and struct.calcsize("2I21q") == C.sizeof(BlockNormIn)
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
        for name in ("clip", "blocknorm", "ffn"):
            getattr(l, f"evg_{name}_destroy").argtypes = [vp]
        _lib = l
    return _lib


class _Operator:
    """What the three have in common: a handle of the library, its stream and the checks of tensors."""

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

    def _at(self, t, shape, what):
        """Address and strides of a tensor of the given shape, [workers, rows, columns] or [workers, columns]."""
        if t.dtype is not self.dtype or t.get_device() != self._index:
            raise ValueError(f"{what} must be {self.dtype} on {self.device}, is {t.dtype} on {t.device}")
        if t.shape != shape:
            raise ValueError(f"{what} must have the shape {tuple(shape)}, has {tuple(t.shape)}")
        stride = t.stride()
        if stride[-1] != 1 and shape[-1] > 1:
            raise ValueError(f"{what}: the last axis must have stride 1")
        return t.data_ptr() or _NOTHING, stride[0], stride[1] if len(stride) == 3 else 0

    def _mat(self, t, shape, what):
        return _MAT(*self._at(t, shape, what))

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
