"""The token operators (include/cbinfer_tokens.h, which has their formulas): what follows the per-frame
network when its answers become tokens and decisions, one token per stream and frame.

Tensors are torch CUDA tensors, float32 or bfloat16.  Work is enqueued on the torch stream that is current
at the call; what a call needs beyond its tensors is allocated on that stream.  As in binding.py this file
marshals arguments and nothing else: there is no fallback, what the library does not take raises CBInferError."""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence

import torch

from .binding import BF16, F32, CBInferError, _last_error, load_library

GATES = {None: 0, "silu": 1, "sigmoid": 2}
EINVAL, EDEVICE = -1, -4

EXPORTS = [
    "cbinfer_log_probs_workspace_bytes", "cbinfer_log_probs", "cbinfer_linear_attention_workspace_bytes",
    "cbinfer_linear_attention", "cbinfer_quantise_weights", "cbinfer_packed_weights_bytes", "cbinfer_pack_weights",
    "cbinfer_quantised_product_workspace_bytes", "cbinfer_quantised_product", "cbinfer_gated_norm",
]


class log_probs_args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("label_bytes", C.c_int32), ("top", C.c_int32), ("reserved", C.c_int32),
                ("outer", C.c_int64), ("classes", C.c_int64), ("inner", C.c_int64), ("outer_stride", C.c_int64),
                ("class_stride", C.c_int64), ("inner_stride", C.c_int64), ("scores", C.c_void_p), ("labels", C.c_void_p),
                ("label", C.c_void_p), ("entropy", C.c_void_p), ("top_values", C.c_void_p), ("top_index", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class linear_attention_args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("streams", C.c_int32), ("tokens", C.c_int32), ("heads", C.c_int32),
                ("kv_heads", C.c_int32), ("key_size", C.c_int32), ("value_size", C.c_int32), ("scale", C.c_float),
                ("q_stride", C.c_int64 * 3), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3), ("o_stride", C.c_int64 * 3),
                ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("o", C.c_void_p), ("state", C.c_void_p),
                ("decay", C.c_void_p), ("lengths", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class quantised_product_args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("group", C.c_int32), ("tokens", C.c_int64), ("rows", C.c_int64), ("cols", C.c_int64),
                ("x_stride", C.c_int64), ("y_stride", C.c_int64), ("x", C.c_void_p), ("packed", C.c_void_p),
                ("bias", C.c_void_p), ("y", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class gated_norm_args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("sum_dtype", C.c_int32), ("gate_kind", C.c_int32), ("group", C.c_int32),
                ("rows", C.c_int64), ("size", C.c_int64), ("x_stride", C.c_int64), ("gate_stride", C.c_int64),
                ("residual_stride", C.c_int64), ("h_stride", C.c_int64), ("y_stride", C.c_int64), ("scale", C.c_float),
                ("eps", C.c_float), ("x", C.c_void_p), ("weight", C.c_void_p), ("gate", C.c_void_p), ("residual", C.c_void_p),
                ("channel_scale", C.c_void_p), ("h", C.c_void_p), ("next_weight", C.c_void_p), ("y", C.c_void_p)]


_lib = None


def _library():
    """The loaded library with the argument types of the token operators set."""
    global _lib
    if _lib is None:
        lib = load_library()
        for name, args in (("log_probs", log_probs_args), ("linear_attention", linear_attention_args),
                           ("quantised_product", quantised_product_args)):
            f = getattr(lib, "cbinfer_%s_workspace_bytes" % name)
            f.argtypes, f.restype = [C.POINTER(args)], C.c_size_t
            f = getattr(lib, "cbinfer_" + name)
            f.argtypes, f.restype = [C.POINTER(args), C.c_void_p], C.c_int
        lib.cbinfer_gated_norm.argtypes, lib.cbinfer_gated_norm.restype = [C.POINTER(gated_norm_args), C.c_void_p], C.c_int
        lib.cbinfer_quantise_weights.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int64, C.c_int64, C.c_int32, C.c_void_p,
                                                 C.c_void_p, C.c_void_p]
        lib.cbinfer_quantise_weights.restype = C.c_int
        lib.cbinfer_packed_weights_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int32]
        lib.cbinfer_packed_weights_bytes.restype = C.c_size_t
        lib.cbinfer_pack_weights.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p]
        lib.cbinfer_pack_weights.restype = C.c_int
        _lib = lib
    return _lib


def _raise(rc: int):
    raise CBInferError(rc, _last_error(_lib))


def _refuse(message: str):
    raise CBInferError(EINVAL, message)


_KINDS = {torch.float32: F32, torch.bfloat16: BF16}


def _dtype(t, what: str) -> int:
    kind = _KINDS.get(t.dtype)
    if kind is None:
        _refuse("%s must be float32 or bfloat16 (got %s)" % (what, t.dtype))
    return kind


def _device(t, what: str):
    """The tensor's device, which has to be the current one: kernels are launched there."""
    if not t.is_cuda:
        if not torch.cuda.is_available():
            raise CBInferError(EDEVICE, "no GPU visible to torch; the HIP path has no CPU fallback")
        _refuse("%s must be a CUDA tensor" % what)
    device = t.device
    if device.index != torch._C._cuda_getDevice():
        _refuse("%s is on %s, the current device is %d" % (what, device, torch.cuda.current_device()))
    return device


def _same_device(t, device, what: str):
    if t.device != device:
        _refuse("%s is on %s, expected %s" % (what, t.device, device))


def _float32(t, device, size: int, what: str):
    if t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != size or not t.is_contiguous():
        _refuse("%s must be a contiguous float32 tensor of %d values" % (what, size))
    _same_device(t, device, what)


def _apart(t) -> bool:
    """Whether no two values of a tensor to be written share their memory, as far as its axes in the order of their strides tell."""
    reach = 0
    for stride, size in sorted((s, n) for n, s in zip(t.shape, t.stride()) if n > 1):
        if stride <= reach:
            return False
        reach += stride * (size - 1)
    return True


def _stream(device) -> int:
    """torch.cuda.current_stream(device).cuda_stream without the objects in between, which cost more than a launch."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _workspace(args, needed: int, device):
    """Allocated on the current stream; the caller keeps it until the launch."""
    if not needed:
        return None
    w = torch.empty(needed + 256, dtype=torch.uint8, device=device)
    args.workspace = (w.data_ptr() + 255) // 256 * 256
    args.workspace_bytes = needed
    return w


# ---- log probabilities --------------------------------------------------------------------------
class LogProbs(NamedTuple):
    """label: log probability of the given labels; entropy: in nats; top, index: the alternatives' log
    probabilities and classes, best first, where the scores have their classes.  None where not asked for."""
    label: Optional[object]
    entropy: object
    top: Optional[object]
    index: Optional[object]


def _joined(shape, strides):
    """Size and stride of several axes as one; None if they do not lie behind one another."""
    n, step = 1, 1
    for size, stride in zip(reversed(shape), reversed(strides)):
        if size == 1:
            continue
        if n == 1:
            step = stride
        elif stride != step * n:
            return None
        n *= size
    return n, step


def _positions(before, before_strides, behind, behind_strides):
    """The axes in front of and behind the classes as (outer, inner), each a size and a stride, and how many axes
    belong to the outer.  Without axes behind the classes those in front may fall into two parts."""
    outer, inner = _joined(before, before_strides), _joined(behind, behind_strides)
    if outer and inner:
        return outer, inner, len(before)
    if inner == (1, 1):
        for cut in range(1, len(before)):
            parts = _joined(before[:cut], before_strides[:cut]), _joined(before[cut:], before_strides[cut:])
            if parts[0] and parts[1]:
                return parts[0], parts[1], cut
    _refuse("scores: the axes in front of the classes, and those behind, must lie behind one another as one; call .contiguous()")


class _ScoresPlan(NamedTuple):
    """What a call of log_probs needs besides addresses: checked arguments, the outputs' shapes, bytes of workspace."""
    args: log_probs_args
    rest: tuple
    top_shape: tuple
    moved: Optional[tuple]
    workspace: int


# By shapes, strides and types: for the smallest calls the checks would take longer than the launch.
_scores_plans: dict = {}


def _scores_plan(scores, labels, dim: int, top: int) -> _ScoresPlan:
    shape, strides, axes = scores.shape, scores.stride(), scores.dim()
    if axes < 1 or not -axes <= dim < axes:
        _refuse("scores have no axis %d" % dim)
    dim %= axes
    if not isinstance(top, int) or top < 0 or top > 64 or top > shape[dim]:
        _refuse("top must be 0 .. 64 and at most the number of classes (got %r)" % (top,))
    a = log_probs_args()
    a.dtype = _dtype(scores, "scores")
    a.top = top
    a.classes, a.class_stride = shape[dim], strides[dim]
    before, behind = shape[:dim], shape[dim + 1:]
    cut = dim
    if scores.numel() == 0:
        a.outer = a.inner = 0
    else:
        (a.outer, a.outer_stride), (a.inner, a.inner_stride), cut = _positions(before, strides[:dim], behind, strides[dim + 1:])
    rest = before + behind
    if labels is not None:
        if labels.shape != rest:
            _refuse("labels must have the shape of the scores without the classes, %s (got %s)" % (tuple(rest), tuple(labels.shape)))
        if labels.dtype not in (torch.int32, torch.int64) or not labels.is_contiguous():
            _refuse("labels must be contiguous int32 or int64")
        a.label_bytes = 4 if labels.dtype == torch.int32 else 8
    return _ScoresPlan(a, rest, rest[:cut] + (top,) + rest[cut:], (cut, dim) if cut != dim else None,
                       _library().cbinfer_log_probs_workspace_bytes(a))


def log_probs(scores, labels=None, *, dim: int = 1, top: int = 0) -> LogProbs:
    """Log probability of `labels` (int32 or int64, the shape of scores without `dim`, or None), entropy, and the
    `top` classes with their log probabilities of float32 or bfloat16 scores of any strides whose classes lie along
    `dim`: the network's [streams][classes][H][W], or [rows][classes] of a vocabulary."""
    device = _device(scores, "scores")
    key = (scores.shape, scores.stride(), scores.dtype, dim, top, None if labels is None else (labels.shape, labels.stride(), labels.dtype))
    plan = _scores_plans.get(key)
    if plan is None:
        plan = _scores_plan(scores, labels, dim, top)
        if len(_scores_plans) >= 1024:
            _scores_plans.clear()
        _scores_plans[key] = plan
    a = log_probs_args.from_buffer_copy(plan.args)
    a.scores = scores.data_ptr()
    label = values = index = None
    entropy = torch.empty(plan.rest, dtype=torch.float32, device=device)
    a.entropy = entropy.data_ptr()
    if labels is not None:
        _same_device(labels, device, "labels")
        label = torch.empty_like(entropy)
        a.labels, a.label = labels.data_ptr(), label.data_ptr()
    if top:
        values = torch.empty(plan.top_shape, dtype=torch.float32, device=device)
        index = torch.empty_like(values, dtype=torch.int32)
        a.top_values, a.top_index = values.data_ptr(), index.data_ptr()
    keep = _workspace(a, plan.workspace, device)  # noqa: F841
    rc = _lib.cbinfer_log_probs(a, _stream(device))
    if rc:
        _raise(rc)
    if top and plan.moved:
        values, index = values.movedim(*plan.moved), index.movedim(*plan.moved)
    return LogProbs(label, entropy, values, index)


class _LayerPlan(NamedTuple):
    """What a layer's call needs besides addresses.  Made whole and kept in one assignment, read in one: calls of other threads
    may come in between."""
    geometry: tuple
    args: C.Structure
    shape: tuple
    workspace: int


# ---- linear attention ---------------------------------------------------------------------------
class LinearAttention:
    """Linear attention with a decay for each head, and the states of `n_streams` streams.

    `state` is carried from call to call, as a CBInfer carries a stream's maps; a caller that moves between torch streams orders the calls itself."""

    def __init__(self, decay: Sequence[float], key_size: int, value_size: int, *, n_streams: int = 1,
                 kv_heads: Optional[int] = None, scale: float = 1.0):
        self.lib = _library()
        if not torch.cuda.is_available():
            raise CBInferError(EDEVICE, "no GPU visible to torch; the HIP path has no CPU fallback")
        decay = [float(g) for g in decay]
        self.heads, self.kv_heads = len(decay), len(decay) if kv_heads is None else int(kv_heads)
        if not decay or not all(0.0 <= g <= 1.0 for g in decay):
            _refuse("decay: one value in 0 .. 1 for each head")
        if self.kv_heads < 1 or self.heads % self.kv_heads:
            _refuse("heads (%d) must be a multiple of kv_heads (%d)" % (self.heads, self.kv_heads))
        if not 1 <= key_size <= 256 or not 1 <= value_size <= 256:
            _refuse("key and value sizes must be 1 .. 256 (got %d and %d)" % (key_size, value_size))
        if n_streams < 1:
            _refuse("n_streams must be >= 1")
        if n_streams * self.heads > 1 << 18:  # here, as the library is told of 32 bits
            _refuse("streams times heads must be at most 2^18 (got %d and %d)" % (n_streams, self.heads))
        self.n_streams, self.key_size, self.value_size, self.scale = int(n_streams), int(key_size), int(value_size), float(scale)
        self._decay = torch.tensor(decay, dtype=torch.float32).cuda()
        self._state = torch.zeros((self.n_streams, self.heads, self.key_size, self.value_size), dtype=torch.float32,
                                  device=self._decay.device)
        self._plan: Optional[_LayerPlan] = None
        a = self._args = linear_attention_args()
        a.streams, a.heads, a.kv_heads = self.n_streams, self.heads, self.kv_heads
        a.key_size, a.value_size, a.scale = self.key_size, self.value_size, self.scale
        a.state, a.decay = self._state.data_ptr(), self._decay.data_ptr()

    @property
    def state(self):
        """[n_streams][heads][key_size][value_size] float32; filled in place to restore what was saved."""
        return self._state

    @property
    def decay(self):
        """[heads] float32."""
        return self._decay

    def reset(self):
        """Forget what the streams have seen."""
        self._state.zero_()

    def process(self, q, k, v, lengths=None, out=None):
        """The next tokens of every stream: q [n_streams][tokens][heads][key_size], k [..][kv_heads][key_size],
        v [..][kv_heads][value_size], the last axis contiguous; lengths: None, or int32 [n_streams], how many of the
        tokens a stream has.  Returns [n_streams][tokens][heads][value_size] and leaves the new state."""
        geometry = (q.shape, q.stride(), k.shape, k.stride(), v.shape, v.stride(), q.dtype, k.dtype, v.dtype, lengths is None,
                    None if out is None else (out.shape, out.stride(), out.dtype))
        plan = self._plan
        if plan is None or plan.geometry != geometry:
            plan = self._plan = self._planned(geometry, q, k, v, lengths, out)
        a = linear_attention_args.from_buffer_copy(plan.args)
        device = _device(q, "q")
        _same_device(k, device, "k")
        _same_device(v, device, "v")
        _same_device(self._state, device, "the state")
        if out is None:
            out = torch.empty(plan.shape, dtype=q.dtype, device=device)
        else:
            _same_device(out, device, "out")
        if lengths is not None:
            if lengths.dtype != torch.int32 or lengths.shape != (self.n_streams,) or not lengths.is_contiguous():
                _refuse("lengths must be a contiguous int32 tensor of n_streams values")
            _same_device(lengths, device, "lengths")
            a.lengths = lengths.data_ptr()
        a.q, a.k, a.v, a.o = q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr()
        keep = _workspace(a, plan.workspace, device)  # noqa: F841
        rc = self.lib.cbinfer_linear_attention(a, _stream(device))
        if rc:
            _raise(rc)
        return out

    def _planned(self, geometry, q, k, v, lengths, out) -> _LayerPlan:
        """Checks of shapes and types, and what follows from them; kept for calls of the same geometry."""
        a = linear_attention_args.from_buffer_copy(self._args)
        if q.dim() != 4:
            _refuse("q must be [streams][tokens][heads][key_size]")
        tokens = q.shape[1]
        if tokens > 1 << 28:
            _refuse("tokens must be at most 2^28 (got %d)" % tokens)
        for t, n, size, what in ((q, self.heads, self.key_size, "q"), (k, self.kv_heads, self.key_size, "k"),
                                 (v, self.kv_heads, self.value_size, "v")):
            if t.shape != (self.n_streams, tokens, n, size):
                _refuse("%s must have the shape %s (got %s)" % (what, (self.n_streams, tokens, n, size), tuple(t.shape)))
            if t.dtype != q.dtype:
                _refuse("q, k and v must have one type")
            if size > 1 and t.stride(3) != 1:
                _refuse("%s: the last axis must be contiguous" % what)
        a.dtype = _dtype(q, "q")
        a.tokens = tokens
        a.q_stride[:], a.k_stride[:], a.v_stride[:] = q.stride()[:3], k.stride()[:3], v.stride()[:3]
        shape = (self.n_streams, tokens, self.heads, self.value_size)
        if out is None:
            a.o_stride[:] = (tokens * self.heads * self.value_size, self.heads * self.value_size, self.value_size)
        else:
            if out.shape != shape or out.dtype != q.dtype or (self.value_size > 1 and out.stride(3) != 1) or not _apart(out):
                _refuse("out must be a tensor like q of shape %s, its values apart in memory" % (shape,))
            a.o_stride[:] = out.stride()[:3]
        a.lengths = None if lengths is None else a.state  # of the workspace it matters only whether there are any
        return _LayerPlan(geometry, a, shape, self.lib.cbinfer_linear_attention_workspace_bytes(a))


# ---- products with 4-bit weights ------------------------------------------------------------------
def quantise_weights(weight, group: int = 64):
    """Codes (uint8 [rows][cols]) and scales (bfloat16 [rows][groups]) of a float matrix, each weight the nearest
    of the 16 values under the scale of its group."""
    lib = _library()
    if weight.dim() != 2 or (weight.shape[1] > 1 and weight.stride(1) != 1):
        _refuse("weight must be a matrix with contiguous rows")
    device, kind = _device(weight, "weight"), _dtype(weight, "weight")
    rows, cols = weight.shape
    if group not in (32, 64, 128):
        _refuse("a group must be 32, 64 or 128 weights (got %r)" % (group,))
    codes = torch.empty((rows, cols), dtype=torch.uint8, device=device)
    scales = torch.empty((rows, -(-cols // group)), dtype=torch.bfloat16, device=device)
    rc = lib.cbinfer_quantise_weights(weight.data_ptr(), kind, rows, cols, weight.stride(0), group, codes.data_ptr(),
                                      scales.data_ptr(), _stream(device))
    if rc:
        _raise(rc)
    return codes, scales


class QuantisedLinear:
    """y = x W^T + bias for few tokens, W of 4-bit codes (uint8 [rows][cols], their lower four bits) with a bfloat16
    scale for each group of 32, 64 or 128 along a row ([rows][ceil(cols / group)]).  The weights are laid out
    once, at construction; codes and scales are not needed afterwards."""

    def __init__(self, codes, scales, bias=None, *, group: int = 64):
        self.lib = _library()
        if codes.dim() != 2 or codes.dtype != torch.uint8 or not codes.is_contiguous():
            _refuse("codes must be a contiguous uint8 matrix")
        device = _device(codes, "codes")
        self.rows, self.cols = codes.shape
        if group not in (32, 64, 128):
            _refuse("a group must be 32, 64 or 128 weights (got %r)" % (group,))
        self.group = int(group)
        nbytes = self.lib.cbinfer_packed_weights_bytes(self.rows, self.cols, self.group)
        if not nbytes:
            _raise(EINVAL)
        want = (self.rows, -(-self.cols // self.group))
        if scales.dtype != torch.bfloat16 or scales.shape != want or not scales.is_contiguous():
            _refuse("scales must be a contiguous bfloat16 tensor of shape %s" % (want,))
        _same_device(scales, device, "scales")
        if bias is not None:
            _float32(bias, device, self.rows, "bias")
        self._bias = bias
        self._memory = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        packed = (self._memory.data_ptr() + 255) // 256 * 256
        rc = self.lib.cbinfer_pack_weights(codes.data_ptr(), scales.data_ptr(), self.rows, self.cols, self.group, packed, _stream(device))
        if rc:
            _raise(rc)
        self._plan: Optional[_LayerPlan] = None
        a = self._args = quantised_product_args()
        a.group, a.rows, a.cols, a.packed = self.group, self.rows, self.cols, packed
        a.bias = None if bias is None else bias.data_ptr()

    @property
    def bias(self):
        """[rows] float32 as given, or None; read by every call, so it may be filled in place."""
        return self._bias

    @classmethod
    def from_weights(cls, weight, bias=None, *, group: int = 64):
        """From a float matrix [rows][cols], quantised here."""
        return cls(*quantise_weights(weight, group), bias, group=group)

    def __call__(self, x, out=None):
        """x [..][cols] float32 or bfloat16 -> [..][rows] of the same type.  Rows of x may lie apart, not their values."""
        geometry = (x.shape, x.stride(), x.dtype)
        plan = self._plan
        if plan is None or plan.geometry != geometry:
            plan = self._plan = self._planned(geometry, x)
        a = quantised_product_args.from_buffer_copy(plan.args)
        device = _device(x, "x")
        _same_device(self._memory, device, "the layer")
        if out is None:
            out = torch.empty(plan.shape, dtype=x.dtype, device=device)
        elif out.shape != plan.shape or out.dtype != x.dtype or out.device != device or not out.is_contiguous():
            _refuse("out must be a contiguous tensor like x of shape %s" % (tuple(plan.shape),))
        a.x, a.y = x.data_ptr(), out.data_ptr()
        keep = _workspace(a, plan.workspace, device)  # noqa: F841
        rc = self.lib.cbinfer_quantised_product(a, _stream(device))
        if rc:
            _raise(rc)
        return out

    def _planned(self, geometry, x) -> _LayerPlan:
        """Checks of shape and type, and what follows from them; kept for calls of the same geometry."""
        a = quantised_product_args.from_buffer_copy(self._args)
        if x.dim() < 1 or x.shape[-1] != self.cols:
            _refuse("x must end in an axis of %d values (got %s)" % (self.cols, tuple(x.shape)))
        if self.cols > 1 and x.stride(-1) != 1:
            _refuse("x: the last axis must be contiguous")
        a.dtype = _dtype(x, "x")
        a.tokens, a.x_stride = _joined_rows(x)
        a.y_stride = self.rows
        return _LayerPlan(geometry, a, x.shape[:-1] + (self.rows,), self.lib.cbinfer_quantised_product_workspace_bytes(a))


def _joined_rows(t):
    """Number of rows in front of the last axis and the stride between them."""
    if t.dim() == 2:
        return t.shape[0], t.stride(0)
    if 0 in t.shape[:-1]:
        return 0, 0
    n, step = 1, t.shape[-1]
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if n == 1:
            step = stride
        elif stride != step * n:
            _refuse("the axes in front of the last must lie behind one another as one; call .contiguous()")
        n *= size
    return n, step


# ---- norms around a block -------------------------------------------------------------------------
def gated_norm(x, weight=None, *, group: int = 0, gate=None, activation: Optional[str] = None, residual=None, scale=1.0,
               next_weight=None, eps: float = 1e-6, sum_out=None):
    """u = x / rms(x, per `group` values) * weight; u *= silu(gate) or sigmoid(gate) (`activation`);
    h = residual + scale * u (scale: a number, or float32 per channel); y = h / rms(h) * next_weight.
    Rows along the last axis; parts that are None are left out.  Returns (h, y): h has the type of the residual
    (float32 or that of x), y (None without next_weight) that of x.  sum_out: where h goes, e.g. the residual itself."""
    device = _device(x, "x")
    key = (x.shape, x.stride(), x.dtype, group, activation, eps, weight is None, next_weight is None,
           None if gate is None else (gate.shape, gate.stride(), gate.dtype),
           None if residual is None else (residual.shape, residual.stride(), residual.dtype),
           None if sum_out is None else (sum_out.shape, sum_out.stride(), sum_out.dtype))
    plan = _norm_plans.get(key)
    if plan is None:
        plan = _norm_plan(x, weight, group, gate, activation, residual, next_weight, eps, sum_out)
        if len(_norm_plans) >= 1024:
            _norm_plans.clear()
        _norm_plans[key] = plan
    a = gated_norm_args.from_buffer_copy(plan[0])
    size = a.size
    a.x = x.data_ptr()
    if weight is not None:
        _float32(weight, device, size, "weight")
        a.weight = weight.data_ptr()
    if gate is not None:
        _same_device(gate, device, "gate")
        a.gate = gate.data_ptr()
    if residual is not None:
        _same_device(residual, device, "residual")
        a.residual = residual.data_ptr()
    if isinstance(scale, torch.Tensor):
        _float32(scale, device, size, "scale")
        a.scale, a.channel_scale = 1.0, scale.data_ptr()
    else:
        a.scale = scale
    if sum_out is None:
        h = torch.empty(x.shape, dtype=plan[1], device=device)
    else:
        h = sum_out
        _same_device(h, device, "sum_out")
    a.h = h.data_ptr()
    y = None
    if next_weight is not None:
        _float32(next_weight, device, size, "next_weight")
        y = torch.empty(x.shape, dtype=x.dtype, device=device)
        a.next_weight, a.y = next_weight.data_ptr(), y.data_ptr()
    rc = _lib.cbinfer_gated_norm(a, _stream(device))
    if rc:
        _raise(rc)
    return h, y


# Checked arguments by shapes, strides and types, as those of log_probs.
_norm_plans: dict = {}


def _norm_plan(x, weight, group, gate, activation, residual, next_weight, eps, sum_out):
    """Everything but addresses and the scale, and the type of the sum."""
    _library()
    a = gated_norm_args()
    shape, kind = x.shape, x.dtype
    a.size = shape[-1] if x.dim() else 0
    if a.size < 1:
        _refuse("x must end in an axis of at least one value")
    a.dtype = a.sum_dtype = _dtype(x, "x")
    a.eps = eps
    a.rows, a.x_stride = _norm_rows(x, shape, "x")
    if weight is not None:
        if not 0 <= group <= a.size:
            _refuse("group must be 0 or divide the size, %d (got %r)" % (a.size, group))
        a.group = group
    elif group:
        _refuse("group without weight")
    if (gate is None) != (activation is None) or activation not in GATES:
        _refuse("gate and activation ('silu' or 'sigmoid') go together")
    if gate is not None:
        if gate.dtype != kind:
            _refuse("gate must have the type of x")
        _, a.gate_stride = _norm_rows(gate, shape, "gate")
        a.gate_kind = GATES[activation]
    sum_kind = kind
    if residual is not None:
        if residual.dtype not in (kind, torch.float32):
            _refuse("residual must be float32 or have the type of x")
        sum_kind = residual.dtype
        a.sum_dtype = _dtype(residual, "residual")
        _, a.residual_stride = _norm_rows(residual, shape, "residual")
    if sum_out is not None:
        if sum_out.dtype != sum_kind:
            _refuse("sum_out must have the type of the residual (without one: of x)")
        _, a.h_stride = _norm_rows(sum_out, shape, "sum_out")
        if not _apart(sum_out):
            _refuse("sum_out: its values must lie apart in memory")
    else:
        a.h_stride = a.size
    a.y_stride = a.size
    return a, sum_kind


def _norm_rows(t, shape, what: str):
    if t.shape != shape:
        _refuse("%s must have the shape of x, %s (got %s)" % (what, tuple(shape), tuple(t.shape)))
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse("%s: the last axis must be contiguous" % what)
    return _joined_rows(t)
