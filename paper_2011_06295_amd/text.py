"""A text model around the sparse convolutions: word vectors, their gradient and a fully connected layer in 8-bit integers; and what trains
the layers behind the convolutions: a fully connected layer with its gradients, a classifier's loss, AdamW steps.

`Embedding`, `Int8Linear`, `Linear`, `cross_entropy` and `AdamW` call the library's operators (include/sparse_conv.h) on PyTorch tensors.  A call's tensors are checked,
and its output and scratch memory allocated, by csrc/text_torch.cpp: calls of few tokens are bound by the host.  There is no fallback.

Autograd does not record these calls: their outputs have no gradient function, also where a table or an input requires a gradient.
`Embedding.backward` and `Linear.backward` are called by the program itself.  A write into a given `out` raises that tensor's version.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B
from .build import TORCH_LIB

try:
    from . import _text_torch as _calls
except ImportError as e:
    raise ImportError(f"{TORCH_LIB} is missing or does not load ({e}): build it with `python -m paper_2011_06295_amd.build`") from e

_DTYPES = {torch.float32: B.SC_F32, torch.float16: B.SC_F16, torch.bfloat16: B.SC_BF16}
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_current_stream = B._current_stream


def _bind():
    import ctypes as C
    lib = B.raw_library()
    _calls.bind(*(C.cast(getattr(lib, "sparse_conv_" + name), C.c_void_p).value for name in (
        "embed", "embed_backward_workspace", "embed_backward", "int8_linear_workspace", "int8_linear", "linear_workspace", "linear",
        "linear_backward_workspace", "linear_backward", "cross_entropy", "adamw", "adamw_count")))


_bind()


class Embedding:
    """Rows of a table [vocab][dim] (fp32, binary16 or bfloat16) for tokens, times `scale`, and the gradient of the table.
    A token outside 0..vocab-1 reads as zeros and has no gradient; the row of token `padding` has no gradient.  `backward` computes
    that gradient when it is called: autograd does not record `forward`."""

    def __init__(self, table: torch.Tensor, scale: float = 1.0, padding: Optional[int] = None):
        if not table.is_cuda or table.dtype not in _DTYPES or table.dim() != 2 or not table.is_contiguous():
            raise ValueError("table must be a contiguous CUDA tensor [vocab][dim] of fp32, binary16 or bfloat16")
        self.table = table
        self.scale = float(scale)
        self.padding = -1 if padding is None else int(padding)
        self.vocab, self.dim = table.shape
        self._device = table.get_device()
        if not -1 <= self.padding < self.vocab:
            raise ValueError("padding must be a token of the table")

    def forward(self, tokens, channels_first: bool = False, out=None):
        """Vectors [..., dim] of tokens [...] (contiguous, 32- or 64-bit integers); with channels_first [sentences][dim][1][words] of
        tokens [sentences][words], the input of a 1-D convolution layer."""
        if self._device != _current_device():      # the library's calls run on the current device
            with torch.cuda.device(self._device):
                return self.forward(tokens, channels_first, out)
        out = _calls.embed(self.table, tokens, out, channels_first, self.scale, _current_stream(self._device))
        if out.__class__ is int:
            B._check(out, "sparse_conv_embed")
        return out

    def backward(self, grad, tokens, channels_first: bool = False, out=None, accumulate: bool = False):
        """Gradient [vocab][dim] of the table (fp32 or the type of grad; without `out` the table's type) from the gradient of
        what forward gave for these tokens.  accumulate: added to what `out` holds."""
        if self._device != _current_device():
            with torch.cuda.device(self._device):
                return self.backward(grad, tokens, channels_first, out, accumulate)
        out = _calls.embed_backward(self.table, grad, tokens, out, channels_first, accumulate, self.scale, self.padding, _current_stream(self._device))
        if out.__class__ is int:
            B._check(out, "sparse_conv_embed_backward")
        return out


def quantize(x: torch.Tensor):
    """(8-bit integers [rows][int8_pitch(K)], fp32 scales [rows]) of the rows of x [rows][K]; row strides may exceed K."""
    if not x.is_cuda or x.dtype not in _DTYPES or x.dim() != 2 or x.shape[1] < 1 or (x.stride(1) != 1 and x.shape[1] > 1):
        raise ValueError("x must be a CUDA tensor [rows][K] of fp32, binary16 or bfloat16 whose rows are contiguous")
    rows, K = x.shape
    ldx = x.stride(0) if rows > 1 else K
    if ldx < K:
        raise ValueError("the rows of x overlap")
    with torch.cuda.device(x.device):
        q = torch.empty((rows, B.int8_pitch(K)), dtype=torch.int8, device=x.device)
        scale = torch.empty(rows, dtype=torch.float32, device=x.device)
        B.sparse_conv_int8_quantize(x.data_ptr(), q.data_ptr(), scale.data_ptr(), rows, K, ldx, _DTYPES[x.dtype], _current_stream(x.get_device()))
    return q, scale


class Int8Linear:
    """Fully connected layer whose weights are 8-bit integers with a scale for each output channel; the input is quantised
    within the call, with a scale for each token (row).  Autograd does not record it; `dequantized` gives the weights that a
    gradient of the input goes through."""

    def __init__(self, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, relu: bool = False):
        """weight: CUDA tensor [N][K] of fp32, binary16 or bfloat16, quantised here; bias: [N] or None."""
        q, scale = quantize(weight)
        self._set(q, scale, weight.shape[1], bias, relu)

    @classmethod
    def from_quantized(cls, weight: torch.Tensor, scale: torch.Tensor, bias: Optional[torch.Tensor] = None, relu: bool = False) -> "Int8Linear":
        """weight: CUDA tensor [N][K] of 8-bit integers, laid out here where K is not a whole number of 128 (else kept as it is,
        not copied); scale: fp32 [N]."""
        if not weight.is_cuda or weight.dtype != torch.int8 or weight.dim() != 2 or min(weight.shape) < 1:
            raise ValueError("weight must be a CUDA tensor [N][K] of 8-bit integers")
        if scale.shape != weight.shape[:1] or scale.dtype != torch.float32 or scale.device != weight.device:
            raise ValueError("scale must be an fp32 tensor [N] on the weight's device")
        self = cls.__new__(cls)
        N, K = weight.shape
        if K == B.int8_pitch(K) and weight.is_contiguous() and weight.data_ptr() % 16 == 0:
            q = weight          # laid out as the library reads it: kept as it is
        else:
            q = torch.zeros((N, B.int8_pitch(K)), dtype=torch.int8, device=weight.device)
            q[:, :K] = weight
        self._set(q, scale.contiguous(), K, bias, relu)
        return self

    def _set(self, q, scale, K, bias, relu):
        self.N, self.K = q.shape[0], K
        self.weight, self.scale, self.relu = q, scale, relu
        if bias is not None:
            if bias.shape != (self.N,) or bias.device != q.device:
                raise ValueError("bias must be a tensor [N] on the weight's device")
            bias = bias.detach().to(torch.float32).contiguous()
        self.bias = bias
        self._device = q.get_device()

    def dequantized(self) -> torch.Tensor:
        """The weights that the 8-bit integers stand for: fp32 [N][K]."""
        return self.weight[:, :self.K].float() * self.scale[:, None]

    def forward(self, x, out=None, dtype: Optional[torch.dtype] = None):
        """[..., N] of x [..., K] (contiguous, or [M][K] with contiguous rows at any stride); dtype: of the output, x's by default."""
        return self._call(x, None, out, dtype)

    def forward_quantized(self, q, scale, out=None, dtype: Optional[torch.dtype] = None):
        """The layer on rows that `quantize` made: q [M][int8_pitch(K)], scale [M]; the output is fp32 by default."""
        return self._call(q, scale, out, dtype)

    def _call(self, x, scale, out, dtype):
        if self._device != _current_device():      # the library's calls run on the current device
            with torch.cuda.device(self._device):
                return self._call(x, scale, out, dtype)
        out = _calls.linear(x, scale, self.weight, self.scale, self.bias, self.K, self.relu, out, dtype, _current_stream(self._device))
        if out.__class__ is int:
            B._check(out, "sparse_conv_int8_linear")
        return out


_ACTIVATIONS = {None: B.SC_ACT_NONE, "relu": B.SC_ACT_RELU, "gelu": B.SC_ACT_GELU, "silu": B.SC_ACT_SILU}


class Linear:
    """Fully connected layer act(x W^T + bias) + residual in the weight's type, summed in fp32, and its gradients.  The weight and the bias are
    read when a call runs: a step that changes them in place needs no new layer.  Autograd does not record the calls: `backward` is called
    by the program itself."""

    def __init__(self, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, activation: Optional[str] = None):
        """weight: CUDA tensor [N][K] of fp32, binary16 or bfloat16 (kept, not copied; rows may lie apart); bias: fp32 [N] or None;
        activation: None, "relu", "gelu" (x Phi(x)) or "silu"."""
        if not weight.is_cuda or weight.dtype not in _DTYPES or weight.dim() != 2 or min(weight.shape) < 1 or (weight.stride(1) != 1 and weight.shape[1] > 1):
            raise ValueError("weight must be a CUDA tensor [N][K] of fp32, binary16 or bfloat16 whose rows are contiguous")
        if bias is not None and (bias.shape != weight.shape[:1] or bias.dtype != torch.float32 or bias.device != weight.device or not bias.is_contiguous()):
            raise ValueError("bias must be a contiguous fp32 tensor [N] on the weight's device")
        if activation not in _ACTIVATIONS:
            raise ValueError('activation must be None, "relu", "gelu" or "silu"')
        self.weight, self.bias, self.activation = weight, bias, activation
        self.N, self.K = weight.shape
        self._act = _ACTIVATIONS[activation]
        self._device = weight.get_device()

    def forward(self, x, residual=None, keep: bool = False, out=None):
        """[..., N] of x [..., K] (contiguous, or [M][K] with contiguous rows at any stride), plus residual [..., N], which may be `out` itself.
        keep: (output, z), z what went into the activation, as `backward` needs it."""
        if self._device != _current_device():      # the library's calls run on the current device
            with torch.cuda.device(self._device):
                return self.forward(x, residual, keep, out)
        out = _calls.layer(x, self.weight, self.bias, residual, out, keep, self._act, _current_stream(self._device))
        if out.__class__ is int:
            B._check(out, "sparse_conv_linear")
        return out

    def backward(self, grad, x, z=None, grad_x=True, grad_weight=True, grad_bias=True, accumulate: bool = False):
        """(gradient of x, of the weight, of the bias (fp32)) from the gradient of the output, which is the residual's as well.  x: what
        forward was given (None where grad_weight is False); z: what it kept, needed with an activation.  Each of the three is made (True), left out
        (False, None comes back) or written to the tensor given; accumulate: the weight's and the bias's are added to those tensors."""
        if self._device != _current_device():
            with torch.cuda.device(self._device):
                return self.backward(grad, x, z, grad_x, grad_weight, grad_bias, accumulate)
        if self.bias is None and grad_bias is True:
            grad_bias = False
        out = _calls.layer_backward(grad, x, self.weight, z, grad_x, grad_weight, grad_bias, accumulate, self._act, _current_stream(self._device))
        if out.__class__ is int:
            B._check(out, "sparse_conv_linear_backward")
        return out


def cross_entropy(logits, labels, weights=None, grad=True, scale: float = 1.0):
    """(losses fp32 [...], gradient of their sum towards the logits [..., classes] or None) of logits [..., classes] and labels [...]:
    scale * weights * -log of the softmax at the label.  A row whose label is no class, or whose weight is 0, counts for nothing.
    grad: True, False or the tensor to write to, which may be `logits` itself.  Autograd does not record the call."""
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda:
        raise ValueError("logits must be a CUDA tensor [..., classes] of fp32, binary16 or bfloat16")
    device = logits.get_device()
    if device != _current_device():
        with torch.cuda.device(device):
            return cross_entropy(logits, labels, weights, grad, scale)
    out = _calls.cross_entropy(logits, labels, weights, grad, float(scale), _current_stream(device))
    if out.__class__ is int:
        B._check(out, "sparse_conv_cross_entropy")
    return out


class AdamW:
    """AdamW steps over many tensors at once, in place: m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
    p = (1 - rate decay) p - rate (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps), in fp32.

    States (`m`, `v`, with 8 bits `m_scale` and `v_scale`, with master `master`) are one array each for all tensors; tensor i's begin at element
    `begins[i]`, a whole number of blocks of 256.  They are zero at first and can be copied out and in, with `steps`, the number of
    steps taken."""

    def __init__(self, params, rate: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, decay: float = 0.01, bits: int = 32, master: bool = False,
                 counted: bool = False):
        """params: contiguous CUDA tensors of one type (fp32, binary16, bfloat16) and device.  bits: 32, or 8: numbers of 8 bits (e4m3)
        with an fp32 scale for each block of 256, and beta1 up to 0.9 (m is rounded to the nearest number, by which a steady gradient may leave it off by a factor
        of 2.25; closer to 1 it would stop following).  master: steps apply to fp32 weights kept here, the parameters receive them rounded
        (else a 16-bit parameter loses every change below half its own rounding).  counted: the number of steps is counted in device
        memory, for steps recorded in a graph (`steps` is then a tensor)."""
        self.params = list(params)
        if not self.params or any(not isinstance(p, torch.Tensor) or not p.is_cuda or p.dtype not in _DTYPES or not p.is_contiguous() for p in self.params):
            raise ValueError("params must be contiguous CUDA tensors of fp32, binary16 or bfloat16")
        first = self.params[0]
        if any(p.dtype != first.dtype or p.device != first.device for p in self.params):
            raise ValueError("params must be of one type and on one device (an optimizer for each)")
        spans = sorted((p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()) for p in self.params if p.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("params must not share memory")
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        beta1, beta2 = (float(b) for b in betas)
        self.rate, self.betas, self.eps, self.decay, self.bits = float(rate), (beta1, beta2), float(eps), float(decay), bits
        if not (0.0 <= beta1 < 1.0 and 0.0 <= beta2 < 1.0 and self.rate >= 0.0 and self.eps >= 0.0 and self.decay >= 0.0):
            raise ValueError("rate, eps and decay must not be negative, betas at least 0 and below 1")
        if bits == 8 and beta1 > 0.9:      # a change of m by less than half a step between numbers of 8 bits is lost
            raise ValueError("with states of 8 bits beta1 is 0.9 at most")
        self.begins = [0]
        for p in self.params:
            self.begins.append(self.begins[-1] + -(-p.numel() // B.SC_ADAMW_BLOCK) * B.SC_ADAMW_BLOCK)
        total, device = self.begins.pop(), first.device
        self.m, self.v = (torch.zeros(total, dtype=torch.float32 if bits == 32 else torch.float8_e4m3fn, device=device) for _ in range(2))
        self.m_scale = self.v_scale = self.master = None
        if bits == 8:
            self.m_scale, self.v_scale = (torch.zeros(total // B.SC_ADAMW_BLOCK, device=device) for _ in range(2))
        if master:
            self.master = torch.zeros(total, device=device)
            for begin, p in zip(self.begins, self.params):
                self.master[begin:begin + p.numel()].copy_(p.detach().reshape(-1))
        self.steps = torch.zeros(1, dtype=torch.int64, device=device) if counted else 0
        self._counted = torch.zeros(B.SC_ADAMW_COUNTED_BYTES // 4, device=device) if counted else None
        self._device = first.get_device()

    def step(self, grads, scale: float = 1.0):
        """One step on scale * grads: a contiguous tensor like each parameter (all fp32 or of the parameters' type; any of the three types where
        parameters are fp32), or None, which leaves the parameter and its states alone.  Rates and scale are kept by a graph as they were when
        it was recorded."""
        if self._device != _current_device():
            with torch.cuda.device(self._device):
                return self.step(grads, scale)
        grads = grads if isinstance(grads, list) else list(grads)
        if self._counted is None and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("a step recorded in a graph would keep its number in every replay: make the optimizer with counted=True")
        counted = None if self._counted is None else (self.steps, self._counted)
        rule = (self.rate, *self.betas, self.eps, self.decay, scale)
        rc = _calls.adamw(self.params, grads, self.m, self.v, self.m_scale, self.v_scale, self.master, counted, rule,
                          self.steps + 1 if counted is None else 1, _current_stream(self._device))
        B._check(rc, "sparse_conv_adamw")
        if counted is None:
            self.steps += 1
