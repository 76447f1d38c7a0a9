"""A text model around the sparse convolutions: word vectors, their gradient and a fully connected layer in 8-bit integers.

`Embedding` and `Int8Linear` call the library's operators (include/sparse_conv.h) on PyTorch tensors.  A call's tensors are checked,
and its output and scratch memory allocated, by csrc/text_torch.cpp: calls of few tokens are bound by the host.  There is no fallback.

Autograd does not record these calls: their outputs have no gradient function, also where a table or an input requires a gradient.
`Embedding.backward` is called by the program itself.  A write into a given `out` raises that tensor's version.
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
        "embed", "embed_backward_workspace", "embed_backward", "int8_linear_workspace", "int8_linear")))


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
