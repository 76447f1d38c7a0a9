"""A text model around the sparse convolutions: word vectors, their gradient and a fully connected layer in 8-bit integers.

`Embedding` and `Int8Linear` marshal arguments for the library's operators (include/sparse_conv.h); tensors are checked here,
scratch memory comes from PyTorch's allocator on the stream that is current at the call.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B

_DTYPES = {torch.float32: B.SC_F32, torch.float16: B.SC_F16, torch.bfloat16: B.SC_BF16}
_lib = B.raw_library()
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


class Embedding:
    """Rows of a table [vocab][dim] (fp32, binary16 or bfloat16) for tokens, times `scale`, and the gradient of the table.
    A token outside 0..vocab-1 reads as zeros and has no gradient; the row of token `padding` has no gradient."""

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
        self._workspaces = {}

    def _tokens(self, tokens, channels_first):
        """(sentences, words, flags) of a call."""
        if (tokens.dtype != torch.int64 and tokens.dtype != torch.int32) or not tokens.is_contiguous() \
                or tokens.get_device() != self._device or (channels_first and tokens.dim() != 2):
            raise ValueError("tokens must be a contiguous tensor of 32- or 64-bit integers on the table's device "
                             "([sentences][words] for channels_first)")
        flags = B.SC_EMBED_TOKENS_64 if tokens.dtype == torch.int64 else 0
        if channels_first:
            return tokens.shape[0], tokens.shape[1], flags | B.SC_EMBED_CHANNELS_FIRST
        return 1, tokens.numel(), flags

    def forward(self, tokens, channels_first: bool = False, out=None):
        """Vectors [..., dim] of tokens [...]; with channels_first [sentences][dim][1][words] of tokens [sentences][words],
        the input of a 1-D convolution layer."""
        if self._device != _current_device():      # the library's calls run on the current device
            with torch.cuda.device(self._device):
                return self.forward(tokens, channels_first, out)
        n, t, flags = self._tokens(tokens, channels_first)
        shape = (n, self.dim, 1, t) if channels_first else (*tokens.shape, self.dim)
        table = self.table
        if out is None:
            out = table.new_empty(shape)
        elif out.shape != shape or out.dtype != table.dtype or out.device != table.device or not out.is_contiguous():
            raise ValueError("bad output tensor")
        rc = _lib.sparse_conv_embed(table.data_ptr(), tokens.data_ptr(), out.data_ptr(), self.vocab, self.dim, n, t, _DTYPES[table.dtype],
                                    self.scale, flags, B._current_stream(self._device) or None)
        if rc:
            B._check(rc, "sparse_conv_embed")
        return out

    def backward(self, grad, tokens, channels_first: bool = False, out=None, accumulate: bool = False):
        """Gradient [vocab][dim] of the table (fp32 or the type of grad; without `out` the table's type) from the gradient of
        what forward gave for these tokens.  accumulate: added to what `out` holds."""
        if self._device != _current_device():
            with torch.cuda.device(self._device):
                return self.backward(grad, tokens, channels_first, out, accumulate)
        n, t, flags = self._tokens(tokens, channels_first)
        shape = (n, self.dim, 1, t) if channels_first else (*tokens.shape, self.dim)
        table = self.table
        if grad.shape != shape or grad.dtype not in _DTYPES or not grad.is_contiguous() or grad.device != table.device:
            raise ValueError("grad must be a contiguous tensor of the shape that forward gives")
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs the tensor to add to")
            out = table.new_empty(table.shape)
        elif out.shape != table.shape or out.device != table.device or not out.is_contiguous():
            raise ValueError("bad output tensor")
        if out.dtype != torch.float32 and out.dtype != grad.dtype:
            raise ValueError("the table's gradient is fp32 or of the type of grad")
        g = _DTYPES[grad.dtype]
        key = (n, t, g, flags)
        nbytes = self._workspaces.get(key)
        if nbytes is None:      # the size for these shapes is asked of the library once
            nbytes = self._workspaces[key] = B.sparse_conv_embed_backward_workspace(self.vocab, self.dim, n, t, g, flags)
        work = table.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
        rc = _lib.sparse_conv_embed_backward(grad.data_ptr(), tokens.data_ptr(), out.data_ptr(), self.vocab, self.dim, n, t, g,
                                             _DTYPES[out.dtype], self.scale, self.padding,
                                             flags | (B.SC_EMBED_ACCUMULATE if accumulate else 0),
                                             work.data_ptr() if nbytes else None, nbytes, B._current_stream(self._device) or None)
        if rc:
            B._check(rc, "sparse_conv_embed_backward")
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
        B.sparse_conv_int8_quantize(x.data_ptr(), q.data_ptr(), scale.data_ptr(), rows, K, ldx, _DTYPES[x.dtype], B._current_stream(x.get_device()))
    return q, scale


class Int8Linear:
    """Fully connected layer whose weights are 8-bit integers with a scale for each output channel; the input is quantised
    within the call, with a scale for each token (row)."""

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
        self.N, self.K, self.pitch = q.shape[0], K, q.shape[1]
        self.weight, self.scale, self.relu = q, scale, relu
        if bias is not None:
            if bias.shape != (self.N,) or bias.device != q.device:
                raise ValueError("bias must be a tensor [N] on the weight's device")
            bias = bias.detach().to(torch.float32).contiguous()
        self.bias = bias
        self._device = q.get_device()
        self._pointers = (q.data_ptr(), scale.data_ptr(), 0 if bias is None else bias.data_ptr())
        self._flags = B.SC_EPILOGUE_RELU if relu else 0
        self._workspaces = {}

    def dequantized(self) -> torch.Tensor:
        """The weights that the 8-bit integers stand for: fp32 [N][K]."""
        return self.weight[:, :self.K].float() * self.scale[:, None]

    def _call(self, x, x_scale, in_dtype, M, ldx, lead, dtype, out):
        if out is None:
            out = x.new_empty((*lead, self.N), dtype=dtype)
            ldo = self.N
        else:
            if out.shape != (*lead, self.N) or out.dtype not in _DTYPES or out.device != x.device:
                raise ValueError("bad output tensor")
            dtype = out.dtype
            if out.is_contiguous():
                ldo = self.N
            elif out.dim() == 2 and (out.stride(1) == 1 or self.N == 1) and out.stride(0) >= self.N:
                ldo = out.stride(0)
            else:
                raise ValueError("bad output tensor")
        od = _DTYPES[dtype]
        key = (M, in_dtype, od)
        nbytes = self._workspaces.get(key)
        if nbytes is None:      # the size for these shapes is asked of the library once
            if len(self._workspaces) > 4096:
                self._workspaces.clear()
            nbytes = self._workspaces[key] = B.sparse_conv_int8_linear_workspace(M, self.N, self.K, in_dtype, od)
        work = self.weight.new_empty(nbytes) if nbytes else None
        w, ws, bias = self._pointers
        rc = _lib.sparse_conv_int8_linear(x.data_ptr(), x_scale, w, ws, bias or None, out.data_ptr(), M, self.N, self.K, ldx, ldo, in_dtype, od,
                                          self._flags, work.data_ptr() if nbytes else None, nbytes, B._current_stream(self._device) or None)
        if rc:
            B._check(rc, "sparse_conv_int8_linear")
        return out

    def forward(self, x, out=None, dtype: Optional[torch.dtype] = None):
        """[..., N] of x [..., K] (contiguous, or [M][K] with contiguous rows at any stride); dtype: of the output, x's by default."""
        if self._device != _current_device():      # the library's calls run on the current device
            with torch.cuda.device(self._device):
                return self.forward(x, out, dtype)
        t = x.dtype
        if t not in _DTYPES or x.get_device() != self._device or x.dim() < 1 or x.shape[-1] != self.K:
            raise ValueError("x must be a tensor [..., K] of fp32, binary16 or bfloat16 on the layer's device")
        if x.is_contiguous():
            ldx = self.K
        elif x.dim() == 2 and (x.stride(1) == 1 or self.K == 1) and x.stride(0) >= self.K:
            ldx = x.stride(0)
        else:
            raise ValueError("x must be contiguous, or [M][K] with contiguous rows that do not overlap")
        return self._call(x, None, _DTYPES[t], x.numel() // self.K, ldx, x.shape[:-1], t if dtype is None else dtype, out)

    def forward_quantized(self, q, scale, out=None, dtype: torch.dtype = torch.float32):
        """The layer on rows that `quantize` made: q [M][int8_pitch(K)], scale [M]."""
        if self._device != _current_device():
            with torch.cuda.device(self._device):
                return self.forward_quantized(q, scale, out, dtype)
        if q.dtype != torch.int8 or q.dim() != 2 or q.shape[1] != self.pitch or not q.is_contiguous() or q.get_device() != self._device \
                or scale.shape != q.shape[:1] or scale.dtype != torch.float32 or not scale.is_contiguous() or scale.device != q.device:
            raise ValueError("q must be [M][int8_pitch(K)] 8-bit integers and scale fp32 [M], as quantize makes them")
        return self._call(q, scale.data_ptr(), B.SC_I8, q.shape[0], self.pitch, q.shape[:1], dtype, out)
