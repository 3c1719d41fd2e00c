"""Training operators of the library (include/novak.h, "Training operators"):
8-bit forms of activations, layer norm, root-mean-square norm with the residual's
addition, activation functions, the weight gradient of a linear layer, token embedding
and its gradient, and orthogonalised updates of matrices, on torch tensors.

A tensor is seen as rows of its last dimension, its address goes to the C entry
point of the same name, and the work is enqueued on torch's current stream of the
tensors' device.  Results are new tensors of that stream.  The marshalling is compiled
(csrc/novak_torch.cpp).  Nothing here records gradients: ``block`` has the autograd side.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import math

import torch

from . import binding as B
from . import build as _build

BLOCK = 32          # elements that share an exponent byte
_TYPE = {torch.float32: B.NOVAK_TYPE_F32, torch.bfloat16: B.NOVAK_TYPE_BF16}
_KIND = {"gelu": B.NOVAK_ACT_GELU, "gelu_tanh": B.NOVAK_ACT_GELU_TANH, "silu": B.NOVAK_ACT_SILU}
_ENTRIES = ("novak_act8_pack", "novak_act8_unpack", "novak_layer_norm", "novak_layer_norm_backward_bytes",
            "novak_layer_norm_backward", "novak_activation", "novak_activation_backward",
            "novak_linear_weight_grad_bytes", "novak_linear_weight_grad", "novak_rms_norm",
            "novak_rms_norm_backward_bytes", "novak_rms_norm_backward", "novak_embedding", "novak_embedding_grad_bytes",
            "novak_embedding_grad", "novak_orthogonalize_bytes", "novak_orthogonalize", "novak_orthogonal_step",
            "novak_orthogonalize_fine_bytes", "novak_orthogonalize_fine", "novak_orthogonal_step_fine", "novak_ops_error")

# The triples (a, b, c) of five Newton-Schulz steps that bring singular values above 1e-3 of the
# largest to between 0.7 and 1.2 (those of the Muon optimiser).
NEWTON_SCHULZ = ((3.4445, -4.7750, 2.0315),) * 5


class _Calls:
    """The host extension, put in this one's place in ``_calls`` by the first call: loading
    it may build it and the library."""

    def __getattr__(self, name: str):
        global _calls
        loader = importlib.machinery.ExtensionFileLoader("_novak_torch", _build.build_torch())
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_novak_torch", loader))
        loader.exec_module(module)
        lib = B.load_library()
        module.bind(B.NovakError, *(ctypes.cast(getattr(lib, entry), ctypes.c_void_p).value for entry in _ENTRIES))
        _calls = module
        return getattr(module, name)


_calls = _Calls()


def _type(dtype, name: str) -> int:
    try:
        return _TYPE[dtype]
    except KeyError:
        raise TypeError(f"{name} must be float32 or bfloat16, got {dtype}") from None


def _folded(shape, rows: int, cols: int):
    shape = (rows, cols) if shape is None else tuple(shape)
    if not shape or shape[-1] != cols or math.prod(shape[:-1]) != rows:
        raise ValueError(f"shape {shape} does not fold into {rows} rows of {cols} elements")
    return shape


class Act8:
    """The 8-bit form of a matrix: ``codes`` (int8, rows x padded columns) and ``exps``
    (uint8, rows x padded columns / 32), see include/novak.h.  ``shape`` is that of the
    tensor it was made from."""

    __slots__ = ("_codes", "_exps", "_both", "rows", "cols", "shape", "codes_ptr", "exps_ptr", "index")

    def __init__(self, codes, exps, cols: int, shape=None):
        rows, pitch = codes.shape
        if codes.dtype != torch.int8 or exps.dtype != torch.uint8:
            raise TypeError("codes must be int8 and exps uint8")
        if cols < 1 or pitch != (cols + BLOCK - 1) // BLOCK * BLOCK or exps.shape != (rows, pitch // BLOCK):
            raise ValueError(f"no 8-bit form of rows of {cols} elements: codes {tuple(codes.shape)}, "
                             f"exps {tuple(exps.shape)}")
        shape = _folded(shape, rows, cols)
        index = codes.get_device()
        if not codes.is_contiguous() or not exps.is_contiguous() or index < 0 or exps.get_device() != index:
            raise ValueError("codes and exps must be contiguous CUDA tensors of one device")
        self.codes_ptr, self.exps_ptr = codes.data_ptr(), exps.data_ptr()
        if self.codes_ptr % 32 and rows:
            raise ValueError("codes must be 32-byte aligned")
        self._codes, self._exps, self._both, self.rows, self.cols, self.index = codes, exps, None, rows, cols, index
        self.shape = shape

    @classmethod
    def from_buffer(cls, buffer, cols: int, shape=None):
        """The form whose ``buffer`` this is (or a copy of it), of rows of ``cols`` elements."""
        if buffer.dtype != torch.uint8 or buffer.dim() != 1 or not buffer.is_contiguous():
            raise TypeError("a form's buffer is one contiguous dimension of uint8")
        size = (cols + BLOCK - 1) // BLOCK * (BLOCK + 1)
        if cols < 1 or buffer.shape[0] % size or buffer.get_device() < 0 or buffer.data_ptr() % 32:
            raise ValueError(f"no buffer of the 8-bit form of rows of {cols} elements: {buffer.shape[0]} bytes on "
                             f"{buffer.device}")
        return cls._of(buffer, cols, _folded(shape, buffer.shape[0] // size, cols))

    @classmethod
    def _of(cls, both, cols: int, shape):
        """The form in a buffer of codes and exponents that an operator has written."""
        self = object.__new__(cls)
        blocks = (cols + BLOCK - 1) // BLOCK
        rows = both.shape[0] // (blocks * (BLOCK + 1))
        self._codes = self._exps = None
        self._both, self.rows, self.cols, self.shape, self.index = both, rows, cols, shape, both.get_device()
        self.codes_ptr = both.data_ptr()
        self.exps_ptr = self.codes_ptr + rows * blocks * BLOCK
        return self

    def _split(self):
        blocks = (self.cols + BLOCK - 1) // BLOCK
        n = self.rows * blocks * BLOCK
        self._codes = self._both[:n].view(torch.int8).view(self.rows, blocks * BLOCK)
        self._exps = self._both[n:].view(self.rows, blocks)

    @property
    def codes(self):
        if self._codes is None:
            self._split()
        return self._codes

    @property
    def exps(self):
        if self._exps is None:
            self._split()
        return self._exps

    @property
    def buffer(self):
        """Codes and exponents as one tensor, codes first: what to keep, move or save of a form."""
        if self._both is None:
            return torch.cat([self._codes.view(torch.uint8).view(-1), self._exps.view(-1)])
        return self._both

    @property
    def device(self):
        return (self._codes if self._both is None else self._both).device

    @property
    def nbytes(self) -> int:
        return self.rows * ((self.cols + BLOCK - 1) // BLOCK) * (BLOCK + 1)

    def __repr__(self):
        return f"Act8(shape={tuple(self.shape)}, {self.nbytes} bytes on {self.device})"


def act8_pack(x) -> Act8:
    """The 8-bit form of x (float32 or bfloat16)."""
    both = _calls.pack(x)
    return Act8._of(both, x.shape[-1], x.shape)


def act8_unpack(kept: Act8, dtype=torch.bfloat16):
    """A tensor of what an 8-bit form stands for (bfloat16 holds it exactly)."""
    _type(dtype, "dtype")
    out = torch.empty(kept.shape, dtype=dtype, device=kept.device)
    _calls.unpack(kept, out)
    return out


def layer_norm(x, weight, bias=None, eps: float = 1e-5, checkpoint: bool = False):
    """Layer norm over the last dimension.  Returns (y, mean, rstd, kept): y like x, the
    statistics fp32 with x's leading dimensions, and with ``checkpoint`` the 8-bit form of
    xhat = (x - mean) rstd (else None), from which ``layer_norm_backward`` and the next
    layer's ``linear_weight_grad`` work."""
    y, mean, rstd, both = _calls.layer_norm(x, weight, bias, eps, checkpoint)
    return y, mean, rstd, Act8._of(both, x.shape[-1], x.shape) if checkpoint else None


def layer_norm_backward(dy, saved, rstd, weight, mean=None, grad_dtype=torch.float32):
    """(dx, dweight, dbias) of ``layer_norm``.  ``saved`` is the 8-bit form of xhat that the
    forward pass left, or its input x (then ``mean`` is needed too)."""
    grad = _type(grad_dtype, "grad_dtype")
    if isinstance(saved, Act8):
        return _calls.layer_norm_backward(dy, saved, None, None, rstd, weight, grad)
    if mean is None:
        raise ValueError("mean is needed beside x")
    return _calls.layer_norm_backward(dy, None, saved, mean, rstd, weight, grad)


def rms_norm(x, weight, residual=None, eps: float = 1e-6, checkpoint: bool = False):
    """Root-mean-square norm over the last dimension, of h = x + residual (``residual`` None:
    of x).  Returns (y, h, rstd, kept): y = h rstd weight and h like x (h is x itself without
    a residual), rstd fp32 with x's leading dimensions, and with ``checkpoint`` the 8-bit form
    of xhat = h rstd (else None), from which ``rms_norm_backward`` and the next layer's
    ``linear_weight_grad`` (affine = (weight, None)) work."""
    y, h, rstd, both = _calls.rms_norm(x, weight, residual, eps, checkpoint)
    return y, h, rstd, Act8._of(both, x.shape[-1], x.shape) if checkpoint else None


def rms_norm_backward(dy, saved, rstd, weight, dh=None, grad_dtype=torch.float32):
    """(dx, dweight) of ``rms_norm``: dx is the gradient of x and of the residual alike.
    ``saved`` is the 8-bit form of xhat that the forward pass left, or its h; ``dh`` the
    gradient that reaches h from elsewhere (the stream's), added to dx."""
    grad = _type(grad_dtype, "grad_dtype")
    if isinstance(saved, Act8):
        return _calls.rms_norm_backward(dy, saved, None, rstd, weight, dh, grad)
    return _calls.rms_norm_backward(dy, None, saved, rstd, weight, dh, grad)


def embedding(ids, table, scale: float = 1.0, dtype=None):
    """out[...] = scale table[ids[...]], of ``dtype`` (None: the table's); ids int64 or int32 of any
    shape.  An id outside [0, rows of the table) stands for no token and gives zeros."""
    return _calls.embedding(ids, table, scale, _type(table.dtype if dtype is None else dtype, "dtype"))


def embedding_grad(dout, ids, vocab: int, scale: float = 1.0, dtype=torch.float32, out=None):
    """The gradient of ``embedding``'s table (vocab x the last dimension of dout) of ``dtype``:
    scale times the sum of dout over the tokens of each id.  With ``out``, that sum is added to
    it, in place, and rows that no token names are not touched."""
    return _calls.embedding_grad(dout, ids, vocab, scale, _type(dtype, "dtype"), out)


def _flat(coefficients):
    flat = []
    for triple in coefficients:
        a, b, c = triple
        flat += (a, b, c)
    return flat


def orthogonalize(matrices, coefficients=NEWTON_SCHULZ, eps: float = 1e-7, fine: bool = False):
    """Matrices brought close to orthogonal (their singular values close to 1) by Newton-Schulz
    products, as new bfloat16 tensors: X = G / max(|G|, eps), then X <- a X + (b A + c A^2) X
    with A = X X^T for each (a, b, c) of ``coefficients``.  ``matrices`` is a tensor or a list of
    tensors of one dtype (float32 or bfloat16), which are worked on together; one of more than two
    dimensions is a batch of matrices.  Matrices that are not small (include/novak.h) go through products of
    fp16 operands, 1e-4 to 1e-3 off for dense matrices and up to 1e-2 where a few elements carry all; with
    ``fine`` operands are of two parts, as the small ones' always are, which makes that 3e-6 to 3e-5, and takes
    two to three times as long."""
    if isinstance(matrices, torch.Tensor):
        return _calls.orthogonalize((matrices,), _flat(coefficients), eps, fine)[0]
    return _calls.orthogonalize(matrices, _flat(coefficients), eps, fine)


def orthogonal_step(params, grads, momenta, steps, momentum: float = 0.95, nesterov: bool = True, decay: float = 1.0,
                    coefficients=NEWTON_SCHULZ, eps: float = 1e-7, fine: bool = False):
    """In place, for each matrix: m <- momentum m + g, G = g + momentum m (``nesterov``) or m,
    theta <- decay theta - step X, X the orthogonalised G (``fine``: see ``orthogonalize``).  ``params`` and ``momenta`` are
    contiguous float32 tensors, none of them twice, ``grads`` of one dtype, ``steps`` one number each.
    To autograd they have changed: it refuses to go back through what was computed from them before."""
    _calls.orthogonal_step(params, grads, momenta, momentum, nesterov, steps, decay, _flat(coefficients), eps, fine)


def _kind(kind) -> int:
    try:
        return _KIND[kind]
    except KeyError:
        raise ValueError(f"kind must be one of {sorted(_KIND)}, got {kind!r}") from None


def activation(u, kind: str = "gelu", save_input: bool = True, save_output: bool = False):
    """(a, kept_u, kept_a): a = f(u) with f one of "gelu", "gelu_tanh", "silu"; the 8-bit
    form of u for ``activation_backward`` and that of a for the next layer's
    ``linear_weight_grad`` (None where not asked for)."""
    a, of_u, of_a = _calls.activation(u, _kind(kind), save_input, save_output)
    return (a, None if of_u is None else Act8._of(of_u, u.shape[-1], u.shape),
            None if of_a is None else Act8._of(of_a, u.shape[-1], u.shape))


def activation_backward(da, saved, kind: str = "gelu"):
    """du = da f'(u); ``saved`` is the 8-bit form of u, or u itself."""
    if isinstance(saved, Act8):
        return _calls.activation_backward(da, saved, None, _kind(kind))
    return _calls.activation_backward(da, None, saved, _kind(kind))


def linear_weight_grad(dy, kept: Act8, affine=None, bias: bool = True, dtype=torch.float32):
    """(dW, db) of a linear layer y = h W^T + b from the gradient of its output (rows x
    n_out) and the 8-bit form of its input (rows x n_in): dW (n_out x n_in) = dy^T h,
    db = the sum of dy's rows (None without ``bias``), both of ``dtype``.  With ``affine``
    = (weight, bias) of a layer norm, ``kept`` is that norm's xhat and
    h = xhat weight + bias, the layer norm's output; its bias may be None."""
    weight, beta = (None, None) if affine is None else affine
    if weight is not None and beta is None:
        beta = torch.zeros_like(weight)
    return _calls.linear_weight_grad(dy, kept, weight, beta, bias, _type(dtype, "dtype"))


def wait_failures() -> int:
    """How many bounded waits inside the kernels of the weight gradient and of the orthogonalised
    updates ran out on the current device since the library was loaded (0, or something is
    broken; see include/novak.h).
    Synchronises torch's current stream."""
    lib, count = B.load_library(), B.c_uint32()
    status = lib.novak_ops_gave_up(B.byref(count), torch.cuda.current_stream().cuda_stream)
    if status:
        raise B.NovakError(status, "novak_ops_gave_up", lib.novak_ops_error().decode())
    return count.value
