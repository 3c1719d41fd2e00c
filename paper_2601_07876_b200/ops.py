"""Training operators of the library (include/novak.h, "Training operators"):
8-bit forms of activations, layer norm, activation functions and the weight
gradient of a linear layer, on torch tensors.

Argument marshalling only: a tensor is seen as rows of its last dimension, its
address goes to the C entry point of the same name, and the work is enqueued on
torch's current stream of the tensors' device.  Results are new tensors of that
stream.  Nothing here records gradients: ``block`` has the autograd side.
"""
from __future__ import annotations

from functools import lru_cache

import torch

from . import binding as B

BLOCK = 32          # elements that share an exponent byte
_TYPE = {torch.float32: B.NOVAK_TYPE_F32, torch.bfloat16: B.NOVAK_TYPE_BF16}
_KIND = {"gelu": B.NOVAK_ACT_GELU, "gelu_tanh": B.NOVAK_ACT_GELU_TANH, "silu": B.NOVAK_ACT_SILU}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_lib = None


def _library():
    """The loaded library.  Loading is put off to the first call: it may build it."""
    global _lib
    if _lib is None:
        _lib = B.load_library()
    return _lib


def _enqueue(name: str, index: int, *args):
    """Calls the C entry point on torch's current stream of device `index`, with that device
    current (the raw lookups where torch has them: the objects cost 2 us per call)."""
    lib = _lib or _library()
    stream = _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream(index).cuda_stream
    if _current_device() == index:
        status = getattr(lib, name)(*args, stream)
    else:
        with torch.cuda.device(index):
            status = getattr(lib, name)(*args, stream)
    if status:
        raise B.NovakError(status, name, lib.novak_ops_error().decode())


def _type(t, name: str) -> int:
    try:
        return _TYPE[t.dtype]
    except KeyError:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}") from None


def _rows(t, name: str):
    """(rows, cols, elements between rows) of a tensor seen as rows of its last dimension;
    the leading dimensions have to fold into one."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    shape = t.shape
    if not shape or shape[-1] == 0:
        raise ValueError(f"{name} needs a last dimension of at least one element")
    cols = shape[-1]
    if t.is_contiguous():
        return (shape[0] if len(shape) == 2 else t.numel() // cols), cols, cols
    st = t.stride()
    if st[-1] != 1 and cols > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    rows, stride = 1, cols
    for size, step in zip(reversed(shape[:-1]), reversed(st[:-1])):
        if size == 1:
            continue
        if rows == 1:
            stride = step
        elif step != stride * rows:
            raise ValueError(f"{name}: the leading dimensions must fold into one stride")
        rows *= size
    if rows > 1 and stride < cols:
        raise ValueError(f"{name}: rows overlap")
    return rows, cols, stride


def _same(t, name: str, index: int, shape, dtype=None):
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{index}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def _vector(t, name: str, index: int, n: int):
    _same(t, name, index, (n,))
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return _type(t, name)


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
        index = codes.get_device()
        if not codes.is_contiguous() or not exps.is_contiguous() or index < 0 or exps.get_device() != index:
            raise ValueError("codes and exps must be contiguous CUDA tensors of one device")
        self.codes_ptr, self.exps_ptr = codes.data_ptr(), exps.data_ptr()
        if self.codes_ptr % 32 and rows:
            raise ValueError("codes must be 32-byte aligned")
        self._codes, self._exps, self._both, self.rows, self.cols, self.index = codes, exps, None, rows, cols, index
        self.shape = (rows, cols) if shape is None else tuple(shape)

    @classmethod
    def empty(cls, rows: int, cols: int, device, shape=None):
        """Uninitialised codes and exponents for rows x cols elements, in one buffer."""
        self = object.__new__(cls)
        blocks = (cols + BLOCK - 1) // BLOCK
        both = torch.empty(rows * blocks * (BLOCK + 1), dtype=torch.uint8, device=device)
        self._codes = self._exps = None
        self._both, self.rows, self.cols, self.index = both, rows, cols, both.get_device()
        self.codes_ptr = both.data_ptr()
        self.exps_ptr = self.codes_ptr + rows * blocks * BLOCK
        self.shape = (rows, cols) if shape is None else shape
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
    def device(self):
        return (self._codes if self._both is None else self._both).device

    @property
    def nbytes(self) -> int:
        return self.rows * ((self.cols + BLOCK - 1) // BLOCK) * (BLOCK + 1)

    def __repr__(self):
        return f"Act8(shape={tuple(self.shape)}, {self.nbytes} bytes on {self.device})"


def _belongs(kept: Act8, rows: int, cols: int, index: int, name: str):
    if kept.rows != rows or kept.cols != cols or kept.index != index:
        raise ValueError(f"the 8-bit form of {kept.rows} x {kept.cols} elements on cuda:{kept.index} does not belong "
                         f"to {name} of {rows} x {cols} on cuda:{index}")


def act8_pack(x) -> Act8:
    """The 8-bit form of x (float32 or bfloat16)."""
    rows, cols, stride = _rows(x, "x")
    kept = Act8.empty(rows, cols, x.device, x.shape)
    _enqueue("novak_act8_pack", kept.index, x.data_ptr(), stride, _type(x, "x"), kept.codes_ptr, kept.exps_ptr,
             rows, cols)
    return kept


def act8_unpack(kept: Act8, dtype=torch.bfloat16):
    """A tensor of what an 8-bit form stands for (bfloat16 holds it exactly)."""
    out = torch.empty(kept.shape, dtype=dtype, device=kept.device)
    _enqueue("novak_act8_unpack", kept.index, kept.codes_ptr, kept.exps_ptr, out.data_ptr(), kept.cols,
             _type(out, "dtype"), kept.rows, kept.cols)
    return out


def layer_norm(x, weight, bias=None, eps: float = 1e-5, checkpoint: bool = False):
    """Layer norm over the last dimension.  Returns (y, mean, rstd, kept): y like x, the
    statistics fp32 with x's leading dimensions, and with ``checkpoint`` the 8-bit form of
    xhat = (x - mean) rstd (else None), from which ``layer_norm_backward`` and the next
    layer's ``linear_weight_grad`` work."""
    rows, cols, stride = _rows(x, "x")
    index, shape, dev = x.get_device(), x.shape, x.device
    param = _vector(weight, "weight", index, cols)
    if bias is not None and _vector(bias, "bias", index, cols) != param:
        raise TypeError("weight and bias must have one dtype")
    y = torch.empty_like(x) if stride == cols else torch.empty(shape, dtype=x.dtype, device=dev)
    mean, rstd = torch.empty((2,) + shape[:-1], dtype=torch.float32, device=dev).unbind(0)
    kept = None
    codes = exps = None
    if checkpoint:
        kept = Act8.empty(rows, cols, dev, shape)
        codes, exps = kept.codes_ptr, kept.exps_ptr
    _enqueue("novak_layer_norm", index, x.data_ptr(), stride, y.data_ptr(), cols, _type(x, "x"), weight.data_ptr(),
             None if bias is None else bias.data_ptr(), param, eps, mean.data_ptr(), rstd.data_ptr(), codes, exps,
             rows, cols)
    return y, mean, rstd, kept


@lru_cache(maxsize=1024)
def _norm_backward_bytes(rows: int, cols: int) -> int:
    return _library().novak_layer_norm_backward_bytes(rows, cols)


def layer_norm_backward(dy, saved, rstd, weight, mean=None, grad_dtype=torch.float32):
    """(dx, dweight, dbias) of ``layer_norm``.  ``saved`` is the 8-bit form of xhat that the
    forward pass left, or its input x (then ``mean`` is needed too)."""
    rows, cols, stride = _rows(dy, "dy")
    index, shape, dev, type_ = dy.get_device(), dy.shape, dy.device, _type(dy, "dy")
    param = _vector(weight, "weight", index, cols)
    _same(rstd, "rstd", index, shape[:-1], torch.float32)
    rstd = rstd.contiguous()
    x_ptr = codes = exps = mean_ptr = None
    x_stride = 0
    if isinstance(saved, Act8):
        _belongs(saved, rows, cols, index, "dy")
        codes, exps = saved.codes_ptr, saved.exps_ptr
    else:
        _same(saved, "x", index, shape, dy.dtype)
        if mean is None:
            raise ValueError("mean is needed beside x")
        _same(mean, "mean", index, shape[:-1], torch.float32)
        mean = mean.contiguous()
        _, _, x_stride = _rows(saved, "x")
        x_ptr, mean_ptr = saved.data_ptr(), mean.data_ptr()
    dx = torch.empty_like(dy) if stride == cols else torch.empty(shape, dtype=dy.dtype, device=dev)
    dw, db = torch.empty((2, cols), dtype=grad_dtype, device=dev).unbind(0)
    need = _norm_backward_bytes(rows, cols)
    work = torch.empty(need, dtype=torch.uint8, device=dev)
    _enqueue("novak_layer_norm_backward", index, dy.data_ptr(), stride, x_ptr, x_stride, type_, mean_ptr,
             rstd.data_ptr(), codes, exps, weight.data_ptr(), param, dx.data_ptr(), cols, dw.data_ptr(), db.data_ptr(),
             _type(dw, "grad_dtype"), work.data_ptr(), need, rows, cols)
    return dx, dw, db


def _kind(kind) -> int:
    try:
        return _KIND[kind]
    except KeyError:
        raise ValueError(f"kind must be one of {sorted(_KIND)}, got {kind!r}") from None


def activation(u, kind: str = "gelu", save_input: bool = True, save_output: bool = False):
    """(a, kept_u, kept_a): a = f(u) with f one of "gelu", "gelu_tanh", "silu"; the 8-bit
    form of u for ``activation_backward`` and that of a for the next layer's
    ``linear_weight_grad`` (None where not asked for)."""
    k = _kind(kind)
    rows, cols, stride = _rows(u, "u")
    dev, shape = u.device, u.shape
    a = torch.empty_like(u) if stride == cols else torch.empty(shape, dtype=u.dtype, device=dev)
    kept_u = kept_a = None
    u_codes = u_exps = a_codes = a_exps = None
    if save_input:
        kept_u = Act8.empty(rows, cols, dev, shape)
        u_codes, u_exps = kept_u.codes_ptr, kept_u.exps_ptr
    if save_output:
        kept_a = Act8.empty(rows, cols, dev, shape)
        a_codes, a_exps = kept_a.codes_ptr, kept_a.exps_ptr
    _enqueue("novak_activation", u.get_device(), u.data_ptr(), stride, a.data_ptr(), cols, _type(u, "u"), k, u_codes,
             u_exps, a_codes, a_exps, rows, cols)
    return a, kept_u, kept_a


def activation_backward(da, saved, kind: str = "gelu"):
    """du = da f'(u); ``saved`` is the 8-bit form of u, or u itself."""
    k = _kind(kind)
    rows, cols, stride = _rows(da, "da")
    index = da.get_device()
    u_ptr = codes = exps = None
    u_stride = 0
    if isinstance(saved, Act8):
        _belongs(saved, rows, cols, index, "da")
        codes, exps = saved.codes_ptr, saved.exps_ptr
    else:
        _same(saved, "u", index, da.shape, da.dtype)
        _, _, u_stride = _rows(saved, "u")
        u_ptr = saved.data_ptr()
    du = torch.empty_like(da) if stride == cols else torch.empty(da.shape, dtype=da.dtype, device=da.device)
    _enqueue("novak_activation_backward", index, da.data_ptr(), stride, u_ptr, u_stride, _type(da, "da"), k, codes,
             exps, du.data_ptr(), cols, rows, cols)
    return du


@lru_cache(maxsize=1024)
def _weight_grad_bytes(aligned: bool, stride: int, type_: int, rows: int, n_out: int, n_in: int) -> int:
    # only the address's alignment matters
    return _library().novak_linear_weight_grad_bytes(256 if aligned else 2, stride, type_, rows, n_out, n_in)


def linear_weight_grad(dy, kept: Act8, affine=None, bias: bool = True, dtype=torch.float32):
    """(dW, db) of a linear layer y = h W^T + b from the gradient of its output (rows x
    n_out) and the 8-bit form of its input (rows x n_in): dW (n_out x n_in) = dy^T h,
    db = the sum of dy's rows (None without ``bias``), both of ``dtype``.  With ``affine``
    = (weight, bias) of a layer norm, ``kept`` is that norm's xhat and
    h = xhat weight + bias, the layer norm's output."""
    rows, n_out, stride = _rows(dy, "dy")
    index, dev, type_, n_in = dy.get_device(), dy.device, _type(dy, "dy"), kept.cols
    _belongs(kept, rows, n_in, index, "dy")
    w_ptr = b_ptr = None
    param = 0
    if affine is not None:
        weight, beta = affine
        param = _vector(weight, "weight", index, n_in)
        if _vector(beta, "bias", index, n_in) != param:
            raise TypeError("weight and bias must have one dtype")
        w_ptr, b_ptr = weight.data_ptr(), beta.data_ptr()
    dw = torch.empty((n_out, n_in), dtype=dtype, device=dev)
    db = torch.empty(n_out, dtype=dtype, device=dev) if bias else None
    ptr = dy.data_ptr()
    need = _weight_grad_bytes(ptr % 16 == 0, stride, type_, rows, n_out, n_in)
    work = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _enqueue("novak_linear_weight_grad", index, ptr, stride, type_, kept.codes_ptr, kept.exps_ptr, w_ptr, b_ptr, param,
             dw.data_ptr(), None if db is None else db.data_ptr(), _type(dw, "dtype"),
             None if work is None else work.data_ptr(), need, rows, n_out, n_in)
    return dw, db


def wait_failures() -> int:
    """How many bounded waits inside the weight gradient's kernel ran out on the current
    device since the library was loaded (0, or something is broken; see include/novak.h).
    Synchronises torch's current stream."""
    count = B.c_uint32()
    _enqueue("novak_ops_gave_up", torch.cuda.current_device(), B.byref(count))
    return count.value
