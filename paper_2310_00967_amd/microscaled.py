"""Microscaled 4-bit matrices (blocks of 32 values with a power of two as their
scale) and their products: layers and logits at a quarter of 16-bit types' bytes
and four times their matrix rate.

Streams, outputs and lifetimes are as in language.py.
"""
import ctypes

from . import _lib
from .language import _Enqueued, _value_types

GROUP, BLOCKS = 128, 4  # values and blocks of a group; a row is whole groups


class PackedMatrix:
    """A rows x cols matrix in blocks of 32 values along its rows.

    codes: uint8, (groups, rows, 64), two values a byte; scales: uint8, (groups, rows,
    4), the exponents of 2 plus 127; groups = cols / 128, rounded up.  Values behind
    cols are 0.  Both are contiguous and may be saved and loaded as they are.  A
    matrix keeps the tensors that it was made of: others make another matrix."""

    __slots__ = ("_parts",)  # (codes, scales, rows, cols), which every call goes by

    def __init__(self, codes, scales, rows, cols):
        rows, cols = int(rows), int(cols)
        if rows < 0 or cols < 0:
            raise ValueError("a side is negative")
        self._check(codes, scales, rows, cols)
        self._parts = (codes, scales, rows, cols)

    @staticmethod
    def _check(codes, scales, rows, cols):
        """(Again at every call: a tensor can be resized, or given other memory.)"""
        import torch
        groups = -(-cols // GROUP)
        for t, name, shape in ((codes, "codes", (groups, rows, GROUP // 2)),
                               (scales, "scales", (groups, rows, BLOCKS))):
            if not isinstance(t, torch.Tensor) or t.dtype != torch.uint8 or not t.is_contiguous():
                raise TypeError(f"{name} must be a contiguous uint8 tensor")
            if tuple(t.shape) != shape:
                raise ValueError(f"{name} of a {rows} x {cols} matrix must have the shape {shape}")
        if codes.device != scales.device:
            raise TypeError("codes and scales must be on one device")

    @classmethod
    def _made(cls, parts):
        """Of a call's own outputs."""
        m = cls.__new__(cls)
        m._parts = parts
        return m

    @property
    def codes(self):
        return self._parts[0]

    @property
    def scales(self):
        return self._parts[1]

    @property
    def rows(self):
        return self._parts[2]

    @property
    def cols(self):
        return self._parts[3]

    @property
    def _c(self):
        codes, scales, rows, cols = self._parts
        self._check(*self._parts)
        return _lib.micro_mx4_matrix(codes.data_ptr(), scales.data_ptr(), rows, cols)

    @property
    def device(self):
        return self._parts[0].device

    @property
    def shape(self):
        return self._parts[2:]

    def __repr__(self):
        return f"PackedMatrix({self.rows} x {self.cols}, {self.device})"


class Microscaled(_Enqueued):
    """Packing and products of 4-bit matrices on one device and stream.

    x and out are float32, float16 or bfloat16, two-dimensional or, where rows
    follow one another, of any shape with the columns last; two-dimensional ones may
    have strided rows (the last dimension adjacent).  Calls are outside autograd: a
    tensor that requires its gradient is refused unless under torch.no_grad(), one
    with a tangent always.  The backward pass of y = x w^T is two products:

        dx = product(pack(dy), pack(w, transposed=True))
        dw = product(pack(dy, transposed=True), pack(x, transposed=True))
    """

    def __init__(self, device=None, stream=None):
        self._bind(device, stream)
        with self._torch.cuda.device(self.device):
            self._handle = _lib.micro_mx4_init(self._raw_stream)
        lib = _lib.load()
        self._types = _value_types()
        self._pack_fn, self._unpack_fn = lib.micro_mx4_pack, lib.micro_mx4_unpack
        self._product_fn, self._linear_fn = lib.micro_mx4_product, lib.micro_mx4_linear
        # the native marshalling of the plain case of these
        self._caller = _lib.load_caller("MxCaller")(
            *(ctypes.cast(fn, ctypes.c_void_p).value for fn in (self._pack_fn, self._unpack_fn, self._product_fn, self._linear_fn)),
            self._handle.value, self._index, self.stream.stream_id)

    def close(self):
        if getattr(self, "_handle", None) is not None:
            self._caller = None
            _lib.micro_mx4_free(self._handle)
            self._handle = None

    def _values(self, t, name):
        """(address, row stride, rows, columns) of a tensor of values."""
        if not isinstance(t, self._tensor) or t.dtype not in self._types or not t.is_cuda or t.get_device() != self._index:
            raise TypeError(f"{name} must be a float32, float16 or bfloat16 tensor on {self.device}")
        self._outside_autograd(t, name)
        if t.dim() < 1:
            raise ValueError(f"{name} must have rows")
        cols = t.shape[-1]
        if t.is_contiguous():
            rows = t.numel() // cols if cols else t.shape[:-1].numel()
            return t.data_ptr(), cols, rows, cols
        if t.dim() != 2 or (cols > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < cols):
            raise TypeError(f"{name} must be contiguous, or two-dimensional with adjacent values in a row")
        return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else cols, t.shape[0], cols

    def _packed(self, m, name):
        if not isinstance(m, PackedMatrix) or m.codes.get_device() != self._index:
            raise TypeError(f"{name} must be a PackedMatrix on {self.device}")
        return m._c

    def _new(self, rows, cols, foreign):
        groups = -(-cols // GROUP)
        u8 = self._torch.uint8
        return PackedMatrix(self._empty((groups, rows, GROUP // 2), u8, foreign),
                            self._empty((groups, rows, BLOCKS), u8, foreign), rows, cols)

    def _kept(self, *what):
        for m in what:
            if isinstance(m, PackedMatrix):
                self._used(m.codes, m.scales)
            else:
                self._used(m)

    def _pack(self, x, straight, transposed):
        handle = self._open()
        done = self._caller.pack(x, straight, transposed)
        if isinstance(done, tuple):
            return (None if done[0] is None else PackedMatrix._made(done[0]),
                    None if done[1] is None else PackedMatrix._made(done[1]))
        if done is not None:
            _lib.check(done)
        foreign = self._foreign()
        at, stride, rows, cols = self._values(x, "x")
        q = self._new(rows, cols, foreign) if straight else None
        t = self._new(cols, rows, foreign) if transposed else None
        _lib.check(self._pack_fn(handle, at, self._types[x.dtype], stride, rows, cols, q._c if q else None,
                                 t._c if t else None))
        if foreign:
            self._kept(x)
        return q, t

    def pack(self, x, transposed=False):
        """x's rows in 4 bits; transposed: those of its transpose, in blocks along
        x's columns."""
        return self._pack(x, not transposed, bool(transposed))[1 if transposed else 0]

    def pack_both(self, x):
        """(pack(x), pack(x, transposed=True)) from one read of x."""
        return self._pack(x, True, True)

    def unpack(self, packed, dtype=None, out=None):
        """The values that a packed matrix stands for (dtype: float32)."""
        handle = self._open()
        if out is None and packed.__class__ is PackedMatrix:
            done = self._caller.unpack(packed._parts, self._types.get(dtype or self._torch.float32, -1))
            if isinstance(done, self._tensor):
                return done
            if done is not None:
                _lib.check(done)
        foreign = self._foreign()
        m = self._packed(packed, "packed")
        out, at, stride = self._out(out, dtype, self._torch.float32, (packed.rows, packed.cols), packed.rows, foreign)
        _lib.check(self._unpack_fn(handle, m, at, self._types[out.dtype], stride))
        if foreign:
            self._kept(packed, out)
        return out

    def _out(self, out, dtype, default, shape, rows, foreign):
        """(tensor, address, row stride) of a call's output."""
        if out is None:
            dtype = default if dtype is None else dtype
            if dtype not in self._types:
                raise TypeError("dtype must be float32, float16 or bfloat16")
            out = self._empty(shape, dtype, foreign)
            return out, out.data_ptr(), shape[-1]
        at, stride, have, cols = self._values(out, "out")
        if dtype is not None and dtype != out.dtype:
            raise TypeError("dtype is not that of out")
        if have != rows or cols != shape[-1]:
            raise ValueError(f"out must hold {rows} rows of {shape[-1]} values")
        return out, at, stride

    def product(self, a, b, dtype=None, out=None, accumulate=False):
        """a b^T of two packed matrices with rows of one length (dtype: float32);
        accumulate adds to the given out."""
        handle = self._open()
        if out is None and not accumulate and a.__class__ is b.__class__ is PackedMatrix:
            done = self._caller.product(a._parts, b._parts, self._types.get(dtype or self._torch.float32, -1))
            if isinstance(done, self._tensor):
                return done
            if done is not None:
                _lib.check(done)
        foreign = self._foreign()
        ca, cb = self._packed(a, "a"), self._packed(b, "b")
        if accumulate and out is None:
            raise ValueError("accumulate needs the out to add to")
        out, at, stride = self._out(out, dtype, self._torch.float32, (a.rows, b.rows), a.rows, foreign)
        _lib.check(self._product_fn(handle, ca, cb, 1 if accumulate else 0, at, self._types[out.dtype], stride))
        if foreign:
            self._kept(a, b, out)
        return out

    def linear(self, x, weight, dtype=None, out=None, accumulate=False):
        """x weight^T, x packed on the way (dtype: x's own)."""
        handle = self._open()
        if out is None and not accumulate and weight.__class__ is PackedMatrix:
            done = self._caller.linear(x, weight._parts, self._types.get(dtype or getattr(x, "dtype", None), -1))
            if isinstance(done, self._tensor):
                return done
            if done is not None:
                _lib.check(done)
        foreign = self._foreign()
        cw = self._packed(weight, "weight")
        at, stride, rows, cols = self._values(x, "x")
        if cols != weight.cols:
            raise ValueError(f"x must have rows of {weight.cols} values")
        if accumulate and out is None:
            raise ValueError("accumulate needs the out to add to")
        out, to, out_stride = self._out(out, dtype, x.dtype, (*x.shape[:-1], weight.rows), rows, foreign)
        q = self._new(rows, cols, foreign)
        _lib.check(self._linear_fn(handle, at, self._types[x.dtype], stride, q._c, cw,
                                   1 if accumulate else 0, to, self._types[out.dtype], out_stride))
        if foreign:
            self._kept(x, weight, out)
        return out
