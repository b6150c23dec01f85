"""The operators around the sparsify step on a language model: a model's
gradients as one clipped flat vector, and the token table's lookup and loss
with their gradients.

Calls are enqueued on the handle's stream (by default the current one when the
handle was made) and return after the launches, without waiting.  Inputs must
be ready on that stream.  Outputs that a call allocates belong to that stream.
Where another stream is current during a call, its tensors are kept from reuse
until the handle's stream is done with them; where the handle's own is current,
as with torch's operators, a tensor that another stream allocated needs the
caller's record_stream.  Calls share their handle's scratch, those that a graph has
captured too: they must not run at once, and the handle must live until the graph's
last replay.
"""
import ctypes
import math
import operator

from . import _lib


def _value_types():
    import torch
    return {torch.float32: _lib.MICRO_TYPE_F32, torch.float16: _lib.MICRO_TYPE_F16,
            torch.bfloat16: _lib.MICRO_TYPE_BF16}


class _Enqueued:
    """A library handle bound to a torch device and stream."""

    def _bind(self, device, stream):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError(f"{type(self).__name__} needs a HIP device")
        dev = torch.device(device) if device is not None else torch.device("cuda")
        if dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        self._torch = torch
        self._tensor = torch.Tensor
        self._forward_ad = torch.autograd.forward_ad
        self.device = dev
        self.stream = stream if stream is not None else torch.cuda.current_stream(dev)
        self._raw_stream = self.stream.cuda_stream
        self._handle = None
        self._index = dev.index

    def _open(self):
        if self._handle is None:
            raise RuntimeError(f"{type(self).__name__} is closed")
        return self._handle

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _foreign(self):
        return self._torch.cuda.current_stream(self._index).cuda_stream != self._raw_stream

    def _empty(self, shape, dtype, foreign):
        torch = self._torch
        if foreign:
            with torch.cuda.stream(self.stream):
                return torch.empty(shape, dtype=dtype, device=self.device)
        return torch.empty(shape, dtype=dtype, device=self.device)

    def _used(self, *tensors):
        """Keeps the memory of tensors made on another stream until the
        enqueued work is done."""
        for t in tensors:
            if t is not None:
                t.record_stream(self.stream)

    def _outside_autograd(self, t, name):
        if t.requires_grad and self._torch.is_grad_enabled():
            raise RuntimeError(f"{name} requires its gradient, which this call does not record: call under "
                               "torch.no_grad() or pass its detach()")
        if self._forward_ad._current_level >= 0 and self._forward_ad.unpack_dual(t).tangent is not None:
            raise RuntimeError(f"{name} has a tangent, which this call does not carry on")

    def _scalar(self, t, name, dtype):
        if not isinstance(t, self._torch.Tensor) or t.dtype != dtype or t.device != self.device or t.numel() != 1:
            raise TypeError(f"{name} must be one {dtype} on {self.device}")
        return t.data_ptr()


class GradientSet(_Enqueued):
    """A model's gradient tensors, in the order of the flat vector that the
    sparsify step reads.

    Contiguous float32, float16 or bfloat16 tensors on one device; no two may
    share memory.  The set holds them, and uses the memory they had when it was
    made, which it keeps allocated.  So it must be made anew when a gradient is
    another tensor or has other memory, as every step's is after torch's
    zero_grad() (set_to_none=True, its default): an old set reads the old values
    without an error.  Making one allocates, uploads and waits for its stream;
    gradients that are zeroed or written in place keep theirs."""

    def __init__(self, tensors, device=None, stream=None):
        tensors = list(tensors)
        if device is None and tensors:
            device = getattr(tensors[0], "device", None)
        self._bind(device, stream)
        types = _value_types()
        for i, t in enumerate(tensors):
            if not isinstance(t, self._torch.Tensor) or t.dtype not in types or t.device != self.device \
                    or not t.is_contiguous():
                raise TypeError(f"tensor {i} must be a contiguous float32, float16 or bfloat16 tensor on "
                                f"{self.device}")
        self.tensors = tensors
        self._memory = [t.detach() for t in tensors]  # whatever becomes of the tensors' data
        self.n_total = sum(t.numel() for t in tensors)
        with self._torch.cuda.device(self.device):
            self._handle = _lib.micro_grads_init([t.data_ptr() for t in tensors], [t.numel() for t in tensors],
                                                 [types[t.dtype] for t in tensors], self._raw_stream)
        lib = _lib.load()
        self._norm_fn, self._clip_fn, self._flatten_fn = (lib.micro_grads_norm, lib.micro_grads_clip,
                                                          lib.micro_grads_flatten)

    def close(self):
        if getattr(self, "_handle", None) is not None:
            _lib.micro_grads_free(self._handle)
            self._handle = None
            self._memory = []

    def sumsq(self):
        """The sum of the squares of all values (a float64 device scalar):
        what workers that hold parts of one model add up before clipping."""
        handle = self._open()
        foreign = self._foreign()
        out = self._empty((), self._torch.float64, foreign)
        _lib.check(self._norm_fn(handle, out.data_ptr(), None))
        if foreign:
            self._used(*self._memory)
        return out

    def norm(self):
        """The global L2 norm (a float32 device scalar)."""
        handle = self._open()
        foreign = self._foreign()
        out = self._empty((), self._torch.float32, foreign)
        _lib.check(self._norm_fn(handle, None, out.data_ptr()))
        if foreign:
            self._used(*self._memory)
        return out

    def clip_(self, max_norm, sumsq=None):
        """Scales every gradient in place by min(1, max_norm / (norm + 1e-6)).
        Returns the norm before clipping (a float32 device scalar).  sumsq: the
        squared norm to clip by, where other workers hold parts of the model."""
        handle = self._open()
        foreign = self._foreign()
        other = None if sumsq is None else self._scalar(sumsq, "sumsq", self._torch.float64)
        norm = self._empty((), self._torch.float32, foreign)
        _lib.check(self._clip_fn(handle, float(max_norm), other, norm.data_ptr()))
        if foreign:
            self._used(sumsq, *self._memory)
        return norm

    def flatten(self, flat, max_norm=None, sumsq=None):
        """Writes the gradients, clipped to max_norm, into `flat` (contiguous
        float32, n_total values).  Returns the norm before clipping (a float32
        device scalar); without max_norm the values are only converted, and None
        is returned."""
        handle = self._open()
        foreign = self._foreign()
        if not isinstance(flat, self._torch.Tensor) or flat.dtype != self._torch.float32 \
                or flat.device != self.device or not flat.is_contiguous():
            raise TypeError(f"flat must be a contiguous float32 tensor on {self.device}")
        if flat.numel() != self.n_total:
            raise ValueError(f"flat must hold {self.n_total} values")
        if max_norm is None:
            if sumsq is not None:
                raise ValueError("sumsq without max_norm")
            _lib.check(self._flatten_fn(handle, math.inf, None, flat.data_ptr(), None))
            if foreign:
                self._used(flat, *self._memory)
            return None
        other = None if sumsq is None else self._scalar(sumsq, "sumsq", self._torch.float64)
        norm = self._empty((), self._torch.float32, foreign)
        _lib.check(self._flatten_fn(handle, float(max_norm), other, flat.data_ptr(), norm.data_ptr()))
        if foreign:
            self._used(flat, sumsq, *self._memory)
        return norm


class TokenTable(_Enqueued):
    """A table of `vocab` token rows of `dim` values: the lookup of rows, the
    softmax cross entropy over the table, and the gradients of both.

    The handle holds sizes and scratch, not the table: `weight` is an argument
    of every call.  Calls take up to max_tokens tokens.  Rows may be strided
    (the last dimension adjacent); ids and targets are int32 or int64, of any
    contiguous shape.  Calls are outside autograd: a tensor that requires its
    gradient is refused unless under torch.no_grad(), one with a tangent always.
    padding_id: an id whose row gets no gradient from lookups; ignore_id: the
    target of a token that does not count; score_bytes: scratch for one token
    block's scores at most."""

    def __init__(self, vocab, dim, max_tokens, dtype=None, padding_id=None, ignore_id=-100, score_bytes=None,
                 device=None, stream=None):
        self._bind(device, stream)
        torch = self._torch
        self.dtype = dtype if dtype is not None else torch.float32
        types = _value_types()
        if self.dtype not in types:
            raise TypeError("dtype must be float32, float16 or bfloat16")
        cfg = _lib.default_table_config()
        if padding_id is not None:
            cfg.padding_id = int(padding_id)
        cfg.ignored = int(ignore_id)
        if score_bytes is not None:
            cfg.score_bytes = int(score_bytes)
        self.config = cfg
        self.vocab, self.dim, self.max_tokens = int(vocab), int(dim), int(max_tokens)
        with torch.cuda.device(self.device):
            self._handle = _lib.micro_table_init(self.vocab, self.dim, self.max_tokens, types[self.dtype],
                                                 self._raw_stream, cfg)
        lib = _lib.load()
        self._lookup_fn, self._lookup_grad_fn = lib.micro_table_lookup, lib.micro_table_lookup_grad
        self._loss_fn, self._loss_grad_fn = lib.micro_table_loss, lib.micro_table_loss_grad
        self._sample_fn = lib.micro_table_sample
        self._value_types = types
        # the native marshalling of the plain case of lookup and sample
        self._caller = _lib.load_caller("TableCaller")(
            *(ctypes.cast(fn, ctypes.c_void_p).value for fn in (self._lookup_fn, self._sample_fn)), self._handle.value, self.vocab, self.dim,
            types[self.dtype], self._index, self.stream.stream_id)
        self._ids_types = {torch.int32: _lib.MICRO_IDS_I32, torch.int64: _lib.MICRO_IDS_I64}

    def close(self):
        if getattr(self, "_handle", None) is not None:
            self._caller = None
            _lib.micro_table_free(self._handle)
            self._handle = None

    def _ids(self, t, name):
        if not isinstance(t, self._tensor) or t.dtype not in self._ids_types or not t.is_cuda \
                or t.get_device() != self._index or not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous int32 or int64 tensor on {self.device}")
        return t.data_ptr(), self._ids_types[t.dtype], t.numel()

    def _rows(self, t, name, rows):
        """(address, row stride) of `rows` rows of dim values."""
        if not isinstance(t, self._tensor) or t.dtype is not self.dtype or not t.is_cuda or t.get_device() != self._index:
            raise TypeError(f"{name} must be a {self.dtype} tensor on {self.device}")
        self._outside_autograd(t, name)
        if t.dim() < 1 or t.shape[-1] != self.dim or t.numel() != rows * self.dim:
            raise ValueError(f"{name} must hold {rows} rows of {self.dim} values")
        if t.is_contiguous():
            return t.data_ptr(), self.dim
        if t.dim() != 2 or (self.dim > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) < self.dim):
            raise TypeError(f"{name} must be contiguous, or two-dimensional with adjacent values in a row")
        return t.data_ptr(), t.stride(0) if rows > 1 else self.dim

    def lookup(self, weight, ids, scale=1.0, out=None):
        """scale * weight[ids], of the shape of ids with dim behind it.  An id
        outside the table gives a row of NaN."""
        handle = self._open()
        if out is None:
            done = self._caller.lookup(weight, ids, scale)
            if isinstance(done, self._tensor):
                return done
            if done is not None:
                _lib.check(done)
        foreign = self._foreign()
        at, kind, tokens = self._ids(ids, "ids")
        w, w_stride = self._rows(weight, "weight", self.vocab)
        if out is None:
            out = self._empty((*ids.shape, self.dim), self.dtype, foreign)
        o, o_stride = self._rows(out, "out", tokens)
        st = self._lookup_fn(handle, w, w_stride, at, kind, tokens, float(scale), o, o_stride)
        if st:
            _lib.check(st)
        if foreign:
            self._used(weight, ids, out)
        return out

    def lookup_grad(self, grad, ids, dweight, scale=1.0, accumulate=False):
        """The lookup's gradient into `dweight`: scale times the sum of grad's
        rows over the tokens of each id, in a fixed order.  accumulate adds it
        to dweight (rows without a token stay as they are); otherwise every row
        is written.  Returns dweight."""
        handle = self._open()
        foreign = self._foreign()
        at, kind, tokens = self._ids(ids, "ids")
        g, g_stride = self._rows(grad, "grad", tokens)
        d, d_stride = self._rows(dweight, "dweight", self.vocab)
        st = self._lookup_grad_fn(handle, g, g_stride, at, kind, tokens, float(scale), 1 if accumulate else 0, d,
                                  d_stride)
        if st:
            _lib.check(st)
        if foreign:
            self._used(grad, ids, dweight)
        return dweight

    @staticmethod
    def _mean(reduction):
        if reduction not in ("mean", "sum"):
            raise ValueError("reduction must be 'mean' or 'sum'")
        return 1 if reduction == "mean" else 0

    def loss(self, hidden, weight, targets, reduction="mean"):
        """The softmax cross entropy of hidden's rows against the table's.
        Returns (loss, losses): the mean or sum over the counted tokens (a
        float32 device scalar) and every token's loss (float32, of the shape of
        targets; 0 where a token does not count)."""
        handle = self._open()
        foreign = self._foreign()
        mean = self._mean(reduction)
        at, kind, tokens = self._ids(targets, "targets")
        h, h_stride = self._rows(hidden, "hidden", tokens)
        w, w_stride = self._rows(weight, "weight", self.vocab)
        losses = self._empty(targets.shape, self._torch.float32, foreign)
        loss = self._empty((), self._torch.float32, foreign)
        st = self._loss_fn(handle, h, h_stride, w, w_stride, at, kind, tokens, mean, losses.data_ptr(),
                           loss.data_ptr())
        if st:
            _lib.check(st)
        if foreign:
            self._used(hidden, weight, targets)
        return loss, losses

    def loss_grad(self, hidden, weight, targets, scale=1.0, reduction="mean", dhidden=None, dweight=None,
                  accumulate=False):
        """The loss with its gradients times `scale`.  Returns (loss, losses,
        dhidden, dweight); given tensors are written, accumulate adds to the
        given dweight.  The losses are not scaled."""
        handle = self._open()
        foreign = self._foreign()
        mean = self._mean(reduction)
        at, kind, tokens = self._ids(targets, "targets")
        h, h_stride = self._rows(hidden, "hidden", tokens)
        w, w_stride = self._rows(weight, "weight", self.vocab)
        if accumulate and dweight is None:
            raise ValueError("accumulate needs the dweight to add to")
        if dhidden is None:
            dhidden = self._empty(hidden.shape, self.dtype, foreign)
        if dweight is None:
            dweight = self._empty((self.vocab, self.dim), self.dtype, foreign)
        dh, dh_stride = self._rows(dhidden, "dhidden", tokens)
        dw, dw_stride = self._rows(dweight, "dweight", self.vocab)
        losses = self._empty(targets.shape, self._torch.float32, foreign)
        loss = self._empty((), self._torch.float32, foreign)
        st = self._loss_grad_fn(handle, h, h_stride, w, w_stride, at, kind, tokens, mean, float(scale),
                                1 if accumulate else 0, losses.data_ptr(), loss.data_ptr(), dh, dh_stride, dw,
                                dw_stride)
        if st:
            _lib.check(st)
        if foreign:
            self._used(hidden, weight, targets, dhidden, dweight)
        return loss, losses, dhidden, dweight

    def _setting(self, sampling, name, value, dtype, rows):
        """Enters one of sample's settings: a number, or a tensor of one a row,
        which is returned."""
        if not isinstance(value, self._tensor):
            if dtype == self._torch.int32:
                value = operator.index(value)
                if not -2 ** 63 <= value < 2 ** 63:  # (ctypes takes one modulo 2^64)
                    raise OverflowError(f"{name} does not fit 64 bits")
            setattr(sampling, name, value)
            return None
        if value.dtype != dtype or not value.is_cuda or value.get_device() != self._index or not value.is_contiguous():
            raise TypeError(f"{name} must be a number or a contiguous {dtype} tensor on {self.device}")
        self._outside_autograd(value, name)
        if value.numel() != rows:
            raise ValueError(f"{name} must hold {rows} values")
        setattr(sampling, name + "s", value.data_ptr())
        return value

    def sample(self, logits, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, out=None):
        """Draws a token from each of the logits' rows by the given random numbers.
        Returns (ids, logprobs) of the shape of uniforms: int64 (or the given int32
        or int64 out) and float32, the logarithm of the drawn token's share of what
        is kept.

        logits: float32, float16 or bfloat16 rows of vocab values, strided or of any
        contiguous shape; uniforms: float32 in [0, 1).  top_k keeps the k largest
        (0: all), top_p of those the fewest that reach that share, min_p of those the
        ones with at least that share of the largest's; equal logits go by their
        index.  Each may be a tensor of one value a row (float32, top_k int32).
        temperature 0 takes the first largest logit.  Logits of -inf or NaN have no
        part; a row without any other gives -1 and NaN."""
        handle = self._open()
        if out is None:
            done = self._caller.sample(logits, uniforms, temperature, top_k, top_p, min_p)
            if isinstance(done, tuple):
                return done
            if done is not None:
                _lib.check(done)
        foreign = self._foreign()
        torch = self._torch
        if not isinstance(uniforms, self._tensor) or uniforms.dtype is not torch.float32 or not uniforms.is_cuda \
                or uniforms.get_device() != self._index or not uniforms.is_contiguous():
            raise TypeError(f"uniforms must be a contiguous float32 tensor on {self.device}")
        self._outside_autograd(uniforms, "uniforms")
        rows = uniforms.numel()
        if not isinstance(logits, self._tensor) or logits.dtype not in self._value_types or not logits.is_cuda \
                or logits.get_device() != self._index:
            raise TypeError(f"logits must be a float32, float16 or bfloat16 tensor on {self.device}")
        if logits.dim() < 1 or logits.shape[-1] != self.vocab or logits.numel() != rows * self.vocab:
            raise ValueError(f"logits must hold {rows} rows of {self.vocab} values")
        self._outside_autograd(logits, "logits")
        stride = self.vocab
        if not logits.is_contiguous():
            if logits.dim() != 2 or (self.vocab > 1 and logits.stride(1) != 1) or \
                    (rows > 1 and logits.stride(0) < self.vocab):
                raise TypeError("logits must be contiguous, or two-dimensional with adjacent values in a row")
            stride = logits.stride(0) if rows > 1 else self.vocab
        sampling = _lib.micro_sampling()
        arrays = [self._setting(sampling, "temperature", temperature, torch.float32, rows),
                  self._setting(sampling, "top_k", top_k, torch.int32, rows),
                  self._setting(sampling, "top_p", top_p, torch.float32, rows),
                  self._setting(sampling, "min_p", min_p, torch.float32, rows)]
        ids = self._empty(uniforms.shape, torch.int64, foreign) if out is None else out
        at, kind, count = self._ids(ids, "out")
        if count != rows:
            raise ValueError(f"out must hold {rows} ids")
        logprobs = self._empty(uniforms.shape, torch.float32, foreign)
        st = self._sample_fn(handle, logits.data_ptr(), self._value_types[logits.dtype], stride, rows, uniforms.data_ptr(),
                             ctypes.byref(sampling), at, kind, logprobs.data_ptr())
        if st:
            _lib.check(st)
        if foreign:
            self._used(logits, uniforms, *arrays, out)
        return ids, logprobs
