"""The operators around a product with decoded weights, on torch tensors: torch supplies memory and the
stream, the library's kernels compute.  A handle keeps what does not change between calls (weights and
a call descriptor), never an input or an output, and is used by one thread at a time.  Every call
enqueues on the current stream of its tensors' device and returns without waiting.

For inference: results carry no graph, and a tensor that requires a gradient is taken by its values."""
from __future__ import annotations

import torch

from . import binding as B
from . import build as _build

_ELEMENT = {torch.bfloat16: B.ANS_BF16, torch.float32: B.ANS_F32, torch.float8_e4m3fn: B.ANS_E4M3}


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _on_device(t: torch.Tensor, device: torch.device, what: str) -> None:
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, the handle on {device}")


def _cuda_device(device) -> torch.device:
    d = torch.device(device)
    if d.type != "cuda":
        raise RuntimeError("the operators need a CUDA device: there is no CPU path")
    return torch.device("cuda", torch.cuda.current_device() if d.index is None else d.index)


# the current device and its current stream, as plain numbers
_current_device = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream


def _form_type():
    """The type that compares tensors' forms, out of the module built in-tree with the library."""
    again = "run paper_2406_06237_b200.build.build() (needs g++ and torch's headers); there is no fallback path"
    try:
        from . import _ans_form
    except ImportError as e:
        raise ImportError(f"{_build.FORM} is missing or does not load: {again}") from e
    if _ans_form.MADE_FOR != _build.form_interface():
        raise ImportError(f"{_build.FORM} was built for {_ans_form.MADE_FOR}, this is {_build.form_interface()}: {again}")
    return _ans_form.Form


class _Handle:
    """A device, and the status word its calls report to.

    A call checks its tensors' types, shapes, strides and devices; where all of them are those of the
    handle's last call (Form in csrc/torch) the checks' result is known and only the pointers change.

    Streams: making a handle waits for its stream, so that what the handle made of its own is complete for a call on
    any other.  What a handle holds is marked as used by each stream it is called on (record_stream), so that a handle may be
    dropped while its calls run.  A graph that holds calls needs the handle for as long as it is replayed."""

    def __init__(self, device):
        self._new_form = _form_type()
        self.device = _cuda_device(device)
        self._index = self.device.index
        self.status = torch.zeros(64, dtype=torch.int32, device=self.device)
        self._status = self.status.data_ptr()

    def _hold(self, *tensors) -> None:
        """The end of making a handle: the tensors that its calls use besides those they are given."""
        self._held = [t for t in (self.status, *tensors) if t is not None and t.device == self.device]
        self._streams = {_current_stream(self._index)}
        with torch.cuda.device(self.device):
            if not torch.cuda.is_current_stream_capturing():
                torch.cuda.current_stream().synchronize()

    def _enter(self) -> int:
        """The current stream; the library launches on the current device."""
        if _current_device() != self._index:
            raise RuntimeError(f"the handle is on {self.device}, which is not the current device")
        stream = _current_stream(self._index)
        if stream not in self._streams:
            for t in self._held:
                t.record_stream(torch.cuda.current_stream())
            self._streams.add(stream)
        return stream

    def read_status(self) -> int:
        """Waits for the stream; ANS_STATUS_* bits that calls have set since the last look (0: all sound)."""
        return B.ans_read_status(self._status, self._enter())


def _rows(t: torch.Tensor, what: str) -> int:
    """Row stride of a matrix whose rows are contiguous."""
    _need(t.dim() == 2, f"{what} must be a matrix")
    rows, width = t.shape
    stride, one = t.stride()
    _need(one == 1 or width <= 1, f"the rows of {what} must be contiguous")
    if stride < width:
        _need(rows <= 1, f"the rows of {what} overlap")
        return width
    return stride


class RmsNorm(_Handle):
    """y = h / sqrt(mean(h^2) + eps) * weight with h = x + residual, rows of `x` by themselves.

    weight: [width], bf16 or fp32, or None (ones; `device` must then be given).  out_dtype: bf16,
    fp32, or float8_e4m3fn: then y is returned as q with one fp32 scale a row, y ~ scale * q."""

    def __init__(self, weight: torch.Tensor | None, eps: float = 1e-6, out_dtype: torch.dtype = torch.bfloat16, device=None):
        super().__init__(weight.device if weight is not None else device or "cuda")
        _need(out_dtype in _ELEMENT, f"out_dtype {out_dtype} is not supported")
        if weight is not None:
            _need(weight.dim() == 1 and weight.is_contiguous(), "weight must be a contiguous vector")
            _need(weight.dtype in (torch.bfloat16, torch.float32), "weight must be bf16 or fp32")
        self.weight, self.eps, self.out_dtype = weight, float(eps), out_dtype
        self._8bit = out_dtype is torch.float8_e4m3fn
        self._form = self._new_form()
        self._desc = d = B.ans_norm_desc()
        d.d_weight = weight.data_ptr() if weight is not None and weight.numel() else None
        d.weight_dtype = _ELEMENT[weight.dtype] if weight is not None else B.ANS_F32
        d.eps, d.out_dtype = self.eps, _ELEMENT[out_dtype]
        self._hold(weight)

    def __call__(self, x: torch.Tensor, residual: torch.Tensor | None = None, out: torch.Tensor | None = None,
                 scales: torch.Tensor | None = None, summed: torch.Tensor | None = None):
        """x, residual: [rows, width] of one type, bf16 or fp32.  Returns (out, scales, summed): scales
        ([rows] fp32) only with an 8-bit output, summed (x + residual in x's type) only with a residual;
        None otherwise.  Buffers given for them are written and returned; summed may be x or residual."""
        st, d = self._enter(), self._desc
        if out is None or (scales is None and self._8bit) or (summed is None and residual is not None):
            out, scales, summed = self._buffers(x, residual, out, scales, summed)
        at = self._form.places(x, residual, out, scales, summed)
        if at is None:
            self._form.keep()
            self._check(x, residual, out, scales, summed)
            self._form.keep(x, residual, out, scales, summed)
            at = self._form.places(x, residual, out, scales, summed)
        d.d_x, d.d_residual, d.d_out, d.d_scales, d.d_sum = at
        B.ans_rms_norm(d, st)
        return out, scales, summed

    def _buffers(self, x, residual, out, scales, summed):
        _need(x.dim() == 2, "x must be a matrix")
        _on_device(x, self.device, "x")
        if out is None:
            out = torch.empty(x.shape, dtype=self.out_dtype, device=self.device)
        if scales is None and self._8bit:
            scales = torch.empty(x.shape[0], dtype=torch.float32, device=self.device)
        if summed is None and residual is not None:
            summed = torch.empty(x.shape, dtype=x.dtype, device=self.device)
        return out, scales, summed

    def _check(self, x, residual, out, scales, summed):
        """Checks one call's tensors and writes all but their places into the descriptor."""
        d, dt = self._desc, x.dtype
        xs = _rows(x, "x")
        rows, width = x.shape
        _need(dt in (torch.bfloat16, torch.float32), "x must be bf16 or fp32")
        _on_device(x, self.device, "x")
        _need(self.weight is None or self.weight.shape[0] == width, "weight and x differ in width")
        _need(out.dtype is self.out_dtype and out.shape == x.shape, "out has the wrong type or shape")
        _on_device(out, self.device, "out")
        if self._8bit:
            _need(scales.dtype is torch.float32 and scales.shape == (rows,) and scales.is_contiguous(), "scales must be fp32 [rows]")
            _on_device(scales, self.device, "scales")
        else:
            _need(scales is None, "scales belong to an 8-bit output")
        if residual is not None:
            _need(residual.dtype is dt and residual.shape == x.shape, "residual and x differ")
            _on_device(residual, self.device, "residual")
            _need(summed.dtype is dt and summed.shape == x.shape, "summed has the wrong type or shape")
            _on_device(summed, self.device, "summed")
            d.residual_stride, d.sum_stride = _rows(residual, "residual"), _rows(summed, "summed")
        else:
            _need(summed is None, "summed belongs to a residual")
        d.x_stride, d.x_dtype, d.rows, d.width = xs, _ELEMENT[dt], rows, width
        d.out_stride = _rows(out, "out")


def symbols_to_e4m3(symbols: torch.Tensor, zero_point: int) -> torch.Tensor:
    """Decoded symbols (uint8, any shape) as e4m3 values q - zero_point: the weights of a Linear in 8 bits,
    whose `scales` is then the layer's scale.  Raises if a difference in use is not exact in e4m3 (those
    of up to 4 bits always are)."""
    table = (torch.arange(256, dtype=torch.float32) - zero_point)
    exact = table.to(torch.float8_e4m3fn).float() == table
    used = torch.bincount(symbols.reshape(-1), minlength=256).cpu() > 0 if symbols.numel() else torch.zeros(256, dtype=torch.bool)
    _need(bool(exact[used].all()), "a symbol minus the zero-point is not exact in e4m3")
    return table.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).to(symbols.device)[symbols.long()].view(torch.float8_e4m3fn)


def _fits(t: torch.Tensor) -> bool:
    """Whether rows are contiguous and, if the first one does, start on 16 bytes."""
    (rows, width), (stride, one) = t.shape, t.stride()
    return (one == 1 or width <= 1) and (rows <= 1 or stride >= width and stride * t.element_size() % 16 == 0)


def _vector(t: torch.Tensor, n: int, device) -> torch.Tensor:
    """One value or n as n fp32 values."""
    return t.to(device=device, dtype=torch.float32).reshape(-1).expand(n).contiguous()


class Linear(_Handle):
    """Y = act(x_scales * scales * X W^T + bias) + residual with W [out features, in features].

    weight: bf16 (as decoded) or float8_e4m3fn (see symbols_to_e4m3).  scales: fp32, one for each
    output feature or one for all (a float or one element), or None.  bias: [out features] or None.
    activation: "none", "relu", "gelu", "gelu_tanh" or "silu".

    The weight is read where it lies, at each call, so that its buffer may be decoded into again.  Where it or its
    rows do not start on 16 bytes, each call lays it out in fresh memory first (a kernel that reads and writes
    the whole weight), unless it is settled.  Scales and bias on the weight's device are read anew in the same way: contiguous fp32
    vectors where they lie, others converted by each call.  What lies on another device, and a plain
    number, is taken once, here.

    settled: weight, scales and bias do not change any more.  The device is synchronised here, what has to be laid out or
    converted is so here once, and calls may read the weight before the work queued ahead of them is done
    (ANS_PRODUCT_WEIGHTS_SETTLED).  Leave it out where the weight's buffer is decoded into again.
    """

    def __init__(self, weight: torch.Tensor, scales=None, bias: torch.Tensor | None = None, activation: str = "none",
                 settled: bool = False):
        super().__init__(weight.device)
        _need(weight.dim() == 2, "weight must be a matrix")
        _need(weight.dtype in (torch.bfloat16, torch.float8_e4m3fn), "weight must be bf16 or float8_e4m3fn")
        _need(activation in B.ACTIVATIONS, f"activation {activation!r} is not one of {', '.join(B.ACTIVATIONS)}")
        n, k = weight.shape
        self.weight = weight
        if scales is not None:
            scales = torch.as_tensor(scales, dtype=None if isinstance(scales, torch.Tensor) else torch.float32)
            _need(scales.numel() in (1, n), "scales must be one or one for each output feature")
        if bias is not None:
            _need(bias.shape == (n,), "bias must have one value for each output feature")
        self.scales, self.bias, self.activation = scales, bias, activation
        self.in_features, self.out_features = k, n
        self._form, self._lies_off = self._new_form(), False
        self._desc = d = B.ans_product_desc()
        d.d_w, d.w_stride = weight.data_ptr() or None, max(weight.stride(0), k)
        self._anew, self._taken = [], []
        for field, t in (("d_w_scales", scales), ("d_bias", bias)):
            if t is None:
                continue
            if t.device == self.device and t.dtype is torch.float32 and t.is_contiguous() and t.numel() == n:
                setattr(d, field, t.data_ptr() or None)
            elif t.device == self.device and not settled:
                self._anew.append((field, t.detach()))
            else:
                self._taken.append(_vector(t.detach(), n, self.device))
                setattr(d, field, self._taken[-1].data_ptr() or None)
        d.n, d.k, d.dtype, d.activation = n, k, _ELEMENT[weight.dtype], B.ACTIVATIONS[activation]
        off = n > 0 and k > 0 and not (_fits(weight) and weight.data_ptr() % 16 == 0)
        strided = off and (k > 1 and weight.stride(1) != 1 or n > 1 and weight.stride(0) < k)
        if settled:
            if off:
                with torch.cuda.device(self.device):
                    self._taken.append(self._lay_out(_current_stream(self._index)))
            torch.cuda.synchronize(self.device)
            d.flags = B.ANS_PRODUCT_WEIGHTS_SETTLED
        elif off and not strided:
            d.flags = B.ANS_PRODUCT_WEIGHTS_ANYWHERE
        # what each call does: lay the weight out by a call of its own; have the product lay it out
        self._weight_strided, self._weight_off = strided and not settled, off and not strided and not settled
        self._hold(weight, scales, bias, *self._taken)

    def __call__(self, x: torch.Tensor, x_scales: torch.Tensor | None = None, residual: torch.Tensor | None = None,
                 out: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
        """x: [rows, in features] of the weight's type; x_scales: [rows] fp32.  Returns out (bf16 or fp32,
        [rows, out features]), the given buffer if there is one; residual is of its type and may be out
        itself.  An x whose rows do not start on 16 bytes is laid out in fresh memory first."""
        st, d = self._enter(), self._desc
        if out is None:
            _need(x.dim() == 2, "x must be [rows, in features]")
            out = torch.empty(x.shape[0], self.out_features, dtype=out_dtype, device=self.device)
        at = self._form.places(x, x_scales, residual, out)
        if at is None:
            self._form.keep()
            self._check(x, x_scales, residual, out)
            self._form.keep(x, x_scales, residual, out)
            at = self._form.places(x, x_scales, residual, out)
        d.d_x, d.d_x_scales, d.d_residual, d.d_y = at
        if self._anew:
            taken = [(field, _vector(t, d.n, self.device)) for field, t in self._anew]     # kept until the call is queued
            for field, t in taken:
                setattr(d, field, t.data_ptr())
        if self._weight_strided:
            laid = self._lay_out(st)                       # kept until the call is queued  # noqa: F841
        if self._weight_off or self._lies_off or at[0] % 16:
            room = torch.empty(B.ans_product_room_bytes(d), dtype=torch.uint8, device=self.device)
            d.d_room, d.room_bytes = room.data_ptr(), room.numel()
        B.ans_product(d, self._status, st)
        return out

    def _lay_out(self, stream: int) -> torch.Tensor:
        """The weight as it is when the stream gets there, in rows that start on 16 bytes; the descriptor names them."""
        d, w = self._desc, self.weight
        pad = 16 // w.element_size()
        d.w_stride = (d.k + pad - 1) // pad * pad
        laid = torch.empty(d.n * d.w_stride, dtype=w.dtype, device=self.device)
        d.d_w = laid.data_ptr()
        B.ans_product_rows(w.data_ptr(), *w.stride(), d.n, d.k, d.dtype, d.d_w, stream)
        return laid

    def _check(self, x, x_scales, residual, out):
        """Checks one call's tensors and writes all but their places into the descriptor."""
        d, dt = self._desc, out.dtype
        _need(x.dim() == 2 and x.shape[1] == self.in_features, "x must be [rows, in features]")
        _need(x.dtype is self.weight.dtype, f"x is {x.dtype}, the weight {self.weight.dtype}")
        _on_device(x, self.device, "x")
        shape = (x.shape[0], self.out_features)
        _need(out.shape == shape, "out has the wrong shape")
        _need(dt in (torch.bfloat16, torch.float32), "the output is bf16 or fp32")
        _on_device(out, self.device, "out")
        if x_scales is not None:
            _need(x_scales.dtype is torch.float32 and x_scales.shape == shape[:1] and x_scales.is_contiguous(), "x_scales must be fp32 [rows]")
            _on_device(x_scales, self.device, "x_scales")
        if residual is not None:
            _need(residual.dtype is dt and residual.shape == shape, "residual and out differ")
            _on_device(residual, self.device, "residual")
            d.residual_stride = _rows(residual, "residual")
        d.x_stride, d.m = _rows(x, "x"), shape[0]
        self._lies_off = not _fits(x)
        d.y_stride, d.y_dtype = _rows(out, "out"), _ELEMENT[dt]


class PagedCache(_Handle):
    """A paged cache of keys and values in 8 or 4 bits, quantised with a scale and a zero-point for every
    `group` values of a (token, head) as they are written (see ans_cache_desc in the header).

    Pages are the caller's to assign: token i of a sequence lies in slot
    table[i // page_size] * page_size + i % page_size.

    group: a multiple of 16 up to 256, head_dim unless given; a cache of other groups can be made, its calls are refused.  The
    cache saves room, not traffic: a step that reads it back moves the codes, writes 2 or 4 bytes a value and reads
    those again."""

    def __init__(self, n_pages: int, page_size: int, heads: int, head_dim: int, bitwidth: int = 8, group: int | None = None, device="cuda"):
        group = head_dim if group is None else group
        _need(bitwidth in (4, 8), "bitwidth must be 8 or 4")
        _need(min(n_pages, page_size, heads, head_dim, group) > 0, "sizes must be positive")
        _need(head_dim % group == 0 and head_dim % 2 == 0, "head_dim must be a multiple of group")
        device = _cuda_device(device)

        def make(last, dtype):
            return torch.zeros(n_pages, page_size, heads, last, dtype=dtype, device=device)

        codes, groups = head_dim * bitwidth // 8, head_dim // group
        self._take(make(codes, torch.uint8), make(groups, torch.float32), make(groups, torch.uint8),
                   make(codes, torch.uint8), make(groups, torch.float32), make(groups, torch.uint8), bitwidth)

    @classmethod
    def wrap(cls, k_codes, k_scales, k_zeros, v_codes, v_scales, v_zeros, bitwidth: int) -> "PagedCache":
        """A cache on existing arrays (shapes as in ans_cache_desc), which are used in place."""
        self = cls.__new__(cls)
        self._take(k_codes, k_scales, k_zeros, v_codes, v_scales, v_zeros, bitwidth)
        return self

    def _take(self, k_codes, k_scales, k_zeros, v_codes, v_scales, v_zeros, bitwidth):
        _Handle.__init__(self, k_codes.device)
        _need(bitwidth in (4, 8), "bitwidth must be 8 or 4")
        _need(k_codes.dim() == 4 and k_scales.dim() == 4, "codes, scales and zeros have four dimensions")
        dim = k_codes.shape[3] * 8 // bitwidth
        groups = k_scales.shape[3]
        _need(groups > 0 and dim % groups == 0, "codes and scales do not fit together")
        params = (*k_codes.shape[:3], groups)
        for t, dtype, shape, what in ((k_codes, torch.uint8, k_codes.shape, "k_codes"), (v_codes, torch.uint8, k_codes.shape, "v_codes"),
                                      (k_scales, torch.float32, params, "k_scales"), (v_scales, torch.float32, params, "v_scales"),
                                      (k_zeros, torch.uint8, params, "k_zeros"), (v_zeros, torch.uint8, params, "v_zeros")):
            _need(t.dtype is dtype and t.shape == shape and t.is_contiguous(), f"{what} must be a contiguous {dtype} tensor of {tuple(shape)}")
            _on_device(t, self.device, what)
        self.k_codes, self.k_scales, self.k_zeros = k_codes, k_scales, k_zeros
        self.v_codes, self.v_scales, self.v_zeros = v_codes, v_scales, v_zeros
        self.n_pages, self.page_size, self.heads = k_codes.shape[:3]
        self.head_dim, self.group, self.bitwidth = dim, dim // groups, bitwidth
        self._wrote, self._read = self._new_form(), self._new_form()
        self._desc = d = B.ans_cache_desc()
        d.d_k_codes, d.d_k_scales, d.d_k_zeros = k_codes.data_ptr(), k_scales.data_ptr(), k_zeros.data_ptr()
        d.d_v_codes, d.d_v_scales, d.d_v_zeros = v_codes.data_ptr(), v_scales.data_ptr(), v_zeros.data_ptr()
        d.n_pages, d.page_size, d.heads, d.head_dim = self.n_pages, self.page_size, self.heads, dim
        d.group, d.bitwidth = self.group, bitwidth
        self._hold(k_codes, k_scales, k_zeros, v_codes, v_scales, v_zeros)

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
        """k, v: [tokens, heads, head_dim], bf16 or fp32, tokens and heads at any stride; slots: [tokens]
        int64, a negative one skips its token."""
        st = self._enter()
        at = self._wrote.places(k, v, slots)
        if at is None:
            self._wrote.keep()
            self._check_write(k, v, slots)
            self._wrote.keep(k, v, slots)
            at = self._wrote.places(k, v, slots)
        dtype, tokens, ks, vs = self._write_args
        B.ans_cache_write(self._desc, at[0], at[1], dtype, tokens, ks, vs, at[2], self._status, st)

    def _check_write(self, k, v, slots):
        def strides(t, what):
            _need(t.dim() == 3 and t.shape[1:] == (self.heads, self.head_dim), f"{what} must be [tokens, heads, head_dim]")
            _need(t.stride(2) == 1, f"the values of a head of {what} must be contiguous")
            _on_device(t, self.device, what)
            return t.stride()[:2]

        ks, vs = strides(k, "k"), strides(v, "v")
        dt, tokens = k.dtype, k.shape[0]
        _need(dt in (torch.bfloat16, torch.float32), "k and v must be bf16 or fp32")
        _need(v.dtype is dt and v.shape[0] == tokens, "k and v differ")
        _need(slots.dtype is torch.int64 and slots.shape == (tokens,) and slots.is_contiguous(), "slots must be int64 [tokens]")
        _on_device(slots, self.device, "slots")
        self._write_args = (_ELEMENT[dt], tokens, ks, vs)

    def read(self, tables: torch.Tensor, starts: torch.Tensor, rows: int | None = None, k_out: torch.Tensor | None = None,
             v_out: torch.Tensor | None = None, out_dtype: torch.dtype = torch.bfloat16):
        """The keys and values of whole sequences, one after the other: [rows, heads, head_dim] each.
        tables: [sequences, pages] int32; starts: [sequences + 1] int32, sequence s is rows starts[s] to
        starts[s + 1].  rows = starts[-1] as a number (the call does not read it from the device), or
        k_out and v_out of that many rows are given.  Returns (k, v).

        A loop whose sequences grow gives the same buffers, long enough for all its steps, and no rows: the
        form of its calls is then the same each time, and their checks' result is known."""
        st = self._enter()
        if (k_out is None) != (v_out is None):
            raise ValueError("give both of k_out and v_out or none")
        if k_out is None:
            _need(rows is not None, "rows is needed where no buffers are given")
            k_out = torch.empty(rows, self.heads, self.head_dim, dtype=out_dtype, device=self.device)
            v_out = torch.empty_like(k_out)
        at = self._read.places(tables, starts, k_out, v_out)
        if at is None or rows != self._read_args[0]:
            self._read.keep()
            self._check_read(tables, starts, rows, k_out, v_out)
            self._read.keep(tables, starts, k_out, v_out)
            at = self._read.places(tables, starts, k_out, v_out)
        _, stride, pages, n, count, dtype = self._read_args
        B.ans_cache_read(self._desc, at[0], stride, pages, n, at[1], count, at[2], at[3], dtype, self._status, st)
        return k_out, v_out

    def _check_read(self, tables, starts, rows, k_out, v_out):
        given, rows = rows, k_out.shape[0] if rows is None else rows
        for t in (k_out, v_out):
            _need(t.dim() == 3 and t.shape[0] >= rows >= 0 and t.shape[1:] == (self.heads, self.head_dim) and t.is_contiguous(),
                  "k_out and v_out must be contiguous [rows, heads, head_dim]")
            _on_device(t, self.device, "an output")
        dt = k_out.dtype
        _need(v_out.dtype is dt, "k_out and v_out differ")
        _need(dt in (torch.bfloat16, torch.float32), "the outputs are bf16 or fp32")
        _need(tables.dtype is torch.int32 and tables.dim() == 2 and (tables.stride(1) == 1 or tables.shape[1] <= 1), "tables must be int32 [sequences, pages]")
        n, pages = tables.shape
        _need(n <= 1 or tables.stride(0) >= pages, "the rows of tables overlap")
        _need(starts.dtype is torch.int32 and starts.shape == (n + 1,) and starts.is_contiguous(), "starts must be int32 [sequences + 1]")
        _on_device(tables, self.device, "tables")
        _on_device(starts, self.device, "starts")
        self._read_args = given, tables.stride(0), pages, n, rows, _ELEMENT[dt]
