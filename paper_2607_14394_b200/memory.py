"""Recurrent memory around the layer: the root-mean-square norm, the 8-bit product, the gated linear recurrence, and
two blocks made of them.

The spectral layer of a 3D+time operator treats time as one more grid dimension; a rollout over many frames needs a
state that is carried from frame to frame instead.  `RmsNorm`, `GatedScan` and `Fp8Linear` are thin wrappers over the
C entry points (`dtst_rms_norm*`, `dtst_gated_scan*`, `dtst_matmul_fp8`): they check arguments, allocate outputs that
the caller did not bring, and pass device pointers on; their arithmetic runs in the CUDA library (`FieldMemory` adds two
pairs of fields with torch).  Every call runs on the current stream, or on the one given as `stream=`; an object may be used
on several streams and from several threads at once (a block, which keeps buffers or states, may not).

`FieldMemory` is a trainable block on channels-first fields [B, C, n..., T] whose last axis is time; `RolloutMemory`
is the serving form on latent vectors [B, T, D] with 8-bit projections, a whole history or one frame at a time.
"""
from __future__ import annotations

import ctypes
from typing import List, Optional, Sequence, Tuple

import torch

from . import binding as Bn

DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
GATES = {"sigmoid": 0, "decay": 1}
FP8 = torch.float8_e4m3fn
BLOCK = 128


def _device(device) -> int:
    d = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    if d.type != "cuda":
        raise ValueError("the memory operators live on a CUDA device")
    return torch.cuda.current_device() if d.index is None else d.index


def _addr(t: Optional[torch.Tensor], name: str, dev: int, dtype: torch.dtype, shape) -> int:
    """Device address of a contiguous tensor of this type and shape (0 for None)."""
    if t is None:
        return 0
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    _on_device(t, name, dev, dtype)
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise ValueError(f"{name} must be contiguous")


def _on_device(t: torch.Tensor, name: str, dev: int, dtype: torch.dtype) -> int:
    """Device address of a tensor of this type; its layout is the caller's business."""
    if t.get_device() != dev:
        raise ValueError(f"{name} must be a tensor on cuda:{dev}, got {t.device}")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _use(stream, dev):
    """A context in which `stream` (a torch stream or a cudaStream_t, 0 being the default stream) is current: the whole
    call, the allocation of its outputs included, runs on it."""
    if not isinstance(stream, torch.cuda.Stream):
        # (an ExternalStream of address 0 is a new stream of torch's own)
        stream = torch.cuda.ExternalStream(int(stream), device=dev) if int(stream) else torch.cuda.default_stream(dev)
    return torch.cuda.stream(stream)


# the current stream of a device as a cudaStream_t; the first form costs a tenth of the second
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device      # (likewise)


def _check(status: int, where: str) -> None:
    if status != Bn.DTST_OK:
        raise Bn.DtstError(status, where)


def _rows16(k: int) -> int:
    """Bytes between rows of k 8-bit values: rows start on 16-byte boundaries."""
    return -(-k // 16) * 16


def empty_fp8(rows: int, k: int, device=None) -> torch.Tensor:
    """An uninitialised [rows, k] 8-bit tensor whose rows start on 16-byte boundaries."""
    return torch.empty_strided((rows, k), (_rows16(k), 1), dtype=FP8, device=torch.device("cuda", _device(device)))


class RmsNorm:
    """y = s rstd weight, s = x + residual, rstd = (mean s^2 + eps)^-1/2 over dimension `dim` of `shape`.

    `dim` is the last dimension (token-major rows) or any other one (channels-first fields).
    """

    def __init__(self, shape: Sequence[int], dim: int = -1, dtype: torch.dtype = torch.float32, eps: float = 1e-6,
                 device=None):
        self.shape = torch.Size(int(n) for n in shape)
        nd = len(self.shape)
        if nd < 1 or not -nd <= dim < nd:
            raise ValueError(f"dim {dim} is no dimension of shape {tuple(self.shape)}")
        if dtype not in DTYPES:
            raise ValueError(f"dtype must be one of {list(DTYPES)}, got {dtype}")
        self.dim, self.dtype, self.eps, self.dev = dim % nd, dtype, float(eps), _device(device)
        self.device = torch.device("cuda", self.dev)
        self.channels = self.shape[self.dim]
        if self.channels < 1:
            raise ValueError("the normalised dimension is empty")
        self.outer = self.shape[:self.dim].numel()
        self.inner = self.shape[self.dim + 1:].numel()
        self._type = DTYPES[dtype]
        self._rest = self.shape[:self.dim] + self.shape[self.dim + 1:]
        self._wshape = torch.Size((self.channels,))
        self._q_like_x = self.channels % 16 == 0 and nd == 2
        self._scale_shape = torch.Size((-(-self.channels // BLOCK), self.outer))
        self._lib = Bn.lib()
        n = ctypes.c_size_t()
        _check(self._lib.dtst_rms_norm_scratch_bytes(self.channels, ctypes.byref(n)), "dtst_rms_norm_scratch_bytes")
        self._scratch_bytes = int(n.value)

    def forward(self, x, weight, residual=None, out=None, sum_out=None, rstd=None, need_backward=True, stream=None):
        """Returns (y, s, rstd); without a residual s is x itself (None where y takes x's place and leaves no s behind).

        In a 16-bit type with a residual, what rounding took from s stays with the rstd that is returned (its attribute
        `sum_low`), so that `backward` has the sum to 24 bits; an rstd that the caller brings may carry such a buffer too
        (a call without a sum to round sets it to None, the next one with a residual makes another).
        need_backward=False: neither is formed, and rstd is None.
        """
        d, t, sh = self.dev, self.dtype, self.shape
        if stream is not None or _current_device() != d:
            with torch.cuda.device(d), _use(torch.cuda.current_stream(d) if stream is None else stream, d):
                return self.forward(x, weight, residual, out, sum_out, rstd, need_backward)
        xp, wp = _addr(x, "x", d, t, sh), _addr(weight, "weight", d, torch.float32, self._wshape)
        rp = sp = 0
        if sum_out is not None:
            sp = _addr(sum_out, "sum_out", d, t, sh)
        if residual is not None:
            rp = _addr(residual, "residual", d, t, sh)
            if sum_out is None:
                sum_out = torch.empty_like(x)
                sp = sum_out.data_ptr()
        if out is None:
            out = torch.empty_like(x)
            yp = out.data_ptr()
        else:
            yp = _addr(out, "out", d, t, sh)
        qp = lp = 0
        if rstd is not None:
            qp = _addr(rstd, "rstd", d, torch.float32, self._rest)
            if self._type and hasattr(rstd, "sum_low"):
                if not sp:                              # s is x itself; what an earlier call's sum lost is not its
                    rstd.sum_low = None
                elif rstd.sum_low is None:
                    rstd.sum_low = torch.empty_like(x)
                lp = _addr(rstd.sum_low, "rstd.sum_low", d, t, sh)
        elif need_backward:
            rstd = weight.new_empty(self._rest)
            qp = rstd.data_ptr()
            if rp and self._type:
                rstd.sum_low = low = torch.empty_like(x)
                lp = low.data_ptr()
        status = self._lib.dtst_rms_norm(self._type, self.outer, self.channels, self.inner, self.eps, xp, rp, wp, sp, lp, yp,
                                         qp, _raw_stream(d))
        if status:
            _check(status, "dtst_rms_norm")
        if sum_out is None and (yp != xp or not xp):
            sum_out = x
        return out, sum_out, rstd

    def forward_fp8(self, x, weight, residual=None, q=None, scale=None, sum_out=None, stream=None):
        """Returns (q, scale, s): the norm of token-major rows in 8 bits, [rows, channels], and its scales
        [ceil(channels / 128), rows] - what Fp8Linear takes."""
        rows, c, d, t, sh = self.outer, self.channels, self.dev, self.dtype, self.shape
        if stream is not None or _current_device() != d:
            with torch.cuda.device(d), _use(torch.cuda.current_stream(d) if stream is None else stream, d):
                return self.forward_fp8(x, weight, residual, q, scale, sum_out)
        if self.inner != 1:
            raise ValueError("an 8-bit output needs the channels in the last dimension")
        xp, wp = _addr(x, "x", d, t, sh), _addr(weight, "weight", d, torch.float32, self._wshape)
        rp = sp = 0
        if sum_out is not None:
            sp = _addr(sum_out, "sum_out", d, t, sh)
        if residual is not None:
            rp = _addr(residual, "residual", d, t, sh)
            if sum_out is None:
                sum_out = torch.empty_like(x)
                sp = sum_out.data_ptr()
        if q is not None:
            ld, qp = _q_stride(q, rows, c), _on_device(q, "q", d, FP8)
        else:
            q = torch.empty_like(x, dtype=FP8) if self._q_like_x else \
                torch.empty_strided((rows, c), (_rows16(c), 1), dtype=FP8, device=self.device)
            ld, qp = _rows16(c), q.data_ptr()
        if scale is None:
            scale = weight.new_empty(self._scale_shape)
            scp = scale.data_ptr()
        else:
            scp = _addr(scale, "scale", d, torch.float32, self._scale_shape)
        status = self._lib.dtst_rms_norm_fp8(self._type, rows, c, self.eps, xp, rp, wp, sp, qp, ld, scp, _raw_stream(d))
        if status:
            _check(status, "dtst_rms_norm_fp8")
        return q, scale, (x if sum_out is None else sum_out)

    def backward(self, grad_y, s, weight, rstd, grad_s=None, grad_x=None, grad_weight=None, need_grad_weight=True,
                 stream=None, sum_low=None):
        """Returns (grad_x, grad_weight); grad_x is the gradient of x and of the residual.  s and rstd as `forward`
        returned them.

        In a 16-bit type the sum is s and the low part that rstd carries (`rstd.sum_low`).  The attribute does not survive a
        clone, a detach or a copy of rstd: pass it on as `sum_low=`, or the gradients are those of the rounded sum."""
        d, t, sh = self.dev, self.dtype, self.shape
        if stream is not None or _current_device() != d:
            with torch.cuda.device(d), _use(torch.cuda.current_stream(d) if stream is None else stream, d):
                return self.backward(grad_y, s, weight, rstd, grad_s, grad_x, grad_weight, need_grad_weight, None, sum_low)
        gp, wp = _addr(grad_y, "grad_y", d, t, sh), _addr(weight, "weight", d, torch.float32, self._wshape)
        if grad_x is None:
            grad_x = torch.empty_like(grad_y)
            xp = grad_x.data_ptr()
        else:
            xp = _addr(grad_x, "grad_x", d, t, sh)
        scratch = nbytes = gwp = 0
        if need_grad_weight:
            if grad_weight is None:
                grad_weight = torch.empty_like(weight)
                gwp = grad_weight.data_ptr()
            else:
                gwp = _addr(grad_weight, "grad_weight", d, torch.float32, self._wshape)
            # the call's own, from the current stream's allocations: calls on other streams may be under way
            partial, nbytes = torch.empty(self._scratch_bytes, dtype=torch.uint8, device=self.device), self._scratch_bytes
            scratch = partial.data_ptr()
        if sum_low is None and self._type:
            sum_low = getattr(rstd, "sum_low", None)
        status = self._lib.dtst_rms_norm_backward(
            self._type, self.outer, self.channels, self.inner, gp, _addr(s, "s", d, t, sh), _addr(sum_low, "sum_low", d, t, sh), wp,
            _addr(rstd, "rstd", d, torch.float32, self._rest), 0 if grad_s is None else _addr(grad_s, "grad_s", d, t, sh),
            xp, gwp, scratch, nbytes, _raw_stream(d))
        if status:
            _check(status, "dtst_rms_norm_backward")
        return grad_x, grad_weight


def _q_stride(q: torch.Tensor, rows: int, k: int) -> int:
    if q.shape != (rows, k):
        raise ValueError(f"8-bit tensor must have shape {(rows, k)}, got {tuple(q.shape)}")
    if k > 1 and q.stride(1) != 1:
        raise ValueError("the rows of an 8-bit tensor must be contiguous")
    return q.stride(0) if rows > 1 else _rows16(k)       # (of one row there is no distance: any that the library takes)


def quantize_fp8(x: torch.Tensor, q=None, scale=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows x [rows, k] (contiguous along k) -> (q [rows, k] in 8 bits, scale [ceil(k / 128), rows])."""
    if x.dim() != 2 or x.dtype not in DTYPES or not x.is_cuda or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError("quantize_fp8 takes CUDA rows [rows, k] of float32, bfloat16 or float16, contiguous along k")
    rows, k = x.shape
    dev, shape = x.get_device(), (-(-k // BLOCK), rows)
    if stream is not None or _current_device() != dev:
        with torch.cuda.device(dev), _use(torch.cuda.current_stream(dev) if stream is None else stream, dev):
            return quantize_fp8(x, q, scale)
    if q is None:
        q = empty_fp8(rows, k, x.device)
    if scale is None:
        scale = x.new_empty(shape, dtype=torch.float32)
    _check(Bn.lib().dtst_quantize_fp8(DTYPES[x.dtype], rows, k, x.data_ptr(), x.stride(0), _on_device(q, "q", dev, FP8),
                                      _q_stride(q, rows, k), _addr(scale, "scale", dev, torch.float32, shape),
                                      _raw_stream(dev)), "dtst_quantize_fp8")
    return q, scale


def quantize_fp8_weight(w: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """w [n, k] -> (8-bit values [n, k], scale [ceil(n / 128), ceil(k / 128)]), one scale per 128 x 128 block."""
    if w.dim() != 2 or w.dtype not in DTYPES or not w.is_cuda or (w.shape[1] > 1 and w.stride(1) != 1):
        raise ValueError("quantize_fp8_weight takes CUDA w [n, k] of float32, bfloat16 or float16, contiguous along k")
    n, k = w.shape
    dev = w.get_device()
    if stream is not None or _current_device() != dev:
        with torch.cuda.device(dev), _use(torch.cuda.current_stream(dev) if stream is None else stream, dev):
            return quantize_fp8_weight(w)
    q = empty_fp8(n, k, w.device)
    scale = w.new_empty((-(-n // BLOCK), -(-k // BLOCK)), dtype=torch.float32)
    _check(Bn.lib().dtst_quantize_fp8_weight(DTYPES[w.dtype], n, k, w.data_ptr(), w.stride(0) if n > 1 else k, q.data_ptr(),
                                             _q_stride(q, n, k), scale.data_ptr(), _raw_stream(dev)),
           "dtst_quantize_fp8_weight")
    return q, scale


class Fp8Linear:
    """out = x w^T for 8-bit x [m, k] (scale [ceil(k / 128), m]) and weights [n, k] (a scale per 128 x 128 block)."""

    def __init__(self, weight: torch.Tensor, weight_scale: torch.Tensor, out_dtype: torch.dtype = torch.bfloat16):
        if weight.dim() != 2 or weight.dtype != FP8:
            raise ValueError("weight must be an 8-bit tensor [n, k] (see from_weight)")
        if out_dtype not in DTYPES:
            raise ValueError(f"out_dtype must be one of {list(DTYPES)}, got {out_dtype}")
        self.dev = weight.get_device()
        if self.dev < 0:
            raise ValueError("weight must be a CUDA tensor")
        self.device = weight.device
        self.n, self.k = weight.shape
        self.weight, self.weight_scale, self.out_dtype = weight, weight_scale, out_dtype
        self._ld = _q_stride(weight, self.n, self.k)
        self._kb = -(-self.k // BLOCK)
        self._w = weight.data_ptr()
        self._ws = _addr(weight_scale, "weight_scale", self.dev, torch.float32, (-(-self.n // BLOCK), self._kb))
        # zeroed memory that calls on any stream may use from now on: a status word, which only a wait that gives up writes
        self.workspace = torch.zeros(256, dtype=torch.uint8, device=self.device)
        torch.cuda.current_stream(self.dev).synchronize()
        self._work = self.workspace.data_ptr()
        self._type = DTYPES[out_dtype]
        self._lib = Bn.lib()

    @classmethod
    def from_weight(cls, w: torch.Tensor, out_dtype: torch.dtype = torch.bfloat16) -> "Fp8Linear":
        """Quantises w [n, k] (float32, bfloat16 or float16) once."""
        return cls(*quantize_fp8_weight(w), out_dtype=out_dtype)

    def forward(self, x: torch.Tensor, x_scale: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None):
        d, k = self.dev, self.k
        if stream is not None or _current_device() != d:
            with torch.cuda.device(d), _use(torch.cuda.current_stream(d) if stream is None else stream, d):
                return self.forward(x, x_scale, out)
        m = x.shape[0]
        xp, ld = _on_device(x, "x", d, FP8), _q_stride(x, m, k)
        sp = _addr(x_scale, "x_scale", d, torch.float32, (self._kb, m))
        if out is None:
            out = x_scale.new_empty((m, self.n), dtype=self.out_dtype)
            op, out_ld = out.data_ptr(), self.n
        else:
            if out.shape != (m, self.n) or (self.n > 1 and out.stride(1) != 1):
                raise ValueError(f"out must have shape {(m, self.n)} and contiguous rows")
            op, out_ld = _on_device(out, "out", d, self.out_dtype), out.stride(0) if m > 1 else self.n
        status = self._lib.dtst_matmul_fp8(self._type, m, self.n, k, xp, ld, sp, self._w, self._ld, self._ws, op, out_ld,
                                           self._work, 256, _raw_stream(d))
        if status:
            _check(status, "dtst_matmul_fp8")
        return out

    __call__ = forward

    def status(self, stream=None) -> int:
        """DTST_OK, or DTST_ERR_DEVICE_TIMEOUT if a bounded wait gave up since the last query; synchronises."""
        with torch.cuda.device(self.dev):
            return int(self._lib.dtst_workspace_status(self._work, Bn._stream_ptr(stream)))


class GatedScan:
    """h_t = a_t h_{t-1} + u_t along dimension `dim` of `shape`, forward and backward.

    gate "sigmoid": a = sigmoid(g), u = (1 - a) v; "decay": a = g, u = v (with |a| > 1 the product of neighbouring gates has to
    stay in float32's range wherever the state is not zero).  The states (h0, h_last) are float32 of the
    shape without `dim`.  v and g may be strided in the dimensions in front of the last (both alike), e.g. the two
    halves of one projection's output; h and the upstream gradient are contiguous.
    """

    def __init__(self, shape: Sequence[int], dim: int = 1, dtype: torch.dtype = torch.float32, gate: str = "sigmoid",
                 device=None):
        self.shape = torch.Size(int(n) for n in shape)
        nd = len(self.shape)
        if nd < 1 or not -nd <= dim < nd:
            raise ValueError(f"dim {dim} is no dimension of shape {tuple(self.shape)}")
        if dtype not in DTYPES:
            raise ValueError(f"dtype must be one of {list(DTYPES)}, got {dtype}")
        if gate not in GATES:
            raise ValueError(f"gate must be one of {list(GATES)}, got {gate!r}")
        self.dim, self.dtype, self.gate, self.dev = dim % nd, dtype, gate, _device(device)
        self.device = torch.device("cuda", self.dev)
        self.length = self.shape[self.dim]
        self.outer_shape, inner_shape = self.shape[:self.dim], self.shape[self.dim + 1:]
        self.outer, self.inner = self.outer_shape.numel(), inner_shape.numel()
        if self.inner < 1:
            raise ValueError("the dimensions behind the recurrence's must not be empty")
        self.state_shape = self.outer_shape + inner_shape
        dense = (self.length * self.inner, self.inner)
        self._dense = dense                              # (outer, step) strides of contiguous tensors
        self._ref = self._describe(dense, dense)
        self._other = (None, None, None)                 # the last description of other strides: v and g's, the gradients'
        self._lib = Bn.lib()
        n = ctypes.c_int64()
        _check(self._lib.dtst_gated_scan_checkpoints(self._ref, ctypes.byref(n)), "dtst_gated_scan_checkpoints")
        self.checkpoint_floats = int(n.value)
        self._ck_shape = torch.Size((self.checkpoint_floats,))

    def new_checkpoints(self) -> torch.Tensor:
        """A buffer for the states that a forward pass saves for its backward pass."""
        return torch.empty(self.checkpoint_floats, dtype=torch.float32, device=self.device)

    def _strides(self, t: torch.Tensor, name: str) -> Tuple[int, int]:
        """(outer, step) strides of t, whose other dimensions must lie together."""
        if t.shape != self.shape:
            raise ValueError(f"{name} must have shape {tuple(self.shape)}, got {tuple(t.shape)}")
        if t.is_contiguous():
            return self._dense
        st, sh, k = t.stride(), self.shape, self.dim

        def joined(dims: range) -> Optional[int]:        # the stride of several dimensions taken as one
            at = None
            for i in reversed(dims):
                if sh[i] == 1:
                    continue
                if at is not None and st[i] != at[1]:
                    raise ValueError(f"{name}: the dimensions on each side of the recurrence's must lie together")
                at = (st[i] if at is None else at[0], st[i] * sh[i])
            return None if at is None else at[0]

        inner, outer = joined(range(k + 1, len(sh))), joined(range(0, k))
        if inner not in (None, 1):
            raise ValueError(f"{name}: the last dimension must be contiguous")
        step = st[k] if sh[k] != 1 else self.inner
        if self.inner == 1 and step != 1:
            raise ValueError(f"{name}: the recurrence's dimension must be contiguous when it is the last one")
        return (self._dense[0] if outer is None else outer), step

    def _describe(self, at, grad_at):
        return ctypes.byref(Bn.ScanDesc(DTYPES[self.dtype], GATES[self.gate], self.outer, self.length, self.inner, at, grad_at))

    def _description(self, at, grad_at):
        """The description for these strides.  One that a call may be reading is never changed."""
        if at is self._dense and grad_at is self._dense:
            return self._ref
        a, b, ref = self._other
        if a != at or b != grad_at:
            ref = self._describe(at, grad_at)
            self._other = (at, grad_at, ref)
        return ref

    def _inputs(self, v, g):
        """Addresses of v and g, and their strides."""
        d, t, sh = self.dev, self.dtype, self.shape
        if v.dtype is t and g.dtype is t and v.shape == sh and g.shape == sh and v.get_device() == d and \
                g.get_device() == d and v.is_contiguous() and g.is_contiguous():
            at = self._dense
        else:
            _on_device(v, "v", d, t)
            _on_device(g, "g", d, t)
            at, b = self._strides(v, "v"), self._strides(g, "g")
            if at != b:
                raise ValueError(f"v and g must have the same strides, got {v.stride()} and {g.stride()}")
        return v.data_ptr(), g.data_ptr(), at

    def forward(self, v, g, h0=None, lengths=None, out=None, h_last=None, checkpoints=None, stream=None):
        """Returns (h, h_last).  lengths: int32 per outer entry; checkpoints: see new_checkpoints."""
        d, state = self.dev, self.state_shape
        if stream is not None or _current_device() != d:
            with torch.cuda.device(d), _use(torch.cuda.current_stream(d) if stream is None else stream, d):
                return self.forward(v, g, h0, lengths, out, h_last, checkpoints)
        vp, gp, at = self._inputs(v, g)
        hp = 0 if h0 is None else _addr(h0, "h0", d, torch.float32, state)
        if out is None:
            out = torch.empty_like(v) if at is self._dense else v.new_empty(self.shape)
            op = out.data_ptr()
        else:
            op = _addr(out, "out", d, self.dtype, self.shape)
        if h_last is None:
            h_last = torch.empty(state, dtype=torch.float32, device=self.device) if h0 is None else torch.empty_like(h0)
            lp = h_last.data_ptr()
        else:
            lp = _addr(h_last, "h_last", d, torch.float32, state)
        status = self._lib.dtst_gated_scan(
            self._description(at, self._dense), vp, gp, hp,
            0 if lengths is None else _addr(lengths, "lengths", d, torch.int32, self.outer_shape), op, lp,
            0 if checkpoints is None else _addr(checkpoints, "checkpoints", d, torch.float32, self._ck_shape),
            _raw_stream(d))
        if status:
            _check(status, "dtst_gated_scan")
        return out, h_last

    def backward(self, grad_h, v, g, checkpoints, h0=None, lengths=None, grad_last=None, grad_v=None, grad_g=None,
                 grad_h0=None, need_grad_h0=True, stream=None):
        """Returns (grad_v, grad_g, grad_h0); v, g, h0, lengths and checkpoints as in the forward call."""
        d, t, state = self.dev, self.dtype, self.state_shape
        if stream is not None or _current_device() != d:
            with torch.cuda.device(d), _use(torch.cuda.current_stream(d) if stream is None else stream, d):
                return self.backward(grad_h, v, g, checkpoints, h0, lengths, grad_last, grad_v, grad_g, grad_h0,
                                     need_grad_h0)
        vp, gp, at = self._inputs(v, g)
        dp = _addr(grad_h, "grad_h", d, t, self.shape)
        if grad_v is None and grad_g is None:
            grad_v, grad_g, to = torch.empty_like(grad_h), torch.empty_like(grad_h), self._dense
        else:
            grad_v = torch.empty_like(grad_h) if grad_v is None else grad_v
            grad_g = torch.empty_like(grad_h) if grad_g is None else grad_g
            _on_device(grad_v, "grad_v", d, t)
            _on_device(grad_g, "grad_g", d, t)
            to, b = self._strides(grad_v, "grad_v"), self._strides(grad_g, "grad_g")
            if to != b:
                raise ValueError(f"grad_v and grad_g must have the same strides, got {grad_v.stride()} and {grad_g.stride()}")
        if grad_h0 is None and need_grad_h0:
            grad_h0 = (torch.empty(state, dtype=torch.float32, device=self.device) if grad_last is None and h0 is None
                       else torch.empty_like(grad_last if h0 is None else h0))
        status = self._lib.dtst_gated_scan_backward(
            self._description(at, to), dp, 0 if grad_last is None else _addr(grad_last, "grad_last", d, torch.float32, state), vp, gp,
            0 if h0 is None else _addr(h0, "h0", d, torch.float32, state),
            0 if lengths is None else _addr(lengths, "lengths", d, torch.int32, self.outer_shape),
            _addr(checkpoints, "checkpoints", d, torch.float32, self._ck_shape), grad_v.data_ptr(), grad_g.data_ptr(),
            _addr(grad_h0, "grad_h0", d, torch.float32, state), _raw_stream(d))
        if status:
            _check(status, "dtst_gated_scan_backward")
        return grad_v, grad_g, grad_h0

    def status(self, stream=None) -> int:
        """DTST_OK, or DTST_ERR_DEVICE_TIMEOUT if a bounded wait of any recurrence gave up on this device since the last
        query; synchronises."""
        with torch.cuda.device(self.dev):
            return int(self._lib.dtst_gated_scan_status(Bn._stream_ptr(stream)))


class FieldMemory:
    """A trainable memory along the time axis of fields x [B, C, n..., T] (float32, T last), pre-normalised and residual:

        y = norm(x);  v = W_v y + b_v;  g = W_g y + b_g;  h = scan(v, g);  out = x + W_o h

    forward(x) -> out and backward(grad_out) -> gradients of x and of every parameter; point-wise maps are
    dtst_pointwise_linear (C <= 32, points % 4 == 0).  Parameters are plain tensors owned by this object.
    """

    def __init__(self, B: int, C: int, grid: Sequence[int], device=None, seed: int = 0):
        shape = (B, C) + tuple(int(n) for n in grid)
        points = torch.Size(shape[2:]).numel()
        if not 1 <= C <= 32 or B < 1 or len(shape) < 3 or points < 4 or points % 4 != 0:
            raise ValueError("FieldMemory takes 1 to 32 channels and a grid whose points are a multiple of 4, got "
                             f"B = {B}, C = {C}, grid = {tuple(grid)}")
        self.norm = RmsNorm(shape, 1, device=device)
        self.scan = GatedScan(shape, len(shape) - 1, device=device)
        dev = self.device = self.norm.device
        self.shape, self.C = shape, C
        gen = torch.Generator(device=dev).manual_seed(seed)
        rn = lambda *s: torch.randn(s, device=dev, generator=gen)
        self.weight = torch.ones(C, device=dev)
        self.W_v, self.W_g, self.W_o = (rn(C, C) / C ** 0.5 for _ in range(3))
        self.b_v, self.b_g = torch.zeros(C, device=dev), torch.full((C,), 2.0, device=dev)
        n = Bn.dtst_pointwise_linear_scratch_bytes(C, C)
        self._scratch = torch.empty(n, dtype=torch.uint8, device=dev)
        new = lambda: torch.empty(shape, device=dev)
        self.y, self.v, self.g, self.h, self.out = new(), new(), new(), new(), new()
        self.rstd = torch.empty((B,) + shape[2:], device=dev)
        self.checkpoints = self.scan.new_checkpoints()
        self.x = self.h0 = None

    def forward(self, x, h0=None, stream=None):
        """Returns (out, h_last); both passes work in this object's buffers."""
        if stream is not None:
            with _use(stream, self.device):
                return self.forward(x, h0)
        self.x, self.h0 = x, h0
        self.norm.forward(x, self.weight, out=self.y, rstd=self.rstd)
        Bn.dtst_pointwise_linear(self.y, self.W_v, self.b_v, self.v)
        Bn.dtst_pointwise_linear(self.y, self.W_g, self.b_g, self.g)
        _, last = self.scan.forward(self.v, self.g, h0, out=self.h, checkpoints=self.checkpoints)
        Bn.dtst_pointwise_linear(self.h, self.W_o, None, self.out)
        self.out.add_(x)
        return self.out, last

    def backward(self, grad_out, grad_last=None, stream=None) -> dict:
        if stream is not None:
            with _use(stream, self.device):
                return self.backward(grad_out, grad_last)
        e = torch.empty_like
        gr = {"W_o": e(self.W_o), "W_v": e(self.W_v), "W_g": e(self.W_g), "b_v": e(self.b_v), "b_g": e(self.b_g)}
        gh, gy, gyg = e(self.h), e(self.y), e(self.y)
        back = Bn.dtst_pointwise_linear_backward
        back(grad_out, self.h, self.W_o, gh, gr["W_o"], None, self._scratch)
        gv, gg, gr["h0"] = self.scan.backward(gh, self.v, self.g, self.checkpoints, self.h0, grad_last=grad_last,
                                              need_grad_h0=self.h0 is not None)
        back(gv, self.y, self.W_v, gy, gr["W_v"], gr["b_v"], self._scratch)
        back(gg, self.y, self.W_g, gyg, gr["W_g"], gr["b_g"], self._scratch)
        gy.add_(gyg)
        # the residual's gradient joins inside the norm's backward pass
        gr["x"], gr["weight"] = self.norm.backward(gy, self.x, self.weight, self.rstd, grad_s=grad_out)
        return gr

    def status(self, stream=None) -> int:
        """DTST_OK, or the status word of a bounded wait that gave up since the last query; synchronises."""
        return self.scan.status(stream)


class RolloutMemory:
    """Recurrent layers on latent vectors with 8-bit projections, for serving: a history [B, T, D] at once, then frame
    by frame [B, 1, D] with the state carried on.

        r_0 = x;  per layer: [v | g] = W_in q(norm(r_l)), h = scan(v, g), r_{l+1} = r_l + W_out q(h);  out = norm(r_L)

    x and out are `dtype` (bfloat16 by default); the residual's addition runs inside the next layer's norm.
    weights: per layer (W_in [2 H, D], W_out [D, H], norm weight [D]); final_weight [D].
    """

    def __init__(self, weights: List[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]], final_weight: torch.Tensor,
                 batch: int, dtype: torch.dtype = torch.bfloat16, eps: float = 1e-6):
        self.B, self.dtype, self.eps = int(batch), dtype, eps
        self.D = final_weight.numel()
        self.final_weight, self.device = final_weight, final_weight.device
        self.layers = []
        for w_in, w_out, nw in weights:
            if w_in.shape[1] != self.D or w_in.shape[0] != 2 * w_out.shape[1] or w_out.shape[0] != self.D or nw.numel() != self.D:
                raise ValueError("RolloutMemory: weights are (W_in [2 H, D], W_out [D, H], norm weight [D])")
            self.layers.append((Fp8Linear.from_weight(w_in, dtype), Fp8Linear.from_weight(w_out, dtype), nw))
        self.states = [torch.zeros((self.B, lin.k), device=self.device) for _, lin, _ in self.layers]
        self._plans: dict = {}

    def reset(self) -> None:
        for s in self.states:
            s.zero_()

    def status(self, stream=None) -> int:
        """DTST_OK, or the status word of a bounded wait that gave up since the last query; synchronises."""
        words = [lin.status(stream) for layer in self.layers for lin in layer[:2]]
        with torch.cuda.device(self.device):
            words.append(int(Bn.lib().dtst_gated_scan_status(Bn._stream_ptr(stream))))
        return next((w for w in words if w != Bn.DTST_OK), Bn.DTST_OK)

    def _plan(self, T: int):
        if T not in self._plans:
            while len(self._plans) >= 8:              # histories may come in any length
                del self._plans[next(iter(self._plans))]
            norm = RmsNorm((self.B * T, self.D), -1, self.dtype, self.eps, self.device)
            scans = [GatedScan((self.B, T, lin.k), 1, self.dtype, device=self.device) for _, lin, _ in self.layers]
            self._plans[T] = (norm, scans)
        return self._plans[T]

    def forward(self, x: torch.Tensor, lengths=None, stream=None) -> torch.Tensor:
        """x [B, T, D] -> out [B, T, D]; the layers' states move on by T frames (by lengths[b] where given)."""
        if stream is not None:
            with _use(stream, self.device):
                return self.forward(x, lengths)
        B, T, D = x.shape
        if (B, D) != (self.B, self.D):
            raise ValueError(f"x must be [{self.B}, T, {self.D}], got {tuple(x.shape)}")
        norm, scans = self._plan(T)
        r, delta = x.view(B * T, D), None
        for (lin_in, lin_out, nw), scan, state in zip(self.layers, scans, self.states):
            q, sc, r = norm.forward_fp8(r, nw, residual=delta)
            vg = lin_in.forward(q, sc).view(B, T, 2 * lin_out.k)
            h, _ = scan.forward(vg[..., :lin_out.k], vg[..., lin_out.k:], state, lengths=lengths, h_last=state)
            delta = lin_out.forward(*quantize_fp8(h.view(B * T, lin_out.k)))
        y, _, _ = norm.forward(r, self.final_weight, residual=delta, need_backward=False)
        return y.view(B, T, D)

    def step(self, frame: torch.Tensor, stream=None) -> torch.Tensor:
        """One new frame [B, D] -> [B, D]."""
        return self.forward(frame.view(self.B, 1, self.D), stream=stream).view(self.B, self.D)
