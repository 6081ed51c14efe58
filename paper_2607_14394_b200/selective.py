"""Selective memory: the layer norm, the short causal convolution and the selective scan, a block made of them, and the
norm of all gradients with which a training step is clipped.

Where `GatedScan` has one gate for every element, the selective scan keeps several states a channel and takes its step,
its input map and its output map from every token.  `LayerNorm`, `CausalConv`, `SelectiveScan` and `GradNorm` are thin wrappers
over the C entry points (`dtst_layer_norm*`, `dtst_causal_conv*`, `dtst_selective_scan*`, `dtst_clip_grad_norm`) in the manner
of the memory operators: they check arguments, allocate outputs that the caller did not bring, and pass device pointers on.
Every call runs on the current stream, or on the one given as `stream=`; an object holds nothing that calls share, so it may be
used on several streams and from several threads at once (a block, which keeps activations, may not).

`SelectiveMemory` is a trainable block on latent vectors [B, T, D], a history at a time or frame by frame.
"""
from __future__ import annotations

import ctypes
from typing import Iterable, List, Optional, Sequence, Tuple

import torch

from . import binding as Bn
from . import memory as Mem
from .memory import DTYPES, _addr, _check, _on_device, _use

ACTIVATIONS = {None: 0, "silu": 1}
_F32, _I32 = torch.float32, torch.int32


def _there(stream, dev):
    """A context in which `dev` is the current device and `stream` (or that device's current stream) the current stream."""
    return _Both(torch.cuda.device(dev), _use(torch.cuda.current_stream(dev) if stream is None else stream, dev))


class _Both:
    def __init__(self, *contexts):
        self.contexts = contexts

    def __enter__(self):
        for c in self.contexts:
            c.__enter__()

    def __exit__(self, *error):
        for c in reversed(self.contexts):
            c.__exit__(*error)


class _Tokens:
    """Checks of one token-major argument: its type, device and shape, and that the dimensions behind the steps lie together."""

    def __init__(self, name: str, dev: int, dtype: torch.dtype, shape):
        self.name, self.dev, self.dtype, self.shape = name, dev, dtype, torch.Size(shape)
        self.seen = (None, None)                         # the last strides that were found right, and what they gave

    def __call__(self, t: torch.Tensor) -> Tuple[int, Tuple[int, int]]:
        """Address and (batch, step) strides."""
        if t.dtype is not self.dtype or t.get_device() != self.dev:
            _on_device(t, self.name, self.dev, self.dtype)
        if t.shape != self.shape:
            raise ValueError(f"{self.name} must have shape {tuple(self.shape)}, got {tuple(t.shape)}")
        st = t.stride()
        was, at = self.seen                              # (one read: another thread may set it)
        if was != st:
            width = 1
            for i in range(len(st) - 1, 1, -1):
                if self.shape[i] != 1 and st[i] != width:
                    raise ValueError(f"{self.name}: the dimensions behind the steps must lie together")
                width *= self.shape[i]
            at = st[:2]
            self.seen = (st, at)
        return t.data_ptr(), at


class LayerNorm:
    """y = (s - mean) rstd weight + bias, s = x + residual, with mean and variance over dimension `dim` of `shape`.

    `dim` is the last dimension (token-major rows) or any other one (channels-first fields).
    """

    def __init__(self, shape: Sequence[int], dim: int = -1, dtype: torch.dtype = torch.float32, eps: float = 1e-5,
                 device=None):
        self.shape = torch.Size(int(n) for n in shape)
        nd = len(self.shape)
        if nd < 1 or not -nd <= dim < nd:
            raise ValueError(f"dim {dim} is no dimension of shape {tuple(self.shape)}")
        if dtype not in DTYPES:
            raise ValueError(f"dtype must be one of {list(DTYPES)}, got {dtype}")
        self.dim, self.dtype, self.eps, self.dev = dim % nd, dtype, float(eps), Mem._device(device)
        self.device = torch.device("cuda", self.dev)
        self.channels = self.shape[self.dim]
        if self.channels < 1:
            raise ValueError("the normalised dimension is empty")
        self.outer = self.shape[:self.dim].numel()
        self.inner = self.shape[self.dim + 1:].numel()
        self._type = DTYPES[dtype]
        self._stats = torch.Size((2,)) + self.shape[:self.dim] + self.shape[self.dim + 1:]
        self._wshape = torch.Size((self.channels,))
        self._lib = Bn.lib()
        n = ctypes.c_size_t()
        _check(self._lib.dtst_layer_norm_scratch_bytes(self.channels, ctypes.byref(n)), "dtst_layer_norm_scratch_bytes")
        self._scratch_bytes = int(n.value)

    def forward(self, x, weight, bias=None, residual=None, out=None, sum_out=None, stats=None, need_backward=True, stream=None):
        """Returns (y, s, stats); stats [2, ...] are the means and the reciprocal deviations; without a residual s is x itself
        (None where y takes x's place and leaves no s behind).

        In a 16-bit type with a residual, what rounding took from s stays with the stats that are returned (their attribute
        `sum_low`), so that `backward` has the sum to 24 bits; stats that the caller brings may carry such a buffer too (a
        call without a sum to round sets it to None, the next one with a residual makes another).
        need_backward=False: neither is formed, and stats is None.
        """
        d, t, sh = self.dev, self.dtype, self.shape
        if stream is not None or Mem._current_device() != d:
            with _there(stream, d):
                return self.forward(x, weight, bias, residual, out, sum_out, stats, need_backward)
        xp, wp = _addr(x, "x", d, t, sh), _addr(weight, "weight", d, _F32, self._wshape)
        bp = 0 if bias is None else _addr(bias, "bias", d, _F32, self._wshape)
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
        if stats is not None:
            qp = _addr(stats, "stats", d, _F32, self._stats)
            if self._type and hasattr(stats, "sum_low"):
                if not sp:                              # s is x itself; what an earlier call's sum lost is not its
                    stats.sum_low = None
                elif stats.sum_low is None:
                    stats.sum_low = torch.empty_like(x)
                lp = _addr(stats.sum_low, "stats.sum_low", d, t, sh)
        elif need_backward:
            stats = weight.new_empty(self._stats)
            qp = stats.data_ptr()
            if rp and self._type:
                stats.sum_low = low = torch.empty_like(x)
                lp = low.data_ptr()
        status = self._lib.dtst_layer_norm(self._type, self.outer, self.channels, self.inner, self.eps, xp, rp, wp, bp, sp, lp, yp,
                                           qp, Mem._raw_stream(d))
        if status:
            _check(status, "dtst_layer_norm")
        if sum_out is None and (yp != xp or not xp):
            sum_out = x
        return out, sum_out, stats

    def backward(self, grad_y, s, weight, stats, grad_s=None, grad_x=None, grad_weight=None, grad_bias=None,
                 need_grad_weight=True, stream=None, sum_low=None):
        """Returns (grad_x, grad_weight, grad_bias); grad_x is the gradient of x and of the residual.  s and stats as `forward`
        returned them (the attribute `sum_low` does not survive a clone, a detach or a copy: pass it on as `sum_low=`, or
        the gradients are those of the rounded sum).  need_grad_weight=False: neither parameter's gradient is formed."""
        d, t, sh = self.dev, self.dtype, self.shape
        if stream is not None or Mem._current_device() != d:
            with _there(stream, d):
                return self.backward(grad_y, s, weight, stats, grad_s, grad_x, grad_weight, grad_bias, need_grad_weight, None, sum_low)
        gp, wp = _addr(grad_y, "grad_y", d, t, sh), _addr(weight, "weight", d, _F32, self._wshape)
        if grad_x is None:
            grad_x = torch.empty_like(grad_y)
            xp = grad_x.data_ptr()
        else:
            xp = _addr(grad_x, "grad_x", d, t, sh)
        scratch = nbytes = gwp = gbp = 0
        if need_grad_weight:
            grad_weight = torch.empty_like(weight) if grad_weight is None else grad_weight
            grad_bias = torch.empty_like(weight) if grad_bias is None else grad_bias
            gwp, gbp = _addr(grad_weight, "grad_weight", d, _F32, self._wshape), _addr(grad_bias, "grad_bias", d, _F32, self._wshape)
            # the call's own, from the current stream's allocations: calls on other streams may be under way
            partial, nbytes = torch.empty(self._scratch_bytes, dtype=torch.uint8, device=self.device), self._scratch_bytes
            scratch = partial.data_ptr()
        if sum_low is None and self._type:
            sum_low = getattr(stats, "sum_low", None)
        status = self._lib.dtst_layer_norm_backward(
            self._type, self.outer, self.channels, self.inner, gp, _addr(s, "s", d, t, sh), _addr(sum_low, "sum_low", d, t, sh), wp,
            _addr(stats, "stats", d, _F32, self._stats), 0 if grad_s is None else _addr(grad_s, "grad_s", d, t, sh),
            xp, gwp, gbp, scratch, nbytes, Mem._raw_stream(d))
        if status:
            _check(status, "dtst_layer_norm_backward")
        return grad_x, grad_weight, grad_bias


class CausalConv:
    """y_t = act(bias + sum_k weight[:, k] u_(t+k)) for every channel of x [B, T, C], u = the width - 1 steps of the state, then x.

    activation None or "silu"; width 1 to 4.  weight [C, width] and bias [C] are float32; the state [B, width - 1, C] is of the
    tensors' type, the oldest step first.  x may be strided in its first two dimensions (a part of a projection's output).
    """

    def __init__(self, shape: Sequence[int], width: int, dtype: torch.dtype = torch.float32, activation: Optional[str] = "silu",
                 device=None):
        self.shape = torch.Size(int(n) for n in shape)
        if len(self.shape) != 3:
            raise ValueError(f"shape must be [batch, length, channels], got {tuple(self.shape)}")
        if dtype not in DTYPES:
            raise ValueError(f"dtype must be one of {list(DTYPES)}, got {dtype}")
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation must be one of {list(ACTIVATIONS)}, got {activation!r}")
        self.width, self.dtype, self.activation, self.dev = int(width), dtype, activation, Mem._device(device)
        self.device = torch.device("cuda", self.dev)
        B, T, C = self.shape
        self.state_shape = torch.Size((B, max(0, self.width - 1), C))
        self._wshape, self._bshape, self._lshape = torch.Size((C, self.width)), torch.Size((C,)), torch.Size((B,))
        self._x, self._grad_x = (_Tokens(n, self.dev, dtype, self.shape) for n in ("x", "grad_x"))
        self._dense = (T * C, C)
        self._ref = self._describe(self._dense, self._dense)
        self._other = (None, None, None)                 # the last description of other strides
        self._lib = Bn.lib()
        n = ctypes.c_size_t()
        _check(self._lib.dtst_causal_conv_scratch_bytes(self._ref, ctypes.byref(n)), "dtst_causal_conv_scratch_bytes")
        self._scratch_bytes = int(n.value)

    def _describe(self, at, to):
        B, T, C = self.shape
        return ctypes.byref(Bn.ConvDesc(DTYPES[self.dtype], ACTIVATIONS[self.activation], B, T, C, self.width, 0, at, to))

    def _description(self, at, to):
        """The description for these strides.  One that a call may be reading is never changed."""
        if at == self._dense and to == self._dense:
            return self._ref
        a, b, ref = self._other
        if a != at or b != to:
            ref = self._describe(at, to)
            self._other = (at, to, ref)
        return ref

    def _params(self, weight, bias, state, lengths):
        d = self.dev
        return (_addr(weight, "weight", d, _F32, self._wshape), 0 if bias is None else _addr(bias, "bias", d, _F32, self._bshape),
                0 if state is None else _addr(state, "state", d, self.dtype, self.state_shape),
                0 if lengths is None else _addr(lengths, "lengths", d, _I32, self._lshape))

    def forward(self, x, weight, bias=None, state=None, lengths=None, out=None, state_out=None, need_state=True, stream=None):
        """Returns (y, new state).  state_out may be the state itself; need_state=False forms none (None)."""
        d, t = self.dev, self.dtype
        if stream is not None or Mem._current_device() != d:
            with _there(stream, d):
                return self.forward(x, weight, bias, state, lengths, out, state_out, need_state)
        xp, at = self._x(x)
        wp, bp, sp, lp = self._params(weight, bias, state, lengths)
        if out is None:
            out = torch.empty_like(x) if at == self._dense else x.new_empty(self.shape)
            yp = out.data_ptr()
        else:
            yp = _addr(out, "out", d, t, self.shape)
        op = 0
        if state_out is not None:
            op = _addr(state_out, "state_out", d, t, self.state_shape)
        elif need_state:
            state_out = x.new_empty(self.state_shape) if state is None else torch.empty_like(state)
            op = state_out.data_ptr()
        status = self._lib.dtst_causal_conv(self._description(at, self._dense), xp, wp, bp, sp, lp, yp, op, Mem._raw_stream(d))
        if status:
            _check(status, "dtst_causal_conv")
        return out, state_out

    def backward(self, grad_y, x, weight, bias=None, state=None, lengths=None, grad_state_out=None, grad_x=None, grad_weight=None,
                 grad_bias=None, grad_state=None, need_grad_weight=True, need_grad_state=True, stream=None):
        """Returns (grad_x, grad_weight, grad_bias, grad_state); x, weight, bias, state (as it was) and lengths as in the forward
        call.  grad_x may be strided like x.  need_grad_weight=False: neither parameter's gradient is formed."""
        d, t = self.dev, self.dtype
        if stream is not None or Mem._current_device() != d:
            with _there(stream, d):
                return self.backward(grad_y, x, weight, bias, state, lengths, grad_state_out, grad_x, grad_weight, grad_bias,
                                     grad_state, need_grad_weight, need_grad_state)
        xp, at = self._x(x)
        wp, bp, sp, lp = self._params(weight, bias, state, lengths)
        gp = _addr(grad_y, "grad_y", d, t, self.shape)
        if grad_x is None:
            grad_x = torch.empty_like(grad_y)
        gxp, to = self._grad_x(grad_x)
        scratch = nbytes = gwp = gbp = gsp = 0
        if need_grad_weight:
            grad_weight = torch.empty_like(weight) if grad_weight is None else grad_weight
            grad_bias = weight.new_empty(self._bshape) if grad_bias is None else grad_bias
            gwp, gbp = _addr(grad_weight, "grad_weight", d, _F32, self._wshape), _addr(grad_bias, "grad_bias", d, _F32, self._bshape)
            partial, nbytes = torch.empty(self._scratch_bytes, dtype=torch.uint8, device=self.device), self._scratch_bytes
            scratch = partial.data_ptr()
        if grad_state is None and need_grad_state:
            grad_state = grad_y.new_empty(self.state_shape)
        if grad_state is not None:
            gsp = _addr(grad_state, "grad_state", d, t, self.state_shape)
        status = self._lib.dtst_causal_conv_backward(
            self._description(at, to), gp, 0 if grad_state_out is None else _addr(grad_state_out, "grad_state_out", d, t, self.state_shape),
            xp, wp, bp, sp, lp, gxp, gwp, gbp, gsp, scratch, nbytes, Mem._raw_stream(d))
        if status:
            _check(status, "dtst_causal_conv_backward")
        return grad_x, grad_weight, grad_bias, grad_state


class SelectiveScan:
    """y_t = (C_t . h_t + D x_t) silu(z_t), h_t = exp(d_t A) h_(t-1) + d_t x_t B_t, d_t = softplus(dt_t + dt_bias), forward and
    backward, for x, dt, z [B, T, C] and maps B, C [B, T, groups, states].

    A [C, states] (meant to be negative), D, dt_bias [C] and the states h0, h_last [B, C, states] are float32; D, z and dt_bias
    may be None.  softplus=False: d_t = dt_t + dt_bias.  1 to 64 states.  x, dt, z and the maps may be strided in their
    first two dimensions (parts of projections' outputs), and so may the gradients that the caller brings.
    """

    NAMES = ("x", "dt", "z", "B", "C")

    def __init__(self, shape: Sequence[int], states: int, groups: int = 1, dtype: torch.dtype = torch.float32,
                 softplus: bool = True, device=None):
        self.shape = torch.Size(int(n) for n in shape)
        if len(self.shape) != 3:
            raise ValueError(f"shape must be [batch, length, channels], got {tuple(self.shape)}")
        if dtype not in DTYPES:
            raise ValueError(f"dtype must be one of {list(DTYPES)}, got {dtype}")
        self.states, self.groups, self.dtype, self.softplus = int(states), int(groups), dtype, bool(softplus)
        B, T, C = self.shape
        if self.groups < 1 or C % self.groups:
            raise ValueError(f"{C} channels do not make {groups} groups")
        self.dev = Mem._device(device)
        self.device = torch.device("cuda", self.dev)
        self.state_shape, self.maps_shape = torch.Size((B, C, self.states)), torch.Size((B, T, self.groups, self.states))
        self._ashape, self._cshape, self._lshape = torch.Size((C, self.states)), torch.Size((C,)), torch.Size((B,))
        self._shapes = (self.shape, self.shape, self.shape, self.maps_shape, self.maps_shape)
        self._checks = [_Tokens(n, self.dev, dtype, sh) for n, sh in zip(self.NAMES, self._shapes)]
        self._grad_checks = [_Tokens("gradient of " + n, self.dev, dtype, sh) for n, sh in zip(self.NAMES, self._shapes)]
        rows, maps = (T * C, C), (T * self.groups * self.states, self.groups * self.states)
        self._dense = (rows, rows, rows, maps, maps)
        self._ref = self._describe(self._dense, self._dense)
        self._other = (None, None, None)                 # the last description of other strides
        self._lib = Bn.lib()
        n = ctypes.c_int64()
        _check(self._lib.dtst_selective_scan_checkpoints(self._ref, ctypes.byref(n)), "dtst_selective_scan_checkpoints")
        self.checkpoint_floats = int(n.value)
        self._ck_shape = torch.Size((self.checkpoint_floats,))
        self._scratch_bytes = [None, None]               # of either pass; asked for where it is used: it goes by the device

    def new_checkpoints(self) -> torch.Tensor:
        """A buffer for the states that a forward pass saves for its backward pass."""
        return torch.empty(self.checkpoint_floats, dtype=torch.float32, device=self.device)

    def _ask_scratch(self, backward: int) -> int:
        n = ctypes.c_size_t()
        _check(self._lib.dtst_selective_scan_scratch_bytes(self._ref, backward, ctypes.byref(n)), "dtst_selective_scan_scratch_bytes")
        self._scratch_bytes[backward] = int(n.value)
        return int(n.value)

    def _describe(self, at, to):
        B, T, C = self.shape
        return ctypes.byref(Bn.SelectiveDesc(DTYPES[self.dtype], int(self.softplus), B, T, C, self.states, self.groups, *at, *to))

    def _description(self, at, to):
        """The description for these strides.  One that a call may be reading is never changed."""
        if at == self._dense and to == self._dense:
            return self._ref
        a, b, ref = self._other
        if a != at or b != to:
            ref = self._describe(at, to)
            self._other = (at, to, ref)
        return ref

    def _inputs(self, tensors, A, D, dt_bias, h0, lengths):
        """The C structure of the inputs, and their strides."""
        d = self.dev
        x, dt, z, B, C = tensors
        cx, cdt, cz, cb, cc = self._checks
        (xp, xs), (tp, ts), (bp, bs), (cp, cs) = cx(x), cdt(dt), cb(B), cc(C)
        zp, zs = (0, self._dense[2]) if z is None else cz(z)
        return Bn.SelectiveInputs(xp, tp, zp, bp, cp, _addr(A, "A", d, _F32, self._ashape), 0 if D is None else _addr(D, "D", d, _F32, self._cshape),
                                  0 if dt_bias is None else _addr(dt_bias, "dt_bias", d, _F32, self._cshape),
                                  0 if h0 is None else _addr(h0, "h0", d, _F32, self.state_shape),
                                  0 if lengths is None else _addr(lengths, "lengths", d, _I32, self._lshape)), (xs, ts, zs, bs, cs)

    def forward(self, x, dt, A, B, C, D=None, z=None, dt_bias=None, h0=None, lengths=None, out=None, h_last=None, checkpoints=None,
                need_state=True, stream=None):
        """Returns (y, h_last).  lengths: int32 per batch entry; checkpoints: see new_checkpoints; h_last may be h0 itself;
        need_state=False forms none (None)."""
        d = self.dev
        if stream is not None or Mem._current_device() != d:
            with _there(stream, d):
                return self.forward(x, dt, A, B, C, D, z, dt_bias, h0, lengths, out, h_last, checkpoints, need_state)
        inputs, at = self._inputs((x, dt, z, B, C), A, D, dt_bias, h0, lengths)
        if out is None:
            out = torch.empty_like(dt) if dt.is_contiguous() else x.new_empty(self.shape)
            yp = out.data_ptr()
        else:
            yp = _addr(out, "out", d, self.dtype, self.shape)
        lp = 0
        if h_last is not None:
            lp = _addr(h_last, "h_last", d, _F32, self.state_shape)
        elif need_state:
            h_last = A.new_empty(self.state_shape) if h0 is None else torch.empty_like(h0)
            lp = h_last.data_ptr()
        # the call's own, from the current stream's allocations: calls on other streams may be under way
        nbytes = self._scratch_bytes[0] if self._scratch_bytes[0] is not None else self._ask_scratch(0)
        sp = 0
        if nbytes:
            scratch = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            sp = scratch.data_ptr()
        status = self._lib.dtst_selective_scan(
            self._description(at, self._dense), ctypes.byref(inputs), yp, lp,
            0 if checkpoints is None else _addr(checkpoints, "checkpoints", d, _F32, self._ck_shape), sp, nbytes, Mem._raw_stream(d))
        if status:
            _check(status, "dtst_selective_scan")
        return out, h_last

    def backward(self, grad_y, x, dt, A, B, C, checkpoints, D=None, z=None, dt_bias=None, h0=None, lengths=None, grad_last=None,
                 out: Optional[dict] = None, stream=None) -> dict:
        """Gradients by name: x, dt, B, C, A, h0, and z, D, dt_bias where these were given.  Inputs and checkpoints as in the
        forward call; `out` may bring buffers by the same names."""
        d, t = self.dev, self.dtype
        if stream is not None or Mem._current_device() != d:
            with _there(stream, d):
                return self.backward(grad_y, x, dt, A, B, C, checkpoints, D, z, dt_bias, h0, lengths, grad_last, out)
        inputs, at = self._inputs((x, dt, z, B, C), A, D, dt_bias, h0, lengths)
        gp = _addr(grad_y, "grad_y", d, t, self.shape)
        grads = dict(out) if out else {}
        ptr, to = [], []
        for name, shape, dense, check in zip(self.NAMES, self._shapes, self._dense, self._grad_checks):
            if name == "z" and z is None:
                ptr.append(0)
                to.append(dense)
                continue
            if name not in grads:
                grads[name] = torch.empty_like(grad_y) if shape is self.shape else grad_y.new_empty(shape)
            p, s = check(grads[name])
            ptr.append(p)
            to.append(s)
        for name, like, shape in (("A", A, self._ashape), ("D", D, self._cshape), ("dt_bias", dt_bias, self._cshape),
                                  ("h0", h0 if h0 is not None else grad_last, self.state_shape)):
            if like is None and name != "h0":
                ptr.append(0)
                continue
            if name not in grads:
                grads[name] = A.new_empty(shape) if like is None else torch.empty_like(like)
            ptr.append(_addr(grads[name], "gradient of " + name, d, _F32, shape))
        desc = self._description(at, tuple(to))
        nbytes = self._scratch_bytes[1] if self._scratch_bytes[1] is not None else self._ask_scratch(1)
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        g = Bn.SelectiveGrads(*ptr)
        status = self._lib.dtst_selective_scan_backward(
            desc, ctypes.byref(inputs), gp, 0 if grad_last is None else _addr(grad_last, "grad_last", d, _F32, self.state_shape),
            _addr(checkpoints, "checkpoints", d, _F32, self._ck_shape), ctypes.byref(g), scratch.data_ptr(), nbytes,
            Mem._raw_stream(d))
        if status:
            _check(status, "dtst_selective_scan_backward")
        return grads


def _flat(grads) -> Iterable[torch.Tensor]:
    if grads is None:
        return
    if isinstance(grads, torch.Tensor):
        yield grads
        return
    for g in (grads.values() if isinstance(grads, dict) else grads):
        yield from _flat(g)


class GradNorm:
    """The norm of a list of gradients taken as one vector, and their clipping by it.

    tensors: contiguous float32, bfloat16, float16 or complex64 tensors of one device (nested lists and dicts of them, as the
    backward passes here return them; None is passed over).  `out`: tensors like them that receive the clipped gradients;
    without it they are scaled where they are.  The object holds on to the tensors: make it once for buffers that a
    program keeps, and use `clip_grad_norm` for gradients that are new in every step.
    """

    def __init__(self, tensors, out=None, device=None):
        self.tensors: List[torch.Tensor] = list(_flat(tensors))
        self.out: List[torch.Tensor] = self.tensors if out is None else list(_flat(out))
        if len(self.out) != len(self.tensors):
            raise ValueError(f"{len(self.tensors)} gradients, {len(self.out)} outputs")
        self.dev = self.tensors[0].get_device() if self.tensors and device is None else Mem._device(device)
        if self.dev < 0 and Mem._current_device() >= 0:
            raise ValueError(f"gradients must be tensors on a CUDA device, got {self.tensors[0].device}")
        self.device = torch.device("cuda", self.dev)
        n = len(self.tensors)
        self._list = (Bn.GradTensor * n)()
        for e, g, o in zip(self._list, self.tensors, self.out):
            dtype = _F32 if g.dtype is torch.complex64 else g.dtype
            if dtype not in DTYPES:
                raise ValueError(f"gradients must be complex64 or one of {list(DTYPES)}, got {g.dtype}")
            size = g.numel() * (2 if g.dtype is torch.complex64 else 1)
            _as_it_lies(g)
            _as_it_lies(o)
            e.grad, e.out = _addr(g, "gradient", self.dev, g.dtype, g.shape), _addr(o, "out", self.dev, g.dtype, g.shape)
            e.n, e.dtype = size, DTYPES[dtype]
        self._only = (Bn.GradTensor * n)(*self._list)
        for e in self._only:
            e.out = None
        self._lib = Bn.lib()
        b = ctypes.c_size_t()
        _check(self._lib.dtst_grad_norm_scratch_bytes(n, ctypes.byref(b)), "dtst_grad_norm_scratch_bytes")
        self._scratch_bytes = int(b.value)
        self._shape = torch.Size(())

    def _run(self, entries, max_norm, eps, norm, stream):
        d = self.dev
        if stream is not None or Mem._current_device() != d:
            with _there(stream, d):
                return self._run(entries, max_norm, eps, norm, None)
        if norm is None:
            norm = torch.empty((), dtype=_F32, device=self.device)
            np = norm.data_ptr()
        else:
            np = _addr(norm, "norm", d, _F32, self._shape)
        # the call's own, from the current stream's allocations: calls on other streams may be under way
        scratch = torch.empty(self._scratch_bytes, dtype=torch.uint8, device=self.device)
        status = self._lib.dtst_clip_grad_norm(entries, len(entries), max_norm, eps, np, scratch.data_ptr(), self._scratch_bytes,
                                               Mem._raw_stream(d))
        if status:
            _check(status, "dtst_clip_grad_norm")
        return norm

    def norm(self, norm=None, stream=None) -> torch.Tensor:
        """The norm, a float32 tensor on the device; nothing is scaled."""
        return self._run(self._only, float("inf"), 1.0, norm, stream)

    def clip(self, max_norm: float, eps: float = 1e-6, norm=None, stream=None) -> torch.Tensor:
        """Scales by min(1, max_norm / (norm + eps)) and returns the norm as it was, a float32 tensor on the device."""
        return self._run(self._list, max_norm, eps, norm, stream)


def _as_it_lies(t: torch.Tensor) -> None:
    if t.is_conj() or t.is_neg():
        raise ValueError("the values of a conjugated or negated view are not those in memory (resolve_conj(), resolve_neg())")


def clip_grad_norm(grads, max_norm: float, eps: float = 1e-6, stream=None) -> torch.Tensor:
    """Clips gradients (nested lists and dicts as the backward passes return them) where they are; returns their norm."""
    return GradNorm(grads).clip(max_norm, eps, stream=stream)


def _meet(a: Optional[torch.Tensor], b: Optional[torch.Tensor]) -> bool:
    """Whether two contiguous tensors share memory."""
    if a is None or b is None:
        return False
    p, q = a.data_ptr(), b.data_ptr()
    return p < q + b.numel() * b.element_size() and q < p + a.numel() * a.element_size()


class SelectiveMemory:
    """A trainable selective memory on latent vectors x [B, T, D] of `dtype`, pre-normalised and residual:

        n = layer_norm(x);  [u | z] = n W_in^T;  u = conv(u);  [r | B | C] = u W_x^T;  dt = r W_dt^T
        y = selective_scan(u, dt, A, B, C, D, z);  out = x + y W_out^T

    forward(x) -> (out, state) and backward(grad_out) -> gradients of x, of the state in front and of every parameter; step() is the
    form for one new frame.  A state is (the convolution's last inputs [B, width - 1, H], h [B, H, states]).  Parameters are
    plain tensors owned by this object (`parameters()`); the projections are plain matrix products.

    Behind an entry's own length `out` is x and the gradient of x that of `out`, whatever they hold there; neither reaches a
    state or a parameter's gradient.
    """

    NAMES = ("norm_weight", "norm_bias", "W_in", "conv_weight", "conv_bias", "W_x", "W_dt", "dt_bias", "A_log", "D", "W_out")

    def __init__(self, D: int, H: int, states: int = 16, rank: Optional[int] = None, width: int = 4, dtype: torch.dtype = torch.bfloat16,
                 device=None, seed: int = 0, eps: float = 1e-5):
        if dtype not in DTYPES:
            raise ValueError(f"dtype must be one of {list(DTYPES)}, got {dtype}")
        self.D_model, self.H, self.states, self.width, self.dtype, self.eps = int(D), int(H), int(states), int(width), dtype, eps
        self.rank = max(1, D // 16) if rank is None else int(rank)
        self.device = dev = torch.device("cuda", Mem._device(device))
        gen = torch.Generator(device=dev).manual_seed(seed)
        rn = lambda *s: torch.randn(s, device=dev, generator=gen)
        self.norm_weight, self.norm_bias = torch.ones(D, device=dev), torch.zeros(D, device=dev)
        self.W_in = (rn(2 * H, D) / D ** 0.5).to(dtype)
        self.conv_weight, self.conv_bias = rn(H, width) / width ** 0.5, torch.zeros(H, device=dev)
        self.W_x = (rn(self.rank + 2 * states, H) / H ** 0.5).to(dtype)
        self.W_dt = (rn(H, self.rank) / self.rank ** 0.5).to(dtype)
        step = torch.exp(torch.rand(H, device=dev, generator=gen) * 4.6 - 6.9)          # 0.001 to 0.1
        self.dt_bias = step + torch.log(-torch.expm1(-step))
        self.A_log = torch.log(torch.arange(1, states + 1, device=dev, dtype=torch.float32)).expand(H, states).contiguous()
        self.D = torch.ones(H, device=dev)
        self.W_out = (rn(D, H) / H ** 0.5).to(dtype)
        self._plans: dict = {}
        self._zero = torch.zeros((), dtype=dtype, device=dev)
        self.saved = None

    def parameters(self) -> dict:
        return {n: getattr(self, n) for n in self.NAMES}

    def new_state(self, B: int) -> Tuple[torch.Tensor, torch.Tensor]:
        return (torch.zeros((B, self.width - 1, self.H), dtype=self.dtype, device=self.device),
                torch.zeros((B, self.H, self.states), device=self.device))

    def _plan(self, B: int, T: int):
        if (B, T) not in self._plans:
            while len(self._plans) >= 8:              # histories may come in any length
                del self._plans[next(iter(self._plans))]
            self._plans[B, T] = (LayerNorm((B, T, self.D_model), -1, self.dtype, self.eps, self.device),
                                 CausalConv((B, T, self.H), self.width, self.dtype, "silu", self.device),
                                 SelectiveScan((B, T, self.H), self.states, 1, self.dtype, True, self.device))
        return self._plans[B, T]

    def _maps(self, u):
        """The step's low-rank form and both maps of the scan."""
        both = u @ self.W_x.t()
        r, s = self.rank, self.states
        return both, both[..., :r], both[..., r:r + s].unsqueeze(2), both[..., r + s:].unsqueeze(2)

    def forward(self, x, state=None, lengths=None, training=True, state_out=None, stream=None):
        """Returns (out, state); training=False keeps nothing for a backward pass.  state_out may be the state itself where
        training is False (a backward pass needs the state as it was)."""
        if stream is not None:
            with _use(stream, self.device):
                return self.forward(x, state, lengths, training, state_out)
        x = x.contiguous()
        B, T, D = x.shape
        norm, conv, scan = self._plan(B, T)
        H = self.H
        before, h0 = (None, None) if state is None else state
        if training and state is not None and state_out is not None and any(_meet(o, i) for o in state_out for i in state):
            raise ValueError("a backward pass needs the state as it was: state_out must be another one where training is True")
        own = seen = None
        if lengths is not None and training:
            # the parameters' gradients are sums over all rows, and zero times a NaN is no zero: chosen, not multiplied
            _addr(lengths, "lengths", norm.dev, _I32, conv._lshape)
            own = torch.arange(T, device=x.device).view(T, 1) < lengths.view(B, 1, 1)
            seen = torch.where(own, x, self._zero)
        n, s, stats = norm.forward(x if seen is None else seen, self.norm_weight, self.norm_bias, need_backward=training)
        uz = n @ self.W_in.t()
        after, h = (None, None) if state_out is None else state_out
        u, after = conv.forward(uz[..., :H], self.conv_weight, self.conv_bias, state=before, lengths=lengths, state_out=after)
        both, r, Bm, Cm = self._maps(u)
        dt = r @ self.W_dt.t()
        A = -torch.exp(self.A_log)
        ck = scan.new_checkpoints() if training else None
        y, h = scan.forward(u, dt, A, Bm, Cm, D=self.D, z=uz[..., H:], dt_bias=self.dt_bias, h0=h0, lengths=lengths, h_last=h,
                            checkpoints=ck)
        out = x + y @ self.W_out.t()
        self.saved = (s, n, stats, uz, u, both, dt, A, y, ck, before, h0, lengths, own) if training else None
        return out, (after, h)

    def step(self, frame, state, stream=None):
        """One new frame [B, D] -> [B, D]; the state moves on where it is."""
        return self.forward(frame.unsqueeze(1), state, training=False, state_out=state, stream=stream)[0].squeeze(1)

    def backward(self, grad_out, grad_state=None, stream=None) -> dict:
        """Gradients of every parameter, of x, and of the state in front ("conv_state", "h0")."""
        if stream is not None:
            with _use(stream, self.device):
                return self.backward(grad_out, grad_state)
        if self.saved is None:
            raise RuntimeError("backward follows a forward pass with training=True")
        s, n, stats, uz, u, both, dt, A, y, ck, before, h0, lengths, own = self.saved
        grad_out = grad_out.contiguous()
        B, T, D = grad_out.shape
        norm, conv, scan = self._plan(B, T)
        H, R, S, flat = self.H, self.rank, self.states, lambda t: t.flatten(0, 1)
        g_after, g_last = (None, None) if grad_state is None else grad_state
        gr = {"W_out": flat(grad_out if own is None else torch.where(own, grad_out, self._zero)).t() @ flat(y)}
        gy = grad_out @ self.W_out
        guz, gboth = torch.empty_like(uz), torch.empty_like(both)
        g = scan.backward(gy, u, dt, A, both[..., R:R + S].unsqueeze(2), both[..., R + S:].unsqueeze(2), ck, D=self.D, z=uz[..., H:],
                          dt_bias=self.dt_bias, h0=h0, lengths=lengths, grad_last=g_last,
                          out={"z": guz[..., H:], "B": gboth[..., R:R + S].unsqueeze(2), "C": gboth[..., R + S:].unsqueeze(2)})
        gr["D"], gr["dt_bias"], gr["A_log"], gr["h0"] = g["D"], g["dt_bias"], g["A"] * A, g["h0"]
        gr["W_dt"] = flat(g["dt"]).t() @ flat(both[..., :R])
        gboth[..., :R] = g["dt"] @ self.W_dt
        gr["W_x"] = flat(gboth).t() @ flat(u)
        gu = g["x"].add_(gboth @ self.W_x)
        _, gr["conv_weight"], gr["conv_bias"], gr["conv_state"] = conv.backward(
            gu, uz[..., :H], self.conv_weight, self.conv_bias, state=before, lengths=lengths, grad_state_out=g_after, grad_x=guz[..., :H])
        gr["W_in"] = flat(guz).t() @ flat(n)
        gr["x"], gr["norm_weight"], gr["norm_bias"] = norm.backward(guz @ self.W_in, s, self.norm_weight, stats, grad_s=grad_out)
        return gr
