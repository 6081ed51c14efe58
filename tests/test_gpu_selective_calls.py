"""The selective memory's operators and block as they are called on the GPU: padded batches, batches of many entries, states that
decay at once, buffers that share memory, against the float64 statement or against the same call in another form.

Tolerances as in test_gpu_selective: a stored value is off by half a unit in its last place (2^-24 of its size in float32, 2^-8
in bfloat16, 2^-11 in float16), sums in 32 bits by 1e-5, the scan's chains by 3e-5.
"""
import ctypes

import numpy as np
import pytest

from oracle import selective_oracle as S

torch = pytest.importorskip("torch")
from test_gpu_selective import BF16, F32, TYPES, close, host, rand, run_scan, scan_inputs

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ the block
@pytest.mark.parametrize("bad", [0.0, float("nan"), float("inf")])
def test_block_trains_on_ragged_batches(bad):
    """What lies behind an entry's end, in x and in the outputs' gradient, reaches no parameter's gradient: they are the sums of those
    of the entries by themselves (float32: the chain of test_block_gradients_against_autograd, sums over entries in another
    order)."""
    from paper_2607_14394_b200 import SelectiveMemory, clip_grad_norm
    B, T, D, H, N = 4, 23, 24, 48, 8
    lengths = [23, 0, 7, 30]                                  # (beyond T: T)
    m = SelectiveMemory(D, H, N, rank=3, dtype=F32, seed=3)
    x, state, go = rand(B, T, D, seed=1), (rand(B, 3, H, seed=2), rand(B, H, N, seed=3)), rand(B, T, D, seed=4)
    gs = (rand(B, 3, H, seed=5), rand(B, H, N, seed=6))
    want, outs = {k: 0.0 for k in m.NAMES}, []
    for b, n in enumerate(lengths):
        n = min(n, T)
        e = slice(b, b + 1)
        out, new = m.forward(x[e, :n], tuple(s[e] for s in state))
        g = m.backward(go[e, :n], tuple(s[e] for s in gs))
        for k in m.NAMES:
            want[k] = want[k] + g[k].double()
        outs.append((out, *new, g["x"], g["conv_state"], g["h0"]))
        x[b, n:], go[b, n:] = bad, bad
    out, new = m.forward(x, state, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    g = m.backward(go, gs)
    for k in m.NAMES:
        close(g[k], host(want[k]), k, 1e-4)
    for b, n in enumerate(lengths):
        got = (out[b:b + 1, :n], *(s[b:b + 1] for s in new), g["x"][b:b + 1, :n], g["conv_state"][b:b + 1], g["h0"][b:b + 1])
        for p, q, name in zip(got, outs[b], ("out", "conv state", "h", "x", "grad conv_state", "grad h0")):
            close(p, host(q), (b, name), 1e-4)
    assert torch.isfinite(clip_grad_norm({k: g[k] for k in m.NAMES}, 1.0))


# ------------------------------------------------------------------------------------------------ scan
@pytest.mark.parametrize("B,T,lengths", [(2, 1, None), (2, 3, [0, 2]), (1, 16, None), (3, 37, [37, 5, 0]), (2, 1000, [1000, 130])])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_states_that_decay_at_once(B, T, lengths, dtype):
    """A of minus infinity (and beyond float32 once in powers of two) keeps nothing of a state from step to step, as an A of
    -1e30 does: the same bits forward and backward, at every length, and a state passes an entry without steps."""
    from paper_2607_14394_b200 import SelectiveScan
    C, N = 20, 6
    v = scan_inputs(B, T, C, N, 1, dtype)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    scan = SelectiveScan((B, T, C), N, 1, dtype)
    gy, gl = rand(B, T, C, dtype=dtype, seed=50), rand(B, C, N, seed=51)
    got = []
    for a in (-1e30, float("-inf"), -3.0e38):
        v["A"][:, 2], v["A"][3] = a, a
        ck = scan.new_checkpoints()
        y, last = scan.forward(lengths=ln, checkpoints=ck, **v)
        got.append([y, last, *scan.backward(gy, checkpoints=ck, lengths=ln, grad_last=gl, **v).values()])
    v["A"][:, 2], v["A"][3] = -1e30, -1e30
    want = S.selective_scan(lengths=lengths, **{k: host(t) for k, t in v.items()})
    close(got[0][0], want[0], "y", 3e-5)
    close(got[0][1], want[1], "h_last", 3e-5)
    for other in got[1:]:
        assert all(torch.equal(p, q) for p, q in zip(got[0], other))


# ------------------------------------------------------------------------------------------------ convolution
@pytest.mark.parametrize("B,T,C,K", [(262145, 1, 2, 4), (262150, 3, 3, 3), (300001, 2, 1, 1), (140000, 130, 1, 2)])
def test_conv_of_many_sequences(B, T, C, K):
    """More runs than a grid's second dimension holds: the bits of the same batch in parts, the state in its own place."""
    from paper_2607_14394_b200 import CausalConv
    x, w, b = rand(B, T, C, seed=1), rand(C, K, seed=2), rand(C, seed=3)
    s, ln = rand(B, K - 1, C, seed=4), torch.arange(B, device="cuda", dtype=torch.int32) % (T + 2)
    y, last = CausalConv((B, T, C), K).forward(x, w, b, state=s, lengths=ln)
    h = B // 3
    for e in (slice(0, h), slice(h, 2 * h), slice(2 * h, B)):
        part, plast = CausalConv((e.stop - e.start, T, C), K).forward(x[e], w, b, state=s[e], lengths=ln[e])
        assert torch.equal(y[e], part) and torch.equal(last[e], plast)
    state = s.clone()
    again, same = CausalConv((B, T, C), K).forward(x, w, b, state=state, lengths=ln, state_out=state)
    assert torch.equal(again, y) and torch.equal(same, last)


def test_conv_backward_without_steps_through_the_entry_point():
    """Strides of an empty tensor make no elements coincide: the new state's gradient passes to the state, and the sums are empty."""
    from paper_2607_14394_b200 import binding as Bn
    B, C, K = 3, 8, 4
    d = Bn.ConvDesc(0, 1, B, 0, C, K, 0, (0, C), (0, C))
    w, b, s, gso = rand(C, K, seed=1), rand(C, seed=2), rand(B, K - 1, C, seed=3), rand(B, K - 1, C, seed=4)
    gw, gb, gs = (torch.full_like(t, 9.0) for t in (w, b, s))
    n = ctypes.c_size_t()
    assert Bn.lib().dtst_causal_conv_scratch_bytes(ctypes.byref(d), ctypes.byref(n)) == Bn.DTST_OK
    scratch = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    p = lambda t: ctypes.c_void_p(0 if t is None else t.data_ptr())
    status = Bn.lib().dtst_causal_conv_backward(ctypes.byref(d), None, p(gso), None, p(w), p(b), p(s), None, None, p(gw), p(gb), p(gs), p(scratch), n.value,
                                                ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert status == Bn.DTST_OK and torch.equal(gs, gso) and not gw.any() and not gb.any()


@pytest.mark.parametrize("K", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype", TYPES)
def test_conv_off_a_vector(K, dtype):
    """Rows that begin anywhere and an odd distance apart take elements one by one: the bits of the same rows in vectors, over many
    runs a warp, ends inside and in front of them, and with no steps at all."""
    from paper_2607_14394_b200 import CausalConv
    B, T, C = 90, 700, 64
    ends = [700, 0, 1, 2, 3, 63, 64, 65, 66, 67, 68, 699] + [int(i) for i in np.random.default_rng(K).integers(0, 701, B - 12)]
    ln = torch.tensor(ends, dtype=torch.int32, device="cuda")
    x, gy, w, b = rand(B, T, C, dtype=dtype, seed=1), rand(B, T, C, dtype=dtype, seed=2), rand(C, K, seed=3), rand(C, seed=4)
    s, gl = rand(B, K - 1, C, dtype=dtype, seed=5), rand(B, K - 1, C, dtype=dtype, seed=6)
    off = torch.empty(B, T, C + 1, dtype=dtype, device="cuda")[..., 1:]
    off.copy_(x)
    conv = CausalConv((B, T, C), K, dtype)
    got = [[*conv.forward(v, w, b, state=s, lengths=ln), *conv.backward(gy, v, w, b, state=s, lengths=ln, grad_state_out=gl)] for v in (x, off)]
    assert all(torch.equal(p, q) for i, (p, q) in enumerate(zip(*got)) if i not in (3, 4))
    # (the parameters' gradients: a CTA holds other channels, so it visits other runs)
    for i in (3, 4):
        close(got[0][i], host(got[1][i]), i, size=(B * T * C) ** 0.5)


# ------------------------------------------------------------------------------------------------ layer norm
@pytest.mark.parametrize("shape", [(2, 21, 514), (1, 24, 3331), (3, 32, 2054), (1, 29, 66), (2, 20, 1000002), (2, 32, 600004)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual", [False, True])
def test_layer_norm_of_fields_of_20_to_32_channels(shape, dtype, residual):
    """One tile and many a CTA, rows of positions that take vectors of four, of two and none."""
    from paper_2607_14394_b200 import LayerNorm
    C = shape[1]
    x, r = rand(*shape, dtype=dtype, seed=1, shift=0.5), rand(*shape, dtype=dtype, seed=2) if residual else None
    gy, gs, w, b = rand(*shape, dtype=dtype, seed=3), rand(*shape, dtype=dtype, seed=4) if residual else None, rand(C, seed=5, shift=1.0), rand(C, seed=6)
    n = LayerNorm(shape, 1, dtype)
    y, s, stats = n.forward(x, w, b, residual=r)
    gx, gw, gb = n.backward(gy, s, w, stats, grad_s=gs)
    d = lambda t: None if t is None else t.double()
    s64 = d(x) if r is None else d(x) + d(r)                                      # (64 bits on the GPU: elementary operations)
    mean = s64.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((s64 - mean) ** 2).mean(1, keepdim=True) + 1e-5)
    n64 = (s64 - mean) * rstd
    g = d(gy) * d(w)[:, None]
    want = rstd * (g - g.mean(1, keepdim=True) - n64 * (g * n64).mean(1, keepdim=True))
    if gs is not None:
        want = want + d(gs)
    close(y, host(n64 * d(w)[:, None] + d(b)[:, None]), "y")
    close(gx, host(want), "grad_x", size=float((g * rstd).norm()))
    close(gw, host((d(gy) * n64).sum((0, 2))), "grad_weight", size=float((d(gy) * n64).norm()))
    close(gb, host(d(gy).sum((0, 2))), "grad_bias", size=float(d(gy).norm()))
    again = n.backward(gy, s, w, stats, grad_s=gs)
    assert all(torch.equal(p, q) for p, q in zip((gx, gw, gb), again))


# ------------------------------------------------------------------------------------------------ every size of state, far and exact places
@pytest.mark.parametrize("B,T,C,N,G,lengths", [(2, 9, 40, 17, 1, [9, 4]), (1, 1, 70, 31, 1, None), (1, 130, 20, 24, 2, None), (2, 33, 24, 32, 1, None),
                                               (2, 500, 12, 20, 1, [500, 131]), (2, 640, 8, 32, 2, [640, 0]), (1, 700, 10, 33, 1, None), (1, 513, 6, 64, 2, None),
                                               (2, 300, 36, 48, 1, [7, 300])])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gated", [False, True])
def test_scan_of_17_to_64_states(B, T, C, N, G, lengths, dtype, gated):
    """Eight and sixteen lanes to a pair of channels, in one segment and in several."""
    v = scan_inputs(B, T, C, N, G, dtype, gated=gated, strided=gated)
    if lengths is not None:
        for i, n in enumerate(lengths):
            for k in ("x", "dt", "B", "C", "z"):
                if v[k] is not None:
                    v[k][i, n:] = float("nan")
    run_scan(v, N, G, dtype, lengths)


def test_far_offsets_backward():
    """More than 2^31 elements: the first and the last steps of a long sequence by themselves.  Decays are e^-60 and less, so neither
    a state nor a gradient is seen from twenty steps away."""
    from paper_2607_14394_b200 import CausalConv, LayerNorm, SelectiveScan
    T, C, N = (1 << 31) // 1024 + 37, 1024, 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, gy = (torch.empty(1, T, C, dtype=BF16, device="cuda").normal_(generator=gen) for _ in range(2))
    w, b = rand(C, 4, seed=1), rand(C, seed=2)
    gx = CausalConv((1, T, C), 4, BF16).backward(gy, x, w, b)[0]
    part = CausalConv((1, 60, C), 4, BF16)
    assert torch.equal(part.backward(gy[:, -60:].contiguous(), x[:, -60:], w, b, state=x[:, -63:-60])[0], gx[:, -60:])
    assert torch.equal(part.backward(gy[:, :60], x[:, :60], w, b)[0][:, :50], gx[:, :50])
    del gx
    n = LayerNorm((T, C), -1, BF16)
    _, _, stats = n.forward(x[0], b)
    gx = n.backward(gy[0], x[0], b, stats)[0]
    for e in (slice(0, 50), slice(T - 50, T)):
        assert torch.equal(LayerNorm((50, C), -1, BF16).backward(gy[0, e], x[0, e], b, stats[:, e].contiguous(), need_grad_weight=False)[0], gx[e])
    del gx, stats
    I = T * C // 16
    f, gf = x.view(-1)[:16 * I].view(1, 16, I), gy.view(-1)[:16 * I].view(1, 16, I)
    n, bf = LayerNorm((1, 16, I), 1, BF16), b[:16].contiguous()
    y, _, stats = n.forward(f, bf)
    gx = n.backward(gf, f, bf, stats)[0]
    at = slice(I - 999, I)
    small, xs, gs = LayerNorm((1, 16, 999), 1, BF16), f[..., at].contiguous(), gf[..., at].contiguous()
    ys, _, st = small.forward(xs, bf)
    assert torch.equal(ys, y[..., at]) and torch.equal(small.backward(gs, xs, bf, st)[0], gx[..., at])
    del y, gx, stats
    maps = rand(1, T, 1, 2 * N, dtype=BF16, seed=3)
    A, bias = torch.full((C, N), -200.0, device="cuda"), torch.full((C,), 4.0, device="cuda")

    def scan(e):
        xs, g, m = (x, gy, maps) if e is None else (x[:, e].contiguous(), gy[:, e].contiguous(), maps[:, e])
        s = SelectiveScan((1, xs.shape[1], C), N, 1, BF16)
        ck = s.new_checkpoints()
        s.forward(xs, xs, A, m[..., :N], m[..., N:], dt_bias=bias, checkpoints=ck)
        return s.backward(g, xs, xs, A, m[..., :N], m[..., N:], ck, dt_bias=bias)

    whole, front, back = scan(None), scan(slice(0, 40)), scan(slice(T - 40, T))
    for k in ("x", "dt", "B", "C"):
        assert torch.equal(whole[k][:, :20], front[k][:, :20]) and torch.equal(whole[k][:, -20:], back[k][:, -20:]), k


class Guard:
    """The library with scratch of exactly the size that a call states, full of NaNs, between bytes that are looked at afterwards."""
    CALLS = ("dtst_layer_norm_backward", "dtst_causal_conv_backward", "dtst_selective_scan", "dtst_selective_scan_backward", "dtst_clip_grad_norm")

    def __init__(self, lib):
        self.lib, self.kept = lib, []

    def __getattr__(self, name):
        f = getattr(self.lib, name)
        if name not in self.CALLS:
            return f

        def call(*args):
            *rest, scratch, size, stream = args
            base = torch.full((size + 512,), 0xff, dtype=torch.uint8, device="cuda")
            base[:256], base[256 + size:] = 77, 77
            self.kept.append((name, base, size))
            return f(*rest, base.data_ptr() + 256 if scratch else scratch, size, stream)
        return call

    def untouched(self):
        for name, base, size in self.kept:
            assert (base[:256] == 77).all() and (base[256 + size:] == 77).all(), name
        return sorted({name for name, _, _ in self.kept})


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scratch_of_the_stated_size_is_enough(dtype):
    from paper_2607_14394_b200 import CausalConv, GradNorm, LayerNorm, SelectiveScan, binding as Bn
    guard = Guard(Bn.lib())

    def twice(op, call):
        want = call(op)
        op._lib = guard
        assert all(torch.equal(p, q) for p, q in zip(want, call(op))), type(op)

    for shape, dim in (((700, 33), 1), ((3, 1001), 1), ((2, 16385), 1), ((2, 20, 999), 1), ((1, 37, 4096), 1), ((2, 131, 70), 1), ((9000, 2048), 1), ((1, 5, 400000), 1)):
        x, g, w = rand(*shape, dtype=dtype, seed=1), rand(*shape, dtype=dtype, seed=2), rand(shape[dim], seed=3)
        n = LayerNorm(shape, dim, dtype)
        _, s, st = n.forward(x, w)
        twice(n, lambda n: n.backward(g, s, w, st))
    for B, T, C, K in ((3, 700, 33, 4), (1, 1, 1, 1), (50, 300, 130, 3), (2, 5000, 4097, 2)):
        x, g, w = rand(B, T, C, dtype=dtype, seed=1), rand(B, T, C, dtype=dtype, seed=2), rand(C, K, seed=3)
        twice(CausalConv((B, T, C), K, dtype), lambda c: c.backward(g, x, w))
    for B, T, C, N, G in ((2, 900, 33, 5, 1), (1, 1, 1, 1, 1), (3, 40, 129, 17, 1), (1, 3000, 21, 33, 3), (2, 130, 2, 3, 1)):
        v, g = scan_inputs(B, T, C, N, G, dtype), rand(B, T, C, dtype=dtype, seed=50)

        def call(s):
            ck = s.new_checkpoints()
            y, last = s.forward(checkpoints=ck, **v)
            return [y, last, *s.backward(g, checkpoints=ck, grad_last=last, **v).values()]
        twice(SelectiveScan((B, T, C), N, G, dtype), call)
    for count in (1, 16, 17, 128, 129, 300):
        many = [rand(1 + (977 * i) % 40000, dtype=dtype, seed=i) for i in range(count)]
        out = [torch.empty_like(t) for t in many]
        twice(GradNorm(many, out=out), lambda n: [n.clip(1.0), *[t.clone() for t in out], n.norm()])
    assert guard.untouched() == sorted(Guard.CALLS)


@pytest.mark.parametrize("dtype", TYPES)
def test_nothing_around_norms_and_clipped_gradients_is_touched(dtype):
    from paper_2607_14394_b200 import GradNorm, LayerNorm

    def guarded(*shape, dtype=dtype):
        size = int(np.prod(shape))
        base = torch.full((size + 128,), 5.0, dtype=dtype, device="cuda")
        kept.append(base)
        return base[64:64 + size].view(shape)

    kept = []
    for shape, dim in (((5, 37), 1), ((3, 1001), 1), ((2, 16385), 1), ((2, 20, 99), 1), ((1, 30, 66), 1), ((1, 37, 41), 1), ((2, 131, 7), 1)):
        x, r, g, w = (rand(*shape, dtype=dtype, seed=1), rand(*shape, dtype=dtype, seed=2), rand(*shape, dtype=dtype, seed=3), rand(shape[dim], seed=4))
        n, C = LayerNorm(shape, dim, dtype), shape[dim]
        rest = shape[:dim] + shape[dim + 1:]
        stats = guarded(2, *rest, dtype=F32)
        if dtype is not F32:
            stats.sum_low = guarded(*shape)
        y, s, _ = n.forward(x, w, residual=r, out=guarded(*shape), sum_out=guarded(*shape), stats=stats)
        n.backward(g, s, w, stats, grad_s=r, grad_x=guarded(*shape), grad_weight=guarded(C, dtype=F32), grad_bias=guarded(C, dtype=F32))
    grads = [rand(k, dtype=dtype, seed=k) for k in (1, 63, 4095, 4096, 4097, 8193)]
    GradNorm(grads, out=[guarded(t.numel()) for t in grads]).clip(0.5, norm=guarded(dtype=F32))
    for base in kept:
        assert (base[:64] == 5.0).all() and (base[-64:] == 5.0).all()
