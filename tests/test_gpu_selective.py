"""Selective-memory operators on the GPU against the float64 statement.

Tolerances (relative L2 of a whole output).  A stored value is rounded once: at most half a unit in the last place, 2^-24 of its
size in float32, 2^-8 in bfloat16, 2^-11 in float16.  Norm, convolution and clipping: sums of a few to a few thousand terms in
32 bits in front of that, as the other operators here 1e-5.  Scan: a decay is off by at most 2^-22 of its size and its product
with the state by 2^-24, an error that lives as long as what it is in, 1 / (1 - a) steps and no longer than the sequence; with
the steps below (0.02 and more, states that decay by 1 or more a unit of time: 50 steps) that is 50 (2^-22 + 2^-24) = 1.5e-5 of a
state at worst, twice that where a gradient has gone through the decays a second time: 3e-5.
"""
import numpy as np
import pytest

from oracle import selective_oracle as S

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
HALF = {F32: 0.0, BF16: 2.0 ** -8, F16: 2.0 ** -11}
EPS = 1e-5


def rand(*shape, dtype=F32, seed=0, scale=1.0, shift=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=gen) * scale + shift).to(dtype)


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def close(got, want, what="", tol=1e-5, size=0.0):
    t = tol + HALF[got.dtype]
    got = host(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert np.isfinite(got).all(), what
    off, norm = np.linalg.norm(got - want), np.linalg.norm(want)
    assert off <= t * max(norm, size), (what, off, norm)


def as3(t, dim):
    return None if t is None else host(t).reshape(int(np.prod(t.shape[:dim])), t.shape[dim], int(np.prod(t.shape[dim + 1:])))


# ------------------------------------------------------------------------------------------------ layer norm
NORM_SHAPES = [((1, 7), 1), ((3, 64), 1), ((5, 250), 1), ((9, 511), 1), ((2, 1000), 1), ((700, 1024), 1), ((3, 2048), 1), ((2, 4100), 1),
               ((3, 8192), 1), ((3, 8190), 1), ((2, 16390), 1), ((2, 3, 40), 2), ((1, 4, 64), 1), ((2, 20, 30, 7), 1), ((1, 32, 1000), 1),
               ((2, 33, 257), 1), ((1, 128, 64), 1), ((2, 150, 90), 1), ((1, 5, 200000), 1), ((1, 16, 2052), 1)]


@pytest.mark.parametrize("shape,dim", NORM_SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual", [False, True])
def test_layer_norm_forward_and_backward(shape, dim, dtype, residual):
    from paper_2607_14394_b200 import LayerNorm
    x, r = rand(*shape, dtype=dtype, seed=1, shift=0.7), rand(*shape, dtype=dtype, seed=2, scale=2.0) if residual else None
    gy, gs = rand(*shape, dtype=dtype, seed=3), rand(*shape, dtype=dtype, seed=4) if residual else None
    w, b = rand(shape[dim], seed=5, scale=0.2, shift=1.0), rand(shape[dim], seed=6, scale=0.3)
    n = LayerNorm(shape, dim, dtype, EPS)
    y, s, stats = n.forward(x, w, b, residual=r)
    ry, rs, mean, rstd = S.layer_norm(as3(x, dim), host(w), host(b), EPS, as3(r, dim))
    v = ry.shape
    close(y.view(v), ry, "y")
    close(s.view(v), rs, "s")
    close(stats[0].reshape(mean.shape), mean, "mean", size=np.linalg.norm(rs) / v[1] ** 0.5)
    close(stats[1].reshape(rstd.shape), rstd, "rstd")
    gx, gw, gb = n.backward(gy, s, w, stats, grad_s=gs)
    rgx, rgw, rgb = S.layer_norm_backward(as3(gy, dim), rs, host(w), mean, rstd, as3(gs, dim))
    size = np.linalg.norm(as3(gy, dim) * host(w)[None, :, None] * rstd[:, None, :])
    close(gx.view(v), rgx, "grad_x", size=size)
    # a sum of terms of both signs is held to the terms' size
    n64 = (rs - mean[:, None, :]) * rstd[:, None, :]
    close(gw, rgw, "grad_weight", size=np.linalg.norm(as3(gy, dim) * n64))
    close(gb, rgb, "grad_bias", size=np.linalg.norm(as3(gy, dim)))
    again = n.backward(gy, s, w, stats, grad_s=gs)
    assert all(torch.equal(p, q) for p, q in zip((gx, gw, gb), again))
    only = n.backward(gy, s, w, stats, grad_s=gs, need_grad_weight=False)
    assert only[1] is None and only[2] is None and torch.equal(only[0], gx)
    assert torch.equal(n.forward(x, w, b, residual=r, need_backward=False)[0], y)
    close(n.forward(x, w, residual=r)[0].view(v), S.layer_norm(as3(x, dim), host(w), None, EPS, as3(r, dim))[0], "no bias")


@pytest.mark.parametrize("dtype", TYPES)
def test_layer_norm_of_a_large_mean(dtype):
    """The variance is of the differences from the mean: an offset of 2^10 spreads costs no bits that the input has."""
    from paper_2607_14394_b200 import LayerNorm
    for shape, dim in [((4, 1000), 1), ((4, 16400), 1), ((2, 20, 50), 1), ((1, 140, 33), 1)]:
        x = rand(*shape, seed=7, scale=1.0, shift=1024.0).to(dtype)
        w = torch.ones(shape[dim], device="cuda")
        y, _, _ = LayerNorm(shape, dim, dtype, EPS).forward(x, w)
        # the sum of C values of 1024 is off by a few units of 2^-24 of its terms' size: 1024 2^-22 of a spread
        want = S.layer_norm(as3(x, dim), host(w), None, EPS)[0]
        close(y.view(want.shape), want, "y", tol=1024 * 2.0 ** -21)


def test_layer_norm_special_values_and_places():
    from paper_2607_14394_b200 import LayerNorm
    n, w = LayerNorm((4, 200), -1, F32, EPS), torch.ones(200, device="cuda")
    x = rand(4, 200, seed=1)
    x[1], x[2, 5] = 3.0, float("nan")
    y, _, stats = n.forward(x, w)
    assert torch.equal(y[1], torch.zeros_like(y[1])) and torch.isnan(y[2]).all()
    assert torch.isfinite(y[0]).all() and torch.isfinite(y[3]).all()           # rows do not touch each other
    for dtype in TYPES:
        for shape, dim in [((6, 1000), 1), ((6, 64), 1), ((2, 20, 36), 1), ((3, 16400), 1)]:
            n = LayerNorm(shape, dim, dtype, EPS)
            x, r, w, b = rand(*shape, dtype=dtype, seed=1), rand(*shape, dtype=dtype, seed=2), rand(shape[dim], seed=3), rand(shape[dim], seed=4)
            y, s, st = n.forward(x, w, b, residual=r)
            x2, r2 = x.clone(), r.clone()
            n.forward(x2, w, b, residual=r2, sum_out=r2, out=x2)
            assert torch.equal(r2, s) and torch.equal(x2, y)
            g = rand(*shape, dtype=dtype, seed=5)
            want, g2 = n.backward(g, s, w, st), g.clone()
            got = n.backward(g2, s, w, st, grad_x=g2)
            assert all(torch.equal(p, q) for p, q in zip(got, want)) and got[0] is g2
    # a view that begins off a vector
    base, w = rand(3 * 64 + 1, dtype=BF16, seed=6), rand(64, seed=7)
    n = LayerNorm((3, 64), -1, BF16)
    assert torch.equal(n.forward(base[1:].view(3, 64), w)[0], n.forward(base[1:].clone().view(3, 64), w)[0])
    e = LayerNorm((0, 8), -1, F32)
    gx, gw, gb = e.backward(torch.empty(0, 8, device="cuda"), torch.empty(0, 8, device="cuda"), torch.ones(8, device="cuda"), torch.empty(2, 0, device="cuda"))
    assert not gw.any() and not gb.any() and gx.shape == (0, 8)


# ------------------------------------------------------------------------------------------------ convolution
def conv_inputs(B, T, C, K, dtype, strided, seed=0):
    x = rand(B, T, 2 * C, dtype=dtype, seed=seed)[..., C:] if strided else rand(B, T, C, dtype=dtype, seed=seed)
    return x, rand(C, K, seed=seed + 1, scale=K ** -0.5), rand(C, seed=seed + 2, scale=0.2), rand(B, K - 1, C, dtype=dtype, seed=seed + 3)


CONV_CASES = [(1, 1, 1, 4, None), (3, 1, 64, 4, None), (2, 2, 7, 4, [0, 2]), (3, 37, 260, 4, [37, 0, 3]), (2, 300, 64, 3, None),
              (4, 65, 33, 2, [1, 64, 65, 200]), (2, 50, 128, 1, [50, -3]), (1, 1000, 8, 4, None), (5, 17, 1024, 4, [2, 16, 17, 1, 0]), (2, 0, 8, 4, None)]


@pytest.mark.parametrize("B,T,C,K,lengths", CONV_CASES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("silu,strided,bare", [(True, True, False), (False, False, False), (True, False, True)])
def test_conv_forward_and_backward(B, T, C, K, lengths, dtype, silu, strided, bare):
    from paper_2607_14394_b200 import CausalConv
    x, w, b, s = conv_inputs(B, T, C, K, dtype, strided)
    gy, gl = rand(B, T, C, dtype=dtype, seed=8), rand(B, K - 1, C, dtype=dtype, seed=9)
    if bare:
        b = s = gl = None
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if lengths is not None:                      # what lies behind a sequence's end is not used
        for i, n in enumerate(lengths):
            x[i, max(n, 0):], gy[i, max(n, 0):] = float("nan"), float("inf")
    conv = CausalConv((B, T, C), K, dtype, "silu" if silu else None)
    y, last = conv.forward(x, w, b, state=s, lengths=ln)
    with np.errstate(invalid="ignore"):
        ry, rl = S.causal_conv(host(x), host(w), host(b), host(s), lengths, silu)
    close(y, ry, "y")
    close(last, rl, "state")
    gx = torch.full((B, T, 2 * C), 7.0, dtype=dtype, device="cuda")
    got = conv.backward(gy, x, w, b, state=s, lengths=ln, grad_state_out=gl, grad_x=gx[..., :C])
    want = S.causal_conv_backward(host(gy), host(x), host(w), host(b), host(s), lengths, host(gl), silu)
    scale = max(1.0, B * T) ** 0.5                 # the sums' terms are of unit size
    for g, r, name, size in zip(got, want, ("grad_x", "grad_weight", "grad_bias", "grad_state"), (0, scale * C ** 0.5, scale * C ** 0.5, 0)):
        close(g, r, name, size=size)
    assert (gx[..., C:] == 7.0).all()
    again = conv.backward(gy, x, w, b, state=s, lengths=ln, grad_state_out=gl)
    assert all(torch.equal(p, q) for p, q in zip(got, again))
    none = conv.backward(gy, x, w, b, state=s, lengths=ln, grad_state_out=gl, need_grad_weight=False, need_grad_state=False)
    assert torch.equal(none[0], got[0]) and none[1:] == (None, None, None)


@pytest.mark.parametrize("dtype", TYPES)
def test_conv_steps_are_the_whole(dtype):
    """A sequence in pieces, the state moving on in its own place, has the same bits as the whole."""
    from paper_2607_14394_b200 import CausalConv
    B, T, C, K = 3, 23, 40, 4
    x, w, b, s = conv_inputs(B, T, C, K, dtype, False)
    y, last = CausalConv((B, T, C), K, dtype).forward(x, w, b, state=s)
    state, parts, t = s.clone(), [], 0
    for n in (1, 1, 2, 7, 1, 11):
        part, out = CausalConv((B, n, C), K, dtype).forward(x[:, t:t + n], w, b, state=state, state_out=state)
        assert out is state
        parts.append(part)
        t += n
    assert torch.equal(torch.cat(parts, 1), y) and torch.equal(state, last)


# ------------------------------------------------------------------------------------------------ scan
def scan_inputs(B, T, C, N, G, dtype, seed=0, gated=True, strided=True, D=True, softplus=True):
    two = rand(B, T, 2 * C, dtype=dtype, seed=seed)
    maps = rand(B, T, 2 * G * N + 3, dtype=dtype, seed=seed + 1)
    v = {"x": two[..., :C] if strided else rand(B, T, C, dtype=dtype, seed=seed + 2),
         "dt": rand(B, T, C, dtype=dtype, seed=seed + 3, scale=0.3) if softplus else rand(B, T, C, seed=seed + 3, scale=0.1, shift=0.3).abs().to(dtype),
         "A": -torch.arange(1, N + 1, device="cuda", dtype=F32) * torch.exp(0.1 * rand(C, N, seed=seed + 4)),
         "B": maps[..., 3:3 + G * N].unflatten(-1, (G, N)), "C": maps[..., 3 + G * N:].unflatten(-1, (G, N)),
         "D": rand(C, seed=seed + 5) if D else None, "z": two[..., C:] if gated else None,
         # steps of about 0.05 to 0.3
         "dt_bias": rand(C, seed=seed + 6, scale=0.5, shift=-2.0) if softplus else None, "h0": rand(B, C, N, seed=seed + 7)}
    return v


def run_scan(v, N, G, dtype, lengths=None, softplus=True, train=True, seed=50, check=True):
    from paper_2607_14394_b200 import SelectiveScan
    B, T, C = v["x"].shape
    scan = SelectiveScan((B, T, C), N, G, dtype, softplus)
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    rest = {k: v[k] for k in ("D", "z", "dt_bias", "h0")}
    args = (v["x"], v["dt"], v["A"], v["B"], v["C"])
    ck = scan.new_checkpoints().fill_(float("nan"))
    y, last = scan.forward(*args, lengths=ln, checkpoints=ck, **rest)
    plain = scan.forward(*args, lengths=ln, **rest)
    assert torch.equal(plain[0], y) and torch.equal(plain[1], last)
    gy, gl = rand(B, T, C, dtype=dtype, seed=seed), rand(B, C, N, seed=seed + 1)
    if lengths is not None:
        for i, n in enumerate(lengths):
            gy[i, max(n, 0):] = float("nan")
    g = scan.backward(gy, *args, ck, lengths=ln, grad_last=gl, **rest)
    again = scan.backward(gy, *args, ck, lengths=ln, grad_last=gl, **rest)
    assert g.keys() == again.keys() and all(torch.equal(g[k], again[k]) for k in g)
    if check:
        h = {k: host(t) for k, t in v.items()}
        with np.errstate(invalid="ignore", over="ignore"):
            ry, rl = S.selective_scan(lengths=lengths, softplus=softplus, **h)
            rg = S.selective_scan_backward(host(gy), lengths=lengths, grad_last=host(gl), softplus=softplus, **h)
        close(y, ry, "y", 3e-5)
        close(last, rl, "h_last", 3e-5)
        assert set(g) == {k for k in rg if k not in ("D", "dt_bias") or v[k] is not None}
        for k in g:
            # (sums over everything: held to their terms' size, the sum over a batch of independent terms)
            size = np.linalg.norm(rg["h0"]) + (B * T) ** 0.5 if k in ("A", "D", "dt_bias") else 0.0
            close(g[k], rg[k], "grad_" + k, 3e-5, size)
    return y, last, g


SCAN_CASES = [(1, 1, 1, 1, 1, None), (4, 1, 96, 16, 1, None), (2, 2, 6, 5, 2, [2, 0]), (2, 7, 64, 16, 1, [7, 3]), (2, 8, 33, 16, 1, None),
              (1, 9, 40, 16, 1, None), (3, 16, 24, 4, 2, [16, 15, 1]), (2, 17, 130, 12, 1, None), (2, 33, 20, 64, 1, [40, -1]), (1, 64, 8, 33, 1, None),
              (1, 129, 16, 16, 2, None), (3, 130, 10, 8, 1, [129, 64, 65]), (1, 300, 66, 16, 1, None), (2, 257, 12, 3, 3, [256, 8])]


@pytest.mark.parametrize("B,T,C,N,G,lengths", SCAN_CASES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gated,strided,full,softplus", [(True, True, True, True), (False, False, False, True), (True, False, True, False)])
def test_scan_forward_and_backward(B, T, C, N, G, lengths, dtype, gated, strided, full, softplus):
    v = scan_inputs(B, T, C, N, G, dtype, gated=gated, strided=strided, D=full, softplus=softplus)
    if lengths is not None:                      # what lies behind a sequence's end is not used
        for i, n in enumerate(lengths):
            n = max(n, 0)
            for k, bad in (("x", float("nan")), ("dt", float("inf")), ("B", float("nan")), ("C", float("-inf")), ("z", float("nan"))):
                if v[k] is not None:
                    v[k][i, n:] = bad
    if not full:
        v["h0"] = v["dt_bias"] = None
        v["dt"] = (v["dt"].float() - 2.0).to(dtype)
    run_scan(v, N, G, dtype, lengths, softplus)


def test_scan_with_many_channels_takes_one_run_a_tile():
    """Enough channels for every SM: the kernels without runs, against the ones with runs on a part of the batch."""
    for dtype in (F32, BF16):
        v = scan_inputs(8, 40, 2500, 16, 1, dtype)
        y, last, g = run_scan(v, 16, 1, dtype, check=False)
        part = {k: t[2:3].contiguous() if k in ("x", "dt", "z", "h0") else t[2:3] if k in ("B", "C") else t for k, t in v.items()}
        part = {k: (t[..., :40] if k in ("x", "dt", "z", "D", "dt_bias") else t[:40] if k == "A" else t[:, :40] if k == "h0" else t) for k, t in part.items()}
        part = {k: t if k in ("B", "C") else t.contiguous() for k, t in part.items()}
        h = {k: host(t) for k, t in part.items()}
        ry, rl = S.selective_scan(**h)
        close(y[2:3, :, :40], ry, "y", 3e-5)
        close(last[2:3, :40], rl, "h_last", 3e-5)
        gy, gl = rand(8, 40, 2500, dtype=dtype, seed=50), rand(8, 2500, 16, seed=51)
        rg = S.selective_scan_backward(host(gy[2:3, :, :40]), grad_last=host(gl[2:3, :40]), **h)
        for k in ("x", "dt", "z"):
            close(g[k][2:3, :, :40], rg[k], k, 3e-5)
        close(g["h0"][2:3, :40], rg["h0"], "h0", 3e-5)
        # sums over all channels and the batch, by the identity that ties them to the others: sum_t,n B gB = sum_c x gx - D x gy'
        lhs = (v["B"].double() * g["B"].double()).sum()
        z = v["z"].double()
        direct = (gy.double() * z * torch.sigmoid(z) * v["x"].double() * v["D"].double())
        rhs = (v["x"].double() * g["x"].double()).sum() - direct.sum()
        size = float((v["x"].double() * g["x"].double()).norm() + direct.norm() + (v["B"].double() * g["B"].double()).norm())
        assert abs(float(lhs - rhs)) <= (3e-5 + 2 * HALF[dtype]) * size * 4


@pytest.mark.parametrize("dtype", TYPES)
def test_scan_steps_are_the_whole(dtype):
    """A sequence in pieces, the state moving on in its own place: the same state and outputs to 32-bit rounding."""
    from paper_2607_14394_b200 import SelectiveScan
    B, T, C, N = 2, 61, 48, 16
    v = scan_inputs(B, T, C, N, 1, dtype)
    rest = {k: v[k] for k in ("D", "dt_bias")}
    y, last = SelectiveScan((B, T, C), N, 1, dtype).forward(v["x"], v["dt"], v["A"], v["B"], v["C"], z=v["z"], h0=v["h0"], **rest)
    h, parts, t = v["h0"].clone(), [], 0
    for n in (1, 1, 2, 30, 1, 26):
        p = slice(t, t + n)
        out, same = SelectiveScan((B, n, C), N, 1, dtype).forward(v["x"][:, p], v["dt"][:, p], v["A"], v["B"][:, p], v["C"][:, p], z=v["z"][:, p],
                                                                 h0=h, h_last=h, **rest)
        assert same is h
        parts.append(out)
        t += n
    close(torch.cat(parts, 1), host(y), "y", 3e-5)
    close(h, host(last), "h", 3e-5)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_state_in_place_of_a_sequence_in_segments(dtype):
    """Few channels and many steps: the state behind may take the place of the state in front while segments still read that."""
    from paper_2607_14394_b200 import SelectiveScan
    B, T, C, N = 2, 5000, 100, 16
    v = scan_inputs(B, T, C, N, 1, dtype)
    v["A"] = v["A"] * 1e-3                                # states that last: what is in front is seen everywhere
    scan = SelectiveScan((B, T, C), N, 1, dtype)
    ck = scan.new_checkpoints()
    y, last = scan.forward(checkpoints=ck, **v)
    h0 = v["h0"].clone()
    gy, gl = rand(B, T, C, dtype=dtype, seed=50), rand(B, C, N, seed=51)
    g = scan.backward(gy, checkpoints=ck, grad_last=gl, **v)
    for _ in range(5):
        v["h0"] = h0.clone()
        again, same = scan.forward(h_last=v["h0"], **v)
        assert same is v["h0"] and torch.equal(again, y) and torch.equal(same, last)
        at = gl.clone()
        h = scan.backward(gy, checkpoints=ck, grad_last=at, out={"h0": at}, **v)
        assert h["h0"] is at and all(torch.equal(h[k], g[k]) for k in g)


def test_scan_without_steps():
    from paper_2607_14394_b200 import SelectiveScan
    v = scan_inputs(2, 0, 10, 5, 1, F32, strided=False)
    scan = SelectiveScan((2, 0, 10), 5)
    ck = scan.new_checkpoints()
    y, last = scan.forward(checkpoints=ck, **v)
    gl = rand(2, 10, 5, seed=3)
    g = scan.backward(torch.empty(2, 0, 10, device="cuda"), checkpoints=ck, grad_last=gl, **v)
    assert y.shape == (2, 0, 10) and torch.equal(last, v["h0"]) and torch.equal(g["h0"], gl)
    assert not g["A"].any() and not g["D"].any() and not g["dt_bias"].any() and g["B"].shape == (2, 0, 1, 5)


def test_scan_gradient_against_differences():
    from paper_2607_14394_b200 import SelectiveScan
    B, T, C, N = 2, 20, 24, 16
    v = scan_inputs(B, T, C, N, 1, F32, strided=False)
    scan = SelectiveScan((B, T, C), N)
    names = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "h0")
    v = {k: v[k].contiguous() for k in names}
    gy, gl = rand(B, T, C, seed=60), rand(B, C, N, seed=61)

    def loss(u):
        y, last = scan.forward(**u)
        return float((y.double() * gy.double()).sum() + (last.double() * gl.double()).sum())

    ck = scan.new_checkpoints()
    scan.forward(checkpoints=ck, **v)
    g = scan.backward(gy, checkpoints=ck, grad_last=gl, **v)
    for i, k in enumerate(names):
        d = rand(*v[k].shape, seed=70 + i)
        d *= 1.0 if k != "A" else v["A"].abs()
        e = 2.0 ** -8                              # e^2 of a third derivative, 2^-24 sqrt(terms) / e of rounding
        fd = (loss({**v, k: v[k] + e * d}) - loss({**v, k: v[k] - e * d})) / (2 * e)
        got = float((g[k].double() * d.double()).sum())
        assert abs(fd - got) <= 5e-3 * float(g[k].double().norm() * d.double().norm()), (k, fd, got)


def test_scan_zero_state_passes_growing_decays():
    """Decays that multiply up beyond float32's range do nothing to a state of zero."""
    from paper_2607_14394_b200 import SelectiveScan
    B, T, C, N = 1, 64, 8, 4
    v = scan_inputs(B, T, C, N, 1, F32, gated=False, strided=False)
    v["A"], v["dt"], v["dt_bias"] = torch.full((C, N), 30.0, device="cuda"), torch.full((B, T, C), 1.0, device="cuda"), None
    v["h0"], v["x"][:] = torch.zeros_like(v["h0"]), 0.0
    y, last = SelectiveScan((B, T, C), N).forward(**v)
    assert not y.any() and not last.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_expanded_and_shifted_inputs(dtype):
    """Inputs that repeat (strides of zero) and rows that begin off a vector give the bits of their dense copies."""
    from paper_2607_14394_b200 import CausalConv, SelectiveScan
    B, T, C, N = 3, 77, 64, 16
    v = scan_inputs(B, T, C, N, 1, dtype, strided=False)
    scan, conv = SelectiveScan((B, T, C), N, 1, dtype), CausalConv((B, T, C), 4, dtype)
    shifted = torch.empty(B, T, C + 1, dtype=dtype, device="cuda")[..., 1:]
    shifted.copy_(v["dt"])
    odd = dict(v, x=v["x"][:1, :1].expand(B, T, C), dt=shifted, z=v["z"][:1].expand(B, T, C), B=v["B"][:, :1].expand(B, T, 1, N))
    dense = {k: t if t is None else t.contiguous() for k, t in odd.items()}
    gy, gl = rand(B, T, C, dtype=dtype, seed=50), rand(B, C, N, seed=51)
    out = []
    for u in (odd, dense):
        ck = scan.new_checkpoints()
        y, last = scan.forward(checkpoints=ck, **u)
        g = scan.backward(gy, checkpoints=ck, grad_last=gl, **u)
        w, b = rand(C, 4, seed=1), rand(C, seed=2)
        out.append([y, last, *g.values(), *conv.forward(u["x"], w, b), *conv.backward(gy, u["dt"], w, b)])
    assert all(torch.equal(p, q) for p, q in zip(*out))


def test_far_offsets():
    """More than 2^31 elements: the last steps of a long sequence, whose states forget within a few steps, by themselves."""
    from paper_2607_14394_b200 import CausalConv, LayerNorm, SelectiveScan
    T, C, N = (1 << 31) // 1024 + 37, 1024, 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(1, T, C, dtype=BF16, device="cuda").normal_(generator=gen)
    w, b = rand(C, 4, seed=1), rand(C, seed=2)
    y, last = CausalConv((1, T, C), 4, BF16).forward(x, w, b)
    part, plast = CausalConv((1, 60, C), 4, BF16).forward(x[:, -60:], w, b, state=x[:, -63:-60])
    assert torch.equal(y[:, -60:], part) and torch.equal(last, plast)
    del y
    n = LayerNorm((T, C), -1, BF16)
    y, _, stats = n.forward(x[0], b)
    assert torch.equal(y[-50:], LayerNorm((50, C), -1, BF16).forward(x[0, -50:], b)[0])
    del y, stats
    maps = rand(1, T, 1, 2 * N, dtype=BF16, seed=3)
    A = torch.full((C, N), -200.0, device="cuda")
    dt = x                                          # softplus of a normal number and the bias: 0.3 and more, decays of e^-60
    bias = torch.full((C,), 4.0, device="cuda")
    y, last = SelectiveScan((1, T, C), N, 1, BF16).forward(x, dt, A, maps[..., :N], maps[..., N:], dt_bias=bias)
    part, plast = SelectiveScan((1, 40, C), N, 1, BF16).forward(x[:, -40:], dt[:, -40:], A, maps[:, -40:, :, :N], maps[:, -40:, :, N:], dt_bias=bias)
    assert torch.equal(y[:, -20:], part[:, -20:]) and torch.equal(last, plast)


# ------------------------------------------------------------------------------------------------ the gradients' norm
def grads_like(seed=0):
    g = [rand(5, 7, seed=seed), rand(4097, dtype=BF16, seed=seed + 1, scale=3.0), torch.view_as_complex(rand(33, 9, 2, seed=seed + 2)), rand(1, seed=seed + 3),
         rand(0, 4, seed=seed + 4), rand(70001, dtype=F16, seed=seed + 5, scale=0.1), rand(3, 8192, seed=seed + 6)]
    return g


@pytest.mark.parametrize("max_norm", [0.0, 1.0, 50.0, 1e9, float("inf")])
def test_clip_against_the_statement(max_norm):
    from paper_2607_14394_b200 import GradNorm, clip_grad_norm
    g = grads_like()
    norm, want = S.clip([t.cpu().numpy() if t.is_complex() else host(t) for t in g], max_norm)
    out = [torch.full_like(t, 9.0) for t in g]
    n = GradNorm(g, out=out)
    got = n.clip(max_norm)
    assert abs(float(got) - norm) <= 2.0 ** -23 * norm and torch.equal(n.norm(), got)
    for o, r, t in zip(out, want, g):
        if t.numel():
            assert o.dtype == t.dtype
            o = torch.view_as_real(o) if o.is_complex() else o
            close(o, torch.view_as_real(torch.from_numpy(r)).numpy() if np.iscomplexobj(r) else r, "out", tol=2.0 ** -22)
    before = [t.clone() for t in g]
    assert torch.equal(clip_grad_norm({"a": g[:3], "b": [g[3], None, g[4:]]}, max_norm), got)
    assert all(torch.equal(t, o) for t, o in zip(g, out))
    if max_norm > 2 * norm:
        assert all(torch.equal(t, o) for t, o in zip(g, before))


def test_clip_of_many_tensors_and_far_values():
    from paper_2607_14394_b200 import GradNorm, clip_grad_norm
    many = [rand(1 + (37 * i) % 600, seed=i) for i in range(300)]             # more than one launch takes
    want = torch.cat([t.double() for t in many]).norm()
    copies = [t.clone() for t in many]
    got = clip_grad_norm(copies, 2.0)
    assert abs(float(got) - float(want)) <= 2.0 ** -23 * float(want)
    flat, ref = torch.cat(copies).double(), torch.cat(many).double() * (2.0 / (want + 1e-6))
    assert float((flat - ref).norm()) <= 2.0 ** -22 * float(ref.norm())
    # squares beyond and below float32's range
    for scale, dtype in ((1e30, F32), (1e30, BF16), (1e-30, F32), (1e-35, BF16)):
        t = rand(5000, seed=3, scale=scale).to(dtype)
        norm = GradNorm([t]).norm()
        assert abs(float(norm) / float(t.double().norm()) - 1) <= 2.0 ** -22
    t = rand(5000, seed=3, scale=1e37)
    clip_grad_norm([t], 1.0)
    assert abs(float(t.double().norm()) - 1.0) <= 1e-6
    t = rand(100, seed=4)
    t[7] = float("inf")
    assert float(clip_grad_norm([t], 1.0)) == float("inf") and torch.isnan(t[7]) and float(t[6]) == 0.0
    t[7] = float("inf")
    before = t.clone()
    assert float(clip_grad_norm([t], float("inf"))) == float("inf") and torch.equal(t, before)       # without a bound nothing is scaled
    t = rand(100, seed=4)
    t[7] = float("nan")
    assert torch.isnan(clip_grad_norm([t], 1.0)) and torch.isnan(t).all()
    assert float(GradNorm([]).norm()) == 0.0
    odd = rand(100001, seed=5)[1:]                                           # begins off a vector
    assert abs(float(GradNorm([odd]).norm()) / float(odd.double().norm()) - 1) <= 2.0 ** -23


def test_clip_of_more_than_2_31_elements():
    from paper_2607_14394_b200 import GradNorm
    g = torch.ones((1 << 31) + 77, dtype=BF16, device="cuda")
    g[-1] = 2.0 ** 20
    norm = GradNorm([g]).clip(2.0 ** 10)
    want = float(np.sqrt((1 << 31) + 76 + 2.0 ** 40))
    assert abs(float(norm) / want - 1) <= 2.0 ** -23
    c = 2.0 ** 10 / want
    assert abs(float(g[-1]) / (c * 2.0 ** 20) - 1) <= 2.0 ** -8 and abs(float(g[5]) / c - 1) <= 2.0 ** -8 and float(g[-2]) == float(g[5])


# ------------------------------------------------------------------------------------------------ how they are called
def every_operator(dtype=BF16, B=2, T=40, C=64, N=16):
    """[(name, a call that takes stream=, returns a list of tensors)]"""
    from paper_2607_14394_b200 import CausalConv, GradNorm, LayerNorm, SelectiveScan
    ln, conv, scan = LayerNorm((B, T, C), -1, dtype), CausalConv((B, T, C), 4, dtype), SelectiveScan((B, T, C), N, 1, dtype)
    x, w, b = rand(B, T, C, dtype=dtype, seed=1), rand(C, seed=2), rand(C, seed=3)
    cw, v, gy = rand(C, 4, seed=4), scan_inputs(B, T, C, N, 1, dtype, seed=5), rand(B, T, C, dtype=dtype, seed=30)
    rest = {k: v[k] for k in ("D", "z", "dt_bias", "h0")}
    args = (v["x"], v["dt"], v["A"], v["B"], v["C"])
    g = grads_like(40)
    out = [torch.empty_like(t) for t in g]

    def norm(stream=None):
        y, s, st = ln.forward(x, w, b, residual=gy, stream=stream)
        return [y, s, *ln.backward(gy, s, w, st, stream=stream)]

    def convolve(stream=None):
        y, last = conv.forward(x, cw, b, stream=stream)
        return [y, last, *conv.backward(gy, x, cw, b, grad_state_out=last, stream=stream)]

    def scanned(stream=None):
        if stream is None:
            ck = scan.new_checkpoints()
        else:
            with torch.cuda.stream(stream):
                ck = scan.new_checkpoints()
        y, last = scan.forward(*args, checkpoints=ck, stream=stream, **rest)
        return [y, last, *scan.backward(gy, *args, ck, grad_last=last, stream=stream, **rest).values()]

    def clipped(stream=None):
        return [GradNorm(g, out=out).clip(1.0, stream=stream), *out]

    return [("norm", norm), ("conv", convolve), ("scan", scanned), ("clip", clipped)]


def test_on_a_stream_of_their_own():
    for name, call in every_operator():
        want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        got = call(stream=side)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), name


def test_captured_and_replayed():
    for name, call in every_operator():
        want = [t.clone() for t in call()]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for t in got:
            t.zero_()
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), name


def test_two_at_once():
    """The same objects on two streams at the same time."""
    calls = every_operator(T=200, C=512)[:3]
    want = [[t.clone() for t in call()] for _, call in calls]
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(3):
        for _, call in calls:
            got.append((call(stream=a), call(stream=b)))
    torch.cuda.synchronize()
    for i, pair in enumerate(got):
        for out in pair:
            assert all(torch.equal(p, q) for p, q in zip(out, want[i % 3])), calls[i % 3][0]


def test_nothing_around_the_outputs_is_touched():
    from paper_2607_14394_b200 import CausalConv, SelectiveScan
    B, T, C, N = 2, 21, 20, 12
    for dtype in (F32, BF16):
        v = scan_inputs(B, T, C, N, 1, dtype)
        x, w, b, s = conv_inputs(B, T, C, 4, dtype, True)
        gy = rand(B, T, C, dtype=dtype, seed=9)

        def guarded(*shape, dtype=dtype):
            n = int(np.prod(shape))
            base = torch.full((n + 128,), 5.0, dtype=dtype, device="cuda")
            return base, base[64:64 + n].view(shape)

        kept = [guarded(B, T, C), guarded(B, 3, C), guarded(B, T, C), guarded(C, 4, dtype=F32), guarded(C, dtype=F32), guarded(B, 3, C)]
        conv = CausalConv((B, T, C), 4, dtype)
        conv.forward(x, w, b, state=s, out=kept[0][1], state_out=kept[1][1])
        conv.backward(gy, x, w, b, state=s, grad_x=kept[2][1], grad_weight=kept[3][1], grad_bias=kept[4][1], grad_state=kept[5][1])
        scan = SelectiveScan((B, T, C), N, 1, dtype)
        rest = {k: v[k] for k in ("D", "z", "dt_bias", "h0")}
        args = (v["x"], v["dt"], v["A"], v["B"], v["C"])
        y, last, ck = guarded(B, T, C), guarded(B, C, N, dtype=F32), guarded(scan.checkpoint_floats, dtype=F32)
        scan.forward(*args, out=y[1], h_last=last[1], checkpoints=ck[1], **rest)
        outs = {k: guarded(*s_, dtype=d) for k, s_, d in (("x", (B, T, C), dtype), ("dt", (B, T, C), dtype), ("z", (B, T, C), dtype), ("B", (B, T, 1, N), dtype),
                                                         ("C", (B, T, 1, N), dtype), ("A", (C, N), F32), ("D", (C,), F32), ("dt_bias", (C,), F32), ("h0", (B, C, N), F32))}
        scan.backward(gy, *args, ck[1], out={k: t[1] for k, t in outs.items()}, **rest)
        for base, view in kept + [y, last, ck] + list(outs.values()):
            assert (base[:64] == 5.0).all() and (base[-64:] == 5.0).all()


# ------------------------------------------------------------------------------------------------ the block and a training step
def block64(p, x, cs, h0, r, N):
    """The block in 64 bits with autograd (elementary operations, one step after the other)."""
    B, T, D = x.shape
    H, K = p["conv_weight"].shape
    mean = x.mean(-1, keepdim=True)
    n = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(-1, keepdim=True) + 1e-5) * p["norm_weight"] + p["norm_bias"]
    uz = n @ p["W_in"].t()
    seq = torch.cat([cs, uz[..., :H]], 1)
    pre = p["conv_bias"] + sum(p["conv_weight"][:, k] * seq[:, k:k + T] for k in range(K))
    u = pre * torch.sigmoid(pre)
    both = u @ p["W_x"].t()
    dt = torch.logaddexp(both[..., :r] @ p["W_dt"].t() + p["dt_bias"], torch.zeros((), dtype=x.dtype, device=x.device))
    A, h, ys = -torch.exp(p["A_log"]), h0, []
    for t in range(T):
        h = torch.exp(dt[:, t, :, None] * A) * h + (dt[:, t] * u[:, t])[..., None] * both[:, t, None, r:r + N]
        ys.append((h * both[:, t, None, r + N:]).sum(-1) + p["D"] * u[:, t])
    z = uz[..., H:]
    y = torch.stack(ys, 1) * z * torch.sigmoid(z)
    return x + y @ p["W_out"].t(), seq[:, T:], h


@pytest.mark.parametrize("T", [1, 19, 70])
def test_block_gradients_against_autograd_in_64_bits(T):
    """The whole chain in float32; the matrix products of the library in full float32 (no TF32): a few roundings of 2^-24 per
    operation over a chain of about ten, and the scan's 3e-5."""
    from paper_2607_14394_b200 import SelectiveMemory, clip_grad_norm
    B, D, H, N = 2, 24, 48, 8
    assert not torch.backends.cuda.matmul.allow_tf32
    m = SelectiveMemory(D, H, N, rank=3, dtype=F32, seed=3)
    x, state = rand(B, T, D, seed=1), (rand(B, 3, H, seed=2), rand(B, H, N, seed=3))
    go, gs = rand(B, T, D, seed=4), (rand(B, 3, H, seed=5), rand(B, H, N, seed=6))
    out, new = m.forward(x, state)
    g = m.backward(go, gs)
    p = {k: t.double().requires_grad_() for k, t in m.parameters().items()}
    leaves = [t.double().requires_grad_() for t in (x, *state)]
    ref = block64(p, *leaves, 3, N)
    loss = (ref[0] * go.double()).sum() + (ref[1] * gs[0].double()).sum() + (ref[2] * gs[1].double()).sum()
    loss.backward()
    for a, b, name in zip((out, *new), ref, ("out", "conv_state", "h")):
        close(a, host(b), name, 5e-5)
    for k in m.NAMES:
        close(g[k], host(p[k].grad), k, 1e-4)
    for k, t in zip(("x", "conv_state", "h0"), leaves):
        close(g[k], host(t.grad), k, 1e-4)
    # a training step: the parameters' gradients, clipped together
    grads = {k: g[k] for k in m.NAMES}
    want = torch.sqrt(sum((t.double() ** 2).sum() for t in grads.values()))
    got = clip_grad_norm(grads, 0.5)
    assert abs(float(got) / float(want) - 1) <= 2.0 ** -22
    after = torch.sqrt(sum((t.double() ** 2).sum() for t in grads.values()))
    assert abs(float(after) / 0.5 - 1) <= 1e-5


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_block_frame_by_frame(dtype):
    """step() against the whole history: in float32 to 32-bit rounding of the chain; in bfloat16 every one of the chain's eight
    stored tensors may round the other way (2^-8 each, averaged over many)."""
    from paper_2607_14394_b200 import SelectiveMemory
    B, T, D, H = 3, 11, 64, 128
    m = SelectiveMemory(D, H, 16, dtype=dtype, seed=5)
    x = rand(B, T, D, dtype=dtype, seed=1)
    out, (cs, h) = m.forward(x, m.new_state(B), training=False)
    state = m.new_state(B)
    steps = torch.stack([m.step(x[:, t], state) for t in range(T)], 1)
    tol = 5e-5 if dtype is F32 else 8 * 2.0 ** -8
    close(steps, host(out), "out", tol)
    close(state[1], host(h), "h", tol)
    close(state[0], host(cs), "conv_state", tol)
    with pytest.raises(RuntimeError):
        m.backward(out)
    # a ragged batch: every entry as by itself
    ln = torch.tensor([11, 0, 5], dtype=torch.int32, device="cuda")
    ragged, (cs, h) = m.forward(x, m.new_state(B), lengths=ln, training=False)
    alone, (_, h5) = m.forward(x[2:, :5].contiguous(), m.new_state(1), training=False)
    close(ragged[2:, :5], host(alone), "ragged", tol)
    close(h[2:], host(h5), "ragged h", tol)
    assert not h[1].any() and not cs[1].any()


def test_network_gradients_are_clipped_in_the_backward_pass():
    from paper_2607_14394_b200 import FNO
    net = FNO((16, 32), (4, 4), B=2, C_a=3, C_u=1, width=8, layers=2, seed=1)
    a, gu = rand(2, 3, 16, 32, seed=1), rand(2, 1, 16, 32, seed=2)
    net.forward(a)
    plain = net.backward(gu, need_grad_a=True)
    net.forward(a)
    clipped = net.backward(gu, need_grad_a=True, max_norm=0.25)
    flat = lambda g: [g["P_w"], g["P_b"], *g["W"], *g["Wb"], g["Q_w"], g["Q_b"]]
    norm = torch.sqrt(sum((t.abs().double() ** 2).sum() for t in flat(plain)))
    assert abs(float(clipped["norm"]) / float(norm) - 1) <= 2.0 ** -22
    c = 0.25 / (float(norm) + 1e-6)
    for p, q in zip(flat(plain), flat(clipped)):
        assert float((q - p * c).abs().max()) <= 2.0 ** -21 * c * float(p.abs().max())
    assert torch.equal(plain["a"], clipped["a"])
