"""Recurrent-memory operators on the GPU against the float64 statement.

Tolerances (relative L2 of a whole output).  A stored value is rounded once: at most half a unit in the last place,
2^-24 of its size in float32, 2^-8 in bfloat16, 2^-11 in float16 (subnormals apart).  The 32-bit arithmetic in front of
it - sums of up to a few thousand terms, states carried over a few hundred steps with a relative error of about 1e-7 per
step - stays within the 1e-5 that the library's other kernels keep to.  So: 1e-5 for float32, 1e-5 + half a unit for the
16-bit types.
"""
import numpy as np
import pytest

from oracle import memory_oracle as M

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
TOL = {F32: 1e-5, BF16: 1e-5 + 2.0 ** -8, F16: 1e-5 + 2.0 ** -11}
EPS = 1e-6


def rand(*shape, dtype=F32, seed=0, scale=1.0, shift=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=gen) * scale + shift).to(dtype)


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, want, dtype, what=""):
    got = host(got)
    assert np.isfinite(got).all() == np.isfinite(want).all(), what
    assert got.shape == want.shape, (what, got.shape, want.shape)
    e = M.rel_l2(got, want)
    assert e <= TOL[dtype], (what, e)


def three(shape, dim):
    return int(np.prod(shape[:dim])), shape[dim], int(np.prod(shape[dim + 1:]))


# ------------------------------------------------------------------------------------------------ norm
NORM_SHAPES = [
    ((1, 1), 1), ((1, 7), 1), ((3, 64), 1), ((5, 250), 1), ((4, 256), 1), ((9, 511), 1), ((2, 1000), 1), ((700, 1024), 1),
    ((3, 2048), 1), ((2, 4100), 1), ((3, 8192), 1), ((2, 16390), 1), ((2, 3, 40), 2),
    ((1, 4, 64), 1), ((2, 20, 30, 7), 1), ((2, 20, 128), 1), ((1, 32, 1000), 1), ((2, 33, 257), 1), ((1, 128, 64), 1),
    ((2, 150, 90), 1), ((3, 1, 5), 1), ((4, 6000), 1), ((3, 8190), 1), ((1, 16, 2052), 1), ((1, 5, 200000), 1),
]


@pytest.mark.parametrize("shape,dim", NORM_SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm_forward_and_backward(shape, dim, dtype, residual):
    from paper_2607_14394_b200 import RmsNorm
    x, r = rand(*shape, dtype=dtype, seed=1), rand(*shape, dtype=dtype, seed=2, scale=2.0) if residual else None
    gy, gs = rand(*shape, dtype=dtype, seed=3), rand(*shape, dtype=dtype, seed=4) if residual else None
    w = rand(shape[dim], seed=5, scale=0.2, shift=1.0)
    n = RmsNorm(shape, dim, dtype, EPS)
    v = three(shape, dim)
    as3 = lambda t: None if t is None else host(t).reshape(v)
    y, s, rstd = n.forward(x, w, residual=r)
    ry, rs, rrstd = M.rms_norm(as3(x), host(w), EPS, as3(r))
    close(y.view(v), ry, dtype, "y")
    close(s.view(v), rs, dtype, "s")
    close(rstd.view(v[0], v[2]), rrstd, F32, "rstd")
    # backward of the unrounded sum: s, and what rounding took from it, which the returned rstd carries
    gx, gw = n.backward(gy, s, w, rstd, grad_s=gs)
    rgx, rgw = M.rms_norm_backward(as3(gy), rs, host(w), rrstd, as3(gs))
    # with one channel (and no eps) grad_x is a difference of equal terms: held to the size of what is subtracted
    size = np.linalg.norm(as3(gy) * host(w)[None, :, None] * host(rstd).reshape(v[0], 1, v[2]))
    assert np.linalg.norm(host(gx).reshape(v) - rgx) <= TOL[dtype] * max(np.linalg.norm(rgx), size)
    close(gw, rgw, F32, "grad_weight") if np.prod(v[:1] + v[2:]) > 1 else None
    again = n.backward(gy, s, w, rstd, grad_s=gs)
    assert torch.equal(gx, again[0]) and torch.equal(gw, again[1])
    only, none = n.backward(gy, s, w, rstd, grad_s=gs, need_grad_weight=False)
    assert none is None and torch.equal(only, gx)
    # ... and of the rounded sum where the low part was not kept
    gx, gw = n.backward(gy, s, w, rstd.clone(), grad_s=gs)
    rgx, rgw = M.rms_norm_backward(as3(gy), as3(s), host(w), host(rstd).reshape(v[0], v[2]), as3(gs))
    assert np.linalg.norm(host(gx).reshape(v) - rgx) <= TOL[dtype] * max(np.linalg.norm(rgx), size)
    close(gw, rgw, F32, "grad_weight") if np.prod(v[:1] + v[2:]) > 1 else None
    assert torch.equal(n.forward(x, w, residual=r, need_backward=False)[0], y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [64, 1000, 4096])
def test_norm_in_place(dtype, c):
    from paper_2607_14394_b200 import RmsNorm
    x, r, w = rand(6, c, dtype=dtype, seed=1), rand(6, c, dtype=dtype, seed=2), rand(c, seed=3)
    n = RmsNorm((6, c), -1, dtype)
    y, s, _ = n.forward(x, w, residual=r)
    r2, x2 = r.clone(), x.clone()
    n.forward(x2, w, residual=r2, sum_out=r2, out=x2)
    assert torch.equal(r2, s) and torch.equal(x2, y)


def test_norm_gradient_against_differences():
    from paper_2607_14394_b200 import RmsNorm
    for shape in [(3, 40), (2, 20, 33)]:
        n = RmsNorm(shape, 1, F32, 1e-3)
        x, gy, w = rand(*shape, seed=1), rand(*shape, seed=2), rand(shape[1], seed=3, shift=1.0)
        d = rand(*shape, seed=4)
        _, s, rstd = n.forward(x, w)
        gx, _ = n.backward(gy, s, w, rstd)
        h = 2.0 ** -6                     # central difference: h^2 of a third derivative, 2^-24 / h of rounding
        up, down = n.forward(x + h * d, w)[0], n.forward(x - h * d, w)[0]
        fd = float(((up.double() - down.double()) / (2 * h) * gy.double()).sum())
        got = float((gx.double() * d.double()).sum())
        assert abs(fd - got) <= 5e-3 * float(gx.double().norm() * d.double().norm()), (fd, got)


def test_norm_special_values():
    from paper_2607_14394_b200 import RmsNorm
    n = RmsNorm((4, 200), -1, F32)
    x, w = rand(4, 200, seed=1), torch.ones(200, device="cuda")
    x[1] = 0.0
    x[2, 5] = float("nan")
    y, _, rstd = n.forward(x, w)
    assert torch.equal(y[1], torch.zeros_like(y[1])) and torch.isnan(y[2]).all()
    assert torch.isfinite(y[0]).all() and torch.isfinite(y[3]).all()        # rows do not touch each other
    assert abs(float(rstd[1]) - EPS ** -0.5) < 1e-3 * EPS ** -0.5


def fp8_rows_ok(q, scale, y):
    """q is the nearest 8-bit number of y / scale (both within 32-bit rounding), scale the block's amax / 448."""
    rows, k = y.shape
    _, want = M.quantize_rows(y)
    assert np.all(np.abs(host(scale) - want) <= 1e-5 * want)
    z = y / host(scale).T[:, np.arange(k) // 128]
    got = host(q)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(z), 1e-30))), -6) - 3)
    assert np.all(np.abs(got - z) <= step * 0.5 + 2e-5 * np.abs(z) + 1e-12)
    assert np.isin(np.abs(got), M.e4m3_values()).all()


@pytest.mark.parametrize("rows,c", [(1, 1), (2, 100), (3, 128), (5, 129), (4, 1000), (1, 2048), (17, 1024), (3, 4097),
                                    (2, 8192), (2, 20000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_and_quantise_to_8_bits(rows, c, dtype):
    from paper_2607_14394_b200 import RmsNorm, quantize_fp8
    x, r, w = rand(rows, c, dtype=dtype, seed=1), rand(rows, c, dtype=dtype, seed=2), rand(c, seed=3)
    n = RmsNorm((rows, c), -1, dtype, EPS)
    q, scale, s = n.forward_fp8(x, w, residual=r)
    y, rs, _ = M.rms_norm(host(x)[..., None], host(w), EPS, host(r)[..., None])
    fp8_rows_ok(q, scale, y[..., 0])
    close(s, rs[..., 0], dtype)
    q, scale = quantize_fp8(x)
    fp8_rows_ok(q, scale, host(x))
    wide = rand(rows, c + 24, dtype=dtype, seed=4)       # rows of a wider tensor
    q, scale = quantize_fp8(wide[:, 8:8 + c])
    fp8_rows_ok(q, scale, host(wide[:, 8:8 + c]))


def test_quantise_special_values():
    from paper_2607_14394_b200 import quantize_fp8
    x = rand(4, 300, seed=1)
    x[0, :128] = 0.0
    x[1, 130] = float("nan")
    x[2, 3] = float("inf")
    x[3] = torch.finfo(F32).min
    q, s = quantize_fp8(x)
    assert torch.equal(q[0, :128].float(), torch.zeros(128, device="cuda")) and float(s[0, 0]) > 0
    nan = torch.isnan(q.float())
    assert nan[1, 130] and int(nan[1].sum()) == 1
    assert torch.isinf(s[0, 2]) and torch.isfinite(s[1:, 2]).all()
    assert torch.equal(q[3].float(), torch.full((300,), -448.0, device="cuda"))


@pytest.mark.parametrize("n,k", [(1, 1), (128, 128), (130, 300), (300, 64), (257, 1000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantise_weight(n, k, dtype):
    from paper_2607_14394_b200 import quantize_fp8_weight
    w = rand(n, k, dtype=dtype, seed=7)
    q, s = quantize_fp8_weight(w)
    _, want = M.quantize_blocks(host(w))
    assert s.shape == want.shape and np.all(np.abs(host(s) - want) <= 1e-6 * want)
    z = host(w) / host(s)[np.arange(n) // 128][:, np.arange(k) // 128]
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(z), 1e-30))), -6) - 3)
    assert np.all(np.abs(host(q) - z) <= step * 0.5 + 2e-5 * np.abs(z))


# ------------------------------------------------------------------------------------------------ 8-bit product
@pytest.mark.parametrize("m,n,k", [
    (1, 1, 1), (1, 128, 128), (3, 200, 100), (4, 4096, 2048), (17, 130, 1000), (32, 64, 256), (33, 64, 256), (64, 500, 4096),
    (65, 129, 272), (128, 256, 384), (129, 257, 130), (200, 1111, 1360), (1000, 96, 640), (513, 640, 2049), (2, 70, 9000),
    (300, 2304, 512), (1500, 1500, 128), (5, 20000, 16), (4200, 333, 256),
    (16, 96, 4096), (48, 1024, 2048), (100, 640, 4096), (2250, 2100, 650), (4865, 1000, 200), (2304, 2304, 1024), (2305, 2309, 16),
])
@pytest.mark.parametrize("dtype", TYPES)
def test_matmul(m, n, k, dtype):
    from paper_2607_14394_b200 import Fp8Linear, quantize_fp8
    q, s = quantize_fp8(rand(m, k, seed=m))
    lin = Fp8Linear.from_weight(rand(n, k, seed=n + 1, scale=k ** -0.5), dtype)
    out = lin(q, s)
    want = M.matmul_fp8(host(q), host(s), host(lin.weight), host(lin.weight_scale))
    # a sum of k products: its rounding errors are relative to the terms, not to what is left of them
    size = np.linalg.norm(M.matmul_fp8(np.abs(host(q)), host(s), np.abs(host(lin.weight)), host(lin.weight_scale)))
    err = np.linalg.norm(host(out) - want)
    assert err <= (TOL[dtype] - 1e-5) * np.linalg.norm(want) + 1e-6 * size, (err, np.linalg.norm(want), size)
    assert torch.equal(out, lin(q, s)) and lin.status() == 0


@pytest.mark.parametrize("m,n,k", [(4, 300, 200), (150, 300, 200)])
def test_matmul_strided_rows_and_neighbours(m, n, k):
    """Operands and output inside larger buffers: nothing beside them is read into the result or written."""
    from paper_2607_14394_b200 import Fp8Linear, quantize_fp8
    from paper_2607_14394_b200.memory import FP8
    q, s = quantize_fp8(rand(m, k, seed=1))
    lin = Fp8Linear.from_weight(rand(n, k, seed=2), F32)
    plain = lin(q, s)
    big = torch.full((m + 2, 512), 0x7f, dtype=torch.uint8, device="cuda").view(FP8)     # NaN around the operand
    big[1:1 + m, 64:64 + k] = q
    out = torch.full((m + 2, n + 11), 7.0, device="cuda")
    got = lin(big[1:1 + m, 64:64 + k], s, out=out[1:1 + m, 5:5 + n])
    assert torch.equal(got, plain)
    out[1:1 + m, 5:5 + n] = 7.0
    assert torch.equal(out, torch.full_like(out, 7.0))
    wide = torch.full((n, 256), 0x7f, dtype=torch.uint8, device="cuda").view(FP8)
    wide[:, :k] = lin.weight
    assert torch.equal(Fp8Linear(wide[:, :k], lin.weight_scale, F32)(q, s), plain)


def test_matmul_special_values_stay_in_their_row():
    from paper_2607_14394_b200 import Fp8Linear, quantize_fp8
    x = rand(40, 256, seed=1)
    x[3, 7] = float("nan")
    q, s = quantize_fp8(x)
    lin = Fp8Linear.from_weight(rand(64, 256, seed=2), F32)
    out = lin(q, s)
    assert torch.isnan(out[3]).all()
    rest = [i for i in range(40) if i != 3]
    assert torch.isfinite(out[rest]).all()


# ------------------------------------------------------------------------------------------------ recurrence
SCAN_SHAPES = [
    # (outer, L, inner)
    (1, 1, 8), (4, 1, 2048), (3, 2, 5), (2, 8, 64), (5, 9, 12), (3, 33, 20), (2, 64, 64), (2, 65, 64), (1, 129, 36), (2, 300, 100),
    (1, 1000, 7), (2, 513, 260), (40, 5, 3), (1, 2500, 64),
    (1, 1, 1), (7, 1, 1), (300, 2, 1), (1000, 16, 1), (515, 17, 1), (1000, 30, 1), (130, 64, 1), (70, 100, 1), (33, 512, 1),
    (9, 513, 1), (3, 2000, 1),
    (50, 7, 1), (200, 8, 1), (131, 9, 1), (64, 15, 1), (20, 127, 1), (11, 255, 1), (5, 504, 1), (5, 505, 1), (4, 511, 1),
    (3, 1016, 1), (2, 1009, 1), (1, 9001, 1), (2, 3000, 20), (1, 4099, 3),
    (3, 256, 40), (3, 257, 40), (2, 511, 33), (2, 513, 5), (1, 5000, 132), (700, 300, 20), (5, 66, 7),
]


def scan_case(outer, L, inner, dtype, gate, ragged, seed=0):
    shape = (outer, L) if inner == 1 else (outer, L, inner)
    v, gh = rand(*shape, dtype=dtype, seed=seed + 1), rand(*shape, dtype=dtype, seed=seed + 2)
    g = rand(*shape, dtype=F32, seed=seed + 3, scale=1.5, shift=1.5)
    g = (torch.sigmoid(g) if gate == "decay" else g).to(dtype)
    state = (outer,) if inner == 1 else (outer, inner)
    h0, gl = rand(*state, seed=seed + 4), rand(*state, seed=seed + 5)
    lengths = None
    if ragged:
        rng = np.random.default_rng(seed + 6)
        n = rng.integers(0, L + 1, outer)
        n[0] = 0
        n[-1] = L
        lengths = torch.from_numpy(n.astype(np.int32)).cuda()
    return shape, v, g, gh, h0, gl, lengths


def scan_reference(outer, L, inner, v, g, gh, h0, gl, lengths, gate):
    d = (outer, L, inner)
    a = [host(t).reshape(d) for t in (v, g, gh)]
    z0, zl = host(h0).reshape(outer, inner), host(gl).reshape(outer, inner)
    n = None if lengths is None else lengths.cpu().numpy()
    h, last, _ = M.gated_scan(a[0], a[1], z0, n, gate)
    return h, last, *M.gated_scan_backward(a[2], a[0], a[1], z0, n, zl, gate)


@pytest.mark.parametrize("outer,L,inner", SCAN_SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gate,ragged", [("sigmoid", False), ("sigmoid", True), ("decay", True)])
def test_scan_forward_and_backward(outer, L, inner, dtype, gate, ragged):
    from paper_2607_14394_b200 import GatedScan
    shape, v, g, gh, h0, gl, lengths = scan_case(outer, L, inner, dtype, gate, ragged)
    plan = GatedScan(shape, 1, dtype, gate)
    ck = plan.new_checkpoints()
    h, last = plan.forward(v, g, h0, lengths=lengths, checkpoints=ck)
    gv, gg, g0 = plan.backward(gh, v, g, ck, h0, lengths=lengths, grad_last=gl)
    want = scan_reference(outer, L, inner, v, g, gh, h0, gl, lengths, gate)
    d = (outer, L, inner)
    for got, ref, kind, what in [(h.view(d), want[0], dtype, "h"), (last.view(outer, inner), want[1], F32, "h_last"),
                                 (gv.view(d), want[2], dtype, "grad_v"), (gg.view(d), want[3], dtype, "grad_g"),
                                 (g0.view(outer, inner), want[4], F32, "grad_h0")]:
        close(got, ref, kind, what)
    again = plan.forward(v, g, h0, lengths=lengths)
    assert torch.equal(again[0], h) and torch.equal(again[1], last)
    assert all(torch.equal(a, b) for a, b in zip(plan.backward(gh, v, g, ck, h0, lengths=lengths, grad_last=gl), (gv, gg, g0)))
    assert plan.status() == 0


@pytest.mark.parametrize("L", [9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257])
@pytest.mark.parametrize("outer,inner", [(5, 12), (3, 129), (300, 4), (7, 516)])
@pytest.mark.parametrize("dtype,gate,ragged", [(F32, "sigmoid", True), (torch.bfloat16, "decay", False), (torch.float16, "sigmoid", False)])
def test_scan_at_the_ends_of_the_tiles(outer, L, inner, dtype, gate, ragged):
    """Lengths on both sides of every tile's, channels by fours and one by one."""
    test_scan_forward_and_backward(outer, L, inner, dtype, gate, ragged)


def test_scan_without_states():
    from paper_2607_14394_b200 import GatedScan
    for shape in [(3, 70, 20), (40, 30), (5, 600)]:
        plan = GatedScan(shape, 1)
        v, g, gh = rand(*shape, seed=1), rand(*shape, seed=2), rand(*shape, seed=3)
        zero = torch.zeros(plan.state_shape, device="cuda")
        ck, ck2 = plan.new_checkpoints(), plan.new_checkpoints()
        a, b = plan.forward(v, g, checkpoints=ck), plan.forward(v, g, zero, checkpoints=ck2)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        x, y = plan.backward(gh, v, g, ck, need_grad_h0=False), plan.backward(gh, v, g, ck2, zero, grad_last=zero)
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and x[2] is None


def test_scan_of_no_steps_passes_the_state_on():
    from paper_2607_14394_b200 import GatedScan
    plan = GatedScan((3, 0, 8), 1)
    e, h0 = torch.empty((3, 0, 8), device="cuda"), rand(3, 8, seed=1)
    h, last = plan.forward(e, e, h0)
    assert h.numel() == 0 and torch.equal(last, h0)
    _, _, g0 = plan.backward(e, e, e, plan.new_checkpoints(), h0, grad_last=h0)
    assert torch.equal(g0, h0)
    plan = GatedScan((0, 5, 8), 1)
    e = torch.empty((0, 5, 8), device="cuda")
    plan.forward(e, e)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,L,D", [(2, 70, 64), (3, 300, 33), (2, 1, 40)])
def test_scan_of_strided_halves(dtype, B, L, D):
    """v and g as the halves of one projection's output, their gradients written into halves of one buffer."""
    from paper_2607_14394_b200 import GatedScan
    vg, gh = rand(B, L, 2 * D, dtype=dtype, seed=1), rand(B, L, D, dtype=dtype, seed=2)
    plan = GatedScan((B, L, D), 1, dtype)
    v, g = vg[..., :D], vg[..., D:]
    ck, ck2 = plan.new_checkpoints(), plan.new_checkpoints()
    h, last = plan.forward(v, g, checkpoints=ck)
    h2, last2 = plan.forward(v.contiguous(), g.contiguous(), checkpoints=ck2)
    # widths that are no multiple of four start the halves off a vector: other loads, the same sums
    assert torch.equal(h, h2) and torch.equal(last, last2) if D % 4 == 0 else M.rel_l2(host(h), host(h2)) < TOL[dtype]
    buf = torch.full((B, L, 2 * D + 4), 7.0, dtype=dtype, device="cuda")
    gv, gg, _ = plan.backward(gh, v, g, ck, grad_v=buf[..., :D], grad_g=buf[..., D:2 * D])
    rv, rg, _ = plan.backward(gh, v.contiguous(), g.contiguous(), ck2)
    assert M.rel_l2(host(gv), host(rv)) <= TOL[dtype] and M.rel_l2(host(gg), host(rg)) <= TOL[dtype]
    assert torch.equal(buf[..., 2 * D:], torch.full_like(buf[..., 2 * D:], 7.0))


@pytest.mark.parametrize("dim", [0, 1, 2, 3])
def test_scan_along_any_axis(dim):
    from paper_2607_14394_b200 import GatedScan
    shape = (6, 10, 4, 9)
    v, g = rand(*shape, seed=1), rand(*shape, seed=2)
    h, last = GatedScan(shape, dim).forward(v, g)
    d = three(shape, dim)
    want, wl, _ = M.gated_scan(host(v).reshape(d), host(g).reshape(d))
    close(h.view(d), want, F32)
    close(last.view(d[0], d[2]), wl, F32)
    # a broadcast input: one entry's gates for all of them
    if dim > 0:
        one = g[:1].expand(shape)
        try:
            h, _ = GatedScan(shape, dim).forward(v.clone()[:1].expand(shape), one)
        except ValueError:
            assert dim > 1          # the outer dimensions no longer lie together
            return
        want, _, _ = M.gated_scan(host(v[:1].expand(shape)).reshape(d), host(one).reshape(d))
        close(h.view(d), want, F32)


@pytest.mark.parametrize("shape", [(3, 200, 40), (3, 200, 5), (40, 30), (3, 700)])
@pytest.mark.parametrize("poison", [float("nan"), float("inf"), torch.finfo(F32).min])
def test_scan_does_not_see_what_lies_behind_a_length(shape, poison):
    from paper_2607_14394_b200 import GatedScan
    outer, L = shape[:2]
    lengths = torch.tensor([(37 * i) % (L + 1) for i in range(outer)], dtype=torch.int32, device="cuda")
    v, g, gh = (rand(*shape, seed=k) for k in (1, 2, 3))
    plan = GatedScan(shape, 1)
    ck = plan.new_checkpoints()
    clean = [*plan.forward(v, g, lengths=lengths, checkpoints=ck), *plan.backward(gh, v, g, ck, lengths=lengths)]
    for t in (v, g, gh):
        for o in range(outer):
            t[o, int(lengths[o]):] = poison
    dirty = [*plan.forward(v, g, lengths=lengths, checkpoints=ck), *plan.backward(gh, v, g, ck, lengths=lengths)]
    for a, b in zip(clean, dirty):
        assert torch.isfinite(b).all() and torch.equal(a, b)
    for o in range(outer):
        assert not clean[0][o, int(lengths[o]):].any() and not clean[2][o, int(lengths[o]):].any()


def test_scan_extreme_gates():
    from paper_2607_14394_b200 import GatedScan
    plan = GatedScan((2, 300, 8), 1)
    v, g, h0 = rand(2, 300, 8, seed=1), torch.full((2, 300, 8), float("inf"), device="cuda"), rand(2, 8, seed=2)
    h, last = plan.forward(v, g, h0)                      # a = 1: the state stays
    assert torch.equal(last, h0) and torch.equal(h, h0[:, None].expand_as(h))
    h, last = plan.forward(v, -g, h0)                     # a = 0: the input passes through
    assert torch.equal(h, v)
    g = rand(2, 300, 8, seed=3, scale=60.0)               # saturated gates both ways
    want, wl, _ = M.gated_scan(host(v), host(g), host(h0))
    h, last = plan.forward(v, g, h0)
    close(h, want, F32)
    # a NaN spoils the rest of its own sequence and channel alone
    v[0, 100, 3] = float("nan")
    h, _ = plan.forward(v, rand(2, 300, 8, seed=4), h0)
    bad = torch.isnan(h)
    assert bad[0, 100:, 3].all() and int(bad.sum()) == 200


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_step_by_step_equals_the_whole(dtype):
    """A history read at once, then frames one by one with the state in place, against the whole at once."""
    from paper_2607_14394_b200 import GatedScan
    v, g = rand(3, 40, 100, dtype=dtype, seed=1), rand(3, 40, 100, dtype=dtype, seed=2)
    h, last = GatedScan((3, 40, 100), 1, dtype).forward(v, g)
    parts, state = [], torch.zeros(3, 100, device="cuda")
    first, one = GatedScan((3, 30, 100), 1, dtype), GatedScan((3, 1, 100), 1, dtype)
    parts.append(first.forward(v[:, :30], g[:, :30], state, h_last=state)[0])
    for t in range(30, 40):
        parts.append(one.forward(v[:, t:t + 1], g[:, t:t + 1], state, h_last=state)[0])
    close(torch.cat(parts, 1), host(h), dtype)
    close(state, host(last), F32)


def test_scan_gradients_against_differences():
    from paper_2607_14394_b200 import GatedScan
    for shape in [(2, 50, 12), (20, 30)]:
        plan = GatedScan(shape, 1)
        v, g, gh, dv, dg = (rand(*shape, seed=k) for k in range(5))
        ck = plan.new_checkpoints()
        plan.forward(v, g, checkpoints=ck)
        gv, gg, _ = plan.backward(gh, v, g, ck)
        e = 2.0 ** -6
        for d, grad, f in [(dv, gv, lambda s: plan.forward(v + s * dv, g)[0]), (dg, gg, lambda s: plan.forward(v, g + s * dg)[0])]:
            fd = float(((f(e).double() - f(-e).double()) / (2 * e) * gh.double()).sum())
            got = float((grad.double() * d.double()).sum())
            assert abs(fd - got) <= 5e-3 * float(grad.double().norm() * d.double().norm())


def test_long_offsets_pass_32_bits():
    """Rows whose first elements lie more than 2^31 elements into the tensors."""
    from paper_2607_14394_b200 import GatedScan, RmsNorm
    outer, L, inner = 70000, 16, 2000                                          # 2.24e9 elements of 16 bits
    v = torch.zeros((outer, L, inner), dtype=BF16, device="cuda")
    v[-1] = rand(L, inner, dtype=BF16, seed=1)
    plan = GatedScan(v.shape, 1, BF16, "decay")
    out = torch.empty_like(v)
    h, last = plan.forward(v, v, out=out)
    want, wl, _ = M.gated_scan(host(v[-1:]), host(v[-1:]), gate="decay")
    close(h[-1:], want, BF16)
    assert not h[:5].any()
    n = RmsNorm((outer * L, inner), -1, BF16)
    y, _, _ = n.forward(v.view(outer * L, inner), torch.ones(inner, device="cuda"), out=out.view(outer * L, inner))
    want, _, _ = M.rms_norm(host(v[-1])[..., None], np.ones(inner), EPS)
    close(y[-L:], want[..., 0], BF16)


# ------------------------------------------------------------------------------------------------ in use
def test_arguments_are_checked():
    from paper_2607_14394_b200 import Fp8Linear, GatedScan, RmsNorm, quantize_fp8
    x, w = rand(4, 64), rand(64)
    n = RmsNorm((4, 64), -1)
    for bad in (dict(x=x.cpu()), dict(x=x.half()), dict(x=rand(4, 65)), dict(x=rand(64, 4).t()), dict(weight=rand(63)),
                dict(weight=w.double()), dict(residual=rand(3, 64))):
        with pytest.raises(ValueError):
            n.forward(**{**dict(x=x, weight=w), **bad})
    with pytest.raises(ValueError):
        RmsNorm((2, 8, 30), 1, F32).forward_fp8(rand(2, 8, 30), rand(8))
    for bad in (dict(dtype=torch.float64), dict(dim=2)):
        with pytest.raises(ValueError):
            RmsNorm(**{**dict(shape=(4, 64)), **bad})
    q, s = quantize_fp8(x)
    lin = Fp8Linear.from_weight(rand(32, 64))
    for bad in (dict(x=x), dict(x_scale=s[:, :3]), dict(x=q[:, :48]), dict(x_scale=s.double()),
                dict(out=torch.empty(4, 32, device="cuda"))):
        with pytest.raises(ValueError):
            lin.forward(**{**dict(x=q, x_scale=s), **bad})
    plan = GatedScan((2, 10, 8), 1)
    v = rand(2, 10, 8)
    for bad in (dict(v=rand(2, 10, 9)), dict(g=v.half()), dict(g=rand(2, 10, 16)[..., :8]), dict(h0=rand(2, 9)),
                dict(lengths=torch.ones(2, device="cuda")), dict(v=rand(2, 8, 10).transpose(1, 2)),
                dict(checkpoints=torch.empty(3, device="cuda"))):
        with pytest.raises(ValueError):
            plan.forward(**{**dict(v=v, g=v), **bad})
    with pytest.raises(ValueError):
        GatedScan((2, 10, 8), 1, gate="relu")


def test_calls_follow_the_stream():
    """On a stream of their own, behind work that is still running there."""
    from paper_2607_14394_b200 import Fp8Linear, GatedScan, RmsNorm
    st = torch.cuda.Stream()
    w, x = rand(512, seed=1), rand(300, 512, dtype=BF16, seed=2)
    n, lin = RmsNorm((300, 512), -1, BF16), Fp8Linear.from_weight(rand(256, 512, seed=3), BF16)
    scan = GatedScan((3, 100, 128), 1, BF16)

    def chain(x_, **k):
        q, s, _ = n.forward_fp8(x_, w, **k)
        vg = lin.forward(q, s, **k).view(3, 100, 256)
        return scan.forward(vg[..., :128], vg[..., 128:], **k)[0]

    want = chain(x)
    torch.cuda.synchronize()
    late = torch.zeros_like(x)
    big = torch.empty(1 << 28, device="cuda")
    with torch.cuda.stream(st):
        for _ in range(20):
            big.mul_(1.0001)
        late.copy_(x)
    for how in (st, st.cuda_stream):
        got = chain(late, stream=how)
        st.synchronize()
        assert torch.equal(got, want)


def test_calls_replay_in_a_graph():
    from paper_2607_14394_b200 import Fp8Linear, GatedScan, RmsNorm
    w, x = rand(256, seed=1), rand(2 * 900, 256, dtype=BF16, seed=2)
    n, lin = RmsNorm((1800, 256), -1, BF16), Fp8Linear.from_weight(rand(128, 256, seed=3), BF16)
    scan = GatedScan((2, 900, 64), 1, BF16)

    def chain():
        q, s, _ = n.forward_fp8(x, w)
        vg = lin.forward(q, s).view(2, 900, 128)
        return scan.forward(vg[..., :64], vg[..., 64:])

    chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, last = chain()
    for seed in (5, 6, 7):
        x.copy_(rand(2 * 900, 256, dtype=BF16, seed=seed))
        graph.replay()
        a = h.clone(), last.clone()
        b = chain()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert lin.status() == 0


def test_field_memory_matches_the_statement():
    """The trainable block on a field with a time axis of 30, forward and backward."""
    from paper_2607_14394_b200 import FieldMemory
    B, C, grid = 2, 20, (6, 8, 30)
    blk = FieldMemory(B, C, grid, seed=3)
    shape = (B, C) + grid
    x, go, h0 = rand(*shape, seed=1), rand(*shape, seed=2), rand(B, C, 6, 8, seed=3)
    out, last = blk.forward(x, h0)
    gr = blk.backward(go)
    P = 6 * 8 * 30
    p = {k: host(getattr(blk, k)) for k in ("W_v", "W_g", "W_o", "b_v", "b_g", "weight")}
    x3, go3 = host(x).reshape(B, C, P), host(go).reshape(B, C, P)
    y, s, rstd = M.rms_norm(x3, p["weight"], EPS)
    lin = lambda W, t: np.einsum("oi,bip->bop", W, t)
    rows = lambda t: t.reshape(B * C * 48, 30, 1)
    v, g = lin(p["W_v"], y) + p["b_v"][None, :, None], lin(p["W_g"], y) + p["b_g"][None, :, None]
    h, wl, _ = M.gated_scan(rows(v), rows(g), host(h0).reshape(-1, 1))
    h = h.reshape(B, C, P)
    close(out.view(B, C, P), x3 + lin(p["W_o"], h), F32, "out")
    close(last.view(-1, 1), wl, F32, "h_last")
    gh = lin(p["W_o"].T, go3)
    gv, gg, g0 = M.gated_scan_backward(rows(gh), rows(v), rows(g), host(h0).reshape(-1, 1))
    gv, gg = gv.reshape(B, C, P), gg.reshape(B, C, P)
    gx, gw = M.rms_norm_backward(lin(p["W_v"].T, gv) + lin(p["W_g"].T, gg), s, p["weight"], rstd, go3)
    outer = lambda a, b: np.einsum("bop,bip->oi", a, b)
    want = {"x": gx.reshape(shape), "weight": gw, "W_o": outer(go3, h), "W_v": outer(gv, y), "W_g": outer(gg, y),
            "b_v": gv.sum((0, 2)), "b_g": gg.sum((0, 2)), "h0": g0.reshape(B, C, 6, 8)}
    for k, ref in want.items():
        close(gr[k], ref, F32, k)


def test_rollout_memory_steps_equal_the_history():
    """A serving rollout: the history at once and frame by frame, ragged beginnings, every layer in 8 bits."""
    from paper_2607_14394_b200 import RolloutMemory
    B, T, D, H = 3, 12, 192, 256
    mk = lambda: [(rand(2 * H, D, seed=10 + i, scale=D ** -0.5), rand(D, H, seed=20 + i, scale=H ** -0.5),
                   1 + rand(D, seed=30 + i, scale=0.1)) for i in range(2)]
    fw = torch.ones(D, device="cuda")
    x = rand(B, T, D, dtype=BF16, seed=1)
    whole, steps = RolloutMemory(mk(), fw, B), RolloutMemory(mk(), fw, B)
    out = whole.forward(x)
    one = torch.stack([steps.step(x[:, t].contiguous()) for t in range(T)], 1)
    assert torch.isfinite(out).all()
    # the same products and norms row by row; the recurrence groups its steps differently, so a 16-bit state may round
    # the other way and an 8-bit value with it (one step of 2^-4 relative among 256)
    assert M.rel_l2(host(one), host(out)) <= 2e-2
    for a, b in zip(whole.states, steps.states):
        assert M.rel_l2(host(a), host(b)) <= 2e-2
    # against the statement in 64 bits, quantised at the same places
    r = host(x).reshape(B * T, D)
    r0 = r
    for w_in, w_out, nw in mk():
        y, _, _ = M.rms_norm(r[..., None], host(nw), EPS)
        q, s = M.quantize_rows(y[..., 0])
        vg = M.matmul_fp8(q, s, *M.quantize_blocks(host(w_in))).reshape(B, T, 2 * H)
        h, _, _ = M.gated_scan(vg[..., :H], vg[..., H:])
        q, s = M.quantize_rows(h.reshape(B * T, H))
        r = r + M.matmul_fp8(q, s, *M.quantize_blocks(host(w_out)))
    y, _, _ = M.rms_norm(r[..., None], np.ones(D), EPS)
    assert np.linalg.norm(r - r0) > 0.1 * np.linalg.norm(r0)
    # 16-bit intermediates flip some 8-bit roundings (each 2^-4 of its value, a few per cent of them): well below 5 %
    assert M.rel_l2(host(out).reshape(B * T, D), y[..., 0]) <= 5e-2
    ragged = RolloutMemory(mk(), fw, B)
    n = torch.tensor([0, 5, 12], dtype=torch.int32, device="cuda")
    part = ragged.forward(x, lengths=n)
    assert torch.equal(part[2], out[2]) and torch.equal(part[1, :5], out[1, :5])
    assert not ragged.states[0][0].any()
