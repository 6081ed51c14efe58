"""Recurrent-memory operators without a GPU: the float64 statement against differences, and the C entry points'
refusals (every one of them is decided before anything is launched)."""
import ctypes

import numpy as np
import pytest

from oracle import memory_oracle as M
from paper_2607_14394_b200 import binding as Bn
from paper_2607_14394_b200 import build as Bd


@pytest.fixture(scope="module", autouse=True)
def _built():
    Bd.build()


def _difference(f, x, d, eps=1e-6):
    return (f(x + eps * d) - f(x - eps * d)) / (2 * eps)


@pytest.mark.parametrize("gate", ["sigmoid", "decay"])
@pytest.mark.parametrize("lengths", [None, [0, 5, 3]])
def test_scan_gradients_match_differences(gate, lengths):
    rng = np.random.default_rng(3)
    v, g, gh = (rng.standard_normal((3, 5, 2)) for _ in range(3))
    h0, gl = rng.standard_normal((3, 2)), rng.standard_normal((3, 2))

    def loss(v_, g_, h_):
        h, last, _ = M.gated_scan(v_, g_, h_, lengths, gate)
        return (h * gh).sum() + (last * gl).sum()

    gv, gg, g0 = M.gated_scan_backward(gh, v, g, h0, lengths, gl, gate)
    for _ in range(4):
        dv, dg, d0 = rng.standard_normal(v.shape), rng.standard_normal(g.shape), rng.standard_normal(h0.shape)
        # central differences of a smooth function of unit size: error about eps^2 + 1e-16 / eps
        assert abs(_difference(lambda x: loss(x, g, h0), v, dv) - (gv * dv).sum()) < 1e-7
        assert abs(_difference(lambda x: loss(v, x, h0), g, dg) - (gg * dg).sum()) < 1e-7
        assert abs(_difference(lambda x: loss(v, g, x), h0, d0) - (g0 * d0).sum()) < 1e-7


def test_norm_gradients_match_differences():
    rng = np.random.default_rng(4)
    x, r, gy, gs = (rng.standard_normal((2, 6, 3)) for _ in range(4))
    w = rng.standard_normal(6)

    def loss(x_, w_):
        y, s, _ = M.rms_norm(x_, w_, 1e-3, r)
        return (y * gy).sum() + (s * gs).sum()

    _, s, rstd = M.rms_norm(x, w, 1e-3, r)
    gx, gw = M.rms_norm_backward(gy, s, w, rstd, gs)
    for _ in range(4):
        dx, dw = rng.standard_normal(x.shape), rng.standard_normal(6)
        assert abs(_difference(lambda t: loss(t, w), x, dx) - (gx * dx).sum()) < 1e-7
        assert abs(_difference(lambda t: loss(x, t), w, dw) - (gw * dw).sum()) < 1e-7


def test_e4m3_rounding_against_torch():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(5)
    x = np.concatenate([rng.standard_normal(4000) * 100, rng.standard_normal(4000) * 0.01, M.e4m3_values(),
                        (M.e4m3_values()[1:] + M.e4m3_values()[:-1]) / 2]).astype(np.float32)
    x = np.clip(x, -448, 448)
    got = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(got, M.to_e4m3(x))


# addresses that no call below may touch: each is refused first
A, B_, C, D, E, F = (ctypes.c_void_p(0x10000 * k) for k in range(1, 7))
WS = ctypes.c_void_p(0x100000)
NULL = ctypes.c_void_p(0)


def _norm(dtype=0, outer=4, c=8, inner=1, eps=1e-6, x=A, res=NULL, w=B_, s=NULL, low=NULL, y=C, rstd=NULL):
    return Bn.lib().dtst_rms_norm(dtype, outer, c, inner, eps, x, res, w, s, low, y, rstd, NULL)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(outer=-1), dict(c=0), dict(inner=-1), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(x=NULL), dict(w=NULL), dict(y=NULL),
                                 dict(x=ctypes.c_void_p(0x10002)), dict(s=C), dict(res=C),
                                 dict(outer=1 << 40, c=1 << 40), dict(low=E), dict(dtype=1, s=D, low=D), dict(dtype=1, low=E), dict(w=ctypes.c_void_p(0x20001))])
def test_norm_refuses(bad):
    assert _norm(**bad) == Bn.DTST_ERR_INVALID_ARG


def test_empty_batches_need_no_pointers():
    L = Bn.lib()
    assert _norm(outer=0, x=NULL, w=NULL, y=NULL) == Bn.DTST_OK
    assert L.dtst_rms_norm_fp8(1, 0, 64, 1e-6, NULL, NULL, NULL, NULL, NULL, 64, NULL, NULL) == Bn.DTST_OK
    assert L.dtst_quantize_fp8(1, 0, 64, NULL, 64, NULL, 64, NULL, NULL) == Bn.DTST_OK
    assert L.dtst_matmul_fp8(1, 0, 8, 16, NULL, 16, NULL, NULL, 16, NULL, NULL, 8, NULL, 0, NULL) == Bn.DTST_OK
    d = Bn.ScanDesc(0, 0, 0, 4, 8, (32, 8), (32, 8))
    assert L.dtst_gated_scan(ctypes.byref(d), NULL, NULL, NULL, NULL, NULL, NULL, NULL, NULL) == Bn.DTST_OK


@pytest.mark.parametrize("bad,want", [
    (dict(gy=NULL), -1), (dict(s=NULL), -1), (dict(rstd=NULL), -1), (dict(gx=NULL), -1), (dict(gx=B_), -1), (dict(low=F), -1),
    (dict(scratch=NULL), -5), (dict(nbytes=16), -5), (dict(c=0), -1), (dict(gw=ctypes.c_void_p(0x30002)), -1)])
def test_norm_backward_refuses(bad, want):
    a = dict(dtype=0, c=8, gy=A, s=B_, low=NULL, w=C, rstd=D, gs=NULL, gx=E, gw=F, scratch=WS, nbytes=1 << 20)
    a.update(bad)
    assert Bn.lib().dtst_rms_norm_backward(a["dtype"], 4, a["c"], 1, a["gy"], a["s"], a["low"], a["w"], a["rstd"], a["gs"], a["gx"],
                                           a["gw"], a["scratch"], a["nbytes"], NULL) == want


@pytest.mark.parametrize("bad,want", [
    (dict(dtype=7), -1), (dict(k=0), -1), (dict(x_ld=48), -1), (dict(x_ld=72), -1), (dict(w_ld=65), -1), (dict(out_ld=7), -1),
    (dict(x=ctypes.c_void_p(0x10008)), -1), (dict(w=NULL), -1), (dict(xs=NULL), -1), (dict(out=ctypes.c_void_p(0x50001)), -1),
    (dict(ws=NULL), -5), (dict(nws=128), -5), (dict(ws=ctypes.c_void_p(0x100010)), -1), (dict(m=-1), -1),
    (dict(m=1 << 33), -2)])
def test_matmul_refuses(bad, want):
    a = dict(dtype=1, m=4, n=8, k=64, x=A, x_ld=64, xs=B_, w=C, w_ld=64, wsc=D, out=E, out_ld=8, ws=WS, nws=256)
    a.update(bad)
    assert Bn.lib().dtst_matmul_fp8(a["dtype"], a["m"], a["n"], a["k"], a["x"], a["x_ld"], a["xs"], a["w"], a["w_ld"],
                                    a["wsc"], a["out"], a["out_ld"], a["ws"], a["nws"], NULL) == want


def test_quantisers_refuse():
    L = Bn.lib()
    assert L.dtst_quantize_fp8(0, 4, 64, A, 32, B_, 64, C, NULL) == -1           # rows overlap
    assert L.dtst_quantize_fp8(0, 4, 64, A, 64, B_, 32, C, NULL) == -1
    assert L.dtst_quantize_fp8(0, 4, 64, A, 64, A, 64, C, NULL) == -1            # in place
    assert L.dtst_quantize_fp8_weight(0, 4, 64, A, 32, B_, 64, C, NULL) == -1
    assert L.dtst_quantize_fp8_weight(9, 4, 64, A, 64, B_, 64, C, NULL) == -1
    assert L.dtst_rms_norm_fp8(1, 4, 64, 1e-6, A, NULL, B_, C, C, 64, D, NULL) == -1   # q is s


@pytest.mark.parametrize("fields,want", [
    (dict(dtype=5), -1), (dict(gate=2), -1), (dict(outer=-1), -1), (dict(length=-1), -1), (dict(inner=0), -1),
    (dict(in_stride=(-1, 8)), -1), (dict(inner=1, in_stride=(4, 2)), -1), (dict(inner=1, in_stride=(4, 1), grad_stride=(4, 3)), -1),
    (dict(length=1 << 32, in_stride=(1 << 35, 8), grad_stride=(1 << 35, 8)), -2), (dict(outer=1 << 44, inner=1 << 44), -1)])
def test_scan_descriptions_are_refused(fields, want):
    f = dict(dtype=0, gate=0, outer=3, length=4, inner=8, in_stride=(32, 8), grad_stride=(32, 8))
    f.update(fields)
    d = Bn.ScanDesc(f["dtype"], f["gate"], f["outer"], f["length"], f["inner"], f["in_stride"], f["grad_stride"])
    c = ctypes.c_int64()
    assert Bn.lib().dtst_gated_scan_checkpoints(ctypes.byref(d), ctypes.byref(c)) == want


def _scan(length=4, grad_stride=(32, 8), back=False, **k):
    d = Bn.ScanDesc(0, 0, 3, length, 8, (length * 8, 8), grad_stride)
    a = dict(v=A, g=B_, h=C, h0=NULL, last=NULL, ck=NULL, gv=D, gg=E, g0=NULL)
    a.update(k)
    r = ctypes.byref(d)
    if back:
        return Bn.lib().dtst_gated_scan_backward(r, a["h"], a["last"], a["v"], a["g"], a["h0"], NULL, a["ck"], a["gv"], a["gg"],
                                                 a["g0"], NULL)
    return Bn.lib().dtst_gated_scan(r, a["v"], a["g"], a["h0"], NULL, a["h"], a["last"], a["ck"], NULL)


def test_scan_refuses():
    assert _scan(v=NULL) == -1 and _scan(h=A) == -1 and _scan(h=ctypes.c_void_p(0x30002)) == -1
    assert _scan(h0=ctypes.c_void_p(0x40001)) == -1
    assert _scan(back=True, gv=E) == -1 and _scan(back=True, gv=A) == -1 and _scan(back=True, gg=NULL) == -1
    assert _scan(back=True, grad_stride=(32, 4)) == -1 and _scan(back=True, grad_stride=(0, 8)) == -1   # elements coincide
    assert _scan(back=True, length=4000, grad_stride=(32000, 8)) == -1                                  # no checkpoints
    assert Bn.lib().dtst_gated_scan(None, A, B_, NULL, NULL, C, NULL, NULL, NULL) == -1
    assert Bn.lib().dtst_workspace_status(NULL, NULL) == -1


def test_scan_checkpoint_counts():
    c = ctypes.c_int64()
    for outer, length, inner in [(3, 0, 8), (3, 1, 8), (2, 1000, 8), (5, 30, 1), (5, 3000, 1)]:
        d = Bn.ScanDesc(1, 0, outer, length, inner, (length * inner, inner), (length * inner, inner))
        assert Bn.lib().dtst_gated_scan_checkpoints(ctypes.byref(d), ctypes.byref(c)) == 0
        assert c.value % (outer * inner) == 0 and (c.value == 0) == (length == 0)
        assert c.value <= outer * inner * (1 + length // 256)
