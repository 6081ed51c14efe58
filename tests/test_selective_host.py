"""Selective-memory operators without a GPU: the float64 statement against differences, the C entry points' refusals (every one
of them is decided before anything is launched), and how the classes call the library."""
import ctypes

import numpy as np
import pytest

from oracle import selective_oracle as S
from paper_2607_14394_b200 import binding as Bn
from paper_2607_14394_b200 import build as Bd
from test_memory_calls_host import Calls

torch = pytest.importorskip("torch")
from paper_2607_14394_b200 import memory as Mem
from paper_2607_14394_b200 import selective as Sel


@pytest.fixture(scope="module", autouse=True)
def _built():
    Bd.build()


def check_gradients(loss, grads, inputs, rng, eps=1e-6):
    """Central differences of a smooth function of unit size: error about eps^2 + 1e-16 / eps times the sum's size."""
    for name, x in inputs.items():
        d = rng.standard_normal(x.shape)
        up, down = dict(inputs), dict(inputs)
        up[name], down[name] = x + eps * d, x - eps * d
        assert abs((loss(**up) - loss(**down)) / (2 * eps) - (grads[name] * d).sum()) < 3e-7, name


def test_layer_norm_gradients_match_differences():
    rng = np.random.default_rng(4)
    x, r, gy, gs = (rng.standard_normal((2, 6, 3)) for _ in range(4))
    w, b = rng.standard_normal(6), rng.standard_normal(6)

    def loss(x, w, b):
        y, s, _, _ = S.layer_norm(x, w, b, 1e-3, r)
        return (y * gy).sum() + (s * gs).sum()

    _, s, mean, rstd = S.layer_norm(x, w, b, 1e-3, r)
    gx, gw, gb = S.layer_norm_backward(gy, s, w, mean, rstd, gs)
    check_gradients(loss, {"x": gx, "w": gw, "b": gb}, {"x": x, "w": w, "b": b}, rng)


@pytest.mark.parametrize("lengths", [None, [0, 5, 2]])
@pytest.mark.parametrize("silu", [False, True])
def test_conv_gradients_match_differences(lengths, silu):
    rng = np.random.default_rng(5)
    x, gy, s, gl = rng.standard_normal((3, 5, 2)), rng.standard_normal((3, 5, 2)), rng.standard_normal((3, 3, 2)), rng.standard_normal((3, 3, 2))
    w, b = rng.standard_normal((2, 4)), rng.standard_normal(2)

    def loss(x, w, b, s):
        y, last = S.causal_conv(x, w, b, s, lengths, silu)
        return (y * gy).sum() + (last * gl).sum()

    gx, gw, gb, gs = S.causal_conv_backward(gy, x, w, b, s, lengths, gl, silu)
    check_gradients(loss, {"x": gx, "w": gw, "b": gb, "s": gs}, {"x": x, "w": w, "b": b, "s": s}, rng)


@pytest.mark.parametrize("lengths", [None, [0, 5, 2]])
@pytest.mark.parametrize("groups,gated,softplus", [(1, True, True), (2, False, True), (2, True, False)])
def test_scan_gradients_match_differences(lengths, groups, gated, softplus):
    rng = np.random.default_rng(6)
    n = lambda *s: rng.standard_normal(s)
    v = {"x": n(3, 5, 4), "dt": n(3, 5, 4) if softplus else 0.3 + 0.1 * n(3, 5, 4), "A": -np.exp(n(4, 3)), "B": n(3, 5, groups, 3),
         "C": n(3, 5, groups, 3), "D": n(4), "dt_bias": 0.1 * n(4), "h0": n(3, 4, 3)}
    if gated:
        v["z"] = n(3, 5, 4)
    gy, gl = n(3, 5, 4), n(3, 4, 3)

    def loss(**v):
        y, last = S.selective_scan(lengths=lengths, softplus=softplus, **v)
        return (y * gy).sum() + (last * gl).sum()

    check_gradients(loss, S.selective_scan_backward(gy, lengths=lengths, grad_last=gl, softplus=softplus, **v), v, rng)


# addresses that no call below may touch: each is refused first
P = [ctypes.c_void_p(0x10000 * k) for k in range(16)]
NULL, ODD = ctypes.c_void_p(0), ctypes.c_void_p(0x10001)
INVALID, UNSUPPORTED, WORKSPACE = Bn.DTST_ERR_INVALID_ARG, -2, -5


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(outer=-1), dict(c=0), dict(inner=-1), dict(eps=-1.0), dict(eps=float("nan")),
                                 dict(x=NULL), dict(w=NULL), dict(y=NULL), dict(x=ODD), dict(s=P[3]), dict(res=P[3]), dict(low=P[5]),
                                 dict(dtype=1, s=P[4], low=P[4]), dict(b=ODD), dict(stats=ODD), dict(outer=1 << 40, c=1 << 40)])
def test_layer_norm_refuses(bad):
    a = dict(dtype=0, outer=4, c=8, inner=1, eps=1e-5, x=P[1], res=NULL, w=P[2], b=NULL, s=NULL, low=NULL, y=P[3], stats=NULL)
    a.update(bad)
    assert Bn.lib().dtst_layer_norm(a["dtype"], a["outer"], a["c"], a["inner"], a["eps"], a["x"], a["res"], a["w"], a["b"], a["s"],
                                    a["low"], a["y"], a["stats"], NULL) == INVALID


@pytest.mark.parametrize("bad,want", [(dict(gy=NULL), INVALID), (dict(s=NULL), INVALID), (dict(stats=NULL), INVALID), (dict(gx=NULL), INVALID),
                                      (dict(gx=P[2]), INVALID), (dict(gb=P[6]), INVALID), (dict(low=P[9]), INVALID), (dict(gw=ODD), INVALID),
                                      (dict(scratch=NULL), WORKSPACE), (dict(nbytes=64), WORKSPACE), (dict(gw=NULL, nbytes=64), WORKSPACE),
                                      (dict(scratch=ctypes.c_void_p(0x100004)), INVALID)])
def test_layer_norm_backward_refuses(bad, want):
    a = dict(gy=P[1], s=P[2], low=NULL, w=P[3], stats=P[4], gs=NULL, gx=P[5], gw=P[6], gb=P[7], scratch=P[8], nbytes=1 << 20)
    a.update(bad)
    assert Bn.lib().dtst_layer_norm_backward(0, 4, 8, 1, a["gy"], a["s"], a["low"], a["w"], a["stats"], a["gs"], a["gx"], a["gw"], a["gb"],
                                             a["scratch"], a["nbytes"], NULL) == want


def conv_desc(dtype=0, act=1, B=2, T=5, C=8, K=4, at=(40, 8), to=(40, 8)):
    return Bn.ConvDesc(dtype, act, B, T, C, K, 0, at, to)


@pytest.mark.parametrize("desc,want", [(dict(dtype=5), INVALID), (dict(act=2), INVALID), (dict(B=-1), INVALID), (dict(C=0), INVALID),
                                       (dict(K=0), INVALID), (dict(K=5), UNSUPPORTED), (dict(at=(-40, 8)), INVALID), (dict(T=1 << 31), UNSUPPORTED),
                                       (dict(B=1 << 40, C=1 << 20), INVALID)])
def test_conv_refuses_descriptions(desc, want):
    d = conv_desc(**desc)
    assert Bn.lib().dtst_causal_conv(ctypes.byref(d), P[1], P[2], P[3], NULL, NULL, P[4], NULL, NULL) == want
    n = ctypes.c_size_t()
    assert Bn.lib().dtst_causal_conv_scratch_bytes(ctypes.byref(d), ctypes.byref(n)) == want


@pytest.mark.parametrize("bad", [dict(x=NULL), dict(w=NULL), dict(y=NULL), dict(y=P[1]), dict(y=P[5], state=P[5]), dict(out=P[1]), dict(out=P[4]),
                                 dict(x=ODD), dict(w=ODD), dict(state=ODD), dict(lengths=ODD)])
def test_conv_refuses(bad):
    a = dict(x=P[1], w=P[2], b=P[3], state=NULL, lengths=NULL, y=P[4], out=NULL)
    a.update(bad)
    assert Bn.lib().dtst_causal_conv(ctypes.byref(conv_desc()), a["x"], a["w"], a["b"], a["state"], a["lengths"], a["y"], a["out"], NULL) == INVALID


@pytest.mark.parametrize("bad,want", [(dict(gx=P[1]), INVALID), (dict(gx=P[2]), INVALID), (dict(gx=NULL), INVALID), (dict(gw=P[7], gb=P[7]), INVALID),
                                      (dict(gs=P[9], gso=P[9]), INVALID), (dict(gs=P[5], state=P[5]), INVALID), (dict(scratch=NULL), WORKSPACE),
                                      (dict(nbytes=8), WORKSPACE), (dict(to=(8, 8)), INVALID), (dict(to=(40, 4)), INVALID)])
def test_conv_backward_refuses(bad, want):
    a = dict(gy=P[1], gso=NULL, x=P[2], w=P[3], b=P[4], state=NULL, gx=P[6], gw=P[7], gb=P[8], gs=NULL, scratch=P[10], nbytes=1 << 30, to=(40, 8))
    a.update(bad)
    assert Bn.lib().dtst_causal_conv_backward(ctypes.byref(conv_desc(to=a["to"])), a["gy"], a["gso"], a["x"], a["w"], a["b"], a["state"], NULL,
                                              a["gx"], a["gw"], a["gb"], a["gs"], a["scratch"], a["nbytes"], NULL) == want


def scan_desc(dtype=0, B=2, T=5, C=8, N=16, G=1, rows=(40, 8), maps=(80, 16), **strides):
    at = [strides.get(k, rows if k[-1] in "xtz" else maps) for k in ("x", "dt", "z", "b", "c", "grad_x", "grad_dt", "grad_z", "grad_b", "grad_c")]
    return Bn.SelectiveDesc(dtype, 1, B, T, C, N, G, *at)


@pytest.mark.parametrize("desc,want", [(dict(dtype=5), INVALID), (dict(B=-1), INVALID), (dict(C=0), INVALID), (dict(N=0), INVALID), (dict(N=65), UNSUPPORTED),
                                       (dict(G=3), INVALID), (dict(G=0), INVALID), (dict(B=1 << 17), UNSUPPORTED), (dict(dt=(0, -1)), INVALID),
                                       (dict(T=1 << 31), UNSUPPORTED), (dict(T=1 << 44), INVALID)])
def test_scan_refuses_descriptions(desc, want):
    d = ctypes.byref(scan_desc(**desc))
    n, m = ctypes.c_int64(), ctypes.c_size_t()
    assert Bn.lib().dtst_selective_scan_checkpoints(d, ctypes.byref(n)) == want
    assert Bn.lib().dtst_selective_scan_scratch_bytes(d, 1, ctypes.byref(m)) == want
    i = Bn.SelectiveInputs(P[1], P[2], P[3], P[4], P[5], P[6], P[7], P[8], NULL, NULL)
    assert Bn.lib().dtst_selective_scan(d, ctypes.byref(i), P[9], NULL, NULL, NULL, 0, NULL) == want


INPUTS = dict(x=P[1], dt=P[2], z=P[3], B=P[4], C=P[5], A=P[6], D=P[7], dt_bias=P[8], h0=NULL, lengths=NULL)


@pytest.mark.parametrize("bad", [dict(x=NULL), dict(dt=NULL), dict(B=NULL), dict(C=NULL), dict(A=NULL), dict(x=ODD), dict(z=ODD), dict(A=ODD), dict(D=ODD),
                                 dict(dt_bias=ODD), dict(h0=ODD), dict(lengths=ODD), dict(y=NULL), dict(y=P[1]), dict(y=P[5]), dict(y=P[3]), dict(ck=P[9]),
                                 dict(last=ODD)])
def test_scan_refuses(bad):
    bad = dict(bad)
    y, ck, last = bad.pop("y", P[10]), bad.pop("ck", NULL), bad.pop("last", NULL)
    ck = ctypes.c_void_p(0x90008) if ck else NULL
    i = Bn.SelectiveInputs(**{**INPUTS, **bad})
    assert Bn.lib().dtst_selective_scan(ctypes.byref(scan_desc()), ctypes.byref(i), y, last, ck, NULL, 0, NULL) == INVALID


GRADS = dict(x=P[10], dt=P[11], z=P[12], B=P[13], C=P[14], A=NULL, D=NULL, dt_bias=NULL, h0=NULL)


@pytest.mark.parametrize("bad,want", [(dict(g=dict(x=NULL)), INVALID), (dict(g=dict(z=NULL)), INVALID), (dict(g=dict(B=P[14])), INVALID), (dict(g=dict(dt=P[1])), INVALID),
                                      (dict(g=dict(x=P[9])), INVALID), (dict(gy=NULL), INVALID), (dict(ck=NULL), INVALID), (dict(g=dict(A=ODD)), INVALID),
                                      (dict(desc=dict(grad_x=(8, 8))), INVALID), (dict(desc=dict(grad_b=(0, 16))), INVALID), (dict(scratch=NULL), WORKSPACE),
                                      (dict(nbytes=16), WORKSPACE)])
def test_scan_backward_refuses(bad, want):
    d, i, g = scan_desc(**bad.get("desc", {})), Bn.SelectiveInputs(**INPUTS), Bn.SelectiveGrads(**{**GRADS, **bad.get("g", {})})
    assert Bn.lib().dtst_selective_scan_backward(ctypes.byref(d), ctypes.byref(i), bad.get("gy", P[9]), NULL, bad.get("ck", P[15]), ctypes.byref(g),
                                                 bad.get("scratch", P[15]), bad.get("nbytes", 1 << 30), NULL) == want


def entries(*spans, dtype=0):
    return (Bn.GradTensor * len(spans))(*[Bn.GradTensor(g, o, n, dtype, 0) for g, o, n in spans])


@pytest.mark.parametrize("spans,more,want", [
    ([(0x1000, 0x1000, 16)], dict(max_norm=-1.0), INVALID), ([(0x1000, 0x1000, 16)], dict(max_norm=float("nan")), INVALID),
    ([(0x1000, 0x1000, 16)], dict(eps=0.0), INVALID), ([(0x1000, 0x1000, 16)], dict(norm=NULL), INVALID), ([(0x1000, 0x1000, 16)], dict(dtype=4), INVALID),
    ([(0, 0, 16)], {}, INVALID), ([(0x1000, 0, -1)], {}, INVALID), ([(0x1002, 0, 4)], {}, INVALID), ([(0x1000, 0x2002, 4)], {}, INVALID),
    ([(0x1000, 0x1000, 16), (0x1000, 0x1000, 16)], {}, INVALID),            # one tensor twice, in place: scaled twice
    ([(0x1000, 0x1000, 16), (0x1020, 0, 16)], {}, INVALID),                 # a gradient inside another's output
    ([(0x1000, 0x1020, 16)], {}, INVALID),                                  # an output that begins inside its own gradient
    ([(0x1000, 0x5000, 16), (0x2000, 0x5010, 16)], {}, INVALID),            # outputs that overlap
    ([(0x1000, 0x1000, 16)], dict(nbytes=8), WORKSPACE), ([(0x1000, 0x1000, 16)], dict(scratch=NULL), WORKSPACE)])
def test_clip_refuses(spans, more, want):
    a = dict(max_norm=1.0, eps=1e-6, norm=P[1], scratch=P[2], nbytes=1 << 20, dtype=0)
    a.update(more)
    e = entries(*spans, dtype=a["dtype"])
    assert Bn.lib().dtst_clip_grad_norm(e, len(spans), a["max_norm"], a["eps"], a["norm"], a["scratch"], a["nbytes"], NULL) == want


def test_empty_batches_need_no_pointers():
    L = Bn.lib()
    assert L.dtst_layer_norm(0, 0, 8, 1, 1e-5, *[NULL] * 9) == Bn.DTST_OK
    assert L.dtst_causal_conv(ctypes.byref(conv_desc(B=0)), *[NULL] * 8) == Bn.DTST_OK
    assert L.dtst_selective_scan(ctypes.byref(scan_desc(B=0)), None, NULL, NULL, NULL, NULL, 0, NULL) == Bn.DTST_OK


# ------------------------------------------------------------------------------------------------ the classes' calls
@pytest.fixture
def calls(monkeypatch):
    """Operators made under this fixture work on CPU tensors (device number -1) and call the stand-in."""
    rec = Calls(Bn.lib())
    rec.dtst_status_string = Bn.lib().dtst_status_string
    monkeypatch.setattr(Bn, "lib", lambda: rec)
    monkeypatch.setattr(Mem, "_device", lambda device: -1)
    monkeypatch.setattr(Mem, "_current_device", lambda: -1)
    monkeypatch.setattr(Mem, "_raw_stream", lambda dev: 0)
    real = torch.device
    monkeypatch.setattr(Sel.torch, "device", lambda *a: real("cpu") if a == ("cuda", -1) else real(*a))
    return rec


def test_shapes_types_and_layouts_are_checked(calls):
    ln, w, x = Sel.LayerNorm((4, 8)), torch.ones(8), torch.zeros(4, 8)
    for bad in (x.to(torch.float64), torch.zeros(4, 9), torch.zeros(8, 4).t()):
        with pytest.raises(ValueError):
            ln.forward(bad, w)
    with pytest.raises(ValueError):
        ln.forward(x, w, bias=torch.zeros(7))
    with pytest.raises(ValueError):
        Sel.CausalConv((2, 3), 4)
    with pytest.raises(ValueError):
        Sel.CausalConv((2, 3, 4), 4, activation="relu")
    with pytest.raises(Bn.DtstError):
        Sel.CausalConv((2, 3, 4), 5)
    with pytest.raises(ValueError):
        Sel.SelectiveScan((2, 3, 6), 4, groups=4)
    with pytest.raises(Bn.DtstError):
        Sel.SelectiveScan((2, 3, 6), 65)
    scan = Sel.SelectiveScan((2, 3, 6), 4)
    x, m, A = torch.zeros(2, 3, 6), torch.zeros(2, 3, 1, 4), torch.zeros(6, 4)
    for args in ((x, x, A, m, m[..., :3]), (x, x.transpose(0, 1), A, m, m), (x, x, A.double(), m, m), (torch.zeros(2, 3, 12)[..., ::2], x, A, m, m)):
        with pytest.raises(ValueError):
            scan.forward(*args)
    with pytest.raises(ValueError):
        Sel.GradNorm([torch.zeros(4, dtype=torch.float64)])
    with pytest.raises(ValueError):
        Sel.GradNorm([torch.zeros(4, 4).t()])
    with pytest.raises(ValueError):
        Sel.GradNorm([torch.zeros(4)], out=[])
    with pytest.raises(ValueError):
        Sel.GradNorm([torch.zeros(4, dtype=torch.complex64).conj()])


def test_parts_of_projections_are_passed_as_they_lie(calls):
    scan = Sel.SelectiveScan((2, 3, 8), 4, groups=2)
    xz, both, A = torch.zeros(2, 3, 16), torch.zeros(2, 3, 20), torch.zeros(8, 4)
    B, C = both[..., 4:12].unflatten(-1, (2, 4)), both[..., 12:].unflatten(-1, (2, 4))
    seen = {}

    class Spy:
        def __call__(self, desc, inputs, *rest):
            d, i = desc._obj, inputs._obj
            seen.update({n: tuple(getattr(d, n + "_stride")) for n in ("x", "dt", "z", "b", "c")}, B=i.B, C=i.C, z=i.z)
            return 0
    calls.dtst_selective_scan = Spy()
    scan.forward(xz[..., :8], torch.zeros(2, 3, 8), A, B, C, z=xz[..., 8:])
    assert seen["x"] == (48, 16) and seen["dt"] == (24, 8) and seen["b"] == seen["c"] == (60, 20)
    assert seen["B"] == both.data_ptr() + 16 and seen["C"] == both.data_ptr() + 48 and seen["z"] == xz.data_ptr() + 32


def test_backward_calls_do_not_share_scratch(calls):
    """Two calls of one object under way at once, as on two streams: each sums in memory of its own."""
    c = Sel.CausalConv((2, 5, 8), 4)
    x, w = torch.zeros(2, 5, 8), torch.zeros(8, 4)
    calls.during = lambda: c.backward(x, x, w)
    c.backward(x, x, w)
    a, b = [args for name, args in calls.seen if name == "dtst_causal_conv_backward"]
    assert a[12] + a[13] <= b[12] or b[12] + b[13] <= a[12]


def test_gradients_of_a_backward_pass_are_found(calls):
    g = {"W": [torch.zeros(3, dtype=torch.complex64), torch.zeros(2)], "b": torch.zeros(5), "a": None}
    n = Sel.GradNorm(g)
    assert [(e.n, e.dtype) for e in n._list] == [(6, 0), (2, 0), (5, 0)]
    assert [e.out for e in n._list] == [t.data_ptr() for t in n.tensors] and [e.out for e in n._only] == [None] * 3
    assert n.tensors[0] is g["W"][0]
