"""How the recurrent-memory operators are called: in place, with buffers used again, on several streams and threads, and
with values at the edge of what they take.  Tolerances are test_gpu_memory's, derived there."""
import numpy as np
import pytest

from oracle import memory_oracle as M

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
EPS = 1e-6

TOL = {F32: 1e-5, BF16: 1e-5 + 2.0 ** -8, F16: 1e-5 + 2.0 ** -11}


def rand(*shape, dtype=F32, seed=0, scale=1.0, shift=0.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=gen) * scale + shift).to(dtype)


def host(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------------------------------------ norm
# a shape for every kernel of the backward pass: rows in registers by length, rows off a vector, rows beyond the registers;
# fields in registers by channels, with and without vectors, and beyond the registers
IN_PLACE = [(3, 64), (5, 250), (700, 1024), (2, 2048), (2, 4096), (3, 4100), (2, 8000), (3, 8190), (2, 9000), (2, 16390),
            (2, 20, 90), (2, 33, 257), (1, 128, 64), (2, 150, 90), (1, 129, 33)]


@pytest.mark.parametrize("shape", IN_PLACE)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("over", ["grad_y", "grad_s"])
def test_norm_backward_in_place(shape, dtype, over):
    """grad_x in grad_y's or grad_s's place: the bits of the call into a buffer of its own."""
    from paper_2607_14394_b200 import RmsNorm
    n = RmsNorm(shape, 1, dtype, EPS)
    x, r, w = rand(*shape, dtype=dtype, seed=1), rand(*shape, dtype=dtype, seed=2), rand(shape[1], seed=3, shift=1.0)
    gy, gs = rand(*shape, dtype=dtype, seed=4), rand(*shape, dtype=dtype, seed=5)
    _, s, rstd = n.forward(x, w, residual=r)
    gx, gw = n.backward(gy, s, w, rstd, grad_s=gs)
    place = {"grad_y": gy, "grad_s": gs}[over]
    gx2, gw2 = n.backward(gy, s, w, rstd, grad_s=gs, grad_x=place)
    assert gx2.data_ptr() == place.data_ptr()
    assert torch.equal(gx2, gx) and torch.equal(gw2, gw)


def test_norm_backward_of_one_object_on_two_streams():
    """Calls of one object on two streams at once give what each gives alone."""
    from paper_2607_14394_b200 import RmsNorm
    n = RmsNorm((20000, 512), -1, F32, EPS)
    w = rand(512, seed=1, shift=1.0)
    sets, want, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(2):
        x, gy = rand(20000, 512, seed=2 + k), rand(20000, 512, seed=4 + k)
        _, s, rstd = n.forward(x, w)
        sets.append((gy, s, w, rstd))
        want.append(n.backward(*sets[k])[1])
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for k in range(2):
            got[k].append(n.backward(*sets[k], stream=streams[k])[1])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(torch.equal(g, want[k]) for g in got[k])


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_statistics_buffer_used_again(dtype):
    """An rstd that a call with a residual returned, used for one without and for one with again."""
    from paper_2607_14394_b200 import RmsNorm
    n = RmsNorm((40, 256), 1, dtype, EPS)
    x, r, w = rand(40, 256, dtype=dtype, seed=1), rand(40, 256, dtype=dtype, seed=2), rand(256, seed=3)
    gy = rand(40, 256, dtype=dtype, seed=4)

    def both(residual, rstd=None):
        _, s, rstd = n.forward(x, w, residual=residual, rstd=rstd)
        return (*n.backward(gy, s, w, rstd), rstd)

    *with_r, rstd = both(r)
    *without, _ = both(None)
    for residual, want in [(None, without), (r, with_r), (None, without)]:
        *got, rstd = both(residual, rstd)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_norm_low_part_passed_beside_the_statistics():
    from paper_2607_14394_b200 import RmsNorm
    n = RmsNorm((40, 256), 1, BF16, EPS)
    x, r, w, gy = (rand(*sh, dtype=t, seed=k) for k, (sh, t) in enumerate([((40, 256), BF16), ((40, 256), BF16), ((256,), F32),
                                                                         ((40, 256), BF16)]))
    _, s, rstd = n.forward(x, w, residual=r)
    want = n.backward(gy, s, w, rstd)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for stream in (None, st):
        got = n.backward(gy, s, w, rstd.detach().clone(), sum_low=rstd.sum_low, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ------------------------------------------------------------------------------------------------ recurrence
def test_scan_of_one_object_in_two_threads():
    """Threads that use one object, one on contiguous tensors and one on halves of a projection."""
    import threading

    from paper_2607_14394_b200 import GatedScan
    B, L, D = 2, 40, 64
    plan = GatedScan((B, L, D), 1)
    vg = rand(B, L, 2 * D, seed=1)
    halves = vg[..., :D], vg[..., D:]
    dense = rand(B, L, D, seed=2), rand(B, L, D, seed=3)
    want = [plan.forward(*t)[0] for t in (halves, dense)]
    bad, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()

    def work(k):
        for _ in range(300):
            h, _ = plan.forward(*(halves, dense)[k], stream=streams[k])
            streams[k].synchronize()
            if not torch.equal(h, want[k]):
                bad.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def scan_all(plan, v, g, gh, h0, gl=None, lengths=None):
    """(h, h_last, grad_v, grad_g, grad_h0)"""
    ck = plan.new_checkpoints()
    h, last = plan.forward(v, g, h0, lengths=lengths, checkpoints=ck)
    return (h, last, *plan.backward(gh, v, g, ck, h0, lengths=lengths, grad_last=gl))


def statement(v, g, gh, h0, gl, gate, lengths=None):
    d = (v.shape[0], v.shape[1], int(np.prod(v.shape[2:])))
    a = [host(t).reshape(d) for t in (v, g, gh)]
    z = [None if t is None else host(t).reshape(d[0], d[2]) for t in (h0, gl)]
    n = None if lengths is None else lengths.cpu().numpy()
    h, last, _ = M.gated_scan(a[0], a[1], z[0], n, gate)
    return (h, last, *M.gated_scan_backward(a[2], a[0], a[1], z[0], n, z[1], gate))


@pytest.mark.parametrize("mean", [-20.0, -14.0, -8.0])
@pytest.mark.parametrize("L", [1, 7, 16, 40, 100, 256, 600])
@pytest.mark.parametrize("inner", [8, 5, 1])
def test_scan_gradients_at_closed_gates(mean, L, inner):
    """a of 2e-9 to 3e-4: every gradient as accurate as at gates around 1, in every layout.

    Of grad_g that of the gates' own size, 1e-5: e^-|g| has a relative error of |g| 2^-24 (the rounding of g log2 e) and a few
    2^-23 more, 5e-6 at most here."""
    from paper_2607_14394_b200 import GatedScan
    shape = (3, L) if inner == 1 else (3, L, inner)
    state = (3,) if inner == 1 else (3, inner)
    v, g, gh = rand(*shape, seed=1), rand(*shape, seed=2, shift=mean, scale=0.25), rand(*shape, seed=3)
    h0, gl = rand(*state, seed=4), rand(*state, seed=5)
    got = scan_all(GatedScan(shape, 1), v, g, gh, h0, gl)
    want = statement(v, g, gh, h0, gl, "sigmoid")
    for what, a, b in zip(("h", "h_last", "grad_v", "grad_g", "grad_h0"), got, want):
        assert M.rel_l2(host(a).reshape(b.shape), b) <= TOL[F32], what


@pytest.mark.parametrize("mean", [8.0, 20.0])
@pytest.mark.parametrize("L", [1, 7, 16, 40, 100, 256, 600])
@pytest.mark.parametrize("inner", [8, 5, 1])
def test_scan_with_a_long_memory(mean, L, inner):
    """1 - a of 2e-9 to 3e-4, so that all of the steps count: an error of a that had one sign would add up.

    Rounded to nearest, a is off by up to 2^-25 and a state by 2^-24 at each step, either way: sqrt(600) of them are 2e-6.  (At
    gates of 20 a rounds to 1, always upward, by 2e-9 a step: 1e-6 in all.)"""
    from paper_2607_14394_b200 import GatedScan
    shape = (3, L) if inner == 1 else (3, L, inner)
    state = (3,) if inner == 1 else (3, inner)
    v, g, gh = rand(*shape, seed=1), rand(*shape, seed=2, shift=mean, scale=0.25), rand(*shape, seed=3)
    h0, gl = rand(*state, seed=4), rand(*state, seed=5)
    got = scan_all(GatedScan(shape, 1), v, g, gh, h0, gl)
    want = statement(v, g, gh, h0, gl, "sigmoid")
    for what, a, b in zip(("h", "h_last", "grad_v", "grad_g", "grad_h0"), got, want):
        assert M.rel_l2(host(a).reshape(b.shape), b) <= TOL[F32], what


def test_scan_gradients_at_saturated_gates():
    """Gates of plus and minus infinity: a is 1 or (below the normal numbers) 0, and nothing of a gate's own gradient is left."""
    from paper_2607_14394_b200 import GatedScan
    inf = float("inf")
    for shape in [(2, 300, 8), (2, 300, 5), (2, 20, 8), (2, 5, 8), (40, 30)]:
        plan = GatedScan(shape, 1)
        v, gh = rand(*shape, seed=1), rand(*shape, seed=2)
        h0 = rand(*plan.state_shape, seed=3)
        for g, gv, g0 in [(inf, torch.zeros_like(gh), gh.sum(1)), (-inf, gh, torch.zeros_like(h0))]:
            out = scan_all(plan, v, torch.full_like(v, g), gh, h0)
            assert torch.equal(out[2], gv) and float(out[3].abs().max()) < 1e-36
            assert M.rel_l2(host(out[4]), host(g0)) <= TOL[F32]


AMPLIFYING = [(2, 20, 8), (2, 200, 8), (2, 250, 5), (2, 600, 8), (2, 600, 5), (1, 9000, 8), (5, 300), (4, 600), (2, 9000), (2400, 1100)]


@pytest.mark.parametrize("shape", AMPLIFYING)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_decays_above_one_leave_a_state_of_zero_alone(shape, dtype):
    """Gates of 1.5, whose product over a tile is beyond float32: zeros until the last 20 steps (gradients: but the first 20)."""
    from paper_2607_14394_b200 import GatedScan
    plan = GatedScan(shape, 1, dtype, "decay")
    v, gh, g = (torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(3))
    v[:, -20:], gh[:, :20], g[:] = rand(*v[:, -20:].shape, dtype=dtype, seed=1), rand(*v[:, :20].shape, dtype=dtype, seed=2), 1.5
    got = scan_all(plan, v, g, gh, None)
    some = slice(0, 3)              # (of many sequences the statement walks a few)
    want = statement(v[some], g[some], gh[some], None, None, "decay")
    for what, a, b, t in zip(("h", "h_last", "grad_v", "grad_g", "grad_h0"), got, want, (dtype, F32, dtype, dtype, F32)):
        assert torch.isfinite(a).all(), what
        assert M.rel_l2(host(a[some]).reshape(b.shape), b) <= TOL[t], what


@pytest.mark.parametrize("shape", [(2, 200, 8), (2, 600, 5), (5, 300), (3, 2000), (40, 30)])
@pytest.mark.parametrize("t", [0, 1, 15, 16, 24, 29])
def test_scan_gate_of_nan_spoils_a_state_of_zero(shape, t):
    """0 times NaN: states behind such a gate are NaN, gradients in front of it, and nothing else is."""
    from paper_2607_14394_b200 import GatedScan
    plan = GatedScan(shape, 1, gate="decay")
    v, gh, g = (torch.zeros(shape, device="cuda") for _ in range(3))
    g[:] = 0.5
    g[1, t] = float("nan")
    got = scan_all(plan, v, g, gh, None)
    want = statement(v, g, gh, None, None, "decay")
    for a, b in zip(got, want):
        assert np.array_equal(np.isnan(host(a)).reshape(b.shape), np.isnan(b))


@pytest.mark.parametrize("shape", [(3, 256, 8), (3, 200, 5), (5, 400)])
def test_scan_decays_above_one_within_the_range(shape):
    """Gates of 0.9 to 1.25 (a product of 1e24 at most over the steps), states and gradients everywhere."""
    from paper_2607_14394_b200 import GatedScan
    L = shape[1]
    v, gh = rand(*shape, seed=1).abs(), rand(*shape, seed=2).abs()
    g = 0.9 + 0.35 * torch.rand(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    plan = GatedScan(shape, 1, gate="decay")
    h0 = rand(*plan.state_shape, seed=4).abs()
    got, want = scan_all(plan, v, g, gh, h0, h0), statement(v, g, gh, h0, h0, "decay")
    for a, b in zip(got, want):
        assert np.isfinite(b).all()
        # terms of one sign: at most 2 L roundings of 2^-24 each in any of them, and twice that in a product of two
        assert M.rel_l2(host(a).reshape(b.shape), b) <= 4 * L * 2.0 ** -24


@pytest.mark.parametrize("shape", [(1, 5000, 64), (2, 4097, 36), (1, 3000, 5), (1, 9001), (3, 30000), (4, 1, 64), (40, 30), (7, 9, 12)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_state_in_place(shape, dtype):
    """h_last in h0's place, also where a cluster shares the sequence and every CTA of it reads h0."""
    from paper_2607_14394_b200 import GatedScan
    plan = GatedScan(shape, 1, dtype)
    v, g = rand(*shape, dtype=dtype, seed=1), rand(*shape, dtype=dtype, seed=2)
    h0 = rand(*plan.state_shape, seed=3)
    h, last = plan.forward(v, g, h0)
    for _ in range(5):
        state = h0.clone()
        h2, last2 = plan.forward(v, g, state, h_last=state)
        assert last2.data_ptr() == state.data_ptr() and torch.equal(h2, h) and torch.equal(state, last)


# ------------------------------------------------------------------------------------------------ 8-bit product
def test_rows_that_overlap_are_refused():
    from paper_2607_14394_b200 import Fp8Linear, quantize_fp8, quantize_fp8_weight
    from paper_2607_14394_b200.binding import DtstError
    q, s = quantize_fp8(rand(4, 64, seed=1))
    lin = Fp8Linear.from_weight(rand(32, 64, seed=2), F32)
    for out in (torch.empty(1, 32, device="cuda").expand(4, 32), torch.empty(128, device="cuda").as_strided((4, 32), (16, 1))):
        with pytest.raises(DtstError):
            lin.forward(q, s, out=out)
    for quantise in (quantize_fp8, quantize_fp8_weight):
        with pytest.raises(DtstError):
            quantise(rand(1, 64, seed=3).expand(4, 64))
    one = quantize_fp8_weight(rand(1, 64, seed=3).expand(1, 64))
    assert one[0].shape == (1, 64)


def test_single_rows_of_any_stride():
    """One row of a buffer whose rows are not 16 bytes apart: operand, weights and the quantiser's output."""
    from paper_2607_14394_b200 import Fp8Linear, quantize_fp8, quantize_fp8_weight
    from paper_2607_14394_b200.memory import FP8
    buffer = lambda: torch.zeros(1, 200, dtype=torch.uint8, device="cuda").view(FP8)[:, :100]
    x, w = rand(1, 100, seed=1), rand(1, 100, seed=2)
    (q, s), (wq, ws) = quantize_fp8(x), quantize_fp8_weight(w)
    want = Fp8Linear(wq, ws, F32)(q, s)
    q2, wq2 = buffer(), buffer()
    wq2.copy_(wq)
    quantize_fp8(x, q=q2, scale=s)
    assert torch.equal(q2.float(), q.float())
    assert torch.equal(Fp8Linear(wq2, ws, F32)(q2, s), want)


# ------------------------------------------------------------------------------------------------ streams
@pytest.mark.parametrize("how", ["stream", "address"])
def test_calls_on_the_default_stream(how):
    """stream= the default stream, whose cudaStream_t is 0, from under another stream, behind work still running on it."""
    from paper_2607_14394_b200 import Fp8Linear, GatedScan, RmsNorm, RolloutMemory, quantize_fp8
    default = torch.cuda.default_stream()
    st = default if how == "stream" else default.cuda_stream
    assert default.cuda_stream == 0
    w, x = rand(256, seed=1), rand(60, 256, dtype=BF16, seed=2)
    n, lin = RmsNorm((60, 256), -1, BF16), Fp8Linear.from_weight(rand(128, 256, seed=3), BF16)
    scan = GatedScan((3, 20, 64), 1, BF16)
    mk = lambda: RolloutMemory([(rand(128, 256, seed=4), rand(256, 64, seed=5), w)], w, 3)

    def chain(x_, blk, **k):
        q, s, _ = n.forward_fp8(x_, w, **k)
        vg = lin.forward(q, s, **k).view(3, 20, 128)
        h, _ = scan.forward(vg[..., :64], vg[..., 64:], **k)
        return h, quantize_fp8(x_, **k)[0], blk.forward(x_.view(3, 20, 256), **k)

    want = chain(x, mk())
    blk, late, big = mk(), torch.zeros_like(x), torch.empty(1 << 28, device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        big.mul_(1.0001)
    late.copy_(x)
    with torch.cuda.stream(torch.cuda.Stream()):
        got = chain(late, blk, stream=st)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.float(), b.float())


_EDGES = """
import ctypes, torch
from paper_2607_14394_b200 import Fp8Linear, GatedScan, RmsNorm, quantize_fp8
w, x = torch.ones(256, device="cuda"), torch.randn(3000, 256, device="cuda")
n, lin = RmsNorm((3000, 256)), Fp8Linear.from_weight(torch.randn(2304, 256, device="cuda"))
few = Fp8Linear.from_weight(torch.randn(64, 2048, device="cuda"))
fq, fs = quantize_fp8(torch.randn(8, 2048, device="cuda"))
scan, row = GatedScan((1, 3000, 256)), GatedScan((1, 20000))
t = torch.randn(1, 20000, device="cuda")
v = torch.randn(1, 3000, 256, device="cuda")
def calls():
    q, s, _ = n.forward_fp8(x, w)
    return lin(q, s), lin(q[:100], s[:, :100].contiguous()), few(fq, fs), scan.forward(v, v), row.forward(t, t)
calls()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph(keep_graph=True)
with torch.cuda.graph(g):
    calls()
rt = ctypes.CDLL("libcudart.so.12")
many, ends = ctypes.c_size_t(0), (ctypes.c_void_p * 64)
print(rt.cudaGraphGetEdges(ctypes.c_void_p(g.raw_cuda_graph()), ends(), ends(), ctypes.byref(ctypes.c_size_t(64))))
"""


@pytest.mark.parametrize("off", [False, True])
def test_launches_without_the_dependent_launch_attribute(off):
    """DTST_NO_PDL=1 holds for the kernels in clusters too: no edge of a captured graph carries more than the plain order
    (the query that can only return plain edges is refused, code 402, where one does)."""
    import os
    import subprocess
    import sys
    env = {k: v for k, v in os.environ.items() if k != "DTST_NO_PDL"}
    if off:
        env["DTST_NO_PDL"] = "1"
    r = subprocess.run([sys.executable, "-c", _EDGES], env=env, capture_output=True, text=True, timeout=300,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stderr
    assert (int(r.stdout.split()[-1]) == 0) == off


# ------------------------------------------------------------------------------------------------ the blocks
@pytest.mark.parametrize("bad", [dict(C=33), dict(C=0), dict(B=0), dict(grid=(3, 5, 7)), dict(grid=()), dict(grid=(2,))])
def test_field_memory_refuses_what_it_cannot_train(bad):
    from paper_2607_14394_b200 import FieldMemory
    with pytest.raises(ValueError):
        FieldMemory(**{**dict(B=1, C=4, grid=(4, 6)), **bad})


def test_field_memory_reports_its_status():
    from paper_2607_14394_b200 import FieldMemory
    blk = FieldMemory(1, 4, (4, 6))
    out, _ = blk.forward(rand(1, 4, 4, 6, seed=1))
    blk.backward(out.clone())
    assert blk.status() == 0


def test_rollout_memory_over_histories_of_many_lengths():
    from paper_2607_14394_b200 import RolloutMemory
    w = torch.ones(64, device="cuda")
    blk = RolloutMemory([(rand(96, 64, seed=1, scale=0.1), rand(64, 48, seed=2, scale=0.1), w)], w, 2)
    x = rand(2, 40, 64, dtype=BF16, seed=3)
    first = blk.forward(x[:, :1].contiguous())
    for T in range(1, 41):
        blk.reset()
        blk.forward(x[:, :T].contiguous())
    assert len(blk._plans) <= 8
    blk.reset()
    assert torch.equal(blk.forward(x[:, :1].contiguous()), first)
    assert blk.status() == 0
