"""How the recurrent-memory classes call the library, without a GPU: CPU tensors, and a stand-in that records the
arguments of each entry point (and can call in again, as another thread would while the library has the first call)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2607_14394_b200 import build as Bd
from paper_2607_14394_b200 import memory as Mem

F32, BF16 = torch.float32, torch.bfloat16


class Calls:
    """A library whose entry points record their arguments and succeed; `during` runs inside the first recorded call."""

    def __init__(self, lib):
        self._real, self.seen, self.during = lib, [], None

    def __getattr__(self, name):
        if name.endswith(("_bytes", "_checkpoints")):      # host arithmetic
            return getattr(self._real, name)

        def call(*args):
            entry = (name, list(args))
            self.seen.append(entry)
            if self.during is not None:
                f, self.during = self.during, None
                f()
            for a in args:                                  # what the library would read of a description now
                if hasattr(a, "_obj") and isinstance(a._obj, Mem.Bn.ScanDesc):
                    d = a._obj
                    entry[1].append((tuple(d.in_stride), tuple(d.grad_stride)))
            return 0

        return call

    def last(self, name):
        return [a for n, a in self.seen if n == name][-1]


@pytest.fixture
def calls(monkeypatch):
    """Operators made under this fixture work on CPU tensors (device number -1) and call the stand-in."""
    Bd.build()
    rec = Calls(Mem.Bn.lib())
    monkeypatch.setattr(Mem.Bn, "lib", lambda: rec)
    monkeypatch.setattr(Mem, "_device", lambda device: -1)
    monkeypatch.setattr(Mem, "_current_device", lambda: -1)
    monkeypatch.setattr(Mem, "_raw_stream", lambda dev: 0)
    real = torch.device
    monkeypatch.setattr(Mem.torch, "device", lambda *a: real("cpu") if a == ("cuda", -1) else real(*a))
    return rec


def test_norm_backward_calls_do_not_share_scratch(calls):
    """Two calls of one object under way at once, as on two streams: each sums the weight gradient in memory of its own."""
    n = Mem.RmsNorm((4, 8), -1)
    x, w = torch.randn(4, 8), torch.ones(8)
    _, s, rstd = n.forward(x, w)
    calls.during = lambda: n.backward(x, s, w, rstd)
    n.backward(x, s, w, rstd)
    a, b = [args for name, args in calls.seen if name == "dtst_rms_norm_backward"]
    (pa, na), (pb, nb) = (a[12], a[13]), (b[12], b[13])
    assert na == nb > 0
    assert pa + na <= pb or pb + nb <= pa


def test_norm_over_its_input_leaves_no_sum(calls):
    """y in x's place without a residual: there is no s to hand to backward, and nothing that looks like one."""
    n = Mem.RmsNorm((4, 8), -1)
    x, w = torch.randn(4, 8), torch.ones(8)
    y, s, rstd = n.forward(x, w, out=x)
    assert y is x and s is None
    n.backward(x, s, w, rstd)
    assert calls.last("dtst_rms_norm_backward")[5] == 0          # which the library refuses
    kept = torch.empty(4, 8)
    assert n.forward(x, w, out=x, sum_out=kept)[1] is kept and n.forward(x, w)[1] is x
    none = torch.empty(0, 8)                                     # (an empty batch has no address to go by)
    assert Mem.RmsNorm((0, 8), -1).forward(none, w)[1] is none
    r = torch.randn(4, 8)
    assert n.forward(x, w, residual=r, out=x, sum_out=r)[1] is r


def test_norm_low_part_belongs_to_the_last_forward_call(calls):
    """An rstd used again: without a residual there is no low part, with one again there is."""
    n = Mem.RmsNorm((4, 8), -1, BF16)
    x, r, w = torch.randn(4, 8, dtype=BF16), torch.randn(4, 8, dtype=BF16), torch.ones(8)
    low = lambda: (calls.last("dtst_rms_norm")[9], calls.last("dtst_rms_norm_backward")[6])
    _, s, rstd = n.forward(x, w, residual=r)
    n.backward(x, s, w, rstd)
    assert low()[0] == low()[1] == rstd.sum_low.data_ptr() != 0
    _, s, rstd = n.forward(x, w, rstd=rstd)
    n.backward(x, s, w, rstd)
    assert low() == (0, 0)
    _, s, rstd = n.forward(x, w, residual=r, rstd=rstd)
    n.backward(x, s, w, rstd)
    assert low()[0] == low()[1] == rstd.sum_low.data_ptr() != 0


def test_norm_low_part_by_itself(calls):
    """Statistics that went through a detach: the low part is passed on beside them."""
    n = Mem.RmsNorm((4, 8), -1, BF16)
    x, w = torch.randn(4, 8, dtype=BF16), torch.ones(8)
    _, s, rstd = n.forward(x, w, residual=x)
    n.backward(x, s, w, rstd.detach().clone(), sum_low=rstd.sum_low)
    assert calls.last("dtst_rms_norm_backward")[6] == rstd.sum_low.data_ptr()
    with pytest.raises(ValueError):
        n.backward(x, s, w, rstd, sum_low=rstd.sum_low[:3])


def test_scan_calls_do_not_share_a_description(calls):
    """A call on contiguous tensors while the library has a call on halves of a projection, and the other way round."""
    B, L, D = 2, 6, 4
    plan = Mem.GatedScan((B, L, D), 1)
    vg, whole = torch.randn(B, L, 2 * D), torch.randn(B, L, D)
    halves, dense = (vg[..., :D], vg[..., D:]), (whole, whole.clone())
    strided = (L * 2 * D, 2 * D)
    flat = (L * D, D)
    ck, gh = torch.empty(plan.checkpoint_floats), torch.randn(B, L, D)
    wide = torch.empty(B, L, 3 * D)

    calls.during = lambda: plan.forward(*dense)
    plan.forward(*halves)
    calls.during = lambda: plan.forward(*halves)
    plan.forward(*dense)
    assert [args[-1][0] for name, args in calls.seen if name == "dtst_gated_scan"] == [strided, flat, flat, strided]

    calls.during = lambda: plan.backward(gh, *dense, ck)
    plan.backward(gh, *halves, ck, grad_v=wide[..., :D], grad_g=wide[..., D:2 * D])
    calls.during = lambda: plan.backward(gh, *halves, ck)
    plan.backward(gh, *dense, ck, grad_v=wide[..., :D], grad_g=wide[..., D:2 * D])
    got = [args[-1] for name, args in calls.seen if name == "dtst_gated_scan_backward"]
    third = (L * 3 * D, 3 * D)
    assert got == [(strided, third), (flat, flat), (flat, third), (strided, flat)]


def test_rows_that_overlap_reach_the_library_as_they_are(calls):
    """One row expanded to many: the library refuses a distance below the row's length, so it has to see that distance."""
    q, s = torch.zeros(4, 32, dtype=Mem.FP8), torch.ones(1, 4)
    lin = Mem.Fp8Linear.__new__(Mem.Fp8Linear)
    lin.dev, lin.n, lin.k, lin._kb, lin._ld, lin.out_dtype, lin._type = -1, 16, 32, 1, 32, F32, 0
    lin._w = lin._ws = lin._work = 0
    lin._lib = calls
    for out, ld in [(torch.empty(4, 16), 16), (torch.empty(4, 24)[:, :16], 24), (torch.empty(1, 16).expand(4, 16), 0),
                    (torch.empty(64).as_strided((4, 16), (8, 1)), 8)]:
        lin.forward(q, s, out=out)
        assert calls.last("dtst_matmul_fp8")[11] == ld
    # a single row has no distance to a next one, whatever its tensor's stride
    for width in (32, 48, 200):
        lin.forward(torch.zeros(1, width, dtype=Mem.FP8)[:, :32], torch.ones(1, 1))
        assert calls.last("dtst_matmul_fp8")[5] % 16 == 0
