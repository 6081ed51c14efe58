"""How the selective memory's classes and entry points are called, without a GPU: what is refused before anything is launched."""
import ctypes

import pytest

from paper_2607_14394_b200 import binding as Bn
from test_selective_host import INVALID, NULL, P, _built, calls, entries                 # noqa: F401  (fixtures)

torch = pytest.importorskip("torch")
from paper_2607_14394_b200 import selective as Sel


def test_views_that_negate_or_conjugate_are_no_gradients(calls):
    """Such a view's values are not those in memory: what is written there would be read with the other sign."""
    z, r = torch.zeros(4, dtype=torch.complex64), torch.zeros(4)
    for bad in (z.conj(), torch._neg_view(r), torch._neg_view(z)):
        like = torch.zeros_like(bad).resolve_conj().resolve_neg()
        for pair in (([bad], None), ([like], [bad])):
            with pytest.raises(ValueError):
                Sel.GradNorm(*pair)
    Sel.GradNorm([z.conj().resolve_conj()], out=[z])


@pytest.mark.parametrize("spans,norm", [([(0x1000, 0x1000, 16)], 0x1004), ([(0x1000, 0, 16)], 0x103c), ([(0x1000, 0x5000, 16), (0x2000, 0x6000, 4)], 0x600c),
                                        ([(0x3000, 0, 2), (0x1000, 0x5000, 16)], 0x1000)])
def test_clip_refuses_a_norm_among_the_gradients(spans, norm):
    """The norm is written while gradients are still read and scaled."""
    L, e = Bn.lib(), entries(*spans)
    call = lambda at: L.dtst_clip_grad_norm(e, len(spans), 1.0, 1e-6, ctypes.c_void_p(at), NULL, 0, NULL)
    assert call(norm) == INVALID
    for clear in (0x0ffc, 0x1040, 0x2ffc, 0x3008, 0x4ffc, 0x5040, 0x6010):          # beside them: what is missing is the scratch
        assert call(clear) == Bn.DTST_ERR_WORKSPACE


def test_training_keeps_the_state_in_front(calls):
    """state_out may not lie where the state does, under whatever name: the backward pass reads the state as it was."""
    B, T, D, H, N = 2, 3, 8, 8, 4
    m = Sel.SelectiveMemory(D, H, N, dtype=torch.float32)
    x, conv, h = torch.zeros(B, T, D), torch.zeros(B, 3, H), torch.zeros(2 * B, H, N)
    for out in ((conv, torch.zeros(B, H, N)), (conv.view_as(conv), torch.zeros(B, H, N)), (torch.zeros_like(conv), h[:B]), (None, h[1:1 + B]),
                (h.view(-1)[:B * 3 * H].view(B, 3, H), torch.zeros(B, H, N))):
        with pytest.raises(ValueError, match="state as it was"):
            m.forward(x, (conv, h[:B]), state_out=out)
    m.forward(x, (conv, h[:B]), state_out=(conv, h[:B]), training=False)
    m.forward(x, (conv, h[:B]), state_out=(torch.zeros_like(conv), h[B:]))
    m.forward(x, (None, h[:B]), state_out=(conv, None))
