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
