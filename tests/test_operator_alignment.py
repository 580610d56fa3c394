"""Pointers off their element's alignment: refused on the host by the losses, every one of them."""
import pytest

from test_operator_refusals import ARG, P, distill, preference


@pytest.mark.parametrize("off", [1, 2, 3])
def test_losses_refuse_misaligned_pointers(off):
    for which, names in (("forward", dict(loss=4, lse=5)), ("backward", dict(lse=5, gl=3)), ("both", dict(loss=4, lse=5, gl=3))):
        for name, i in names.items():
            assert distill(which, **{name: P[i] + off}) == ARG, (which, name)
    inputs = dict(z=0, ref=1, c=2, r=3)
    for which, names in (("forward", dict(loss=5, margin=6)), ("backward", dict(gl=4, g=7)), ("both", dict(loss=5, margin=6, gl=4, g=7))):
        for name, i in {**inputs, **names}.items():
            assert preference(which, **{name: P[i] + off}) == ARG, (which, name)
