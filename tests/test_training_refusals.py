"""CPU tests of what the training-step operators refuse before anything is
launched: pointers that are not aligned to their elements."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_26430_gb300 import framefb as ffb


@pytest.fixture(scope="module", autouse=True)
def built_library():
    from paper_2608_26430_gb300.build import build
    build()


A = 1 << 20  # an aligned address (nothing is read from it)


def xent(N=4, **over):
    """A packed framefb_xent of 16 columns and 32 words whose addresses are all aligned, but for `over`."""
    p = dict(target=A, loss=A, lse=A, loss_mean=A, dloss=A, dH=0, dW=0)
    p.update(over)
    return ffb._XENT.pack(N, 16, 32, -100, p["target"], A, 16, A, 16, p["loss"], p["lse"], p["loss_mean"], p["dloss"],
                          p["dH"], 16, p["dW"], 16, 1.0, 0)


@pytest.mark.parametrize("N", [4, 0])
@pytest.mark.parametrize("field,off", [("target", 4), ("loss", 2), ("lse", 1), ("loss_mean", 2)])
def test_misaligned_vectors_of_the_loss(N, field, off):
    assert ffb.lib().framefb_xent_forward(xent(N, **{field: A + off}), ffb.FRAMEFB_BF16, None, 0, None) == ffb.FRAMEFB_EINVAL


@pytest.mark.parametrize("field,off", [("target", 4), ("lse", 2), ("dloss", 2)])
def test_misaligned_vectors_of_the_gradients(field, off):
    for out in ("dH", "dW"):
        s = xent(**{field: A + off, out: A})
        assert ffb.lib().framefb_xent_backward(s, ffb.FRAMEFB_BF16, None, 0, None) == ffb.FRAMEFB_EINVAL
