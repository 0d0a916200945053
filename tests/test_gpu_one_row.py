"""One token out of a wider buffer: its stride does not matter, the results
are those of the token alone."""
import pytest

torch = pytest.importorskip("torch")

from paper_2608_26430_gb300 import framefb as ffb
from tests.test_gpu_norm import DEV, built  # noqa: F401

pytestmark = pytest.mark.gpu


def one_row(t):
    """t's row at the start of rows whose leading dimension is odd, between values that must not be touched."""
    buf = torch.full((2, t.shape[1] + 9 + t.shape[1] % 2), 7.0, dtype=t.dtype, device=DEV)
    assert buf.stride(0) % 2 == 1
    buf[:1, :t.shape[1]] = t
    return buf[:1, :t.shape[1]], buf


def untouched(buf, d):
    return bool((buf[0, d:] == 7).all() and (buf[1] == 7).all())


@pytest.mark.parametrize("d", [12, 768, 4096])
def test_norm_and_dropout(d):
    x = torch.randn((1, d), generator=torch.Generator(device=DEV).manual_seed(d), device=DEV).bfloat16()
    xs, _ = one_row(x)
    for call in (lambda a, o: ffb.framefb_layernorm_forward(a, None, None, o), lambda a, o: ffb.framefb_dropout(a, o, 0.3, 1)):
        want = torch.empty_like(x)
        call(x, want)
        got, buf = one_row(torch.zeros_like(x))
        call(xs, got)
        assert torch.equal(got, want) and untouched(buf, d)


@pytest.mark.parametrize("d", [12, 72])
@pytest.mark.parametrize("V", [1, 300])
def test_cross_entropy(d, V):
    g = torch.Generator(device=DEV).manual_seed(d + V)
    pad = lambda t: torch.nn.functional.pad(t, (0, -d % 8))[:, :d]  # noqa: E731
    h, w = (pad(torch.randn((n, d), generator=g, device=DEV).bfloat16()) for n in (1, V))
    t = torch.zeros(1, dtype=torch.int64, device=DEV)

    def run(h, dh):
        loss, lse = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
        ffb.framefb_xent_forward(h, w, t, loss, lse, ws=ffb.xent_workspace(1, d, V, ffb.XENT_FORWARD, DEV))
        dw = pad(torch.zeros_like(w))
        ffb.framefb_xent_backward(h, w, t, lse, dH=dh, dW=dw, ws=ffb.xent_workspace(1, d, V, ffb.XENT_DH | ffb.XENT_DW, DEV))
        return loss, lse, dh, dw
    hs, _ = one_row(h)
    got, buf = one_row(torch.zeros_like(h))
    for a, b in zip(run(hs, got), run(h, pad(torch.zeros_like(h)))):
        assert torch.equal(a, b)
    assert untouched(buf, d)
