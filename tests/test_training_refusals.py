"""CPU tests of what the training-step operators refuse before anything is
launched: pointers that are not aligned to their elements, tensors that are
not on the current CUDA device, workspaces that are not what they seem."""
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


class Elsewhere:
    """What the binding looks at of a CPU tensor, as a tensor of another device."""

    def __init__(self, t, dev):
        self.t, self.dev = t, dev

    def get_device(self):
        return self.dev

    def __getattr__(self, name):
        return getattr(self.t, name)


def calls(dev):
    """One call of every operator on tensors of device `dev` (-1: CPU), with rows, and without rows but with
    outputs that are written all the same."""
    on = (lambda t: t) if dev < 0 else (lambda t: Elsewhere(t, dev))
    x, g, v = on(torch.zeros(4, 8)), on(torch.zeros(8)), on(torch.zeros(4))
    h, w = on(torch.zeros(4, 16, dtype=torch.bfloat16)), on(torch.zeros(32, 16, dtype=torch.bfloat16))
    t, m, ws = on(torch.zeros(4, dtype=torch.int64)), on(torch.zeros(1)), on(torch.zeros(1 << 20, dtype=torch.uint8))
    x0, h0, v0, t0 = on(torch.zeros(0, 8)), on(torch.zeros(0, 16, dtype=torch.bfloat16)), on(torch.zeros(0)), on(torch.zeros(0, dtype=torch.int64))
    return {
        "dropout": lambda: ffb.framefb_dropout(x, x, 0.1, 0, stream=0),
        "norm": lambda: ffb.framefb_layernorm_forward(x, g, g, x, stream=0),
        "norm gradient": lambda: ffb.framefb_layernorm_backward(x, x, g, v, v, x, g, g, ws=ws, stream=0),
        "norm gradient, no rows": lambda: ffb.framefb_layernorm_backward(x0, x0, g, v0, v0, x0, g, stream=0),
        "loss": lambda: ffb.framefb_xent_forward(h, w, t, v, v, ws=ws, stream=0),
        "loss, no rows": lambda: ffb.framefb_xent_forward(h0, w, t0, v0, v0, m, stream=0),
        "dH": lambda: ffb.framefb_xent_backward(h, w, t, v, dH=h, ws=ws, stream=0),
        "dW, no rows": lambda: ffb.framefb_xent_backward(h0, w, t0, v0, dW=w, stream=0),
    }


@pytest.mark.parametrize("dev", [-1, 1])
@pytest.mark.parametrize("name", list(calls(-1)))
def test_tensors_that_are_not_on_the_current_device(name, dev, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError) as e:
        calls(dev)[name]()
    assert e.value.status == ffb.FRAMEFB_EINVAL


def test_sizes_and_types_are_refused_before_the_device():
    x = torch.zeros(4, 16385)
    with pytest.raises(ffb.FramefbError) as e:
        ffb.framefb_layernorm_backward(x, x, None, torch.zeros(4), torch.zeros(4), x, stream=0)
    assert e.value.status == ffb.FRAMEFB_EUNSUPPORTED


def test_workspaces():
    x, v, g = torch.zeros(4, 8), torch.zeros(4), torch.zeros(8)
    h, w, t = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(32, 16, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    space = torch.zeros(1 << 20, dtype=torch.uint8)
    # elsewhere; fewer bytes than numel() says; bytes that are not its own in between
    for ws in (Elsewhere(space, 0), space[:1].expand(1 << 20), space[::2]):
        for call in (lambda: ffb.framefb_layernorm_backward(x, x, g, v, v, x, g, g, ws=ws, stream=0),
                     lambda: ffb.framefb_xent_forward(h, w, t, v, v, ws=ws, stream=0),
                     lambda: ffb.framefb_xent_backward(h, w, t, v, dH=h, ws=ws, stream=0)):
            with pytest.raises(ValueError, match="ws"):
                call()


@pytest.mark.parametrize("d", [1, 12, 16])
def test_the_stride_of_one_row_does_not_matter(d):
    # one token out of a wider buffer, or broadcast: its row starts where it starts
    for t in (torch.zeros(2, 17)[:1, :d], torch.zeros(3, d)[1:2], torch.zeros(d).expand(1, d)):
        ptr, ld = ffb._rows(t, "t", ffb._Like(t))
        assert ptr == t.data_ptr() and ld >= d and ld % 8 == 0
    assert ffb._rows(torch.zeros(2, 17)[:, :d], "t", ffb._Like(torch.zeros(2, d)))[1] == 17
