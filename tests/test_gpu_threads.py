"""Calls from several host threads, each with a stream of its own: a call's
launch does not depend on what another thread launches with the same kernel."""
import threading

import pytest

torch = pytest.importorskip("torch")

from paper_2608_26430_gb300 import framefb as ffb
from paper_2608_26430_gb300 import workloads as wl
from paper_2608_26430_gb300.batch import AdapterBatch
from tests.test_gpu_xent import Case

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_26430_gb300.build import build
    build()
    ffb.lib()


def at_once(calls, times):
    """Each of `calls` (a function of a stream) `times` times in a thread of its own; the errors they raised."""
    errors, gate = [], threading.Barrier(len(calls))

    def work(call):
        torch.cuda.set_device(DEV)
        stream = torch.cuda.Stream()
        gate.wait()
        try:
            for i in range(times):
                call(stream)
                if i % 200 == 199:
                    stream.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return errors


def test_norms_of_unlike_shared_memory():
    # one kernel of the gradient, with a third input (96 KB of shared memory) and without (64 KB); the descriptors
    # are laid out before, so that the threads meet in the library and not at the interpreter's lock
    N, d = 2, 4096
    g = torch.Generator(device=DEV).manual_seed(1)
    dY, Z, dZin = (torch.randn((N, d), generator=g, device=DEV).bfloat16() for _ in range(3))
    mean, rstd = torch.zeros(N, device=DEV), torch.ones(N, device=DEV)
    outs, want = ([torch.empty_like(dY) for _ in range(4)] for _ in range(2))
    for i, o in enumerate(want):
        ffb.framefb_layernorm_backward(dY, Z, None, mean, rstd, o, dZin=(None, dZin)[i % 2])

    def call(i):
        rows = lambda t: (t.data_ptr(), d)  # noqa: E731
        s = ffb._NORM.pack(N, d, 0.0, 0, 0, 0, mean.data_ptr(), rstd.data_ptr(), *rows(Z), 0, 0, 0, 0, 0, 0, *rows(dY),
                           *(rows(dZin) if i % 2 else (0, 0)), *rows(outs[i]), 0, 0, 0, 0)
        f = ffb.lib().framefb_layernorm_backward

        def run(stream):
            status = f(s, ffb.FRAMEFB_BF16, None, 0, stream.cuda_stream)
            if status != ffb.FRAMEFB_OK:
                raise ffb.FramefbError(status, "framefb_layernorm_backward")
        return run
    assert at_once([call(i) for i in range(4)], 4000) == []
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("dtype,dims,rho2", [("f32", (256, 768), False), ("bf16", (256, 768), False), ("bf16", (384, 768), True)])
def test_adapters_of_unlike_shared_memory(dtype, dims, rho2):
    # two widths of one kernel, of the structured and of the contraction path
    def batch(d, ops=7):
        frames = ((d, d // 2, 2),) if rho2 else ()
        w = wl.Workload(f"threads_{d}", (wl.MatSpec("w", d, d),), N=64, nnz=128, dtype=dtype, c_std=0.02, frames=frames)
        b = AdapterBatch(w, DEV, ops=ops)
        return b, b.workspace(ops)
    batches, alone = [batch(d) for d in dims], [batch(d) for d in dims]
    times = 600

    def call(b, ws):
        return lambda stream: ffb.framefb_run(b.mats, ffb.OP_BACKWARD_DX | ffb.OP_GRAD_COEFF, b.dtype_code, ws, stream)
    for b, ws in alone:
        call(b, ws)(None)
    assert at_once([call(b, ws) for b, ws in batches], times) == []
    for (a, _), (b, _) in zip(batches, alone):
        assert torch.equal(a.dC, b.dC)


def in_new_thread(call):
    """What `call` raised as the first CUDA work of a host thread (None: nothing)."""
    got = []

    def work():
        try:
            call()
            got.append(None)
        except Exception as e:  # noqa: BLE001
            got.append(e)
    torch.cuda.synchronize()
    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    return got[0]


@pytest.mark.parametrize("rho2", [False, True])
def test_adapters_as_a_threads_first_work(rho2):
    w = wl.Workload("thread", (wl.MatSpec("w", 384, 384),), N=64, nnz=128, dtype="bf16", c_std=0.02,
                    frames=((384, 192, 2),) if rho2 else ())
    b = AdapterBatch(w, DEV)
    ws = b.workspace(7)
    b.run(7, ws)
    want = b.dC.clone()
    b.dC.zero_()
    assert in_new_thread(lambda: b.run(7, ws, stream=0)) is None
    assert torch.equal(b.dC, want)


@pytest.mark.parametrize("N", [1, 64])
def test_cross_entropy_as_a_threads_first_work(N):
    c = Case(N, 72, 300)
    want = c.forward()
    grads = c.backward(want[1])
    got = [torch.empty_like(x) for x in want]
    ws = [ffb.xent_workspace(N, 72, 300, ops, DEV) for ops in (ffb.XENT_FORWARD, ffb.XENT_DH | ffb.XENT_DW)]
    dH, dW = c.H.clone(), c.W.clone()
    assert in_new_thread(lambda: ffb.framefb_xent_forward(c.H, c.W, c.t, *got, ws=ws[0], stream=0)) is None
    assert in_new_thread(lambda: ffb.framefb_xent_backward(c.H, c.W, c.t, want[1], dH=dH, dW=dW, ws=ws[1], stream=0)) is None
    for a, b in zip(got + [dH, dW], want + grads):
        assert torch.equal(a, b)


def test_norm_and_dropout_as_a_threads_first_work():
    x = torch.randn((8, 768), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).bfloat16()
    y, z = torch.empty_like(x), torch.empty_like(x)
    for call in (lambda o: ffb.framefb_layernorm_forward(x, None, None, o, stream=0),
                 lambda o: ffb.framefb_dropout(x, o, 0.5, 3, stream=0)):
        call(y)
        assert in_new_thread(lambda: call(z)) is None
        assert torch.equal(y, z)
