"""How near the cross entropy's loss and lse come to 64 bits on average: the
worst case over signs that bounds single tokens elsewhere is some hundred
times the usual error.

Tolerances, for random logits whose partial sums stay within the largest logit
`top` of their row (U32 = 2^-24).  The tensor cores add d / 16 steps, each of
which loses half a unit 2^-23 of the sum on average, towards zero: (d / 16 + 16)
U32 top.  Few tokens' sums round to nearest, d / 64 additions in sequence and a
tree of 6, and roundings average out: sqrt(d / 64 + 6) U32 top.  The exponent's
base, exp2 and log add 8 U32 (top + 1).  The loss takes two such numbers.
"""
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_xent import U32, Case, built  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [3, 64, 300])
@pytest.mark.parametrize("d", [256, 1024, 4096])
def test_average_error_of_the_loss(N, d):
    c = Case(N, d, 9001, seed=9).reference()
    loss, lse, mean = c.forward()
    top = float(c.top.mean())
    sums = (d / 64 + 6) ** 0.5 if N <= 4 else d / 16 + 16
    tol = U32 * (sums * top + 8 * (top + 1))
    assert float((lse.double() - c.lse).abs().mean()) <= tol
    assert float((loss.double() - c.loss).abs().mean()) <= 2 * tol
    # the mean adds N numbers in 32 bits, in runs of N / 256 and a tree
    assert abs(float(mean) - float(c.loss.mean())) <= 2 * tol + (N / 256 + 16) * U32 * float(c.loss.abs().mean())
