"""Layer norm of wide rows (one row takes a whole block) against the oracle:
rows that do not start on 16 bytes, and enough rows that every block has
several and every warp of the column sums' pass more than one.  The checks and
tolerances are those of the narrower rows."""
import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_norm as narrow
from tests.test_gpu_norm import BF16, F32, built  # noqa: F401

pytestmark = pytest.mark.gpu

UNALIGNED = [(3, 8193, 0, 0), (37, 9001, 1, 1), (5, 16383, 0, 0), (5, 16384, 3, 1)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,d,pad,offset", UNALIGNED)
@pytest.mark.parametrize("res,p", [(False, 0.0), (True, 0.2)])
def test_forward(dtype, N, d, pad, offset, res, p):
    narrow.test_layernorm_forward(dtype, N, d, pad, offset, res, p)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,d,pad,offset", UNALIGNED)
@pytest.mark.parametrize("skip,p", [(False, 0.0), (True, 0.2)])
def test_backward(dtype, N, d, pad, offset, skip, p):
    narrow.test_layernorm_backward(dtype, N, d, pad, offset, skip, p)


@pytest.mark.parametrize("dtype,d", [(BF16, 9232), (F32, 8200), (BF16, 8201), (F32, 8201)])
def test_many_rows(dtype, d):
    # more rows than SMs, and tens of rows for each warp of the column sums
    narrow.test_layernorm_forward(dtype, 331, d, 0, 0, True, 0.2)
    narrow.test_layernorm_backward(dtype, 331, d, 0, 0, True, 0.2)
    narrow.test_layernorm_backward(dtype, 1300, d, 0, 0, False, 0.0)
