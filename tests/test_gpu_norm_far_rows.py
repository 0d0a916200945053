"""The layer norm's gradient on rows far from zero: xh = (Z - mean) rstd with
the mean given is nearly exact, however large the mean.

Tolerances: Z - mean is one rounding at most (none where both are within a
factor of two), the product with rstd another, so xh carries 3 U32 |xh| (U32 =
2^-24); sums and products are fp32 as in the other tests of the gradient.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import training as tr
from paper_2608_26430_gb300 import framefb as ffb
from tests.oracle_side import host64
from tests.test_gpu_norm import DEV, F32, U32, assert_close, built, empty, rows, vec  # noqa: F401

pytestmark = pytest.mark.gpu


def gradients(dY, Z, gamma, mean, rstd, p=0.0):
    N, d = Z.shape
    dZ = empty(N, d, Z.dtype)
    more = dict(dX=empty(N, d, Z.dtype), drop=ffb.framefb_dropout_params(p, 3, 4)) if p else {}
    dgamma, dbeta = (torch.full((d,), float("nan"), device=DEV) for _ in range(2))
    ffb.framefb_layernorm_backward(dY, Z, gamma, mean, rstd, dZ, dgamma, dbeta, ws=ffb.layernorm_workspace(N, d, DEV), **more)
    return dZ, dgamma, dbeta


@pytest.mark.parametrize("p", [0.0, 0.3])  # (the dropout makes dX only, by another variant of the kernel)
@pytest.mark.parametrize("d", [768, 1023, 9000, 9001])  # in registers, unaligned; with a pass for the column sums
def test_gradient_of_rows_far_from_zero(d, p):
    rng = np.random.default_rng(d)
    N = 37
    x = rng.standard_normal((N, d))
    Z = rows(x + 2.0 ** 12 * rng.choice([-1.0, 1.0], (N, 1)), F32)  # 4096 standard deviations
    dY = rows(x + 0.5 * rng.standard_normal((N, d)), F32)           # mean(a xh) is about 1
    gamma = vec(1 + 0.2 * rng.standard_normal(d))
    _, mu, rs = tr.layernorm(host64(Z))
    mean, rstd = vec(mu), vec(rs)
    dZ, dgamma, dbeta = gradients(dY, Z, gamma, mean, rstd, p)
    z, dy, g = host64(Z), host64(dY), host64(gamma)
    mu, rs = host64(mean)[:, None], host64(rstd)[:, None]
    dz, dg, db = tr.layernorm_grad(dy, z, g, mu[:, 0], rs[:, 0])
    xh, a = (z - mu) * rs, dy * g
    e_xh = 3 * U32 * np.abs(xh)
    mean1, mean2 = np.abs(a).mean(axis=1, keepdims=True), np.abs(a * xh).mean(axis=1, keepdims=True)
    slack = rs * (8 * U32 * (np.abs(a) + mean1 + np.abs(xh) * mean2) + 64 * U32 * (mean1 + np.abs(xh) * mean2)
                  + e_xh * mean2 + np.abs(xh) * (np.abs(a) * e_xh).mean(axis=1, keepdims=True))
    assert_close(dZ, dz, F32, slack, "dZ")
    assert_close(dgamma, dg, F32, (N + 64) * U32 * np.abs(dy * xh).sum(axis=0) + (np.abs(dy) * e_xh).sum(axis=0), "dgamma")
    assert_close(dbeta, db, F32, (N + 64) * U32 * np.abs(dy).sum(axis=0), "dbeta")


@pytest.mark.parametrize("p", [0.0, 0.3])
@pytest.mark.parametrize("d", [768, 9001])
def test_a_constant_row_has_no_direction(d, p):
    # xh of a row equal to its mean is 0: nothing of it reaches dgamma
    c = np.float32(1000.1)
    Z, dY = rows(np.full((3, d), c), F32), rows(np.random.default_rng(d).standard_normal((3, d)), F32)
    _, dgamma, _ = gradients(dY, Z, None, vec([c] * 3), vec([1e-5 ** -0.5] * 3), p)
    assert not dgamma.any()
