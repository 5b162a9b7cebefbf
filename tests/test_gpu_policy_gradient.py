"""The gradient of the logits near the largest of a row, where most of the sum is, and far below it.

Rows of -inf but for n equal logits of a power of two: a / temperature times log2(e) is exact up to the constant's own rounding, so
every exponent is 0, the sum n, and the gradient of a logit that was not chosen -u / n with u = grad_scale w / temperature dL/dlogp.
What is left are a power of two of 0 (twice, one unit in the last place each: 4 * 2^-24) and two products: 6 * 2^-24 in all."""
import numpy as np
import pytest
import torch

import paper_2504_19925_amd as symi
from tests.test_gpu_policy import call, context

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
POWERS = [2.0 ** k for k in range(-6, 3)] + [-2.0 ** k for k in range(-6, 3)]
LARGE = [sign * 2.0 ** k for k in (24, 27, 28, 30, 40, 60) for sign in (1, -1)]


def flat_rows(values, V, n):
    """Rows whose first, last and n - 2 middle columns are one of `values`; the first is chosen and has the advantage 1 at a ratio of 1."""
    T = len(values)
    z = torch.full((T, V), float("-inf"), device="cuda")
    at = torch.linspace(0, V - 1, n, device="cuda").long()
    z[:, at] = torch.tensor(values, device="cuda")[:, None]
    f = lambda x: torch.full((T,), x, device="cuda")   # noqa: E731
    return dict(z=z, action=torch.zeros(T, dtype=torch.int32, device="cuda"), old=f(-float(np.log(n))), ref=None, advantage=f(1.0),
                weight=f(1.0)), at


@pytest.mark.parametrize("V", [64, 2100, 20000, 70000])
@pytest.mark.parametrize("values", [POWERS, LARGE], ids=["small", "large"])
def test_equal_logits_share_the_slope(values, V):
    for rows in (values, values * (300 // len(values) + 1)):        # split over workgroups, and not
        for tau in (1.0, 0.6, 0.7, 0.8, 1.1, 1.3, 1.7):
            for n in (2, 8):
                b, at = flat_rows(rows, V, n)
                hp = symi.SymiPolicy.make(temperature=tau, dtype="f32")
                _, _, dz = call(context(len(rows)), hp, b, V)
                got = dz[:, at].double()
                u = -1.0 / tau                                      # up to the rounding of the ratio: 1 + 4 * 2^-24 ln n and a few units
                assert ((got[:, 1:] * -n / u - 1).abs() <= 6 * U32 + 24 * U32).all(), (tau, n)
                # what the chosen one gets is what the others lose: no part of u is left over but roundings of the n values
                assert (got.sum(1).abs() <= 8 * U32 * abs(u)).all(), (tau, n, got.sum(1).abs().max().item() / U32)
                rest = torch.ones(V, dtype=torch.bool, device="cuda")
                rest[at] = False
                assert not dz[:, rest].any()


def test_far_below_the_largest():
    """Powers below the smallest normal number times a large scale: a relative error of 24 units for exponents of up to 140."""
    V = 64
    z = torch.full((2, V), -95.0, device="cuda")
    z[:, 0] = 0.0
    f = lambda x: torch.full((2,), x, device="cuda")   # noqa: E731
    b = dict(z=z, action=torch.zeros(2, dtype=torch.int32, device="cuda"), old=f(0.0), ref=None, advantage=f(1.0), weight=f(1.0))
    hp = symi.SymiPolicy.make(grad_scale=2.0 ** 30, dtype="f32")
    _, _, dz = call(context(2), hp, b, V)
    want = 2.0 ** 30 * np.exp(-95.0)
    # the exponent 137 is off by two roundings of it and the constant's: 3 * 2^-24 * 137 ln 2
    assert ((dz[:, 1:].double() / want - 1).abs() <= (24 + 3 * 95) * U32).all()


@pytest.mark.parametrize("V,rows", [(64, 600), (2100, 600), (2100, 200)])
@pytest.mark.parametrize("tau", [1.0, 0.7, 1.3])
def test_probabilities_near_the_largest(V, rows, tau):
    """Pairs of logits a > b, b's share of the slope against e^b / (e^a + e^b).  The pairs are those, of two million, whose exponents are
    furthest off if they are taken from the largest less 24 in single precision (up to 2^-19, or 22 * 2^-24 of the power): exponents near
    0 have to keep their own last bits.  The chosen logit is 80 below, so that its gradient is the slope itself.  Bound, in units of 2^-24:
    the power's root twice 4, exponents 1.4 for each of the two powers, products 2, quotient 1, the powers in the sum 2, additions
    1, corrections by the rounding of the largest exponent 2 in either: 17."""
    rng = np.random.default_rng(V)
    hp = symi.SymiPolicy.make(temperature=tau, dtype="f32")
    c = np.float64(np.float32(1.4426950408889634 * hp.inv_temperature))
    a = (rng.random(2000000) * 5 * tau).astype(np.float32)
    b = (a - rng.random(2000000) * 1.3 * tau).astype(np.float32)
    m = (a.astype(np.float64) * c).astype(np.float32)
    moved = (m - np.float32(24)).astype(np.float64)
    off = (b.astype(np.float64) * c - moved).astype(np.float32).astype(np.float64) - (b.astype(np.float64) * c - m.astype(np.float64) + 24)
    worst = np.argsort(-np.abs(off))[:rows]
    a, b = a[worst], b[worst]
    z = np.full((rows, V), -np.inf, np.float32)
    z[:, 0], z[:, V // 3], z[:, V // 2] = a - 80 * tau, a, b
    z64 = z[:, [0, V // 3, V // 2]].astype(np.float64) * hp.inv_temperature
    lse = z64[:, 1] + np.log(np.exp(z64 - z64[:, 1:2]).sum(1))
    t = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()   # noqa: E731
    inputs = dict(z=t(z), action=torch.zeros(rows, dtype=torch.int32, device="cuda"), old=t(z64[:, 0] - lse), ref=None, advantage=t(np.ones(rows)),
                  weight=t(np.ones(rows)))
    dz = call(context(rows), hp, inputs, V)[2].double().cpu().numpy()
    for at, k in ((V // 3, 1), (V // 2, 2)):
        share = -dz[:, at] / dz[:, 0]
        error = np.abs(share / np.exp(z64[:, k] - lse) - 1)
        assert (error <= 17 * U32).all(), error.max() / U32
