"""8-bit states of gradients around 1e-19: v lies on both sides of the smallest normal number, 2^-126, and eps decides nothing.

Bounds (u = 2^-24): those of test_gpu_adamw.py, and for v three roundings of denormal numbers more (the
decoded value, its decay, the new square: 0.7e-45 each), which its root inherits by half of their part of v; a code is the oracle's wherever the random number is not within 1e-4, or those roundings' part of the step between the two
codes, of the threshold, and one off at most elsewhere."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import ends_oracle as O
from tests.test_gpu_adamw import HP, U32, adam, context, gen, make, states

pytestmark = pytest.mark.gpu
UNIT = 2.1e-45


def step_and_check(t, step, eps, seed):
    w0, g = Hn.npf(t["param"]).astype(np.float64), Hn.npf(t["grad"]).astype(np.float64)
    m0, v0 = states(t)
    symi.symi_adamw_step(context(), symi.symi_adamw_create([t]), adam(step, eps=eps), None, seed)
    eps = float(np.float32(eps))
    w, m, v = O.adamw(w0, g, m0, v0, HP["lr"], HP["beta1"], HP["beta2"], eps, HP["wd"], step)
    fix = 1 - HP["beta1"] ** step
    root = np.sqrt(v / (1 - HP["beta2"] ** step)) + eps
    dm = 4 * U32 * (np.abs(HP["beta1"] * m0) + np.abs((1 - HP["beta1"]) * g)) + UNIT
    dv = 6 * U32 * v + UNIT
    up = np.abs(m) / fix / root
    part = np.where(v > 0, dv / np.maximum(v, UNIT) / 2, 0)
    tol = 2 * U32 * (np.abs(w0) + np.abs(w)) + HP["lr"] * (dm / fix / root + up * (20 * U32 + part) + 4 * U32 * HP["wd"] * np.abs(w0))
    got = Hn.npf(t["param"]).astype(np.float64)
    assert np.isfinite(got).all()
    assert (np.abs(got - w) <= tol).all(), (np.abs(got - w) / tol).max()
    n = len(w)
    for name, x, power, top, u, scale in (("m", np.abs(m), 2, 127, O.random_numbers(seed, step, 0, n)[0], "m_scale"),
                                          ("v", v, 4, 255, O.random_numbers(seed, step, 0, n)[1], "v_scale")):
        big = np.repeat(O.block_max(x), 256)[:n]
        kept = big >= 2.0 ** -125                  # of blocks that are not stored as zeros, whatever the last unit is
        assert (np.abs(np.repeat(Hn.npf(t[scale]), 256)[:n] - big) <= 1e-5 * big + UNIT)[kept].all()
        code, near = O.encode(x, power, top, u)
        if name == "v":
            code = np.where(x > 2 * UNIT, np.maximum(code, 1), code)
        lo = np.clip(np.floor(top * (x / np.maximum(big, 1e-300)) ** (1 / power)), 0, top - 1)
        size = (((lo + 1) / top) ** power - (lo / top) ** power) * big
        off = np.abs(np.abs(Hn.npf(t[name]).astype(np.int64)) - code)
        sure = near > 1e-4 + 2 * UNIT / np.maximum(size, 1e-300)
        assert (off[kept] <= 1).all() and (off[kept & sure] == 0).all(), (name, off[kept].max(), int((off[kept & sure] > 0).sum()))
    return kept


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("n", [256 * 40, 4096 + 77, 200])
def test_denormal_second_moments(n, grad):
    t = make(n, "f32", grad, 8, fresh=True, seed=n)
    g = gen(n + 1)
    size = 10.0 ** (torch.rand(n, generator=g, device="cuda") * 2.2 - 19.5)
    t["grad"].copy_(size * torch.randn(n, generator=g, device="cuda").sign())
    for step in (1, 2, 3):
        kept = step_and_check(t, step, 1e-24, 10 + step)
        assert kept.any()
        t["grad"].copy_(t["grad"].float() * 0.7)


@pytest.mark.parametrize("eps", [1e-39, 1e-44])
def test_a_denormal_eps(eps):
    """Nothing has a gradient: no weight moves but by the decay; with one, the updates are those of the definition."""
    t = make(1000, "f32", "f32", 8, fresh=True, seed=1)
    t["grad"].zero_()
    w0 = t["param"].double()
    symi.symi_adamw_step(context(), symi.symi_adamw_create([t]), adam(1, eps=eps), None, 0)
    assert ((t["param"].double() - w0 * (1 - HP["lr"] * HP["wd"])).abs() <= 4 * U32 * w0.abs()).all()
    t["grad"][::2] = 1.0
    step_and_check(t, 2, eps, 3)
