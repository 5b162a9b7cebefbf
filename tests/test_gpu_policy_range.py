"""Logits of any finite size: parts of a row, or all of it, at the numbers that masks are made of (-1e10, -1e30, the type's lowest), and
rows whose product with the temperature is beyond single precision.

Only differences to the largest logit of a row matter.  In 64 bits they give logp and the probabilities p; the bound is that of
test_gpu_policy.py with Z the largest of those differences among the logits that count (nearer than 110: the others have less than
e^-110 and may come out as 0): |logp error| <= u (6 Z + V / 64 + 24 + 2 |logp|), u = 2^-24, plus u |logp| for the double differences'
constant."""
import pytest
import torch

import paper_2504_19925_amd as symi
from tests.test_gpu_policy import call, context

pytestmark = pytest.mark.gpu
U32, U16 = 2.0 ** -24, 2.0 ** -8
MASKS = (-1e9, -1e10, -3e12, -1e15, -1e30, -2.3e38, -3e38)


def rows(V, dt, T):
    """(logits, chosen tokens): a normal row with its second, first or middle part masked, rows of one value, rows of two."""
    g = torch.Generator(device="cuda").manual_seed(V)
    lowest, highest = torch.finfo(dt).min, torch.finfo(dt).max
    out, action = [], []
    j = torch.arange(V, device="cuda")
    for x in (*MASKS, lowest):
        for part in (j >= V // 2, j < V // 2, (j > V // 4) & (j < V - V // 4)):
            z = torch.randn(V, generator=g, device="cuda") * 3
            z[part] = x
            out.append(z)
            action.append(int(torch.nonzero(~part)[V // 5]))
    for x in (*MASKS, lowest, highest, 1e9, 1e10, 7e22, 3e38):
        out.append(torch.full((V,), x, device="cuda"))
        action.append(V // 3)
    for low, high in ((lowest, highest), (-1e30, 1e30), (1.0, 1e12), (lowest, 0.0), (-3e38, -1e30), (-1e10, -1e10 + 4096), (1e10, 1e10 + 1024)):
        z = torch.where(j % 3 == 1, high, low)
        out.append(z)
        action.append(1)
    z = torch.full((V,), lowest, device="cuda")       # nothing but the chosen token
    z[V - 1] = 2.0
    out.append(z)
    action.append(V - 1)
    n = len(out)
    z = torch.stack(out).to(dt)
    at = torch.arange(T, device="cuda") % n
    return z[at].contiguous(), torch.tensor(action, device="cuda", dtype=torch.int32)[at].contiguous(), n


@pytest.mark.parametrize("tau", [1.0, 0.125, 30.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,T", [(2, 46), (21, 46), (700, 46), (9001, 46), (9001, 300), (40000, 46), (40000, 300), (140001, 46), (140001, 270)])
def test_any_finite_logits(V, T, dtype, tau):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    if V == 2:
        z = torch.tensor([[a, b] for a in (*MASKS, 0.0, 1e10, 3e38) for b in (*MASKS, 0.0, 1e10, 3e38)], device="cuda").to(dt)
        T = len(z)
        action = z.float().argmax(1).to(torch.int32)
    else:
        z, action, _ = rows(V, dt, T)
    hp = symi.SymiPolicy.make(0.5, 0.5, 0.0, tau, 1.0, dtype)
    d = (z.double() - z.double().amax(1, keepdim=True)) * hp.inv_temperature
    lse = d.exp().sum(1, keepdim=True).log()
    a = action.long()[:, None]
    lp = (d.gather(1, a) - lse)[:, 0]
    f = lambda x: torch.full((T,), x, device="cuda")   # noqa: E731
    b = dict(z=z, action=action, old=lp.float(), ref=None, advantage=f(1.0), weight=f(1.0))
    Z = torch.where(d > -110, -d, 0.0).amax(1)
    e = U32 * (6 * Z + V / 64 + 24 + 3 * lp.abs())
    ctx = context(T)
    logp, stats, dz = call(ctx, hp, b, V)
    print(f"[policy] {dtype} V={V} T={T} tau={tau}: {int(logp.isnan().sum())} NaN", flush=True)
    alone, alone_stats, _ = call(ctx, hp, b, V, grad=False)
    single = torch.full((T,), float("nan"), device="cuda")
    symi.symi_token_logp(ctx, hp, z, V, V, action, None, single)
    for got in (logp, alone, single):
        assert ((got.double() - lp).abs() <= e).all()
    # the ratio is 1 up to logp's error and old's rounding
    ratio = torch.exp(lp - b["old"].double())
    rel = 2 * e + U32 * (16 + 4 * lp.abs())
    for got in (stats, alone_stats):
        assert abs(got[0].double() + ratio.sum()) <= (ratio * rel).sum() + 8 * U32 * T
        assert got[2] == 0 and got[3] == 0
    p = torch.exp(d - lse)
    u = -hp.inv_temperature * ratio[:, None]
    want = -u * p
    want.scatter_add_(1, a, u)
    part = p.scatter_add(1, a, torch.ones_like(lp)[:, None])
    bound = u.abs() * 2 * rel[:, None] * part + (U16 if dtype == "bf16" else U32) * 1.01 * want.abs() + 1e-38
    assert ((dz.double() - want).abs() <= bound).all()


def test_the_log_probability_of_a_masked_token():
    for dtype, dt in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        for V in (50, 5000, 70000):
            z = torch.randn(len(MASKS), V, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dt)
            z[:, V // 2:] = torch.tensor(MASKS, device="cuda")[:, None].to(dt)
            action = torch.full((len(MASKS),), V - 1, dtype=torch.int32, device="cuda")
            logp = torch.full((len(MASKS),), float("nan"), device="cuda")
            hp = symi.SymiPolicy.make(dtype=dtype)
            symi.symi_token_logp(context(len(MASKS)), hp, z, V, V, action, None, logp)
            want = torch.log_softmax(z.double(), 1)[:, V - 1]
            assert ((logp.double() - want).abs() <= 3 * U32 * want.abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_inverse_temperature(dtype):
    """The constant of the exponents has to stay finite: the chosen token, the largest of its row, has all the probability."""
    V, T = 1000, 5
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    z = torch.randn(T, V, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(dt)
    z[:, 77] = 9.0
    hp = symi.SymiPolicy.make(dtype=dtype)
    hp.inv_temperature = 3.4e38
    f = lambda x: torch.full((T,), x, device="cuda")   # noqa: E731
    b = dict(z=z, action=torch.full((T,), 77, dtype=torch.int32, device="cuda"), old=f(0.0), ref=None, advantage=f(0.0), weight=f(1.0))
    logp, stats, dz = call(context(T), hp, b, V)
    assert not logp.any() and not stats.any() and not dz.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tau", [0.1, 0.003, 3e-4, 1.1e-4, 1e-5])
def test_low_temperatures(tau, dtype):
    """Exponents of the largest logit from some hundred to some million: on both sides of where they are taken in one operation."""
    T, dt = 40, torch.bfloat16 if dtype == "bf16" else torch.float32
    for V, rows in ((300, T), (20000, T), (20000, 300)):
        g = torch.Generator(device="cuda").manual_seed(V)
        top = torch.linspace(-40, 40, rows, device="cuda")[:, None]
        z = top - torch.rand(rows, V, generator=g, device="cuda") * 40 * tau      # as near as the temperature lets them count
        z = z.to(dt)
        hp = symi.SymiPolicy.make(0.5, 0.5, 0.0, tau, 1.0, dtype)
        d = (z.double() - z.double().amax(1, keepdim=True)) * hp.inv_temperature
        a = torch.randint(0, V, (rows, 1), generator=g, device="cuda")
        lp = torch.log_softmax(d, 1).gather(1, a)[:, 0]
        f = lambda x: torch.full((rows,), x, device="cuda")   # noqa: E731
        b = dict(z=z, action=a[:, 0].to(torch.int32), old=lp.float(), ref=None, advantage=f(1.0), weight=f(1.0))
        Z = torch.where(d > -110, -d, 0.0).amax(1)
        e = U32 * (6 * Z + V / 64 + 24 + 3 * lp.abs())
        logp, stats, dz = call(context(rows), hp, b, V)
        assert ((logp.double() - lp).abs() <= e).all()
        ratio = torch.exp(lp - b["old"].double())
        rel = 2 * e + U32 * (16 + 4 * lp.abs())
        p, u = torch.softmax(d, 1), -hp.inv_temperature * ratio[:, None]
        want = (-u * p).scatter_add_(1, a, u)
        part = p.scatter_add(1, a, torch.ones_like(u))
        bound = u.abs() * 2 * rel[:, None] * part + (U16 if dtype == "bf16" else U32) * 1.01 * want.abs() + 1e-38
        assert ((dz.double() - want).abs() <= bound).all()
