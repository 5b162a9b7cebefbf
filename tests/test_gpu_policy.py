"""Log probabilities, the clipped policy loss and its gradient against binary64.

Bounds (u = 2^-24).  With Z the largest |logit| / temperature of a row, the exponent of every summand is off by at most
3 u Z (two roundings of the product, one of the constant), a power of two by 2 u, the sum by u for each of its additions in
a row: V / 64 + 16 at most (64 threads or more, then a tree), the logarithm and the last subtraction by 2 u each of their
size.  So |logp error| <= u (6 Z + V / 64 + 24 + 2 |logp|) =: e.  The ratio inherits e and its own exponent's rounding; the gradient
of a logit is (indicator + p) times the slope, each with a relative error of e and a few u; bf16 outputs are rounded once."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import ends_oracle as O

pytestmark = pytest.mark.gpu
U32, U16 = 2.0 ** -24, 2.0 ** -8
LOW, HIGH, KL = (float(np.float32(x)) for x in (0.2, 0.3, 0.05))


def context(T, flags=0):
    return symi.symi_create(symi.SymiCfg.make(T, 1, 1, 8, 8, 1, 1, 0, "f32"), flags)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def batch(T, V, ld, dtype, seed=0, tau=1.0, ref=True, peak=3.0):
    """Inputs of a step: ratios off the kinks of the loss by 1e-2, so that both sides take the same branch."""
    g = gen(seed)
    z = (torch.randn(T, ld, generator=g, device="cuda") * peak * (1 + torch.arange(T, device="cuda")[:, None] % 4)).to(
        torch.bfloat16 if dtype == "bf16" else torch.float32)
    z[:, V:] = float("nan")            # columns that are not of the vocabulary
    action = torch.randint(0, V, (T,), generator=g, device="cuda")
    best = z[:, :V].float().argmax(1)
    action = torch.where(torch.rand(T, generator=g, device="cuda") < 0.4, best, action).to(torch.int32)
    lp = torch.log_softmax(z[:, :V].double() / tau, 1).gather(1, action.long()[:, None])[:, 0]
    ratio = torch.exp(0.3 * torch.randn(T, generator=g, device="cuda"))
    for kink in (1 - LOW, 1 + HIGH):
        ratio = torch.where((ratio - kink).abs() < 1e-2, kink + 2e-2, ratio)
    weight = torch.rand(T, generator=g, device="cuda") / T
    weight[torch.rand(T, generator=g, device="cuda") < 0.3] = 0
    return dict(z=z, action=action, old=(lp - torch.log(ratio)).float(), ref=(lp + 0.2 * torch.randn(T, generator=g, device="cuda")).float() if ref else None,
                advantage=torch.randn(T, generator=g, device="cuda"), weight=weight)


def call(ctx, hp, b, V, grad=True, out=None, shift=0):
    """logp, stats, dlogits of symi_policy_loss on poisoned outputs."""
    T, ld = b["z"].shape

    def new(n, dtype):
        return torch.full((n + shift,), float("nan"), dtype=dtype, device="cuda")[shift:]

    logp, stats = new(T, torch.float32), new(4, torch.float32)
    dz = out if out is not None else new(T * ld, b["z"].dtype).view(T, ld) if grad else None
    ws = torch.full((symi.symi_policy_workspace_bytes(ctx),), 0xA5, dtype=torch.uint8, device="cuda")
    symi.symi_policy_loss(ctx, hp, b["z"], V, ld, b["action"], b["old"], b["ref"], b["advantage"], b["weight"], logp, stats, dz, ws)
    return logp, stats, dz


def oracle(b, V, hp):
    f = lambda k: None if b[k] is None else Hn.npf(b[k])   # noqa: E731
    return O.policy(f("z"), V, f("action"), f("old"), f("ref"), f("advantage"), f("weight"), hp.clip_low, hp.clip_high,
                    hp.kl_coef, hp.inv_temperature, hp.grad_scale)


def logp_bound(b, V, hp, want):
    Z = np.abs(np.where(np.isfinite(Hn.npf(b["z"])[:, :V]), Hn.npf(b["z"])[:, :V], 0)).max(axis=1) * hp.inv_temperature
    return U32 * (6 * Z + V / 64 + 24 + 2 * np.abs(want))


def check(b, V, hp, logp, stats, dz):
    want = oracle(b, V, hp)
    e = logp_bound(b, V, hp, want["logp"])
    assert (np.abs(Hn.npf(logp) - want["logp"]) <= e).all()
    w, A, r = Hn.npf(b["weight"]).astype(np.float64), np.abs(Hn.npf(b["advantage"])), want["ratio"]
    near = np.abs(want["e"]) + (1 if b["ref"] is not None else 0)
    distance = np.abs(Hn.npf(b["old"]).astype(np.float64)) + np.abs(want["logp"]) + (0 if b["ref"] is None else np.abs(Hn.npf(b["ref"])))
    rel = 2 * e + U32 * (16 + 2 * distance)          # of a ratio
    each = w[:, None] * np.stack([A * r * rel + hp.kl_coef * near * rel, A * r * rel, near * rel, 0 * r], axis=1)
    assert (np.abs(Hn.npf(stats) - want["stats"]) <= each.sum(axis=0) + 8 * U32 * np.abs(want["terms"]).sum(axis=0)).all()
    if dz is None:
        return
    got = Hn.npf(dz)
    assert (got[:, V:] == 0).all()
    size = abs(hp.grad_scale) * hp.inv_temperature * w * (A * r + hp.kl_coef * near)
    part = want["p"].copy()
    live = (w != 0) & (Hn.npf(b["action"]) >= 0) & (Hn.npf(b["action"]) < V)
    part[np.nonzero(live)[0], Hn.npf(b["action"])[live].astype(int)] += 1
    bound = (size * 2 * rel)[:, None] * part + (U16 if dz.dtype == torch.bfloat16 else U32) * np.abs(want["dlogits"][:, :V]) * 1.01 + 1e-38
    assert (got[~live] == 0).all()
    assert (np.abs(got[:, :V] - want["dlogits"][:, :V]) <= bound).all()


SHAPES = [(1, 1, 1), (1, 2, 2), (3, 5, 8), (2, 63, 64), (7, 255, 255), (5, 511, 517), (4, 2047, 2048), (9, 2049, 2049),
          (3, 4099, 4160), (3, 8191, 8191), (5, 8193, 8256), (2, 16385, 16385), (3, 32003, 32003), (2, 50001, 50048), (2, 65537, 65537),
          (3, 70001, 70016), (2, 131073, 131080), (2, 200003, 200003)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,ld", SHAPES)
def test_loss_and_gradient(T, V, ld, dtype):
    for i, (tau, ref) in enumerate(((1.0, True), (0.6, False), (1.7, True))):
        print(f"[policy] {dtype} T={T} V={V} ld={ld} tau={tau} ref={ref}", flush=True)
        ctx = context(T)
        b = batch(T, V, ld, dtype, 7 * i + V, tau, ref)
        if i == 2:
            b["weight"].fill_(1.0)
        hp = symi.SymiPolicy.make(LOW, HIGH, KL if ref else 0.0, tau, (1.0, 3.0, 0.5)[i], dtype)
        logp, stats, dz = call(ctx, hp, b, V)
        check(b, V, hp, logp, stats, dz)
        logp1, stats1, _ = call(ctx, hp, b, V, grad=False)            # the loss alone
        check(b, V, hp, logp1, stats1, None)
        alone = torch.full((T,), float("nan"), device="cuda")
        symi.symi_token_logp(ctx, hp, b["z"], V, ld, b["action"], b["weight"], alone)
        assert torch.equal(alone, logp1)
        again = call(ctx, hp, b, V, shift=1)                          # the same bits, wherever the outputs lie
        assert torch.equal(logp, again[0]) and torch.equal(stats, again[1]) and torch.equal(dz, again[2])
        if ref:                                                       # in place of the logits
            b["z"][:, V:] = 0
            dz2 = call(ctx, hp, b, V, out=b["z"])[2]
            assert torch.equal(dz, dz2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_alignment(dtype):
    T, V, ld = 6, 3001, 3011
    ctx = context(T)
    b = batch(T, V, ld, dtype, 1)
    hp = symi.SymiPolicy.make(LOW, HIGH, KL, dtype=dtype)
    for by in (1, 3):
        flat = torch.zeros(T * ld + by, dtype=b["z"].dtype, device="cuda")
        flat[by:] = b["z"].reshape(-1)
        got = call(ctx, hp, dict(b, z=flat[by:].view(T, ld)), V, shift=by + 1)
        check(b, V, hp, *got)


@pytest.mark.parametrize("V", [700, 9001, 140001])
def test_masked_columns_and_rows(V):
    """-inf columns have no probability; a token that does not count may have anything in its row; the type's lowest value is a
    number like others."""
    T = 8
    for dtype in ("bf16", "f32"):
        ctx = context(T)
        b = batch(T, V, V, dtype, 3)
        b["weight"].fill_(0.25)
        cut = torch.arange(V, device="cuda") % 3 == 1
        cut = cut[None, :] & (torch.arange(V, device="cuda")[None, :] != b["action"][:, None])
        z = b["z"]
        z[0] = torch.where(cut[0], float("-inf"), z[0])
        z[1] = torch.where(cut[1], torch.finfo(z.dtype).min, z[1])
        z[2] = float("nan")
        b["weight"][2] = 0
        z[3] = float("-inf")
        b["action"][3] = -100
        z[4] = float("inf")
        b["action"][4] = V
        z[5] = float("-inf")                       # all of the row but the chosen token
        z[5, b["action"][5].long()] = 1.5
        z[6, :] = 4.0                              # no largest value
        lp = torch.log_softmax(z.double(), 1).gather(1, b["action"].clamp(0, V - 1).long()[:, None])[:, 0]
        live = torch.tensor([0, 1, 5, 6, 7], device="cuda")
        b["old"][live] = lp[live].float() - 0.05
        b["ref"][live] = lp[live].float() + 0.1
        hp = symi.SymiPolicy.make(LOW, HIGH, KL, dtype=dtype)
        out = call(ctx, hp, b, V)
        print(f"[policy] masked {dtype} V={V} {out[0].tolist()}", flush=True)
        bound_z = z.clone()
        bound_z[1] = torch.where(cut[1], 0, z[1])  # far below the largest: whatever their error, their power of two is 0
        want = oracle(b, V, hp)
        e = logp_bound(dict(b, z=bound_z), V, hp, want["logp"])
        assert (np.abs(Hn.npf(out[0]) - want["logp"]) <= e).all()
        got = Hn.npf(out[2])
        assert np.isfinite(got).all() and np.isfinite(Hn.npf(out[1])).all()
        assert (got[2:5] == 0).all() and (Hn.npf(out[0])[2:5] == 0).all()
        assert (got[0][Hn.npf(cut[0]).astype(bool)] == 0).all() and (got[1][Hn.npf(cut[1]).astype(bool)] == 0).all()
        # a row without any probability left, or with an infinite one, has no log probability: NaN in it alone
        for bad in (float("-inf"), float("nan"), float("inf")):
            z2 = z.clone()
            z2[7] = bad
            logp, stats, dz = call(ctx, hp, dict(b, z=z2), V)
            assert logp[7].isnan() and stats[0].isnan() and dz[7].isnan().all()
            assert not logp[:7].isnan().any() and not dz[:7].isnan().any()
            assert torch.equal(dz[:7], out[2][:7])


def test_kl_near_zero_and_far():
    """exp(x) - x - 1 of x from 1e-6 to 8: relative errors of 2^-20 and the error of x itself."""
    x = torch.cat([torch.logspace(-6, 0.9, 64, device="cuda"), -torch.logspace(-6, 0.9, 64, device="cuda")])
    for one in x.tolist():
        ctx = context(1)
        z = torch.zeros(1, 2, device="cuda")                 # logp = -ln 2
        old = torch.full((1,), -float(np.log(2)), device="cuda")
        ref = torch.tensor([-np.log(2) + one], device="cuda", dtype=torch.float32)
        hp = symi.SymiPolicy.make(LOW, HIGH, 1.0, dtype="f32")
        b = dict(z=z, action=torch.zeros(1, dtype=torch.int32, device="cuda"), old=old, ref=ref, advantage=torch.zeros(1, device="cuda"),
                 weight=torch.ones(1, device="cuda"))
        logp, stats, _ = call(ctx, hp, b, 2, grad=False)
        far = float(ref.double()) - float(logp.double())     # of the kernel's own logp: the series is what is looked at
        want = np.expm1(far) - far
        tol = 2.0 ** -20 * want + 2 * U32 * abs(far) * max(abs(np.expm1(far)), abs(far)) + 4 * U32 * abs(np.expm1(far))
        assert abs(float(stats[2]) - want) <= tol, (one, float(stats[2]), want)


def test_terms_without_a_say_may_be_infinite():
    """A KL that is only looked at (coefficient 0) and a ratio without an advantage: neither makes the loss or the gradient infinite."""
    T, V = 3, 40
    ctx = context(T)
    b = batch(T, V, V, "f32", 9)
    b["weight"].fill_(1.0)
    b["ref"][0] = 300.0                       # exp(300 - logp) is infinite
    b["old"][1], b["advantage"][1] = -400.0, 0.0
    hp = symi.SymiPolicy.make(LOW, HIGH, 0.0, dtype="f32")
    logp, stats, dz = call(ctx, hp, b, V)
    assert stats[2].isinf() and stats[[0, 1, 3]].isfinite().all() and dz.isfinite().all()
    assert not dz[1].any()
    rest = {k: v.clone() for k, v in b.items()}
    rest["ref"][0], rest["old"][1] = 0.0, 0.0
    want = oracle(rest, V, hp)
    assert np.abs(Hn.npf(stats)[:2] - want["stats"][:2]).max() <= 1e-4 * np.abs(want["terms"]).sum()
    assert np.abs(Hn.npf(dz) - want["dlogits"]).max() <= 1e-4


def test_gradient_against_differences():
    """Directional derivatives: (loss(z + h D) - loss(z - h D)) / 2 h of the binary64 loss = <dlogits, D>, for the kernel's
    gradient of fp32 logits (whose errors are below 1e-4 of the summands' sizes); h^2 / 6 of the third derivative is below 1e-7."""
    T, V = 12, 257
    ctx = context(T)
    b = batch(T, V, V, "f32", 5)
    hp = symi.SymiPolicy.make(LOW, HIGH, KL, 0.8, 1.0, "f32")
    dz = Hn.npf(call(ctx, hp, b, V)[2]).astype(np.float64)
    z = Hn.npf(b["z"]).astype(np.float64)
    rng = np.random.default_rng(0)
    for _ in range(8):
        D = rng.standard_normal(z.shape)
        loss = [O.policy(z + s * 1e-4 * D, V, *(Hn.npf(b[k]) for k in ("action", "old", "ref", "advantage", "weight")), hp.clip_low,
                         hp.clip_high, hp.kl_coef, hp.inv_temperature)["stats"][0] for s in (1, -1)]
        assert abs((loss[0] - loss[1]) / 2e-4 - (dz * D).sum()) <= 1e-4 * np.abs(dz * D).sum() + 1e-7


def test_offsets_beyond_32_bits():
    """More than 2^31 logits: the last rows."""
    T, V, ld = 17000, 131000, 131072
    ctx = context(T)
    z = torch.zeros(T, ld, dtype=torch.bfloat16, device="cuda")
    z[-3:] = torch.randn(3, ld, generator=gen(1), device="cuda").to(torch.bfloat16)
    weight = torch.zeros(T, device="cuda")
    weight[-3:] = 1.0
    weight[0] = 1.0
    action = torch.full((T,), 17, dtype=torch.int32, device="cuda")
    hp = symi.SymiPolicy.make(LOW, HIGH, dtype="bf16")
    flat = torch.zeros(T, device="cuda")
    b = dict(z=z, action=action, old=flat - 11.0, ref=None, advantage=flat + 1.0, weight=weight)
    logp, stats, dz = call(ctx, hp, b, V)
    small = {k: None if v is None else torch.cat([v[:1], v[-3:]]) for k, v in b.items()}
    ctx4 = context(4)
    logp4, stats4, dz4 = call(ctx4, hp, small, V)
    check(small, V, hp, logp4, stats4, dz4)
    assert torch.equal(logp[-3:], logp4[1:]) and torch.equal(dz[-3:], dz4[1:]) and torch.equal(dz[0], dz4[0])
    assert torch.equal(stats, stats4) and not dz[1:-3].any()


def test_many_short_rows_and_none():
    T, V = 100003, 3
    ctx = context(T)
    b = batch(T, V, 4, "f32", 2)
    hp = symi.SymiPolicy.make(LOW, HIGH, KL, dtype="f32")
    check(b, V, hp, *call(ctx, hp, b, V))
    none = {k: v[:0] for k, v in b.items()}
    ctx0 = context(0)
    logp, stats, dz = call(ctx0, hp, none, V)
    assert not stats.any() and dz.numel() == 0
    symi.symi_token_logp(ctx0, hp, none["z"], V, 4, none["action"], None, logp)


def test_another_stream_and_a_graph():
    T, V, ld = 300, 5003, 5056
    ctx = context(T)
    hp = symi.SymiPolicy.make(LOW, HIGH, KL, dtype="bf16")
    b = batch(T, V, ld, "bf16", 1)
    want = call(ctx, hp, b, V)
    logp, stats, dz = torch.empty(T, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(b["z"])
    ws = torch.empty(symi.symi_policy_workspace_bytes(ctx), dtype=torch.uint8, device="cuda")

    def one():
        symi.symi_policy_loss(ctx, hp, b["z"], V, ld, b["action"], b["old"], b["ref"], b["advantage"], b["weight"], logp, stats, dz, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        one()
    side.synchronize()
    assert torch.equal(logp, want[0]) and torch.equal(stats, want[1]) and torch.equal(dz, want[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    for i in range(4):
        for k, v in batch(T, V, ld, "bf16", 20 + i).items():
            b[k].copy_(v)
        want = call(ctx, hp, b, V)
        dz.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(logp, want[0]) and torch.equal(stats, want[1]) and torch.equal(dz, want[2])


def test_refusals():
    T, V, ld = 4, 10, 12
    ctx = context(T)
    b = batch(T, V, ld, "bf16", 1)
    hp = symi.SymiPolicy.make(LOW, HIGH, KL, dtype="bf16")
    for change in (dict(z=b["z"].float()), dict(action=b["action"].long()), dict(old=b["old"].double()), dict(weight=b["weight"][:-1]),
                   dict(ref=None), dict(advantage=b["advantage"].cpu())):
        with pytest.raises(symi.SymiError):
            call(ctx, hp, dict(b, **change), V)
    with pytest.raises(symi.SymiError, match="ld"):
        call(ctx, hp, b, ld + 1)
    with pytest.raises(symi.SymiError):
        call(ctx, hp, b, 0)
    for kw in (dict(clip_low=1.5), dict(clip_low=-0.1), dict(clip_high=-0.1), dict(kl_coef=-1.0), dict(temperature=-1.0),
               dict(temperature=float("inf")), dict(clip_low=float("nan")), dict(kl_coef=float("nan")), dict(grad_scale=float("nan"))):
        bad = symi.SymiPolicy.make(**{**dict(clip_low=LOW, clip_high=HIGH, kl_coef=KL, dtype="bf16"), **kw})
        with pytest.raises(symi.SymiError):
            call(ctx, bad, b, V)
    with pytest.raises(symi.SymiError):
        symi.symi_token_logp(ctx, hp, b["z"], V, ld, b["action"], None, torch.empty(T - 1, device="cuda"))
    L = symi.lib()
    import ctypes
    assert L.symi_token_logp(ctx.ptr, ctypes.byref(hp), None, V, ld, None, None, None, None) == -1 and "NULL" in symi.symi_last_error()
    assert L.symi_policy_loss(ctx.ptr, None, None, V, ld, None, None, None, None, None, None, None, None, None, None) == -1
