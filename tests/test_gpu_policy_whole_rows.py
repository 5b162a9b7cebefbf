"""Rows of logits in workgroups of several wavefronts, as batches that are too large to be split over workgroups take them: every
length class with its gradient, in both types, beginning anywhere, in place of the logits too; and the loss without a gradient of
many long rows.  Against binary64 with the bounds of test_gpu_policy.py."""
import pytest
import torch

import paper_2504_19925_amd as symi
from tests.test_gpu_policy import HIGH, KL, LOW, U16, U32, batch, call, context

pytestmark = pytest.mark.gpu
SPLIT_ROWS = 256       # a batch of more rows is not split, whatever their length
# 16-byte pieces of a row: both ends of what 128, 256, 512 and 1024 threads with 4 to 16 pieces each take; from 8193 on rows are read again
# in part, as pieces beyond 1024 x 8 (up to 12800) and beyond 1024 x 16 do not stay
PIECES = [257, 512, 513, 1024, 1025, 2048, 2049, 3000, 3001, 4608, 4609, 8192, 8193, 10001, 12800, 12801, 16384, 16385, 20011]


def reference(b, V, hp):
    """The definition in 64 bits on the device: logp, terms [T, 4], p, the slope of logp, and the errors of logp and of a ratio."""
    z = b["z"][:, :V].double() * hp.inv_temperature
    a = b["action"].long()[:, None]
    live = b["weight"] != 0
    lp = torch.log_softmax(z, 1).gather(1, a)[:, 0]
    e = U32 * (6 * z.abs().amax(1) + V / 64 + 24 + 2 * lp.abs())
    A, w = b["advantage"].double(), b["weight"].double()
    r = torch.exp(lp - b["old"].double())
    bounded = r.clamp(1 - float(hp.clip_low), 1 + float(hp.clip_high))
    clipped = bounded * A < r * A
    gain = -torch.minimum(r * A, bounded * A)
    far = b["ref"].double() - lp if b["ref"] is not None else torch.zeros_like(lp)
    kl = torch.expm1(far) - far
    slope = torch.where(clipped, 0.0, -A * r) - hp.kl_coef * torch.expm1(far)
    terms = torch.stack([w * (gain + hp.kl_coef * kl), w * gain, w * kl, w * clipped], 1)
    distance = b["old"].double().abs() + lp.abs() + (0 if b["ref"] is None else b["ref"].double().abs())
    rel = 2 * e + U32 * (16 + 2 * distance)
    near = torch.expm1(far).abs() + (1 if b["ref"] is not None else 0)
    each = w[:, None] * torch.stack([A.abs() * r * rel + hp.kl_coef * near * rel, A.abs() * r * rel, near * rel, 0 * r], 1)
    return dict(z=z, a=a, live=live, lp=torch.where(live, lp, 0.0), e=e, slope=slope, terms=terms, rel=rel, each=each,
                size=hp.grad_scale * hp.inv_temperature * w * (A.abs() * r + hp.kl_coef * near))


def check(b, V, hp, R, logp, stats, dz):
    assert ((logp.double() - R["lp"]).abs() <= R["e"]).all()
    assert ((stats.double() - R["terms"].sum(0)).abs() <= R["each"].sum(0) + 8 * U32 * R["terms"].abs().sum(0)).all()
    if dz is None:
        return
    assert not dz[:, V:].any() and not dz[~R["live"]].any()
    p = torch.softmax(R["z"], 1)
    u = (hp.grad_scale * hp.inv_temperature * b["weight"].double() * R["slope"])[:, None]
    want = (-u * p).scatter_add_(1, R["a"], u)
    bound = (R["size"] * 2 * R["rel"])[:, None] * p.scatter_add_(1, R["a"], torch.ones_like(u)) + \
        (U16 if dz.dtype == torch.bfloat16 else U32) * 1.01 * want.abs() + 1e-38
    assert ((dz[:, :V].double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pieces", PIECES)
def test_gradient(pieces, dtype):
    T, n = SPLIT_ROWS + 4, 8 if dtype == "bf16" else 4
    for V, ld, by in ((pieces * n, pieces * n, 0), (pieces * n - 3, pieces * n - 3, 1), (pieces * n - n + 1, pieces * n + 5, 3)):
        print(f"[policy] {dtype} pieces={pieces} V={V} ld={ld} by={by}", flush=True)
        hp = symi.SymiPolicy.make(LOW, HIGH, KL, 0.9, 2.0, dtype)
        b = batch(T, V, ld, dtype, pieces, 0.9)
        b["z"][:, V:] = 0
        flat = torch.zeros(T * ld + by, dtype=b["z"].dtype, device="cuda")
        flat[by:] = b["z"].reshape(-1)
        b["z"] = flat[by:].view(T, ld)
        ctx, R = context(T), reference(b, V, hp)
        logp, stats, dz = call(ctx, hp, b, V, shift=2)
        check(b, V, hp, R, logp, stats, dz)
        logp2, stats2, dz2 = call(ctx, hp, b, V, out=b["z"])            # in place of the logits
        assert torch.equal(logp, logp2) and torch.equal(stats, stats2) and torch.equal(dz, dz2)
        del R, dz, dz2, flat, b


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pieces", [1025, 2048, 2049, 5003, 9001])
def test_loss_alone_of_many_rows(pieces, dtype):
    T, n = 4 * torch.cuda.get_device_properties(0).multi_processor_count + 1, 8 if dtype == "bf16" else 4
    for V, ld, by in ((pieces * n, pieces * n, 0), (pieces * n - 3, pieces * n - 3, 1)):
        print(f"[policy] {dtype} pieces={pieces} V={V} ld={ld} by={by}", flush=True)
        hp = symi.SymiPolicy.make(LOW, HIGH, KL, 0.9, 1.0, dtype)
        b = batch(T, V, ld, dtype, pieces, 0.9)
        flat = torch.zeros(T * ld + by, dtype=b["z"].dtype, device="cuda")
        flat[by:] = b["z"].reshape(-1)
        b["z"] = flat[by:].view(T, ld)
        ctx, R = context(T), reference(b, V, hp)
        logp, stats, _ = call(ctx, hp, b, V, grad=False)
        check(b, V, hp, R, logp, stats, None)
        alone = torch.full((T,), float("nan"), device="cuda")
        symi.symi_token_logp(ctx, hp, b["z"], V, ld, b["action"], b["weight"], alone)
        assert torch.equal(alone, logp)
        del R, flat, b
