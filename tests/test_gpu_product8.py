"""Products of 8-bit values over slots, and the experts made of them, against binary64.

Where codes are small whole numbers and powers differ by little, every partial sum has fewer than 24 bits, so fp32 sums are exact in any order and
results have to be equal.  Elsewhere a sum of n products in any order, also one that cuts digits off in place of rounding, is within
2 n U32 of the sum of their sizes.  The 8-bit matrix instruction of bf16 contexts drops more: of 8 neighbouring products each loses less than 2^-13
of the largest, 7 of them at most 7 2^-13 of the sum of the sizes."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import way_oracle as O

pytestmark = pytest.mark.gpu
U32, U16 = 2.0 ** -24, 2.0 ** -8


def context(T, S, dtype, d=8, f=8, k=1, flags=0):
    return symi.symi_create(symi.SymiCfg.make(T, min(S, 1024), k, d, f, S, 1, 0, dtype), flags)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def offsets_of(counts):
    at = np.concatenate([[0], np.cumsum(counts)])
    return at, torch.from_numpy(at.astype(np.int32)).cuda()


def whole(seed, *shape):
    """Values whose codes are small whole numbers, in blocks of different powers."""
    g = gen(seed)
    x = torch.randint(-3, 4, shape, generator=g, device="cuda").float()
    x *= 2.0 ** torch.randint(-2, 3, shape[:-1] + (1,), generator=g, device="cuda")
    return x


def quant(ctx, X, block):
    groups, rows, n = X.shape
    q = torch.empty(groups, rows, symi.symi_pitch8(n), dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.empty(groups, -(-rows // block), symi.symi_scale_pitch8(n), dtype=torch.uint8, device="cuda")
    symi.symi_quant8(ctx, X.to(ctx.torch_dtype), groups, rows, n, block, q, s)
    back = torch.empty(X.shape, dtype=torch.float32, device="cuda")
    other = context(1, 1, "f32")
    symi.symi_dequant8(other, q, s, groups, rows, n, block, back)
    return q, s, Hn.npf(back).astype(np.float64)


def scratch(ctx):
    return torch.full((symi.symi_workspace8_bytes(ctx),), 0xA5, dtype=torch.uint8, device="cuda")


def check(counts, R, n, dtype, extra=0, exact=True):
    """extra: rows behind the last slot."""
    A, S = sum(counts) + extra, len(counts)
    ctx = context(A, S, dtype)
    print(f"[product8] {dtype} rows {counts} + {extra} R={R} n={n} exact={exact}", flush=True)
    at, offs = offsets_of(counts)
    make = whole if exact else lambda seed, *s: torch.randn(*s, generator=gen(seed), device="cuda") * torch.exp(torch.randn(*s[:-1], 1, generator=gen(seed + 1), device="cuda"))
    aq, a_s, a = quant(ctx, make(1, 1, A, n), 1)
    wq, w_s, w = quant(ctx, make(2, S, R, n), 128)
    Y = torch.full((A, R), 640.0, dtype=ctx.torch_dtype, device="cuda")
    ws = scratch(ctx)
    symi.symi_product8(ctx, aq, a_s, offs, wq, w_s, R, n, Y, ws)
    want, size = O.product(a[0], w, at)
    got = Hn.npf(Y).astype(np.float64)
    assert (got[at[-1]:] == 640.0).all()
    got, want, size = got[:at[-1]], want[:at[-1]], size[:at[-1]]
    half = U16 if dtype == "bf16" else 0.0
    if exact and dtype == "f32":
        assert (got == want).all()
    elif exact:
        assert (got == Hn.npf(torch.from_numpy(want).float().to(torch.bfloat16))).all()
    else:
        dropped = 7 * 2.0 ** -13 if dtype == "bf16" else 0.0
        assert (np.abs(got - want) <= (2 * n * U32 + dropped) * size * (1 + half) + half * np.abs(want)).all()
        if dtype == "f32" and got.size:     # and on the whole much nearer: rounding errors of n / 16 steps or more would be a wrong way to sum
            assert np.linalg.norm(got - want) <= (2 * np.sqrt(n) + 4) * U32 * np.linalg.norm(size)
    return ctx, aq, a_s, offs, wq, w_s, Y


COUNTS = [[1], [5, 0, 3], [16, 17, 1, 0, 15], [127, 128, 129], [255, 0, 0, 256, 257], [0, 0], [300, 2, 64, 63, 65, 32, 33, 31]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("R,n", [(8, 8), (128, 128), (264, 136), (320, 1160)])
def test_product(counts, R, n, dtype):
    check(counts, R, n, dtype, extra=3)
    check(counts, R, n, dtype, exact=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,R,n", [([1000, 24, 513], 776, 640), ([700, 0, 90, 1500], 520, 4104), ([3, 1, 2, 0, 9], 4104, 2056), ([2], 264, 16392), ([40, 7], 1032, 512)], ids=str)
def test_larger_products(counts, R, n, dtype):
    check(counts, R, n, dtype)
    check(counts, R, n, dtype, exact=False)


def test_many_slots():
    rng = np.random.default_rng(1)
    check(rng.integers(0, 4, 300).tolist(), 136, 264, "f32")
    check((rng.integers(0, 2, 1100) * rng.integers(0, 40, 1100)).tolist(), 72, 136, "bf16")


@pytest.mark.parametrize("counts", [[3, 20], [300, 200]], ids=str)
def test_rows_and_weights_that_are_not_finite(counts):
    """A NaN reaches the results of its row, or of its weight's column in its slot, and no others."""
    ctx, aq, a_s, offs, wq, w_s, Y = check(counts, 72, 264, "f32")
    clean = Y.clone()
    aq.view(torch.uint8)[0, 1, 200] = 0x7F
    wq.view(torch.uint8)[1, 40, 7] = 0xFF
    symi.symi_product8(ctx, aq, a_s, offs, wq, w_s, 72, 264, Y, scratch(ctx))
    bad = torch.zeros_like(Y, dtype=torch.bool)
    bad[1], bad[counts[0]:, 40] = True, True
    assert torch.isnan(Y[bad]).all() and torch.equal(Y[~bad], clean[~bad])


def test_powers_from_end_to_end():
    """Every byte of a scale counts as its power of two, also where one operand's makes up for the other's."""
    n, R = 128, 256
    A = 255
    ctx = context(A, 1, "f32")
    a = torch.zeros(1, A, n, device="cuda")
    a[0, :, 0] = 1.5
    q = torch.zeros(1, A, 128, dtype=torch.uint8, device="cuda")
    q[0, :, 0] = 0x3C            # 1.5
    s = torch.zeros(1, A, 4, dtype=torch.uint8, device="cuda")
    s[0, :, 0] = torch.arange(A, device="cuda")
    _, offs = offsets_of([A])
    for power in (0, 1, 60, 127, 200, 254):
        wq = torch.zeros(1, R, 128, dtype=torch.uint8, device="cuda")
        wq[0, :, 0] = 0x38       # 1
        w_s = torch.zeros(1, 2, 4, dtype=torch.uint8, device="cuda")
        w_s[0, :, 0] = power
        Y = torch.full((A, R), 640.0, device="cuda")
        symi.symi_product8(ctx, q.view(torch.float8_e4m3fn), s, offs, wq.view(torch.float8_e4m3fn), w_s, R, n, Y, scratch(ctx))
        with np.errstate(over="ignore"):
            want = (1.5 * 2.0 ** (np.arange(A) + power - 254.0)).astype(np.float32)
        got = Y[:, 0].cpu().numpy()
        normal = (want >= 2.0 ** -126) | (want == 0)
        assert (got[normal] == want[normal]).all() and (np.abs(got[~normal] - want[~normal]) <= 2.0 ** -126).all()


# ---- the experts

def near_codes(h, eps):
    """How far a hidden unit's value in 8 bits may move where it is within eps of h, relatively: over its own move and its block's largest value's."""
    base = O.values(*O.quant(h, 1), 1)
    off = np.zeros_like(h)
    blocks = -(-h.shape[1] // 128)
    pad = np.pad(np.abs(h), ((0, 0), (0, blocks * 128 - h.shape[1]))).reshape(len(h), blocks, 128).max(axis=2)
    for move_top in (1 - eps, 1 + eps):
        s = np.vectorize(O.power)(pad * move_top)
        scale = np.repeat(2.0 ** (s - 127.0), 128, axis=1)[:, :h.shape[1]]
        for move in (1 - eps, 1, 1 + eps):
            off = np.maximum(off, np.abs(O.to_e4m3(np.clip(h * move / scale, -448, 448)) * scale - base))
    return base, off


def check_experts(counts, d, f, extra=0, keep=True, k=1):
    S = len(counts)
    A = sum(counts) + extra
    A += -A % k
    ctx = context(A // k, S, "bf16", d, f, k)
    print(f"[expert8] rows {counts} + {extra} d={d} f={f} keep={keep}", flush=True)
    at, offs = offsets_of(counts)
    # u and v come out of sums that are exact, of a size where the gate bends
    X = whole(1, A, d).to(torch.bfloat16)
    _, _, x = quant(ctx, X[None].float(), 1)
    w1q, w1s, w1 = quant(ctx, whole(2, S, 2 * f, d) * 2.0 ** -round(np.log2(8 * np.sqrt(d))), 128)
    w2q, w2s, w2 = quant(ctx, torch.randn(S, d, f, generator=gen(3), device="cuda"), 128)
    new = lambda *s: torch.full(s, 640.0, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    UV, H, Yp = new(A, 2 * f) if keep else None, new(A, f) if keep else None, new(A, d)
    ws = scratch(ctx)
    symi.symi_expert_fwd8(ctx, X, offs, w1q, w1s, w2q, w2s, UV, H, Yp, ws)
    n = at[-1]
    for t in (UV, H, Yp):
        assert t is None or (t[n:] == 640.0).all()
    uv, _ = O.product(x[0], w1, at)
    uv = uv[:n]
    h = O.silu_product(uv[:, :f], uv[:, f:])
    # an exponential of |u| <= 2^7 with a relative error of (2 |u| + 8) roundings, a reciprocal and four products
    eps = (2 * min(np.abs(uv).max(), 128) + 24) * U32 if n else 0
    if keep:
        assert (Hn.npf(UV)[:n] == Hn.npf(torch.from_numpy(uv).float().to(torch.bfloat16))).all()
        assert (np.abs(Hn.npf(H)[:n] - h) <= (U16 * 1.01 + eps) * np.abs(h) + 2.0 ** -133).all()
    if n:
        base, off = near_codes(h, eps)
        y, size = O.product(base, w2, at)
        slack = sum_over_slots(off, w2, at)
        assert (np.abs(Hn.npf(Yp)[:n] - y) <= slack + (2 * f * U32 + 7 * 2.0 ** -13) * size * 1.01 + U16 * 1.01 * (np.abs(y) + slack)).all()
    return ctx, (X, offs, w1q, w1s, w2q, w2s), (UV, H, Yp)


def sum_over_slots(off, w, at):
    out = np.zeros((at[-1], w.shape[1]))
    for p in range(len(w)):
        rows = slice(at[p], at[p + 1])
        out[rows] = off[rows] @ np.abs(w[p]).T
    return out


@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("d,f", [(8, 8), (128, 256), (264, 136), (520, 1416)])
def test_experts(counts, d, f):
    check_experts(counts, d, f, extra=2)
    check_experts(counts, d, f, keep=False, k=min(2, len(counts)))


@pytest.mark.parametrize("counts,d,f", [([900, 0, 260, 31], 1032, 520), ([2, 1, 1], 1160, 2744)], ids=str)
def test_larger_experts(counts, d, f):
    full = check_experts(counts, d, f)
    only = check_experts(counts, d, f, keep=False)
    assert torch.equal(full[2][2], only[2][2])


def test_refusals():
    ctx = context(4, 2, "bf16", 64, 32)
    codes = lambda *s: torch.zeros(*s, dtype=torch.float8_e4m3fn, device="cuda")   # noqa: E731
    scales = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")   # noqa: E731
    offs = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    a, a_s, w, w_s, ws = codes(4, 128), scales(4, 4), codes(2, 64, 128), scales(2, 1, 4), scratch(ctx)
    Y = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    symi.symi_product8(ctx, a, a_s, offs, w, w_s, 64, 64, Y, ws)
    for R, n, said in ((64, 60, "multiple of 8"), (60, 64, "R must be"), (0, 64, "R must be")):
        with pytest.raises(symi.SymiError, match=said):
            symi.symi_product8(ctx, a, a_s, offs, w, w_s, R, n, Y, ws)
    big = torch.zeros(2 * 64 * 128 + 64, dtype=torch.uint8, device="cuda")
    with pytest.raises(symi.SymiError, match="16-byte"):
        symi.symi_product8(ctx, a, a_s, offs, big[8:8 + 2 * 64 * 128].view(torch.float8_e4m3fn), w_s, 64, 64, Y, ws)
    with pytest.raises(symi.SymiError, match="4-byte"):
        symi.symi_product8(ctx, a, big[2:2 + 16], offs, w, w_s, 64, 64, Y, ws)
    X, UV, H = (torch.zeros(4, n, dtype=torch.bfloat16, device="cuda") for n in (64, 64, 32))
    w2, w2_s = codes(2, 64, 128), scales(2, 1, 4)
    symi.symi_expert_fwd8(ctx, X, offs, w, w_s, w2, w2_s, UV, H, Y, ws)
    for uv, h in ((None, H), (UV, None)):
        with pytest.raises(symi.SymiError, match="both or neither"):
            symi.symi_expert_fwd8(ctx, X, offs, w, w_s, w2, w2_s, uv, h, Y, ws)
    single = context(4, 2, "f32", 64, 32)
    with pytest.raises(symi.SymiError, match="bf16 context"):
        symi.symi_expert_fwd8(single, X.float(), offs, w, w_s, w2, w2_s, None, None, Y.float(), scratch(single))
    none = context(0, 2, "bf16", 64, 32)
    e = torch.empty(0, dtype=torch.bfloat16, device="cuda")
    symi.symi_expert_fwd8(none, e, offs, w, w_s, w2, w2_s, None, None, e, scratch(none))
    symi.symi_product8(none, codes(0), scales(0), offs, w, w_s, 64, 64, e, scratch(none))
    torch.cuda.synchronize()


@pytest.mark.parametrize("A", [3, 40], ids=["thin", "large"])
def test_weights_beyond_four_gigabytes(A):
    """Offsets into a slot's weight pass 32 bits: columns on both sides of that, and the last ones."""
    n, R = 4104, 1040008                     # 4224 bytes a row: 4.39e9
    ctx = context(A, 1, "bf16")
    p, sp = symi.symi_pitch8(n), symi.symi_scale_pitch8(n)
    assert p * R > 2 ** 32
    g = gen(1)
    aq, a_s, a = quant(ctx, whole(1, 1, A, n), 1)
    wq = torch.zeros(1, R, p, dtype=torch.uint8, device="cuda")
    w_s = torch.full((1, -(-R // 128), sp), 127, dtype=torch.uint8, device="cuda")
    at = sorted({0, 127, 2 ** 32 // p - 1, 2 ** 32 // p, 2 ** 32 // p + 1, 2 ** 31 // p + 1, R - 9, R - 1})
    few = torch.randint(-3, 4, (len(at), n), generator=g, device="cuda").float()
    wq[0, at, :n] = few.to(torch.float8_e4m3fn).view(torch.uint8)
    Y = torch.full((A, R), 640.0, dtype=torch.bfloat16, device="cuda")
    _, offs = offsets_of([A])
    symi.symi_product8(ctx, aq, a_s, offs, wq.view(torch.float8_e4m3fn), w_s, R, n, Y, scratch(ctx))
    want = torch.from_numpy(a[0] @ Hn.npf(few).astype(np.float64).T).float().to(torch.bfloat16).cuda()
    assert torch.equal(Y[:, at], want)
    Y[:, at] = 0
    assert not Y.any()


def test_more_columns_than_a_launch_has_are_refused():
    L, some = symi.lib(), 256                # refused before anything is read
    for dtype in ("bf16", "f32"):
        ctx = context(1, 1, dtype)
        assert L.symi_product8(ctx.ptr, some, some, some, some, some, 65535 * 64 + 8, 1024, some, some, None) == -2
        assert "tiles" in symi.symi_last_error()
