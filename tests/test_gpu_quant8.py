"""Values in 8 bits, bit for bit against binary64: powers of two and one rounding leave nothing to tolerate."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import way_oracle as O

pytestmark = pytest.mark.gpu


def context(dtype, T=1, S=1, d=8, f=8, k=1, flags=0):
    return symi.symi_create(symi.SymiCfg.make(T, S, k, d, f, S, 1, 0, dtype), flags)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def room(groups, rows, n, block):
    """Codes and scales, filled with what must not stay."""
    q = torch.full((groups, rows, symi.symi_pitch8(n)), 0x55, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    return q, torch.full((groups, -(-rows // block), symi.symi_scale_pitch8(n)), 0x55, dtype=torch.uint8, device="cuda")


def check(ctx, X, block):
    groups, rows, n = X.shape
    q, s = room(groups, rows, n, block)
    symi.symi_quant8(ctx, X, groups, rows, n, block, q, s)
    back = torch.full_like(X, 3.0)
    symi.symi_dequant8(ctx, q, s, groups, rows, n, block, back)
    blocks = -(-n // 128)
    assert not q[:, :, n:].view(torch.uint8).any() and not s[:, :, blocks:].any()
    x, codes, scales, got = Hn.npf(X), q.float().cpu().numpy(), s.cpu().numpy(), Hn.npf(back)
    for g in range(groups):
        want_q, want_s = O.quant(x[g], block)
        assert (scales[g, :, :blocks] == want_s).all()
        np.testing.assert_array_equal(codes[g, :, :n], want_q)
        with np.errstate(all="ignore"):
            v = O.values(want_q, want_s, block).astype(np.float32)
        np.testing.assert_array_equal(got[g], v if X.dtype == torch.float32 else Hn.npf(torch.from_numpy(v).to(torch.bfloat16)))
    return q, s


SIZES = [(1, 1, 8, 1), (1, 1, 4096, 1), (1, 17, 136, 1), (3, 5, 520, 1), (1, 129, 1160, 1), (1, 3, 40008, 1), (1, 8, 8, 128), (2, 128, 128, 128),
         (3, 130, 264, 128), (1, 1, 1024, 128), (5, 127, 72, 128), (2, 400, 1160, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("groups,rows,n,block", SIZES)
def test_codes_and_values(groups, rows, n, block, dtype):
    ctx = context(dtype)
    print(f"[quant8] {dtype} {groups} x {rows} x {n} block {block}", flush=True)
    x = torch.randn(groups, rows, n, generator=gen(1), device="cuda") * torch.exp(2 * torch.randn(groups, rows, 1, generator=gen(2), device="cuda"))
    x[:, ::3] = torch.randint(-64, 65, x[:, ::3].shape, generator=gen(3), device="cuda") * 0.25      # ties between two codes
    if rows > 1:
        x[:, 1] = 0
    check(ctx, x.to(ctx.torch_dtype), block)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [1, 128])
def test_every_power_its_borders_and_what_is_not_finite(dtype, block):
    ctx = context(dtype)
    n, rows = 256, 256 if block == 1 else 256 * 128
    x = torch.zeros(rows, n)
    tiny = torch.finfo(torch.float32).smallest_normal
    for e in range(256):     # the largest value of a block just below, at and above 448 * 2 ^ i, from denormal numbers to the largest
        top = 2.0 ** (e - 149) * 1.75 if e < 240 else 2.0 ** (e - 128 - 0) * 1.75 if e < 255 else torch.finfo(torch.float32).max
        if not np.isfinite(np.float32(top)):
            top = torch.finfo(torch.float32).max
        r = e * (1 if block == 1 else 128)
        x[r, 3], x[r, 5] = top, -top / 3
        with np.errstate(over="ignore"):
            x[r, 130] = float(np.nextafter(np.float32(top), np.float32(np.inf if e % 2 else 0)))
        x[r, 200] = tiny * (e % 3)
    x = torch.nan_to_num(x, posinf=torch.finfo(torch.bfloat16).max)
    X = x.to(ctx.torch_dtype).cuda()
    X = torch.where(torch.isfinite(X), X, 1.0)
    check(ctx, X[None], block)
    X[2, 0], X[2, 1], X[2, 131], X[4] = float("nan"), float("inf"), -float("inf"), float("nan")
    check(ctx, X[None], block)


def test_any_alignment_of_values_and_refusals():
    ctx = context("bf16")
    x = torch.randn(1, 40, 200, generator=gen(1), device="cuda").to(torch.bfloat16)
    for block in (1, 128):
        q, s = check(ctx, x, block)
        flat = torch.empty(x.numel() + 3, dtype=x.dtype, device="cuda")
        flat[3:] = x.view(-1)
        q2, s2 = room(1, 40, 200, block)
        symi.symi_quant8(ctx, flat[3:], 1, 40, 200, block, q2, s2)
        assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s, s2)
        back, moved = torch.empty_like(x), torch.zeros_like(flat)
        symi.symi_dequant8(ctx, q, s, 1, 40, 200, block, back)
        symi.symi_dequant8(ctx, q, s, 1, 40, 200, block, moved[3:])
        assert torch.equal(moved[3:], back.view(-1))
    big = torch.empty(40 * 256 + 16, dtype=torch.uint8, device="cuda")
    q, s = room(1, 40, 200, 1)
    for bad_q, bad_s, said in ((big[8:8 + 40 * 256].view(torch.float8_e4m3fn), s, "16-byte"), (q, big[1:1 + 160], "4-byte")):
        with pytest.raises(symi.SymiError, match=said):
            symi.symi_quant8(ctx, x, 1, 40, 200, 1, bad_q, bad_s)
        with pytest.raises(symi.SymiError, match=said):
            symi.symi_dequant8(ctx, bad_q, bad_s, 1, 40, 200, 1, x)
    for groups, rows, n, block, said in ((1, 40, 100, 1, "multiple of 8"), (1, 40, 0, 1, "multiple of 8"), (-1, 40, 200, 1, "negative"),
                                         (1, -1, 200, 1, "negative"), (1, 40, 200, 2, "block"), (1, 40, 200, 0, "block")):
        with pytest.raises(symi.SymiError, match=said):
            symi.symi_quant8(ctx, x, groups, rows, n, block, q, s)
        with pytest.raises(symi.SymiError, match=said):
            symi.symi_dequant8(ctx, q, s, groups, rows, n, block, x)
    for groups, rows in ((0, 40), (3, 0)):     # nothing to do
        symi.symi_quant8(ctx, x, groups, rows, 200, 128, q, s)
        symi.symi_dequant8(ctx, q, s, groups, rows, 200, 128, x)
    torch.cuda.synchronize()
