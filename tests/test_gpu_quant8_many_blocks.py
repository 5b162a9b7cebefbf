"""Weights of more blocks than one dimension of a launch holds: it ends at 2^32 threads, which 2^24 blocks of a workgroup each pass."""
import pytest
import torch

import paper_2504_19925_amd as symi

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_small_weights(dtype):
    """2^22 + 3 weights of one row of 8 values are four bytes of scales each, and so 2^24 + 12 blocks; values that are next to a code times a power."""
    groups, n = (1 << 22) + 3, 8
    ctx = symi.symi_create(symi.SymiCfg.make(1, 1, 1, 8, 8, 1, 1, 0, dtype))
    g = torch.Generator(device="cuda").manual_seed(1)
    power = torch.randint(-20, 21, (groups, 1, 1), generator=g, device="cuda")
    x = torch.randint(-15, 16, (groups, 1, n), generator=g, device="cuda").float()
    x[:, :, 0] = 16                  # the largest: 16 2^p = 256 2^(p - 4)
    x[5], x[groups - 2] = 0, 0
    X = (x * 2.0 ** power).to(ctx.torch_dtype)
    q = torch.full((groups, 1, symi.symi_pitch8(n)), 0x55, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    s = torch.full((groups, 1, symi.symi_scale_pitch8(n)), 0x55, dtype=torch.uint8, device="cuda")
    symi.symi_quant8(ctx, X, groups, 1, n, 128, q, s)
    empty = x[:, 0, 0] == 0
    want = torch.where(empty, 0, power[:, 0, 0] - 4 + 127).to(torch.uint8)
    assert torch.equal(s[:, 0, 0], want) and not s[:, :, 1:].any()
    assert not q[:, :, n:].view(torch.uint8).any()
    assert torch.equal(q[:, :, :n].float(), x * 16)
    back = torch.full_like(X, 3.0)
    symi.symi_dequant8(ctx, q, s, groups, 1, n, 128, back)
    # the device's pow is off by a unit in the last place for some powers: codes are the nearest, and what they stand for has exact powers
    exact = ((power.int() + 127) << 23).view(torch.float32)
    assert torch.equal(back.float(), x * exact)
