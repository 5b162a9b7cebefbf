"""How exact the hidden units of the 8-bit experts are on their way into 8 bits.  The second weight is the identity, so that the outputs are the hidden units'
values in 8 bits, which bf16 holds exactly; only 8 neighbouring inputs of a row are not zero, so that sums are short.

A sum of 8 products in fp32, in any order, is within 2 * 8 U32 of the sum of their sizes.  In tiles of more than 16 rows the 8-bit instruction drops 7 2^-13 of it at
most.  The exponential is within (2 |u| + 24) U32, relatively, and silu's slope at most 1.1.  A value in 8 bits may be any that a hidden unit within these bounds has."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import way_oracle as O
from tests.test_gpu_product8 import U32, context, gen, offsets_of, quant, scratch
from tests.test_gpu_product8_large_tiles import tile_rows

pytestmark = pytest.mark.gpu


def reach(h, off):
    """(value in 8 bits, how far from it the value may be of anything within `off` of h and of the block's largest)."""
    blocks = h.shape[1] // 128
    tops = [np.max((np.abs(h) + sign * off).reshape(len(h), blocks, 128), axis=2) for sign in (-1, 1)]
    base = O.values(*O.quant(h, 1), 1)
    far = np.zeros_like(h)
    for top in tops:
        scale = np.repeat(2.0 ** (np.vectorize(O.power)(np.maximum(top, 0)) - 127.0), 128, axis=1)
        for x in (h - off, h + off):
            far = np.maximum(far, np.abs(O.to_e4m3(np.clip(x / scale, -448, 448)) * scale - base))
    return base, far


@pytest.mark.parametrize("counts,rows", [([12, 0, 16, 9, 17, 1, 20, 21], 16), ([300, 2, 64, 200], 128), ([700, 129, 255, 256, 257, 0, 511, 130, 384, 1, 900, 640], 256)],
                         ids=["16", "128", "256"])
@pytest.mark.parametrize("seed", [1, 2])
def test_hidden_units_have_the_digits_of_their_sums(counts, rows, seed):
    A, S, d = sum(counts), len(counts), 1024
    assert max(tile_rows(A, S, d, True), tile_rows(A, S, d, False)) == rows
    ctx = context(A, S, "bf16", d, d)
    print(f"[expert8 digits] rows {counts} seed {seed}", flush=True)
    at, offs = offsets_of(counts)
    X = torch.zeros(A, d, dtype=torch.bfloat16, device="cuda")
    X[:, 8:16] = torch.randn(A, 8, generator=gen(seed), device="cuda").to(torch.bfloat16)
    _, _, x = quant(ctx, X[None].float(), 1)
    w1q, w1s, w1 = quant(ctx, torch.randn(S, 2 * d, d, generator=gen(seed + 10), device="cuda"), 128)
    w2q, w2s, w2 = quant(ctx, torch.eye(d, device="cuda").expand(S, d, d), 128)
    assert (w2 == np.eye(d)).all()
    Y = torch.full((A, d), 640.0, dtype=torch.bfloat16, device="cuda")
    symi.symi_expert_fwd8(ctx, X, offs, w1q, w1s, w2q, w2s, None, None, Y, scratch(ctx))
    uv, size = O.product(x[0], w1, at)
    u, v = uv[:, :d], uv[:, d:]
    lost = (2 * 8 * U32 + (7 * 2.0 ** -13 if rows > 16 else 0)) * size * 1.01
    h = O.silu_product(u, v)
    off = 1.1 * (np.abs(v) + lost[:, d:]) * lost[:, :d] + np.abs(O.silu_product(u, 1.0)) * lost[:, d:] + (2 * np.abs(u) + 24) * U32 * np.abs(h)
    base, far = reach(h, off)
    got = Hn.npf(Y).astype(np.float64)
    print(f"[expert8 digits] {int((got != base).sum())} of {got.size} another code, {int((far > 0).sum())} may", flush=True)
    assert (np.abs(got - base) <= far).all()
