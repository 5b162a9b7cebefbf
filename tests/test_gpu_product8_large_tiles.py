"""The 8-bit products' and experts' tiles of 256 rows, which training batches run on; buffers at any element; blocks of zeros beside others.

Oracle and bounds are those of the products' other tests: where codes are small whole numbers results have to be equal, elsewhere every
summand may lose what its sum's order and the 8-bit instruction drop."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import way_oracle as O
from tests.test_gpu_product8 import check, check_experts, context, gen, offsets_of, quant, scratch, whole

pytestmark = pytest.mark.gpu


def tile_rows(A, S, R, expert, dtype="bf16"):
    """Rows of a product's tiles, by the library's rule."""
    if A <= (32 if dtype == "f32" else 12) * S:
        return 16
    if dtype == "f32":
        return 128
    units = torch.cuda.get_device_properties(0).multi_processor_count
    return 128 if (A // 128 + S // 2) * -(-R // (128 if expert else 256)) <= units else 256


# last tiles of 1, 128, 129, 188, 255 and 256 rows, a slot without rows, one that ends a tile of 128 late
COUNTS = [700, 129, 255, 256, 257, 0, 511, 130, 384, 1, 900, 640]


@pytest.mark.parametrize("n", [8, 136, 264, 512, 640, 1416])     # 1, 2, 3, 4, 5, 12 blocks
@pytest.mark.parametrize("R", [1800, 2048])
def test_product(R, n):
    assert tile_rows(sum(COUNTS), len(COUNTS), R, False) == 256
    check(COUNTS, R, n, "bf16", extra=5)
    first = check(COUNTS, R, n, "bf16", exact=False)
    ctx, aq, a_s, offs, wq, w_s, Y = first
    again = torch.full_like(Y, 640.0)
    symi.symi_product8(ctx, aq, a_s, offs, wq, w_s, R, n, again, scratch(ctx))
    assert torch.equal(again, Y)


@pytest.mark.parametrize("d,f", [(136, 1032), (264, 1416), (512, 1160), (520, 1304), (1032, 1024)])
def test_experts(d, f):
    """1 to 12 blocks of either reduction; hidden units that end inside a block and with one."""
    assert max(tile_rows(sum(COUNTS), len(COUNTS), f, True), tile_rows(sum(COUNTS), len(COUNTS), d, False)) == 256
    ctx, inputs, (UV, H, Yp) = check_experts(COUNTS, d, f, extra=5)
    only = check_experts(COUNTS, d, f, extra=5, keep=False)
    assert torch.equal(only[2][2], Yp)
    new = [torch.full_like(t, 640.0) for t in (UV, H, Yp)]
    symi.symi_expert_fwd8(ctx, *inputs, *new, scratch(ctx))
    assert all(torch.equal(x, y) for x, y in zip(new, (UV, H, Yp)))


def moved(t, by):
    """(all of a buffer, t's place in it from element `by` on), with elements behind it."""
    flat = torch.full((t.numel() + by + 9,), 7.0, dtype=t.dtype, device="cuda")
    flat[by:by + t.numel()] = t.reshape(-1)
    return flat, flat[by:by + t.numel()].view(t.shape)


def untouched(flat, by, numel):
    return (flat[:by] == 7.0).all() and (flat[by + numel:] == 7.0).all()


@pytest.mark.parametrize("by", [1, 3])
@pytest.mark.parametrize("counts,d,f,rows", [(COUNTS, 264, 1032, 256), ([300, 2, 64, 200], 264, 136, 128), ([3, 0, 9], 136, 264, 16)], ids=["256", "128", "16"])
def test_rows_and_results_at_any_element(counts, d, f, rows, by):
    A, S = sum(counts), len(counts)
    assert max(tile_rows(A, S, f, True), tile_rows(A, S, d, False)) == rows
    ctx, (X, offs, w1q, w1s, w2q, w2s), (UV, H, Yp) = check_experts(counts, d, f)
    flats = [moved(torch.full_like(t, 640.0), by) for t in (UV, H, Yp)]
    symi.symi_expert_fwd8(ctx, moved(X, by)[1], offs, w1q, w1s, w2q, w2s, *[v for _, v in flats], scratch(ctx))
    for (flat, view), t in zip(flats, (UV, H, Yp)):
        assert torch.equal(view, t) and untouched(flat, by, t.numel())
    flat, view = moved(torch.full_like(Yp, 640.0), by)
    symi.symi_expert_fwd8(ctx, moved(X, by)[1], offs, w1q, w1s, w2q, w2s, None, None, view, scratch(ctx))
    assert torch.equal(view, Yp) and untouched(flat, by, Yp.numel())


@pytest.mark.parametrize("by", [1, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,R", [(COUNTS, 1800), ([300, 2, 64, 200], 264), ([3, 0, 9], 136)], ids=["256", "128", "16"])
def test_product_at_any_element(counts, R, dtype, by):
    A, S = sum(counts), len(counts)
    assert tile_rows(A, S, R, False, dtype) == (16 if A < 100 else 128 if A < 1000 or dtype == "f32" else 256)
    ctx, aq, a_s, offs, wq, w_s, Y = check(counts, R, 392, dtype, exact=False)
    flat, view = moved(torch.full_like(Y, 640.0), by)
    symi.symi_product8(ctx, aq, a_s, offs, wq, w_s, R, 392, view, scratch(ctx))
    assert torch.equal(view, Y) and untouched(flat, by, Y.numel())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,R", [(COUNTS, 1800), ([300, 2, 64, 200], 264), ([3, 0, 9], 136)], ids=["256", "128", "16"])
def test_blocks_of_zeros_beside_others(counts, R, dtype):
    """Padding rows, a masked column block, rows with one block that is not zero, weights with blocks of zeros and a slot whose weight is zero:
    their powers are 0, the smallest there is, and count for nothing."""
    n, A, S = 640, sum(counts), len(counts)
    ctx = context(A, S, dtype)
    print(f"[product8 zeros] {dtype} rows {counts} R={R}", flush=True)
    at, offs = offsets_of(counts)
    x, v = whole(1, 1, A, n), whole(2, S, R, n)
    x[:, ::10] = 0
    x[:, 1::10, 128:] = 0
    x[:, :, 256:384] = 0
    v[:, :128, :128] = 0
    v[0] = 0
    aq, a_s, a = quant(ctx, x, 1)
    wq, w_s, w = quant(ctx, v, 128)
    assert (a_s[0, ::10] == 0).all() and (a_s[0, :, 2] == 0).all() and (w_s[1:, 0, 0] == 0).all() and (w_s[0] == 0).all()
    Y = torch.full((A, R), 640.0, dtype=ctx.torch_dtype, device="cuda")
    symi.symi_product8(ctx, aq, a_s, offs, wq, w_s, R, n, Y, scratch(ctx))
    want, _ = O.product(a[0], w, at)
    want = torch.from_numpy(want).float().to(ctx.torch_dtype)
    assert (Hn.npf(Y) == Hn.npf(want)).all() and np.abs(Hn.npf(want)).max() > 0


@pytest.mark.parametrize("counts,d,f", [(COUNTS, 264, 1032), ([300, 2, 64, 200], 264, 136), ([3, 0, 9], 136, 264)], ids=["256", "128", "16"])
def test_rows_and_weights_of_the_experts_that_are_not_finite(counts, d, f):
    """A NaN or an infinity reaches the results of its row, or of its weight's slot, and no others."""
    ctx, (X, offs, w1q, w1s, w2q, w2s), clean = check_experts(counts, d, f)
    X, w1q, n = X.clone(), w1q.clone(), counts[0]
    X[0, 3], X[2, d - 1] = float("nan"), -float("inf")
    w1q.view(torch.uint8)[2, f + 5, 7] = 0x7F        # an up row of the third slot
    bad = [torch.full_like(t, 640.0) for t in clean]
    symi.symi_expert_fwd8(ctx, X, offs, w1q, w1s, w2q, w2s, *bad, scratch(ctx))
    rows = torch.zeros(sum(counts), dtype=torch.bool, device="cuda")
    rows[0] = rows[2] = True
    third = slice(int(offs[2]), int(offs[3]))
    UV, H, Y = bad
    assert torch.isnan(UV[rows]).all() and torch.isnan(H[rows]).all() and torch.isnan(Y[rows]).all()
    assert torch.isnan(UV[third, f + 5]).all() and torch.isnan(H[third, 5]).all() and torch.isnan(Y[third]).all()
    rows[third] = True
    assert all(torch.equal(t[~rows], c[~rows]) for t, c in zip(bad, clean)) and n > 2
    others = torch.ones(2 * f, dtype=torch.bool, device="cuda")
    others[f + 5] = False
    assert torch.equal(UV[third][:, others], clean[0][third][:, others])


def test_more_tiles_than_a_launch_has_threads_for_are_refused():
    """2^24 workgroups of 256 threads.  Refused before anything is read."""
    L, some = symi.lib(), 256
    for dtype, T in (("bf16", 8000000), ("f32", 4000000)):
        ctx = context(T, 1, dtype)
        assert L.symi_product8(ctx.ptr, some, some, some, some, some, 1 << 22, 1024, some, some, None) == -2
        assert "tiles" in symi.symi_last_error()
    ctx = context(8000000, 4000, "bf16", d=256, f=1 << 19)
    assert L.symi_expert_fwd8(ctx.ptr, some, some, some, some, some, some, None, None, some, some, None) == -2
    assert "tiles" in symi.symi_last_error()
