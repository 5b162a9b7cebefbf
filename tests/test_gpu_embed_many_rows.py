"""The lookup of batches that take two rows at a time: one product in single precision, rounded once more in bf16, is what torch's
own product of the same rows is, bit for bit."""
import pytest
import torch

import paper_2504_19925_amd as symi
from tests.test_gpu_embed import context, gen, make_tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 16, 24, 136, 1000, 1024, 2048, 2056, 4096])
def test_two_rows_at_a_time(d, dtype):
    pieces, lanes = d // (8 if dtype == "bf16" else 4), 1
    while lanes < 256 and lanes < pieces:
        lanes *= 2
    least = 8 * torch.cuda.get_device_properties(0).multi_processor_count * (256 // lanes)   # rows from which on it does
    V, scale = 5003, 0.37
    table = torch.randn(V, d, generator=gen(d), device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    for T, kind in ((least - 1, "padded"), (least, "skewed"), (least + 1, "padded"), (least + 2, "uniform"), (2 * least + 33, "padded"), (least + 7, "none")):
        print(f"[embed] {dtype} T={T} d={d} {kind}", flush=True)
        ctx = context(T, d, dtype)
        tokens = make_tokens(kind, T, V, T)
        for by in (0, 3):
            X = torch.full((T * d + by + 8,), 7.0, dtype=table.dtype, device="cuda")
            symi.symi_embed_fwd(ctx, tokens, table, V, scale, X[by:by + T * d].view(T, d))
            inside = (tokens >= 0) & (tokens < V)
            want = torch.where(inside[:, None], table[tokens.long().clamp(0, V - 1)].float() * scale, 0.0).to(table.dtype)
            assert torch.equal(X[by:by + T * d].view(T, d), want)
            assert (X[:by] == 7).all() and (X[by + T * d:] == 7).all()
