"""AdamW over lists of more than 2^23 values, whose tensors are cut into whole chunks of 4096 values with four blocks in flight, and
their decoding by two workgroups a chunk: every kind of tensor, ragged around the chunks, at any alignment.  Against binary64 with the
bounds of test_gpu_adamw.py."""
import numpy as np
import pytest
import torch

import harness as Hn
import paper_2504_19925_amd as symi
from oracle import ends_oracle as O
from tests.test_gpu_adamw import U32, adam, check, context, make, snapshot, states

pytestmark = pytest.mark.gpu
SIZES = [4095, 4096, 4097, 3 * 4096 + 200, 8192, 8192 + 1025, 70, 20001, 4096 + 4095]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("param", ["f32", "bf16"])
def test_whole_chunks(param, grad, bits, monkeypatch):
    ctx = context()
    tensors = [make(n, param, grad, bits, (1.0, 0.0, 0.5)[i % 3], i, by=i % 4) for i, n in enumerate(SIZES)]
    rest = make((1 << 23) + 5, param, grad, bits, seed=99)       # its last 4096 values and what is behind them are looked at below
    opt = symi.symi_adamw_create(tensors + [rest])
    for step, scale, seed in ((7, None, 1), (8, -0.25, 2 ** 31)):
        before = snapshot(tensors + [rest])
        clip = None if scale is None else torch.full((1,), scale, device="cuda")
        symi.symi_adamw_step(ctx, opt, adam(step, 0.5), clip, seed)
        check(before[:-1], tensors, step, 0.5 * (1.0 if scale is None else scale), seed)
        at = (1 << 23) - 4096
        cut = lambda t: {k: (x if not isinstance(x, torch.Tensor) else x[at // 256:] if "scale" in k else x[at:]) for k, x in t.items()}   # noqa: E731
        place = sum(-(-n // 256) for n in SIZES) + at // 256
        shift = O.random_numbers
        monkeypatch.setattr(O, "random_numbers", lambda seed, step, first, n: shift(seed, step, first + place, n))
        check([cut(before[-1])], [cut(rest)], step, 0.5 * (1.0 if scale is None else scale), seed)
        monkeypatch.undo()
    n = symi.symi_adamw_values(opt)
    m, v = torch.full((n,), -7.0, device="cuda"), torch.full((n,), -7.0, device="cuda")
    symi.symi_adamw_decode(ctx, opt, m, v)
    at = 0
    for t in tensors + [rest]:
        size = t["param"].numel()
        m64, v64 = states(t)
        assert (np.abs(Hn.npf(m[at:at + size]) - m64) <= 4 * U32 * np.abs(m64)).all()
        assert (np.abs(Hn.npf(v[at:at + size]) - v64) <= 6 * U32 * v64).all()
        end = at + -(-size // 256) * 256
        assert (m[at + size:end] == -7).all() and (v[at + size:end] == -7).all()
        at = end
