"""As many tensors as make more workgroups of the decoding than one dimension of a launch has threads for: 2^23 tensors of one value,
which are also so many values that a chunk has two workgroups."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2504_19925_amd as symi
from paper_2504_19925_amd.binding import SymiAdamWTensor
from tests.test_gpu_adamw import HP, adam, context

pytestmark = pytest.mark.gpu


def test_eight_million_tensors():
    n = 1 << 23
    g = torch.Generator(device="cuda").manual_seed(1)
    w, grad, m, v = (torch.randn(n, generator=g, device="cuda") for _ in range(4))
    v.square_()
    kind = np.dtype([(k, np.uint64) for k in ("param", "master", "grad", "m", "v", "m_scale", "v_scale")] +
                    [("n", np.int64), ("decay", np.float32), ("param_dtype", np.int32), ("grad_dtype", np.int32), ("state_bits", np.int32)])
    assert kind.itemsize == ctypes.sizeof(SymiAdamWTensor)
    list_ = np.zeros(n, kind)
    for name, x in (("param", w), ("grad", grad), ("m", m), ("v", v)):
        list_[name] = x.data_ptr() + 4 * np.arange(n, dtype=np.uint64)
    list_["n"], list_["state_bits"] = 1, 32
    L, out = symi.lib(), ctypes.c_void_p()
    at = ctypes.cast(list_.ctypes.data, ctypes.POINTER(SymiAdamWTensor))
    table = torch.empty(L.symi_adamw_table_bytes(at, n), dtype=torch.uint8, device="cuda")
    assert L.symi_adamw_create(at, n, ctypes.c_void_p(table.data_ptr()), ctypes.byref(out), None) == 0
    opt = symi.SymiAdamW(out, [], table)
    ctx = context()
    print("[adamw] step", flush=True)
    m0, w0 = m.clone(), w.clone()
    symi.symi_adamw_step(ctx, opt, adam(2), None, 0)
    want = m0 * HP["beta1"] + grad * (1 - HP["beta1"])
    assert (m - want).abs().max() <= 1e-6 and not torch.equal(w, w0)
    values = symi.symi_adamw_values(opt)
    assert values == 256 * n
    print("[adamw] decode", flush=True)
    for which, state in ((0, m), (1, v)):                   # one after the other: 8.6 GB each
        outs = [torch.full((values,), -7.0, device="cuda") for _ in range(2)]
        symi.symi_adamw_decode(ctx, opt, *outs)
        got = outs[which].view(n, 256)
        assert torch.equal(got[:, 0], state)
        got[:, 0] = -7.0
        assert got.min() == -7 and got.max() == -7
        del outs, got
