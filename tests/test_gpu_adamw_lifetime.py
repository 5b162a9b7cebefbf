"""The optimizer's handle may be dropped while its steps are queued on another stream than the one that made it: neither the table
nor tensors that only the handle holds are handed to anybody else before the step has run."""
import pytest
import torch

import paper_2504_19925_amd as symi
from tests.test_gpu_adamw import adam, check, context, make, snapshot

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("through", ["marshal", "ctypes"])
@pytest.mark.parametrize("bits", [32, 8])
def test_dropped_while_a_side_stream_still_has_to_step(bits, through):
    ctx, n = context(), 1 << 20
    step = symi.symi_adamw_step if through == "marshal" else symi.symi_adamw_step.through_ctypes
    a = torch.randn(8192, 8192, device="cuda").to(torch.bfloat16)
    product = a @ a                                     # the first calls of all that runs below load their kernels
    _ = [torch.full((1000,), 1, dtype=x, device="cuda") for x in (torch.int32, torch.uint8)]
    side = torch.cuda.Stream()
    step(ctx, symi.symi_adamw_create([make(n, bits=bits)]), adam(1), None, 0)
    for _ in range(2):
        t = make(n, bits=bits, seed=bits)
        before = snapshot([t])
        opt = symi.symi_adamw_create([t])
        keep = {k: t[k] for k in ("param", "grad", "m", "v", "m_scale", "v_scale") if k in t and k != "grad"}
        t["grad"] = None
        held = [opt.table, opt.tensors[0]["grad"]]      # what the handle alone holds
        places, sizes = [x.data_ptr() for x in held], [x.numel() * x.element_size() for x in held]
        del held, t
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(60):                         # about a millisecond each
                torch.mm(a, a, out=product)
            busy = torch.cuda.Event()
            busy.record()
            step(ctx, opt, adam(3), None, 5)
        del opt
        new = [torch.full((size // 4 if size % 4 == 0 else size,), 1, dtype=torch.int32 if size % 4 == 0 else torch.uint8, device="cuda") for size in sizes]
        waiting = not busy.query()
        if waiting:                                     # the step had not begun when the new memory was handed out
            assert not {x.data_ptr() for x in new} & set(places)
        torch.cuda.synchronize()
        assert waiting
        check(before, [{**before[0], **keep}], 3, 1.0, 5)


def test_every_stream_is_noted_once():
    ctx = context()
    t = make(300, "bf16", "f32", 8)
    opt = symi.symi_adamw_create([t])
    home, side = torch.cuda.current_stream(), torch.cuda.Stream()
    assert opt.streams == {home.cuda_stream} and opt.stream == home.cuda_stream
    symi.symi_adamw_step(ctx, opt, adam(1), None, 0)
    side.wait_stream(home)
    with torch.cuda.stream(side):
        symi.symi_adamw_step(ctx, opt, adam(2), None, 0)
        assert opt.streams == {home.cuda_stream, side.cuda_stream} and opt.stream == side.cuda_stream
        symi.symi_adamw_step(ctx, opt, adam(3), None, 0)
    home.wait_stream(side)
    m, v = torch.empty(512, device="cuda"), torch.empty(512, device="cuda")
    symi.symi_adamw_decode(ctx, opt, m, v)
    assert opt.stream == home.cuda_stream and len(opt.streams) == 2
    torch.cuda.synchronize()
