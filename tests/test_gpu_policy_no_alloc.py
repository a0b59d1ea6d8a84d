"""The C entry points of the operators around the layer step take all memory from the caller: once a kernel's code is loaded, a call leaves the
device's free memory and the allocator's count of requests as they were."""
import ctypes

import pytest
import torch

from paper_2512_23353_amd import isopo

pytestmark = pytest.mark.gpu


def test_calls_allocate_nothing(gpu_device):
    lib, s = isopo.load(), torch.cuda.current_stream().cuda_stream
    n, d_in, d_out, vocab = 96, 2056, 264, 1000
    mk = lambda *shape: torch.randn(shape, device=gpu_device)  # noqa: E731
    calls = []
    for code, t in ((isopo.F32, torch.float32), (isopo.BF16, torch.bfloat16)):
        X, W, Y, Z = mk(n, d_in).to(t), mk(d_out, d_in).to(t), mk(n, d_out).to(t), mk(n, d_out).to(t)
        delta, dx, db = torch.empty_like(Y), torch.empty_like(X), mk(d_out)
        ws = torch.empty(max(256, lib.isopo_linear_workspace(n, d_in, d_out, code), lib.isopo_linear_backward_workspace(n, d_in, d_out, code)), dtype=torch.uint8,
                         device=gpu_device)
        logits, targets, f = mk(n, vocab).to(t), torch.zeros(n, dtype=torch.int32, device=gpu_device), mk(4, n)
        lse, g = mk(n, 2), torch.empty_like(logits)
        lay = isopo._LinearLayer(X.data_ptr(), W.data_ptr(), None, None, code, isopo.ACT_SILU, n, d_in, d_out, 0, 0, 0)
        arg = isopo._TokenLogits(logits.data_ptr(), code, n, vocab, 0, targets.data_ptr(), 1.0)
        keep = (X, W, Y, Z, delta, dx, db, ws, logits, targets, f, lse, g)
        calls += [
            (keep, lambda lay=lay, Y=Y, Z=Z, ws=ws: lib.isopo_linear(lay, Y.data_ptr(), Z.data_ptr(), ws.data_ptr(), ws.numel(), s)),
            (keep, lambda Y=Y, W=W, Z=Z, code=code, delta=delta, dx=dx, db=db, ws=ws: lib.isopo_linear_backward(
                Y.data_ptr(), 0, W.data_ptr(), Z.data_ptr(), code, isopo.ACT_SILU, n, d_in, d_out, delta.data_ptr(), dx.data_ptr(), db.data_ptr(),
                ws.data_ptr(), ws.numel(), s)),
            (keep, lambda arg=arg, f=f, lse=lse, g=g: lib.isopo_token_logprob(arg, f[0].data_ptr(), lse.data_ptr(), f[1].data_ptr(), f[2].data_ptr(), g.data_ptr(), 0, s)),
            (keep, lambda arg=arg, f=f, lse=lse, g=g: lib.isopo_token_logprob_backward(arg, lse.data_ptr(), f[2].data_ptr(), f[1].data_ptr(), f[3].data_ptr(),
                                                                                     g.data_ptr(), 0, s)),
        ]
    for bits in (8, 32):
        opt = isopo.AdamW([mk(5000), mk(300)], state_bits=bits)
        grads, norm = [mk(5000), mk(300)], mk(1)
        arr = opt._pointers(*[x.data_ptr() for x in grads])
        opt._args.lr, opt._args.max_norm, opt._args.step = 1e-3, 1.0, 1
        keep = (opt, grads, norm, arr)
        calls.append((keep, lambda opt=opt, arr=arr, norm=norm: lib.isopo_adamw_clipped(opt._tensors, arr, 2, opt._args, norm.data_ptr(), opt._norm_ws.data_ptr(),
                                                                                       opt._norm_ws.numel(), s)))
        if bits == 8:
            out = mk(2, 5000)
            calls.append(((opt, out), lambda opt=opt, out=out: lib.isopo_adamw_state(
                ctypes.c_void_p(opt.m[0].data_ptr()), opt.m_scales[0].data_ptr(), opt.v[0].data_ptr(), opt.v_scales[0].data_ptr(), 5000, isopo.F32,
                out[0].data_ptr(), out[1].data_ptr(), s)))
    for _, call in calls:
        assert call() == 0
    torch.cuda.synchronize()
    free, asked = torch.cuda.mem_get_info()[0], torch.cuda.memory_stats()["allocation.all.allocated"]
    for _ in range(3):
        for _, call in calls:
            assert call() == 0
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] >= free and torch.cuda.memory_stats()["allocation.all.allocated"] == asked
