"""Empty batches through every block operator: a successful call that launches nothing."""
import pytest
import torch

from paper_2410_15352_b200 import binding as cb
from paper_2410_15352_b200 import block
from paper_2410_15352_b200.build import build_library


@pytest.mark.parametrize("dtype", [cb.BF16, cb.F32])
def test_norm_backward_of_no_tokens_needs_no_output(dtype):
    """A frozen weight leaves dX alone, and a matrix of no rows has no memory."""
    build_library()
    before = cb.kernel_launch_count()
    assert block.lib().compact_rms_norm_bwd(dtype, 0, 64, None, 64, None, 64, None, None, None, 0, None, 64, None, 0, None, 0, None) == cb.OK
    assert block.lib().compact_rms_norm_bwd(dtype, 1, 64, 0x1000, 64, 0x1000, 64, 0x1000, 0x1000, None, 0, None, 64, None, 0, None, 0, None) == cb.ERR_INVALID_ARG
    assert cb.kernel_launch_count() == before


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_empty_batches(dtype):
    build_library()
    n = 640
    x, w, dw = (torch.ones(s, dtype=t, device="cuda") for s, t in (((0, n), dtype), ((n,), dtype), ((n,), torch.float32)))
    norm, product, rotary = block.RMSNorm(n, dtype=dtype), block.Fp8Product(), block.Rotary(64)
    w8 = block.quantize_rows(torch.ones((72, n), dtype=dtype, device="cuda"))
    before = cb.kernel_launch_count()
    for residual in (None, x):
        o = norm.forward(x, w, residual=residual, want_fp8=True)
        assert o.y.shape == o.h.shape == (0, n) and o.q.data.shape == (0, n) and o.rstd.shape == (0,)
        dx, none = norm.backward(o.y, o.h, w, o.rstd, residual_grad=residual, need_dweight=False)
        assert dx.shape == (0, n) and none is None
        none, same = norm.backward(o.y, o.h, w, o.rstd, need_dx=False, dweight=dw, accumulate=True)
        assert none is None and bool((same == 1).all())
        dx, zero = norm.backward(o.y, o.h, w, o.rstd)
        assert dx.shape == (0, n) and bool((zero == 0).all())
    q = block.quantize_rows(x)
    assert product(q, w8).shape == (0, 72) and product.status() == cb.OK
    b, bt = block.quantize_blocks(x)
    assert b.data.shape == (0, n) and bt.data.shape == (n, 0)
    a, c = rotary.forward(x.view(0, 10, 64), x.view(0, 10, 64), torch.zeros(0, dtype=torch.int64, device="cuda"))
    assert a.shape == c.shape == (0, 10, 64)
    assert cb.kernel_launch_count() == before
