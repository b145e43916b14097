"""The norm's kernels where a group of threads goes round its ring of rows: sizes that give every layout more rows to a group than it has
stages.  All outputs are compared with the formulas in 64 bits.

Tolerances as in test_block_gpu, u = 2^-24: rstd 2.1e-6, y 3e-6 |y|, dx 1e-5 of the sum of its terms' magnitudes.  dweight: a
group adds up at most 50 rows, a CTA at most 24 groups, the last kernel 5 parts to a warp and 32 warps in 5 steps, each within u; a
product of three factors before it, 3 u more, and rstd as the forward rounded it, 2.1e-6: below 90 u + 2.1e-6 = 7.5e-6 of the sum of magnitudes."""
import pytest
import torch

from paper_2410_15352_b200 import block
from paper_2410_15352_b200.build import build_library
from test_block_gpu import BF, E4, E5, F32, defined_scales, gen, half_ulp, norm_reference, normal, padded, scale_table, widen

pytestmark = pytest.mark.gpu
# a layout each, forward or backward: one warp to a row and several, one unit to a thread and two, weight in registers and in shared memory
ROUNDS = [(20001, 256), (20000, 512), (16000, 1000), (9003, 1376), (9001, 2048), (4000, 2736), (5001, 4096), (4000, 5000), (2500, 8192), (1501, 11008),
          (1200, 16384), (15001, 130)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def inputs(tokens, n, dtype, residual):
    g = gen(tokens + 1000 * n)
    x = normal(g, (tokens, n))
    x[:, n // 3] *= 20.0
    x[tokens // 2] = 0.0
    x = padded(x.to(dtype))
    r = padded(normal(g, (tokens, n), dtype), 48) if residual else None
    return g, x, r, (1.0 + 0.1 * normal(g, (n,))).to(dtype)


def check_forward(o, x, r, w, eps, fp8):
    dtype, n = x.dtype, x.shape[1]
    h = x if r is None else (x.float() + r.float()).to(dtype)
    assert torch.equal(o.h, h)
    h64 = h.double()
    rstd = 1.0 / torch.sqrt(h64.square().mean(1) + eps)
    assert bool(((o.rstd.double() - rstd).abs() <= 2.1e-6 * rstd).all())
    y = h64 * rstd[:, None] * w.double()
    if o.y is not None:
        assert bool(((o.y.double() - y).abs() <= half_ulp(dtype, y, 3e-6 * y.abs())).all())
    if o.q is not None:
        exps, past = scale_table(o.q.scales, n)
        assert bool((past == 0).all())
        assert bool(((exps == defined_scales(y * (1 - 3e-6), fp8, 1)) | (exps == defined_scales(y * (1 + 3e-6), fp8, 1))).all())
        s = torch.exp2(exps.double()).repeat_interleave(128, 1)[:, :n]
        # half a step of the type: three mantissa bits, least step 2^-9; two and 2^-16
        rel, least = (2.0 ** -4, 2.0 ** -10) if fp8 == E4 else (2.0 ** -3, 2.0 ** -17)
        assert bool(((widen(o.q) - y).abs() <= torch.maximum(y.abs() * rel, s * least) + 3e-6 * y.abs()).all())


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens, n", ROUNDS)
def test_forward(tokens, n, dtype, residual):
    _, x, r, w = inputs(tokens, n, dtype, residual)
    norm = block.RMSNorm(n, eps=1e-5, dtype=dtype)
    for want_y, want_fp8, fp8 in ((True, True, E4), (True, False, E4), (False, True, E5)):
        check_forward(norm.forward(x, w, residual=r, want_y=want_y, want_fp8=want_fp8, fp8_dtype=fp8), x, r, w, 1e-5, fp8)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens, n", [(20001, 256), (4000, 2736), (5001, 4096), (2500, 8192)])
def test_forward_in_place(tokens, n, dtype):
    """h over x or over the residual, while later rows are on their way."""
    _, x, r, w = inputs(tokens, n, dtype, True)
    norm = block.RMSNorm(n, eps=1e-5, dtype=dtype)
    for over_x in (True, False):
        a, b = x.clone(memory_format=torch.preserve_format), r.clone(memory_format=torch.preserve_format)
        a, b = padded(a), padded(b, 48)
        target = a if over_x else b
        o = norm.forward(a, w, residual=b, want_fp8=True, h=target)
        assert o.h is target or o.h.data_ptr() == target.data_ptr()
        check_forward(o, x, r, w, 1e-5, E4)
    # h alone
    o = norm.forward(x, w, residual=r, want_y=False)
    assert o.y is None and o.q is None
    check_forward(o, x, r, w, 1e-5, E4)


@pytest.mark.parametrize("extra", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens, n", ROUNDS)
def test_backward(tokens, n, dtype, extra):
    g, h, dr, w = inputs(tokens, n, dtype, extra)
    dy = padded(normal(g, (tokens, n), dtype), 32)
    norm = block.RMSNorm(n, eps=1e-5, dtype=dtype)
    rstd = norm.forward(h, w).rstd
    dx, dw = norm.backward(dy, h, w, rstd, residual_grad=dr)
    h64, w64 = h.double().requires_grad_(), w.double().requires_grad_()
    gx, gw = torch.autograd.grad(norm_reference(h64, w64, 1e-5), (h64, w64), dy.double())
    if dr is not None:
        gx = gx + dr.double()
    r64 = rstd.double()[:, None]
    gm = (dy.double() * w.double()).abs()
    size = r64 * (gm + h.double().abs() * r64 * (gm * h.double().abs() * r64).mean(1, keepdim=True))
    if dr is not None:
        size = size + dr.double().abs()
    assert bool(((dx.double() - gx).abs() <= half_ulp(dtype, gx, 1e-5 * size)).all())
    terms = (dy.double() * h.double() * r64).abs().sum(0)
    assert bool(((dw.double() - gw).abs() <= 7.5e-6 * terms).all())
    dx2, dw2 = norm.backward(dy, h, w, rstd, residual_grad=dr)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    for over_dy in (True, False):
        if not over_dy and dr is None:
            continue
        a, b = padded(dy, 32), None if dr is None else padded(dr, 48)
        got, none = norm.backward(a, h, w, rstd, residual_grad=b, dx=a if over_dy else b, need_dweight=False)
        assert none is None and torch.equal(got, dx)


@pytest.mark.parametrize("extra", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens, n", [(10, 1000), (700, 1376), (3000, 600), (3000, 2048), (5001, 4096)])
def test_the_order_of_the_weight_gradient(tokens, n, dtype, extra):
    """The same bits wherever the matrices lie, with dx or without it, alone or after another."""
    g, h, dr, w = inputs(tokens, n, dtype, extra)
    dy = normal(g, (tokens, n), dtype)
    norm = block.RMSNorm(n, eps=1e-5, dtype=dtype)
    rstd = norm.forward(h, w).rstd
    _, dw = norm.backward(padded(dy), h, w, rstd, residual_grad=dr)
    _, alone = norm.backward(padded(dy, 64), padded(h, 32), w.clone(), rstd.clone(), residual_grad=None if dr is None else padded(dr, 16), need_dx=False)
    assert torch.equal(dw, alone)
    into = torch.zeros_like(dw)
    norm.backward(padded(dy), h, w, rstd, residual_grad=dr, dweight=into, accumulate=True)
    assert torch.equal(dw, into)
