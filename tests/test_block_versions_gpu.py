"""Tensors that a block operator writes into count as changed, so that autograd refuses a backward pass through what it saved of them."""
import pytest
import torch

from paper_2410_15352_b200 import block
from paper_2410_15352_b200.build import build_library

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_what_a_call_writes_changes_its_version():
    build_library()
    t, n = 48, 256
    x, r, dy = (torch.randn((t, n), device="cuda").to(BF) for _ in range(3))
    w, dw = torch.ones(n, dtype=BF, device="cuda"), torch.zeros(n, device="cuda")
    norm, product, rotary = block.RMSNorm(n), block.Fp8Product(), block.Rotary(64)
    q8, w8, wt8 = block.new_fp8(t, n), block.new_fp8(n, n), block.new_fp8(n, n)
    h, y, dx, c = (torch.empty_like(x) for _ in range(4))
    square = torch.randn((n, n), device="cuda").to(BF)
    heads = x.clone().view(t, 4, 64)
    calls = [
        (lambda: block.quantize_rows(x, out=q8), q8), (lambda: block.quantize_blocks(square, out=w8, out_t=wt8), (*w8, *wt8)),
        (lambda: norm.forward(x, w, residual=r, h=h, y=y, q=q8), (h, y, *q8)),
        (lambda: norm.backward(dy, h, w, torch.ones(t, device="cuda"), dx=dx, dweight=dw), (dx, dw)),
        (lambda: rotary.forward(heads, heads[:, :2], q_out=heads, k_out=y.view(t, 4, 64)[:, 2:]), (heads, y)), (lambda: product(q8, w8, out=c), (c,)),
    ]
    rest = [x, r, dy, w, square]
    for call, outputs in calls:
        before, still = [o._version for o in outputs], [o._version for o in rest]
        call()
        assert all(o._version > b for o, b in zip(outputs, before))
        assert [o._version for o in rest] == still


def test_a_refused_call_changes_none():
    build_library()
    x = torch.ones((4, 64), dtype=BF, device="cuda")
    out = block.new_fp8(5, 64)
    before = [o._version for o in out]
    with pytest.raises(Exception):
        block.quantize_rows(x, out=out)
    assert [o._version for o in out] == before


def test_autograd_notices_an_output_in_place():
    build_library()
    rotary = block.Rotary(64)
    leaf = torch.randn((8, 2, 64), device="cuda", requires_grad=True)
    q = leaf * 2.0
    loss = (q * q).sum()                                       # saves q
    with torch.no_grad():
        rotary.forward(q, None, q_out=q)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_inference_tensors_are_written_as_well():
    build_library()
    rotary = block.Rotary(64)
    with torch.inference_mode():
        q = torch.randn((8, 2, 64), device="cuda")
        want = rotary.forward(q, None)[0]
        assert torch.equal(rotary.forward(q, None, q_out=q)[0], want)
