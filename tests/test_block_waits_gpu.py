"""The bounded waits of the product kernels: with operand tiles left out every wait that depends on them runs out, the kernel returns, the
status word says so once, and work goes on with the same bits as before."""
import pytest
import torch

from paper_2410_15352_b200 import binding as cb
from paper_2410_15352_b200 import block
from paper_2410_15352_b200.build import build_library
from test_block_gpu import BF, operands


def test_withhold_refusals():
    build_library()
    call = block.lib().compact_debug_fp8_product_withhold
    assert call(None, 1) == cb.ERR_INVALID_ARG
    p = block.Fp8Product()
    p.debug_withhold(3)
    p.debug_withhold(-1)
    assert p.status() == cb.OK


# kernel; M, N, K; k-steps that are loaded, fewer than K has
CASES = [
    (1, 200, 256, 700, 0), (1, 200, 256, 700, 2),                     # a tile to a pair, two k-steps to a barrier
    (1, 60001, 104, 1345, 4),                                         # several
    (1, 5000, 4000, 700, 1), (1, 9001, 1376, 1300, 8),                # wide tiles; 256 columns and K longer than the ring
    (2, 1, 512, 4096, 0), (2, 1, 512, 4096, 6), (2, 77, 1000, 2736, 12), (2, 300, 130, 200, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("which, M, N, K, loaded", CASES)
def test_tiles_that_never_come(which, M, N, K, loaded):
    build_library()
    a, b = operands(M + N, M, N, K)
    p, other = block.Fp8Product(), block.Fp8Product()
    block.set_product_kernel(which)
    try:
        want = p(a, b)
        other(a, b)
        assert p.status() == cb.OK
        p.debug_withhold(loaded)
        p(a, b)
        assert other.status() == cb.OK                                # another handle's status word is its own
        assert p.status() == cb.ERR_DEVICE_TIMEOUT
        assert p.status() == cb.OK                                    # reading cleared it
        # the request was for one product; the context is intact
        got = p(a, b)
        assert torch.equal(got, want) and p.status() == cb.OK
        # and with a good product behind the bad one in the stream
        p.debug_withhold(loaded)
        p(a, b)
        got = p(a, b)
        assert p.status() == cb.ERR_DEVICE_TIMEOUT and torch.equal(got, want)
    finally:
        block.set_product_kernel(0)


@pytest.mark.gpu
def test_all_steps_loaded_is_an_ordinary_product():
    build_library()
    a, b = operands(5, 300, 264, 700)
    p = block.Fp8Product()
    want = p(a, b)
    p.debug_withhold(6)
    assert torch.equal(p(a, b), want) and p.status() == cb.OK
    assert want.dtype == BF


@pytest.mark.gpu
@pytest.mark.parametrize("which", [1, 2])
def test_a_replayed_graph_forgets_nothing(which):
    """A handle whose first product was captured: replays must not clear what an earlier product, or an earlier replay, reported."""
    build_library()
    a, b = operands(7, 200, 256, 700)
    block.set_product_kernel(which)
    try:
        want = block.Fp8Product()(a, b)
        p, out = block.Fp8Product(), torch.empty_like(want)
        good, bad = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(good):
            p(a, b, out=out)
        p.debug_withhold(2)
        with torch.cuda.graph(bad):
            p(a, b, out=out)
        good.replay()
        assert p.status() == cb.OK and torch.equal(out, want)
        bad.replay()
        good.replay()
        good.replay()
        assert p.status() == cb.ERR_DEVICE_TIMEOUT and torch.equal(out, want)
        assert p.status() == cb.OK
        p.debug_withhold(0)
        p(a, b, out=out)
        good.replay()
        assert p.status() == cb.ERR_DEVICE_TIMEOUT and torch.equal(out, want)
    finally:
        block.set_product_kernel(0)


@pytest.mark.gpu
def test_a_slot_passes_from_handle_to_handle():
    """What an earlier handle of the slot left is not taken for the later one's, and does not hide it."""
    build_library()
    a, b = operands(8, 200, 256, 700)
    first = block.Fp8Product()
    first.debug_withhold(0)
    first(a, b)
    del first                                                          # unread, and perhaps still running
    second = block.Fp8Product()                                        # in its slot
    second(a, b)
    assert second.status() == cb.OK
    second.debug_withhold(0)
    second(a, b)
    assert second.status() == cb.ERR_DEVICE_TIMEOUT and second.status() == cb.OK
    second.debug_withhold(0)
    second(a, b)
    del second
    assert block.Fp8Product().status() == cb.OK                        # nothing launched
    third = block.Fp8Product()
    third(a, b)
    assert third.status() == cb.OK
