"""The pairs' product kernel where a pair has several tiles: both accumulators and their barriers, tiles of every width class (two k-steps
to a barrier up to 128 columns, one above; more than 128 rows of B with scales of their own; 256 columns, whose accumulators share 32
of them), scales carried from tile to tile, panels of column tiles.  The plan of each shape is asserted, so that it stays on the path
it was chosen for.  Bounds as in test_block_gpu: an instruction adds 32 exact products to the accumulator with an error below 2^-22 of the
magnitudes summed so far, and K / 32 of them make a sum."""
import pytest
import torch

from paper_2410_15352_b200 import binding as cb
from paper_2410_15352_b200 import block
from paper_2410_15352_b200.build import build_library
from test_block_gpu import BF, E4, E5, F32, check_product, operands

PAIRS = 74      # of the GPU's 148 SMs
# M, N, K; columns of a tile, k-steps to a barrier, panels; least number of tiles of some pair
SHAPES = [
    (40001, 96, 136, 96, 2, 1, 3),
    (60001, 104, 70, 128, 2, 1, 4),            # K within one k-step
    (60001, 104, 1345, 128, 2, 1, 4),
    (20000, 264, 1100, 160, 1, 1, 3),
    (3333, 2736, 520, 192, 1, 1, 3),
    (5000, 4000, 700, 224, 1, 1, 5),
    (4321, 3750, 504, 224, 1, 1, 4),           # one group of scales to a tile
    (9001, 1376, 300, 256, 1, 1, 3),
    (15411, 1012, 1800, 256, 1, 1, 4),
    (16384, 4096, 640, 256, 1, 1, 14),
    (700, 12552, 4112, 192, 1, 2, 3),          # B of 49 MB
    (2100, 12552, 4112, 224, 1, 2, 7),
    (5200, 13000, 4112, 256, 1, 2, 15),
]


@pytest.mark.parametrize("M, N, K, width, per_barrier, panels, rounds", SHAPES)
def test_the_plans_are_the_ones_meant(M, N, K, width, per_barrier, panels, rounds):
    build_library()
    p = block.debug_product_plan(M, N, K)
    assert (p.kernel, p.width, p.per_barrier, p.panels) == (1, width, per_barrier, panels)
    assert -(-p.tiles // PAIRS) == rounds


def test_plan_refusals():
    build_library()
    for bad in ((0, 8, 8), (8, 0, 8), (8, 8, 0), (1 << 31, 8, 8)):
        with pytest.raises(cb.CompactError) as e:
            block.debug_product_plan(*bad)
        assert e.value.code == cb.ERR_INVALID_ARG
    with pytest.raises(cb.CompactError) as e:
        block.debug_product_plan(0x7fffff00, 0x7fffff00, 128)
    assert e.value.code == cb.ERR_SHAPE


@pytest.mark.gpu
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("M, N, K", [s[:3] for s in SHAPES])
def test_several_tiles_to_a_pair(M, N, K, out):
    build_library()
    a, b = operands(M + N + K, M, N, K, E5 if K % 8 == 4 else E4)
    p = block.Fp8Product()
    c = torch.full((M, N + 24 + -N % 8), 7.0, dtype=out, device="cuda")
    p(a, b, out=c[:, 8: 8 + N])
    again = p(a, b, dtype=out)
    assert p.status() == cb.OK
    assert torch.equal(c[:, 8: 8 + N], again)
    assert bool((c[:, :8] == 7.0).all()) and bool((c[:, 8 + N:] == 7.0).all())
    del c
    # in pieces of rows, each against the 64-bit product of what the 8 bits stand for
    for i in range(0, M, 8192):
        rows = block.Fp8Matrix(a.data[i: i + 8192], a.scales[:, i: i + 8192])
        check_product(again[i: i + 8192], rows, b)


@pytest.mark.gpu
@pytest.mark.parametrize("which", [1, 2])
def test_scales_far_apart(which):
    """Rows whose scales lie up to 2^200 apart on either side, with products of ordinary size."""
    build_library()
    g = torch.Generator(device="cuda").manual_seed(3)
    M, N, K = 300, 264, 700
    up = torch.tensor([-100.0, -60.0, 0.0, 60.0, 100.0], device="cuda")
    for e in up:
        a = torch.randn((M, K), generator=g, device="cuda") * 2.0 ** float(e)
        b = torch.randn((N, K), generator=g, device="cuda") * 2.0 ** -float(e)
        wide = [torch.zeros((x.shape[0], 704), device="cuda") for x in (a, b)]
        for x, w in zip((a, b), wide):
            w[:, :K] = x
        qa, qb = (block.quantize_rows(w[:, :K]) for w in wide)
        block.set_product_kernel(which)
        p = block.Fp8Product()
        c = p(qa, qb, dtype=F32)
        block.set_product_kernel(0)
        assert p.status() == cb.OK
        check_product(c, qa, qb)
