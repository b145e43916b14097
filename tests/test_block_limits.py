"""Numbers at the ends of their ranges in the block operators' arguments.  """
import pytest

from paper_2410_15352_b200 import binding as cb
from paper_2410_15352_b200 import block
from paper_2410_15352_b200.build import build_library


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


@pytest.mark.parametrize("kw", [
    dict(scaling="linear", factor=1e-310), dict(scaling="by_parts", factor=1e-310, trained_length=1.0), dict(scaling="base", factor=1e-320),
    dict(scaling="base", factor=1e305, base=1e9)])
def test_rotary_speeds_that_are_not_numbers_are_refused(kw):
    """An infinite speed has no fraction of a turn; a base out of range has no speeds."""
    with pytest.raises(cb.CompactError) as e:
        block.Rotary(64, **kw)
    assert e.value.code == cb.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=1e-300), dict(scaling="linear", factor=1e300), dict(scaling="base", factor=1e-3),
                                dict(scaling="by_parts", factor=1e-300), dict(base=1e300)])
def test_rotary_speeds_at_the_ends_of_the_range(kw):
    block.Rotary(64, **kw)


@pytest.mark.parametrize("eps", [float("inf"), float("nan"), -1.0, 1e39])
def test_norm_eps_beyond_a_float_is_refused(eps):
    """1e39 is finite as a double and infinite as the kernel's float, which would make every output zero."""
    with pytest.raises(cb.CompactError) as e:
        block.RMSNorm(64, eps=eps)
    assert e.value.code == cb.ERR_INVALID_ARG


@pytest.mark.parametrize("tokens", [0, 4])
def test_norm_infinite_eps_is_refused_by_the_library(tokens):
    p = 0x1000      # an aligned address: no refused call looks behind it
    call = block.lib().compact_rms_norm_fwd
    assert call(cb.BF16, tokens, 64, float("inf"), p, 64, None, 0, p, None, 0, p, 64, None, 0, None, 0, None, 0, None) == cb.ERR_INVALID_ARG


def test_rotary_outputs_that_run_into_each_other_are_refused():
    """Heads or tokens written to one place, or closer than a head is long: which of them stays is chance."""
    rot, p = block.Rotary(64), 0x1000

    def call(tokens=2, heads=2, kv=2, qo=(128, 64), ko=(128, 64)):
        return block.lib().compact_rotary_apply(rot._h, cb.BF16, tokens, heads, kv, p, 0, 0, p, 0, 0, None, 64, 0, 0, p, *qo, p, *ko, None)

    for bad in ((0, 64), (128, 0), (128, 63), (63, 64), (-63, 64), (128, -32)):
        assert call(qo=bad) == cb.ERR_INVALID_ARG and call(ko=bad) == cb.ERR_INVALID_ARG
    # an address off its element's boundary is looked at later: these strides pass
    p += 1
    for good in ((128, 64), (64, 128), (-64, 128), (128, -64)):
        assert call(qo=good) == cb.ERR_ALIGNMENT
    assert call(tokens=1, qo=(0, 64), ko=(0, 64)) == call(heads=1, kv=1, qo=(64, 0), ko=(64, 0)) == cb.ERR_ALIGNMENT
    assert call(kv=0, ko=(0, 0)) == cb.ERR_ALIGNMENT


@pytest.mark.gpu
def test_rotary_broadcast_output_is_refused_and_input_is_not():
    import torch

    rot = block.Rotary(64)
    one = torch.randn((1, 2, 64), device="cuda")
    many = one.expand(4, 2, 64)
    with pytest.raises(cb.CompactError) as e:
        rot.forward(one.repeat(4, 1, 1), None, q_out=many)
    assert e.value.code == cb.ERR_INVALID_ARG
    assert torch.equal(rot.forward(many, None)[0], rot.forward(many.contiguous(), None)[0])
