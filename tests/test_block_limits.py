"""Numbers at the ends of their ranges in the block operators' arguments.  Nothing is launched."""
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
