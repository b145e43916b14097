"""What the sources of the block operators must not say."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_15352_b200", "csrc")


def test_no_kernel_promises_that_its_inputs_stand_still():
    """Their kernels are launched before their predecessors end: an input may be written until griddepcontrol.wait, so that neither
    __restrict__ nor the read-only path may be used for one."""
    files = glob.glob(os.path.join(CSRC, "block_*.cuh")) + [os.path.join(CSRC, "block_api.cu")]
    assert len(files) >= 6
    for path in files:
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(path).read(), flags=re.S)
        assert not re.search(r"__restrict|__ldg\b|ld\.global(\.\w+)*\.nc\b", code), path


def test_every_kernel_waits_for_its_predecessors():
    for path in glob.glob(os.path.join(CSRC, "block_*.cuh")):
        code = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(path).read(), flags=re.S)
        kernels = re.split(r"__global__", code)[1:]
        for k in kernels:
            assert "let_successor_start();" in k and "wait_for_predecessors();" in k, path
