"""The bits of the device status word tell the waits apart: read from the sources, since no test makes most of them expire."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_06564_b200", "csrc")


def _bits():
    with open(os.path.join(CSRC, "ptx.cuh")) as f:
        return {name: int(bit) for name, bit in re.findall(r"(kStatusTimeout\w+) = 1u << (\d+)", f.read())}


def _users(name):
    found = set()
    for path in glob.glob(os.path.join(CSRC, "*.cu")):
        with open(path) as f:
            if re.search(rf"\b{name}\b", f.read()):
                found.add(os.path.basename(path))
    return found


def test_every_bit_is_its_own():
    bits = _bits()
    assert len(bits) >= 5 and len(set(bits.values())) == len(bits) and max(bits.values()) < 32


def test_the_bits_of_one_kernel_alone():
    assert _users("kStatusTimeoutUnpack") == {"gemm_w4a8.cu"}
    assert _users("kStatusTimeoutScales") == {"gemm_fp8.cu"}
    assert _users("kStatusTimeoutSelfTest") == {"api.cu"}
