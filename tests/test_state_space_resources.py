"""What the compiler made of the state space operators' kernels, read from the metadata of the built library."""
import re

from tests.test_kernel_resources import notes  # noqa: F401  (a fixture)

KERNELS = r"\d+(convolution_(forward|backward|step|sum)|selective_(forward|back_maps|backward|line|carry|widen|step|sum)|block_norm_(forward|backward|wide_backward|sum))_kernel"


def test_no_scratch(notes):  # noqa: F811
    """States, rows and windows that a lane holds stay in registers."""
    kernels = {k: v for k, v in notes.items() if re.search(KERNELS, k)}
    assert len([k for k in kernels if "selective" in k]) > 80 and len([k for k in kernels if "convolution" in k]) > 60 and len([k for k in kernels if "block_norm" in k]) > 60
    assert not {k: v for k, v in kernels.items() if v[0]}


def test_two_waves_of_the_reverse_scan_share_a_simd(notes):  # noqa: F811
    kernels = {k: v for k, v in notes.items() if re.search(r"selective_backward_kernelI\w+ELi1EEE", k)}
    assert len(kernels) == 12
    assert not {k: v for k, v in kernels.items() if v[2] > 256 or v[1] > 160 * 1024 // 8}
