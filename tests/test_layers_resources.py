"""What the compiler made of the layer operators' kernels, read from the metadata of the built library."""
import re

from tests.test_kernel_resources import notes, resources  # noqa: F401  (fixtures)


def test_no_scratch_where_arrays_lie_as_allocated(resources):  # noqa: F811
    """Maps, rows and moments that a thread holds between two passes over them stay in registers.  (Kernels for elements of 16 bits at addresses
    that are no multiple of four bytes are left out: those of the recurrence without scalar addressing.)"""
    kernels = {k: v for k, (v, _) in resources.items() if re.search(r"recurrence_\w+_kernel|norm_\w+_kernel|adamw_\w+_kernel", k)}
    assert len([k for k in kernels if "norm_" in k and "adamw" not in k]) > 50 and len([k for k in kernels if "recurrence" in k]) > 50
    slow = re.compile(r"recurrence_(forward|backward)_kernelI\w+?Lb0E")
    assert not {k: v for k, v in kernels.items() if v and not slow.search(k)}


def test_workgroups_of_a_recurrence_share_a_compute_unit(notes):  # noqa: F811
    """Blocks that hand their maps on wait for each other: three workgroups a compute unit forward, two in reverse."""
    forward = {k: v for k, v in notes.items() if re.search(r"recurrence_forward_kernelI(f|DF16b|DF16_)Lb1ELi\dELi8ELi4ELb1", k)}
    backward = {k: v for k, v in notes.items() if re.search(r"recurrence_backward_kernelI(f|DF16b|DF16_)Lb1ELi\dELi8ELi4ELb1", k)}
    assert len(forward) == len(backward) == 6
    assert not {k: v for k, v in forward.items() if v[2] > 168 or v[1] > 160 * 1024 // 3}
    assert not {k: v for k, v in backward.items() if v[2] > 256 or v[1] > 160 * 1024 // 2}
