"""No kernel of the layer operators uses scratch memory, none excepted."""
import re

from tests.test_kernel_resources import notes, resources  # noqa: F401  (fixtures)


def test_no_scratch_in_any_kernel(resources):  # noqa: F811
    """Maps, rows and moments that a thread holds between two passes over them stay in registers, at any alignment, in workgroups of one
    block or of all."""
    of = lambda pattern: {k: v for k, (v, _) in resources.items() if re.search(pattern, k)}  # noqa: E731
    recurrence, norm, adamw = of(r"\d+recurrence_\w+_kernel"), of(r"\d+norm_\w+_kernel"), of(r"\d+adamw_\w+_kernel")
    # whole sequences: 3 types x 2 kinds x 3 ways of access x 6 launches (2 or 8 positions with one wave; two, four and eight waves; ahead)
    assert len([k for k in recurrence if re.search("(forward|backward)_kernel", k)]) == 2 * 3 * 2 * 3 * 6
    assert len(norm) > 150 and len(adamw) >= 8
    assert not {k: v for kernels in (recurrence, norm, adamw) for k, v in kernels.items() if v}
