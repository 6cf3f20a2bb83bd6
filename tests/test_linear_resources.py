"""Registers of the kernels of linear attention and group norm, from the built library: a value
in scratch memory lies within the serial chain of every chunk (addresses kept there took a
fifth of the gradients' time), and in every row's.  A few registers that are read once a chunk
or once a row may lie there: 8 of a work item."""

import re

from test_kernel_resources import kernels  # noqa: F401  (a fixture)

NAME = re.compile(r"k_lin_(forward|backward|backward_by_two|backward_kv|state|scan|step|decay|"
                  r"decay_sum)\w*|k_gn_\w+")


def test_next_to_no_value_lies_in_scratch_memory(kernels):  # noqa: F811
    mine = {n: k for n, k in kernels.items() if NAME.search(n)}
    assert len([n for n in mine if "k_lin_" in n]) > 40 and any("k_gn_" in n for n in mine)
    bad = {n: k[".private_segment_fixed_size"] for n, k in mine.items()
           if k[".private_segment_fixed_size"] > 32 or k[".vgpr_spill_count"] > 8}
    assert not bad, bad
