"""Which kernels of the explainer operators use private memory, by the compiler's report: the
norm gradients of rows past 8192 columns, in every type, and no other."""
import re

from test_nn_kernel_resources import kernels


def test_what_spills():
    spilled = {name for _, name, _, scratch, _ in kernels() if scratch > 0}
    wide = {name for kind, name, *_ in kernels() if kind == "norm_grad_kernel" and
            re.search(r"I(DF16b|DF16_)Li1024ELi2E|IfLi1024ELi4E", name)}
    assert spilled == wide and len(wide) == 6
