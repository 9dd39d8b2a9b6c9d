"""Registers of the kernels of the calls around a reduced activation, read from the built
library (no GPU needed).  Scratch is memory traffic that results do not show."""
import re

from test_kernel_resources import code_objects, kernels  # noqa: F401 (fixtures)

NEW = re.compile(r"(fold_norm|norm_grad|norm_dweight|route|route_grad|plan_count|plan_place|dispatch"
                 r"|combine|combine_grad)_kernel")
# norm_grad_kernel of 4 and 8 pieces a thread: 9 to 20 registers of 128 are spilled
SPILLS = re.compile(r"norm_grad_kernelINS_\d+T\w+?ELi[48]ELi0E")


def test_scratch(kernels):  # noqa: F811
    got = {n: scratch for n, (_, scratch) in kernels.items() if NEW.search(n)}
    assert len(got) > 200
    spills = [n for n in got if SPILLS.search(n)]
    assert len(spills) == 4, spills
    bad = [(n, s) for n, s in got.items() if s > (84 if n in spills else 0)]
    assert not bad, bad
