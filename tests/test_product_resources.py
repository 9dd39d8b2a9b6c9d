"""Registers of the kernels of the experts' products, the gated activation and 4-bit rows,
read from the built library (no GPU needed).  Scratch is memory traffic that results do not
show."""
import re

from test_kernel_resources import code_objects, kernels  # noqa: F401 (fixtures)

NEW = re.compile(r"\d(product|product_narrow|product_wide|gate|quant_mx4|dequant_mx4)_kernelI")
WIDE = re.compile(r"product_wide_kernelI")           # spills at the ends of tiles, some bytes more or less
LOOSE = re.compile(r"product_kernelI.*Lb0ELi[12]E")  # operands off the grid, in registers


def test_scratch(kernels):  # noqa: F811
    got = {n: scratch for n, (_, scratch) in kernels.items() if NEW.search(n)}
    assert len([n for n in got if "product_narrow" in n]) == 16
    assert len([n for n in got if "product_wide_kernelINS_5PE4M3" in n]) == 3
    assert len([n for n in got if "gate_kernel" in n]) == 6 and len([n for n in got if "mx4_kernel" in n]) == 6
    most = lambda n: 800 if WIDE.search(n) else 128 if LOOSE.search(n) else 0
    bad = [(n, s) for n, s in got.items() if s > most(n)]
    assert not bad, bad
    # the kernels of the common types on the grid, with outputs of their own type
    for own in ("5PBF16ENS_5TBF16", "4PF16ENS_4TF16"):
        for kind in ("Lb0ELb0ELb0ELb1", "Lb1ELb1ELb0ELb1"):
            assert [s for n, s in got.items() if "product_wide_kernelINS_%sE%s" % (own, kind) in n] == [0], (own, kind)
