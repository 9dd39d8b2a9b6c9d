"""Scratch of the experts' products, family by family, close to what the built kernels have (no
GPU needed): bytes of a lane.  Results of 256 x 256 tiles on their way out need them, most
where they are fp32 or added to what is there, and operands that come by way of registers."""
import re

from test_kernel_resources import code_objects, kernels  # noqa: F401 (fixtures)

WIDE = "product_wide_kernelINS_%sENS_%sELb%sELb%sELb%sELb%sEEEv"   # gradient, transposed, adding, on the grid
TILES = "product_kernelINS_%sELb%sELb%sELb%sELi%sELi%sELb%sEEEv"   # gradient, transposed, on the grid, two sizes, halves
HALF, OWN = r"(\d)P(BF16|F16)", r"\dT\2"
FAMILIES = [   # name, most bytes
    # 16-bit operands on the grid, results of their own type; added to
    (WIDE % (HALF, OWN, "[01]", "[01]", "0", "1"), 16), (WIDE % (HALF, OWN, "1", "1", "1", "1"), 400),
    # the same off the grid, through registers
    (WIDE % (HALF, OWN, "0", "[01]", "0", "0"), 200),
    # fp32 results of 16-bit operands: weights as they lie and gradients; transposed; added to
    (WIDE % (HALF, "4TF32", "0", "0", "0", "1"), 464), (WIDE % (HALF, "4TF32", "1", "1", "0", "1"), 464),
    (WIDE % (HALF, "4TF32", "0", "1", "0", "1"), 528), (WIDE % (HALF, "4TF32", "1", "1", "1", "1"), 0),
    # fp32 operands, on the grid and off it
    (WIDE % ("4PF32", "4TF32", "0", "0", "0", "1"), 528), (WIDE % ("4PF32", "4TF32", "0", "1", "0", "1"), 592),
    (WIDE % ("4PF32", "4TF32", "0", "[01]", "0", "0"), 768),
    (WIDE % ("5PE4M3", r"\dT\w+", "0", "0", "0", "1"), 0),
    (WIDE % ("4PMx4", r"\dT(?:BF16|F16)", "0", "0", "0", "1"), 32), (WIDE % ("4PMx4", "4TF32", "0", "0", "0", "1"), 592),
    (r"product_narrow_kernelINS_\dP\w+ELb[01]ELb[01]EEEv", 0),
    (TILES % (r"\dP\w+", "[01]", "[01]", "1", "[12]", "[12]", "0"), 0),              # on the grid
    (TILES % (r"\dP\w+", "0", "[01]", "[01]", "1", "1", "1"), 0),                     # of far rows
    (TILES % (r"\dP(?:BF16|F16|F32)", "0", "[01]", "0", "[12]", "[12]", "0"), 0),    # off the grid
    (TILES % (r"\dP(?:BF16|F16|F32)", "1", "1", "0", "[12]", "[12]", "0"), 24),
    (TILES % ("5PE4M3", "0", "0", "0", "[12]", "[12]", "0"), 64),
    (TILES % ("4PMx4", "0", "0", "0", "1", "1", "0"), 64), (TILES % ("4PMx4", "0", "0", "0", "2", "2", "0"), 128)]


def test_every_kernel_keeps_to_its_familys_scratch(kernels):  # noqa: F811
    names = [n for n in kernels if re.search(r"\dproduct(_narrow|_wide)?_kernelI", n)]
    bad, used = [], set()
    for n in names:
        of = [(f, most) for f, most in FAMILIES if re.search(f, n)]
        assert len(of) == 1, (n, of)
        used.add(of[0][0])
        if kernels[n][1] > of[0][1]:
            bad.append((n, kernels[n][1], of[0][1]))
    assert not bad, bad
    assert len(used) == len(FAMILIES), [f for f, _ in FAMILIES if f not in used]
