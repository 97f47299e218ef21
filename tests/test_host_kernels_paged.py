"""Kernels of attention over the paged cache that the library has: the shapes that plans ask for (csrc/lq_plan_paged.h), all of them and
no others."""
import itertools
import re

from paper_2503_19950_amd import binding


def test_the_library_has_the_kernels_that_plans_ask_for():
    with open(binding.LIB_PATH, "rb") as f:
        names = re.findall(rb"attn_paged_kernelILb([01])ELi(\d+)ELi(\d+)ELi([12])ELi([01])ELb([01])ELb([01])E", f.read())
    got = {tuple(int(x) for x in name) for name in names}
    # type, head dimension, wavefronts, sets of 16 heads, rows alike or listed, step, scores changed
    want = set(itertools.product((0, 1), (64, 96, 128), (4, 8), (1,), (0, 1), (0, 1), (0, 1)))
    want |= set(itertools.product((0, 1), (64, 96, 128), (4,), (2,), (0, 1), (0, 1), (0, 1)))
    want |= set(itertools.product((0, 1), (64,), (16,), (1,), (1,), (0, 1), (0, 1)))
    assert got == want, sorted(got ^ want)
