"""Kernels that are launched while the one before them on the stream still runs (programmatic launches) wait for it before they read memory.  What they
read may be written while they are resident already, so it must not come through the non-coherent cache.  Neither shows in results: the sources are checked."""
import os
import re

import pytest

from paper_1511_05950_b200 import build

# files whose kernels all start with wait_for_earlier() (units.cuh: what they share)
DEPENDENT = ("units.cuh", "pack_kernels.cuh", "norm_kernels.cuh", "mma_kernels.cuh", "head_kernels.cuh")


def code(name):
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", DEPENDENT)
def test_no_load_through_the_non_coherent_cache(name):
    assert not re.findall(r"__ldg\b|ld\.global\.nc|__restrict__", code(name))


@pytest.mark.parametrize("name", DEPENDENT[1:])
def test_every_kernel_waits_before_it_lets_the_next_one_start(name):
    text = code(name)
    bodies = [text[m.start():] for m in re.finditer(r"__global__", text)]
    assert bodies
    for body in bodies:
        kernel = re.search(r"(\w+)\((?:const|unsigned|[A-Z])[^;]*?\)\s*\{", body).group(1)
        waits, starts = body.find("wait_for_earlier()"), body.find("let_next_start()")
        if kernel == "order_kernel":               # always the first of its call, launched plainly
            waits = 0
        assert 0 <= waits < starts, kernel
