"""Kernels of the language-model operators in the built library: none that no call can reach."""
import os
import re

import pytest

from test_scratch import _code_objects, _kernels, entry


@pytest.fixture(scope="module")
def kernels():
    if not os.path.exists(entry.LIB):
        pytest.skip("libbns.so is not built")
    names = set()
    for elf in _code_objects(open(entry.LIB, "rb").read()):
        names |= set(_kernels(elf))
    return names


def arguments(kernels, kernel):
    """The integer and truth-value arguments of a template's kernels."""
    found = [tuple(int(v) for v in re.findall(r"L[ib](\d+)E", n)) for n in kernels if re.search(r"\d" + kernel + "I", n)]
    assert found, kernel
    return found


def test_gradients_laid_out_in_parts_have_tiles_of_32_tokens_at_least(kernels):
    statistics, gradient, parts = range(3)
    for kernel, at in (("direct_logits_kernel", 1), ("stream_logits_kernel", 1)):
        tiles = {e: {a[at] for a in arguments(kernels, kernel) if a[5 if "direct" in kernel else 2] == e} for e in (statistics, gradient, parts)}
        least = 16 if "direct" in kernel else 1             # (stream: in units of 16)
        assert min(tiles[statistics]) == min(tiles[gradient]) == least and min(tiles[parts]) == 2 * least


def test_plans_of_few_rows_of_the_norm_have_no_non_temporal_form(kernels):
    forms = {}
    for tpr, vpt, _, nt in arguments(kernels, "rms_forward_kernel"):
        forms.setdefault((tpr, vpt), set()).add(nt)
    assert forms[256, 1] == forms[1024, 1] == {0} and forms[256, 2] == forms[512, 4] == {0, 1}
