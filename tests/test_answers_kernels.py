"""Kernels of the queries' and keys' calls in the built library: none that no call can reach, and none missing."""
import re

from test_lm_kernels import kernels  # noqa: F401  (a fixture)


def plan(width, rotated, f32, interleaved):
    """(elements of a chunk, lanes of a head) as the calls choose them."""
    for e in (4 if f32 else 8, 4, 2):
        if width % e or rotated % (e if interleaved else 2 * e):
            continue
        units = (width // e + 1) // 2 if interleaved else rotated // (2 * e) + ((width - rotated) // e + 1) // 2
        of_lane, group = (2, 8) if e == 2 else (1, 4)
        while group * of_lane < units:
            group *= 2
        assert group <= 64 and group * of_lane * e * 2 >= width
        return e, group
    return (1, 16) if (width + 1) // 2 <= 64 else (1, 64)


def test_the_layouts_of_heads_are_those_that_calls_choose(kernels):  # noqa: F811
    reached = set()
    for f32 in (True, False):
        for interleaved in (True, False):
            for width in range(1, 513):
                for rotated in range(0, width + 1, 2):
                    e, group = plan(width, rotated, f32, interleaved)
                    neighbours, whole = interleaved and e > 1, e == (4 if f32 else 8)
                    reached |= {(f32, e, group, neighbours, nt) for nt in ((False, True) if whole else (False,))}
    for direction in ("forward", "backward"):
        built = set()
        for name in kernels:
            m = re.search(rf"\dqk_{direction}_kernelI(f|N3bns6bf16_tE|NS\w*_6bf16_tE)Li(\d+)ELi(\d+)ELi\d+ELb([01])ELb([01])E", name)
            if m:
                built.add((m[1] == "f", int(m[2]), int(m[3]), m[4] == "1", m[5] == "1"))
        assert built == reached
