"""Kernels of the queries' and keys' calls in the built library: none that no call can reach, and none missing."""
import re

from test_lm_kernels import kernels  # noqa: F401  (a fixture)


def plan(width, rotated, f32, interleaved):
    """(elements of a chunk, lanes of a head, whether chunks overlap) as the calls choose them."""
    whole, rest, part = 4 if f32 else 8, width - rotated, rotated if interleaved else rotated // 2
    for e in (whole, whole // 2, whole // 4):
        if e < 2 or width < e or 0 < part < e:
            continue
        turned, others = -(-part // e), -(-rest // e)
        units, of_lane = (turned + others + 1) // 2 if interleaved else turned + (others + 1) // 2, 2 if e == 2 else 1
        if units > 64 * of_lane:
            continue
        if e < whole:
            group = 8 if e == 4 and units <= 8 else 16 if units <= 16 * of_lane else 64
        else:
            group = max(4, 1 << (units - 1).bit_length())
        # every unit has a lane, every angle of a token a place
        assert group <= 64 and units <= group * of_lane and rotated // 2 <= group * of_lane * e
        return e, group, e < whole or part % e > 0 or rest % e > 0
    assert (width + 1) // 2 <= 256
    return 1, 16 if (width + 1) // 2 <= 64 else 64, False


def test_the_layouts_of_heads_are_those_that_calls_choose(kernels):  # noqa: F811
    reached = set()
    for f32 in (True, False):
        for interleaved in (True, False):
            for width in range(1, 513):
                for rotated in range(0, width + 1, 2):
                    e, group, ragged = plan(width, rotated, f32, interleaved)
                    reached |= {(f32, e, group, interleaved and e > 1, ragged, nt) for nt in ((False, True) if e > 1 and not ragged else (False,))}
    for direction in ("forward", "backward"):
        built = set()
        for name in kernels:
            m = re.search(rf"\dqk_{direction}_kernelI(f|N3bns6bf16_tE|NS\w*_6bf16_tE)Li(\d+)ELi(\d+)ELi\d+ELb([01])ELb([01])ELb([01])E", name)
            if m:
                built.add((m[1] == "f", int(m[2]), int(m[3]), m[4] == "1", m[5] == "1", m[6] == "1"))
        assert built == reached
