"""Kernels of the queries' and keys' calls in the built library: none that no call can reach, and none missing."""
import re

from test_lm_kernels import kernels  # noqa: F401  (a fixture)


def plan(width, rotated, f32, interleaved):
    """(elements of a chunk, lanes of a head, 0: whole chunks, 1: ragged ones, 2: rotated inside one) as the calls choose them."""
    largest, half = 4 if f32 else 8, rotated // 2
    for e in (largest, largest // 2, largest // 4):
        inner = not interleaved and 0 < rotated <= e
        if e < 2 or width < e or (not interleaved and not inner and 0 < half < e):
            continue
        turned = 0 if inner else -(-(rotated if interleaved else half) // e)
        begin = 0 if inner else turned * e if interleaved and turned * e <= width else rotated
        others = -(-(width - begin) // e)
        units, of_lane = (turned + others + 1) // 2 if interleaved else turned + (others + 1) // 2, 2 if e == 2 else 1
        if units > 64 * of_lane:
            continue
        if e < largest:
            group = 8 if e == 4 and units <= 8 else 16 if units <= 16 * of_lane else 64
        else:
            group = 1 << (units - 1).bit_length()
        # every unit has a lane, every angle of a token a place, and chunks that begin further down begin in the head
        assert group <= 64 and units <= group * of_lane and rotated // 2 <= group * of_lane * e
        assert not interleaved or turned * e <= width or rotated >= e
        return e, group, 2 if inner else int(e < largest or width % e > 0 or rotated % (e if interleaved else 2 * e) > 0)
    assert (width + 1) // 2 <= 256
    return 1, 16 if (width + 1) // 2 <= 64 else 64, 0


def test_the_layouts_of_heads_are_those_that_calls_choose(kernels):  # noqa: F811
    reached = set()
    for f32 in (True, False):
        for interleaved in (True, False):
            for width in range(1, 513):
                for rotated in range(0, width + 1, 2):
                    e, group, form = plan(width, rotated, f32, interleaved)
                    reached |= {(f32, e, group, interleaved and e > 1, form, nt) for nt in ((False, True) if e > 1 and form == 0 else (False,))}
    for direction in ("forward", "backward"):
        built = set()
        for name in kernels:
            m = re.search(rf"\dqk_{direction}_kernelI(f|N3bns6bf16_tE|NS\w*_6bf16_tE)Li(\d+)ELi(\d+)ELi\d+ELb([01])ELi([012])ELb([01])E", name)
            if m:
                built.add((m[1] == "f", int(m[2]), int(m[3]), m[4] == "1", int(m[5]), m[6] == "1"))
        assert built == reached
