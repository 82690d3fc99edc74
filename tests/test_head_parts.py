"""The three bf16 parts of an fp32 value and the six products of two values' parts, on the CPU: what test_gpu_head_values expects of a product is what all six
give, and none of them can be left out or taken twice without a bit that changes."""
import pytest
import torch

from test_gpu_head_values import three_parts

PAIRS = [(0, 2), (2, 0), (1, 1), (0, 1), (1, 0), (0, 0)]       # smallest first


def parts(x):
    hi = x.bfloat16().float()
    mid = (x - hi).bfloat16().float()
    return hi, mid, (x - hi - mid).bfloat16().float()


def product(x, y, pairs):
    a, b, total = parts(x), parts(y), torch.zeros_like(x)
    for i, j in pairs:
        total = total + a[i] * b[j]
    return total


CASES = {"hidden": (8 * three_parts(30, 1), torch.full((30,), 8.0)), "weight": (torch.full((30,), 8.0), 8 * three_parts(30, 2)),
         "middle": (torch.full((30,), 8 * (1 + 2.0 ** -9)), torch.full((30,), 8 * (1 + 2.0 ** -9)))}


@pytest.mark.parametrize("x,y", CASES.values(), ids=CASES)
def test_six_products_are_the_whole(x, y):
    assert torch.equal(sum(p.double() for p in parts(x)), x.double())
    assert torch.equal(product(x, y, PAIRS).double(), x.double() * y.double())


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("times", [0, 2])
def test_each_of_them_shows(pair, times):
    others = [p for p in PAIRS if p != pair] + [pair] * times
    assert any(not torch.equal(product(x, y, others).double(), x.double() * y.double()) for x, y in CASES.values())
