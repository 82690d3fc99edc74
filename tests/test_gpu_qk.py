"""Queries and keys on the GPU (norm of every head, rotation by position, and their gradients) against the definition in 64 bits (answers_reference).

Tolerances, with u = 2^-24.  A head's sum of squares has 16 terms a lane in turn and six steps between lanes, all positive: 22 u relative, the mean and eps
3 u more; r carries half of that and 2 u of the estimate: 15 u; v = x (r w) two roundings more: V = 17 u.  An angle's remainder is rounded to fp32 (u of at most
0.79), as are its factor and their product (0.79 * 3 u), and the series have 2 u each of rounding and 0.03 u of truncation: C = 5 u absolute for cos and sin, besides
four roundings of the product in fp64, here and in the reference, 2^-51 of the angle.  A rotated element is then off by (|v_a| + |v_b|) (V + C + 3 u), and by
half a unit of its type.  Backward: g the same without V (G = C + 3 u); x^ 16 u; the mean of weight g x^ its terms' errors and 28 u of their magnitudes."""
import math
from fractions import Fraction

import pytest
import torch

import answers_reference as ref
from answers_reference import HALF_ULP, TYPES, U, Strided, tail_is_whole, written
from paper_1810_10962_amd import bns

pytestmark = pytest.mark.gpu
EPS = 1e-6


def layout(kind, tokens, heads, width):
    """Strides from token to token and head to head."""
    return {"dense": (heads * width, width), "packed": ((heads + 3) * width + 8, width), "loose": (heads * (width + 5) + 3, width + 5),
            "head_major": (width, tokens * width), "head_major_loose": (width + 3, tokens * (width + 3) + 1)}[kind]


def make(tokens, heads, width, dtype, seed, far):
    g = torch.Generator().manual_seed(seed * 7919 + tokens * 31 + heads * 7 + width)
    x = (torch.randn(tokens, heads, width, generator=g) * torch.exp(torch.randn(tokens, heads, 1, generator=g))).to(TYPES[dtype])
    return x, (1 + 0.3 * torch.randn(width, generator=g)), torch.randint(-far, far, (tokens,), generator=g), torch.randn(tokens, heads, width, generator=g).to(TYPES[dtype])


def frequencies(rotated):
    return 10000.0 ** (-torch.arange(rotated // 2, dtype=torch.float64) * 2 / max(1, rotated))


def angle_off(positions, f):
    """C of the docstring for every element of a head, with the fp64 part."""
    return 5 * U + 2.0 ** -51 * float(positions.abs().max() if len(positions) else 0) * float(f.max() if len(f) else 0)


def assert_forward(got, x, weight, positions, f, rotated, interleaved, dtype):
    want, v = ref.qk_forward(x.double(), None if weight is None else weight.double(), positions, f, rotated, interleaved, EPS)
    v_off = 0 if weight is None else 17 * U
    off = ref.beside(v, rotated, interleaved) * (v_off + angle_off(positions, f) + 3 * U) + HALF_ULP[dtype] * want.abs() + 1e-37
    worst = ((got.double().cpu() - want).abs() - off).max().item()
    assert worst <= 0, f"worst excess {worst:.3e}"


def assert_backward(got, got_dw, x, weight, positions, f, dy, rotated, interleaved, dtype):
    w = None if weight is None else weight.double()
    want, dw, g, r = ref.qk_backward(x.double(), w, positions, f, dy.double(), rotated, interleaved, EPS)
    g_off = ref.beside(g, rotated, interleaved) * (angle_off(positions, f) + 3 * U)
    off = g_off
    if weight is not None:
        xh = x.double() * r
        mean = (w * g * xh).mean(-1, keepdim=True)
        mean_off = ((w * xh).abs() * g_off + 28 * U * (w * g * xh).abs()).mean(-1, keepdim=True) + 18 * U * mean.abs()
        off = r * (w.abs() * g_off + 3 * U * (w * g).abs() + xh.abs() * mean_off + 18 * U * (xh * mean).abs()) + 16 * U * want.abs()
        n = x.shape[0] * x.shape[1]
        terms = (xh * g).abs().sum((0, 1))
        dw_off = (xh.abs() * g_off).sum((0, 1)) + (17 + min(n, 300) + 100) * U * terms + 1e-37     # (a lane's terms in turn, then 32 slots, 32 and 32 sums)
        worst = ((got_dw.double().cpu() - dw).abs() - dw_off).max().item()
        assert worst <= 0, f"dweight: worst excess {worst:.3e}"
    worst = ((got.double().cpu() - want).abs() - (off + HALF_ULP[dtype] * want.abs() + 1e-37)).max().item()
    assert worst <= 0, f"dx: worst excess {worst:.3e}"


CASES = [  # tokens, q heads, k heads, width, rotated, interleaved, norm, layout, far
    (1, 1, 1, 2, 2, False, True, "dense", 4),
    (1, 32, 8, 128, 128, False, True, "packed", 2 ** 20),
    (3, 5, 1, 128, 128, True, True, "loose", 1000),
    (37, 7, 2, 64, 64, False, True, "packed", 5000),
    (130, 3, 3, 96, 48, False, True, "dense", 5000),
    (29, 9, 3, 80, 80, False, True, "head_major", 5000),
    (65, 6, 2, 256, 64, True, True, "packed", 2 ** 17),
    (18, 2, 1, 512, 512, False, True, "loose", 100),
    (17, 2, 1, 512, 0, True, True, "dense", 100),
    (33, 4, 4, 100, 50, True, True, "dense", 5000),
    (21, 3, 1, 101, 100, False, True, "loose", 5000),
    (9, 3, 2, 1, 0, False, True, "dense", 5),
    (6, 2, 2, 3, 2, True, True, "loose", 50),
    (11, 2, 1, 501, 250, False, True, "head_major_loose", 5000),
    (40, 12, 0, 32, 32, False, True, "dense", 5000),
    (40, 0, 5, 16, 8, False, True, "packed", 5000),
    (26, 70, 2, 24, 16, False, True, "dense", 5000),
    (50, 4, 2, 128, 128, False, False, "packed", 5000),
    (50, 4, 2, 60, 20, True, False, "loose", 5000),
    (1500, 3, 2, 48, 32, True, True, "dense", 2 ** 30),
    (14, 3, 2, 390, 260, False, True, "loose", 5000),
    (23, 5, 1, 130, 64, True, True, "packed", 5000),
    (7, 2, 2, 514 - 4, 510, True, True, "dense", 5000),
    (5, 40, 24, 6, 4, False, True, "dense", 5000),
    (3000, 33, 1, 16, 16, False, True, "packed", 5000),
    (31, 3, 3, 20, 8, False, True, "packed", 5000),
    (31, 5, 2, 84, 40, False, True, "loose", 5000),
    (12, 2, 1, 236, 236, True, True, "packed", 5000),
    (12, 2, 1, 500, 252, True, True, "dense", 5000),
    (19, 4, 2, 66, 34, True, True, "packed", 5000),
    (8, 2, 1, 250, 250, True, True, "dense", 5000),
    (70, 6, 2, 83, 40, True, True, "dense", 5000),
    (70, 6, 2, 83, 40, False, True, "packed", 5000),
    (90, 23, 5, 46, 10, False, True, "dense", 5000),
    (33, 30, 30, 47, 46, False, True, "loose", 5000),
    (33, 7, 3, 47, 46, True, False, "dense", 5000),
    (12, 5, 2, 213, 212, True, True, "packed", 5000),
    (12, 5, 2, 243, 242, False, True, "head_major", 5000),
    (9, 2, 1, 507, 10, False, True, "dense", 5000),
    (9, 2, 1, 511, 36, False, True, "packed", 5000),
    (9, 2, 1, 509, 18, True, True, "head_major_loose", 5000),
    (1, 3, 1, 31, 30, False, True, "dense", 5000),
    (40, 3, 2, 9, 8, True, True, "packed", 5000),
    (40, 3, 2, 17, 16, False, True, "dense", 5000),
    (40, 3, 2, 26, 0, False, True, "dense", 5000),
    (40, 3, 2, 14, 12, True, True, "loose", 5000),
    (600, 16, 16, 25, 18, False, True, "dense", 5000),
    (2, 32, 8, 128, 128, False, True, "packed", 5000),      # (the sums of one block: up to 8 turns of a wave)
    (3, 32, 8, 128, 128, False, True, "packed", 5000),
    (2, 0, 8, 64, 64, True, True, "dense", 5000),
    (1, 5, 0, 243, 242, False, True, "dense", 5000),
    (32, 4, 4, 16, 16, False, True, "dense", 5000),
    (33, 4, 4, 16, 16, False, True, "dense", 5000),
    (40, 9, 3, 16, 4, False, True, "dense", 5000),
    (40, 9, 3, 16, 4, True, True, "packed", 5000),
    (40, 9, 3, 16, 8, False, True, "dense", 5000),
    (40, 9, 3, 9, 8, False, True, "dense", 5000),
    (40, 9, 3, 9, 2, False, True, "packed", 5000),
    (40, 9, 3, 9, 6, True, True, "dense", 5000),
    (40, 5, 3, 11, 10, True, True, "dense", 5000),
    (40, 5, 3, 10, 6, False, True, "dense", 5000),
    (40, 5, 3, 7, 6, False, True, "loose", 5000),
    (40, 5, 3, 5, 4, True, True, "dense", 5000),
    (40, 5, 3, 13, 6, False, False, "dense", 5000),
    (20, 5, 3, 101, 2, True, True, "dense", 5000),
    (20, 5, 3, 101, 2, False, True, "dense", 5000),
    (20, 5, 3, 509, 6, False, True, "dense", 5000),
    (20, 5, 3, 2, 0, False, True, "dense", 5000),
    (20, 5, 3, 12, 12, True, True, "dense", 5000),
    (300, 70, 1, 16, 16, False, True, "packed", 5000),
    (300, 64, 63, 8, 8, True, True, "dense", 5000),
    (1000, 2, 1, 8, 0, False, True, "head_major", 5000),
    (500, 33, 8, 32, 16, False, True, "loose", 5000),
    (200, 130, 5, 15, 14, True, True, "dense", 5000),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward_and_backward(case, dtype):
    tokens, hq, hk, width, rotated, interleaved, norm, kind, far = CASES[case]
    print(f"[gpu-case] qk {CASES[case]} {dtype}", flush=True)
    f = frequencies(rotated)
    data = [make(tokens, h, width, dtype, seed, far) for seed, h in enumerate((hq, hk))]
    positions = data[0][2]
    weight_dtype = "bf16" if case % 3 == 2 else "f32"
    weights = [d[1].to(TYPES[weight_dtype]) if norm else None for d in data]
    strides = [layout(kind, tokens, h, width) for h in (hq, hk)]
    other = [layout("loose" if kind == "dense" else "dense", tokens, h, width) for h in (hq, hk)]
    x = [Strided(d[0], (*s, 1)) if h else None for d, s, h in zip(data, strides, (hq, hk))]
    dy = [Strided(d[3], (*s, 1)) if h else None for d, s, h in zip(data, other, (hq, hk))]
    empty = [torch.zeros(tokens, h, width, dtype=TYPES[dtype]) for h in (hq, hk)]
    out = [Strided(e, (*s, 1), written=True) if h else None for e, s, h in zip(empty, other, (hq, hk))]
    dx = [Strided(e, (*s, 1), written=True) if h else None for e, s, h in zip(empty, strides, (hq, hk))]
    spec = bns.make_qk(tokens, hq, hk, width, dtype, rotated=rotated, interleaved=interleaved, weight_dtype=weight_dtype, eps=EPS, q=strides[0], k=strides[1],
                       q_out=other[0], k_out=other[1], dq=strides[0], dk=strides[1])
    def sliced(t):          # at an element's alignment only
        return None if t is None else torch.cat([t[:1], t]).cuda()[1:]

    cw = [sliced(w) for w in weights]
    cp, cf = (sliced(positions), sliced(f)) if rotated else (None, None)
    bns.bns_qk_forward(spec, x[0], x[1], *cw, cp, cf, out[0], out[1])
    room = bns.bns_qk_workspace_bytes(spec)
    workspace, space = written(room, dtype=torch.uint8)
    dw = [written(width) if norm else (None, None) for _ in range(2)]
    bns.bns_qk_backward(spec, x[0] if norm else None, x[1] if norm else None, *cw, cp, cf, dy[0], dy[1], dx[0], dx[1], dw[0][1], dw[1][1], space)
    for i, h in enumerate((hq, hk)):
        if not h:
            if norm:
                assert bool((dw[i][1] == 0).all())
            continue
        assert_forward(out[i].check(), data[i][0], weights[i], positions, f, rotated, interleaved, dtype)
        assert_backward(dx[i].check(), dw[i][1], data[i][0], weights[i], positions, f, data[i][3], rotated, interleaved, dtype)
        if norm:
            tail_is_whole(dw[i][0], width)
    tail_is_whole(workspace, room)


@pytest.mark.parametrize("dtype,width", [("f32", 4), ("f32", 12), ("bf16", 8), ("bf16", 24), ("bf16", 20), ("bf16", 4), ("bf16", 6), ("f32", 6), ("bf16", 9), ("bf16", 22), ("f32", 10)])
def test_angles_of_an_earlier_call_that_are_nan(dtype, width):
    """Neighbours paired and turned all, an odd number of chunks: the last lane has one chunk, and the other's angles are whatever lies behind those of the
    head.  A call before whose angles are all NaN is what may lie there."""
    tokens, heads, rotated = 2048, 64, width // 2 * 2
    print(f"[gpu-case] qk after NaN {dtype} {width}", flush=True)
    wide = bns.make_qk(tokens, heads, heads, 512, dtype, rotated=512, interleaved=True)
    x = torch.ones(tokens, heads, 512, dtype=TYPES[dtype], device="cuda")
    bns.bns_qk_forward(wide, x, x, None, None, torch.ones(tokens, dtype=torch.int64, device="cuda"),
                       torch.full((256,), float("nan"), dtype=torch.float64, device="cuda"), torch.empty_like(x), torch.empty_like(x))
    f = frequencies(rotated)
    data = [make(tokens, heads, width, dtype, seed, 5000) for seed in (0, 1)]
    spec = bns.make_qk(tokens, heads, heads, width, dtype, rotated=rotated, interleaved=True, eps=EPS)
    w = [d[1].cuda() for d in data]
    dx = [torch.empty_like(d[0], device="cuda") for d in data]
    dw = [torch.empty(width, device="cuda") for _ in data]
    workspace = torch.empty(bns.bns_qk_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
    bns.bns_qk_backward(spec, *[d[0].cuda() for d in data], *w, data[0][2].cuda(), f.cuda(), *[d[3].cuda() for d in data], *dx, *dw, workspace)
    for i in range(2):
        assert_backward(dx[i], dw[i], data[i][0], data[i][1], data[0][2], f, data[i][3], rotated, True, dtype)


def test_one_weight_and_no_tokens():
    """Weights on one side only, of few and of many tokens; without tokens the weights' gradients are zero."""
    print("[gpu-case] qk one weight", flush=True)
    for tokens in (0, 2, 300):
        x, dy = (torch.randn(tokens, 4, 64, device="cuda") for _ in range(2))
        weight, turns = torch.rand(64, device="cuda") + 0.5, frequencies(64).cuda()
        positions = torch.arange(tokens, device="cuda")
        spec = bns.make_qk(tokens, 4, 4, 64, "f32", eps=EPS)
        workspace = torch.empty(bns.bns_qk_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
        results = []
        for weights in ((weight, None), (None, weight), (weight, weight)):
            dx = [torch.empty_like(x) for _ in "qk"]
            dw = [None if w is None else torch.full((64,), 7.0, device="cuda") for w in weights]
            bns.bns_qk_backward(spec, x, x, *weights, positions, turns, dy, dy, *dx, *dw, workspace)
            results.append((dx, dw))
        (a, da), (b, db), (both, dboth) = results
        assert torch.equal(a[0], both[0]) and torch.equal(b[1], both[1]) and torch.equal(both[0], both[1]) and torch.equal(a[1], b[0])
        assert torch.equal(da[0], dboth[0]) and torch.equal(db[1], dboth[1]) and torch.equal(dboth[0], dboth[1])
        assert da[1] is None and (tokens > 0 or not bool(dboth[0].any()))


@pytest.mark.parametrize("dtype,width,rotated,interleaved", [("f32", 64, 64, False), ("bf16", 128, 64, True), ("bf16", 83, 40, False), ("f32", 16, 4, False), ("bf16", 1, 0, False)])
def test_without_tokens_only_the_weights_gradients_are_written(dtype, width, rotated, interleaved):
    """No tokens: nothing is turned, so that positions and frequencies may be NULL as the tensors may; weights on either side have gradients of zero."""
    print(f"[gpu-case] qk without tokens {dtype} {width} {rotated}", flush=True)
    weight = torch.ones(width, device="cuda")
    for hq, hk in ((4, 2), (4, 0), (0, 0)):
        spec = bns.make_qk(0, hq, hk, width, dtype, rotated=rotated, interleaved=interleaved, eps=EPS)
        workspace = torch.full((bns.bns_qk_workspace_bytes(spec),), 255, dtype=torch.uint8, device="cuda")
        bns.bns_qk_forward(spec, None, None, weight, weight, None, None, None, None)
        for both in ((weight, weight), (weight, None), (None, weight), (None, None)):
            made = [None if w is None else written(width) for w in both]
            dw = [None if m is None else m[1] for m in made]
            bns.bns_qk_backward(spec, None, None, *both, None, None, None, None, None, None, *dw, workspace)
            for m in made:
                if m is not None:
                    assert not bool(m[1].any())
                    tail_is_whole(m[0], width)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [8, 1000])
def test_sums_of_the_weights_gradients_lose_nothing_small(tokens, dtype):
    """Terms that are whole numbers (x of one everywhere has r = 1): 2^25 and -2^25 in different lanes of one block, or in different blocks, and ones between them, which fp32
    drops beside those.  A lane has one term of a large magnitude and else zeros, so that its sum is exact, and so is a block's in fp64.  Blocks' sums are rounded to fp32, where numbers
    from 2^25 on are 4 apart: the two that have a large term and ones (blocks of bf16 have eight tokens, of fp32 four) may each be off by 2."""
    print(f"[gpu-case] qk sums of large and small terms {tokens} {dtype}", flush=True)
    heads, width = 8, 64
    dy = torch.zeros(tokens, heads, width)
    if tokens == 8:         # (one block)
        dy[:, 1:7] = 1
        dy[0, 0], dy[0, 7] = 2.0 ** 25, -2.0 ** 25
    else:
        dy[5::4, 3] = 1
        dy[0, 0], dy[tokens - 1, 7] = 2.0 ** 25, -2.0 ** 25
        dy[tokens - 3, 3] = 0
    want = dy.double().sum((0, 1))
    x = torch.ones(tokens, heads, width, dtype=TYPES[dtype], device="cuda")
    dw = [torch.empty(width, device="cuda") for _ in "qk"]
    spec = bns.make_qk(tokens, heads, heads, width, dtype, rotated=0, eps=0.0)
    ones, dy = torch.ones(width, device="cuda"), dy.to(TYPES[dtype]).cuda()
    bns.bns_qk_backward(spec, x, x, ones, ones, None, None, dy, dy, torch.empty_like(x), torch.empty_like(x), *dw,
                        torch.empty(bns.bns_qk_workspace_bytes(spec), dtype=torch.uint8, device="cuda"))
    for got in dw:
        assert float((got.double().cpu() - want).abs().max()) <= (0 if tokens == 8 else 2 * 2), (float(got[0]), float(want[0]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width,rotated", [(128, 128), (64, 32), (50, 20), (37, 34), (75, 22)])
def test_in_place_in_a_projection_s_result(width, rotated, dtype):
    """Queries and keys beside their values, replaced where they are; the values stay.  Then the same backward, gradients in place."""
    tokens, hq, hk = 45, 6, 2
    print(f"[gpu-case] qk in place {width} {rotated} {dtype}", flush=True)
    g = torch.Generator().manual_seed(width)
    whole = torch.randn(tokens, (hq + 2 * hk) * width, generator=g).to(TYPES[dtype]).cuda()
    positions, f = torch.arange(tokens, device="cuda") + 7, frequencies(rotated).cuda()
    weights = [(1 + 0.1 * torch.randn(width, generator=g)).cuda() for _ in range(2)]

    def parts(t):
        return t[:, :hq * width].view(tokens, hq, width), t[:, hq * width:(hq + hk) * width].view(tokens, hk, width)

    row = (whole.stride(0), width)
    apart = bns.make_qk(tokens, hq, hk, width, dtype, rotated=rotated, eps=EPS, q=row, k=row)
    here = bns.make_qk(tokens, hq, hk, width, dtype, rotated=rotated, eps=EPS, q=row, k=row, q_out=row, k_out=row, dq=row, dk=row)
    want = [torch.empty(tokens, h, width, dtype=TYPES[dtype], device="cuda") for h in (hq, hk)]
    bns.bns_qk_forward(apart, *parts(whole), *weights, positions, f, *want)
    changed = whole.clone()
    bns.bns_qk_forward(here, *parts(changed), *weights, positions, f, *parts(changed))
    for a, b in zip(parts(changed), want):
        assert torch.equal(a, b)
    assert torch.equal(changed[:, (hq + hk) * width:], whole[:, (hq + hk) * width:])
    dy = torch.randn(whole.shape, generator=g).to(TYPES[dtype]).cuda()
    space = torch.empty(bns.bns_qk_workspace_bytes(here), dtype=torch.uint8, device="cuda")
    dense = bns.make_qk(tokens, hq, hk, width, dtype, rotated=rotated, eps=EPS, q=row, k=row, q_out=row, k_out=row)
    dw = [torch.empty(width, device="cuda") for _ in range(4)]
    bns.bns_qk_backward(dense, *parts(whole), *weights, positions, f, *parts(dy), *want, dw[0], dw[1], space)
    changed = dy.clone()
    bns.bns_qk_backward(here, *parts(whole), *weights, positions, f, *parts(changed), *parts(changed), dw[2], dw[3], space)
    for a, b in zip(parts(changed), want):
        assert torch.equal(a, b)
    assert torch.equal(changed[:, (hq + hk) * width:], dy[:, (hq + hk) * width:]) and torch.equal(dw[0], dw[2]) and torch.equal(dw[1], dw[3])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_values_stay_in_their_heads(dtype):
    """A head of zeros, one with NaN, one with infinity, one whose squares overflow, and clean ones beside them (dweight: NaN where theirs are)."""
    tokens, hq, width = 2, 8, 64
    print(f"[gpu-case] qk special values {dtype}", flush=True)
    x, weight, positions, dy = make(tokens, hq, width, dtype, 3, 100)
    f = frequencies(width)
    x[0, 0], x[0, 1, 5], x[0, 2, 6], x[0, 3, 7] = 0, float("nan"), float("inf"), 1e30
    spec = bns.make_qk(tokens, hq, 0, width, dtype, eps=EPS)
    out, dx, dw = torch.empty_like(x, device="cuda"), torch.empty_like(x, device="cuda"), torch.empty(width, device="cuda")
    space = torch.empty(bns.bns_qk_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
    args = (x.cuda(), None, weight.cuda(), None, positions.cuda(), f.cuda())
    bns.bns_qk_forward(spec, *args, out, None)
    bns.bns_qk_backward(spec, *args, dy.cuda(), None, dx, None, dw, None, space)
    assert bool((out[0, 0] == 0).all()) and bool(out[0, 1].isnan().all()) and bool((out[0, 3] == 0).all())
    assert bool(torch.isfinite(dx[0, 0]).all()) and bool(dx[0, 1].isnan().all())
    clean = torch.ones(tokens, hq, dtype=torch.bool)
    clean[0, 1:4] = False
    for t in range(tokens):
        rows = clean[t]
        part = slice(t, t + 1)
        assert_forward(out[part][:, rows], x[part][:, rows], weight, positions[part], f, width, False, dtype)
        want = ref.qk_backward(x[part][:, rows].double(), weight.double(), positions[part], f, dy[part][:, rows].double(), width, False, EPS)[0]
        got = dx[part][:, rows].double().cpu()
        assert bool(((got - want).abs() <= (HALF_ULP[dtype] + 200 * U) * want.abs().amax(-1, keepdim=True) + 1e-37).all())


def test_far_positions_turn_exactly():
    """A rotation by 2^31 - 1 against the angle in 64 bits: what is left of it is rounded to fp32 only after it was reduced."""
    width, tokens = 64, 8
    print("[gpu-case] qk far positions", flush=True)
    positions = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 10 ** 9 + 7, 123456789, 2 ** 24 + 1, -5, 0])
    f = frequencies(width)
    x, _, _, _ = make(tokens, 2, width, "f32", 1, 10)
    out = torch.empty(tokens, 2, width, device="cuda")
    bns.bns_qk_forward(bns.make_qk(tokens, 2, 0, width, "f32"), x.cuda(), None, None, None, positions.cuda(), f.cuda(), out, None)
    for t in range(tokens):
        part = slice(t, t + 1)
        assert_forward(out[part], x[part], None, positions[part], f, width, False, "f32")
    assert torch.equal(out[-1].cpu(), x[-1])


def test_far_positions_turn_as_exactly_as_near_ones():
    """cos and sin alone, (1, 0) turned, against angles that are reduced as fractions with 70 digits of pi: C = 5 u of the docstring, without a part that grows with the position."""
    print("[gpu-case] qk angles of far positions", flush=True)
    pi = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")
    positions = [2 ** 31, -2 ** 31, 2 ** 31 - 1, 2 ** 30 + 1, 10 ** 9 + 7, 2 ** 24 + 1, 12345, 1, -1, 0]
    g = torch.Generator().manual_seed(11)
    f = torch.cat([0.5 + 2.5 * torch.rand(128, generator=g, dtype=torch.float64), 10000.0 ** (-torch.arange(120, dtype=torch.float64) / 120),
                   2.0 ** 16 * torch.rand(8, generator=g, dtype=torch.float64)])
    want = torch.empty(len(positions), 2, len(f), dtype=torch.float64)
    for t, position in enumerate(positions):
        for i, frequency in enumerate(f.tolist()):
            angle = position * Fraction(frequency)
            left = float(angle - round(angle / (2 * pi)) * 2 * pi)
            want[t, 0, i], want[t, 1, i] = math.cos(left), math.sin(left)
    x = torch.zeros(len(positions), 1, 512)
    x[:, :, :256] = 1
    out = torch.empty_like(x, device="cuda")
    bns.bns_qk_forward(bns.make_qk(len(positions), 1, 0, 512, "f32"), x.cuda(), None, None, None, torch.tensor(positions).cuda(), f.cuda(), out, None)
    worst = (out.double().cpu().reshape(want.shape) - want).abs().amax((1, 2)) / U
    assert bool((worst <= 5).all()), worst


def test_gradients_against_differences():
    """The change of sum(c * y) along directions of x and weight, central difference with step 2^-6 in fp32: third order h^2 / 6 = 4e-5, rounding 1e-6 / h = 6e-5."""
    tokens, heads, width, h = 12, 3, 48, 2.0 ** -6
    print("[gpu-case] qk gradients against differences", flush=True)
    x, weight, positions, c = make(tokens, heads, width, "f32", 5, 3000)
    x = x / x.abs().amax(-1, keepdim=True)
    f = frequencies(32)
    spec = bns.make_qk(tokens, heads, 0, width, "f32", rotated=32, eps=EPS)
    g = torch.Generator().manual_seed(9)
    ex, ew = torch.randn(x.shape, generator=g), torch.randn(weight.shape, generator=g)
    out = torch.empty(x.shape, device="cuda")

    def value(step):
        bns.bns_qk_forward(spec, (x + step * 0.1 * ex).cuda(), None, (weight + step * ew).cuda(), None, positions.cuda(), f.cuda(), out, None)
        return float((out.double().cpu() * c.double()).sum())

    measured = (value(h) - value(-h)) / (2 * h)
    dx, dw = torch.empty(x.shape, device="cuda"), torch.empty(width, device="cuda")
    space = torch.empty(bns.bns_qk_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
    bns.bns_qk_backward(spec, x.cuda(), None, weight.cuda(), None, positions.cuda(), f.cuda(), c.cuda(), None, dx, None, dw, None, space)
    slope = float((dx.double().cpu() * 0.1 * ex.double()).sum() + (dw.double().cpu() * ew.double()).sum())
    size = float(dx.norm()) * 0.1 * float(ex.norm()) / x.numel() ** 0.5 + float(dw.norm()) * float(ew.norm()) / width ** 0.5
    assert abs(slope - measured) < 2e-3 * size


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_tokens_are_the_same_bits_again_and_as_few(dtype):
    """More tokens than a launch has waves; twice the same bits; a head's result does not depend on what is beside it."""
    tokens, hq, hk, width = 20000, 4, 2, 64
    print(f"[gpu-case] qk many tokens {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, dq_out, dk_out = (torch.randn(tokens, h, width, generator=g, device="cuda").to(TYPES[dtype]) for h in (hq, hk, hq, hk))
    w = [1 + 0.1 * torch.randn(width, generator=g, device="cuda") for _ in range(2)]
    positions, f = torch.arange(tokens, device="cuda"), frequencies(width).cuda()
    spec = bns.make_qk(tokens, hq, hk, width, dtype, eps=EPS)
    space = torch.empty(bns.bns_qk_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
    runs = []
    for _ in range(2):
        out = [torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k), torch.empty(width, device="cuda"), torch.empty(width, device="cuda")]
        bns.bns_qk_forward(spec, q, k, *w, positions, f, out[0], out[1])
        bns.bns_qk_backward(spec, q, k, *w, positions, f, dq_out, dk_out, *out[2:], space)
        runs.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    few = slice(19990, 20000)
    small = [torch.empty_like(q[few]), torch.empty_like(k[few]), torch.empty_like(q[few]), torch.empty_like(k[few])]
    part = bns.make_qk(10, hq, hk, width, dtype, eps=EPS)
    bns.bns_qk_forward(part, q[few], k[few], *w, positions[few].contiguous(), f, small[0], small[1])
    assert torch.equal(small[0], runs[0][0][few]) and torch.equal(small[1], runs[0][1][few])
    x, dy = q.double().cpu(), dq_out.double().cpu()
    _, dw, gg, r = ref.qk_backward(x, w[0].double().cpu(), positions.cpu(), f.cpu(), dy, width, False, EPS)
    # (tokens x heads terms: some 40 in turn in a lane, then 32, 32 and 32)
    terms = (gg * x * r).abs().sum((0, 1))
    assert bool(((runs[0][4].double().cpu() - dw).abs() <= (17 + 8 + 400) * U * terms).all())
