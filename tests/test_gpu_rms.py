"""Root-mean-square norm on the GPU against its definition in 64 bits (lm_reference).

Tolerances.  The sum of squares of a row has at most 32 terms per thread, which are added in turn, and 10 levels of a tree above them, every one with an error of half
a unit: (32 + 10) 2^-24, half of which reaches 1 / sqrt; two products and the reciprocal root (one unit) follow: below 5e-6 relative.  A
result in 16 bits is rounded once more, 2^-8.  The 8-bit type keeps four significant bits, 2^-4 relative, and 2^-10 of the scale below its
smallest normal number.  dx has two such sums, one of which is taken off: its error is relative to the terms, not to their difference."""
import pytest
import torch

import lm_reference as ref
from lm_reference import HALF_ULP, TYPES, Rows, vector, written
from paper_1810_10962_amd import bns

pytestmark = pytest.mark.gpu
SUM = 5e-6
EPS = 1e-6


def make(rows, width, dtype, seed=0, residual=True):
    g = torch.Generator().manual_seed(seed * 7919 + rows * 31 + width)
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = (rnd(rows, width) * torch.exp(rnd(rows, 1))).to(TYPES[dtype])
    return x, rnd(rows, width).to(TYPES[dtype]) if residual else None, 1 + 0.2 * rnd(width), rnd(rows, width).to(TYPES[dtype]), rnd(rows, width).to(TYPES[dtype])


def near(got, want, relative, absolute=0.0):
    got, want = got.double().cpu(), want.double()
    off = (got - want).abs() - (relative * want.abs() + absolute)
    assert bool((off <= 0).all()), f"worst excess {off.max().item():.3e}, at most {(got - want).abs().max().item():.3e} off"


SHAPES = [(1, 1), (1, 4096), (3, 7), (2, 64), (5, 65), (4, 511), (3, 520), (1500, 96), (1030, 1001), (1100, 2048), (1024, 2056), (2, 8192), (1025, 4099), (1, 16384),
          (3, 8200), (9, 16383)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", SHAPES)
def test_forward(rows, width, dtype):
    for residual, pad, weight_dtype in [(True, 0, "f32"), (False, 3, "bf16"), (True, 5, "bf16")]:
        print(f"[gpu-case] rms forward {rows}x{width} {dtype} residual={residual} pad={pad}", flush=True)
        x, r, w, _, _ = make(rows, width, dtype, residual=residual)
        w = w.to(TYPES[weight_dtype])
        stride = width + pad if pad else 0
        dx, dr = Rows(x, stride), Rows(r, stride + 1 if pad else 0) if residual else None
        s = Rows(torch.zeros(rows, width), stride, TYPES[dtype], written=True) if residual else None
        y = Rows(torch.zeros(rows, width), stride + 2 if pad else 0, TYPES[dtype], written=True)
        rstd = written(rows)
        spec = bns.make_rms(rows, width, dtype, weight_dtype=weight_dtype, eps=EPS, x_stride=stride, residual_stride=dr.stride if dr else 0,
                            sum_stride=stride, y_stride=y.stride)
        bns.bns_rms_forward(spec, dx, dr, w.cuda(), s, y, None, rstd)
        total, want_rstd, want = ref.rms_forward(x.double(), None if r is None else r.double(), w.double(), EPS)
        # the addition itself rounds once in fp32, on top of SUM
        near(rstd.check()[0], want_rstd, SUM)
        near(y.check(), want, SUM + HALF_ULP[dtype], 1e-7 * float((want_rstd[:, None] * w.double()).abs().max()) if residual else 0.0)
        if residual:
            assert torch.equal(s.check().cpu(), (x.float() + r.float()).to(TYPES[dtype]))


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("pow2", [False, True])
@pytest.mark.parametrize("rows,width,dtype", [(1, 4096, "bf16"), (3, 1000, "bf16"), (1100, 160, "f32"), (1030, 1001, "bf16"), (5, 33, "f32"), (2, 8199, "bf16"),
                                              (2, 1, "f32"), (1050, 5120, "bf16")])
def test_forward_in_8_bits(rows, width, dtype, group, pow2):
    print(f"[gpu-case] rms forward e4m3 {rows}x{width} {dtype} group={group} pow2={pow2}", flush=True)
    x, r, w, _, _ = make(rows, width, dtype, seed=1)
    x[0, : min(width, 40)] = 0
    r[0, : min(width, 40)] = 0
    groups = -(-width // group) if group else 1
    y = Rows(torch.zeros(rows, width), width + 5, torch.float8_e4m3fn, written=True)
    scales = Rows(torch.zeros(rows, groups), written=True)
    s = torch.empty(rows, width, dtype=TYPES[dtype], device="cuda")
    spec = bns.make_rms(rows, width, dtype, out="e4m3", group=group, pow2_scales=pow2, eps=EPS, y_stride=width + 5)
    bns.bns_rms_forward(spec, x.cuda(), r.cuda(), w.cuda(), s, y, scales, None)
    _, rstd, v = ref.rms_forward(x.double(), r.double(), w.double(), EPS)
    q, scale = y.check().float().double().cpu(), scales.check().double().cpu()
    wide = torch.nn.functional.pad(v, (0, groups * (group or width) - width)).view(rows, groups, -1)
    most = wide.abs().amax(2).clamp(min=448 * 2.0 ** -126)
    slack = SUM + 2e-7 + 1e-7 * float((rstd[:, None] * w.double()).abs().max() / most.min()) if float(most.min()) > 1e-30 else 1.0
    assert bool((scale >= 2.0 ** -126).all())
    big = most > 1e-30
    if pow2:
        mantissa, _ = torch.frexp(scale)
        assert bool((mantissa == 0.5).all())
        assert bool((most <= 448 * scale * (1 + 1e-5)).all()) and bool((most[big] > 224 * scale[big] * (1 - 1e-5)).all())
    else:
        near(scale[big], most[big] / 448, min(slack, 1e-5))
    each = scale.repeat_interleave(group or width, 1)[:, :width]
    # one rounding to four significant bits (or to the spacing of the smallest numbers), of a value that is SUM off
    bound = torch.maximum(v.abs() * 2.0 ** -4, each * 2.0 ** -10) * (1 + 1e-4) + v.abs() * 1e-5 + 2e-7 * (rstd[:, None] * w.double()).abs()
    assert bool(((q * each - v).abs() <= bound).all())
    assert bool((q.abs() <= 448).all())


def test_forward_in_8_bits_special_values():
    x = torch.zeros(4, 256)
    x[0, 3] = float("nan")
    x[0, 200] = 1.0
    x[2] = torch.randn(256, generator=torch.Generator().manual_seed(1)) * 1e-30
    x[3, 5] = float("inf")
    y, scales = torch.empty(4, 256, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(4, 2, device="cuda")
    spec = bns.make_rms(4, 256, "f32", out="e4m3", group=128, eps=EPS)
    print("[gpu-case] rms forward e4m3 special values", flush=True)
    bns.bns_rms_forward(spec, x.cuda(), None, torch.ones(256, device="cuda"), None, y, scales, None)
    q = y.float().cpu()
    assert bool(torch.isnan(q[0]).all())                     # a NaN reaches the whole row through its norm
    assert bool((q[1] == 0).all()) and bool((scales[1] == 2.0 ** -126).all())
    assert float(q[2].abs().max()) == 448.0                  # values far below 1 use the whole range
    assert bool(torch.isnan(q[3, 5])) and bool((q[3, 6:] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", SHAPES + [(0, 64), (5000, 40), (777, 1001)])
def test_backward(rows, width, dtype):
    for use_dsum, pad in [(True, 0), (False, 3), (True, 7)]:
        print(f"[gpu-case] rms backward {rows}x{width} {dtype} dsum={use_dsum} pad={pad}", flush=True)
        x, _, w, dy, dsum = make(rows, width, dtype, seed=2)
        dsum = dsum if use_dsum else None
        rstd = (1.0 / torch.sqrt(x.double().pow(2).mean(1) + EPS)).float()
        stride = width + pad if pad else 0
        out, dw = Rows(torch.zeros(rows, width), stride, TYPES[dtype], written=True), written(width)
        spec = bns.make_rms(rows, width, dtype, eps=EPS, x_stride=stride, residual_stride=stride + 1 if pad else 0, sum_stride=stride, y_stride=stride)
        ws = torch.empty(bns.bns_rms_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
        bns.bns_rms_backward(spec, Rows(x, stride), w.cuda(), vector(rstd), Rows(dy, stride),
                             Rows(dsum, stride + 1 if pad else 0) if use_dsum else None, out, dw, ws)
        wx, wr, wdy = x.double(), rstd.double(), dy.double()
        want_dx, want_dw = ref.rms_backward(wx, w.double(), wr, wdy, None if dsum is None else dsum.double())
        xh, g = wx * wr[:, None], w.double() * wdy
        terms = wr[:, None] * (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True)) + (0 if dsum is None else dsum.double().abs())
        near(out.check(), want_dx, HALF_ULP[dtype], SUM * terms)
        # dweight: at most rows / 512 + 1 terms in turn, then 32 + 16 partial sums
        near(dw.check()[0], want_dw, 0.0, (rows / 512 + 60) * 2.0 ** -24 * (wdy * xh).abs().sum(0) + 1e-30)


def test_gradient_against_differences():
    """The forward kernel's own change along a direction, central difference with step 2^-7: the error of third order is about h^2 = 6e-5 of the
    gradient's size, the rounding error of the outputs (2^-24 each, independent) some 1e-6 / h."""
    rows, width, h = 40, 640, 2.0 ** -7
    x, r, w, dy, dsum = make(rows, width, "f32", seed=3)
    g = torch.Generator().manual_seed(11)
    d, dwt = torch.randn(rows, width, generator=g), torch.randn(width, generator=g)
    spec = bns.make_rms(rows, width, "f32", eps=EPS)
    dev = "cuda"

    def value(step):
        y, s, rstd = (torch.empty(rows, width, device=dev) for _ in range(2)), None, None
        y, s = y
        rstd = torch.empty(rows, device=dev)
        bns.bns_rms_forward(spec, (x + step * d).to(dev), r.to(dev), (w + step * dwt).to(dev), s, y, None, rstd)
        return float((y.double().cpu() * dy.double()).sum() + (s.double().cpu() * dsum.double()).sum()), s, rstd

    print("[gpu-case] rms gradient against differences", flush=True)
    _, s, rstd = value(0.0)
    dx, dw = torch.empty(rows, width, device=dev), torch.empty(width, device=dev)
    ws = torch.empty(bns.bns_rms_workspace_bytes(spec), dtype=torch.uint8, device=dev)
    bns.bns_rms_backward(spec, s, w.to(dev), rstd, dy.to(dev), dsum.to(dev), dx, dw, ws)
    slope = float((dx.double().cpu() * d.double()).sum() + (dw.double().cpu() * dwt.double()).sum())
    measured = (value(h)[0] - value(-h)[0]) / (2 * h)
    size = float((dx.double().cpu().norm() * d.double().norm()))
    assert abs(slope - measured) < 1e-3 * size


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(dtype):
    rows, width = 70, 1000
    x, r, w, dy, dsum = (t.cuda() for t in make(rows, width, dtype, seed=4))
    spec = bns.make_rms(rows, width, dtype, eps=EPS)
    rstd, y, s = torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    print(f"[gpu-case] rms in place {dtype}", flush=True)
    bns.bns_rms_forward(spec, x, r, w, s, y, None, rstd)
    for place in ("residual", "x"):
        x2, r2, y2 = x.clone(), r.clone(), torch.empty_like(x)
        at = r2 if place == "residual" else x2
        bns.bns_rms_forward(spec, x2, r2, w, at, y2, None, None)
        assert torch.equal(at, s) and torch.equal(y2, y)
    alone, alone2 = torch.empty_like(x), x.clone()
    bns.bns_rms_forward(spec, x, None, w, None, alone, None, None)
    bns.bns_rms_forward(spec, alone2, None, w, None, alone2, None, None)
    assert torch.equal(alone, alone2)
    dx, dw, dw2 = torch.empty_like(x), torch.empty(width, device="cuda"), torch.empty(width, device="cuda")
    ws = torch.empty(bns.bns_rms_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
    bns.bns_rms_backward(spec, s, w, rstd, dy, dsum, dx, dw, ws)
    for place in ("dy", "dsum"):
        dy2, ds2 = dy.clone(), dsum.clone()
        at = dy2 if place == "dy" else ds2
        bns.bns_rms_backward(spec, s, w, rstd, dy2, ds2, at, dw2, ws)
        assert torch.equal(at, dx) and torch.equal(dw2, dw)      # and the same bits from run to run


def test_columns_of_a_wider_matrix_and_another_stream():
    """Two halves of one matrix: x in the left columns, y in the right ones, on a stream of its own."""
    rows, width = 33, 256
    x, _, w, _, _ = make(rows, width, "bf16", residual=False)
    both = torch.zeros(rows, 2 * width, dtype=torch.bfloat16, device="cuda")
    both[:, :width] = x.cuda()
    w = w.cuda()
    spec = bns.make_rms(rows, width, "bf16", eps=EPS, x_stride=2 * width, y_stride=2 * width)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    print("[gpu-case] rms halves of a matrix", flush=True)
    with torch.cuda.stream(stream):
        bns.bns_rms_forward(spec, both, None, w, None, both[:, width:], None, None)
    stream.synchronize()
    want = ref.rms_forward(x.double(), None, w.double().cpu(), EPS)[2]
    near(both[:, width:], want, SUM + HALF_ULP["bf16"])
    assert torch.equal(both[:, :width].cpu(), x)
