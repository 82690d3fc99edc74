"""Language-model operators on the GPU in calls that move more than the memory-side cache holds, which have kernels of their own (non-temporal accesses), in calls with more
rows than a launch has blocks, and beyond 2^31 elements.  Rows are independent, so a large call has to leave the bits that calls on some of its rows leave, which are
small enough for the kernels that the other tests hold to 64 bits, and which begin at addresses of their own."""
import pytest
import torch

from lm_reference import TYPES
from paper_1810_10962_amd import bns

pytestmark = pytest.mark.gpu
CACHE = 224 << 20
CHUNK = 1104        # rows of a small call: enough for the plans of many rows, a multiple of 16 so that every base is aligned


def filled(rows, width, stride, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty(rows * stride, dtype=TYPES[dtype], device="cuda")
    for at in range(0, t.numel(), 1 << 28):
        t[at:at + (1 << 28)].normal_(0.0, std, generator=g)
    return t.as_strided((rows, width), (stride, 1))


def blank(rows, width, stride, dtype):
    return torch.zeros(rows * stride, dtype=dtype, device="cuda").as_strided((rows, width), (stride, 1))


def same(a, b):
    whole = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    assert bool(a[:64].view(whole).any()) and bool(a[-64:].view(whole).any()), "nothing was written"
    return all(torch.equal(x.view(whole), y.view(whole)) for x, y in zip(a.split(1 << 16), b.split(1 << 16)))


# One width for each plan of many rows.
FORWARD_WIDTHS = [512, 1000, 2048, 4096, 5120, 8192, 16384]
BACKWARD_WIDTHS = [512, 1000, 2048, 4096, 8192, 16384]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", FORWARD_WIDTHS)
@pytest.mark.parametrize("out,group", [("same", 0), ("e4m3", 0), ("e4m3", 32), ("e4m3", 128)])
def test_norm_beyond_the_cache(out, group, width, dtype):
    e, ye = TYPES[dtype].itemsize, 1 if out == "e4m3" else TYPES[dtype].itemsize
    row = width * (3 * e + ye)
    chunk = CHUNK if CHUNK * row <= CACHE else CHUNK // 2           # (so long a row has one plan for any number of them)
    rows = (CACHE // row // CHUNK + 1) * CHUNK
    assert chunk * row <= CACHE < rows * row
    pad, groups = (3 if group == 32 else 0), -(-width // group) if group else 1
    stride = width + pad
    print(f"[gpu-case] rms beyond the cache {rows}x{width} {dtype} {out} {group}", flush=True)
    x, r, w = filled(rows, width, stride, dtype, 1), filled(rows, width, stride, dtype, 2), 1 + 0.1 * filled(1, width, width, "f32", 3)[0]

    def call(at, count, x, r, s):
        y = blank(count, width, stride, torch.float8_e4m3fn if out == "e4m3" else TYPES[dtype])
        scales, rstd = torch.zeros(count, groups, device="cuda") if out == "e4m3" else None, torch.zeros(count, device="cuda")
        spec = bns.make_rms(count, width, dtype, out=out, group=group, pow2_scales=group == 32, x_stride=stride, residual_stride=stride, sum_stride=stride, y_stride=stride)
        bns.bns_rms_forward(spec, x[at:], r[at:], w, s[at:], y, scales, rstd)
        return y, scales, rstd

    total, place = blank(rows, width, stride, TYPES[dtype]), r.clone() if pad == 0 else None
    y, scales, rstd = call(0, rows, x, r, total)
    if place is not None:
        assert same(call(0, rows, x, place, place)[0], y) and same(place, total)
    part = blank(rows, width, stride, TYPES[dtype])
    for at in range(0, rows, chunk):
        py, pscales, prstd = call(at, chunk, x, r, part)
        assert same(py, y[at:at + chunk]) and torch.equal(prstd, rstd[at:at + chunk]), at
        assert scales is None or torch.equal(pscales, scales[at:at + chunk]), at
    assert same(part, total)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", BACKWARD_WIDTHS)
def test_norm_backward_beyond_the_cache(width, dtype):
    e = TYPES[dtype].itemsize
    rows = (CACHE // (width * 4 * e) // CHUNK + 1) * CHUNK
    chunk = CHUNK // (2 if CHUNK * width * 4 * e > CACHE else 1)
    pad = 5 if width % 512 else 0
    stride = width + pad
    print(f"[gpu-case] rms backward beyond the cache {rows}x{width} {dtype}", flush=True)
    x, dy, ds = (filled(rows, width, stride, dtype, s) for s in (1, 2, 3))
    w, rstd = 1 + 0.1 * filled(1, width, width, "f32", 4)[0], filled(1, rows, rows, "f32", 5)[0].exp()

    def call(at, count, dx):
        spec = bns.make_rms(count, width, dtype, x_stride=stride, residual_stride=stride, sum_stride=stride, y_stride=stride)
        ws, dw = torch.empty(bns.bns_rms_workspace_bytes(spec), dtype=torch.uint8, device="cuda"), torch.zeros(width, device="cuda")
        bns.bns_rms_backward(spec, x[at:], w, rstd[at:], dy[at:], ds[at:], dx, dw, ws)
        return dw

    dx, size = blank(rows, width, stride, TYPES[dtype]), torch.zeros(width, dtype=torch.float64, device="cuda")
    dw, parts = call(0, rows, dx), torch.zeros(width, dtype=torch.float64, device="cuda")
    for at in range(0, rows, chunk):
        part = blank(chunk, width, stride, TYPES[dtype])
        parts += call(at, chunk, part).double()
        size += (dy[at:at + chunk].double() * x[at:at + chunk].double() * rstd[at:at + chunk, None].double()).abs().sum(0)
        assert same(part, dx[at:at + chunk]), at
    # both sides add in fp32: at most rows / 512 + 1 terms in turn, then 32 + 16 partial sums
    assert bool(((dw.double() - parts).abs() <= 2 * (rows / 512 + 60) * 2.0 ** -24 * size).all())


def entries(tokens, vocab, k, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(-1, vocab, (tokens, k), generator=g, device="cuda")
    if k > 1:
        ids[:, k - 1] = ids[:, 0]                            # (an id comes twice)
    return ids, torch.randn(tokens, k, generator=g, device="cuda"), torch.rand(tokens, generator=g, device="cuda") + 0.5


# Logits of bf16, one vocabulary for each number of registers that hold a row, the last two beyond them; half of it in fp32.
VOCABULARIES = [5, 4001, 8000, 16001, 32003, 65000, 98001, 131072, 140001, 262151]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", VOCABULARIES)
def test_distillation_beyond_the_cache(vocab, dtype):
    e, tau, k = TYPES[dtype].itemsize, 2.0, 3 if vocab == 5 else 70
    if dtype == "f32" and vocab > 5:
        vocab = vocab // 2 + vocab % 2
    stride = vocab + (vocab % 2) * 2
    few = 16 if vocab > 100 else 1 << 16
    tokens = (CACHE // (vocab * 2 * e) // few + 2) * few
    print(f"[gpu-case] distill beyond the cache {tokens}x{vocab} {dtype}", flush=True)
    z = filled(tokens, vocab, stride, dtype, 1, std=2.0)
    ids, teacher, dloss = entries(tokens, vocab, k, 2)

    def call(at, count, out, back):
        loss, lse = torch.zeros(count, device="cuda"), torch.zeros(count, device="cuda")
        spec = bns.make_distill(count, vocab, k, dtype, temperature=tau, logits_stride=stride, dlogits_stride=stride)
        bns.bns_distill_forward(spec, z[at:], ids[at:], teacher[at:], dloss[at:], loss, lse, out)
        bns.bns_distill_backward(spec, z[at:], ids[at:], teacher[at:], lse, dloss[at:], back)
        return loss, lse

    out, back = blank(tokens, vocab, stride, TYPES[dtype]), blank(tokens, vocab, stride, TYPES[dtype])
    loss, lse = call(0, tokens, out, back)
    chunk = max(few, CACHE // 8 // (vocab * 2 * e) // few * few)
    assert chunk * vocab * 2 * e <= CACHE
    for at in range(0, tokens, chunk):
        count = min(chunk, tokens - at)
        pout, pback = blank(count, vocab, stride, TYPES[dtype]), blank(count, vocab, stride, TYPES[dtype])
        ploss, plse = call(at, count, pout, pback)
        assert torch.equal(ploss, loss[at:at + count]) and torch.equal(plse, lse[at:at + count]), at
        assert same(pout, out[at:at + count]) and same(pback, back[at:at + count]), at
    place = torch.empty_strided((tokens, vocab), (stride, 1), dtype=TYPES[dtype], device="cuda")
    spec = bns.make_distill(tokens, vocab, k, dtype, temperature=tau, logits_stride=stride, dlogits_stride=stride)
    for want in (out, back):
        place.copy_(z)
        if want is out:
            bns.bns_distill_forward(spec, place, ids, teacher, dloss, loss, lse, place)
        else:
            bns.bns_distill_backward(spec, place, ids, teacher, lse, dloss, place)
        assert same(place, want)


def test_norm_of_more_rows_than_a_launch_has_blocks():
    """A wave per row: 4 x 2^20 rows at a time, so that the rest takes a second turn."""
    rows, width, at = (1 << 22) + 5008, 40, (1 << 22) - 1024
    print(f"[gpu-case] rms {rows}x{width}", flush=True)
    for dtype, out in (("bf16", "same"), ("f32", "e4m3")):
        x, w = filled(rows, width, width, dtype, 1), 1 + 0.1 * filled(1, width, width, "f32", 3)[0]
        got = []
        for first, count in ((0, rows), (at, rows - at)):
            y = torch.zeros(count, width, dtype=torch.float8_e4m3fn if out == "e4m3" else TYPES[dtype], device="cuda")
            scales = torch.zeros(count, 2, device="cuda") if out == "e4m3" else None
            bns.bns_rms_forward(bns.make_rms(count, width, dtype, out=out, group=32 if scales is not None else 0), x[first:], None, w, None, y, scales, None)
            got.append((y, scales))
        (y, scales), (py, pscales) = got
        assert same(y[at:], py) and (scales is None or torch.equal(scales[at:], pscales))


@pytest.mark.parametrize("out", ["same", "e4m3"])
def test_norm_beyond_31_bits(out):
    """More elements than 2^31 and, with a block per row, more rows than a launch has blocks."""
    rows, width = (1 << 20) + 40 * CHUNK, 2056
    print(f"[gpu-case] rms {rows}x{width} {out}", flush=True)
    x, w = filled(rows, width, width, "bf16", 1), 1 + 0.1 * filled(1, width, width, "f32", 3)[0]

    def call(at, count):
        y = torch.zeros(count, width, dtype=torch.float8_e4m3fn if out == "e4m3" else torch.bfloat16, device="cuda")
        scales = torch.zeros(count, -(-width // 64), device="cuda") if out == "e4m3" else None
        bns.bns_rms_forward(bns.make_rms(count, width, "bf16", out=out, group=64 if scales is not None else 0), x[at:], None, w, None, y, scales, None)
        return y, scales

    y, scales = call(0, rows)
    for at in (0, (1 << 20) - 1024, rows - 16 * CHUNK):
        py, pscales = call(at, 16 * CHUNK)
        assert same(py, y[at:at + 16 * CHUNK]) and (scales is None or torch.equal(pscales, scales[at:at + 16 * CHUNK])), at
    if out == "same":
        dx, dw, rstd = torch.zeros_like(x), torch.zeros(width, device="cuda"), torch.full((rows,), 0.7, device="cuda")
        for at, count, to in ((0, rows, dx), (rows - CHUNK, CHUNK, torch.zeros(CHUNK, width, dtype=torch.bfloat16, device="cuda"))):
            spec = bns.make_rms(count, width, "bf16")
            ws = torch.empty(bns.bns_rms_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
            bns.bns_rms_backward(spec, x[at:], w, rstd[at:], y[at:], None, to, dw, ws)
        assert same(to, dx[rows - CHUNK:])


def test_distillation_beyond_31_bits():
    tokens, vocab, k = (1 << 20) + 4096, 2100, 3
    print(f"[gpu-case] distill {tokens}x{vocab}", flush=True)
    z = filled(tokens, vocab, vocab, "bf16", 1)
    ids, teacher, dloss = entries(tokens, vocab, k, 2)
    got = []
    for at, count in ((0, tokens), (tokens - 8192, 8192)):
        spec = bns.make_distill(count, vocab, k, "bf16")
        loss, lse, out, back = torch.zeros(count, device="cuda"), torch.zeros(count, device="cuda"), torch.zeros_like(z[at:]), torch.zeros_like(z[at:])
        bns.bns_distill_forward(spec, z[at:], ids[at:], teacher[at:], dloss[at:], loss, lse, out)
        bns.bns_distill_backward(spec, z[at:], ids[at:], teacher[at:], lse, dloss[at:], back)
        got.append((loss[-8192:], lse[-8192:], out[-8192:], back[-8192:]))
    assert all(same(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("tokens,vocab,hidden_stride,weight_stride", [(16, 270000, 64, 8192), (300, 270000, 64, 8192), (300000, 270, 8192, 64)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_loss_over_the_vocabulary_with_strides_beyond_31_bits(tokens, vocab, hidden_stride, weight_stride, dtype):
    """The same bits as from dense matrices."""
    width = 64
    print(f"[gpu-case] head {tokens}x{width}x{vocab} {dtype} strides {hidden_stride} {weight_stride}", flush=True)
    hidden, weight = filled(tokens, width, width, dtype, 1), filled(vocab, width, width, dtype, 2, std=0.2)
    targets, dloss = torch.randint(0, vocab, (tokens,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)), torch.ones(tokens, device="cuda")
    got = []
    for hs, wst in ((width, width), (hidden_stride, weight_stride)):
        h, w = (torch.empty(n * s, dtype=TYPES[dtype], device="cuda").as_strided((n, width), (s, 1)) for n, s in ((tokens, hs), (vocab, wst)))
        h.copy_(hidden), w.copy_(weight)
        spec = bns.make_head(tokens, width, vocab, dtype, hidden_stride=hs, weight_stride=wst)
        ws = torch.empty(bns.bns_head_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
        loss, lse, dh, dw = torch.zeros(tokens, device="cuda"), torch.zeros(tokens, device="cuda"), torch.zeros_like(hidden), torch.zeros_like(weight)
        bns.bns_head_forward(spec, h, w, targets, loss, lse, ws)
        bns.bns_head_backward(spec, h, w, targets, lse, dloss, dh, dw, ws)
        got.append((loss[:, None], lse[:, None], dh, dw))
    assert all(same(a, b) for a, b in zip(*got)) and bool(torch.isfinite(got[0][0]).all())


def test_gradients_of_the_vocabulary_beyond_31_bits():
    """A gradient of more than 2^31 elements: its ends against the product of g, in fp32 from the call's own lse, with the hidden states.  g is rounded to bf16
    (2^-8) and so is the result."""
    tokens, width, vocab = 8, 2048, 1100000
    print(f"[gpu-case] head {tokens}x{width}x{vocab}", flush=True)
    hidden, weight = filled(tokens, width, width, "bf16", 1), filled(vocab, width, width, "bf16", 2, std=0.05)
    targets, dloss = torch.arange(tokens, device="cuda") * (vocab // tokens) + vocab // tokens - 1, torch.full((tokens,), 1000.0, device="cuda")
    spec = bns.make_head(tokens, width, vocab, "bf16")
    ws = torch.empty(bns.bns_head_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
    loss, lse, dh, dw = torch.zeros(tokens, device="cuda"), torch.zeros(tokens, device="cuda"), torch.zeros_like(hidden), torch.zeros_like(weight)
    bns.bns_head_forward(spec, hidden, weight, targets, loss, lse, ws)
    bns.bns_head_backward(spec, hidden, weight, targets, lse, dloss, dh, dw, ws)
    z = torch.cat([hidden.float() @ w.float().T for w in weight.split(1 << 16)], 1)
    assert bool(((torch.logsumexp(z, 1) - lse).abs() <= 1e-4).all())
    g = torch.exp(z - lse[:, None])
    g[torch.arange(tokens, device="cuda"), targets] -= 1
    g *= dloss[:, None]
    for rows in (slice(0, 1000), slice((1 << 31) // width - 500, (1 << 31) // width + 500), slice(vocab - 1000, vocab)):
        want, size = g[:, rows].T @ hidden.float(), g[:, rows].abs().T @ hidden.float().abs()
        assert bool(((dw[rows].float() - want).abs() <= 2.0 ** -8 * (want.abs() + size) * 1.01 + 1e-3 * size).all())
