"""Loss over the vocabulary on the GPU: logits that are infinite, NaN or as low as the type goes, in tokens that count.  A masked row of the vocabulary holds
-infinity or the type's lowest value in a column that is positive in every token, as a bias does; what it adds to a softmax is nothing, so the definition (lm_reference) is
evaluated without those rows, with the tolerances of test_gpu_head."""
import pytest
import torch

from lm_reference import TYPES
from paper_1810_10962_amd import bns
from test_gpu_head import check_backward, check_forward, make, path, run  # noqa: F401

pytestmark = pytest.mark.gpu
BIAS, MASKED = 7, 40        # the column, and how many of the vocabulary's last rows are masked


def masked(tokens, width, vocab, dtype, value):
    hidden, weight, targets, dloss = make(tokens, width, vocab, dtype, seed=11)
    targets = torch.where((targets >= vocab - MASKED) & (targets < vocab), targets - MASKED, targets)
    weight[:, BIAS] = 0
    # one, which is its own first part, values with three parts of mixed signs, one whose product with the lowest value overflows
    hidden[:, BIAS] = torch.tensor([1.0, 0.1, 1.5, 300.7, 1e-3, 0.7])[torch.arange(tokens) % 6].to(TYPES[dtype])
    weight[vocab - MASKED:, BIAS] = value
    return hidden, weight, targets, dloss


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,width,vocab", [(9, 64, 300), (140, 72, 700), (20, 512, 1100)])
def test_masked_rows_of_the_vocabulary_count_for_nothing(tokens, width, vocab, dtype, path):  # noqa: F811
    for value in (-float("inf"), float(torch.finfo(TYPES[dtype]).min)):
        print(f"[gpu-case] head masked by {value} {tokens}x{width}x{vocab} {dtype} {path}", flush=True)
        hidden, weight, targets, dloss = masked(tokens, width, vocab, dtype, value)
        left = torch.where(targets >= vocab - MASKED, -1, targets)      # (a target outside the smaller vocabulary is one outside the larger)
        loss, lse, dh, dw = run(hidden, weight, targets, dloss, dtype)
        check_forward(loss, lse, hidden, weight[:-MASKED], left, dtype)
        assert bool((dw[-MASKED:] == 0).all())
        clean = weight[:-MASKED]
        if value == -float("inf"):          # zero times infinity: the column's gradient is NaN by the formula
            dh = dh.clone()
            dh[:, BIAS] = 0
        check_backward(dh, dw[:-MASKED], hidden, clean, left, dloss, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens,width,vocab", [(9, 64, 300), (140, 72, 700)])
def test_infinity_and_nan_stay_in_their_token(tokens, width, vocab, dtype, path):  # noqa: F811
    hidden, weight, targets, dloss = masked(tokens, width, vocab, dtype, -float("inf"))
    targets = torch.randint(0, vocab - MASKED, (tokens,), generator=torch.Generator().manual_seed(3))
    hidden[1, BIAS] = -0.3                  # logits of +infinity
    hidden[3, 5] = float("nan")
    hidden[4, BIAS] = 0                     # zero times infinity
    hidden[6, 2] = float("inf")             # logits of both infinities
    targets[7] = vocab - 3                  # a target that is masked
    print(f"[gpu-case] head infinity and NaN {tokens}x{width}x{vocab} {dtype} {path}", flush=True)
    loss, lse, _, _ = run(hidden, weight, targets, dloss, dtype)
    loss, lse = loss.cpu(), lse.cpu()
    for t in (1, 3, 4, 6):
        assert not bool(torch.isfinite(loss[t])) and not bool(torch.isfinite(lse[t])), t
    assert bool(torch.isnan(loss[3])) and bool(torch.isnan(lse[3]))
    assert float(loss[7]) == float("inf") and bool(torch.isfinite(lse[7]))
    rest = torch.tensor([t not in (1, 3, 4, 6, 7) for t in range(tokens)])
    check_forward(loss[rest], lse[rest], hidden[rest], weight[:-MASKED], targets[rest], dtype)
    check_forward(lse[7:8] * 0, lse[7:8], hidden[7:8], weight[:-MASKED], torch.tensor([-1]), dtype)


def test_the_whole_range_of_fp32(path):  # noqa: F811
    """Operands from the largest finite value down, one product a logit, and the other a power of two: every logit is exact, so is the difference of two of them."""
    tokens, width, vocab = 30, 64, 300
    big = torch.tensor([torch.finfo(torch.float32).max, 3.3961775292304957e38, 3.39e38, 3.3895313892515355e38, 1.7e38, 1e30])
    weight, hidden = torch.zeros(vocab, width), torch.zeros(tokens, width)
    weight[torch.arange(tokens), torch.arange(tokens)] = big[torch.arange(tokens) % 6]
    hidden[torch.arange(tokens), torch.arange(tokens)] = 2.0 ** -(121 + torch.arange(tokens).float() % 3)
    weight[vocab - 1], hidden[:, width - 1] = 0, 0
    want = (weight[:tokens].double() * hidden.double()).sum(1)          # every token has one logit that is not zero
    print(f"[gpu-case] head range of fp32 {path}", flush=True)
    spec = bns.make_head(tokens, width, vocab, "f32")
    ws = torch.empty(bns.bns_head_workspace_bytes(spec), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    bns.bns_head_forward(spec, hidden.cuda(), weight.cuda(), torch.full((tokens,), vocab - 1).cuda(), loss, lse, ws)
    top = torch.log(torch.exp(want) + vocab - 1)
    assert bool(((loss.double().cpu() - top).abs() <= 2.0 ** -20 * (1 + top.abs())).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1, 8, 32])
def test_the_loss_of_a_sure_model_is_zero(scale, dtype, path):  # noqa: F811
    """Logits scale (32 + t) on the target, zero and below elsewhere, all exact: what a softmax leaves to the others is below 700 exp(-32) = 1e-11, so the loss is
    neither negative nor more than a unit in the last place of one, and lse is the target's logit."""
    tokens, width, vocab = 64, 64, 700
    weight = torch.zeros(vocab, width)
    weight[torch.arange(vocab), torch.arange(vocab) % width] = float(scale)
    weight[width:] *= -1
    top = 32.0 + torch.arange(tokens)
    hidden, targets = torch.diag(top), torch.arange(tokens)
    print(f"[gpu-case] head sure {scale} {dtype} {path}", flush=True)
    loss, lse, _, _ = run(hidden.to(TYPES[dtype]), weight.to(TYPES[dtype]), targets, torch.ones(tokens), dtype)
    assert bool((loss >= 0).all()) and bool((loss <= 2.0 ** -23).all())
    assert torch.equal(lse.cpu(), scale * top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("base", [0.0, 512.0, -2048.0])
@pytest.mark.parametrize("tokens", [12, 130])
def test_logits_far_from_zero(tokens, base, dtype, path):  # noqa: F811
    """Exact logits, base plus multiples of 1/8 between -4 and 4: the loss does not depend on the base.  Exponents below 12 in powers of two and an exponential's own unit cost
    (12 + 2) 2^-24 of a term, the sums in turn and in a tree 30 2^-24, the logarithm two units of a number below 16: 3e-6 + 2e-6."""
    width, vocab = 64, 700
    g = torch.Generator().manual_seed(17)
    weight, hidden = torch.zeros(vocab, width), torch.zeros(tokens, width)
    weight[:, 0], weight[:, 1], weight[:, 2] = base, torch.randint(-16, 17, (vocab,), generator=g) / 8.0, torch.randint(-16, 17, (vocab,), generator=g) / 8.0
    hidden[:, 0] = 1
    hidden[torch.arange(tokens), 1 + torch.arange(tokens) % 2] = 2.0 - (torch.arange(tokens) % 4).float()
    targets = torch.randint(0, vocab, (tokens,), generator=g)
    print(f"[gpu-case] head base {base} {tokens} {dtype} {path}", flush=True)
    loss, lse, _, _ = run(hidden.to(TYPES[dtype]), weight.to(TYPES[dtype]), targets, torch.ones(tokens), dtype)
    z = hidden.double() @ weight.double().T
    want = torch.logsumexp(z, 1)
    assert bool(((loss.double().cpu() - (want - z[torch.arange(tokens), targets])).abs() <= 5e-6).all())
    assert bool(((lse.double().cpu() - want).abs() <= 5e-6 + 2.0 ** -24 * want.abs()).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [12, 130])
def test_logits_at_the_ends_of_the_range(tokens, dtype, path):  # noqa: F811
    """All logits of a token are the type's lowest value, or its largest: alike, so the loss is log(vocab)."""
    width, vocab = 64, 700
    weight, hidden = torch.zeros(vocab, width), torch.zeros(tokens, width)
    weight[:, 0] = torch.finfo(TYPES[dtype]).max
    hidden[:, 0] = 1.0 - 2 * (torch.arange(tokens) % 2)
    print(f"[gpu-case] head ends of the range {tokens} {dtype} {path}", flush=True)
    loss, lse, _, _ = run(hidden.to(TYPES[dtype]), weight.to(TYPES[dtype]), torch.arange(tokens), torch.ones(tokens), dtype)
    assert bool(((loss.double().cpu() - torch.log(torch.tensor(float(vocab), dtype=torch.float64))).abs() <= 5e-6).all())
    assert torch.equal(lse.cpu(), hidden[:, 0] * torch.finfo(TYPES[dtype]).max)


def three_parts(n, seed):
    """Values in [1, 2) with 24 significant bits, each of whose three parts is needed."""
    return 1 + (torch.randint(0, 2 ** 22, (n,), generator=torch.Generator().manual_seed(seed)) * 2 + 1).float() * 2.0 ** -23


@pytest.mark.parametrize("tokens,width,vocab", [(30, 64, 300), (30, 200, 1500), (140, 192, 700), (250, 256, 3000)])
@pytest.mark.parametrize("which", ["hidden", "weight", "dloss", "middle"])
def test_every_part_of_an_fp32_product_counts(which, tokens, width, vocab, path):  # noqa: F811
    """Token t has one product that is not zero, x_t y_t = 64 to 128, with row 2 t of the vocabulary; its target is row 2 t + 1, whose logit is zero.  What the softmax
    leaves to all other rows is below 3000 exp(-64) = 1e-24, so that loss = lse = x_t y_t, g = dloss and -dloss, and every result is a single product, which is exact in
    fp32 where one factor is a power of two, or where both are 1 + 2^-9 times one (whose product of second parts is 2^-18 of the whole).  A pair of parts that is left out or
    taken twice changes bits."""
    t = torch.arange(tokens)
    x, y, d = torch.full((tokens,), 8.0), torch.full((tokens,), 8.0), torch.full((tokens,), 0.25)
    if which == "hidden":
        x = x * three_parts(tokens, 1)
    elif which == "weight":
        y = y * three_parts(tokens, 2)
    elif which == "dloss":
        d = d * three_parts(tokens, 3)
    else:
        x, y, d = (v * (1 + 2.0 ** -9) for v in (x, y, d))
    hidden, weight = torch.zeros(tokens, width), torch.zeros(vocab, width)
    hidden[t, t], weight[2 * t, t] = x, y
    print(f"[gpu-case] head parts {which} {tokens}x{width}x{vocab} {path}", flush=True)
    loss, lse, dh, dw = (o.cpu() for o in run(hidden, weight, 2 * t + 1, d, "f32"))
    assert torch.equal(loss, x * y) and torch.equal(lse, x * y)
    assert torch.equal(dh[t, t], d * y)
    assert torch.equal(dw[2 * t, t], d * x) and torch.equal(dw[2 * t + 1, t], -d * x)
