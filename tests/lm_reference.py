"""The last layers of a language model in 64 bits, from their definitions (include/bns.h), on the CPU, and what the tests need around the calls:
rows with strides, guards around what is written."""
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# Half a unit in the last place, relative: what one rounding to the type may cost.
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
GUARD = 4096


def rms_forward(x, residual, weight, eps):
    s = x if residual is None else x + residual
    rstd = 1.0 / torch.sqrt(s.pow(2).mean(1) + eps)
    return s, rstd, weight * s * rstd[:, None]


def rms_backward(x, weight, rstd, dy, dsum):
    xh = x * rstd[:, None]
    g = weight * dy
    dx = rstd[:, None] * (g - xh * (g * xh).mean(1, keepdim=True))
    return dx if dsum is None else dx + dsum, (dy * xh).sum(0)


def head(hidden, weight, targets, dloss):
    """loss, lse, p, g, dhidden, dweight; tokens that are left out count as zeros whatever they hold."""
    kept = (targets >= 0) & (targets < weight.shape[0])
    z = hidden @ weight.T
    lse = torch.logsumexp(z, 1)
    at = z.gather(1, torch.where(kept, targets, 0)[:, None])[:, 0]
    loss = torch.where(kept, lse - at, torch.zeros_like(lse))
    p = torch.exp(z - lse[:, None])
    one = torch.zeros_like(p)
    one[torch.arange(len(targets))[kept], targets[kept]] = 1.0
    g = torch.where(kept[:, None], dloss[:, None] * (p - one), torch.zeros_like(p))
    return loss, lse, p, g, g @ weight, g.T @ torch.where(kept[:, None], hidden, torch.zeros_like(hidden))


def distill(logits, ids, teacher, tau, dloss):
    """loss, lse, dlogits."""
    tokens, vocab = logits.shape
    z = logits / tau
    lse = torch.logsumexp(z, 1)
    loss, dz = torch.zeros(tokens, dtype=torch.float64), torch.zeros_like(z)
    for t in range(tokens):
        keep = (ids[t] >= 0) & (ids[t] < vocab) & ~(teacher[t] == -torch.inf)
        if not bool(keep.any()):
            continue
        j = ids[t][keep]
        logq = torch.log_softmax(teacher[t][keep] / tau, 0)
        q = logq.exp()
        loss[t] = tau * tau * torch.where(q > 0, q * (logq - (z[t, j] - lse[t])), torch.zeros_like(q)).sum()
        dz[t] = torch.exp(z[t] - lse[t]) * tau * dloss[t]
        dz[t].index_add_(0, j, -q * tau * dloss[t])
    return loss, lse, dz


class Rows:
    """A matrix on the GPU whose rows lie `stride` elements apart, between guards: NaN (a read outside would show) or, for an output, a pattern
    that `check` looks for, also between the rows."""

    def __init__(self, values, stride=0, dtype=None, written=False):
        rows, width = values.shape
        self.stride, self.width, self.rows = stride or width, width, rows
        dtype = dtype or values.dtype
        self.fill = 1.5 if written else float("nan")
        whole = torch.full((2 * GUARD + (rows * self.stride + 15) // 16 * 16,), self.fill, dtype=torch.float32).to(dtype).cuda()
        self.whole = whole
        self.t = whole[GUARD:].as_strided((rows, width), (self.stride, 1))
        if dtype.itemsize == 1:
            whole.view(torch.uint8)[GUARD:].as_strided((rows, width), (self.stride, 1)).copy_(torch.zeros(rows, width, dtype=torch.uint8))
        else:
            self.t.copy_(values.to(dtype))
        self.before = whole.clone()

    def __getattr__(self, name):            # data_ptr, nbytes, get_device, device: those of the matrix
        return getattr(self.t, name)

    def check(self):
        now, before = self.whole.clone(), self.before.clone()
        for w in (now, before):
            v = w.view(torch.uint8) if w.dtype.itemsize == 1 else w
            v[GUARD:].as_strided((self.rows, self.width), (self.stride, 1)).fill_(0)
        assert torch.equal(now.view(torch.uint8), before.view(torch.uint8)), "written outside the rows"
        return self.t


def vector(values, dtype=torch.float32):
    return values.to(dtype).cuda()


def written(n, dtype=torch.float32):
    return Rows(torch.zeros(1, n), dtype=dtype, written=True)
