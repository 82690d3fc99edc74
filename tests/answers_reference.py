"""A step on a language model's own answers in 64 bits, from its definitions (include/bns.h), on the CPU, and tensors of any layout between guards."""
import math

import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U = 2.0 ** -24
GUARD = 1003                # elements; odd, so that what lies behind begins at an element's alignment only


def turns(positions, frequencies):
    w = positions.double()[:, None] * frequencies
    return torch.cos(w)[:, None], torch.sin(w)[:, None]


def rotate(v, cos, sin, rotated, interleaved):
    out = v.clone()
    a, b = (slice(0, rotated, 2), slice(1, rotated, 2)) if interleaved else (slice(0, rotated // 2), slice(rotated // 2, rotated))
    out[..., a], out[..., b] = v[..., a] * cos - v[..., b] * sin, v[..., a] * sin + v[..., b] * cos
    return out


def beside(v, rotated, interleaved):
    """|v_a| + |v_b| of the pair of every element (|v| where nothing is rotated): what an error of the rotation is relative to."""
    out = v.abs()
    a, b = (slice(0, rotated, 2), slice(1, rotated, 2)) if interleaved else (slice(0, rotated // 2), slice(rotated // 2, rotated))
    out[..., a] = out[..., b] = v[..., a].abs() + v[..., b].abs()
    return out


def qk_forward(x, weight, positions, frequencies, rotated, interleaved, eps):
    """y, v."""
    v = x if weight is None else weight * x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps)
    return rotate(v, *turns(positions, frequencies), rotated, interleaved), v


def qk_backward(x, weight, positions, frequencies, dy, rotated, interleaved, eps):
    """dx, dweight, g, r."""
    cos, sin = turns(positions, frequencies)
    g = rotate(dy, cos, -sin, rotated, interleaved)
    if weight is None:
        return g, None, g, None
    r = 1 / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps)
    xh, wg = x * r, weight * g
    return r * (wg - xh * (wg * xh).mean(-1, keepdim=True)), (g * xh).sum((0, 1)), g, r


def logprob(logits, targets, tau):
    """largest, s, log p, logp, entropy; rows of -infinity as include/bns.h has them."""
    m = logits.amax(1)
    empty = m == -math.inf
    z = torch.where(empty[:, None], -math.inf, (logits - m[:, None]) / tau)
    s = torch.where(empty, 0.0, torch.log(torch.exp(z).sum(1)))
    logp = z - s[:, None]
    p = torch.exp(logp)
    entropy = -torch.where(p == 0, 0.0, p * logp).sum(1)
    kept = (targets >= 0) & (targets < logits.shape[1])
    given = torch.where(kept, logp.gather(1, torch.where(kept, targets, 0)[:, None])[:, 0], 0.0)
    return m, s, logp, given, entropy


def top(logits, k):
    """Indices of the k largest in falling order, the lowest first among equals; NaN as -infinity."""
    x = torch.where(logits.isnan(), -math.inf, logits)
    return torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]


def logprob_backward(logits, targets, stats, entropy, dlogp, dentropy, tau):
    """dlogits, log p, p; from the stats as they are given."""
    logp = (logits - stats[:, :1]) / tau - stats[:, 1:]
    p = torch.exp(logp)
    kept = (targets >= 0) & (targets < logits.shape[1])
    g = torch.where(kept, dlogp, 0.0)[:, None]
    dz = torch.where(p == 0, 0.0, -p * (g + dentropy[:, None] * (logp + entropy[:, None])))
    dz.scatter_add_(1, torch.where(kept, targets, 0)[:, None], g)
    none = ((g[:, 0] == 0) & (dentropy == 0)) | (stats[:, 0] == -math.inf)
    return torch.where(none[:, None], 0.0, dz) / tau, logp, p


class Strided:
    """A tensor [a][b][width] of given strides on the GPU, GUARD elements inside a buffer of NaN (a read outside would show) or, for an output, of a pattern that
    `check` looks for wherever the tensor has no element."""

    def __init__(self, values, strides=None, written=False):
        shape = tuple(values.shape)
        strides = tuple(strides or values.contiguous().stride())
        reach = 1 + sum((n - 1) * s for n, s in zip(shape, strides)) if values.numel() else 0
        self.fill = 1.5 if written else float("nan")
        self.whole = torch.full((2 * GUARD + reach,), self.fill, dtype=values.dtype, device="cuda")
        self.at = self.whole[GUARD:]
        self.shape, self.strides = shape, strides
        self.t = self.view(self.whole)
        if values.numel():
            self.t.copy_(values)
        self.before = self.whole.clone()

    def view(self, whole):
        return whole[GUARD:].as_strided(self.shape, self.strides)

    def data_ptr(self):
        return self.at.data_ptr()

    def get_device(self):
        return self.whole.get_device()

    @property
    def device(self):
        return self.whole.device

    @property
    def nbytes(self):
        return self.at.nbytes

    def check(self):
        now, before = self.whole.clone(), self.before.clone()
        if self.t.numel():
            self.view(now).fill_(0), self.view(before).fill_(0)
        bits = torch.int16 if now.element_size() == 2 else torch.int32 if now.element_size() == 4 else torch.int64
        assert torch.equal(now.view(bits), before.view(bits)), "written outside the tensor"
        return self.t


def written(*shape, dtype=torch.float32):
    """A vector that a call writes, on 16 bytes, with a pattern behind it that `tail` looks for."""
    n = math.prod(shape)
    whole = torch.full((n + 64,), 7, dtype=dtype, device="cuda")
    return whole, whole[:n].view(shape)


def tail_is_whole(whole, n):
    assert bool((whole[n:] == 7).all()), "written behind the end"
