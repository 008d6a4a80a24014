"""Plain 64-bit references of the operators at the ends of a training step."""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step, relative to the value
U = 2.0 ** -24


def normal(shape, seed, std=1.0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype)


def assert_within(got, want, tol, what):
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    tol = torch.as_tensor(tol, dtype=torch.float64).cpu().expand(want.shape)
    bad = ~((got - want).abs() <= tol) & ~(got == want)
    if bad.any():
        i = tuple(int(k[0]) for k in torch.nonzero(bad, as_tuple=True))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: got {float(got[i])}, want {float(want[i])}, "
                             f"tolerance {float(tol[i])}")


# ------------------------------------------------------------------------------------------------- heads ----
def pairs(rotary, interleaved):
    """Places of the first and second elements of the pairs that turn."""
    i = torch.arange(rotary // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)


def turned(u, positions, inv_freq, interleaved, back=False):
    """u: [rows, heads, dim] in 64 bits."""
    if inv_freq is None:
        return u
    first, second = pairs(2 * len(inv_freq), interleaved)
    t = positions.double()[:, None, None] * inv_freq.double()
    c, s = torch.cos(t), torch.sin(t) * (-1 if back else 1)
    out = u.clone()
    out[..., first] = u[..., first] * c - u[..., second] * s
    out[..., second] = u[..., second] * c + u[..., first] * s
    return out


def heads_fwd(x, hq, hk, gain_q, gain_k, eps, inv_freq, positions, interleaved):
    """x: [rows, (hq + hk) * dim] in 64 bits."""
    h = x.unflatten(1, (hq + hk, -1))
    dim = h.shape[2]
    one = torch.ones(dim, dtype=torch.float64)
    gain = torch.cat([(one if gain_q is None else gain_q.double()).expand(hq, -1), (one if gain_k is None else gain_k.double()).expand(hk, -1)])
    n = h / (h.square().mean(2, keepdim=True) + eps).sqrt()
    return turned(n * gain, positions, inv_freq, interleaved).flatten(1)


def beside(v, rotary, interleaved):
    """Magnitudes of the elements and of their partners, added."""
    if not rotary:
        return v.abs()
    first, second = pairs(rotary, interleaved)
    out = v.abs()
    out[..., first] = v[..., first].abs() + v[..., second].abs()
    out[..., second] = out[..., first]
    return out


# ----------------------------------------------------------------------------------------------- logprob ----
class Softmax:
    """Of scale * logits, row by row, with the bounds of what binary32 can lose.  Rows of nothing but minus infinities have probability 0 everywhere."""

    def __init__(self, logits, scale):
        x = logits.double()
        self.top = x.max(1, keepdim=True).values
        self.empty = torch.isinf(self.top[:, 0])
        d = torch.where(self.empty[:, None], -math.inf, (x - torch.where(torch.isinf(self.top), 0.0, self.top)) * scale)
        self.log_total = torch.log(torch.exp(d).sum(1, keepdim=True))
        self.lse = (torch.where(torch.isinf(self.top), 0.0, self.top) * scale + self.log_total)[:, 0]
        self.lse = torch.where(self.lse.abs() >= 2.0 ** 128, torch.copysign(torch.tensor(math.inf, dtype=torch.float64), self.lse), self.lse)  # (as binary32 rounds it)
        self.log_p = torch.where(self.empty[:, None], -math.inf, d - torch.where(self.empty[:, None], 0.0, self.log_total))
        self.p = torch.exp(self.log_p)
        self.surprise = torch.where(torch.isinf(self.log_p), 0.0, -self.log_p)
        self.entropy = (self.p * self.surprise).sum(1)
        far = torch.where(torch.isinf(d), 0.0, -d)
        self.mean, self.square = (self.p * far).sum(1), (self.p * far * far).sum(1)
        # A sum's terms: chains of vocab / 1024 additions and some 30 beyond them; 2^-22 for the exponential; a difference is off by four
        # roundings, which moves its term by that times the difference.
        self.steps = (logits.shape[1] / 1024 + 30) * U + 2.0 ** -21
        self.sum_off = self.steps + 4 * U * self.mean
        self.entropy_off = 2 * self.steps * (1 + self.mean) + 8 * U * (self.mean + self.square) + 4 * U * self.entropy
        self.lse_off = self.sum_off + 2 * U * (self.lse.abs().nan_to_num(posinf=0.0) + (self.top[:, 0] * scale).abs().nan_to_num(posinf=0))

    def log_p_off(self):
        """Of a log probability that is taken from the largest logit and the sum."""
        return self.sum_off[:, None] + 4 * U * (self.surprise + self.log_total.nan_to_num(neginf=0))

    def grad(self, targets, dlogprob, dentropy, scale):
        """The gradient and how far binary32 may be off it, before the rounding to the output's type."""
        rows, vocab = self.p.shape
        there = (targets >= 0) & (targets < vocab)
        hit = torch.zeros_like(self.p)
        hit[there, targets[there].long()] = 1.0
        w = torch.zeros(rows, dtype=torch.float64) if dlogprob is None else torch.where(there, dlogprob.double(), 0.0)
        e = torch.zeros(rows, dtype=torch.float64) if dentropy is None else dentropy.double()
        w, e = w[:, None], e[:, None]
        g = w * (hit - self.p) + e * self.p * (self.surprise - self.entropy[:, None])
        off = self.log_p_off() + 2.0 ** -21 + 2 * U * self.surprise
        tol = w.abs() * (self.p * off + 4 * U * (hit + self.p))
        tol = tol + e.abs() * self.p * ((self.surprise + self.entropy[:, None]) * (off + 8 * U) + self.log_p_off() + self.entropy_off[:, None])
        # probabilities below the smallest normal binary32 number are taken for 0
        tol = tol + self.p.clamp_max(2.0 ** -126) * (w.abs() + e.abs() * (self.surprise + self.entropy[:, None]))
        zero = self.empty[:, None]
        return torch.where(zero, 0.0, g * scale), torch.where(zero, 0.0, tol * scale)


def top_of(logits, top):
    """Places of the largest, equal ones by index."""
    return torch.sort(logits.double(), dim=1, descending=True, stable=True).indices[:, :top]
