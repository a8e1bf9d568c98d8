"""Plain 64-bit models of the ragged caches (bf16, fp32 or 8-bit) and of the
rows that single queries and drafted trees read from them, on the CPU.

Tolerances of a row o = sum_j p_j v_j / sum_j p_j, with A = sum_j p_j |v_j| and p
normalised.  u = 2^-24.  A logit is a sum of d products in fp32 and is then
scaled: its error is at most delta = (d + 4) u max_j sum_i |q_i k_ji| / sqrt(d)
+ 4 u max_j |logit_j|, and that of its weight delta + 4 u relative (an exp2 within
4 u); numerator and denominator each add n of them one by one at worst.  So
    fp32  |err| <= (2 delta + (2 n + 16) u) (A + |o|)
    bf16  the weights of the numerator and the output are rounded as well, half
          a step, 2^-8, each: + 2^-8 A + 2^-8 |o|
Rows of the 8-bit cache are compared with a model that holds the same codes, so
their quantisation is no part of it.
"""
import math

import torch

import oracle

SLIDING, ALIGNED, BLOCKED = 0, 1, 2
U = 2.0 ** -24


def first_position(window, p, W, C):
    lo = max(0, p - W + 1)
    return lo // C * C if window == ALIGNED else p // W * W if window == BLOCKED else lo


def quantise(x):
    """[..., d] -> (codes as float8_e4m3fn, exponent bytes), the 8-bit cache's rows."""
    x = x.float()
    top = torch.where(torch.isfinite(x), x, 0).abs().amax(-1)
    m, e = torch.frexp(top)
    e = torch.where(top > 0, e - 9 + (m > 0.875).int(), 0).clamp(-126, 119)
    scaled = torch.where(torch.isfinite(x), torch.ldexp(x, -e.unsqueeze(-1)), math.nan)
    return scaled.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def value(codes, exp):
    return codes.double() * torch.pow(2.0, exp.double() - 127).unsqueeze(-1)


def plain(x):
    return x.double()


def quantised(x):
    return value(*quantise(x))


def summary(k, v):
    """Mean key and softmax-weighted value of one chunk [C, d]."""
    ks, vs = oracle.summaries(k.numpy(), v.numpy(), k.shape[0])
    return torch.from_numpy(ks[0]), torch.from_numpy(vs[0])


class Model:
    """One (sequence, kv head): rows as the cache holds them, by position.

    k, v, Ks, Vs: the prompt's rows and summaries as given to the fill; `held`
    turns given rows into held ones."""

    def __init__(self, k, v, Ks, Vs, W, C, window, held):
        self.W, self.C, self.window, self.held = W, C, window, held
        self.k, self.v = list(held(k)), list(held(v))
        self.ks, self.vs = list(held(Ks)), list(held(Vs))

    def append(self, k, v):
        self.k.append(self.held(k))
        self.v.append(self.held(v))
        n = len(self.k)
        if n % self.C == 0:
            ks, vs = summary(torch.stack(self.k[n - self.C:]), torch.stack(self.v[n - self.C:]))
            self.ks.append(ks)
            self.vs.append(vs)
            self.round_summary()

    def round_summary(self):
        # as the cache's own type holds it; the 8-bit one's is compared, and
        # taken over, by the tests that need it
        pass

    def keys(self, p, extra=()):
        """(keys, values, log-weights) of the row at position p over the cache's
        rows below and the `extra` (k, v) rows."""
        n = len(self.k)
        lo = first_position(self.window, p, self.W, self.C)
        s = lo // self.C
        pick = list(range(lo, min(n, p + 1)))
        k = self.ks[:s] + [self.k[i] for i in pick] + [e[0] for e in extra]
        v = self.vs[:s] + [self.v[i] for i in pick] + [e[1] for e in extra]
        bias = torch.zeros(len(k), dtype=torch.float64)
        bias[:s] = math.log(self.C)
        return torch.stack(k), torch.stack(v), bias


def row(q, k, v, bias, dtype):
    """Rows q [heads, d] over keys and values: (o, bound)."""
    d = q.shape[-1]
    q = q.double()
    s = q @ k.T / math.sqrt(d) + bias
    p = torch.softmax(s, -1)
    o, A = p @ v, p @ v.abs()
    size = (q.abs() @ k.abs().T / math.sqrt(d)).amax(-1, keepdim=True)
    delta = (d + 4) * U * size + 4 * U * s.abs().amax(-1, keepdim=True)
    bound = (2 * delta + (2 * len(k) + 16) * U) * (A + o.abs())
    if dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (A + o.abs())
    return o, bound


def line_of(parents, t):
    """Node t and the nodes it continues, the root first."""
    line = []
    while 0 <= t < len(parents) and (not line or t < line[-1]):
        line.append(t)
        t = int(parents[t])
    return line[::-1]


def random_tree(B, T, gen):
    """Parents of a mixture of chains and branches."""
    t = torch.arange(T)
    any_ = (torch.rand(B, T, generator=gen) * (t + 1)).long() - 1
    return torch.where(torch.rand(B, T, generator=gen) < 0.5, t - 1, torch.minimum(any_, t - 1)).int()
