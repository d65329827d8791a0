"""Plain float64 implementations of the uncompressed layers' operators (CPU, torch)."""
import math

import torch

TOP = {0: 127.0, 1: 448.0}


def rope_turns(R, theta, scaling, factor=1.0, L0=0, lo=0.0, hi=0.0):
    """Frequencies f_j of the R/2 pairs."""
    f = [theta ** (-2.0 * j / R) for j in range(R // 2)]
    if scaling == 1:
        f = [x / factor for x in f]
    elif scaling == 2:
        f = [(theta * factor ** (R / (R - 2.0))) ** (-2.0 * j / R) for j in range(R // 2)]
    elif scaling == 3:
        lo, hi = (lo, hi) if hi else (1.0, 4.0)
        w = [min(max((L0 * x / (2 * math.pi) - lo) / (hi - lo), 0.0), 1.0) for x in f]
        f = [x * (u + (1 - u) / factor) for x, u in zip(f, w)]
    elif scaling == 4:
        lo, hi = (lo, hi) if hi else (1.0, 32.0)

        def at(n):
            return R * math.log(L0 / (2 * math.pi * n)) / (2 * math.log(theta))
        j0, j1 = max(math.floor(at(hi)), 0), min(math.ceil(at(lo)), R - 1)
        r = [min(max((j - j0) / max(j1 - j0, 1e-3), 0.0), 1.0) for j in range(R // 2)]
        f = [x * (1 - u) + x / factor * u for x, u in zip(f, r)]
    return torch.tensor(f, dtype=torch.float64)


def rope(x, pos, f, interleaved, gain=1.0, inverse=False):
    """x [..., H, d] float64 at pos [...]; the first 2 len(f) channels are rotated."""
    R = 2 * len(f)
    a = pos.double()[..., None, None] * f * (-1.0 if inverse else 1.0)
    c, s = torch.cos(a) * gain, torch.sin(a) * gain
    p = torch.arange(0, R, 2) if interleaved else torch.arange(R // 2)
    q = p + 1 if interleaved else p + R // 2
    y = x.clone()
    y[..., p] = x[..., p] * c - x[..., q] * s
    y[..., q] = x[..., q] * c + x[..., p] * s
    return y


def grid(code):
    """The non-negative values of the code, in order."""
    if code == 0:
        return torch.arange(128, dtype=torch.float64)
    return torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
                         for e in range(16) for m in range(8)][:127], dtype=torch.float64)


def quantize(x, code):
    """Blocks [..., T, d]: signed grid values and fp32 scales [...].  A border between two
    codes goes to the even one; a block with a NaN or an infinity has scale NaN and codes 0."""
    x = x.double()
    s = (x.abs().amax((-2, -1)) / torch.tensor(TOP[code], dtype=torch.float64)).float()
    bad = ~torch.isfinite(x).all(-1).all(-1)
    s = torch.where(bad, math.nan, s)
    d = s.double()[..., None, None]
    a = torch.where(d > 0, x.abs() / d, 0.0)
    g = grid(code)
    mid = (g[1:] + g[:-1]) / 2
    lo, hi = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)
    i = torch.where(lo % 2 == 0, lo, hi)
    v = torch.where(bad[..., None, None], 0.0, torch.sign(x) * g[i])
    return v, s


def cached(x, code, T):
    """Rows x [n][d] of one head as the cache holds them."""
    n = x.shape[0] // T * T
    y = x.double().clone()
    if n:
        v, s = quantize(x[:n].reshape(-1, T, x.shape[1]), code)
        y[:n] = (v * s.double()[:, None, None]).reshape(n, -1)
    return y


def attend(q, K, V, scale, first):
    """q [m][d] (query tokens of one head), K, V [n][d] float64; query j sees tokens up to
    first + j.  Returns (out [m][d], sum p |v|, sum over channels |q k| scale at most, p [m][n])."""
    m, n = q.shape[0], K.shape[0]
    seen = torch.arange(n)[None] <= first + torch.arange(m)[:, None]
    s = q.double() @ K.T * scale
    mag = (q.double().abs() @ K.abs().T * scale)
    s = torch.where(seen, s, -math.inf)
    top = s.amax(-1, keepdim=True) if n else torch.zeros(m, 1, dtype=torch.float64)
    p = torch.where(seen, torch.exp(s - torch.where(top > -math.inf, top, 0.0)), 0.0)
    l = p.sum(-1, keepdim=True)
    p = torch.where(l > 0, p / torch.where(l > 0, l, 1.0), torch.where(l == 0, 0.0, l))
    big = torch.where(seen, mag, 0.0).amax(-1) if n else torch.zeros(m, dtype=torch.float64)
    # a token that is not seen has no part in the sum, whatever it holds
    o = torch.stack([p[j, :max(first + j + 1, 0)] @ V[:max(first + j + 1, 0)] for j in range(m)])
    a = torch.stack([p[j, :max(first + j + 1, 0)] @ V[:max(first + j + 1, 0)].abs()
                     for j in range(m)])
    return o, a, big, p


def evict(w, table, ctx, T, keep, sink, recent):
    """One head: (table, weights, tokens)."""
    J, n = len(w), ctx // T
    gone = max(n - keep, 0) // 2 * 2

    def key(i):
        return (math.inf, 1) if math.isnan(w[i]) else (w[i] + 0.0, 0)
    free = sorted(range(min(sink, n), max(n - recent, sink)), key=lambda i: (key(i), -i))
    out = set(free[:gone])
    order = [i for i in range(n) if i not in out] + sorted(out) + list(range(n, J))
    w2 = [w[i] for i in order[:n - gone]] + [0.0] * (J - n + gone)
    if n < J:
        w2[n - gone] = w[n]
    return [table[i] for i in order], w2, ctx - gone * T
