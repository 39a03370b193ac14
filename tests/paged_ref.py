"""Plain 64-bit implementations of the paged cache and the sampler, on the CPU: loops over tokens, from the definitions."""
import math

import torch

BLOCK = 16


def table(positions, rd, theta=1.0e4):
    f = theta ** (-2.0 * torch.arange(rd // 2, dtype=torch.float64) / rd)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def rotate(x, tab, pos, layout):
    """x [heads][hd] in 64 bits, at one position."""
    if tab is None:
        return x
    c, s = tab[pos, :, 0].double(), tab[pos, :, 1].double()
    half = c.numel()
    y = x.clone()
    lo = slice(0, half) if layout == "half" else slice(0, 2 * half, 2)
    hi = slice(half, 2 * half) if layout == "half" else slice(1, 2 * half, 2)
    y[:, lo] = x[:, lo] * c - x[:, hi] * s
    y[:, hi] = x[:, hi] * c + x[:, lo] * s
    return y


def scale_exponent(amax):
    """Biased exponent of the smallest power of two with amax <= 448 times it."""
    if amax == 0.0:
        return 0
    e = -127
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return e + 127


def values(codes, scales):
    """64-bit values of pages [..., page, hd] of codes with scales [..., page / 16]."""
    f = torch.exp2(scales.double() - 127)
    return codes.view(torch.float8_e4m3fn).double() * f.repeat_interleave(BLOCK, -1)[..., None]


def attention(q, keys, vals, see, scale):
    """q [n][H][hd], keys and vals [T][Hk][hd], see [n][T]: only the seen entries are touched."""
    n, H, hd = q.shape
    G = H // keys.shape[1]
    out = torch.zeros(n, H, hd, dtype=torch.float64)
    size = 0.0  # the largest sum of |q||k| of a score: what its rounding scales with
    for i in range(n):
        t = see[i].nonzero()[:, 0]
        if not t.numel():
            continue
        for h in range(H):
            k, v = keys[t, h // G], vals[t, h // G]
            s = (k @ q[i, h]) * scale
            size = max(size, float((k.abs() @ q[i, h].abs()).max()) * abs(scale))
            out[i, h] = torch.softmax(s, 0) @ v
    return out, size


def ancestors(parent):
    n = len(parent)
    see = torch.zeros(n, n, dtype=torch.bool)
    depth = [0] * n
    for i in range(n):
        if i:
            see[i] = see[parent[i]]
            depth[i] = depth[parent[i]] + 1
        see[i, i] = True
    return see, torch.tensor(depth)


def sample(z, T, k, p, min_p, u):
    """(token, logp, kept, distance of the draw from the nearest border, as a share of the total) of one row."""
    z = torch.where(torch.isnan(z), -math.inf, z.double()).clamp(max=3.4028234663852886e38)
    V = z.numel()
    if not bool((z > -math.inf).any()):
        return -1, -math.inf, 0, 1.0
    if not T > 0:
        T, k = 1.0, 1
    order = sorted(range(V), key=lambda i: (-float(z[i]), i))
    order = [i for i in order if z[i] > -math.inf][:k if k > 0 else V]
    w = [math.exp((float(z[i]) - float(z[order[0]])) / T) for i in order]
    if p < 1:
        total, run, n = math.fsum(w), 0.0, 0
        while n < len(w) and (n == 0 or run < p * total):
            run += w[n]
            n += 1
        order, w = order[:n], w[:n]
    n = max(1, sum(x >= min_p for x in w)) if min_p > 0 else len(w)
    order, w = order[:n], w[:n]
    total, run, tok, near = math.fsum(w), 0.0, None, 1.0
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    for i, x in sorted(zip(order, w)):
        run += x
        near = min(near, abs(run / total - u)) if x > 2.0 ** -44 else near
        if tok is None and run > u * total and x > 2.0 ** -44:
            tok = i
    if tok is None:
        tok = max(i for i, x in zip(order, w) if x > 2.0 ** -44)
    return tok, (float(z[tok]) - float(z[order[0]])) / T - math.log(total), n, near
