"""Plain 64-bit forms of the rotation with head norms, of the weights that query rows pay and of eviction, on the CPU, from the definitions in fastav.h."""
import math

import torch


def turned(x, pos, frequencies, axis=None, interleaved=False, norm=None, eps=0.0):
    """x [tokens, heads, dim] (any type) normed and rotated; pos [axes, tokens] or [tokens].  (result, of each element the magnitude of its pair
    before the rotation.)  The angle is reduced modulo a turn as integers would: positions and frequencies are exact, their product is taken in parts."""
    x = x.double()
    if norm is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * norm.double()
    y, size = x.clone(), x.abs()
    half = len(frequencies)
    pos = pos.reshape(-1, x.shape[0])
    for p, f in enumerate(frequencies):
        at = pos[0 if axis is None else axis[p]].tolist()
        t = torch.tensor([angle(n, f) for n in at], dtype=torch.float64)[:, None]
        a, b = (2 * p, 2 * p + 1) if interleaved else (p, p + half)
        y[..., a] = x[..., a] * torch.cos(t) - x[..., b] * torch.sin(t)
        y[..., b] = x[..., b] * torch.cos(t) + x[..., a] * torch.sin(t)
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def _arctan_of_inverse(x: int, bits: int) -> int:
    """arctan(1 / x) in units of 2^-bits, by its series."""
    term = total = (1 << bits) // x
    n = 1
    while term:
        term //= -x * x
        n += 2
        total += term // n
    return total


_BITS = 900
TWO_PI = 8 * (4 * _arctan_of_inverse(5, _BITS + 40) - _arctan_of_inverse(239, _BITS + 40)) >> 40  # Machin's formula, in units of 2^-_BITS


def angle(n: int, f: float) -> float:
    """n * f modulo 2 pi, within 2^-52 of a turn: whole-number arithmetic on the exact fraction that f is."""
    num, den = f.as_integer_ratio()
    num *= n
    scaled = (num << _BITS) // den
    return (scaled % TWO_PI) / (1 << _BITS)


def weigh(weights, decay, fresh, q, keys, lse, sees, scale):
    """One sequence: weights [n, Hkv] before, of which the first `fresh` count; q [R, Hq, d], keys [n, Hkv, d] (float64), lse [R, Hq].  (weights after, sum of
    what was paid times its own possible error in units: magnitude of the logit's terms + |lse| + 1.)"""
    n, hkv = keys.shape[:2]
    group = q.shape[1] // hkv
    out = torch.zeros(n, hkv, dtype=torch.float64)
    out[:fresh] = decay * weights[:fresh].double() if decay else 0.0
    size = torch.zeros_like(out)
    q, lse = q.double(), lse.double()
    for h in range(q.shape[1]):
        k = keys[:, h // group]
        for r in range(q.shape[0]):
            m = max(0, min(n, int(sees[r])))
            if m == 0 or torch.isinf(lse[r, h]):
                continue
            p = torch.exp(k[:m] @ q[r, h] * scale - lse[r, h])
            out[:m, h // group] += p
            size[:m, h // group] += p * (k[:m].abs() @ q[r, h].abs() * scale + lse[r, h].abs() + 1)
    return out, size


def survivors(weights, keep, first, recent):
    """Indices that stay, ascending: weights [n] (float), the heaviest, ties to the lower index, NaN lowest, the first and the recent above all."""
    n = len(weights)

    def rank(j):
        if j < first or j >= n - recent:
            return (0, 0.0, j)
        w = float(weights[j])
        return (2, 0.0, j) if math.isnan(w) else (1, -w, j)

    return sorted(sorted(range(n), key=rank)[:max(0, min(keep, n))])
