"""Plain 64-bit forms of the 8-bit K/V cache and of the attention over it, on the CPU, from the definitions in fastav.h."""
import math

import torch

LARGEST = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}


def e4m3(y: torch.Tensor) -> torch.Tensor:
    """float64 -> nearest e4m3 value, ties to even: three bits behind the first, steps of 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def quantise(x: torch.Tensor, code: torch.dtype):
    """Rows x [..., dim] (bf16) -> codes (float64) and scales (float32); a row with a value that is not finite gets codes 0 and scale NaN."""
    x = x.double()
    top = x.abs().amax(-1)
    good = torch.isfinite(top)
    largest = LARGEST[code]
    y = torch.where((good & (top > 0))[..., None], x * largest / top[..., None], torch.zeros_like(x))
    y = torch.round(y) if code == torch.int8 else e4m3(y)
    scale = torch.where(good, top.float() / largest, torch.full_like(top, math.nan).float())
    return torch.where(good[..., None], y, torch.zeros_like(y)), scale


def attend(q, keys, values, sees, scale):
    """One sequence: q [R, Hq, d], keys and values [n, Hkv, d] (float64), row r sees the first sees[r] of them.  (out, lse, weight of
    |v|: sum_j p_j |v_j|, largest sum_i |q_i k_ji| times scale, n max_j p_j max_i |v_ji|)."""
    rows, hq, dim = q.shape
    group = hq // keys.shape[1]
    q = q.double()
    out, lse = torch.zeros(rows, hq, dim, dtype=torch.float64), torch.full((rows, hq), -math.inf, dtype=torch.float64)
    mass, size, most = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(lse)
    for h in range(hq):
        k, v = keys[:, h // group], values[:, h // group]
        for r in range(rows):
            n = int(sees[r])
            if n <= 0:
                continue
            z = k[:n] @ q[r, h] * scale
            lse[r, h] = torch.logsumexp(z, 0)
            p = torch.exp(z - lse[r, h])
            out[r, h] = p @ v[:n]
            mass[r, h] = p @ v[:n].abs()
            size[r, h] = (k[:n].abs() @ q[r, h].abs()).max() * scale
            most[r, h] = n * (p * v[:n].abs().amax(1)).max()
    return out, lse, mass, size, most
