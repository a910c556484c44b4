"""Problems for fastav_attend with chosen queries, keys and values, at row counts that reach each of its kernels."""
import math

import torch

import cache_reference as ref
from test_gpu_attend import CODE, Problem

# Query rows per sequence at four heads per KV head: one (the kernel for few rows), 32 stacked rows (the kernel for many, both of its streams on the
# same rows) and 160 (a stream for each half).
GROUP = 4
ROWS = [1, 8, 40]


def direction(dim, seed=1):
    """A row of +-1: keys along it have codes of one magnitude, and logits that are known."""
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(0, 2, (dim,), generator=gen).float() * 2 - 1


def along(logits, dim):
    """Keys [n, dim] whose logits (base 2, softmax scale 1 / sqrt(dim)) with `direction` are about `logits`."""
    return logits[:, None] * (math.sqrt(dim) / (dim * math.log2(math.e))) * direction(dim)


def place(p, b, k=None, v=None):
    """Puts rows k and v ([n, heads, dim]) in the place of what sequence b of the problem holds (b >= len(p.lens): a prefix)."""
    table = p.tables[0][b] if b < len(p.lens) else p.tables[1][b - len(p.lens)]
    for x, pool, scales, which in ((k, p.cache.k, p.cache.k_scale, 0), (v, p.cache.v, p.cache.v_scale, 1)):
        if x is None:
            continue
        codes, scale = ref.quantise(x.to(torch.bfloat16), CODE[p.fmt])
        t = torch.arange(len(x))
        to, slot = table.long()[t // p.page], t % p.page
        pool.view(torch.int8)[to.cuda(), :, slot.cuda()] = codes.float().to(CODE[p.fmt]).view(torch.int8).cuda()
        scales[to.cuda(), :, slot.cuda()] = scale.cuda()
        p.tokens[b][which] = codes * scale.double()[..., None]


def set_queries(p, q):
    p.q = q.expand(p.total, p.hq, p.dim).to(torch.bfloat16)
    p.qd = p.q.cuda()


def long_problem(rows, fmt="int8", hkv=8, dim=64, n=9000, **more):
    """One sequence on so many units that a warp, or a block, has several one behind the other."""
    return Problem(GROUP * hkv, hkv, dim, fmt, 64, [n], [rows], **more)
