"""The serving operators' definitions in 64 bits (CPU) and error bounds of their results, for the tests of those operators."""
import ctypes
import math

import torch

from paper_2311_02382_amd import lss

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of the type, relative to the value
DTYPES = [torch.bfloat16, torch.float32]


def normal(*shape, seed, dtype=torch.bfloat16, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen, dtype=torch.float32) * std).to(dtype)


def starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32)


def frequencies(rot, base=10000.0):
    return base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)


def tables(lengths, page, seed, spare=2, extra=0):
    """(table [B, most pages + extra] with the unused entries -1, number of pages): pages in random order, `spare` of them nobody's"""
    need = [-(-max(n, 0) // page) for n in lengths]
    order = torch.randperm(sum(need) + spare, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lengths), max(need + [1]) + extra), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare


def rotate(x, positions, freq, interleaved):
    """(rotated, bound of |error| apart from the rounding to the type) of x [rows, heads, d] in 64 bits.

    An angle is wrong by at most pi 2^-24 (its part of a turn, rounded to 32 bits), its cosine and sine by 4 2^-24 more, and the two products and
    their sum round by 2^-24 of |x| + |y| at most each."""
    out, slack = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    if freq is None:
        return out, slack
    rot = 2 * len(freq)
    one = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    two = one + 1 if interleaved else one + rot // 2
    a = positions.double()[:, None, None] * freq
    u, w = x.double()[..., one], x.double()[..., two]
    out[..., one], out[..., two] = u * a.cos() - w * a.sin(), u * a.sin() + w * a.cos()
    slack[..., one] = slack[..., two] = (math.pi + 4 + 3) * 2.0 ** -24 * (u.abs() + w.abs())
    return out, slack


def attention(q, k, v, seen, dtype):
    """One head: rows q [n, d], row i sees the first seen[i] keys.  Returns (out, lse, bounds of their errors).

    A score's sum of d products is off by at most (d + 2) 2^-24 of the sum of their sizes (in units of the softmax's exponent), an
    exponential by 2^-21 of itself (its own error and its argument's rounding, scores below 32), the sums over n keys by (n + 8) 2^-24; a weight
    rounded to the type before it multiplies a value by half a step of it, and so is the result."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = k.shape
    score = q @ k.T / math.sqrt(d)
    hidden = torch.arange(n, device=q.device) >= seen[:, None]
    size = (q.abs() @ k.abs().T / math.sqrt(d)).masked_fill(hidden, 0.0).amax(-1) if n else torch.zeros(len(q), dtype=torch.float64, device=q.device)
    score = score.masked_fill(hidden, -math.inf)
    lse = torch.logsumexp(score, -1) if n else torch.full((len(q),), -math.inf, dtype=torch.float64, device=q.device)
    weight = (score - lse[:, None]).exp().masked_fill(hidden, 0.0)
    out, absolute = weight @ v, weight @ v.abs()
    each = (d + 2) * 2.0 ** -24 * size + 2.0 ** -21 + (n + 8) * 2.0 ** -24
    out_bound = HALF[dtype] * out.abs() + (HALF[dtype] + 2 * each)[:, None] * absolute
    lse_bound = each + 2.0 ** -21 + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0.0)
    return out, lse, out_bound, lse_bound


def check(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got - want).abs() <= bound) & ~((got == want) & torch.isinf(want))
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values are off, first at {at}: {float(got[at])} for {float(want[at])} +- {float(bound[at]):.3g}")


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu()


def packed_plan(rows_q, rows_k, B, H, H_kv, d, dtype=torch.bfloat16):
    """(blocks of 32 rows, groups of wavefronts, key splits) of a packed launch (csrc/lss_plan.h)"""
    plan = (ctypes.c_int * 3)()
    lss._check(lss.load().lss_plan_packed(*map(ctypes.c_int64, (rows_q, rows_k, B, H, H_kv, d)), ctypes.c_int(dtype.itemsize), plan))
    return tuple(plan)
