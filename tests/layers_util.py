"""Plain 64-bit forms of the layers over packed batches (causal attention of whole prompts, linear attention with decays), written out as their
definitions, and the bounds that the kernels' roundings leave."""
import math

import torch

from cache_util import BF16_HALF, FP32_HALF, attention


def starts_of(lens, first=0):
    return torch.tensor([first + sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32)


def prompts(q, k, v, starts, scale):
    """q [T,Hq,d], k/v [T,Hkv,d] on the CPU -> out [T,Hq,d], lse [Hq,T] and the bounds of their errors (cache_util.attention); 0 for rows of no
    sequence."""
    T, Hq, d = q.shape
    G = Hq // k.shape[1]
    out, lse = torch.zeros(T, Hq, d, dtype=torch.float64), torch.zeros(Hq, T, dtype=torch.float64)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for a, e in zip(starts[:-1].tolist(), starts[1:].tolist()):
        if e <= a:
            continue
        see = torch.ones(e - a, e - a, dtype=torch.bool).tril()
        o, z, eo, ez = attention(q[a:e][None], scale, lambda b, t: (k[a:e, t // G].double(), v[a:e, t // G].double(), see))
        out[a:e], lse[:, a:e], e_out[a:e], e_lse[:, a:e] = o[0], z[0], eo[0], ez[0]
    return out, lse, e_out, e_lse


def check_prompts(got, ref, rows=None, what=""):
    (o, z), (out, lse, e_out, e_lse) = got, ref
    bf16 = o.dtype == torch.bfloat16
    o, z = o.double().cpu(), z.double().cpu()
    rows = slice(None) if rows is None else rows
    off, bound = (o - out).abs()[rows], (e_out + (BF16_HALF * (out.abs() + e_out) if bf16 else 0.0) + 1e-30)[rows]
    assert torch.isfinite(o[rows]).all(), what
    assert (off <= bound).all(), f"{what}: out off by {float((off / bound).max()):.2f} of the bound"
    off = (z - lse).abs()[:, rows]
    assert (off <= e_lse[:, rows]).all(), f"{what}: lse off by {float((off / e_lse[:, rows]).max()):.2f} of the bound"


def linear(q, k, v, decay, scale, state, chunked):
    """One sequence: q [n,Hq,d] (or None), k/v [n,Hkv,d], decay [Hkv] or [n,Hkv] (<= 0), state [Hkv,d,d] -> out [n,Hq,d], the states behind every
    row [n+1,Hkv,d,d], and the bounds of their errors; all in 64 bits.

    Bounds. With A the state of the same recurrence over absolute values, no number of the state, nor any sum on the way to it, is larger
    than A. Row by row in fp32, a step rounds the decay's factor, the product with it and the sum (k v is exact): 3 * 2^-24 A, and earlier errors
    shrink with the decays. By chunks of 32: a weight exp(c) is off by 2^-22 and by the rounding of c, a sum of up to 32 numbers in five
    steps after a product each, 8 * 2^-24 |c| with |c| <= `most`, the largest sum of |decay| log2(e) over a chunk (decays below 2^-150 count as
    that); a chunk's 96 products (32 keys, three parts of v) are added one by one: (100 + 8 most) 2^-24 A for each chunk. The factors' own
    roundings do not add up beyond that.
    out is scale q . S: in fp32 sums of d products, by (d + 8) 2^-24 of scale |q| A, and the state's error. By chunks the state's numbers
    or the weights of the chunk's rows are rounded to bf16 (2^-8), the weights after a sum of d products."""
    n, Hkv, d = k.shape
    g = decay.double().expand(n, Hkv) if decay.dim() == 1 else decay.double()
    S = state.double().clone()
    A, E = S.abs(), torch.zeros_like(S)
    states, errors, out, e_out = [S], [E], [], []
    low = g.clamp(min=-150 * math.log(2)).abs() / math.log(2)
    most = max([float(low[i:i + 32].sum(0).max()) for i in range(0, n, 32)] or [0.0])
    for i in range(n):
        f = torch.exp(g[i])[:, None, None]
        kv = k[i].double()[:, :, None] * v[i].double()[:, None, :]
        S = S * f + kv
        A = A * f + kv.abs()
        steps = 3 * (i + 1) if not chunked else (100 + 8 * most) * (i // 32 + 1)
        E = steps * FP32_HALF * A
        states.append(S)
        errors.append(E)
        if q is not None:
            x = q[i].double().view(Hkv, -1, d)
            out.append(scale * torch.matmul(x, S).reshape(-1, d))
            part = (d + 8) * FP32_HALF + (1.05 * BF16_HALF + (d + 40 + 16 * most) * FP32_HALF if chunked else 0.0)
            e_out.append(abs(scale) * torch.matmul(x.abs(), E + part * A).reshape(-1, d))
    none = torch.zeros(0, 0, d, dtype=torch.float64)
    return torch.stack(out) if out else none, torch.stack(states), torch.stack(e_out) if e_out else none, torch.stack(errors)


def check_linear(got, out, e_out, what=""):
    bf16 = got.dtype == torch.bfloat16
    o = got.double().cpu()
    assert torch.isfinite(o).all(), what
    off, bound = (o - out).abs(), e_out + (BF16_HALF * (out.abs() + e_out) if bf16 else 0.0) + 1e-30
    assert (off <= bound).all(), f"{what}: off by {float((off / bound).max()):.2f} of the bound"
