"""Plain 64-bit forms of the operators around a small cache (4-bit cache, window attention), written out as their definitions,
and the bounds that the kernels' roundings leave."""
import math

import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BF16_HALF = 2.0 ** -8          # torch.finfo(torch.bfloat16).eps / 2: a bf16's rounding, relative
FP32_HALF = 2.0 ** -24


def quantise(x):
    """bf16 tensor [..., d] -> (codes [..., d/2], scales [..., d/32]) uint8 numpy arrays, group by group as the definition says."""
    x = x.double().numpy()
    g = x.reshape(*x.shape[:-1], -1, 32)
    with np.errstate(all="ignore"):
        a = np.abs(g).max(-1)
        bad = ~np.isfinite(g).all(-1)
        a = np.where(bad | (a == 0), 1.0, a)
        low = np.floor(np.log2(a))
        e = np.clip(low - 2 + (a > 1.75 * 2.0 ** low), -125, 125)
        e = np.where((np.abs(g).max(-1) == 0) & ~bad, -125, e)
        y = np.abs(np.where(bad[..., None], 0.0, g)) / 2.0 ** e[..., None]
    dist = np.abs(y[..., None] - GRID)
    near = dist.min(-1, keepdims=True)
    pick = np.where(dist == near, np.where(np.arange(8) % 2 == 0, 2, 1), 0).argmax(-1)      # of two equally near ones the even
    code = np.where(bad[..., None], 0, pick + 8 * np.signbit(g)).astype(np.uint8).reshape(x.shape)
    scale = np.where(bad, 255, e + 127).astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def values(codes, scales):
    """float64 tensor [..., d] of codes [..., d/2] and scales [..., d/32] (uint8 tensors or arrays)."""
    c, s = np.asarray(codes), np.asarray(scales).astype(np.int64)
    nib = np.stack((c & 15, c >> 4), -1).reshape(*c.shape[:-1], -1).astype(np.int64)
    v = GRID[nib & 7] * np.where(nib >> 3, -1.0, 1.0)
    f = np.where(s == 255, np.nan, 2.0 ** (s - 127.0))
    return torch.from_numpy(v * np.repeat(f, 32, -1))


def packed_cache(B, Hkv, N, d, g, std=0.5, page=0, spare=3):
    """A random 4-bit cache and the values it stands for: (codes, scales, table or None, k, v [B,Hkv,N,d] float64); with `page`, pools
    of pages in random order."""
    k, v = (torch.randn(B, Hkv, N, d, generator=g).mul(std).to(torch.bfloat16) for _ in range(2))
    (kc, ks), (vc, vs) = quantise(k), quantise(v)
    codes, scales = torch.from_numpy(np.stack((kc, vc), 3)), torch.from_numpy(np.stack((ks, vs), 3))
    kv, vv = values(kc, ks), values(vc, vs)
    if not page:
        return codes, scales, None, kv, vv
    return (*(to_pages(t, page, g, spare, seed=5) for t in (codes, scales)), table_of(B, N, page, g, spare, seed=5), kv, vv)


def table_of(B, N, page, g, spare=3, seed=5):
    per = -(-N // page)
    return torch.randperm(B * per + spare, generator=torch.Generator().manual_seed(seed))[: B * per].to(torch.int32).view(B, per)


def to_pages(t, page, g, spare=3, seed=5):
    """[B,H,N,...] -> pool [pages,H,page,...] in the order of table_of; what no token fills is 0xff or NaN."""
    B, H, N = t.shape[:3]
    table = table_of(B, N, page, g, spare, seed)
    pool = torch.full((B * table.shape[1] + spare, H, page, *t.shape[3:]), 255 if t.dtype == torch.uint8 else float("nan"), dtype=t.dtype)
    for b in range(B):
        for j, p in enumerate(table[b].tolist()):
            part = t[b, :, j * page:(j + 1) * page]
            pool[p, :, : part.shape[1]] = part
    return pool


def attention(q, scale, keys, k_new=None, v_new=None, causal=True, q_halves=False):
    """q [B,Tq,Hq,d] bf16; keys(b, t) -> K, V [n,d] float64 and see [Tq,n] of query head t, all rows listed in order (a repeated one
    counts as often). Returns out, lse in 64 bits and the bounds of their errors.

    Bounds. The scaled scores are fp32 sums of d exact products: off by at most dS = |scale| (d + 8) 2^-24 sum |q||k|; with q_halves, Q's
    values off by 2^-17 of the largest of their 32, by |scale| 2^-17 sum_groups max|q| sum|k| more. A weight is then off by a factor
    exp(2 dS), rounded to bf16 (2^-8), its exponential by 2^-20; sums over n keys in fp32 by (n / 8 + 64) 2^-24 (eight lanes at least
    share them). The output is off by that part of sum p|v| / sum p, the logarithm by dS and the sum's part."""
    B, Tq, Hq, d = q.shape
    out, lse = torch.zeros(B, Tq, Hq, d, dtype=torch.float64), torch.full((B, Hq, Tq), -math.inf, dtype=torch.float64)
    e_out, e_lse = torch.zeros_like(out), torch.zeros_like(lse)
    x = q.double()
    for b in range(B):
        for t in range(Hq):
            K, V, see = keys(b, t)
            if k_new is not None:
                h = t // (Hq // k_new.shape[2])
                K, V = torch.cat((K, k_new[b, :, h].double())), torch.cat((V, v_new[b, :, h].double()))
                own = torch.ones(Tq, Tq, dtype=torch.bool)
                see = torch.cat((see, own.tril() if causal else own), 1)
            if K.shape[0] == 0:
                continue
            qt = x[b, :, t]
            s = scale * (qt @ K.T)
            d_s = abs(scale) * (d + 8) * FP32_HALF * (qt.abs() @ K.abs().T)
            if q_halves:
                most = qt.abs().reshape(Tq, -1, 32).amax(-1)
                d_s = d_s + abs(scale) * 2.0 ** -17 * (most @ K.abs().reshape(K.shape[0], -1, 32).sum(-1).T)
            s = torch.where(see, s, -math.inf)
            z = torch.logsumexp(s, -1)
            live = torch.isfinite(z)
            if not live.any():
                continue
            p = torch.exp(s[live] - z[live, None])
            p = torch.where(see[live], p, 0.0)
            out[b, live, t] = p @ torch.where(see[live].any(0)[:, None], V, 0.0)
            lse[b, t] = z
            worst = torch.where(see, d_s, 0.0)[live].amax(-1)
            sums = (K.shape[0] / 8 + 64) * FP32_HALF
            part = BF16_HALF + 2.2 * worst + 2.0 ** -20 + sums
            e_out[b, live, t] = part[:, None] * (p @ V.abs().nan_to_num(0.0))
            e_lse[b, t, live] = worst + sums + 2.0 ** -20 + 2.0 ** -22 * z[live].abs()
    return out, lse, e_out, e_lse


def check(got, ref, what=""):
    """(out, lse) of a call against attention()'s."""
    (o, l), (out, lse, e_out, e_lse) = got, ref
    bf16 = o.dtype == torch.bfloat16
    o, l = o.double().cpu(), l.double().cpu()
    assert torch.isfinite(o).all(), what
    off = (o - out).abs()
    bound = e_out + (BF16_HALF * (out.abs() + e_out) if bf16 else 0.0) + 1e-30
    assert (off <= bound).all(), f"{what}: out off by {float((off / bound).max()):.2f} of the bound"
    empty = torch.isneginf(lse)
    assert torch.equal(torch.isneginf(l), empty), what
    off = (l - lse).abs()[~empty]
    assert (off <= e_lse[~empty]).all(), f"{what}: lse off by {float((off / e_lse[~empty]).max()):.2f} of the bound"
    assert (o[empty.transpose(1, 2)] == 0).all(), what
