"""The operators around a cache that is kept small: what a serving program asks of them.

Every case is one call, or the calls that belong together, at one shape (`op`):

  store   rows of K and V go into the 4-bit cache, and are read back as the bf16 values that the cache
          holds for them
  load    every row of a 4-bit cache as bf16 values
  attn4   verification attention over the 4-bit cache: all tokens, or index lists
  window  attention with a sliding window and a few first tokens that stay visible, bf16 cache: single
          tokens, verification blocks, chunks of a prompt

The 4-bit cache: per token and KV head d/2 bytes of codes for K, then for V (two to a byte, the even
channel in the low half; a sign bit and one of 0 0.5 1 1.5 2 3 4 6), and one byte per 32 channels for the
power of two that they are multiplied by.

`own` false: elementary torch operations in 32 bits. `own` true: the framework's calls.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"

# target layer shapes (query heads, KV heads, head size): 8B- and 70B-shaped, and a draft layer
SHAPES = {"8b": (32, 8, 128), "70b": (64, 8, 128), "draft": (32, 8, 64)}
# of a drawn case: no more than the largest listed cases ask for
MOST_BYTES, MOST_FLOPS = 5.7e8, 1.3e11
MOST_PAIRS = 2.1e9       # (query row, key) pairs that the plain form of `window` writes down


def listed():
    return [
        # A verification step appends five tokens to each of four sequences: launches and latency.
        {"name": "store-step-b4", "op": "store", "shape": "8b", "B": 4, "T": 5, "N": 4096, "page": 0, "padded": False},
        # A chunk of 8191 prompt tokens of two sequences, the second shorter, into a pool of pages.
        {"name": "store-chunk-paged", "op": "store", "shape": "8b", "B": 2, "T": 8191, "N": 20000, "page": 16, "padded": True},
        # A sequence of 100003 tokens leaves the 4-bit cache for a bf16 one.
        {"name": "load-100k", "op": "load", "shape": "8b", "B": 1, "N": 100003, "page": 0},
        # One token of one sequence at 4K of context: the smallest attention call.
        {"name": "attn4-decode-4k", "op": "attn4", "shape": "8b", "B": 1, "N": 4096, "Tq": 1, "k": 0, "page": 1, "paged": False, "tail": False, "ragged": False},
        # A layer that is not pruned, 128K of context, batch 4, the block's own candidates appended.
        {"name": "attn4-dense-128k-b4", "op": "attn4", "shape": "8b", "B": 4, "N": 131072, "Tq": 5, "k": 0, "page": 1, "paged": False, "tail": True, "ragged": False},
        # The benchmark's headline over a 4-bit cache: 10% of 128K, batch 4, a list per draft head.
        {"name": "attn4-lists-128k-b4", "op": "attn4", "shape": "8b", "B": 4, "N": 131072, "Tq": 5, "k": 13108, "page": 1, "paged": False, "tail": True, "ragged": False},
        # 70B-shaped, eight candidates, three sequences of different lengths in a pool of pages.
        {"name": "attn4-70b-paged", "op": "attn4", "shape": "70b", "B": 3, "N": 50003, "Tq": 8, "k": 0, "page": 16, "paged": True, "tail": False, "ragged": True},
        # Decoding of 16 sequences, one token each, window of 4096 behind 4 sinks, lengths up to 32K.
        {"name": "window-decode-b16", "op": "window", "shape": "8b", "B": 16, "N": 32768, "Tq": 1, "window": 4096, "sinks": 4, "page": 0, "tail": False, "ragged": True},
        # A verification block of one sequence, its own candidates not in the (paged) cache yet.
        {"name": "window-verify-paged", "op": "window", "shape": "8b", "B": 1, "N": 8193, "Tq": 5, "window": 1024, "sinks": 4, "page": 16, "tail": True, "ragged": False},
        # A prompt of 8192 tokens at once, window of 1024.
        {"name": "window-prompt-8k", "op": "window", "shape": "8b", "B": 1, "N": 8192, "Tq": 8192, "window": 1024, "sinks": 4, "page": 0, "tail": False, "ragged": False},
        # A chunk of 1999 tokens at the end of a 33001-token context, window of 4096.
        {"name": "window-chunk-33k", "op": "window", "shape": "8b", "B": 1, "N": 33001, "Tq": 1999, "window": 4096, "sinks": 4, "page": 0, "tail": False, "ragged": False},
        # Draft layer (head size 64), two prompts of different lengths in a padded batch.
        {"name": "window-draft-4k", "op": "window", "shape": "draft", "B": 2, "N": 4096, "Tq": 4000, "window": 512, "sinks": 16, "page": 0, "tail": False, "ragged": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["store", "load", "attn4", "attn4", "attn4", "window", "window", "window", "window"])
        shape = rng.choice(["8b", "8b", "70b", "draft"])
        B = rng.choice([1, 1, 2, 3, 4, 7, 8])
        c = {"op": op, "shape": shape, "B": B}
        if op == "store":
            T = _log(rng, 1, 16000)
            c.update(T=T, N=T + rng.randint(0, 20000), page=rng.choice([0, 0, 8, 16, 32]), padded=rng.random() < 0.5)
        elif op == "load":
            c.update(N=_log(rng, 100, 200000), page=rng.choice([0, 0, 8, 16, 32]))
        elif op == "attn4":
            N = _log(rng, 100, 300000)
            lists = rng.random() < 0.5
            paged = rng.random() < 0.4
            page = rng.choice([8, 16, 32]) if paged or (lists and rng.random() < 0.3) else 1
            blocks = -(-N // page)
            k = max(1, min(blocks, int(blocks * rng.uniform(0.02, 0.25)))) if lists else 0
            c.update(N=N, Tq=rng.randint(1, 9), k=k, page=page, paged=paged, tail=rng.random() < 0.5, ragged=not lists and rng.random() < 0.5)
        else:
            tail = False
            if rng.random() < 0.5:
                Tq, tail = rng.randint(1, 9), rng.random() < 0.5
                N = _log(rng, 100, 100000)
            else:
                Tq = _log(rng, 20, 8000)
                N = Tq + (0 if rng.random() < 0.5 else rng.randint(0, 30000))
            c.update(N=N, Tq=Tq, window=_log(rng, 64, 5000), sinks=rng.choice([0, 1, 4, 16, 100]), page=rng.choice([0, 0, 16, 32]), tail=tail,
                     ragged=rng.random() < 0.5)
        w = work(c)
        Hq = SHAPES[shape][0]
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS and (op != "window" or B * Hq * c["Tq"] * c["N"] <= MOST_PAIRS):
            return c


# ------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(g, *shape, std):
    """Normal bf16 values; keys and values of one layer have channels of different sizes."""
    x = torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)
    x *= std * (0.5 + torch.rand(shape[-1], generator=g, device=DEV))
    return x.to(torch.bfloat16)


def _pages(g, B, N, page):
    """A page table over a pool in random order, with some pages that belong to nobody."""
    per = -(-N // page)
    total = B * per + 7
    return torch.randperm(total, generator=g, device=DEV)[: B * per].to(torch.int32).view(B, per), total


def _lens(g, B, lo, hi):
    return torch.randint(lo, hi + 1, (B,), generator=g, device=DEV, dtype=torch.int32)


def prepare(c, seed):
    g = _gen(seed)
    Hq, Hkv, d = SHAPES[c["shape"]]
    B, N, op = c["B"], c["N"], c["op"]
    paged = c["paged"] if op == "attn4" else c["page"] > 0
    s = {"c": c, "table": None, "lens": None, "pos": None, "k_new": None, "v_new": None, "idx": None, "cnt": None, "head_map": None}
    room, slots = B, N
    if paged:
        s["table"], room = _pages(g, B, N, c["page"])
        slots = c["page"]
    if op == "window":
        s["k"] = _rows(g, room, Hkv, slots, d, std=0.5)
        s["v"] = _rows(g, room, Hkv, slots, d, std=0.5)
    elif op == "store":
        s["codes"] = torch.zeros(room, Hkv, slots, 2, d // 2, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.zeros(room, Hkv, slots, 2, d // 32, dtype=torch.uint8, device=DEV)
        s["k"] = _rows(g, B, c["T"], Hkv, d, std=0.5)
        s["v"] = _rows(g, B, c["T"], Hkv, d, std=0.5)
        s["pos"] = _lens(g, B, 0, N - c["T"])
        if c["padded"]:
            s["lens"] = _lens(g, B, c["T"] // 2, c["T"])
        s["k_out"] = torch.zeros_like(s["k"])
        s["v_out"] = torch.zeros_like(s["v"])
    else:
        # a cache that is there already: rows quantised as the store does it
        s["codes"] = torch.empty(room, Hkv, slots, 2, d // 2, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty(room, Hkv, slots, 2, d // 32, dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 26) // (Hkv * slots * d)) if paged else 1
        for i in range(0, room, step):
            for j in range(2):
                x = _rows(g, min(step, room - i), Hkv, slots, d, std=0.5)
                s["codes"][i:i + step, :, :, j], s["scales"][i:i + step, :, :, j] = _to_codes(x)
    if op in ("attn4", "window"):
        Tq = c["Tq"]
        s["q"] = torch.randn(B, Tq, Hq, d, generator=g, device=DEV).to(torch.bfloat16)
        s["scale"] = 1.0 / math.sqrt(d)
        if c["ragged"]:
            s["lens"] = _lens(g, B, N // 2, N)
        if c["tail"]:
            s["k_new"] = _rows(g, B, Tq, Hkv, d, std=0.5)
            s["v_new"] = _rows(g, B, Tq, Hkv, d, std=0.5)
    if op == "attn4" and c["k"]:
        # two neighbouring query heads are mapped to one draft head and share its list
        Hd, blocks = Hq // 2, -(-N // c["page"])
        lists = torch.rand(B, Hd, blocks, generator=g, device=DEV).topk(c["k"], dim=-1).indices.sort(dim=-1).values
        s["idx"] = lists.repeat_interleave(2, dim=1).to(torch.int32).contiguous()
        s["cnt"] = torch.full((B, Hq), c["k"], dtype=torch.int32, device=DEV)
        s["head_map"] = [t // 2 for t in range(Hq)]
    return s


# --------------------------------------------------------------------------- the plain forms

def _to_codes(x):
    """bf16 [..., d] -> codes [..., d/2], scales [..., d/32] (uint8)."""
    y = x.float().unflatten(-1, (-1, 32))
    a = y.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(a)                          # a = m * 2^e, m in [0.5, 1)
    e = torch.where(a > 0, e - 3 + (m > 0.875).to(torch.int32), torch.full_like(e, -125)).clamp(-125, 125)
    bad = ~torch.isfinite(a)
    y = torch.ldexp(y, -e)
    z = y.abs()
    code = ((z > 0.25).to(torch.uint8) + (z >= 0.75) + (z > 1.25) + (z >= 1.75) + (z > 2.5) + (z >= 3.5) + (z > 5.0)).to(torch.uint8)
    code = torch.where(bad, torch.zeros_like(code), code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2)
    scale = torch.where(bad, torch.full_like(e, 255), e + 127).squeeze(-1).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def _from_codes(codes, scales):
    """The fp32 values [..., d] of codes [..., d/2] and scales [..., d/32]."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    powers = torch.exp2(torch.arange(256, device=codes.device, dtype=torch.float64) - 127).float()
    powers[255] = float("nan")
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1).flatten(-2)
    return (v.unflatten(-1, (-1, 32)) * powers[scales.int()].unsqueeze(-1)).flatten(-2)


def _token_rows(s, first, count):
    """Places of tokens first_b .. first_b + count - 1 of every sequence: (batch element or page, slot), each [B, count]."""
    B, page = s["c"]["B"], s["c"]["page"]
    n = torch.arange(count, device=DEV)[None, :] + (first[:, None] if first is not None else torch.zeros(B, 1, dtype=torch.int64, device=DEV))
    if s["table"] is None:
        return torch.arange(B, device=DEV)[:, None].expand_as(n), n
    return torch.gather(s["table"].long(), 1, n.long() // page), n % page


def _whole(s, x):
    """A cache tensor as [B, Hkv, N, ...], its pages in the sequences' order."""
    if s["table"] is None:
        return x
    y = x[s["table"].long()]                                  # [B, pages, Hkv, page, ...]
    return y.transpose(1, 2).flatten(2, 3)[:, :, : s["c"]["N"]]


def _plain_store(s):
    T = s["c"]["T"]
    where, slot = _token_rows(s, s["pos"], T)
    live = torch.ones_like(slot, dtype=torch.bool) if s["lens"] is None else torch.arange(T, device=DEV)[None, :] < s["lens"][:, None]
    w, t = where[live].long(), slot[live].long()
    k, v = s["k"][live], s["v"][live]                         # [tokens, Hkv, d]
    (kc, ks), (vc, vs) = _to_codes(k), _to_codes(v)
    s["codes"][w, :, t] = torch.stack((kc, vc), -2)
    s["scales"][w, :, t] = torch.stack((ks, vs), -2)
    back = _from_codes(s["codes"][w, :, t], s["scales"][w, :, t])
    s["k_out"][live] = back[..., 0, :].to(torch.bfloat16)
    s["v_out"][live] = back[..., 1, :].to(torch.bfloat16)
    return s["k_out"], s["v_out"]


def _plain_load(s):
    x = _from_codes(_whole(s, s["codes"]), _whole(s, s["scales"])).to(torch.bfloat16).transpose(1, 2)
    return x[..., 0, :].contiguous(), x[..., 1, :].contiguous()


def _times(p, x):
    """p [B,Hkv,G,Tq,n] times x [B,Hkv,G or 1,n,m]."""
    if x.shape[2] != 1:
        return torch.matmul(p, x)
    return torch.matmul(p.flatten(2, 3), x.squeeze(2)).unflatten(2, p.shape[2:4])


def _softmax_out(x, v):
    """Scores x [..., rows, keys] (-inf where a key is not visible) and values -> out [..., rows, d], lse [..., rows]."""
    m = x.amax(-1, keepdim=True)
    m0 = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = x.sub_(m0).exp_()
    z = p.sum(-1, keepdim=True)
    out = _times(p, v) / torch.where(z > 0, z, torch.ones_like(z))
    return out, (m0 + torch.log(z)).squeeze(-1)


def _with_tail(s, x, v, q):
    """The block's own keys, causally behind the cached ones: scores [B,Hkv,G,Tq,n] and values [B,Hkv,1,n,d]."""
    if s["k_new"] is None:
        return x, v
    Tq = q.shape[3]
    kn, vn = (s[t].float().permute(0, 2, 1, 3).unsqueeze(2) for t in ("k_new", "v_new"))
    xn = _times(q, kn.transpose(-1, -2)) * s["scale"]
    later = torch.arange(Tq, device=DEV)[None, :] > torch.arange(Tq, device=DEV)[:, None]
    return torch.cat((x, xn.masked_fill(later, float("-inf"))), -1), torch.cat((v, vn.expand(*v.shape[:3], *vn.shape[3:])), 3)


def _heads(s, Hkv):
    """q as [B, Hkv, G, Tq, d] in 32 bits."""
    q = s["q"].float()
    B, Tq, Hq, d = q.shape
    return q.view(B, Tq, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4)


def _back(out, lse):
    B, Hkv, G, Tq, d = out.shape
    return out.permute(0, 3, 1, 2, 4).reshape(B, Tq, Hkv * G, d).to(torch.bfloat16), lse.reshape(B, Hkv * G, Tq)


def _plain_attn4(s):
    c = s["c"]
    N, page = c["N"], c["page"]
    codes, scales = _whole(s, s["codes"]), _whole(s, s["scales"])
    Hkv = codes.shape[1]
    q = _heads(s, Hkv)
    if s["idx"] is None:
        kv = _from_codes(codes, scales)
        k, v = kv[..., 0, :].unsqueeze(2), kv[..., 1, :].unsqueeze(2)          # [B,Hkv,1,N,d]
        hidden = None if s["lens"] is None else torch.arange(N, device=DEV)[None, :] >= s["lens"][:, None]
        hidden = None if hidden is None else hidden[:, None, None, None, :]
    else:
        B, Hq, kk = s["idx"].shape
        tok = (s["idx"].long()[..., None] * page + torch.arange(page, device=DEV)).flatten(2)
        hidden = (tok >= N).view(B, Hkv, Hq // Hkv, 1, -1)
        tok = tok.clamp(max=N - 1).view(B, Hkv, -1)
        bb, hh = torch.arange(B, device=DEV)[:, None, None], torch.arange(Hkv, device=DEV)[None, :, None]
        kv = _from_codes(codes[bb, hh, tok], scales[bb, hh, tok]).unflatten(2, (Hq // Hkv, -1))
        k, v = kv[..., 0, :], kv[..., 1, :]                                    # [B,Hkv,G,k,d]
    x = _times(q, k.transpose(-1, -2)).mul_(s["scale"])
    if hidden is not None:
        x.masked_fill_(hidden, float("-inf"))
    x, v = _with_tail(s, x, v, q)
    return _back(*_softmax_out(x, v))


def _plain_window(s):
    c = s["c"]
    N, Tq = c["N"], c["Tq"]
    k, v = _whole(s, s["k"]).float().unsqueeze(2), _whole(s, s["v"]).float().unsqueeze(2)
    q = _heads(s, k.shape[1])
    lens = s["lens"] if s["lens"] is not None else torch.full((c["B"],), N, dtype=torch.int32, device=DEV)
    p = lens[:, None] - (0 if c["tail"] else Tq) + torch.arange(Tq, device=DEV)[None, :]            # [B, Tq]
    n = torch.arange(N, device=DEV)
    seen = (n <= p[..., None]) & ((n < c["sinks"]) | (n > p[..., None] - c["window"])) & (n < lens[:, None, None])
    x = _times(q, k.transpose(-1, -2)).mul_(s["scale"]).masked_fill_(~seen[:, None, None], float("-inf"))
    x, v = _with_tail(s, x, v, q)
    return _back(*_softmax_out(x, v))


# --------------------------------------------------------------------------------- the calls

def _framework(s):
    import paper_2605_15508_amd as sts

    c = s["c"]
    op = c["op"]
    where = {"page_size": max(1, c["page"]), "block_table": s["table"], "N": c["N"]}
    if op == "store":
        sts.sts_packed_store(s["k"], s["v"], s["codes"], s["scales"], pos=s["pos"], lens=s["lens"], **where)
        return sts.sts_packed_load(s["codes"], s["scales"], c["T"], pos=s["pos"], lens=s["lens"], out=(s["k_out"], s["v_out"]), **where)
    if op == "load":
        return sts.sts_packed_load(s["codes"], s["scales"], c["N"], **where)
    if "call" not in s:      # a serving loop builds the call on its buffers once
        new = {"seq_lens": s["lens"], "k_new": s["k_new"], "v_new": s["v_new"], "prepare": True, **where}
        if op == "attn4":
            s["call"] = sts.sts_packed_attn(s["q"], s["codes"], s["scales"], s["scale"], indices=s["idx"], counts=s["cnt"], head_map=s["head_map"], **new)
        else:
            s["call"] = sts.sts_window_attn(s["q"], s["k"], s["v"], s["scale"], c["window"], sinks=c["sinks"], **new)
    return s["call"]()


def run(s):
    if own:
        return _framework(s)
    return {"store": _plain_store, "load": _plain_load, "attn4": _plain_attn4, "window": _plain_window}[s["c"]["op"]](s)


# ------------------------------------------------------------------------------ what it takes

def work(c):
    Hq, Hkv, d = SHAPES[c["shape"]]
    B, op = c["B"], c["op"]
    row4, row16 = 2 * (d // 2 + d // 32), 4 * d             # bytes of a token's K and V for one KV head
    if op == "store":
        rows = B * c["T"] * Hkv
        return {"bytes": rows * (2 * row16 + 2 * row4), "flops": rows * 2 * d * 4}
    if op == "load":
        rows = B * c["N"] * Hkv
        return {"bytes": rows * (row16 + row4), "flops": rows * 2 * d}
    Tq = c["Tq"]
    ends = B * Tq * Hq * (4 * d + 4) + (B * Tq * Hkv * row16 if c["tail"] else 0)      # q, out, lse, own rows
    if op == "attn4":
        if c["k"]:
            keys = min(c["N"], c["k"] * c["page"])
            lists = B * (Hq // 2) * keys                     # two heads share a list
            return {"bytes": lists * row4 + B * Hq * c["k"] * 4 + ends, "flops": B * Hq * Tq * keys * 4 * d}
        keys = c["N"] if not c["ragged"] else 3 * c["N"] // 4
        return {"bytes": B * Hkv * keys * row4 + ends, "flops": B * Hq * Tq * keys * 4 * d}
    # (query row, key) pairs, the lengths at three quarters of the bound where they vary
    L = c["N"] if not c["ragged"] else 3 * c["N"] // 4
    p0 = L if c["tail"] else L - Tq
    pairs = sum(min(p + 1, c["window"] + c["sinks"]) for p in range(max(p0, 0), p0 + Tq))
    keys = min(L, c["window"] + c["sinks"] + Tq)
    return {"bytes": B * Hkv * keys * row16 + ends, "flops": B * Hq * pairs * 4 * d}


# --------------------------------------------------------------------- the definition, 64 bits

def _values64(codes, scales):
    mag = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)
    out = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=DEV)
    for half in range(2):
        nib = (codes >> (4 * half)) & 15
        out[..., half::2] = mag[(nib & 7).long()] * (1.0 - 2.0 * (nib >> 3).double())
    return out * torch.pow(2.0, scales.double() - 127.0).repeat_interleave(32, dim=-1)


def _quantised64(x):
    x = x.double()
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)
    a = x.unflatten(-1, (-1, 32)).abs().amax(-1).repeat_interleave(32, dim=-1)
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -140)))
    e = (e - 2 + (a > 1.75 * torch.pow(2.0, e)).double()).clamp(-125, 125)
    y = x.abs() / torch.pow(2.0, e)
    dist = (y[..., None] - grid).abs()
    near = dist.amin(-1, keepdim=True)
    even = torch.arange(8, device=DEV) % 2 == 0
    pick = torch.where(dist == near, torch.where(even, 2, 1), 0).argmax(-1)     # the nearest, of two the even one
    return torch.sign(x) * grid[pick] * torch.pow(2.0, e)


def _sequence(s, x, b):
    """Cache tensor x of batch element b as [Hkv, N, ...]."""
    if s["table"] is None:
        return x[b]
    return torch.cat([x[int(p)] for p in s["table"][b].tolist()], dim=1)[:, : s["c"]["N"]]


def exact(c, seed):
    s = prepare(c, seed)
    op, B, N = c["op"], c["B"], c["N"]
    if op == "store":
        k, v = (torch.zeros(*s["k"].shape, dtype=torch.float64, device=DEV) for _ in range(2))
        for b in range(B):
            n = c["T"] if s["lens"] is None else int(s["lens"][b])
            for t in range(0, n, 512):
                k[b, t:min(n, t + 512)] = _quantised64(s["k"][b, t:min(n, t + 512)])
                v[b, t:min(n, t + 512)] = _quantised64(s["v"][b, t:min(n, t + 512)])
        return k, v
    if op == "load":
        both = torch.stack([_values64(_sequence(s, s["codes"], b), _sequence(s, s["scales"], b)) for b in range(B)])
        return both[..., 0, :].transpose(1, 2).contiguous(), both[..., 1, :].transpose(1, 2).contiguous()
    Hq, Hkv, d = SHAPES[c["shape"]]
    Tq, G = c["Tq"], Hq // Hkv
    out = torch.zeros(B, Tq, Hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq, Tq), float("-inf"), dtype=torch.float64, device=DEV)
    for b in range(B):
        L = N if s["lens"] is None else int(s["lens"][b])
        if op == "attn4":
            codes, scales = _sequence(s, s["codes"], b), _sequence(s, s["scales"], b)
        else:
            cached = _sequence(s, s["k"], b), _sequence(s, s["v"], b)
        for h in range(Hq):
            g = h // G
            if op == "attn4":
                rows = torch.arange(L, device=DEV)
                if s["idx"] is not None:
                    rows = torch.cat([rows[e * c["page"]:(e + 1) * c["page"]] for e in s["idx"][b, h].tolist()]) if c["page"] > 1 else s["idx"][b, h].long()
                kv = _values64(codes[g][rows], scales[g][rows])
                K, V = kv[:, 0], kv[:, 1]
                see = torch.ones(Tq, K.shape[0], dtype=torch.bool, device=DEV)
            else:
                at = torch.arange(Tq, device=DEV) + (L if c["tail"] else L - Tq)
                lo = max(0, (L if c["tail"] else L - Tq) - c["window"])
                first = min(c["sinks"], lo)
                rows = torch.cat((torch.arange(first, device=DEV), torch.arange(lo, L, device=DEV)))
                K, V = cached[0][g][rows].double(), cached[1][g][rows].double()
                see = (rows[None, :] <= at[:, None]) & ((rows[None, :] < c["sinks"]) | (at[:, None] - rows[None, :] < c["window"]))
            if c["tail"]:
                K, V = torch.cat((K, s["k_new"][b, :, g].double())), torch.cat((V, s["v_new"][b, :, g].double()))
                see = torch.cat((see, torch.ones(Tq, Tq, dtype=torch.bool, device=DEV).tril()), 1)
            w = (s["q"][b, :, h].double() @ K.T) / math.sqrt(d)
            w = torch.where(see, w, torch.full_like(w, float("-inf")))
            z = torch.logsumexp(w, -1)
            live = torch.isfinite(z)
            out[b, live, h] = torch.exp(w[live] - z[live, None]) @ V
            lse[b, h] = z
    return out, lse
