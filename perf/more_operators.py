"""The layers of a target that no draft's lists prune, over packed batches: what a serving program asks of them.

Every case is one call, or the calls that belong together, at one shape (`op`):

  prompt  causal attention over whole prompts of different lengths, their rows packed one after the other
  linear  linear attention with a decay for each head: packed prompts, single tokens, verification blocks that are then
          committed as far as they were accepted

`own` false: elementary torch operations in 32 bits (decays are summed in 64). `own` true: the framework's calls.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"

# layer shapes (query heads, KV heads, head size): 8B- and 70B-shaped, a draft layer, and layers without grouped heads
SHAPES = {"8b": (32, 8, 128), "70b": (64, 8, 128), "draft": (32, 8, 64), "even": (32, 32, 128), "small": (16, 16, 64)}
# of a drawn case: no more than the largest listed cases ask for
MOST_BYTES, MOST_FLOPS = 6.0e8, 2.1e12


def listed():
    return [
        # One short prompt: the smallest call, where latency counts.
        {"name": "prompt-100", "op": "prompt", "shape": "8b", "B": 1, "lo": 100, "hi": 100, "empty": False, "fused": False},
        # Eight prompts that came in together, 33 to 2049 tokens, K and V as slices of one projection's output.
        {"name": "prompt-b8-mixed", "op": "prompt", "shape": "8b", "B": 8, "lo": 33, "hi": 2049, "empty": False, "fused": True},
        # One prompt of 8192 tokens.
        {"name": "prompt-8k", "op": "prompt", "shape": "8b", "B": 1, "lo": 8192, "hi": 8192, "empty": False, "fused": False},
        # 70B-shaped, three prompts and a place of the batch without one.
        {"name": "prompt-70b-b4", "op": "prompt", "shape": "70b", "B": 4, "lo": 999, "hi": 4001, "empty": True, "fused": False},
        # Draft layer (head size 64), sixteen prompts.
        {"name": "prompt-draft-b16", "op": "prompt", "shape": "draft", "B": 16, "lo": 100, "hi": 4000, "empty": False, "fused": True},
        # A document of 16000 tokens: the largest.
        {"name": "prompt-16k", "op": "prompt", "shape": "8b", "B": 1, "lo": 16000, "hi": 16000, "empty": False, "fused": False},
        # One token of one sequence.
        {"name": "linear-token-b1", "op": "linear", "shape": "8b", "B": 1, "Tq": 1, "gates": False, "carried": True, "accepted": False},
        # Decoding of 64 sequences, decays that depend on the token.
        {"name": "linear-token-b64", "op": "linear", "shape": "even", "B": 64, "Tq": 1, "gates": True, "carried": True, "accepted": False},
        # A verification step of eight sequences: five rows each from the kept states, then the accepted rows into new ones.
        {"name": "linear-verify-b8", "op": "linear", "shape": "8b", "B": 8, "Tq": 5, "gates": True, "carried": True, "accepted": True},
        # One prompt of 8192 tokens, no grouped heads, decays that depend on the token.
        {"name": "linear-prompt-8k", "op": "linear", "shape": "even", "B": 1, "Tq": 0, "lo": 8192, "hi": 8192, "empty": False, "gates": True, "carried": False, "fused": False},
        # Chunks of six prompts behind what is there of them already, grouped heads, one decay per head.
        {"name": "linear-prompts-b6", "op": "linear", "shape": "8b", "B": 6, "Tq": 0, "lo": 77, "hi": 6001, "empty": False, "gates": False, "carried": True, "fused": True},
        # Sixteen prompts through a small layer (head size 64).
        {"name": "linear-small-b16", "op": "linear", "shape": "small", "B": 16, "Tq": 0, "lo": 500, "hi": 4000, "empty": False, "gates": True, "carried": False, "fused": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["prompt", "linear"])
        c = {"op": op, "shape": rng.choice(["8b", "8b", "70b", "draft"] if op == "prompt" else ["8b", "even", "even", "draft", "small"])}
        if op == "linear":
            c.update(gates=rng.random() < 0.5, carried=rng.random() < 0.6)
        if op == "linear" and rng.random() < 0.5:
            c.update(B=_log(rng, 1, 100), Tq=rng.choice([1, 1, rng.randint(2, 16)]))
            c["accepted"] = c["Tq"] > 1 and rng.random() < 0.5
        else:
            if op == "linear":
                c["Tq"] = 0
            hi = _log(rng, 20, 20000)
            c.update(B=rng.choice([1, 1, 2, 3, 5, 8, 13, 20]), lo=max(1, int(hi * rng.uniform(0.02, 1.0))), hi=hi, empty=rng.random() < 0.2, fused=rng.random() < 0.5)
            c["empty"] = c["empty"] and c["B"] > 1
        w = work(c)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return c


def _lengths(c):
    """The lengths of a case's sequences: from `lo` to `hi` in equal ratios, in a mixed order; one of them empty if asked for."""
    B = c["B"]
    if c.get("Tq"):
        return [c["Tq"]] * B
    n = [int(round(c["lo"] * (c["hi"] / c["lo"]) ** (i / max(1, B - 1)))) if B > 1 else c["hi"] for i in range(B)]
    step = next(s for s in range(max(1, B // 2) + 1, 2 * B + 2) if math.gcd(s, B) == 1)
    n = [n[(B - 1 + i * step) % B] for i in range(B)]
    if c["empty"]:
        n[B // 2] = 0
    return n


# ------------------------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(g, *shape, std):
    """Normal bf16 values; the channels of a layer are of different sizes."""
    x = torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)
    x *= std * (0.5 + torch.rand(shape[-1], generator=g, device=DEV))
    return x.to(torch.bfloat16)


def prepare(c, seed):
    g = _gen(seed)
    Hq, Hkv, d = SHAPES[c["shape"]]
    n = _lengths(c)
    B, T = c["B"], sum(n)
    s = {"c": c, "n": n, "scale": 1.0 / math.sqrt(d)}
    # where the sequences begin, on the host for the plain form's loops and on the GPU for the calls
    s["at"] = [sum(n[:b]) for b in range(B + 1)]
    s["starts"] = torch.tensor(s["at"], dtype=torch.int32, device=DEV)
    if c.get("fused"):
        kv = _rows(g, T, 2, Hkv, d, std=0.5)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
    else:
        s["k"], s["v"] = _rows(g, T, Hkv, d, std=0.5), _rows(g, T, Hkv, d, std=0.5)
    s["q"] = torch.randn(T, Hq, d, generator=g, device=DEV).to(torch.bfloat16)
    if c["op"] == "prompt":
        return s
    # natural logarithms of the decays: of heads that forget within some 30 to 4000 tokens, or gates of every token
    if c["gates"]:
        x = 2.0 + 2.0 * torch.randn(T, Hkv, generator=g, device=DEV)
        s["decay"] = -torch.log1p(torch.exp(-x)) / 8.0
    else:
        s["decay"] = torch.log1p(-torch.exp2(-5.0 - 7.0 * torch.rand(Hkv, generator=g, device=DEV)))
    s["state"] = s["slots"] = s["lens"] = None
    if c["carried"]:
        # a pool of states; the sequences' lie anywhere in it
        s["state"] = 2.0 * torch.randn(B + 3, Hkv, d, d, generator=g, device=DEV)
        s["slots"] = torch.randperm(B + 3, generator=g, device=DEV)[:B].to(torch.int32)
    if c.get("accepted"):
        s["lens"] = torch.randint(1, c["Tq"] + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    s["state_out"] = torch.empty(B, Hkv, d, d, dtype=torch.float32, device=DEV)
    if c["Tq"]:
        s["rows"] = {k: s[k].view(B, c["Tq"], *s[k].shape[1:]) for k in ("q", "k", "v")}
        s["rows"]["decay"] = s["decay"].view(B, c["Tq"], Hkv) if c["gates"] else s["decay"]
    return s


# --------------------------------------------------------------------------- the plain forms

def _plain_prompt(s):
    q, k, v = s["q"], s["k"], s["v"]
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    out, lse = torch.empty_like(q), torch.empty(Hq, T, dtype=torch.float32, device=DEV)
    for b, L in enumerate(s["n"]):
        if L == 0:
            continue
        r0 = s["at"][b]
        K = k[r0:r0 + L].float().transpose(0, 1).contiguous()                          # [Hkv, L, d]
        V = v[r0:r0 + L].float().transpose(0, 1).contiguous()
        step = max(64, (1 << 28) // (Hq * L))                                          # rows at a time: 1 GB of scores
        for i in range(0, L, step):
            m = min(step, L - i)
            Q = q[r0 + i:r0 + i + m].float().view(m, Hkv, G, d).permute(1, 2, 0, 3).reshape(Hkv, G * m, d)
            x = torch.matmul(Q, K[:, : i + m].transpose(1, 2)).mul_(s["scale"]).view(Hkv, G, m, i + m)
            later = torch.arange(i + m, device=DEV)[None, :] > torch.arange(i, i + m, device=DEV)[:, None]
            x.masked_fill_(later, float("-inf"))
            top = x.amax(-1, keepdim=True)
            p = x.sub_(top).exp_()
            z = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(Hkv, G * m, i + m), V[:, : i + m]).view(Hkv, G, m, d) / z
            out[r0 + i:r0 + i + m] = o.permute(2, 0, 1, 3).reshape(m, Hq, d).to(torch.bfloat16)
            lse[:, r0 + i:r0 + i + m] = (top + torch.log(z)).view(Hq, m)
    return out, lse


def _first_states(s):
    B, (Hq, Hkv, d) = s["c"]["B"], SHAPES[s["c"]["shape"]]
    if s["state"] is None:
        return torch.zeros(B, Hkv, d, d, dtype=torch.float32, device=DEV)
    return s["state"][s["slots"].long()]


def _plain_linear_rows(s):
    """Token by token: single tokens and short blocks."""
    c, r = s["c"], s["rows"]
    Hq, Hkv, d = SHAPES[c["shape"]]
    B, Tq, G = c["B"], c["Tq"], Hq // Hkv
    S = _first_states(s)
    q, k, v = r["q"].float().view(B, Tq, Hkv, G, d), r["k"].float(), r["v"].float()
    f = torch.exp(r["decay"].view(B, Tq, Hkv) if c["gates"] else r["decay"].expand(B, Tq, Hkv))
    out = []
    kept = S
    for i in range(Tq):
        S = S * f[:, i, :, None, None] + k[:, i, :, :, None] * v[:, i, :, None, :]
        out.append(torch.matmul(q[:, i], S) * s["scale"])                              # [B, Hkv, G, d]
        if s["lens"] is not None:
            kept = torch.where((s["lens"] > i)[:, None, None, None], S, kept)
    out = torch.stack(out, 1).reshape(B, Tq, Hq, d).to(torch.bfloat16)
    s["state_out"].copy_(S if s["lens"] is None else kept)
    return out, s["state_out"]


def _plain_linear_prompts(s):
    """256 rows at a time: what the state before them gives, what they give each other, and the state behind them."""
    c = s["c"]
    Hq, Hkv, d = SHAPES[c["shape"]]
    G, T, C = Hq // Hkv, s["q"].shape[0], 256
    states = _first_states(s)
    out = torch.empty(T, Hq, d, dtype=torch.bfloat16, device=DEV)
    for b, L in enumerate(s["n"]):
        S = states[b]                                                                  # [Hkv, d, d]
        for i in range(0, L, C):
            m = min(C, L - i)
            at = slice(s["at"][b] + i, s["at"][b] + i + m)
            Q = s["q"][at].float().view(m, Hkv, G, d).permute(1, 2, 0, 3)              # [Hkv, G, m, d]
            K, V = s["k"][at].float().transpose(0, 1), s["v"][at].float().transpose(0, 1)
            g = (s["decay"][at] if c["gates"] else s["decay"].expand(m, Hkv)).double().cumsum(0).t()      # [Hkv, m]
            far = torch.exp(g).float()
            near = torch.exp(g[:, :, None] - g[:, None, :]).float().tril()
            w = torch.matmul(Q.reshape(Hkv, G * m, d), K.transpose(1, 2)).view(Hkv, G, m, m) * near[:, None]
            o = torch.matmul(w.view(Hkv, G * m, m), V) + torch.matmul((Q * far[:, None, :, None]).reshape(Hkv, G * m, d), S)
            out[at] = (o.view(Hkv, G, m, d) * s["scale"]).permute(2, 0, 1, 3).reshape(m, Hq, d).to(torch.bfloat16)
            left = torch.exp(g[:, -1:] - g).float()
            S = S * far[:, -1, None, None] + torch.matmul((K * left[:, :, None]).transpose(1, 2), V)
        s["state_out"][b] = S
    return out, s["state_out"]


# --------------------------------------------------------------------------------- the calls

def _framework(s):
    import paper_2605_15508_amd as sts

    c = s["c"]
    if "calls" not in s:      # a serving loop builds its calls on its buffers once
        if c["op"] == "prompt":
            s["calls"] = [sts.sts_prompt_attn(s["q"], s["k"], s["v"], s["starts"], s["scale"], prepare=True)]
        elif not c["Tq"]:
            s["calls"] = [sts.sts_linear_attn(s["q"], s["k"], s["v"], s["decay"], s["scale"], starts=s["starts"], max_len=max(s["n"]), state=s["state"], slots=s["slots"],
                                              state_out=s["state_out"], prepare=True)]
        else:
            r = s["rows"]
            from_state = {"state": s["state"], "slots": s["slots"], "prepare": True}
            if s["lens"] is None:
                s["calls"] = [sts.sts_linear_attn(r["q"], r["k"], r["v"], r["decay"], s["scale"], state_out=s["state_out"], **from_state)]
            else:             # the block's results; then the states behind the rows that were accepted
                s["calls"] = [sts.sts_linear_attn(r["q"], r["k"], r["v"], r["decay"], s["scale"], **from_state),
                              sts.sts_linear_attn(None, r["k"], r["v"], r["decay"], s["scale"], lens=s["lens"], state_out=s["state_out"], **from_state)]
    first = s["calls"][0]()
    if c["op"] == "prompt":
        return first
    for call in s["calls"][1:]:
        call()
    return first[0], s["state_out"]


def run(s):
    if own:
        return _framework(s)
    if s["c"]["op"] == "prompt":
        return _plain_prompt(s)
    return _plain_linear_rows(s) if s["c"]["Tq"] else _plain_linear_prompts(s)


# ------------------------------------------------------------------------------ what it takes

def work(c):
    Hq, Hkv, d = SHAPES[c["shape"]]
    n = _lengths(c)
    T = sum(n)
    rows = T * (2 * Hq + 2 * Hkv) * d * 2                                              # q, k, v, out
    if c["op"] == "prompt":
        return {"bytes": rows + 4 * Hq * T, "flops": sum(L * (L + 1) // 2 for L in n) * Hq * 4 * d}
    states = c["B"] * Hkv * d * d * 4 * (2 if c["carried"] else 1)
    # a row's product with the state, and the state's update: a product by the decay, one and a sum for k and v
    return {"bytes": rows + states + (4 * T * Hkv if c["gates"] else 4 * Hkv), "flops": T * (2 * Hq + 3 * Hkv) * d * d}


# --------------------------------------------------------------------- the definition, 64 bits

def exact(c, seed):
    s = prepare(c, seed)
    Hq, Hkv, d = SHAPES[c["shape"]]
    T, G = s["q"].shape[0], Hq // Hkv
    if c["op"] == "prompt":
        out = torch.zeros(T, Hq, d, dtype=torch.float64, device=DEV)
        lse = torch.zeros(Hq, T, dtype=torch.float64, device=DEV)
        for b, L in enumerate(s["n"]):
            a = s["at"][b]
            for h in range(Hq if L else 0):
                K, V = s["k"][a:a + L, h // G].double(), s["v"][a:a + L, h // G].double()
                for i in range(0, L, 4096):
                    e = min(L, i + 4096)
                    w = s["q"][a + i:a + e, h].double() @ K[:e].T / math.sqrt(d)
                    w = w + torch.full_like(w, float("-inf")).triu(i + 1)
                    z = torch.logsumexp(w, -1)
                    lse[h, a + i:a + e] = z
                    out[a + i:a + e, h] = torch.exp(w - z[:, None]) @ V[:e]
        return out, lse
    # the recurrence itself
    out = torch.zeros(T, Hq, d, dtype=torch.float64, device=DEV)
    states = torch.zeros(c["B"], Hkv, d, d, dtype=torch.float64, device=DEV)
    f = torch.exp(s["decay"].double())
    for b, L in enumerate(s["n"]):
        S = torch.zeros(Hkv, d, d, dtype=torch.float64, device=DEV) if s["state"] is None else s["state"][int(s["slots"][b])].double()
        keep = L if s["lens"] is None else int(s["lens"][b])
        a = s["at"][b]
        q, k, v = (s[t][a:a + L].double() for t in ("q", "k", "v"))
        if keep == 0 or L == 0:
            states[b] = S
        for i in range(L):
            S = torch.baddbmm(S * (f[a + i] if c["gates"] else f).view(Hkv, 1, 1), k[i].unsqueeze(2), v[i].unsqueeze(1))
            out[a + i] = torch.bmm(q[i].view(Hkv, G, d), S).view(Hq, d) / math.sqrt(d)
            if i + 1 == keep:
                states[b] = S
    return out, states
