"""The operators around a small cache at the ends of their numbers, against 64 bits (cache_util.attention)."""
import math

import pytest
import torch

import paper_2605_15508_amd as sts
from cache_util import attention, check, packed_cache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def bf16(*shape, g):
    return torch.randn(*shape, generator=g).to(torch.bfloat16)


def on(t):
    return t.to(DEV) if isinstance(t, torch.Tensor) else t


@pytest.mark.parametrize("low", ["overflow", "infinity"])
@pytest.mark.parametrize("N", [40, 3000])
@pytest.mark.parametrize("op", ["packed", "lists", "window"])
@pytest.mark.parametrize("d", [64, 128])
def test_own_tokens_that_score_below_the_range(d, op, N, low):
    """Nothing cached (a sequence's length, or its lists', is 0), and an own token whose score is -inf in fp32: its weight is 0, whether the workgroup
    that has the unit takes the own tokens in (40 tokens) or the combine kernel (3000)."""
    B, Tq, Hq, Hkv, scale = 2, 5, 4, 2, 0.1
    g = gen(N + d)
    codes, scales, _, k, v = packed_cache(B, Hkv, N, d, g)
    kb, vb = bf16(B, Hkv, N, d, g=g), bf16(B, Hkv, N, d, g=g)
    q, kn, vn = bf16(B, Tq, Hq, d, g=g), bf16(B, Tq, Hkv, d, g=g), bf16(B, Tq, Hkv, d, g=g)
    # in sequence 0, KV head 1: tokens 0 and 3 score -inf with rows 1 .. of one channel, which the others do not have
    q[0, :, :, 7], kn[0, :, :, 7] = 0, 0
    q[0, 1:, 2:, 7] = 1e10
    kn[0, [0, 3], 1, 7] = -3e38 if low == "overflow" else -math.inf
    lens = torch.tensor([0, N], dtype=torch.int32)
    kw = dict(k_new=kn, v_new=vn, out_dtype=torch.float32)
    if op == "window":
        got = sts.sts_window_attn(on(q), on(kb), on(vb), scale, 500, sinks=2, seq_lens=on(lens), **{a: on(t) for a, t in kw.items()})
    else:
        if op == "lists":
            kw.update(indices=torch.arange(N, dtype=torch.int32).expand(B, Hq, N).contiguous(), counts=lens[:, None].expand(B, Hq).contiguous())
        else:
            kw.update(seq_lens=lens)
        got = sts.sts_packed_attn(on(q), on(codes), on(scales), scale, **{a: on(t) for a, t in kw.items()})
    # the definition: those two tokens are as not seen (e^-1e46 of the others); row 0 has no such channel
    own = kn[:1].double()
    own[0, :, :, 7] = 0
    see = [torch.ones(Tq, Tq, dtype=torch.bool).tril() for _ in range(2)]
    see[1][1:, [0, 3]] = False
    ref = attention(q[:1], scale, lambda b, t: (own[0, :, t // 2], vn[0, :, t // 2].double(), see[t // 2]))
    skip = torch.zeros(1, Tq, Hq, dtype=torch.bool)
    skip[:, 0, 2:] = low == "infinity"            # 0 times an infinity
    out, lse = got[0][:1].cpu(), got[1][:1].cpu()
    assert torch.isnan(out[skip]).all()
    out[skip], lse[skip.transpose(1, 2)] = ref[0][skip].float(), ref[1][skip.transpose(1, 2)].float()
    check((out, lse), ref)
    # the sequence beside it
    p = torch.arange(N, N + Tq)[:, None]
    n = torch.arange(N)
    seen = ((n < 2) | (n > p - 500)) if op == "window" else torch.ones(Tq, N, dtype=torch.bool)
    rows = (kb[1].double(), vb[1].double()) if op == "window" else (k[1], v[1])
    ref = attention(q[1:], scale, lambda b, t: (rows[0][t // 2], rows[1][t // 2], seen), kn[1:], vn[1:], q_halves=op != "window")
    check((got[0][1:], got[1][1:]), ref)
