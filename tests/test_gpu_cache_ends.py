"""The operators around a small cache at the ends of their numbers: own tokens that score below the fp32 range, scales at the ends of a byte,
values that are no numbers in pages and in blocks that several workgroups share; against 64 bits (cache_util.attention)."""
import math

import pytest
import torch

import paper_2605_15508_amd as sts
from cache_util import attention, check, packed_cache, table_of, to_pages, values

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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("s", [0, 1, 2, 3, 127, 251, 252])
def test_scale_bytes_are_read_as_they_say(s, d):
    """All codes under every such byte, loaded (exactly) and attended to."""
    g = gen(s)
    B, Hkv, N, Hq, Tq = 1, 2, 90, 4, 3
    codes = torch.randint(0, 256, (B, Hkv, N, 2, d // 2), generator=g, dtype=torch.uint8)
    scales = torch.full((B, Hkv, N, 2, d // 32), s, dtype=torch.uint8)
    k, v = (values(codes[:, :, :, j], scales[:, :, :, j]) for j in range(2))
    for got, want in zip(sts.sts_packed_load(on(codes), on(scales), N), (k, v)):
        assert torch.equal(got.cpu().double(), want.transpose(1, 2))
    # K under the byte, queries that bring the scores back to a few units
    # (no smaller than 2^-113, where they are held to 2^-17 of their group's largest: the rest is the call's scale)
    q = (torch.randn(B, Tq, Hq, d, generator=g) * 2.0 ** (127 - min(max(s, 2), 240))).to(torch.bfloat16)
    scale = 0.05 * 2.0 ** -max(0, s - 240)
    usual = torch.full_like(scales[:, :, :, 1], 126)
    v_usual = values(codes[:, :, :, 1], usual)
    mixed = scales.clone()
    mixed[:, :, :, 1] = usual
    see = torch.ones(Tq, N, dtype=torch.bool)
    check(sts.sts_packed_attn(on(q), on(codes), on(mixed), scale, out_dtype=torch.float32),
          attention(q, scale, lambda b, t: (k[b, t // 2], v_usual[b, t // 2], see), q_halves=True))
    # V under the byte. The sums of weights times values and the result are fp32, whose steps below 2^-126 are 2^-149: a
    # step for every key and one for the last product more than the other bound. Sums of large values may leave fp32: one token of those.
    n = N if s < 200 else 1
    mixed = scales.clone()
    mixed[:, :, :, 0] = 126
    k_usual = values(codes[:, :, :, 0], usual)
    q = bf16(B, Tq, Hq, d, g=g)
    o, _ = sts.sts_packed_attn(on(q), on(codes), on(mixed), 0.05, seq_lens=on(torch.tensor([n], dtype=torch.int32)), out_dtype=torch.float32)
    out, _, bound, _ = attention(q, 0.05, lambda b, t: (k_usual[b, t // 2, :n], v[b, t // 2, :n], see[:, :n]), q_halves=True)
    assert ((o.cpu().double() - out).abs() <= bound + (n + 1) * 2.0 ** -149).all()


def windowed(q, k, v, window, sinks, page, apart=0):
    """sts_window_attn over a contiguous cache, pages, or pages `apart` elements from each other."""
    kw = dict(sinks=sinks, out_dtype=torch.float32)
    if not page:
        return sts.sts_window_attn(on(q), on(k), on(v), 0.1, window, **kw)
    spare = 1 if apart else 3
    kp, vp = (to_pages(t, page, None, spare) for t in (k, v))
    kw.update(page_size=page, N=k.shape[2], block_table=on(table_of(k.shape[0], k.shape[2], page, None, spare)))
    if not apart:
        return sts.sts_window_attn(on(q), on(kp), on(vp), 0.1, window, **kw)
    one = kp[0].numel()
    pool = torch.empty((kp.shape[0] - 1) * apart + 2 * one, dtype=torch.bfloat16, device=DEV)
    far = [pool[j * one:].as_strided(kp.shape, (apart, *kp.stride()[1:])) for j in range(2)]
    try:
        for t, rows in zip(far, (kp, vp)):
            t.copy_(rows)
        return tuple(t.cpu() for t in sts.sts_window_attn(on(q), *far, 0.1, window, **kw))
    finally:
        del far, pool
        torch.cuda.empty_cache()


def odd_values_case(B, Tq, N, window, sinks, spots, bad, d, page, apart=0):
    g = gen(9)
    q, k, v = bf16(B, Tq, 4, d, g=g), bf16(B, 2, N, d, g=g), bf16(B, 2, N, d, g=g)
    p, n = torch.arange(N - Tq, N)[:, None], torch.arange(N)
    see = (n <= p) & ((n < sinks) | (n > p - window))
    clean = v.clone()
    for s in spots:                    # one channel of KV head 0, all of KV head 1
        v[:, 0, s, 3] = bad
        v[:, 1, s] = bad
        clean[:, 0, s, 3] = 0
        clean[:, 1, s] = 0
    unseen = ~see.any(0)
    k[:, :, unseen], v[:, :, unseen] = math.nan, math.nan
    o, l = (t.cpu() for t in windowed(q, k, v, window, sinks, page, apart))
    hit = see[:, spots].any(1)
    assert hit.any() and not hit.all()
    some = see.any(0)
    ref = attention(q, 0.1, lambda b, t: (k[b, t // 2, some].double(), clean[b, t // 2, some].double(), see[:, some]))
    for t in range(4):
        chans = slice(3, 4) if t < 2 else slice(None)
        got = o[:, :, t, chans]
        assert torch.isfinite(got[:, ~hit]).all()
        assert (torch.isnan(got) if math.isnan(bad) else got == bad)[:, hit].all()
        o[:, :, t, chans] = torch.where(hit[:, None], ref[0][:, :, t, chans].float(), got)
    check((o, l), ref)


BAD = [math.nan, math.inf, -math.inf]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("page", [1, 16, 32])
@pytest.mark.parametrize("B,Tq,N,window,sinks,spots", [(1, 5, 300, 70, 3, [100, 227, 299]), (2, 3, 64, 5, 1, [62]), (2, 40, 200, 30, 4, [150, 151, 190]),
                                                       (1, 100, 100, 33, 0, [60, 61])])
def test_values_that_are_no_numbers_in_pages(B, Tq, N, window, sinks, spots, page, bad, d):
    odd_values_case(B, Tq, N, window, sinks, spots, bad, d, page)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("Tq,N,window,sinks,spots", [(40, 2000, 1500, 4, [465, 490]), (40, 2000, 1500, 4, [1985, 1999]), (40, 2000, 1500, 0, [462, 1999, 1971]),
                                                     (5, 4000, 3000, 3, [997, 999]), (5, 4000, 3000, 3, [3998])])
def test_values_that_are_no_numbers_in_blocks_that_several_workgroups_share(Tq, N, window, sinks, spots, page, bad, d):
    odd_values_case(1, Tq, N, window, sinks, spots, bad, d, page)


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("Tq", [5, 40])
def test_values_that_are_no_numbers_in_pages_that_lie_far_apart(Tq, bad):
    """Pages 8 GB apart, head size 128."""
    odd_values_case(1, Tq, 50, 20, 2, [47, 48], bad, 128, 8, apart=2 ** 32)
