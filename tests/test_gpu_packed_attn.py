"""sts_packed_attn: attention over a 4-bit cache against the definition in 64 bits on the values that the cache stands for, within
bounds derived from the roundings (cache_util.attention)."""
import math

import numpy as np
import pytest
import torch

import paper_2605_15508_amd as sts
from cache_util import attention, check, packed_cache, to_pages

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def queries(B, Tq, Hq, d, g, outliers=False):
    q = torch.randn(B, Tq, Hq, d, generator=g)
    if outliers:             # channels of very different sizes
        q = q * torch.exp(2.5 * torch.randn(d, generator=g))
        q = q / q.norm(dim=-1, keepdim=True) * math.sqrt(d)
    return q.to(torch.bfloat16)


def all_tokens(k, v, Hq, Tq, lens=None):
    G = Hq // k.shape[1]

    def keys(b, t):
        n = k.shape[2] if lens is None else max(0, min(int(lens[b]), k.shape[2]))
        return k[b, t // G, :n], v[b, t // G, :n], torch.ones(Tq, n, dtype=torch.bool)
    return keys


def listed(k, v, Hq, Tq, idx, cnt, page=1):
    G, N = Hq // k.shape[1], k.shape[2]

    def keys(b, t):
        e = idx[b, t, : int(cnt[b, t]) if cnt is not None else None].long()
        n = (e[:, None] * page + torch.arange(page)).reshape(-1)
        n = n[n < N]
        return k[b, t // G, n], v[b, t // G, n], torch.ones(Tq, len(n), dtype=torch.bool)
    return keys


def run(q, codes, scales, scale, table=None, **kw):
    kw = {a: x.to(DEV) if isinstance(x, torch.Tensor) else x for a, x in kw.items()}
    return sts.sts_packed_attn(q.to(DEV), codes.to(DEV), scales.to(DEV), scale, block_table=None if table is None else table.to(DEV), **kw)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Tq,Hq,Hkv,N", [(1, 1, 1, 1, 1), (1, 1, 4, 1, 31), (2, 5, 8, 2, 33), (1, 16, 4, 4, 100), (3, 3, 6, 2, 257), (1, 8, 16, 2, 700),
                                           (1, 2, 16, 1, 64), (2, 16, 16, 1, 130), (1, 1, 2, 2, 5000)])
def test_all_tokens(B, Tq, Hq, Hkv, N, d):
    g = gen(N + Tq)
    codes, scales, _, k, v = packed_cache(B, Hkv, N, d, g)
    q = queries(B, Tq, Hq, d, g)
    s = 1 / math.sqrt(d)
    for dt in (torch.float32, torch.bfloat16):
        check(run(q, codes, scales, s, out_dtype=dt), attention(q, s, all_tokens(k, v, Hq, Tq), q_halves=True), f"{dt}")


@pytest.mark.parametrize("scale", [0.125, -0.2, 0.0, 1.7])
def test_scales_of_both_signs(scale):
    g = gen(1)
    codes, scales, _, k, v = packed_cache(2, 2, 300, 128, g)
    q = queries(2, 3, 8, 128, g)
    check(run(q, codes, scales, scale, out_dtype=torch.float32), attention(q, scale, all_tokens(k, v, 8, 3), q_halves=True))


@pytest.mark.parametrize("d", [64, 128])
def test_queries_with_channels_of_very_different_sizes(d):
    g = gen(2)
    codes, scales, _, k, v = packed_cache(1, 2, 200, d, g)
    q = queries(1, 6, 4, d, g, outliers=True)
    q[0, 0] = 0
    q[0, 1, 0] = 0
    q[0, 1, 0, 0] = 1e37 if d == 64 else 1e-38          # next to the ends of the range
    q[0, 2] *= 2.0 ** -100
    s = 1e-37 if d == 64 else 1 / math.sqrt(d)
    check(run(q, codes, scales, s, out_dtype=torch.float32), attention(q, s, all_tokens(k, v, 4, 6), q_halves=True))


def test_lengths_of_the_batch():
    g = gen(3)
    B, N, Hq, Tq, d = 6, 333, 8, 4, 128
    codes, scales, _, k, v = packed_cache(B, 2, N, d, g)
    lens = torch.tensor([0, 1, 333, 32, 400, -5], dtype=torch.int32)
    for b in range(B):                # what lies behind a sequence's end is never looked at
        codes[b, :, max(0, int(lens[b])):] = 0x77
        scales[b, :, max(0, int(lens[b])):] = 255
    q = queries(B, Tq, Hq, d, g)
    ref = attention(q, 0.09, all_tokens(k, v, Hq, Tq, lens), q_halves=True)
    check(run(q, codes, scales, 0.09, seq_lens=lens, out_dtype=torch.float32), ref)
    kn, vn = (torch.randn(B, Tq, 2, d, generator=g).to(torch.bfloat16) for _ in range(2))
    for causal in (True, False):
        ref = attention(q, 0.09, all_tokens(k, v, Hq, Tq, lens), kn, vn, causal, q_halves=True)
        check(run(q, codes, scales, 0.09, seq_lens=lens, k_new=kn, v_new=vn, causal=causal, out_dtype=torch.float32), ref, f"tail {causal}")


def lists(B, Hq, blocks, kmax, g, groups=1):
    heads = Hq // groups
    one = torch.stack([torch.stack([torch.randperm(blocks, generator=g)[:kmax].sort().values for _ in range(heads)]) for _ in range(B)])
    return one.repeat_interleave(groups, 1).to(torch.int32).contiguous()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,kmax,page,groups", [(50, 1, 1, 1), (400, 33, 1, 1), (1000, 600, 1, 2), (401, 20, 8, 4), (130, 5, 32, 2), (99, 13, 8, 1), (3000, 1500, 2, 4)])
def test_lists(N, kmax, page, groups, d):
    g = gen(N)
    B, Tq, Hq, Hkv = 2, 5, 8, 2
    codes, scales, _, k, v = packed_cache(B, Hkv, N, d, g)
    blocks = -(-N // page)
    idx = lists(B, Hq, blocks, min(kmax, blocks), g, groups)
    q = queries(B, Tq, Hq, d, g)
    hm = [t // groups for t in range(Hq)]
    s = 1 / math.sqrt(d)
    ref = attention(q, s, listed(k, v, Hq, Tq, idx, None, page), q_halves=True)
    check(run(q, codes, scales, s, indices=idx, page_size=page, out_dtype=torch.float32), ref)
    check(run(q, codes, scales, s, indices=idx, head_map=hm, page_size=page, out_dtype=torch.float32), ref, "shared lists")
    # lists that end early: what lies behind their end names no token, and the rows there are NaN
    cnt = torch.from_numpy(np.random.default_rng(N).integers(0, idx.shape[2] + 1, (B, Hq // groups)).repeat(groups, 1).astype(np.int32))
    cnt[0, :groups] = 0
    cut = idx.clone()
    used = torch.zeros(B, Hkv, N, dtype=torch.bool)
    for b in range(B):
        for t in range(Hq):
            cut[b, t, int(cnt[b, t]):] = -1 if t % 2 else 2 ** 31 - 1
            for e in idx[b, t, : int(cnt[b, t])].tolist():
                used[b, t // (Hq // Hkv), e * page:(e + 1) * page] = True
    sc = scales.clone()
    sc[~used] = 255
    kn, vn = (torch.randn(B, Tq, Hkv, d, generator=g).to(torch.bfloat16) for _ in range(2))
    check(run(q, codes, sc, s, indices=cut, counts=cnt, head_map=hm, page_size=page, out_dtype=torch.float32),
          attention(q, s, listed(k, v, Hq, Tq, idx, cnt, page), q_halves=True), "counts")
    check(run(q, codes, sc, s, indices=cut, counts=cnt, head_map=hm, page_size=page, k_new=kn, v_new=vn),
          attention(q, s, listed(k, v, Hq, Tq, idx, cnt, page), kn, vn, q_halves=True), "counts and own tokens")


def test_a_repeated_entry_counts_as_often_and_entries_are_kept_in_range():
    g = gen(4)
    codes, scales, _, k, v = packed_cache(1, 1, 60, 128, g)
    q = queries(1, 2, 2, 128, g)
    idx = torch.tensor([[[5, 5, 7, 5], [0, 0, 0, 0]]], dtype=torch.int32)
    check(run(q, codes, scales, 0.1, indices=idx, out_dtype=torch.float32), attention(q, 0.1, listed(k, v, 2, 2, idx, None), q_halves=True))
    wild = torch.tensor([[[-9, 70, 7, 2 ** 31 - 1], [0, -(2 ** 31), 59, 60]]], dtype=torch.int32)
    check(run(q, codes, scales, 0.1, indices=wild, out_dtype=torch.float32), attention(q, 0.1, listed(k, v, 2, 2, wild.clamp(0, 59), None), q_halves=True))


def test_empty_lists():
    g = gen(5)
    codes, scales, _, k, v = packed_cache(2, 2, 20, 64, g)
    q = queries(2, 3, 4, 64, g)
    for e, N in ((torch.zeros(2, 4, 0, dtype=torch.int32), 20), (torch.zeros(2, 4, 0, dtype=torch.int32), 0)):
        o, l = run(q, codes, scales, 0.1, indices=e, N=N)
        assert (o == 0).all() and torch.isneginf(l).all()
    o, l = run(q, codes, scales, 0.1, N=0)
    assert (o == 0).all() and torch.isneginf(l).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 4, 16, 32])
def test_pages(page, d):
    g = gen(page)
    B, Tq, Hq, Hkv, N = 3, 4, 8, 2, 217
    codes, scales, table, k, v = packed_cache(B, Hkv, N, d, g, page=page)
    q = queries(B, Tq, Hq, d, g)
    lens = torch.tensor([217, 1, 100], dtype=torch.int32)
    check(run(q, codes, scales, 0.1, table, page_size=page, N=N, seq_lens=lens, out_dtype=torch.float32),
          attention(q, 0.1, all_tokens(k, v, Hq, Tq, lens), q_halves=True))
    blocks = -(-N // page)
    idx = lists(B, Hq, blocks, max(1, blocks // 3), g, 2)
    idx[:, :, -1] = blocks - 1                  # the last block, which the cache's end cuts
    kn, vn = (torch.randn(B, Tq, Hkv, d, generator=g).to(torch.bfloat16) for _ in range(2))
    check(run(q, codes, scales, 0.1, table, page_size=page, N=N, indices=idx, head_map=[t // 2 for t in range(Hq)], k_new=kn, v_new=vn, out_dtype=torch.float32),
          attention(q, 0.1, listed(k, v, Hq, Tq, idx, None, page), kn, vn, q_halves=True))
    # page numbers out of range are kept in it
    wild = table.clone()
    wild[0, 0], wild[1, 0] = -3, 2 ** 30
    sane = wild.clamp(0, codes.shape[0] - 1)
    a = run(q, codes, scales, 0.1, wild, page_size=page, N=N, out_dtype=torch.float32)
    b = run(q, codes, scales, 0.1, sane, page_size=page, N=N, out_dtype=torch.float32)
    assert all(torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0)) for x, y in zip(a, b))


def test_strides_and_slices():
    """Tokens before heads, a slice of a wider cache, lists that are a slice of heads of wider ones."""
    g = gen(6)
    B, Tq, Hq, Hkv, N, d = 2, 5, 8, 2, 150, 128
    codes, scales, _, k, v = packed_cache(B, Hkv, N, d, g)
    wide_c = torch.full((B, N + 9, Hkv + 1, 2, d // 2), 0x55, dtype=torch.uint8)
    wide_s = torch.full((B, N + 9, Hkv + 1, 2, d // 32), 255, dtype=torch.uint8)
    wide_c[:, :N, 1:] = codes.transpose(1, 2)
    wide_s[:, :N, 1:] = scales.transpose(1, 2)
    c, s = (w.to(DEV)[:, :, 1:].transpose(1, 2) for w in (wide_c, wide_s))
    q = queries(B, Tq, Hq, d, g)
    check(run(q, c, s, 0.1, N=N, out_dtype=torch.float32), attention(q, 0.1, all_tokens(k, v, Hq, Tq), q_halves=True))
    idx = lists(B, 3 * Hq, N, 40, g).to(DEV)
    cnt = torch.randint(0, 41, (B, 3 * Hq), generator=g, dtype=torch.int32).to(DEV)
    part, pcnt = idx[:, Hq:2 * Hq], cnt[:, Hq:2 * Hq]
    check(sts.sts_packed_attn(q.to(DEV), c, s, 0.1, indices=part, counts=pcnt, N=N, out_dtype=torch.float32),
          attention(q, 0.1, listed(k, v, Hq, Tq, part.cpu(), pcnt.cpu()), q_halves=True))


def test_rows_beyond_32_bits():
    """Tokens 64 KB apart, 70000 of them: offsets of more than 32 bits, with and without lists."""
    g = gen(7)
    N, d, step = 70000, 128, 65536
    big = torch.full((N * step,), 0x11, dtype=torch.uint8, device=DEV)
    c = big.as_strided((1, 1, N, 2, 64), (0, 0, step, 64, 1))
    codes, scales, _, k, v = packed_cache(1, 1, N, d, g)
    c.copy_(codes)
    q = queries(1, 2, 2, d, g)
    check(run(q, c, scales, 0.1, out_dtype=torch.float32), attention(q, 0.1, all_tokens(k, v, 2, 2), q_halves=True))
    idx = torch.tensor([[[0, 3, 65535, 65536, 69998, 69999], [1, 2, 65537, 68000, 69000, 69999]]], dtype=torch.int32)
    check(run(q, c, scales, 0.1, indices=idx, out_dtype=torch.float32), attention(q, 0.1, listed(k, v, 2, 2, idx, None), q_halves=True))


def test_nan_groups_reach_those_that_see_them():
    g = gen(8)
    codes, scales, _, k, v = packed_cache(1, 2, 64, 128, g)
    scales[0, 0, 10, 1, 2] = 255              # channels 64..95 of V of one token of KV head 0
    scales[0, 1, 20, 0, 0] = 255              # K of one token of KV head 1
    q = queries(1, 2, 4, 128, g)
    o, _ = run(q, codes, scales, 0.1, out_dtype=torch.float32)
    o = o.cpu()
    assert torch.isnan(o[0, :, :2, 64:96]).all() and torch.isfinite(o[0, :, :2, :64]).all() and torch.isfinite(o[0, :, :2, 96:]).all()
    assert torch.isnan(o[0, :, 2:]).all()
    idx = torch.tensor([[[1, 2, 3]] * 4], dtype=torch.int32)
    assert torch.isfinite(run(q, codes, scales, 0.1, indices=idx)[0]).all()


def test_one_call_is_like_another():
    """Results do not change from run to run, nor with what the workspace held."""
    g = gen(9)
    codes, scales, _, k, v = packed_cache(2, 2, 3000, 128, g)
    q = queries(2, 5, 8, 128, g)
    ws = torch.full((1 << 24,), 0xFF, dtype=torch.uint8, device=DEV)
    a = run(q, codes, scales, 0.1, workspace=ws)
    ws.fill_(0)
    b = run(q, codes, scales, 0.1, workspace=ws)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_from_the_draft_to_the_output_and_back_into_the_cache():
    """As a serving step uses them: the selection ranks draft scores, attention over the 4-bit cache takes the lists and the block's
    own tokens, and these are then stored behind the cached ones, where the next step finds them. Captured and replayed too."""
    g = gen(10)
    B, Tq, Hq, Hkv, d, N = 2, 5, 8, 2, 128, 500
    room = N + 3 * Tq
    codes, scales, _, k, v = packed_cache(B, Hkv, room, d, g)
    codes, scales = codes.to(DEV), scales.to(DEV)
    lens = torch.tensor([N, N - 77], dtype=torch.int32, device=DEV)
    hm = [t // 2 for t in range(Hq)]
    kept = 60
    q = queries(B, Tq, Hq, d, g).to(DEV)
    kn, vn = (torch.randn(B, Tq, Hkv, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    scores = torch.rand(B, Hq // 2, Tq, room, generator=g).to(DEV)
    idx, cnt, _ = sts.sts_select(scores, hm, kept, seq_lens=lens)
    out = torch.empty(B, Tq, Hq, d, dtype=torch.float32, device=DEV)
    lse = torch.empty(B, Hq, Tq, dtype=torch.float32, device=DEV)
    ref = attention(q.cpu(), 0.09, listed(k, v, Hq, Tq, idx.cpu(), cnt.cpu()), kn.cpu(), vn.cpu(), q_halves=True)

    def step():
        sts.sts_select(scores, hm, kept, seq_lens=lens, out=(idx, cnt))
        sts.sts_packed_attn(q, codes, scales, 0.09, indices=idx, counts=cnt, head_map=hm, k_new=kn, v_new=vn, out=out, lse_out=lse)
        sts.sts_packed_store(kn, vn, codes, scales, pos=lens)

    step()
    check((out, lse), ref)
    back = sts.sts_packed_load(codes, scales, Tq, pos=lens)
    from cache_util import quantise, values
    for got, rows in zip(back, (kn, vn)):
        assert torch.equal(got.cpu().double(), values(*quantise(rows.cpu())))
    # the next step, over all tokens, sees them
    after = lens + Tq
    kv = [t.clone() for t in (k, v)]
    for b in range(B):
        n = int(lens[b])
        for t, rows in zip(kv, (kn, vn)):
            t[b, :, n:n + Tq] = values(*quantise(rows.cpu()))[b].transpose(0, 1)
    check(sts.sts_packed_attn(q, codes, scales, 0.09, seq_lens=after, out_dtype=torch.float32),
          attention(q.cpu(), 0.09, all_tokens(*kv, Hq, Tq, after.cpu()), q_halves=True))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        q.copy_(queries(B, Tq, Hq, d, g))
        kn.copy_(torch.randn(B, Tq, Hkv, d, generator=g))
        scores.copy_(torch.rand(B, Hq // 2, Tq, room, generator=g))
        lens.add_(1)
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (idx, out, lse, codes, scales)]
        for t in (out, lse):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (idx, out, lse, codes, scales))), i


def test_prepared_calls_do_not_share_scratch():
    """Two prepared calls on two streams at once, each on the stream it was prepared on or not."""
    g = gen(11)
    sets = []
    for i in range(2):
        codes, scales, _, k, v = packed_cache(1, 2, 2000, 128, g)
        q = queries(1, 3, 8, 128, g).to(DEV)
        call = sts.sts_packed_attn(q, codes.to(DEV), scales.to(DEV), 0.1, prepare=True, out_dtype=torch.float32)
        call()
        torch.cuda.synchronize()
        sets.append((call, [t.clone() for t in call.result]))
    streams = [torch.cuda.Stream() for _ in sets]
    for t in range(4):
        for (call, _), s in zip(sets, streams):
            with torch.cuda.stream(s):
                call()
    torch.cuda.synchronize()
    for call, want in sets:
        assert all(torch.equal(a, b) for a, b in zip(call.result, want))


@pytest.mark.parametrize("N", [40, 2000])
def test_keys_that_are_no_numbers(N):
    """One key, and all of them: their rows have no result, whatever the rest is split into."""
    g = gen(12)
    codes, scales, _, k, v = packed_cache(1, 2, N, 128, g)
    q = queries(1, 2, 4, 128, g)
    ref = attention(q, 0.1, all_tokens(k, v, 4, 2), q_halves=True)
    for bad in (slice(N - 1, N), slice(0, N // 2), slice(0, N)):
        sc = scales.clone()
        sc[:, 1, bad, 0, 1] = 255
        o, l = (x.cpu() for x in run(q, codes, sc, 0.1, out_dtype=torch.float32))
        assert torch.isnan(o[:, :, 2:]).all() and not torch.isfinite(l[:, 2:]).any()
        assert ((o[:, :, :2].double() - ref[0][:, :, :2]).abs() <= ref[2][:, :, :2]).all()
    q[0, 1, 3, 5] = float("inf")
    o = run(q, codes, scales, 0.1, out_dtype=torch.float32)[0].cpu()
    assert torch.isnan(o[0, 1, 3]).all() and torch.isfinite(o[0, 0]).all() and torch.isfinite(o[0, 1, :3]).all()


def test_a_batch_over_one_cache_and_calls_without_results_of_their_own():
    """One cache for the whole batch (a stride of 0), no lse asked for, no batch and no rows at all."""
    g = gen(13)
    codes, scales, _, k, v = packed_cache(1, 2, 150, 128, g)
    c, s = (t.to(DEV).expand(3, -1, -1, -1, -1) for t in (codes, scales))
    q = queries(3, 4, 8, 128, g)
    got = sts.sts_packed_attn(q.to(DEV), c, s, 0.1, out_dtype=torch.float32)
    check(got, attention(q, 0.1, all_tokens(k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1), 8, 4), q_halves=True))
    o, none = sts.sts_packed_attn(q.to(DEV), c, s, 0.1, out_dtype=torch.float32, want_lse=False)
    assert none is None and torch.equal(o, got[0])
    o, l = sts.sts_packed_attn(q[:0].to(DEV), c[:0], s[:0], 0.1)
    assert o.shape == (0, 4, 8, 128) and l.shape == (0, 8, 4)
    a, b = sts.sts_packed_load(c, s, 0)
    assert a.shape == b.shape == (3, 0, 2, 128)
    sts.sts_packed_store(a, b, codes.to(DEV).expand(3, -1, -1, -1, -1), s)
    a, b = sts.sts_packed_load(c[:0], s[:0], 7)
    assert a.shape == (0, 7, 2, 128)


def test_shapes_and_types_that_the_binding_refuses():
    g = gen(14)
    codes, scales, _, _, _ = packed_cache(1, 2, 40, 128, g)
    codes, scales = codes.to(DEV), scales.to(DEV)
    q = queries(1, 2, 4, 128, g).to(DEV)
    rows = torch.zeros(1, 3, 2, 128, dtype=torch.bfloat16, device=DEV)
    one = torch.zeros(1, dtype=torch.int32, device=DEV)
    for call in (lambda: sts.sts_packed_attn(q.float(), codes, scales, 0.1), lambda: sts.sts_packed_attn(q, codes.view(torch.int8), scales, 0.1),
                 lambda: sts.sts_packed_attn(q, codes, scales[:, :, :39], 0.1), lambda: sts.sts_packed_attn(q[..., :64].contiguous(), codes, scales, 0.1),
                 lambda: sts.sts_packed_attn(q, codes, scales, 0.1, N=41), lambda: sts.sts_packed_attn(q, codes, scales, 0.1, counts=one),
                 lambda: sts.sts_packed_attn(q, codes, scales, 0.1, seq_lens=one.long()), lambda: sts.sts_packed_attn(q, codes, scales, 0.1, k_new=rows),
                 lambda: sts.sts_packed_store(rows.half(), rows, codes, scales), lambda: sts.sts_packed_store(rows[:, :, :1], rows, codes, scales),
                 lambda: sts.sts_packed_store(rows, rows, codes, scales, pos=one.cpu()), lambda: sts.sts_packed_load(codes, scales, 3, out=(rows, rows[:, :2])),
                 lambda: sts.sts_packed_load(codes, scales, 3, block_table=one.view(1, 1)), lambda: sts.sts_packed_load(codes.transpose(3, 4), scales, 3)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: sts.sts_packed_store(rows.cpu(), rows.cpu(), codes.cpu(), scales.cpu()), lambda: sts.sts_packed_attn(q, codes, scales, float("nan")),
                 lambda: sts.sts_packed_attn(torch.zeros(1, 17, 4, 128, dtype=torch.bfloat16, device=DEV), codes, scales, 0.1),
                 lambda: sts.sts_packed_attn(q, codes, scales, 0.1, workspace=torch.empty(0, dtype=torch.uint8, device=DEV)),
                 lambda: sts.sts_packed_store(rows, rows, codes, scales, page_size=3)):
        with pytest.raises(sts.StsError):
            call()


@pytest.mark.parametrize("scale", [-0.1, 0.0])
def test_own_tokens_at_scales_of_both_signs(scale):
    g = gen(15)
    codes, scales, _, k, v = packed_cache(2, 2, 90, 128, g)
    q = queries(2, 5, 8, 128, g)
    kn, vn = (torch.randn(2, 5, 2, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    check(run(q, codes, scales, scale, k_new=kn, v_new=vn, out_dtype=torch.float32), attention(q, scale, all_tokens(k, v, 8, 5), kn, vn, q_halves=True))


@pytest.mark.parametrize("Tq,Hq,Hkv,listed_heads", [(2, 256, 256, False), (16, 256, 16, False), (1, 256, 32, True), (3, 240, 16, True)])
def test_many_heads(Tq, Hq, Hkv, listed_heads):
    g = gen(16)
    codes, scales, _, k, v = packed_cache(1, Hkv, 70, 64, g)
    q = queries(1, Tq, Hq, 64, g)
    idx = lists(1, Hq, 70, 40, g) if listed_heads else None
    ref = attention(q, 0.1, listed(k, v, Hq, Tq, idx, None) if listed_heads else all_tokens(k, v, Hq, Tq), q_halves=True)
    check(run(q, codes, scales, 0.1, indices=idx, out_dtype=torch.float32), ref)


def test_large_batches():
    """More sequences than a grid's last dimension has, of one token each: the output is its value."""
    B, d = 40001, 64
    g = gen(17)
    rows = torch.randn(2, B, 1, 1, d, generator=g).to(torch.bfloat16).to(DEV)
    codes, scales = torch.zeros(B, 1, 1, 2, d // 2, dtype=torch.uint8, device=DEV), torch.zeros(B, 1, 1, 2, d // 32, dtype=torch.uint8, device=DEV)
    sts.sts_packed_store(rows[0], rows[1], codes, scales)
    back = sts.sts_packed_load(codes, scales, 1)
    q = torch.randn(B, 1, 1, d, generator=g).to(torch.bfloat16).to(DEV)
    for kw in ({}, {"indices": torch.zeros(B, 1, 1, dtype=torch.int32, device=DEV)}):
        assert torch.equal(sts.sts_packed_attn(q, codes, scales, 0.1, **kw)[0], back[1])
    assert torch.equal(sts.sts_packed_attn(q, codes, scales, 0.0, k_new=rows[0], v_new=back[1])[0], back[1])


@pytest.mark.parametrize("Tq,causal", [(1, True), (4, False), (5, True), (9, False), (16, True)])
@pytest.mark.parametrize("d", [64, 128])
def test_own_tokens_after_short_lists(Tq, causal, d):
    """Lists that one workgroup has whole, with own tokens: one launch, no other kernel merges anything. Own tokens that a row does not see
    may be anything."""
    g = gen(18 + Tq)
    codes, scales, _, k, v = packed_cache(3, 2, 300, d, g)
    q = queries(3, Tq, 8, d, g)
    idx = lists(3, 8, 300, 70, g)
    cnt = torch.randint(0, 71, (3, 8), generator=g, dtype=torch.int32)
    cnt[0] = 0
    kn, vn = (torch.randn(3, Tq, 2, d, generator=g).to(torch.bfloat16) for _ in range(2))
    ref = attention(q, 0.1, listed(k, v, 8, Tq, idx, cnt), kn, vn, causal, q_halves=True)
    got = run(q, codes, scales, 0.1, indices=idx, counts=cnt, k_new=kn, v_new=vn, causal=causal, out_dtype=torch.float32)
    check(got, ref)
    if causal and Tq > 1:
        kn[:, -1], vn[:, -1] = float("nan"), float("inf")
        bad = run(q, codes, scales, 0.1, indices=idx, counts=cnt, k_new=kn, v_new=vn, out_dtype=torch.float32)
        assert torch.equal(bad[0][:, :-1], got[0][:, :-1]) and torch.equal(bad[1][..., :-1], got[1][..., :-1])
        assert torch.isnan(bad[0][:, -1]).all()
    sts.prof_enable(True)
    sts.prof_reset()
    try:
        run(q, codes, scales, 0.1, indices=idx, counts=cnt, k_new=kn, v_new=vn, causal=causal)
        counts = sts.prof_read()
        assert counts["packed_attn"][0] == 1 and counts["attn_combine"][0] == 0
    finally:
        sts.prof_enable(False)
        sts.prof_reset()
