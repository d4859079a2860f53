"""sts_window_attn: attention with a sliding window and sinks against the definition in 64 bits, single tokens to prompts, within bounds
derived from the roundings (cache_util.attention)."""
import math

import pytest
import torch

import paper_2605_15508_amd as sts
from cache_util import attention, check, table_of, to_pages

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def data(B, Tq, Hq, Hkv, N, d, seed, tail=False):
    g = gen(seed)
    q = torch.randn(B, Tq, Hq, d, generator=g).to(torch.bfloat16)
    k, v = (torch.randn(B, Hkv, N, d, generator=g).to(torch.bfloat16) for _ in range(2))
    new = [torch.randn(B, Tq, Hkv, d, generator=g).to(torch.bfloat16) for _ in range(2)] if tail else [None, None]
    return q, k, v, *new


def visible(B, Tq, N, window, sinks, lens, tail):
    """see [Tq, N] of a batch element"""
    def see(b):
        L = N if lens is None else max(0, min(int(lens[b]), N))
        p = torch.arange(Tq) + (L if tail else L - Tq)
        n = torch.arange(N)
        return (n <= p[:, None]) & (n < L) & ((n < sinks) | (n > p[:, None] - window))
    return see


def reference(q, k, v, scale, window, sinks, lens=None, kn=None, vn=None):
    B, Tq, Hq, _ = q.shape
    G = Hq // k.shape[1]
    see = visible(B, Tq, k.shape[2], window, sinks, lens, kn is not None)

    def keys(b, t):
        s = see(b)
        some = s.any(0)
        return k[b, t // G, some].double(), v[b, t // G, some].double(), s[:, some]
    return attention(q, scale, keys, kn, vn)


def run(q, k, v, scale, window, sinks, **kw):
    kw = {a: x.to(DEV) if isinstance(x, torch.Tensor) else x for a, x in kw.items()}
    return sts.sts_window_attn(q.to(DEV), k.to(DEV), v.to(DEV), scale, window, sinks=sinks, **kw)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Tq,Hq,Hkv,N,window,sinks", [
    (1, 1, 1, 1, 1, 1, 0), (1, 1, 4, 1, 100, 1, 0), (2, 1, 8, 2, 300, 64, 4), (1, 5, 4, 2, 500, 33, 1), (2, 16, 8, 1, 200, 100, 40), (1, 3, 16, 1, 97, 1000, 0),
    (1, 16, 16, 1, 400, 7, 3), (1, 2, 2, 2, 64, 32, 32), (1, 4, 4, 4, 1000, 400, 500), (3, 8, 8, 8, 129, 128, 1), (1, 16, 4, 2, 16, 5, 2),
    (1, 17, 1, 1, 17, 1, 0), (1, 40, 4, 1, 300, 64, 4), (2, 130, 8, 2, 130, 33, 1), (1, 33, 6, 2, 700, 600, 5), (1, 200, 16, 1, 201, 1, 1), (2, 90, 3, 1, 400, 10 ** 9, 0),
    (1, 300, 5, 5, 300, 65, 63), (1, 65, 8, 2, 260, 64, 64), (1, 129, 2, 2, 512, 128, 300)])
def test_windows(B, Tq, Hq, Hkv, N, window, sinks, d):
    q, k, v, _, _ = data(B, Tq, Hq, Hkv, N, d, N + window)
    s = 1 / math.sqrt(d)
    ref = reference(q, k, v, s, window, sinks)
    for dt in (torch.float32, torch.bfloat16):
        check(run(q, k, v, s, window, sinks, out_dtype=dt), ref, f"{dt}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Tq", [4, 60])
def test_lengths_of_the_batch(Tq, d):
    """Sequences of all lengths, shorter than the block too: rows before the first token see nothing."""
    B, N = 8, 260
    q, k, v, _, _ = data(B, Tq, 4, 2, N, d, 3)
    lens = torch.tensor([0, 1, Tq - 1, Tq, Tq + 1, 100, 260, 999], dtype=torch.int32)
    for b in range(B):              # what lies behind a sequence's end is never looked at
        k[b, :, max(0, int(lens[b])):] = float("nan")
        v[b, :, max(0, int(lens[b])):] = float("inf")
    for window, sinks in ((50, 4), (300, 0), (1, 1)):
        check(run(q, k, v, 0.1, window, sinks, seq_lens=lens, out_dtype=torch.float32), reference(q, k, v, 0.1, window, sinks, lens), f"{window}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Tq,window,sinks", [(1, 1, 0), (5, 5, 0), (5, 64, 4), (16, 16, 1), (16, 500, 3), (8, 40, 200)])
def test_own_tokens_that_are_not_in_the_cache_yet(Tq, window, sinks, d):
    B, N = 3, 210
    q, k, v, kn, vn = data(B, Tq, 8, 2, N, d, 4, tail=True)
    lens = torch.tensor([210, 0, 33], dtype=torch.int32)
    for b in range(B):
        v[b, :, int(lens[b]):] = float("nan")
    ref = reference(q, k, v, 0.1, window, sinks, lens, kn, vn)
    check(run(q, k, v, 0.1, window, sinks, seq_lens=lens, k_new=kn, v_new=vn, out_dtype=torch.float32), ref)
    # the same tokens in the cache: the block's rows are its last ones
    full_k, full_v = (torch.cat((t, torch.zeros(B, 2, Tq, d, dtype=t.dtype)), 2) for t in (k, v))
    for b in range(B):
        n = int(lens[b])
        full_k[b, :, n:n + Tq], full_v[b, :, n:n + Tq] = kn[b].transpose(0, 1), vn[b].transpose(0, 1)
    check(run(q, full_k, full_v, 0.1, window, sinks, seq_lens=lens + Tq, out_dtype=torch.float32), ref, "in the cache")


@pytest.mark.parametrize("page", [1, 2, 16, 32])
@pytest.mark.parametrize("Tq,window,sinks", [(1, 20, 4), (6, 300, 0), (70, 45, 18), (150, 64, 1)])
def test_pages(Tq, window, sinks, page):
    B, N, d = 2, 233, 128
    q, k, v, _, _ = data(B, Tq, 4, 2, N, d, page)
    lens = torch.tensor([233, 77], dtype=torch.int32)
    ref = reference(q, k, v, 0.1, window, sinks, lens)
    kp, vp = (to_pages(t, page, None) for t in (k, v))
    table = table_of(B, N, page, None)
    kw = dict(page_size=page, N=N, seq_lens=lens, out_dtype=torch.float32)
    check(run(q, kp, vp, 0.1, window, sinks, block_table=table, **kw), ref)
    # pages that no row looks at may be gone: their numbers and what lies there do not matter
    gone = table.clone()
    for b in range(B):
        first = max(0, int(lens[b]) - Tq - window + 1)
        for j in range(table.shape[1]):
            if j * page >= sinks and (j + 1) * page <= first or j * page >= int(lens[b]):
                kp[table[b, j]], vp[table[b, j]] = float("nan"), float("nan")
                gone[b, j] = 2 ** 31 - 1 if j % 2 else -7
    check(run(q, kp, vp, 0.1, window, sinks, block_table=gone, **kw), ref, "released pages")


@pytest.mark.parametrize("scale", [-0.1, 0.0, 0.7])
@pytest.mark.parametrize("Tq", [3, 50])
def test_scales_of_both_signs(Tq, scale):
    q, k, v, _, _ = data(1, Tq, 4, 2, 200, 128, 6)
    check(run(q, k, v, scale, 60, 2, out_dtype=torch.float32), reference(q, k, v, scale, 60, 2))


def test_strides():
    """Tokens before heads, K and V interleaved, a bound below the tensor's length."""
    B, N, d, Hkv = 2, 180, 128, 2
    for Tq in (4, 70):
        q, k, v, _, _ = data(B, Tq, 4, Hkv, N, d, 7)
        wide = torch.full((B, N + 5, Hkv + 1, 2, d), float("nan"), dtype=torch.bfloat16)
        wide[:, :N, 1:, 0], wide[:, :N, 1:, 1] = k.transpose(1, 2), v.transpose(1, 2)
        wide = wide.to(DEV)
        kk, vv = (wide[:, :, 1:, j].transpose(1, 2) for j in range(2))
        check(run(q, kk, vv, 0.1, 64, 3, N=N, out_dtype=torch.float32), reference(q, k, v, 0.1, 64, 3))


@pytest.mark.parametrize("Tq", [2, 40])
def test_rows_beyond_32_bits(Tq):
    """Tokens 128 KB apart, 40000 of them: sinks and window lie 5 GB from each other."""
    N, d, step = 40000, 64, 65536
    big = torch.zeros(N * step, dtype=torch.bfloat16, device=DEV)
    kk = big.as_strided((1, 1, N, d), (0, 0, step, 1))
    vv = big[d:].as_strided((1, 1, N, d), (0, 0, step, 1))
    q, k, v, _, _ = data(1, Tq, 2, 1, N, d, 8)
    kk.copy_(k), vv.copy_(v)
    check(run(q, kk, vv, 0.1, 100, 5, out_dtype=torch.float32), reference(q, k, v, 0.1, 100, 5))
    check(run(q[:, :, :1], kk, vv, 0.1, 39990, 5, out_dtype=torch.float32), reference(q[:, :, :1], k, v, 0.1, 39990, 5))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("B,Tq,N,window,sinks,spots", [(2, 40, 200, 30, 4, [10, 50, 150]), (1, 100, 100, 33, 0, [60, 61]), (1, 5, 300, 70, 3, [2, 100, 231, 299, 297]),
                                                       (1, 12, 90, 20, 5, [0, 40, 80]), (1, 70, 160, 1000, 0, [100]), (2, 3, 64, 5, 1, [62])])
def test_values_that_are_no_numbers_reach_those_that_see_them_alone(B, Tq, N, window, sinks, spots, bad, d):
    q, k, v, _, _ = data(B, Tq, 4, 2, N, d, 9)
    for n in spots:
        v[:, 0, n, 3] = bad
        v[:, 1, n] = bad
    first = N - Tq - window + 1
    for n in range(sinks, first):            # nobody sees these
        k[:, :, n], v[:, :, n] = float("nan"), float("nan")
    o, l = run(q, k, v, 0.1, window, sinks, out_dtype=torch.float32)
    see = visible(B, Tq, N, window, sinks, None, False)(0)
    hit = see[:, [n for n in spots if n < sinks or n >= first]].any(1)
    clean = v.clone()
    for n in spots:
        clean[:, 0, n, 3] = 0
        clean[:, 1, n] = 0
    ref = reference(q, k, clean, 0.1, window, sinks)
    o = o.cpu()
    for t in range(4):
        chans = slice(3, 4) if t < 2 else slice(None)
        got = o[:, :, t, chans]
        assert torch.isfinite(got[:, ~hit]).all()
        same = torch.isnan(got) if math.isnan(bad) else got == bad
        assert same[:, hit].all()
        o[:, :, t, chans] = torch.where(hit[:, None], ref[0][:, :, t, chans].float(), got)
    check((o, l), ref)


def test_a_prompt_in_chunks_is_the_prompt_at_once():
    """As a serving program uses it: chunks of a prompt, then single tokens, each appended to a paged cache before its call; captured and
    replayed too."""
    B, Hq, Hkv, d, T, page, window, sinks = 2, 8, 2, 128, 150, 16, 48, 4
    q, k, v, _, _ = data(B, T, Hq, Hkv, T, d, 10)
    ref = reference(q, k, v, 0.09, window, sinks)
    kp, vp = (to_pages(t, page, None).to(DEV) for t in (k, v))
    table = table_of(B, T, page, None).to(DEV)
    at, outs, lses = 0, [], []
    for n in (64, 17, 33, 16, 13, 1, 1, 5):
        lens = torch.full((B,), at + n, dtype=torch.int32, device=DEV)
        o, l = sts.sts_window_attn(q[:, at:at + n].contiguous().to(DEV), kp, vp, 0.09, window, sinks=sinks, seq_lens=lens, page_size=page, block_table=table, N=T,
                                   out_dtype=torch.float32)
        outs.append(o), lses.append(l)
        at += n
    assert at == T
    check((torch.cat(outs, 1), torch.cat(lses, 2)), ref)
    for n in (1, 9, 70):
        qs = q[:, :n].contiguous().to(DEV)
        lens = torch.full((B,), n, dtype=torch.int32, device=DEV)
        out, lse = torch.empty(B, n, Hq, d, device=DEV), torch.empty(B, Hq, n, device=DEV)

        def step():
            sts.sts_window_attn(qs, kp, vp, 0.09, window, sinks=sinks, seq_lens=lens, page_size=page, block_table=table, N=T, out=out, lse_out=lse)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for i in range(3):
            qs.copy_(torch.randn(B, n, Hq, d, generator=gen(i)))
            lens.fill_(n + 20 * i)
            step()
            torch.cuda.synchronize()
            want = out.clone(), lse.clone()
            out.fill_(7), lse.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_two_captured_graphs_at_once():
    """Graphs captured from the same stream have scratch of their own: replayed on two streams at once they do not disturb each other."""
    sets = []
    for i, Tq in enumerate((3, 40)):
        q, k, v, _, _ = (t.to(DEV) if t is not None else None for t in data(1, Tq, 8, 2, 3000, 128, 20 + i))
        out, lse = torch.empty(1, Tq, 8, 128, device=DEV), torch.empty(1, 8, Tq, device=DEV)
        call = lambda q=q, k=k, v=v, out=out, lse=lse: sts.sts_window_attn(q, k, v, 0.09, 2500, sinks=4, out=out, lse_out=lse)  # noqa: E731
        call()
        torch.cuda.synchronize()
        want = out.clone(), lse.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        sets.append((graph, out, lse, want, torch.cuda.Stream(), call))          # the call holds its inputs
    for _ in range(4):
        for graph, out, lse, _, s, _ in sets:
            with torch.cuda.stream(s):
                out.fill_(0), lse.fill_(0)
                graph.replay()
        torch.cuda.synchronize()
        for _, out, lse, want, _, _ in sets:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("Tq,N,window", [(2000, 2000, 500), (600, 9000, 4096), (48, 20000, 9000), (1, 50000, 30000)])
def test_long_windows(Tq, N, window):
    """Many blocks, and few that are split over their keys, against 64 bits on the GPU at some heads."""
    q, k, v, _, _ = data(1, Tq, 8, 2, N, 128, 11)
    o, l = run(q, k, v, 0.09, window, 4, out_dtype=torch.float32)
    n = torch.arange(N, device=DEV)
    p = torch.arange(N - Tq, N, device=DEV)[:, None]
    see = (n <= p) & ((n < 4) | (n > p - window))
    for t in (0, 5):
        K, V, Q = k[0, t // 4].to(DEV).double(), v[0, t // 4].to(DEV).double(), q[0, :, t].to(DEV).double()
        s = torch.where(see, 0.09 * (Q @ K.T), -math.inf)
        z = torch.logsumexp(s, -1)
        w = torch.exp(s - z[:, None])
        want, size = w @ V, w @ V.abs()
        # scores of 128 products in fp32, |q||k| under 400; weights to 2^-8; sums of N
        d_s = 0.09 * 136 * 2.0 ** -24 * float((Q.abs() @ K.abs().T).max())
        sums = (N / 8 + 64) * 2.0 ** -24
        assert ((o[0, :, t].double() - want).abs() <= (2.0 ** -8 + 2.2 * d_s + 2.0 ** -20 + sums) * size).all()
        assert ((l[0, t].double() - z).abs() <= d_s + sums + 2.0 ** -20 + 2.0 ** -22 * z.abs()).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Tq,N,window,sinks", [(1, 3, 900, 700, 4), (1, 1, 40, 40, 0), (2, 40, 900, 700, 4), (4, 300, 300, 90, 2)])
def test_keys_that_are_no_numbers(B, Tq, N, window, sinks, d):
    """One key, and all of them: who sees one has no result, whatever the rest is split into; who does not is as without."""
    q, k, v, _, _ = data(B, Tq, 4, 2, N, d, 12)
    see = visible(B, Tq, N, window, sinks, None, False)(0)
    for bad in ([N - 2], list(range(N - min(window, N) // 2, N)), list(range(N))):
        kk = k.clone()
        kk[:, 1, bad] = float("nan")
        o, _ = run(q, kk, v, 0.1, window, sinks, out_dtype=torch.float32)
        hit = see[:, bad].any(1)
        o = o.cpu()
        assert torch.isnan(o[:, hit, 2:]).all()
        ref = reference(q, k, v, 0.1, window, sinks)
        assert ((o[:, :, :2].double() - ref[0][:, :, :2]).abs() <= ref[2][:, :, :2]).all()
        assert ((o[:, ~hit, 2:].double() - ref[0][:, ~hit, 2:]).abs() <= ref[2][:, ~hit, 2:] + 1e-30).all()


@pytest.mark.parametrize("Tq,window", [(1, 1), (4, 4), (1, 3)])
def test_the_cache_is_not_looked_at_where_the_window_is_the_block(Tq, window):
    """Own tokens fill the window, or nearly: the cached ones that nobody sees may be anything."""
    q, k, v, kn, vn = data(1, Tq, 4, 2, 70, 128, 13, tail=True)
    ref = reference(q, k, v, 0.1, window, 0, None, kn, vn)
    k[:, :, : 70 - window + 1], v[:, :, : 70 - window + 1] = float("inf"), float("nan")
    check(run(q, k, v, 0.1, window, 0, k_new=kn, v_new=vn, out_dtype=torch.float32), ref)


@pytest.mark.parametrize("Tq", [3, 60])
def test_windows_and_sinks_beyond_any_cache(Tq):
    q, k, v, _, _ = data(1, Tq, 4, 2, 90, 64, 14)
    ref = reference(q, k, v, 0.1, 1000, 0)
    for window, sinks in ((10 ** 12, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 10 ** 12)):
        check(run(q, k, v, 0.1, window, sinks, out_dtype=torch.float32), ref, f"{window} {sinks}")
    with pytest.raises(sts.StsError):
        run(q, k, v, 0.1, -(2 ** 31), 0)


@pytest.mark.parametrize("apart", [2 ** 29, 2 ** 32])
@pytest.mark.parametrize("Tq", [5, 40])
def test_pages_that_lie_far_apart(Tq, apart):
    """Pages 1 GB apart and 8 GB apart: offsets of more than 32 bits, and of more than 32 bits of 16 bytes."""
    N, d, page, Hkv = 70, 64, 8, 2
    q, k, v, _, _ = data(1, Tq, 4, Hkv, N, d, 15)
    ref = reference(q, k, v, 0.1, 45, 3)
    kp, vp = (to_pages(t, page, None, 1) for t in (k, v))
    pool = torch.empty((kp.shape[0] - 1) * apart + 2 * kp[0].numel(), dtype=torch.bfloat16, device=DEV)
    far = [pool[j * kp[0].numel():].as_strided(kp.shape, (apart, page * d, d, 1)) for j in range(2)]
    for t, rows in zip(far, (kp, vp)):
        t.copy_(rows)
    try:
        check(run(q, *far, 0.1, 45, 3, page_size=page, N=N, block_table=table_of(1, N, page, None, 1), out_dtype=torch.float32), ref)
    finally:
        del far, pool
        torch.cuda.empty_cache()


@pytest.mark.parametrize("Tq", [4, 50])
def test_a_batch_over_one_cache_and_calls_without_results_of_their_own(Tq):
    """One cache for the whole batch (a stride of 0), no lse asked for, no batch at all; and what the measurement aid counts."""
    q, k, v, _, _ = data(3, Tq, 4, 2, 200, 128, 16)
    k, v = (t[:1].expand(3, -1, -1, -1) for t in (k, v))
    ref = reference(q, k, v, 0.1, 60, 3)
    kd, vd = (t[:1].to(DEV).expand(3, -1, -1, -1) for t in (k, v))
    got = sts.sts_window_attn(q.to(DEV), kd, vd, 0.1, 60, sinks=3, out_dtype=torch.float32)
    check(got, ref)
    sts.prof_enable(True)
    sts.prof_reset()
    try:
        o, none = sts.sts_window_attn(q.to(DEV), kd, vd, 0.1, 60, sinks=3, out_dtype=torch.float32, want_lse=False)
        assert sts.prof_read()["window"][0] == 1
    finally:
        sts.prof_enable(False)
        sts.prof_reset()
    assert none is None and torch.equal(o, got[0])
    o, l = sts.sts_window_attn(q[:0].to(DEV), kd[:0], vd[:0], 0.1, 60, sinks=3)
    assert o.shape == (0, Tq, 4, 128) and l.shape == (0, 4, Tq)


@pytest.mark.parametrize("scale", [-0.1, 0.0])
def test_own_tokens_at_scales_of_both_signs(scale):
    q, k, v, kn, vn = data(2, 5, 4, 2, 90, 128, 17, tail=True)
    check(run(q, k, v, scale, 40, 2, k_new=kn, v_new=vn, out_dtype=torch.float32), reference(q, k, v, scale, 40, 2, None, kn, vn))


@pytest.mark.parametrize("Tq,Hq,Hkv", [(2, 256, 256), (16, 256, 16), (1, 256, 32), (20, 256, 256), (30, 240, 16)])
def test_many_heads(Tq, Hq, Hkv):
    q, k, v, _, _ = data(1, Tq, Hq, Hkv, 70, 64, 18)
    check(run(q, k, v, 0.1, 33, 2, out_dtype=torch.float32), reference(q, k, v, 0.1, 33, 2))


@pytest.mark.parametrize("Tq", [1, 17])
def test_large_batches(Tq):
    """More sequences than a grid's last dimension has; the first row that sees a key sees the first alone."""
    B, d = 40001, 64
    q, k, v = (torch.randn(*s, generator=gen(19)).to(torch.bfloat16).to(DEV) for s in ((B, Tq, 1, d), (B, 1, 1, d), (B, 1, 1, d)))
    o, l = sts.sts_window_attn(q, k, v, 0.1, 5)
    assert torch.equal(o[:, -1], v[:, :, 0]) and (o[:, :-1] == 0).all()
    s = 0.1 * (q[:, -1, 0].double() * k[:, 0, 0].double()).sum(-1)
    # one key: lse is its score, 64 products in fp32 of |q||k| under 10 each at 0.1, and two conversions between base 2 and e
    assert ((l[:, 0, -1].double() - s).abs() <= 64 * 2.0 ** -24 * 64 + 2.0 ** -22 * s.abs()).all() and torch.isneginf(l[:, 0, :-1]).all()
