"""sts_prompt_attn: causal attention over packed prompts against the definition in 64 bits, within bounds derived from the
roundings (cache_util.attention)."""
import math

import pytest
import torch

import paper_2605_15508_amd as sts
from layers_util import check_prompts, prompts, starts_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def data(T, Hq, Hkv, d, seed):
    g = torch.Generator().manual_seed(seed)
    return tuple(torch.randn(T, h, d, generator=g).to(torch.bfloat16) for h in (Hq, Hkv, Hkv))


def run(q, k, v, starts, scale, **kw):
    return sts.sts_prompt_attn(q.to(DEV), k.to(DEV), v.to(DEV), starts.to(DEV), scale, **kw)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,lens", [(1, 1, [1]), (4, 1, [2]), (2, 2, [0, 1, 0]), (8, 2, [63, 64, 65]), (4, 4, [127, 128, 129]), (16, 1, [7, 8, 9, 0, 70]), (6, 2, [42, 43, 1, 100]),
                                         (8, 8, [300]), (32, 8, [31, 32, 33, 34]), (3, 1, [257, 5]), (10, 2, [200, 1, 1, 1, 63])])
def test_lengths_and_heads(Hq, Hkv, lens, d):
    starts = starts_of(lens)
    q, k, v = data(int(starts[-1]), Hq, Hkv, d, sum(lens) + Hq)
    ref = prompts(q, k, v, starts, 1 / math.sqrt(d))
    for dt in (torch.float32, torch.bfloat16):
        check_prompts(run(q, k, v, starts, 1 / math.sqrt(d), out_dtype=dt), ref, what=f"{dt}")


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_scales(scale):
    starts = starts_of([70, 90])
    q, k, v = data(160, 4, 2, 128, 5)
    check_prompts(run(q, k, v, starts, scale, out_dtype=torch.float32), prompts(q, k, v, starts, scale))


@pytest.mark.parametrize("d", [64, 128])
def test_slices_of_one_projection(d):
    starts = starts_of([50, 0, 77])
    g = torch.Generator().manual_seed(6)
    rows = torch.randn(127, 8 + 2 * 2, d, generator=g).to(torch.bfloat16)
    q, k, v = rows[:, :8], rows[:, 8:10], rows[:, 10:]
    ref = prompts(q, k, v, starts, 0.1)
    on = rows.to(DEV)
    check_prompts(sts.sts_prompt_attn(on[:, :8], on[:, 8:10], on[:, 10:], starts.to(DEV), 0.1, out_dtype=torch.float32), ref)
    # heads first in memory
    qh, kh, vh = (t.transpose(0, 1).contiguous().to(DEV).transpose(0, 1) for t in (q, k, v))
    check_prompts(sts.sts_prompt_attn(qh, kh, vh, starts.to(DEV), 0.1, out_dtype=torch.float32), ref, what="heads first")


@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_no_sequence_stay_as_they_are(d):
    lens, first, T = [40, 0, 33], 13, 100
    starts = starts_of(lens, first)
    q, k, v = data(T, 4, 2, d, 8)
    for t in (q, k, v):
        t[:first], t[first + 73:] = float("nan"), float("inf")
    out, lse = torch.full((T, 4, d), 7.0, device=DEV), torch.full((4, T), 9.0, device=DEV)
    got = run(q, k, v, starts, 0.1, out=out, lse_out=lse)
    check_prompts(got, prompts(q, k, v, starts, 0.1), rows=slice(first, first + 73))
    assert (out[:first] == 7).all() and (out[first + 73:] == 7).all() and (lse[:, :first] == 9).all() and (lse[:, first + 73:] == 9).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,at", [(1, 0), (4, 5), (4, 64), (1, 127), (2, 130), (4, 149)])
def test_values_that_are_no_numbers_reach_no_row_before_them(Hq, at, d):
    """Row `at` of the middle sequence: the rows before it and the other sequences are as if it were not there."""
    lens = [20, 150, 30]
    starts = starts_of(lens)
    q, k, v = data(200, Hq, 1, d, 9)
    ref = prompts(q, k, v, starts, 0.1)
    kept = torch.cat((torch.arange(20 + at), torch.arange(170, 200)))
    for which, what in ((0, float("nan")), (0, float("inf")), (1, float("nan")), (1, float("-inf"))):
        x = [k.clone(), v.clone()]
        x[which][20 + at] = what
        out, lse = run(q, x[0], x[1], starts, 0.1, out_dtype=torch.float32)
        o, z = out.clone(), lse.clone()
        o[20 + at:170], z[:, 20 + at:170] = ref[0][20 + at:170].float().to(DEV), ref[1][:, 20 + at:170].float().to(DEV)
        check_prompts((o, z), ref, rows=kept, what=f"{which} {what}")
        if which == 1:
            assert not torch.isfinite(out[20 + at:170]).any()
            assert torch.isfinite(lse).all()
        if which == 0 and math.isnan(what):
            assert torch.isnan(out[20 + at:170]).all() and torch.isneginf(lse[:, 20 + at:170]).all()


@pytest.mark.parametrize("d", [64, 128])
def test_offsets_beyond_32_bits(d):
    """Rows 2^24 elements apart (the most there may be), behind one another in 4 GB and more."""
    lens = [100, 3, 70]
    T, starts = sum(lens), starts_of(lens)
    q, k, v = data(T, 2, 1, d, 13)
    big = torch.empty(T * 2 ** 24, dtype=torch.bfloat16, device=DEV).view(T, 2 ** 24 // d, d)
    dq, dk, dv = big[:, :2], big[:, 5:6], big[:, 9:10]
    for to, x in ((dq, q), (dk, k), (dv, v)):
        to.copy_(x)
    check_prompts(sts.sts_prompt_attn(dq, dk, dv, starts.to(DEV), 0.1, out_dtype=torch.float32), prompts(q, k, v, starts, 0.1))


@pytest.mark.parametrize("size", [1e-20, 1e36])
def test_values_of_all_sizes(size):
    starts = starts_of([90, 40])
    q, k, v = data(130, 4, 2, 128, 14)
    v = (v.float() * size).to(torch.bfloat16)
    check_prompts(run(q, k, v, starts, 0.1, out_dtype=torch.float32), prompts(q, k, v, starts, 0.1))


def test_scores_far_apart():
    """Scores from -4000 to 4000, of which nearly all weights are 0, in an order that raises the maximum again and again."""
    starts = starts_of([200])
    q, k, v = data(200, 2, 1, 64, 15)
    q[:] = 4.0
    k = (torch.arange(200).float()[:, None, None] * 20 - 2000).expand(200, 1, 64) / 64
    k = k.to(torch.bfloat16).contiguous()
    k[::3] = -k[::3]
    check_prompts(run(q, k, v, starts, 0.5, out_dtype=torch.float32), prompts(q, k, v, starts, 0.5))


def test_two_streams_at_once():
    inputs = [[t.to(DEV) for t in data(700, 8, 2, 128, 16 + i)] for i in range(2)]
    starts = starts_of([300, 0, 400]).to(DEV)
    want = [sts.sts_prompt_attn(*x, starts, 0.1) for x in inputs]
    streams = [torch.cuda.Stream() for _ in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for x, s, to in zip(inputs, streams, got):
            with torch.cuda.stream(s):
                to.append(sts.sts_prompt_attn(*x, starts, 0.1))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for o, z in g:
            assert torch.equal(o, w[0]) and torch.equal(z, w[1])


def test_many_sequences():
    """More than are looked through at once: 200 and 5000 of them, many empty."""
    g = torch.Generator().manual_seed(3)
    for B, most in ((200, 9), (5000, 3)):
        lens = torch.randint(0, most, (B,), generator=g).tolist()
        starts = starts_of(lens)
        T = int(starts[-1])
        q, k, v = data(T, 2, 1, 64, B)
        out, lse = run(q, k, v, starts, 0.125, out_dtype=torch.float32)
        some = torch.randint(0, B, (150,), generator=g).tolist()
        for b in some + [0, B - 1]:
            a, e = int(starts[b]), int(starts[b + 1])
            if e > a:
                check_prompts((out[a:e], lse[:, a:e]), prompts(q[a:e], k[a:e], v[a:e], starts_of([e - a]), 0.125), what=f"{b}")


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 4, 4)])
def test_long_prompts(d, Hq, Hkv):
    """Many tiles, against 64 bits on the GPU: some rows of each."""
    lens = [3001, 1, 4999]
    starts = starts_of(lens)
    q, k, v = (t.to(DEV) for t in data(sum(lens), Hq, Hkv, d, 11))
    out, lse = sts.sts_prompt_attn(q, k, v, starts.to(DEV), 0.1, out_dtype=torch.float32)
    for a, L in ((0, 3001), (3002, 4999)):
        for i in (0, 1, 63, 64, 1000, 2047, 2500, L - 1):
            for t in range(Hq):
                K, V, x = (y.double() for y in (k[a:a + i + 1, t * Hkv // Hq], v[a:a + i + 1, t * Hkv // Hq], q[a + i, t]))
                s = 0.1 * (K @ x)
                z = torch.logsumexp(s, 0)
                p = torch.exp(s - z)
                d_s = 0.1 * (d + 8) * 2.0 ** -24 * float((K.abs() @ x.abs()).max())       # as in cache_util.attention
                sums = ((i + 1) / 8 + 64) * 2.0 ** -24
                assert ((out[a + i, t] - p @ V).abs() <= (2.0 ** -8 + 2.2 * d_s + 2.0 ** -20 + sums) * (p @ V.abs())).all()
                assert abs(float(lse[t, a + i] - z)) <= d_s + sums + 2.0 ** -20 + 2.0 ** -22 * abs(float(z))


def test_the_same_from_run_to_run_and_without_lse():
    starts = starts_of([600, 35, 290]).to(DEV)
    q, k, v = (t.to(DEV) for t in data(925, 8, 2, 128, 12))
    first = sts.sts_prompt_attn(q, k, v, starts, 0.1)
    for _ in range(3):
        again = sts.sts_prompt_attn(q, k, v, starts, 0.1)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    out, lse = sts.sts_prompt_attn(q, k, v, starts, 0.1, want_lse=False)
    assert lse is None and torch.equal(out, first[0])


@pytest.mark.parametrize("d,B,Hq,Hkv", [(64, 14, 16, 4), (128, 7, 32, 8), (128, 3, 16, 16)])
def test_a_full_chip_gives_the_same_from_run_to_run(d, B, Hq, Hkv):
    """More workgroups than run at once, so that some begin where others have ended, at another pace."""
    lens = [2500 - 171 * b for b in range(B)]
    starts = starts_of(lens)
    q, k, v = (t.to(DEV) for t in data(sum(lens), Hq, Hkv, d, 18))
    first = sts.sts_prompt_attn(q, k, v, starts.to(DEV), 0.1)
    for _ in range(20):
        again = sts.sts_prompt_attn(q, k, v, starts.to(DEV), 0.1)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    a, e, G = int(starts[-2]), int(starts[-1]), Hq // Hkv                 # and that is right: the last sequence's last heads
    ref = prompts(q[a:e, Hq - G:].cpu(), k[a:e, Hkv - 1:].cpu(), v[a:e, Hkv - 1:].cpu(), starts_of([e - a]), 0.1)
    check_prompts((first[0][a:e, Hq - G:], first[1][Hq - G:, a:e]), ref)


def test_starts_that_make_no_sense_touch_nothing_else():
    """Out of order and out of range: results are not defined, but nothing behind the tensors is written to."""
    T = 300
    q, k, v = (t.to(DEV) for t in data(T, 4, 2, 64, 13))
    for starts in ([0, 500, 100], [250, 20, 300], [-5, 10, 2 ** 31 - 1], [300, 0, 300], [2 ** 31 - 1, -2 ** 31, 7], [0, 300, 0]):
        buf, zbuf = torch.full((T + 64, 4, 64), 5.0, device=DEV), torch.full((4 * T + 64,), 6.0, device=DEV)
        sts.sts_prompt_attn(q, k, v, torch.tensor(starts, dtype=torch.int32, device=DEV), 0.1, out=buf[32:32 + T], lse_out=zbuf[32:32 + 4 * T].view(4, T))
        assert (buf[:32] == 5).all() and (buf[32 + T:] == 5).all() and (zbuf[:32] == 6).all() and (zbuf[32 + 4 * T:] == 6).all()


def test_prepared_and_captured_calls():
    starts = starts_of([100, 0, 129]).to(DEV)
    q, k, v = (t.to(DEV) for t in data(229, 4, 2, 128, 14))
    call = sts.sts_prompt_attn(q, k, v, starts, 0.1, prepare=True)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out, lse = call()
    for seed in (1, 2, 3):
        for t, x in zip((q, k, v), data(229, 4, 2, 128, seed)):
            t.copy_(x)
        starts.copy_(starts_of([[100, 0, 129], [0, 229, 0], [1, 2, 226]][seed - 1]))
        want = sts.sts_prompt_attn(q, k, v, starts, 0.1)
        out.zero_(), lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_empty_batches():
    q, k, v = (t.to(DEV) for t in data(5, 4, 2, 64, 15))
    out = torch.full((5, 4, 64), 3.0, device=DEV, dtype=torch.bfloat16)
    sts.sts_prompt_attn(q, k, v, torch.zeros(1, dtype=torch.int32, device=DEV), 0.1, out=out)
    sts.sts_prompt_attn(q, k, v, torch.full((4,), 5, dtype=torch.int32, device=DEV), 0.1, out=out)
    assert (out == 3).all()
    got = sts.sts_prompt_attn(q[:0], k[:0], v[:0], torch.zeros(3, dtype=torch.int32, device=DEV), 0.1)
    assert got[0].shape == (0, 4, 64) and got[1].shape == (4, 0)


def test_wrong_arguments_are_refused():
    starts = starts_of([5]).to(DEV)
    q, k, v = (t.to(DEV) for t in data(5, 4, 2, 64, 16))
    for bad in (lambda: sts.sts_prompt_attn(q.float(), k, v, starts, 0.1), lambda: sts.sts_prompt_attn(q, k, v[:4], starts, 0.1),
                lambda: sts.sts_prompt_attn(q, k, v.transpose(1, 2), starts, 0.1), lambda: sts.sts_prompt_attn(q, k, v, starts.long(), 0.1),
                lambda: sts.sts_prompt_attn(q, k, v, starts.cpu(), 0.1), lambda: sts.sts_prompt_attn(q[:, :3], k, v, starts, 0.1),
                lambda: sts.sts_prompt_attn(q, k, v, starts, float("inf")), lambda: sts.sts_prompt_attn(q[:, :, :32], k[:, :, :32], v[:, :, :32], starts, 0.1),
                lambda: sts.sts_prompt_attn(q, k, v, starts, 0.1, out=torch.empty(5, 4, 64, device=DEV, dtype=torch.float16))):
        with pytest.raises((AssertionError, sts.StsError)):
            bad()
