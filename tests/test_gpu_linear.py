"""sts_linear_attn: single tokens, verification blocks and prompts against the recurrence in 64 bits, within bounds derived from the roundings
(layers_util.linear)."""
import math

import pytest
import torch

import paper_2605_15508_amd as sts
from layers_util import check_linear, linear, starts_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def data(T, Hq, Hkv, d, seed, gates=True, strength=0.05):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(T, h, d, generator=g).to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    decay = -strength * torch.rand((T, Hkv) if gates else (Hkv,), generator=g)
    return q, k, v, decay


def states(n, Hkv, d, seed):
    return torch.randn(n, Hkv, d, d, generator=torch.Generator().manual_seed(seed))


def on(x):
    return x.to(DEV) if isinstance(x, torch.Tensor) else x


def run(q, k, v, decay, scale, **kw):
    return sts.sts_linear_attn(on(q), on(k), on(v), on(decay), scale, **{a: on(x) for a, x in kw.items()})


def rows(decay, a, e):
    return decay if decay.dim() == 1 else decay[a:e]


def check(got, q, k, v, decay, scale, starts, first, chunked, lens=None, out=True, what=""):
    """Results and states of every sequence; `first` [B,Hkv,d,d]."""
    o, S = got
    for b in range(len(starts) - 1):
        a, e = int(starts[b]), int(starts[b + 1])
        if lens is not None:
            e = a + max(0, min(int(lens[b]), e - a))
        ref, all_s, e_ref, e_s = linear(q[a:e] if out else None, k[a:e], v[a:e], rows(decay, a, e), scale, first[b], chunked)
        if out and e > a:
            check_linear(o[a:e], ref, e_ref, f"{what} sequence {b}")
        if S is not None:
            check_linear(S[b], all_s[-1], e_s[-1], f"{what} state {b}")


BLOCKS = [(1, 1, 1, 1), (3, 1, 4, 1), (2, 5, 8, 2), (1, 16, 16, 1), (2, 7, 6, 2), (40, 1, 4, 4), (2, 16, 10, 2), (2, 7, 3, 3), (1, 16, 2, 2), (3, 5, 4, 2), (1, 2, 2, 1)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gates", [True, False])
@pytest.mark.parametrize("B,n,Hq,Hkv", BLOCKS)
def test_blocks(B, n, Hq, Hkv, gates, d):
    q, k, v, decay = data(B * n, Hq, Hkv, d, n + Hq, gates)
    first = states(B, Hkv, d, 3)
    shaped = [t.view(B, n, *t.shape[1:]) for t in (q, k, v)] + [decay.view(B, n, Hkv) if gates else decay]
    starts = starts_of([n] * B)
    for dt in (torch.float32, torch.bfloat16):
        out, S = run(*shaped, 0.1, state=first, state_out=torch.empty(B, Hkv, d, d), out_dtype=dt)
        check((out.view(B * n, Hq, d), S), q, k, v, decay, 0.1, starts, first, False, what=f"{dt}")
    out, S = run(*shaped, 0.1)                       # from nothing, and not kept
    assert S is None
    check((out.view(B * n, Hq, d), None), q, k, v, decay, 0.1, starts, torch.zeros_like(first), False, what="from zeros")
    _, S = run(None, *shaped[1:], 0.1, state=first, state_out=torch.empty(B, Hkv, d, d))
    check((None, S), q, k, v, decay, 0.1, starts, first, False, out=False, what="states only")


PROMPTS = [(1, 1, [17]), (2, 2, [0, 20, 0]), (4, 2, [0, 140, 0, 0]), (4, 1, [31, 32, 33]), (2, 2, [1, 0, 64, 65]), (8, 2, [100, 0, 257, 1]), (4, 4, [128, 129, 127]), (16, 1, [40, 385]), (3, 1, [300]), (32, 8, [50, 160])]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gates", [True, False])
@pytest.mark.parametrize("Hq,Hkv,lens", PROMPTS)
def test_prompts(Hq, Hkv, lens, gates, d):
    starts, B = starts_of(lens), len(lens)
    q, k, v, decay = data(int(starts[-1]), Hq, Hkv, d, sum(lens), gates)
    first = states(B, Hkv, d, 4)
    for dt in (torch.float32, torch.bfloat16):
        got = run(q, k, v, decay, 0.1, starts=starts, max_len=max(lens), state=first, state_out=torch.empty(B, Hkv, d, d), out_dtype=dt)
        check(got, q, k, v, decay, 0.1, starts, first, True, what=f"{dt}")
    got = run(q, k, v, decay, 0.1, starts=starts)    # the longest not known; from nothing, not kept
    check((got[0], None), q, k, v, decay, 0.1, starts, torch.zeros_like(first), True, what="from zeros")
    got = run(None, k, v, decay, 0.1, starts=starts, max_len=max(lens), state=first, state_out=torch.empty(B, Hkv, d, d))
    check((None, got[1]), q, k, v, decay, 0.1, starts, first, True, out=False, what="states only")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("strength", [0.0, 0.5, 8.0, 200.0, math.inf])
def test_decays_from_none_to_all(strength, d):
    """exp(-200) is 0 in fp32, and so is exp(-inf); some rows of the last case forget all that was, the others nothing."""
    lens = [70, 200]
    starts = starts_of(lens)
    q, k, v, decay = data(270, 4, 2, d, 21, True, 1.0)
    decay = torch.where(decay < -0.9, -math.inf, 0.0) if math.isinf(strength) else decay * strength
    first = states(2, 2, d, 5)
    got = run(q, k, v, decay, 0.1, starts=starts, max_len=200, state=first, state_out=torch.empty(2, 2, d, d), out_dtype=torch.float32)
    check(got, q, k, v, decay, 0.1, starts, first, True)
    blocks = [t[:15].view(1, 15, *t.shape[1:]) for t in (q, k, v, decay)]
    out, S = run(*blocks, 0.1, state=first[:1], state_out=torch.empty(1, 2, d, d), out_dtype=torch.float32)
    check((out[0], S), q, k, v, decay, 0.1, starts_of([15]), first, False)


@pytest.mark.parametrize("lens", [[5, 5, 5], [40, 300, 17]])
def test_slots(lens):
    """States anywhere in a pool that is wider than this layer's, sequences without one, states that are not kept, in place."""
    d, Hkv, B = 64, 2, 3
    starts = starts_of(lens)
    chunked = max(lens) > 16
    q, k, v, decay = data(sum(lens), 4, Hkv, d, 22)
    wide = states(7, 2 * Hkv, d, 6).to(DEV)
    pool = wide[:, Hkv:]
    before = wide.clone()
    slots, out_slots = torch.tensor([4, -1, 2], dtype=torch.int32), torch.tensor([0, 5, 7], dtype=torch.int32)
    first = torch.stack([pool[4], torch.zeros_like(pool[0]), pool[2]]).cpu()
    o, S = run(q, k, v, decay, 0.1, starts=starts, max_len=max(lens), state=pool, slots=slots, state_out=pool, slots_out=out_slots, out_dtype=torch.float32)
    kept = torch.stack([pool[0], pool[5], pool[0]])
    for b in range(2):
        a, e = int(starts[b]), int(starts[b + 1])
        check((o[a:e], kept[b:b + 1]), q[a:e], k[a:e], v[a:e], decay[a:e], 0.1, starts_of([e - a]), first[b:b + 1], chunked)
    check((o, None), q, k, v, decay, 0.1, starts, first, chunked)
    for s in (1, 2, 3, 4, 6):
        assert torch.equal(wide[s], before[s])
    assert torch.equal(wide[:, :Hkv], before[:, :Hkv])
    # in place
    slots = torch.tensor([6, 1, 3], dtype=torch.int32)
    first = before[[6, 1, 3], Hkv:].cpu()
    pool.copy_(before[:, Hkv:])
    o, S = run(q, k, v, decay, 0.1, starts=starts, max_len=max(lens), state=pool, slots=slots, state_out=pool, out_dtype=torch.float32)
    assert S is pool
    check((o, pool[[6, 1, 3]]), q, k, v, decay, 0.1, starts, first, chunked)
    # nothing of either pool where every slot is outside it
    pool.copy_(before[:, Hkv:])
    none = torch.tensor([-1, 7, 2 ** 31 - 1], dtype=torch.int32)
    o, _ = run(q, k, v, decay, 0.1, starts=starts, max_len=max(lens), state=pool, slots=none, state_out=pool, out_dtype=torch.float32)
    check((o, None), q, k, v, decay, 0.1, starts, torch.zeros_like(first), chunked)
    assert torch.equal(wide, before)


@pytest.mark.parametrize("n", [9, 150])
def test_rows_that_count(n):
    """lens: rows behind them are as they were in out and do not reach the state, whatever lies there; none at all copies the state."""
    d, B = 128, 5
    q, k, v, decay = data(B * n, 4, 2, d, 23)
    lens = torch.tensor([n, 0, 1, n - 1, -3], dtype=torch.int32)
    starts = starts_of([n] * B)
    for b in range(B):
        for t in (q, k, v, decay):
            t[b * n + max(0, int(lens[b])):(b + 1) * n] = float("nan")
    first = states(B, 2, d, 7)
    shaped = [t.view(B, n, *t.shape[1:]) for t in (q, k, v, decay)]
    out = torch.full((B, n, 4, d), 5.0, device=DEV)
    got = run(*shaped, 0.1, lens=lens, state=first, state_out=torch.empty(B, 2, d, d), out=out)
    check((got[0].view(B * n, 4, d), got[1]), q, k, v, decay, 0.1, starts, first, n > 16, lens=lens)
    for b in range(B):
        assert (out[b, max(0, int(lens[b])):] == 5).all()
    assert torch.equal(got[1][1].cpu(), first[1]) and torch.equal(got[1][4].cpu(), first[4])


@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (2, 2)])
def test_a_verification_block_and_its_commit(Hq, Hkv):
    B, n, d = 4, 6, 128
    q, k, v, decay = data(B * n, Hq, Hkv, d, 24)
    shaped = [on(t.view(B, n, *t.shape[1:])) for t in (q, k, v, decay)]
    pool = states(B, Hkv, d, 8).to(DEV)
    first = pool.clone()
    out, _ = sts.sts_linear_attn(*shaped, 0.1, state=pool, out_dtype=torch.float32)
    assert torch.equal(pool, first)
    accepted = torch.tensor([1, 6, 3, 0], dtype=torch.int32, device=DEV)
    sts.sts_linear_attn(None, *shaped[1:], 0.1, lens=accepted, state=pool, state_out=pool)
    check((out.view(B * n, Hq, d), None), q, k, v, decay, 0.1, starts_of([n] * B), first.cpu(), False)
    check((None, pool), q, k, v, decay, 0.1, starts_of([n] * B), first.cpu(), False, lens=accepted.cpu(), out=False)


@pytest.mark.parametrize("d", [64, 128])
def test_a_prompt_in_parts_is_the_prompt(d):
    """A prompt at once, in two calls, and the last rows token by token give the same results but for roundings."""
    n = 210
    q, k, v, decay = data(n, 4, 2, d, 25)
    pool = torch.zeros(1, 2, d, d, device=DEV)
    parts = []
    for a, e in ((0, 97), (97, 200)):
        parts.append(run(q[a:e], k[a:e], v[a:e], decay[a:e], 0.1, starts=starts_of([e - a]), state=pool, state_out=pool, out_dtype=torch.float32)[0])
    for i in range(200, n):
        parts.append(run(*[t[i][None, None] for t in (q, k, v, decay)], 0.1, state=pool, state_out=pool, out_dtype=torch.float32)[0][0])
    zero = torch.zeros(1, 2, d, d)
    check((torch.cat(parts), pool), q, k, v, decay, 0.1, starts_of([n]), zero, True)


@pytest.mark.parametrize("d", [64, 128])
def test_slices_and_gaps(d):
    """K and V out of one projection, rows of no sequence before, behind: not read, and left as they were."""
    lens, first, T = [33, 0, 140, 2], 5, 200
    starts = starts_of(lens, first)
    g = torch.Generator().manual_seed(26)
    x = torch.randn(T, 4 + 2 + 2, d, generator=g).to(torch.bfloat16)
    decay = -0.1 * torch.rand(T, 2, generator=g)
    x[:first], x[first + 175:], decay[:first], decay[first + 175:] = float("nan"), float("nan"), float("nan"), float("nan")
    dx = x.to(DEV)
    out = torch.full((T, 4, d), 5.0, device=DEV)
    S = torch.empty(4, 2, d, d, device=DEV)
    got = sts.sts_linear_attn(dx[:, :4], dx[:, 4:6], dx[:, 6:], on(decay), -0.3, starts=on(starts), state_out=S, out=out)
    check(got, x[:, :4], x[:, 4:6], x[:, 6:], decay, -0.3, starts, torch.zeros(4, 2, d, d), True)
    assert (out[:first] == 5).all() and (out[first + 175:] == 5).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [0, 1, 15, 16, 31, 32, 60, 99, 140])
def test_values_that_are_no_numbers_reach_no_row_before_them(at, d):
    lens = [20, 150, 30]
    starts = starts_of(lens)
    q, k, v, decay = data(200, 4, 2, d, 27)
    zero = torch.zeros(3, 2, d, d)
    for which, what in ((0, float("nan")), (0, float("inf")), (1, float("nan")), (1, float("inf"))):
        x = [k.clone(), v.clone()]
        x[which][20 + at, 0, 3] = what               # one channel of one head
        out, S = run(q, x[0], x[1], decay, 0.1, starts=starts, state_out=torch.empty(3, 2, d, d), out_dtype=torch.float32)
        for b, n in ((0, 20), (1, at), (2, 30)):
            a = int(starts[b])
            if n:
                ref, _, e_ref, _ = linear(q[a:a + n], k[a:a + n], v[a:a + n], decay[a:a + n], 0.1, zero[0], True)
                check_linear(out[a:a + n], ref, e_ref, f"{which} {what} {b}")
        rest = out[20 + at:170]
        assert torch.isfinite(rest[:, 2:]).all() and torch.isfinite(S[1, 1]).all()         # the other head's
        bad = rest[:, :2] if which == 0 else rest[:, :2, 3]
        assert not torch.isfinite(bad).any()
        if which == 1:                               # one column of the state
            others = [c for c in range(d) if c != 3]
            assert torch.isfinite(rest[:, :2, others]).all() and torch.isfinite(S[1, 0][:, others]).all() and not torch.isfinite(S[1, 0][:, 3]).any()


@pytest.mark.parametrize("d,past", [(64, 9), (128, 18)])
def test_segments_of_many_chunks(d, past):
    """Sixteen heads of a group, 256 in all: few segments, so that each has more chunks than a workgroup works out the decays of at once (nine
    or eighteen). Chunks on both sides of that border forget nearly all (2^-200), or grow, or all but stay as they are."""
    n = 1400
    q, k, v, decay = data(n, 256, 16, d, 37, True, 0.1)
    for chunk, value in ((past - 1, -4.0), (past, -6.0), (past + 1, 0.0), (past + 3, 0.02), (0, -5.0)):
        for segment in range(0, n, 352 if d == 64 else 704):
            decay[segment + 32 * chunk:segment + 32 * chunk + 32, 0] = value
    first = states(1, 16, d, 10)
    for out in (True, False):
        o, S = run(q if out else None, k, v, decay, 0.1, starts=starts_of([n]), state=first, state_out=torch.empty(1, 16, d, d), out_dtype=torch.float32)
        for g in (0, 13):
            h, kv = slice(16 * g, 16 * g + 16), slice(g, g + 1)
            check((o[:, h] if out else None, S[:, kv]), q[:, h], k[:, kv], v[:, kv], decay[:, kv], 0.1, starts_of([n]), first[:, kv], True, out=out, what=f"head {g}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("up", [0.02, 0.6, 3.0])
def test_states_that_grow(up, d):
    """Decays above 0: some rows by little, or by more than is taken back."""
    n = 150
    q, k, v, _ = data(n, 4, 2, d, 38)
    g = torch.Generator().manual_seed(39)
    decay = up * (torch.rand(n, 2, generator=g) * 2 - 1)
    first = states(1, 2, d, 11)
    got = run(q, k, v, decay, 0.1, starts=starts_of([n]), state=first, state_out=torch.empty(1, 2, d, d), out_dtype=torch.float32)
    check(got, q, k, v, decay, 0.1, starts_of([n]), first, True)
    blocks = [t[:16].view(1, 16, *t.shape[1:]) for t in (q, k, v, decay)]
    out, S = run(*blocks, 0.1, state=first, state_out=torch.empty(1, 2, d, d), out_dtype=torch.float32)
    check((out[0], S), q, k, v, decay, 0.1, starts_of([16]), first, False)


@pytest.mark.parametrize("size", [1e35, 1e-20])
@pytest.mark.parametrize("n", [10, 300])
def test_values_of_all_sizes(n, size):
    """Values whose sums are near the ends of fp32, with decays that take the state through many powers of two."""
    d = 64
    q, k, v, decay = data(n, 2, 2, d, 40, True, 0.4)
    v = (v.float() * size).to(torch.bfloat16)
    first = states(1, 2, d, 12) * size
    got = run(q, k, v, decay, 0.1, starts=starts_of([n]), max_len=n, state=first, state_out=torch.empty(1, 2, d, d), out_dtype=torch.float32)
    check(got, q, k, v, decay, 0.1, starts_of([n]), first, n > 16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [0, 31, 32, 77, 149])
def test_a_decay_that_is_no_number(at, d):
    """Rows before it and the other head do not see it; from there on the head's results and its state are no numbers."""
    n = 150
    q, k, v, decay = data(n, 4, 2, d, 41)
    decay[at, 0] = float("nan")
    zero = torch.zeros(2, d, d)
    for rows_, chunked in ((n, True), (min(at + 1, 16), False)):
        if not chunked and at >= 16:
            continue
        out, S = run(q[:rows_], k[:rows_], v[:rows_], decay[:rows_], 0.1, starts=starts_of([rows_]), max_len=rows_, state_out=torch.empty(1, 2, d, d), out_dtype=torch.float32)
        if at:
            ref, _, e_ref, _ = linear(q[:at], k[:at], v[:at], decay[:at], 0.1, zero, chunked)
            check_linear(out[:at], ref, e_ref, "before")
        ref, all_s, e_ref, e_s = linear(q[:rows_, 2:], k[:rows_, 1:], v[:rows_, 1:], decay[:rows_, 1:], 0.1, zero[1:], chunked)
        check_linear(out[:, 2:], ref, e_ref, "the other head")
        check_linear(S[0, 1:], all_s[-1], e_s[-1], "the other head's state")
        assert torch.isnan(out[at:, :2]).all() and torch.isnan(S[0, 0]).all()


@pytest.mark.parametrize("max_len,lens", [(7, [20, 3, 9]), (40, [100, 30, 41])])
def test_rows_behind_the_longest_are_left_out(max_len, lens):
    d = 64
    starts = starts_of(lens)
    q, k, v, decay = data(sum(lens), 4, 2, d, 42)
    first = states(3, 2, d, 13)
    out = torch.full((sum(lens), 4, d), 5.0, device=DEV)
    got = run(q, k, v, decay, 0.1, starts=starts, max_len=max_len, state=first, state_out=torch.empty(3, 2, d, d), out=out)
    check(got, q, k, v, decay, 0.1, starts, first, max_len > 16, lens=torch.full((3,), max_len))
    for b, n in enumerate(lens):
        assert (out[int(starts[b]) + min(n, max_len):int(starts[b]) + n] == 5).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
def test_nothing_behind_a_sequence_is_written(dt, d):
    """The last chunk of a segment and of a sequence is not whole: the rows behind belong to the next sequence, or to nobody."""
    lens = [131, 1, 45]
    starts = starts_of(lens)
    q, k, v, decay = data(200, 4, 1, d, 43)
    out = torch.full((200, 4, d), 5.0, device=DEV, dtype=dt)
    for b in range(3):                                # one at a time, each between rows that are not its own
        only = torch.tensor([int(starts[b]), int(starts[b + 1])], dtype=torch.int32)
        before = out.clone()
        got = run(q, k, v, decay, 0.1, starts=only, out=out)
        a, e = only.tolist()
        assert torch.equal(out[:a], before[:a]) and torch.equal(out[e:], before[e:])
        check((got[0][a:e], None), q[a:e], k[a:e], v[a:e], decay[a:e], 0.1, starts_of([e - a]), torch.zeros(1, 1, d, d), True)


@pytest.mark.parametrize("lens", [[9, 8], [100, 40]])
def test_offsets_beyond_32_bits(lens):
    """Rows 2^24 elements apart (the most there may be), behind one another in 4 GB and more."""
    d, T = 64, sum(lens)
    q, k, v, decay = data(T, 2, 1, d, 44)
    big = torch.empty(T * 2 ** 24, dtype=torch.bfloat16, device=DEV).view(T, 2 ** 18, d)
    dq, dk, dv = big[:, :2], big[:, 5:6], big[:, 9:10]
    for to, x in ((dq, q), (dk, k), (dv, v)):
        to.copy_(x)
    starts = starts_of(lens)
    got = sts.sts_linear_attn(dq, dk, dv, on(decay), 0.1, starts=on(starts), max_len=max(lens), state_out=torch.empty(2, 1, d, d, device=DEV), out_dtype=torch.float32)
    check(got, q, k, v, decay, 0.1, starts, torch.zeros(2, 1, d, d), max(lens) > 16)


@pytest.mark.parametrize("n", [8, 500])
def test_two_streams_at_once(n):
    """Calls on two streams, which overlap as they like, with workspaces of their own give what they give one after the other."""
    inputs = [[on(t) for t in data(2 * n, 8, 2, 128, 45 + i)] for i in range(2)]
    starts = starts_of([n, n]).to(DEV)
    want = [sts.sts_linear_attn(*x, 0.1, starts=starts, max_len=n, state_out=torch.empty(2, 2, 128, 128, device=DEV)) for x in inputs]
    streams = [torch.cuda.Stream() for _ in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for x, s, to in zip(inputs, streams, got):
            with torch.cuda.stream(s):
                to.append(sts.sts_linear_attn(*x, 0.1, starts=starts, max_len=n, state_out=torch.empty(2, 2, 128, 128, device=DEV)))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for o, S in g:
            assert torch.equal(o, w[0]) and torch.equal(S, w[1])


def test_a_long_sequence_of_one_decay():
    """4096 rows with a decay close to 1: its factor's rounding is the same in every chunk and must not add up. On the GPU in 64 bits."""
    n, d = 4096, 64
    q, k, v, _ = data(n, 2, 2, d, 28)
    decay = torch.log1p(-torch.tensor([2.0 ** -12, 2.0 ** -9]))
    out, S = run(q, k, v, decay, 0.1, starts=starts_of([n]), state_out=torch.empty(1, 2, d, d), out_dtype=torch.float32)
    w = torch.exp(decay.double()[:, None] * torch.arange(n - 1, -1, -1).double())            # [2, n]
    kk, vv = k.double().transpose(0, 1), v.double().transpose(0, 1)
    want, most = (torch.matmul((x * w[:, :, None]).transpose(1, 2), y) for x, y in ((kk, vv), (kk.abs(), vv.abs())))
    # (100 + 8 * 32 * 0.003) 2^-24 for each of 128 chunks at worst, as in layers_util.linear
    assert ((S[0].cpu().double() - want).abs() <= 128 * 101 * 2.0 ** -24 * most).all()
    # and as measured by its size: sums of rounded numbers err at random, a factor off by 2^-25 in each of 128 chunks would not. 128 chunks'
    # sums of 96 products: sqrt(128 * 96) 2^-24 = 6.6e-6 of a number's size; such a factor alone: 128 * 2^-25 = 3.8e-6
    err = (S[0].cpu().double() - want).square().mean().sqrt() / want.square().mean().sqrt()
    assert err < 6.6e-6


@pytest.mark.parametrize("n", [12, 300])
def test_the_same_from_run_to_run(n):
    q, k, v, decay = (on(t) for t in data(2 * n, 8, 2, 128, 29))
    starts = starts_of([n, n]).to(DEV)
    first = sts.sts_linear_attn(q, k, v, decay, 0.1, starts=starts, max_len=n, state_out=torch.empty(2, 2, 128, 128, device=DEV))
    for _ in range(3):
        again = sts.sts_linear_attn(q, k, v, decay, 0.1, starts=starts, max_len=n, state_out=torch.empty(2, 2, 128, 128, device=DEV))
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("d,B,Hq,Hkv", [(64, 14, 16, 16), (128, 3, 32, 8), (128, 4, 16, 16)])
def test_a_full_chip_gives_the_same_from_run_to_run(d, B, Hq, Hkv):
    """More workgroups than run at once, so that some begin where others have ended, at another pace."""
    lens = [2000 - 133 * b for b in range(B)]
    q, k, v, decay = (on(t) for t in data(sum(lens), Hq, Hkv, d, 47))
    starts = starts_of(lens).to(DEV)
    call = lambda: sts.sts_linear_attn(q, k, v, decay, 0.1, starts=starts, max_len=2000, state_out=torch.empty(B, Hkv, d, d, device=DEV))  # noqa: E731
    first = call()
    for _ in range(20):
        again = call()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    b, g = B - 1, Hkv - 1                             # and that is right: the last sequence's last head
    h, kv = slice(Hq - Hq // Hkv, Hq), slice(g, g + 1)
    a, e = int(starts[b]), int(starts[b + 1])
    rows_ = [t.cpu()[a:e] for t in (q[:, h], k[:, kv], v[:, kv], decay[:, kv])]
    check((first[0][a:e, h], first[1][b:, kv]), *rows_, 0.1, starts_of([e - a]), torch.zeros(1, 1, d, d), True)


def test_many_sequences():
    g = torch.Generator().manual_seed(30)
    lens = torch.randint(0, 4, (5000,), generator=g).tolist()
    lens[77], lens[4000] = 150, 40
    starts = starts_of(lens)
    q, k, v, decay = data(sum(lens), 1, 1, 64, 31)
    out, _ = run(q, k, v, decay, 0.1, starts=starts, out_dtype=torch.float32)
    for b in torch.randint(0, 5000, (100,), generator=g).tolist() + [0, 77, 4000, 4999]:
        a, e = int(starts[b]), int(starts[b + 1])
        check((out[a:e], None), q[a:e], k[a:e], v[a:e], decay[a:e], 0.1, starts_of([e - a]), torch.zeros(1, 1, 64, 64), True)


@pytest.mark.parametrize("max_len", [8, 40, None])
def test_starts_that_make_no_sense_touch_nothing_else(max_len):
    T = 300
    q, k, v, decay = (on(t) for t in data(T, 4, 2, 64, 32))
    for starts in ([0, 500, 100], [250, 20, 300], [-5, 10, 2 ** 31 - 1], [300, 0, 300], [2 ** 31 - 1, -2 ** 31, 7], [0, 300, 0]):
        buf, pool = torch.full((T + 64, 4, 64), 5.0, device=DEV), torch.full((4, 2, 64, 64), 6.0, device=DEV)
        sts.sts_linear_attn(q, k, v, decay, 0.1, starts=torch.tensor(starts, dtype=torch.int32, device=DEV), max_len=max_len, state_out=pool[1:3], out=buf[32:32 + T])
        assert (buf[:32] == 5).all() and (buf[32 + T:] == 5).all() and (pool[0] == 6).all() and (pool[3] == 6).all()


@pytest.mark.parametrize("n", [4, 200])
def test_prepared_and_captured_calls(n):
    """Two calls captured into one graph with a workspace each; replayed with other inputs and lengths."""
    B, d = 2, 64
    T = B * n
    q, k, v, decay = (on(t) for t in data(T, 4, 2, d, 33))
    starts = starts_of([n] * B).to(DEV)
    pools = [torch.zeros(B, 2, d, d, device=DEV) for _ in range(2)]
    calls = [sts.sts_linear_attn(q, k, v, decay, s, starts=starts, max_len=T if n > 16 else n, state=p, state_out=p, prepare=True) for s, p in ((0.1, pools[0]), (-0.2, pools[1]))]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = [call()[0] for call in calls]
    for seed in (1, 2, 3):
        for t, x in zip((q, k, v, decay), data(T, 4, 2, d, seed)):
            t.copy_(x)
        if n > 16:
            starts.copy_(starts_of([[n, n], [0, T], [T - 1, 1]][seed - 1]))
        start = states(B, 2, d, seed)
        wants = []
        for s in (0.1, -0.2):
            p = start.to(DEV)
            wants.append((sts.sts_linear_attn(q, k, v, decay, s, starts=starts, max_len=T if n > 16 else n, state=p, state_out=p)[0], p))
        for p in pools:
            p.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        for o, p, (wo, wp) in zip(got, pools, wants):
            assert torch.equal(o, wo) and torch.equal(p, wp)


def test_empty_batches():
    q, k, v, decay = (on(t) for t in data(5, 4, 2, 64, 34))
    out = torch.full((5, 4, 64), 3.0, device=DEV, dtype=torch.bfloat16)
    sts.sts_linear_attn(q, k, v, decay, 0.1, starts=torch.zeros(1, dtype=torch.int32, device=DEV), out=out)
    pool, first = torch.zeros(3, 2, 64, 64, device=DEV), states(3, 2, 64, 9).to(DEV)
    sts.sts_linear_attn(q, k, v, decay, 0.1, starts=torch.full((4,), 5, dtype=torch.int32, device=DEV), state=first, state_out=pool, out=out)
    assert (out == 3).all() and torch.equal(pool, first)
    pool.zero_()
    pool.zero_()                                    # blocks of no rows
    o, _ = sts.sts_linear_attn(q[:0].view(3, 0, 4, 64), k[:0].view(3, 0, 2, 64), v[:0].view(3, 0, 2, 64), decay[:0].view(3, 0, 2), 0.1, state=first, state_out=pool)
    assert o.shape == (3, 0, 4, 64) and torch.equal(pool, first)
    pool.zero_()
    o, _ = sts.sts_linear_attn(q[:0], k[:0], v[:0], decay[:0], 0.1, starts=torch.zeros(4, dtype=torch.int32, device=DEV), state=first, state_out=pool)
    assert o.shape == (0, 4, 64) and torch.equal(pool, first)


def test_wrong_arguments_are_refused():
    starts = starts_of([5]).to(DEV)
    q, k, v, decay = (on(t) for t in data(5, 4, 2, 64, 35))
    pool = torch.zeros(2, 2, 64, 64, device=DEV)
    one = torch.zeros(1, dtype=torch.int32, device=DEV)
    f = sts.sts_linear_attn
    for bad in (lambda: f(q.float(), k, v, decay, 0.1, starts=starts), lambda: f(q, k, v, decay.double(), 0.1, starts=starts), lambda: f(q, k, v, decay[:, :1], 0.1, starts=starts),
                lambda: f(q, k, v, decay, 0.1), lambda: f(q, k, v, decay, 0.1, starts=starts, slots=one), lambda: f(q, k, v, decay, 0.1, starts=starts, state=pool.bfloat16()),
                lambda: f(q, k, v, decay, 0.1, starts=starts, state=pool.transpose(2, 3)), lambda: f(q, k, v, decay, 0.1, starts=starts, state=pool[:0]),
                lambda: f(q, k, v, decay, 0.1, starts=starts, max_len=-1), lambda: f(q, k, v, decay, float("nan"), starts=starts),
                lambda: f(q, k, v, decay, 0.1, starts=starts, lens=one.long()), lambda: f(None, k, v, decay, 0.1, starts=starts, out=torch.empty_like(q))):
        with pytest.raises((AssertionError, sts.StsError)):
            bad()


def test_both_layers_of_a_prompt_and_what_follows():
    """As a program with both kinds of layers runs them: three packed prompts, then verification blocks whose accepted rows are kept, against the
    whole sequences at once."""
    d, Hq, Hkv, n = 128, 4, 2, 5
    lens, accepted = [70, 1, 33], [2, 5, 1]
    g = torch.Generator().manual_seed(36)
    seqs = [[torch.randn(L + n, h, d, generator=g).to(torch.bfloat16) for h in (Hq, Hkv, Hkv)] + [-0.1 * torch.rand(L + n, Hkv, generator=g)] for L in lens]
    packed = [torch.cat([s[i][:L] for s, L in zip(seqs, lens)]).to(DEV) for i in range(4)]
    block = [torch.stack([s[i][L:] for s, L in zip(seqs, lens)]).to(DEV) for i in range(4)]
    starts = starts_of(lens).to(DEV)
    # the prompts
    out, _ = sts.sts_prompt_attn(*packed[:3], starts, 0.1, out_dtype=torch.float32)
    pool = torch.empty(3, Hkv, d, d, device=DEV)
    lin, _ = sts.sts_linear_attn(*packed, 0.1, starts=starts, max_len=max(lens), state_out=pool, out_dtype=torch.float32)
    cache = torch.zeros(2, 3, Hkv, 80, d, dtype=torch.bfloat16, device=DEV)
    for b, L in enumerate(lens):
        for i in range(2):
            cache[i, b, :, :L] = packed[1 + i][int(starts[b]):int(starts[b + 1])].transpose(0, 1)
    # the block: attention over the cache and its own rows, the linear layer from the kept states
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    vout, _, _ = sts.sts_dense_attn(block[0], cache[0], cache[1], 0.1, seq_lens=length, k_new=block[1], v_new=block[2], out_dtype=torch.float32)
    vlin, _ = sts.sts_linear_attn(*block, 0.1, state=pool, out_dtype=torch.float32)
    sts.sts_linear_attn(None, *block[1:], 0.1, lens=torch.tensor(accepted, dtype=torch.int32, device=DEV), state=pool, state_out=pool)
    for b, (s, L) in enumerate(zip(seqs, lens)):
        both = torch.cat((out[int(starts[b]):int(starts[b + 1])], vout[b]))
        whole, z = sts.sts_prompt_attn(*[t.to(DEV) for t in s[:3]], starts_of([L + n]).to(DEV), 0.1, out_dtype=torch.float32)
        from layers_util import check_prompts, prompts

        ref = prompts(*s[:3], starts_of([L + n]), 0.1)
        check_prompts((both, z), ref)
        check_prompts((whole, z), ref)
        want, all_s, e, e_s = linear(*s, 0.1, torch.zeros(Hkv, d, d), True)
        check_linear(torch.cat((lin[int(starts[b]):int(starts[b + 1])], vlin[b])), want, e)
        check_linear(pool[b], all_s[L + accepted[b]], e_s[L + accepted[b]])
